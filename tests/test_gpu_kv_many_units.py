"""The many-row kernel with more units (runs of 256 rows) than a CTA has threads: each thread plans several."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2609_25451_b200 import gms  # noqa: E402

if torch.cuda.is_available():
    from kv_attn_harness import Problem  # noqa: E402


@pytest.mark.parametrize("seqs,q,heads,kv_heads,dim", [(450, 20, 8, 1, 64), (800, 33, 4, 2, 64), (385, 70, 4, 1, 128)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (60, 2)])
def test_many_units(seqs, q, heads, kv_heads, dim, window, sinks):
    q_lens = [(q * (s % 7 + 1)) // 7 for s in range(seqs)]
    kv_lens = [a + (31 * s) % 200 for s, a in enumerate(q_lens)]
    p = Problem(1, heads=heads, kv_heads=kv_heads, dim=dim, block=64, q_lens=q_lens, kv_lens=kv_lens, window=window, sinks=sinks)
    w = torch.zeros((seqs, kv_heads, max(kv_lens)), device="cuda")
    p.run(gms.kv_weights(None, w))
    ref = p.reference()
    p.check(ref)
    for s, n in enumerate(kv_lens):
        assert not bool(((w[s, :, :n].double() - ref[s][4]).abs() > ref[s][5] + 2.0 ** -23 * (q * heads + 2) * ref[s][4]).any()), s


@pytest.mark.parametrize("groups", [400, 1])
def test_many_units_behind_prefixes(groups):
    """A prefix pass of 400 units, and an own pass of 400."""
    seqs, q = 400, 20
    gs = list(range(401)) if groups == 400 else [0, 400]
    p = Problem(2, heads=8, kv_heads=1, dim=64, block=64, q_lens=[q] * seqs, kv_lens=[q + s % 50 for s in range(seqs)],
                prefix_lens=[40 + s % 100 for s in range(groups)], groups=gs)
    p.run(prefix=p.make_prefix())
    p.check()
