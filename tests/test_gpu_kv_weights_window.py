"""Accumulated weights under windows of many sizes: the kept logits lie in the order of the tiles that are seen."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2609_25451_b200 import gms  # noqa: E402

if torch.cuda.is_available():
    from kv_attn_harness import Problem  # noqa: E402


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 1), (17, 16), (33, 17), (100, 40), (250, 0), (1000, 5), (15, 300)])
@pytest.mark.parametrize("q", [1, 3])
def test_windows(dtype, window, sinks, q):
    kv_lens = (400, q, 16 + q, 31 + q, 47 + q, 1200, 255, 256, 257)
    p = Problem(1, dtype=dtype, heads=8, kv_heads=2, q_lens=(q,) * len(kv_lens), kv_lens=kv_lens, window=window, sinks=sinks, decode=q == 1)
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    w_in = torch.rand((len(kv_lens), 2, 1200), device="cuda", generator=g)
    w = torch.full_like(w_in, -5.0)
    p.run(gms.kv_weights(w_in, w, decay=0.5))
    ref = p.reference()
    p.check(ref)
    for s, n in enumerate(kv_lens):
        want = 0.5 * w_in[s, :, :n].double() + ref[s][4]
        assert not bool(((w[s, :, :n].double() - want).abs() > ref[s][5] + 2.0 ** -23 * (q * 8 + 2) * want).any()), s
        assert bool((w[s, :, n:] == -5).all())
