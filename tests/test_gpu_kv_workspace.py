"""A server's batch shrinks and grows under one workspace, sized once for the largest call."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2609_25451_b200 import gms  # noqa: E402

if torch.cuda.is_available():
    from kv_attn_harness import Problem  # noqa: E402


@pytest.mark.parametrize("weights", [False, True])
def test_batches_of_many_sizes(weights):
    largest = Problem(1, heads=32, kv_heads=8, q_lens=(6,) * 64, kv_lens=(700,) * 64)
    w = torch.zeros((64, 8, 700), device="cuda")
    n = gms.gms_kv_attention_workspace(largest.desc, largest.layout, largest.attn, gms.kv_weights(None, w) if weights else None)
    ws = torch.full((n + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    for seqs, q, kv in ((64, 6, 700), (64, 1, 300), (50, 1, 700), (48, 4, 699), (37, 5, 64), (36, 1, 200), (16, 1, 700), (3, 2, 40), (1, 1, 1)):
        p = Problem(seqs, heads=32, kv_heads=8, q_lens=(q,) * seqs, kv_lens=tuple(kv - s % kv // 2 for s in range(seqs)), decode=q == 1)
        p.attn.set_workspace(ws[:n])
        gms.gms_kv_attention(p.desc, p.layout, p.attn, gms.kv_weights(None, w) if weights else None)
        torch.cuda.synchronize()
        assert int(p.status.item()) == 0 and bool((ws[n:] == 0xFF).all())
        ref = p.reference()
        p.check(ref)
        for s, m in enumerate(p.kv_lens if weights else ()):
            want = ref[s][4]
            assert not bool(((w[s, :, :m].double() - want).abs() > ref[s][5] + 2.0 ** -23 * (q * 32 + 2) * want).any())
