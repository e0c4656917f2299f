"""Infinities and NaN in keys and values: what they reach, and what they cost."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2609_25451_b200 import gms  # noqa: E402

if torch.cuda.is_available():
    from kv_attn_harness import Problem  # noqa: E402


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,kv_heads,q", [(6, 2, 33), (3, 1, 7), (8, 2, 33), (5, 5, 21), (4, 2, 1)])
def test_a_logit_of_minus_infinity_weighs_nothing(dtype, heads, kv_heads, q):
    """Row counts that are and are not multiples of the matrix instruction's eight."""
    p = Problem(1, dtype=dtype, heads=heads, kv_heads=kv_heads, dim=64, block=64, q_lens=(q,), kv_lens=(400,))
    p.q[:, :, 0] = 1.0
    p.K[0][10, :, 0] = -math.inf
    p.store(p.kp, p.table_h[0], p.K[0])
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    w_in = torch.rand((1, kv_heads, 400), device="cuda", generator=g)
    w = torch.zeros_like(w_in)
    p.run(gms.kv_weights(w_in, w, decay=0.5))
    assert bool(torch.isfinite(p.out).all()) and bool(torch.isfinite(w).all())
    assert torch.equal(w[:, :, 10], 0.5 * w_in[:, :, 10])
    total = (w.double() - 0.5 * w_in.double()).sum(2)
    assert float((total - q * heads // kv_heads).abs().max()) < 2.0 ** -20 * 400 * q * heads
