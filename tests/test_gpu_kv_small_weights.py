"""Many tokens of tiny weight behind one that dominates (a sink): together they count, also in fp16, whose smallest number is
2^-24."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2609_25451_b200 import gms  # noqa: E402

if torch.cuda.is_available():
    from kv_attn_harness import Problem  # noqa: E402


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("q,n", [(1, 60000), (2, 60000), (1, 1500), (3, 1500), (40, 30000), (40, 1500), (200, 1500)])
def test_a_dominant_sink(dtype, q, n):
    """Token 0 has logit 17.5 and value 0, all others logit 0 and value 1: each weighs e^-17.5 = 2^-25.2 of the sink.  Their
    weights round alike, so the sum is off by the rounding of one: u relative (a normal number of the type), in fp16 at most
    2^-25 absolute against the largest, which the kernels keep at 2^7 or more; then one rounding of the output, u."""
    p = Problem(1, dtype=dtype, heads=8, kv_heads=2, dim=64, block=64, q_lens=(q,), kv_lens=(n,), decode=q == 1)
    p.qfull.zero_()
    p.q[:, :, 0] = 1.0
    p.K[0].zero_()
    p.K[0][0, :, 0] = 17.5
    p.V[0].fill_(1.0)
    p.V[0][0] = 0.0
    p.store(p.kp, p.table_h[0], p.K[0])
    p.store(p.vp, p.table_h[0], p.V[0])
    p.scale = p.attn.scale = 1.0
    p.run()
    u = torch.finfo(dtype).eps / 2
    for i in range(q):
        rest = (n - q + i) * math.exp(-17.5)
        want = rest / (1 + rest)
        rel = 2 * u + 2.0 ** -19
        if dtype == torch.float16:
            rel += 2.0 ** -25 / (math.exp(-17.5) * 2.0 ** 7)
        got = p.out[i].double()
        # outputs below 2^-14 are spaced 2^-24 in fp16
        assert float((got - want).abs().max()) <= rel * want + (2.0 ** -25 if dtype == torch.float16 else 0), (i, float(got.min()), want)
        assert abs(float(p.lse[i, 0]) - (17.5 + math.log1p(rest))) < 1e-4
