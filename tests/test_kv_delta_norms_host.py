"""The norms that hold gms_kv_delta to its precision (tests/kv_delta_norms.py), on results that are right and on such that are not."""
import pytest

torch = pytest.importorskip("torch")

import kv_delta_norms as norms  # noqa: E402


def problem(n, dtype, D=64, H=2):
    g = torch.Generator().manual_seed(n + D)
    q, k, v = (torch.randn((n, H, D), generator=g).to(dtype) for _ in range(3))
    gates = -torch.nn.functional.softplus(torch.randn((n, H), generator=g) - 1)
    beta = torch.sigmoid(torch.randn((n, H), generator=g))
    S = 0.3 * torch.randn((H, D, D), generator=g)
    return norms.unit(q, 1e-6), norms.unit(k, 1e-6), v, gates, beta, S, D ** -0.5


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n", [1, 20, 64, 130, 500])
def test_what_is_let_through(n, dtype):
    out, S, size = norms.rule(*problem(n, dtype))
    assert norms.state_errors(S.float(), S).max() < norms.STATE
    assert norms.out_errors(out.to(dtype), out, size, dtype).max() <= 1
    # outputs of zeros, of another row, a block that lacks its own rows' part or has lost an eighth of itself; states in one term
    for wrong in (torch.zeros_like(out), out.roll(1, 2), out * 0.875):
        assert (norms.out_errors(wrong.to(dtype), out, size, dtype) > 1).all()
    assert norms.state_errors(S.to(dtype), S).min() > norms.STATE
    lost = out.clone()
    lost[n // 2] = 0
    assert norms.out_errors(lost.to(dtype), out, size, dtype).max() > 1


def test_the_rule_itself():
    """Against the same in matrices: S_n = prod(e^g (I - b k k^T)) S_0 + ..., a row at a time."""
    q, k, v, g, beta, S, scale = problem(7, torch.bfloat16, D=8)
    out, end, size = norms.rule(q, k, v, g, beta, S, scale)
    for h in range(2):
        M = S[h].double()
        for t in range(7):
            kk, b = k[t, h][:, None], beta[t, h].double()
            M = (torch.eye(8).double() - b * kk @ kk.T) @ (g[t, h].double().exp() * M) + b * kk @ v[t, h].double()[None, :]
            assert torch.allclose(out[t, h], scale * (M.T @ q[t, h]), rtol=1e-12, atol=1e-14)
        assert torch.allclose(end[h], M, rtol=1e-12, atol=1e-14)
