"""gms_kv_delta where numbers of one chunk are far apart: gates above 0, rows much longer than others."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from kv_delta_harness import BF16, F16, Delta  # noqa: E402
from kv_delta_norms import check  # noqa: E402

# head_dim, sequences of 4 heads: one slice of a state a CTA, two, a warp each
FORMS = [(128, 1), (128, 6), (128, 12), (64, 1), (64, 12), (64, 20)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("D,S", FORMS)
@pytest.mark.parametrize("up", [12.0, 15.0, 18.0, 20.0, 23.0, 27.0, 30.0, 40.0])
def test_a_gate_above_zero(up, D, S, dtype):
    """What a gate takes the next one gives back (in between the state has nothing new, or fp16 could not hold what comes of it)."""
    d = Delta(1, lens=(130,) * S, D=D, dtype=dtype)
    for s in range(S):
        r = d.cu_h[s] + 40 + s
        d.g[r], d.g[r + 1] = -up, up
        d.beta[r] = 0
    check(d)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("D,S", FORMS)
@pytest.mark.parametrize("up", [0.8, 1.5])
def test_gates_up_and_down(up, D, S, dtype):
    d = Delta(2, lens=(130,) * S, D=D, dtype=dtype)
    d.g.copy_(torch.where(torch.arange(d.T, device="cuda")[:, None] % 2 == 0, -up, up))
    check(d)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("D,S", FORMS)
@pytest.mark.parametrize("what", ["q", "k"])
def test_a_long_row(what, D, S, dtype):
    """A query 2^26 times the others, or a key 2^10 times, with a strength that goes with it."""
    d = Delta(3, lens=(130,) * S, D=D, dtype=dtype, unit=False, scale=0.25)
    rows = torch.tensor([d.cu_h[s] + 50 + s for s in range(S)], device="cuda")
    if what == "q":
        d.q.mul_(2.0 ** -11)
        d.q[rows] *= 2.0 ** 26
    else:
        d.k[rows] *= 2.0 ** 10
        d.beta[rows] *= 2.0 ** -20
    check(d)
