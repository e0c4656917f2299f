"""gms_kv_delta where numbers of one chunk are far apart: gates above 0, rows and keys of very different lengths, values near the types' ends."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from kv_delta_harness import BF16, F16, Delta  # noqa: E402
from kv_delta_norms import check, expected, out_errors  # noqa: E402

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


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("D,S", FORMS)
@pytest.mark.parametrize("apart", [16, 20, 26])
def test_keys_of_many_lengths(apart, D, S, dtype):
    """Keys that are brought to unit length, from 2^-12 of it on."""
    d = Delta(4, lens=(130,) * S, D=D, dtype=dtype)
    g = torch.Generator(device="cuda").manual_seed(apart)
    d.k.mul_(torch.exp2(-12 + apart * torch.rand((d.T, d.K, 1), device="cuda", generator=g)))
    check(d)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("D,S", FORMS)
def test_keys_of_zero(D, S, dtype):
    d = Delta(5, lens=(130,) * S, D=D, dtype=dtype)
    d.eps = 1e-12
    d.k[3::5] = 0
    d.make()
    check(d, one_term=True)  # (a row without a key has nothing but the state's part, which its query may all but miss)


@pytest.mark.parametrize("D,S", FORMS)
@pytest.mark.parametrize("at", [40, 72, 79, 127])
@pytest.mark.parametrize("what", ["value", "two values", "state"])
def test_a_difference_beyond_the_range(what, at, D, S):
    """A row whose difference between value and state 32 bits cannot hold: rows before it, and columns beside it, are as without it."""
    kw = dict(lens=(130,) * S, D=D, unit=False, gates=False)
    clean, d = Delta(6, **kw), Delta(6, **kw)
    row, col = d.cu_h[S - 1] + at, 5
    if what == "state":  # finite, but not its product with the row's key
        for x in (clean, d):
            x.place(x.raw, x.src_h, S - 1, 1)[:, col] = 2e37
        d.k[row, 0] = 16.0
        heads = [0, 1]  # (of the key)
    else:
        for x in (clean, d):
            x.beta[row - 1:row + 1] = 2.0
            x.k[row] = x.k[row - 1]
        if what == "two values":
            d.v[row - 1, 1, col] = -3e38
        d.v[row, 1, col] = 3e38
        heads = [1]
    before = clean.raw.clone()
    clean.run()
    d.run()
    for s, (r, out, _, size) in enumerate(expected(clean, before)):
        stop = r.stop if s < S - 1 else row - (what == "two values")
        part = slice(r.start, stop)
        n = stop - r.start
        for x in (clean, d):
            got = x.out[part]
            assert torch.isfinite(got.float()).all(), s
            assert out_errors(got, out[:n], size[:n], BF16).max() <= 1, s
    for h in range(4):
        cols = slice(0, D) if h in heads and what == "state" else slice(col, col + 1)
        if h in heads:
            d.out[row - 1:, h, cols] = clean.out[row - 1:, h, cols]
            got = d.place(d.raw, d.dst_h, S - 1, h)
            got[:, cols] = clean.place(clean.raw, clean.dst_h, S - 1, h)[:, cols]
    assert torch.isfinite(d.out.float()).all() and torch.isfinite(d.raw).all()
    # (what is left of the sequence may have been computed row by row)
    assert ((d.out.float() - clean.out.float()).abs() <= 2.0 ** -7 * clean.out.float().abs() + 0.02).all() or what == "state"


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("D,S", FORMS)
@pytest.mark.parametrize("size", [1e9, 1e13, 1e16, 1e22])
def test_states_far_from_one(size, D, S, dtype):
    """Also beyond what fp16's terms can be scaled to."""
    check(Delta(7, lens=(130,) * S, D=D, dtype=dtype, state_scale=size, scale=0.1 / size))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("D,S", FORMS)
@pytest.mark.parametrize("up", [12.0, 20.0, 30.0, 40.0, 55.0])
def test_a_gate_above_zero_in_the_next_chunk(up, D, S, dtype):
    """The state between the two chunks is e^-up of what it was and becomes."""
    d = Delta(8, lens=(150,) * S, D=D, dtype=dtype)
    for s in range(S):
        r = d.cu_h[s] + (63 if s % 2 == 0 else 127)
        d.g[r], d.g[r + 1] = -up, up
        d.beta[r] = 0
    check(d)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("D,S", FORMS)
@pytest.mark.parametrize("size", [1e-6, 1e-12, 1e-20])
def test_states_near_zero(size, D, S, dtype):
    """Values of zero: nothing else is in them.  (Gates that leave e^-2 of a state: full decay, e^-60, ends where 32 bits do, 2^-126, or
    where the second of two bf16 terms does, 2^-109.)"""
    d = Delta(9, lens=(150,) * S, D=D, dtype=dtype, state_scale=size, scale=0.1 / size, decay=0.03)
    d.v.zero_()
    check(d)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("D,S", FORMS)
def test_states_of_zero_under_a_gate_above_zero(D, S, dtype):
    d = Delta(10, lens=(70,) * S, D=D, dtype=dtype, fresh=tuple(range(S)))
    d.v.zero_()
    d.g[20] = 75.0
    d.run()
    assert (d.out == 0).all()
    for s in range(S):
        for h in range(4):
            assert (d.place(d.raw, d.dst_h, s, h) == 0).all()
