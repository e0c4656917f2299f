"""gms_kv_delta against the rule in 64 bits, row by row (tests/kv_delta_harness.py derives how far results may be off)."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from kv_delta_harness import BF16, F16, Delta  # noqa: E402
from paper_2609_25451_b200 import gms  # noqa: E402


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 3, 8, 9, 16, 17, 33, 63, 64, 65, 127, 128, 129, 200, 500])
def test_lengths(dtype, D, n):
    Delta(n, dtype=dtype, D=D, lens=(n,)).check()


@pytest.mark.parametrize("H,K", [(1, 1), (2, 1), (6, 2), (5, 5), (16, 4), (3, 1)])
@pytest.mark.parametrize("lens", [(1, 1, 1), (3, 0, 130), (64, 1, 0, 65, 20)])
def test_heads_and_ragged_batches(H, K, lens):
    Delta(H, H=H, K=K, lens=lens, fresh=(0, 2)).check()


@pytest.mark.parametrize("n", [1, 4, 150])
@pytest.mark.parametrize("kw", [dict(unit=False), dict(gates=False), dict(betas=False), dict(gates=False, betas=False), dict(fused=False), dict(in_place=True),
                                dict(per=1), dict(per=1, D=64), dict(per=8, D=64, H=12, K=3), dict(plane=2, gap=64), dict(scale=-3.0), dict(decay=30.0),
                                dict(beta_scale=2.0), dict(pad_rows=5), dict(same_source=True), dict(fresh=(0, 1)), dict(dtype=F16, unit=False, decay=4.0)])
def test_forms(n, kw):
    Delta(n, lens=(n, n, n // 2), **kw).check()


@pytest.mark.parametrize("S", [1, 7, 64])
@pytest.mark.parametrize("D", [64, 128])
def test_one_row_each_without_offsets(S, D):
    Delta(S, lens=(1,) * S, decode=True, D=D, H=8, K=4, fresh=(0,) if S > 1 else ()).check()


@pytest.mark.parametrize("n", [40, 64, 300])
def test_keys_that_are_nearly_alike(n):
    """I + A is far from the identity: ones all over its lower triangle."""
    Delta(n, lens=(n,), key_noise=0.01, betas=False, gates=False).check()
    Delta(n, lens=(n,), key_noise=0.0, beta_scale=1.0, decay=0.01).check()
    Delta(n, lens=(n,), key_noise=0.05, beta_scale=2.0, decay=0.01, dtype=F16).check()


@pytest.mark.parametrize("n", [3, 100])
def test_gates_that_clear_the_state(n):
    d = Delta(5, lens=(n, n), H=4, K=4)
    d.g[1, 0], d.g[n // 2, 1], d.g[n, 2], d.g[n + 1, 3] = -float("inf"), -float("inf"), -150.0, -1e30
    d.g[n - 1, 0] = -float("inf")
    ref = Delta(5, lens=(n, n), H=4, K=4)
    d.check()
    assert torch.equal(ref.v, d.v)


def test_strengths_of_zero_leave_the_state():
    d = Delta(6, lens=(90, 1), gates=False)
    d.beta.zero_()
    before = d.raw.clone()
    d.check()
    for s in range(2):
        for h in range(d.H):
            assert torch.equal(d.place(d.raw, d.dst_h, s, h), d.place(before, d.src_h, s, h))


@pytest.mark.parametrize("n", [1, 70])
def test_holes(n):
    d = Delta(7, lens=(n, n, n), H=4, per=2)
    d.src_h[0, 1], d.dst_h[1, 0], d.src_h[2, 0], d.dst_h[2, 0] = -1, d.n_blocks, 10**6, -5
    d.make()
    d.check()


@pytest.mark.parametrize("max_q", [1, 50, 64, 100])
def test_rows_beyond_max_q_are_left_alone(max_q):
    Delta(8, lens=(130, 20, 64), max_q=max_q).check()


def test_nothing_to_do():
    d = Delta(9, lens=(0, 0), fresh=(1,), pad_rows=3)
    d.check()
    e = Delta(10, lens=(4,))
    e.args.n_seq = 0
    e.args.total_q = e.args.max_q = 0
    before = e.raw.clone()
    e.run()
    assert torch.equal(before, e.raw) and (e.out_full == 3).all()


@pytest.mark.parametrize("n,at", [(6, 3), (64, 0), (64, 63), (200, 70), (200, 130)])
@pytest.mark.parametrize("what", ["v", "k", "q", "beta", "g"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_a_row_does_not_depend_on_cannot_reach_it(n, at, what, bad):
    """A value that is not finite at row `at` of the second sequence: rows before it, other sequences and other heads (and for a
    value's column, other columns) are as without it; from it on the head (the column, the row alone for q) is not finite."""
    kw = dict(lens=(n, n, 3), H=4, K=2, D=64, per=8)
    clean, d = Delta(11, **kw), Delta(11, **kw)
    row = d.cu_h[1] + at
    if what == "v":
        d.v[row, 1, 5] = bad
    elif what in "kq":
        getattr(d, what)[row, 0, 5] = bad
    else:
        getattr(d, what)[row, 1] = bad
    clean.run()
    d.run()
    heads = [0, 1] if what in ("k", "q") else [1]
    end = d.cu_h[2]
    cols = [5] if what == "v" else list(range(64))
    if what == "q":
        end = row + 1
    for h in heads:
        touched = d.out[row:end, h][:, cols].float()
        assert not torch.isfinite(touched).any()
        d.out[row:end, h, cols[0]:cols[-1] + 1] = clean.out[row:end, h, cols[0]:cols[-1] + 1]
        if what != "q":
            st, want = d.place(d.raw, d.dst_h, 1, h), clean.place(clean.raw, clean.dst_h, 1, h)
            assert not torch.isfinite(st[:, cols]).all()
            st[:, cols[0]:cols[-1] + 1] = want[:, cols[0]:cols[-1] + 1]
    # what is left of that sequence may have been computed another way: it stays within its bounds
    before = torch.where(torch.isfinite(d.raw), d.raw, clean.raw)
    ref = clean.reference(before)
    for s in (0, 2):
        r = slice(d.cu_h[s], d.cu_h[s + 1])
        assert torch.equal(d.out[r], clean.out[r])
    n1, out, S, bound, e = ref[1]
    r = slice(d.cu_h[1], d.cu_h[2])
    assert ((d.out[r].double() - out).abs() <= bound).all()
    for h in range(4):
        assert (d.place(d.raw, d.dst_h, 1, h).double() - S[h]).norm() <= e[h]


@pytest.mark.parametrize("n", [1, 100])
def test_captured_and_replayed_in_place(n):
    """Steps of a graph go on from the state that the last one left; another stream."""
    d = Delta(12, lens=(n, n), in_place=True)
    start = d.raw.clone()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        gms.gms_kv_delta(d.desc, d.state, d.args)
    assert torch.equal(start, d.raw)
    for step in range(3):
        was = d.raw.clone()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        now = d.raw.clone()
        d.raw.copy_(was)
        ref = d.reference(d.raw)
        d.raw.copy_(now)
        for q, (m, out, S, bound, e) in enumerate(ref):
            r = slice(d.cu_h[q], d.cu_h[q] + m)
            assert ((d.out[r].double() - out).abs() <= bound).all()
            for h in range(d.H):
                assert (d.place(d.raw, d.dst_h, q, h).double() - S[h]).norm() <= e[h]
        d.v.copy_(torch.randn(d.v.shape, device="cuda"))
        torch.cuda.synchronize()


def test_two_calls_at_once():
    a, b = (Delta(seed, lens=(300, 40), H=8, K=4) for seed in (13, 14))
    befores = a.raw.clone(), b.raw.clone()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        gms.gms_kv_delta(a.desc, a.state, a.args, s)
        gms.gms_kv_delta(b.desc, b.state, b.args, t)
    torch.cuda.synchronize()
    for x, before in zip((a, b), befores):
        for q, (m, out, S, bound, e) in enumerate(x.reference(before)):
            r = slice(x.cu_h[q], x.cu_h[q] + m)
            assert ((x.out[r].double() - out).abs() <= bound).all()


def test_equal_calls_give_equal_bits():
    d = Delta(15, lens=(700, 64, 1, 129), H=8, K=2)
    d.run()
    out, raw = d.out_full.clone(), d.raw.clone()
    for _ in range(5):
        d.ws.random_(0, 256)
        d.run()
        assert torch.equal(out, d.out_full) and torch.equal(raw, d.raw)


def test_one_workspace_for_smaller_calls():
    big = Delta(16, lens=(300, 200, 100), H=4, K=2)
    for lens in ((300,), (64, 1), (1, 1, 1), (65, 64, 63)):
        d = Delta(17, lens=lens, H=4, K=2)
        assert gms.gms_kv_delta_workspace(d.desc, d.state, d.args) <= gms.gms_kv_delta_workspace(big.desc, big.state, big.args)
        d.args.set_workspace(big.ws)
        d.check()


def test_a_long_prompt_with_long_memory():
    Delta(18, lens=(4000,), H=2, K=1, decay=0.001, D=64, per=8).check()
