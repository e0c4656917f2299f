"""gms_kv_delta with many states (whole ones through a ring of buffers) and with batches in which short and long sequences meet."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from kv_delta_harness import BF16, F16, Delta  # noqa: E402
from paper_2609_25451_b200 import gms  # noqa: E402


@pytest.mark.parametrize("D,per", [(64, 8), (128, 2)])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("S", [38, 75, 101])
def test_one_row_each(D, per, dtype, S):
    Delta(S, lens=(1,) * S, decode=True, D=D, per=per, H=8, K=4, dtype=dtype, fresh=(1, S - 1)).check()


@pytest.mark.parametrize("D,per", [(64, 5), (128, 1)])
@pytest.mark.parametrize("kw", [dict(), dict(in_place=True), dict(unit=False, gates=False), dict(betas=False, fused=False), dict(gap=64, plane=1)])
def test_ragged_few_rows(D, per, kw):
    lens = tuple((i * 7) % 12 for i in range(80))  # none to eleven rows: more than a batch of eight among them
    Delta(3, lens=lens, D=D, per=per, H=10, K=5, fresh=(0, 5, 79), **kw).check()


@pytest.mark.parametrize("D,per", [(64, 8), (128, 2)])
def test_short_and_long_sequences(D, per):
    lens = tuple(70 if i % 19 == 3 else 200 if i == 40 else i % 4 for i in range(80))
    Delta(4, lens=lens, D=D, per=per, H=8, K=8, fresh=(3, 10)).check()


def test_holes():
    d = Delta(5, lens=(2,) * 90, H=4, per=2, fresh=(7,))
    for s in range(0, 90, 9):
        d.src_h[s, 0] = -1
        d.dst_h[(s + 4) % 90, 1] = d.n_blocks + s
    d.make()
    d.check()


def test_sequences_that_go_on_from_one_state():
    Delta(6, lens=(3,) * 100, H=4, per=2, same_source=True).check()


@pytest.mark.parametrize("extra", [-1, 0, 1, 2])
def test_around_the_number_of_states_where_the_kernel_changes(extra):
    Delta(7, lens=(1,) * (148 + extra), decode=True, H=2, K=1, per=2).check()
    Delta(8, lens=(1,) * (148 + extra), decode=True, H=4, K=2, per=8, D=64).check()


def test_nothing_but_long_sequences():
    Delta(9, lens=(30,) * 60, H=8, K=4, D=64, per=8).check()


def test_equal_calls_give_equal_bits():
    d = Delta(10, lens=(2, 1, 5) * 40, H=4, K=4, D=128)
    d.run()
    out, raw = d.out_full.clone(), d.raw.clone()
    for _ in range(5):
        d.run()
        assert torch.equal(out, d.out_full) and torch.equal(raw, d.raw)


@pytest.mark.parametrize("D,per,H", [(64, 8, 16), (128, 2, 4), (128, 2, 32)])
def test_a_long_sequence_among_single_rows(D, per, H):
    lens = tuple(700 if i == 21 else 1 for i in range(40))
    Delta(11, lens=lens, D=D, per=per, H=H, K=H // 2, dtype=F16 if D == 64 else BF16, fresh=(21,)).check()


def test_more_sequences_than_threads_make_the_order():
    lens = tuple((i * 37) % 90 for i in range(300))  # most of them in chunks, some alike, some without rows
    Delta(12, lens=lens, D=64, per=2, H=2, K=1, fresh=(0, 299)).check()


def test_a_bound_above_the_longest_sequence():
    Delta(13, lens=(30, 64, 3, 100, 90) * 6, D=128, per=2, H=4, K=4, max_q=1500).check()


def test_a_replayed_call_orders_the_sequences_anew():
    lens = [1] * 30
    lens[2] = 400
    d = Delta(14, lens=lens, D=128, per=2, H=4, K=2)
    d.run()
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        gms.gms_kv_delta(d.desc, d.state, d.args, s.cuda_stream)
    for at in ([(27, 400)], [(5, 140), (6, 200), (29, 62)]):
        lens = [1] * 30
        for i, n in at:
            lens[i] = n
        lens[0] += d.T - sum(lens)
        d.lens = lens
        d.cu_h = [0]
        for n in lens:
            d.cu_h.append(d.cu_h[-1] + n)
        d.cu.copy_(torch.tensor(d.cu_h, dtype=torch.int32))
        d.out_full.fill_(3.0)
        before = d.raw.clone()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        after, out = d.raw.clone(), d.out_full.clone()
        d.raw.copy_(before)
        d.run()                                     # the same call without a graph
        assert torch.equal(after, d.raw) and torch.equal(out, d.out_full)
        d.raw.copy_(before)
        d.check()
        assert torch.equal(out, d.out_full)


@pytest.mark.parametrize("lens", [(1, 300, 2, 70, 24, 25) * 3, (900,) + (1,) * 60])
def test_calls_one_behind_the_other(lens):
    """What follows on the stream finds states and outputs, of long sequences and of short ones."""
    a, b = (Delta(15, lens=lens, H=8, K=4, in_place=True) for _ in range(2))
    seen = []
    for _ in range(4):
        a.run()
        seen.append(a.out_full.clone())
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        for want in seen:
            b.out_full.fill_(3.0)
            gms.gms_kv_delta(b.desc, b.state, b.args, s.cuda_stream)
            want.sub_(b.out_full)
    torch.cuda.synchronize()
    assert all(not x.any() for x in seen) and torch.equal(a.raw, b.raw)


# (with row 40's own strength, f16 and up = 30 have no finite answer: the row's d k^T, of about 1, times e^30 = 10^13 is read at row 41)
@pytest.mark.parametrize("dtype,up,strength", [(BF16, 3.0, 1), (BF16, 30.0, 1), (F16, 3.0, 1), (BF16, 30.0, 0), (F16, 30.0, 0)])
def test_a_gate_far_above_zero(dtype, up, strength):
    d = Delta(16, lens=(130,), H=4, K=2, dtype=dtype)
    d.g[40], d.g[41] = -up, up  # what is lost comes back
    d.beta[40] *= strength
    d.check()


@pytest.mark.parametrize("n", [19, 20, 21, 22])
def test_around_the_length_from_which_chunks_are_taken(n):
    Delta(17, lens=(n, 40, n), H=4, K=2).check()


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("D", [64, 128])
def test_many_long_sequences_captured(D, dtype):
    d = Delta(18, lens=tuple(90 + i for i in range(30)), D=D, H=4, K=2, dtype=dtype, in_place=True)
    first = d.raw.clone()
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(g, stream=s):
        gms.gms_kv_delta(d.desc, d.state, d.args, s.cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(d.raw, first)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    after, out = d.raw.clone(), d.out_full.clone()
    d.raw.copy_(first)
    for _ in range(2):
        d.run()
    before = d.raw.clone()
    d.run()
    assert torch.equal(after, d.raw) and torch.equal(out, d.out_full)
    d.raw.copy_(before)
    d.check()


@pytest.mark.parametrize("D,per,S", [(64, 8, 12), (64, 8, 34), (128, 2, 6), (128, 2, 15)])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("what", ["v", "k", "q", "beta", "g", "state"])
def test_what_is_not_finite_stays_with_what_depends_on_it(D, per, S, dtype, what):
    """As for few sequences, with as many as let a CTA have two slices of a state or a warp one of its own."""
    n, at, bad = 130, 70, float("inf") if what in ("v", "beta") else float("nan")
    kw = dict(lens=(n,) * S, H=4, K=2, D=D, per=per, dtype=dtype)
    clean, d = Delta(19, **kw), Delta(19, **kw)
    row, start = d.cu_h[1] + at, d.cu_h[1]
    if what == "v":
        d.v[row, 1, 5] = bad
    elif what in "kq":
        getattr(d, what)[row, 0, 5] = bad
    elif what == "state":
        d.place(d.raw, d.src_h, 1, 1)[3, 5] = bad
        row = start
    else:
        getattr(d, what)[row, 1] = bad
    clean.run()
    d.run()
    cols = [5] if what in ("v", "state") else list(range(D))
    end = row + 1 if what == "q" else d.cu_h[2]
    for h in [0, 1] if what in ("k", "q") else [1]:
        assert not torch.isfinite(d.out[row:end, h][:, cols].float()).any()
        d.out[row:end, h, cols[0]:cols[-1] + 1] = clean.out[row:end, h, cols[0]:cols[-1] + 1]
        if what != "q":
            st, want = d.place(d.raw, d.dst_h, 1, h), clean.place(clean.raw, clean.dst_h, 1, h)
            assert not torch.isfinite(st[:, cols]).all()
            st[:, cols[0]:cols[-1] + 1] = want[:, cols[0]:cols[-1] + 1]
    if what == "state":
        d.place(d.raw, d.src_h, 1, 1)[3, 5] = clean.place(clean.raw, clean.src_h, 1, 1)[3, 5]
    n1, out, want, bound, e = clean.reference(clean.raw)[1]
    r = slice(start, d.cu_h[2])
    assert ((d.out[r].double() - out).abs() <= bound).all()
    for h in range(4):
        assert (d.place(d.raw, d.dst_h, 1, h).double() - want[h]).norm() <= e[h]
    d.out[r] = clean.out[r]
    for h in range(4):
        d.place(d.raw, d.dst_h, 1, h).copy_(clean.place(clean.raw, clean.dst_h, 1, h))
    assert torch.equal(d.out_full, clean.out_full) and torch.equal(d.raw, clean.raw)  # nothing else differs


@pytest.mark.parametrize("D,per,H,S,loose", [(128, 2, 4, 150, True), (128, 2, 32, 38, True), (64, 8, 8, 160, True), (64, 8, 16, 300, False), (128, 2, 8, 300, False)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_more_long_sequences_than_ctas(D, per, H, S, loose, dtype):
    """CTAs that go through several sequences; `loose`: more of them are long than the largest length lets expect."""
    lens = tuple(15 + (i * 29) % 60 + (130 if i % 31 == 5 else 0) for i in range(S))
    Delta(20, lens=lens, D=D, per=per, H=H, K=H // 2, dtype=dtype, fresh=(0, 7), max_q=sum(lens) if loose else None).check()
