"""gms_kv_delta with many states (whole ones through a ring of buffers) and with batches in which short and long sequences meet."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from kv_delta_harness import BF16, F16, Delta  # noqa: E402


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
