"""gms_kv_delta's states and outputs by their norms (tests/kv_delta_norms.py says how far they may be off)."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from kv_delta_harness import BF16, F16, Delta  # noqa: E402
from kv_delta_norms import check  # noqa: E402

# head_dim, sequences of 4 heads: one slice of a state a CTA, two, a warp each
FORMS = [(128, 1), (128, 6), (128, 12), (64, 1), (64, 12), (64, 20)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("D,S", FORMS)
@pytest.mark.parametrize("n", [1, 4, 20, 21, 64, 65, 130, 500])
def test_lengths(n, D, S, dtype):
    if n * S > 3000:
        S = max(3000 // n, 1)
    check(Delta(n, lens=(n,) * S, D=D, dtype=dtype, fresh=(0,) if S > 1 else ()))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("kw", [dict(unit=False), dict(gates=False), dict(betas=False), dict(decay=0.01), dict(decay=30.0), dict(beta_scale=2.0),
                                dict(scale=-3.0), dict(key_noise=0.3)])
def test_forms(kw, dtype):
    check(Delta(2, lens=(150, 1, 70), dtype=dtype, **kw))
    check(Delta(3, lens=(100, 90) * 8, dtype=dtype, D=64, per=8, **kw))


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_a_long_prompt(dtype):
    check(Delta(4, lens=(2500,), H=2, K=1, decay=0.01, D=64, per=8, dtype=dtype))


@pytest.mark.parametrize("D,per", [(64, 8), (128, 2)])
def test_steps_of_one_batch_in_place(D, per):
    """Prompts of some, then tokens: each step goes on from the state that the last one left."""
    first = None
    for step, lens in enumerate(([40, 1, 0, 170, 33], [1, 1, 30, 1, 1], [1, 0, 100, 2, 1], [3, 3, 3, 3, 3], [1, 1, 1, 1, 1])):
        d = Delta(40 + step, lens=lens, H=8, K=4, D=D, per=per, in_place=True)
        if first is None:
            first = d
        else:
            d.raw.copy_(first.raw)
            d.src_h = first.src_h
            d.dst_h = first.src_h
            d.make()
        check(d, one_term=True)  # (blocks of one row)
        first.raw.copy_(d.raw)


@pytest.mark.parametrize("n", [20, 21, 22, 41, 42, 63, 64, 65, 85])
@pytest.mark.parametrize("others", [1, 7, 20])
def test_where_the_workspace_has_no_room_for_short_sequences(n, others):
    """Some sequences in chunks among many that are not, so that slots go by where rows begin."""
    lens = [n if i % 9 == 4 else (i * 5) % (others + 1) for i in range(60)]
    d = Delta(n, lens=lens, H=2, K=1, D=64, per=2)
    most = (-(-sum(lens) // 21) + 1) * 2 * 23000 + 256
    assert n < 21 or d.ws.numel() <= most
    check(d, one_term=True)  # (blocks of few rows)
