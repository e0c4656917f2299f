"""What infinities and NaN in the values cost: rows that see them are non-finite whatever is done, and only rows that share a
tile with one that they do not see are worked over again.  Results against the 64-bit reference, times against a limit."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2609_25451_b200 import gms  # noqa: E402

if torch.cuda.is_available():
    from kv_attn_harness import Problem  # noqa: E402


def early_infinity(p):
    p.V[0][10, :, 5] = math.inf


def left_the_window(p):
    p.V[0][50] = math.nan


def two_places(p):
    p.V[0][700, :, 3] = math.nan
    p.V[0][2500, :, 70] = -math.inf


def one_column(p):
    p.V[0][:, :, 5] = math.nan


def newest_column(p):
    p.V[0][-300:, :, 64] = math.inf


def everything(p):
    p.V[0][:] = math.nan


@pytest.mark.parametrize("poison", [early_infinity, left_the_window, two_places, one_column, newest_column, everything])
@pytest.mark.parametrize("window,sinks,q", [(0, 0, 1500), (256, 4, 1500), (0, 0, 4), (256, 4, 4)])
def test_time_and_result(poison, window, sinks, q):
    """8 / 2 heads of 128 over 4,000 tokens take some 50 us; the rows of one tile done again, token by token, a few ms.  (All
    rows that see an infinity done again would be hundreds of ms.)"""
    p = Problem(2, heads=8, kv_heads=2, q_lens=(q, 1), kv_lens=(4000, 300), window=window, sinks=sinks, poison=poison)
    p.run()
    p.check()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    gms.gms_kv_attention(p.desc, p.layout, p.attn)
    b.record()
    torch.cuda.synchronize()
    assert a.elapsed_time(b) < 15.0


@pytest.mark.parametrize("poison", [early_infinity, newest_column, everything])
def test_behind_a_prefix(poison):
    def both(p):
        poison(p)
        p.PV[0][20, :, 9] = math.nan

    p = Problem(3, heads=8, kv_heads=2, q_lens=(40, 3), kv_lens=(2000, 90), prefix_lens=(1000, 33), groups=[0, 1, 2], poison=both)
    x = p.make_prefix()
    p.run(prefix=x)
    p.check()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    gms.gms_kv_attention_shared(p.desc, p.layout, p.attn, x)
    b.record()
    torch.cuda.synchronize()
    assert a.elapsed_time(b) < 15.0


def test_more_items_than_one_turn_looks_at():
    """1,600 items of 256 rows; in some sequences, the last ones too, values that the newest queries alone see are infinite."""
    def poison(p):
        for s in (0, 7, 123, 250, 398, 399):
            p.V[s][-1, :, s % 64] = math.inf
            p.V[s][-40, 1, 3] = math.nan

    p = Problem(4, heads=4, kv_heads=2, dim=64, block=64, q_lens=(140,) * 400, kv_lens=tuple(140 + s % 90 for s in range(400)), poison=poison)
    p.run()
    p.check()
