"""Calls whose device arrays go beyond what the host announced (max_q, max_kv, max_group_q): what is left out changes nothing
about the positions, and so the masks, of what is processed.  Tolerances are derived in kv_attn_harness."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2609_25451_b200 import gms  # noqa: E402

if torch.cuda.is_available():
    from kv_attn_harness import Problem  # noqa: E402


def first_tokens_only(p, max_kv):
    """Tokens from max_kv on are seen by nobody."""
    plain = p.visible

    def visible(s):
        v = plain(s)
        v[:, max_kv:] = False
        return v

    p.visible = visible
    p.attn.max_kv = max_kv


def check_rows(p, processed):
    """Rows processed[s] of each sequence are right, the others are as they were."""
    left = []
    for s, (out, otol, lse, ltol, _, _) in enumerate(p.reference()):
        k, b = processed[s], p.cu_h[s]
        got, glse = p.out[b:p.cu_h[s + 1]].double(), p.lse[b:p.cu_h[s + 1]].double()
        assert not bool(((got - out).abs()[:k] > otol[:k]).any()), f"sequence {s}: out off by {float((got - out).abs()[:k].max())}"
        empty = lse[:k] == -math.inf
        assert bool((glse[:k][empty] == -math.inf).all()) and bool((got[:k][empty] == 0).all())
        assert not bool(((glse - lse).abs()[:k][~empty] > ltol[:k][~empty]).any()), f"sequence {s}: lse"
        assert bool((got[k:] == 3).all()) and bool((glse[k:] == 77).all()), f"sequence {s}: rows that are not processed"
        left.append(got.shape[0] - k)
    return left


def weight_sums(p, s, rows):
    """Sums of the weights of the first `rows` queries of sequence s, in 64 bits: [kv heads, tokens]."""
    G, b = p.H // p.C, p.cu_h[s]
    vis = p.visible(s)[:rows]
    w = torch.zeros((p.C, p.kv_lens[s]), dtype=torch.float64, device="cuda")
    for h in range(p.H):
        x = p.q[b:b + rows, h].double() @ p.K[s][:, h // G].double().T * p.scale
        e = torch.where(vis, torch.exp(x - x.amax(1, keepdim=True)), 0.0)
        w[h // G] += (e / e.sum(1, keepdim=True).clamp_min(1e-300)).sum(0)
    return w


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 2)])
@pytest.mark.parametrize("q_lens,max_q", [((5, 9, 1, 2), 2), ((5, 1, 3, 2), 1), ((200, 9, 1, 150), 100), ((70, 9, 12, 40), 20)])
def test_more_queries_than_announced(dtype, window, sinks, q_lens, max_q):
    kv_lens = (300, 40, 77, 160)
    p = Problem(1, dtype=dtype, heads=8, kv_heads=2, q_lens=q_lens, kv_lens=kv_lens, window=window, sinks=sinks)
    p.attn.max_q = max_q
    w = torch.full((4, 2, 300), -5.0, device="cuda")
    p.run(gms.kv_weights(None, w))
    done = [min(q, max_q) for q in q_lens]
    assert sum(check_rows(p, done)) == sum(q_lens) - sum(done) > 0
    for s, n in enumerate(kv_lens):
        want = weight_sums(p, s, done[s])
        # a weight is off by its logit's error (bounded by 2^-12 at these sizes) and the sum's roundings
        assert not bool(((w[s, :, :n].double() - want).abs() > 2.0 ** -11 * want + 1e-9).any()), s
        assert bool((w[s, :, n:] == -5).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("window,sinks", [(0, 0), (90, 3), (20, 0), (20, 150)])
@pytest.mark.parametrize("q", [1, 3, 130])
@pytest.mark.parametrize("max_kv", [200, 100])
def test_more_tokens_than_announced(dtype, window, sinks, q, max_kv):
    """The queries keep their places behind tokens that the call does not reach; a window may then leave them nothing to see."""
    kv_lens = (300, q + 30, 210 + q)
    p = Problem(2, dtype=dtype, heads=8, kv_heads=2, q_lens=(q,) * 3, kv_lens=kv_lens, window=window, sinks=sinks, decode=q == 1)
    first_tokens_only(p, max_kv)
    w = torch.full((3, 2, 400), -5.0, device="cuda")
    p.run(gms.kv_weights(None, w))
    check_rows(p, (q,) * 3)
    for s, n in enumerate(kv_lens):
        n = min(n, max_kv)
        want = weight_sums(p, s, q)[:, :n]
        assert not bool(((w[s, :, :n].double() - want).abs() > 2.0 ** -11 * want + 1e-9).any()), s
        assert bool((w[s, :, n:] == -5).all())


@pytest.mark.parametrize("q_lens,max_group_q", [((1,) * 20, 7), ((30, 1, 40, 1, 1), 31)])
def test_more_rows_in_a_group_than_announced(q_lens, max_group_q):
    """Rows of a group beyond max_group_q are not processed (their prefix would be missing)."""
    S = len(q_lens)
    p = Problem(3, heads=8, kv_heads=2, q_lens=q_lens, kv_lens=tuple(50 + s for s in range(S)), prefix_lens=(300, 41), groups=[0, S - 1, S])
    x = p.make_prefix()
    x.max_group_q = max_group_q
    p.run(prefix=x)
    done, before = [], 0
    for s, q in enumerate(q_lens):
        if s == S - 1:
            before = 0
        done.append(max(0, min(q, max_group_q - before)))
        before += q
    assert sum(check_rows(p, done)) > 0
