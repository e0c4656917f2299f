"""Errors of the gated delta rule as norms: of a head's state, and of its outputs in blocks of 16 rows.

How far they may be off:

  state: 3e-5 of its norm.  What goes into a state in chunks does so in two 16-bit terms (2^-16 = 1.5e-5 relative at most each, of
         either sign); one term instead (2^-9 for bf16, 2^-12 for fp16 at the least) is 2e-4 to 4e-3.
  out:   its last rounding is off by at most u of each element (2^-8, fp16 2^-11), so by u of a block's norm; what an error of the
         state allows comes to it: 3e-5 |scale| |q_i| |S_i| of each row (Frobenius norms); fp16: 2^-25 an element below its normal range.
         In chunks the state before the chunk, S_0, enters an output as one 16-bit term: each element off by u of itself at most, so
         a column's part scale e^G q^T S_0 by u |scale| e^G |q|^T |S_0|, element for element.  Where that part does not cancel, this
         is within what the last rounding is allowed above its average; where it may, `one_term` adds it.
"""
from __future__ import annotations

import math

import torch

STATE = 3e-5
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
BLOCK = 16


def rule(q, k, v, g, beta, S, scale):
    """Row by row in 64 bits.  q, k, v [rows, heads, dim], g, beta [rows, heads], S [heads, key, value]: outputs, state, and what
    each row's output is measured by, all in 64 bits: |scale| |q| |S|, and the norm of |scale| e^G |q|^T |S_0| with S_0 the state before
    the row's 64 (0 where a sequence has no more than 20 rows, which are not done in chunks)."""
    q, k, v, g, beta, S = (x.double() for x in (q, k, v, g, beta, S))
    out, size = torch.zeros_like(v), torch.zeros(v.shape[:2] + (2,), dtype=torch.float64, device=v.device)
    gate = g.exp()
    for t in range(v.shape[0]):
        if t % 64 == 0:
            start = S.abs() if v.shape[0] > 20 else torch.zeros_like(S)
        start = start * gate[t][:, None, None]
        S = S * gate[t][:, None, None]
        d = beta[t][:, None] * (v[t] - torch.einsum("hkv,hk->hv", S, k[t]))
        S = S + k[t][:, :, None] * d[:, None, :]
        out[t] = scale * torch.einsum("hkv,hk->hv", S, q[t])
        size[t, :, 0] = abs(scale) * q[t].norm(dim=-1) * S.flatten(1).norm(dim=1)
        size[t, :, 1] = abs(scale) * torch.einsum("hkv,hk->hv", start, q[t].abs()).norm(dim=1)
    return out, S, size


def unit(x, eps):
    x = x.double()
    return x / ((x * x).sum(-1, keepdim=True) + eps).sqrt()


def state_errors(got, want):
    """Errors of states [heads, key, value] over their norms."""
    return (got.double() - want).flatten(1).norm(dim=1) / want.flatten(1).norm(dim=1).clamp(min=1e-300)


def out_errors(got, want, size, dtype, one_term=False):
    """Errors of outputs [rows, heads, dim] over what they may be, a block of rows and head each."""
    n, H, D = want.shape
    pad = -n % BLOCK

    def blocks(x):  # norms
        x = torch.cat([x, torch.zeros((pad, H, x.shape[2]), dtype=torch.float64, device=x.device)])
        return x.reshape(-1, BLOCK, H, x.shape[2]).transpose(1, 2).flatten(2).norm(dim=2)

    may = U[dtype] * blocks(want) + STATE * blocks(size[:, :, :1]) + (U[dtype] * blocks(size[:, :, 1:]) if one_term else 0)
    if dtype == torch.float16:
        may = may + 2.0 ** -25 * math.sqrt(BLOCK * D)
    return blocks(got.double() - want) / may.clamp(min=1e-300)


def expected(d, raw):
    """For a problem of kv_delta_harness (with the pool as it was): per sequence its rows, outputs, state and the outputs' sizes."""
    inputs = []
    for s, n in enumerate(d.lens):
        n = min(n, d.max_q)
        r = slice(d.cu_h[s], d.cu_h[s] + n)
        q, k = ((unit(x[r], d.eps) if d.unit else x[r].double()).repeat_interleave(d.H // d.K, 1) for x in (d.q, d.k))
        g = d.g[r] if d.g is not None else torch.zeros((n, d.H), device=q.device)
        beta = d.beta[r] if d.beta is not None else torch.ones((n, d.H), device=q.device)
        S = torch.zeros((d.H, d.D, d.D), dtype=torch.float64, device=q.device)
        for h in range(d.H):
            x = None if d.fresh[s] else d.place(raw, d.src_h, s, h)
            if x is not None:
                S[h] = x
        inputs.append((r, q, k, d.v[r], g, beta, S))
    res = [None] * len(inputs)
    for n in {x[3].shape[0] for x in inputs}:  # sequences of one length side by side
        which = [s for s, x in enumerate(inputs) if x[3].shape[0] == n]
        q, k, v, g, beta = (torch.cat([inputs[s][i] for s in which], 1) for i in range(1, 6))
        out, S, size = rule(q, k, v, g, beta, torch.cat([inputs[s][6] for s in which]), d.scale)
        for i, s in enumerate(which):
            h = slice(i * d.H, (i + 1) * d.H)
            res[s] = (inputs[s][0], out[:, h], S[h], size[:, h])
    return res


def check(d, run=True, one_term=False):
    """Runs a problem (without holes) and holds its outputs and states to the limits; returns the largest errors, over the limits."""
    before = d.raw.clone()
    if run:
        d.run()
    worst = [0.0, 0.0]
    for s, (r, out, S, size) in enumerate(expected(d, before)):
        got = torch.stack([d.place(d.raw, d.dst_h, s, h) for h in range(d.H)])
        errs = state_errors(got, S) / STATE
        assert torch.isfinite(got).all() and errs.max() <= 1, ("state", s, errs.tolist())
        worst[0] = max(worst[0], float(errs.max()))
        if out.shape[0]:
            errs = out_errors(d.out[r], out, size, d.dtype, one_term)
            assert torch.isfinite(d.out[r].float()).all() and errs.max() <= 1, ("out", s, errs.max(), errs.argmax())
            worst[1] = max(worst[1], float(errs.max()))
    return worst
