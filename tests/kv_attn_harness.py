"""Problems and 64-bit reference of the attention and eviction calls on the paged KV pool.

The reference gathers every sequence's keys and values token by token, masks them one (query, token) pair at a time and
works in float64; it shares nothing with the library.  `bounds` derives how far a result may be off:

  logits: products of 16-bit numbers are exact in 32 bits, their sum of D terms and the scaling are off by at most
          dx = (D + 8) 2^-24 scale sum|q k| + 2^-22 (|x| + |m|)  (exponent argument formed in 32 bits)
  softmax weights p: relative 2 dx (its own logit and the normaliser's) + 2^-21 (exponential, quotient)
          + n 2^-24 (the sum of n terms), then one rounding to the pool's type, u = eps / 2 of the type: 2^-8 (bf16) or 2^-11 (f16; below
          2^-14 of the running maximum absolute 2^-25)
  out:    sum p |v| times (that + u + n 2^-24) for the products' sum, plus u |out| for the last rounding
"""
from __future__ import annotations

import math

import numpy as np
import torch

from paper_2609_25451_b200 import gms

U = {t: torch.finfo(t).eps / 2 for t in (torch.bfloat16, torch.float16)}  # unit roundoff, round to nearest


class Problem:
    """A pool with shuffled tables, ragged queries and outputs surrounded by canaries."""

    def __init__(self, seed, *, dtype=torch.bfloat16, heads=8, kv_heads=2, dim=128, block=16, order="token", q_lens=(1,),
                 kv_lens=(37,), window=0, sinks=0, prefix_lens=(), groups=None, pad_block=0, plane_gap=0, head_gap=0, max_extra=0,
                 planes=(0, 1), poison=None, q_scale=1.5, v_scale=1.0, holes=(), q_pad=0, lse=True, decode=False, table_pad=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.dtype, self.H, self.C, self.D, self.B, self.order = dtype, heads, kv_heads, dim, block, order
        self.q_lens, self.kv_lens, self.window, self.sinks = list(q_lens), list(kv_lens), window, sinks
        self.prefix_lens = list(prefix_lens)
        self.groups = groups
        S = len(self.kv_lens)
        if order == "token":
            hs, ts = dim * 2 + head_gap, kv_heads * (dim * 2 + head_gap)
        else:
            ts, hs = dim * 2 + head_gap, block * (dim * 2 + head_gap)
        used = (block - 1) * ts + (kv_heads - 1) * hs + dim * 2
        self.block_bytes = (used + 4095) // 4096 * 4096
        assert self.block_bytes <= 131072
        self.ts, self.hs = ts, hs
        self.block_stride = self.block_bytes + pad_block
        need = [(n + block - 1) // block for n in self.kv_lens]
        pneed = [(n + block - 1) // block for n in self.prefix_lens]
        self.n_blocks = sum(need) + sum(pneed) + 3
        self.plane_stride = self.n_blocks * self.block_stride + plane_gap
        self.n_planes = max(planes) + 1
        self.kp, self.vp = planes
        # every byte of the pool is random bits at first (NaN patterns included); then the tokens that exist get values
        self.raw = torch.randint(0, 256, (self.n_planes * self.plane_stride,), dtype=torch.uint8, device="cuda", generator=g)
        ids = list(rng.permutation(self.n_blocks))
        self.table_h = [[int(ids.pop()) for _ in range(k)] for k in need]
        self.prefix_h = [[int(ids.pop()) for _ in range(k)] for k in pneed]
        self.K = [torch.randn((n, kv_heads, dim), device="cuda", generator=g).to(dtype) for n in self.kv_lens]
        self.V = [(torch.randn((n, kv_heads, dim), device="cuda", generator=g) * v_scale).to(dtype) for n in self.kv_lens]
        self.PK = [torch.randn((n, kv_heads, dim), device="cuda", generator=g).to(dtype) for n in self.prefix_lens]
        self.PV = [(torch.randn((n, kv_heads, dim), device="cuda", generator=g) * v_scale).to(dtype) for n in self.prefix_lens]
        self.seen_by_none = []
        if poison is not None:
            poison(self)
        for t, k, v in zip(self.table_h + self.prefix_h, self.K + self.PK, self.V + self.PV):
            self.store(self.kp, t, k)
            self.store(self.vp, t, v)
        for s, j, bad in holes:  # block j of sequence s is taken out of the table
            self.table_h[s][j] = bad
        width = max([1] + need) + table_pad
        self.table = torch.tensor([r + [-7] * (width - len(r)) for r in self.table_h], dtype=torch.int32, device="cuda").view(S, width)
        pw = max([1] + pneed)
        self.prefix = torch.tensor([r + [-7] * (pw - len(r)) for r in self.prefix_h], dtype=torch.int32, device="cuda")
        T = sum(self.q_lens)
        self.T = T
        self.qfull = torch.randn((T, heads + q_pad, dim), device="cuda", generator=g).mul_(q_scale).to(dtype)
        self.q = self.qfull[:, :heads]
        self.ofull = torch.full((T + 2, heads + q_pad, dim), 3.0, dtype=dtype, device="cuda")
        self.out = self.ofull[1:T + 1, :heads]
        self.lfull = torch.full((T + 2, heads), 77.0, device="cuda")
        self.lse = self.lfull[1:T + 1] if lse else None
        self.cu_h = np.concatenate([[0], np.cumsum(self.q_lens)]).tolist()
        self.cu = torch.tensor(self.cu_h, dtype=torch.int32, device="cuda")
        self.lens = torch.tensor(self.kv_lens, dtype=torch.int32, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int64, device="cuda")
        self.scale = 1.0 / math.sqrt(dim)
        self.desc = gms.KvPool(base=self.raw.data_ptr(), plane_stride=self.plane_stride, block_stride=self.block_stride,
                               n_planes=self.n_planes, n_blocks=self.n_blocks, block_bytes=self.block_bytes)
        self.layout = gms.KvLayout(k_plane=self.kp, v_plane=self.vp, n_kv_heads=kv_heads, head_dim=dim, block_tokens=block,
                                   dtype=gms.DTYPE_BF16 if dtype == torch.bfloat16 else gms.DTYPE_F16, token_stride=ts, head_stride=hs)
        self.attn = gms.kv_attn(q=self.q, out=self.out, lse=self.lse, cu_q=None if decode else self.cu, kv_lens=self.lens,
                                block_table=self.table, max_q=max([1] + self.q_lens) if T else 0, max_kv=max([0] + self.kv_lens) + max_extra,
                                window=window, sinks=sinks, scale=self.scale, status=self.status)

    def view(self, plane):
        """[blocks, tokens, heads, dim] view of one plane."""
        x = self.raw[plane * self.plane_stride:].view(self.dtype)
        return torch.as_strided(x, (self.n_blocks, self.B, self.C, self.D),
                                (self.block_stride // 2, self.ts // 2, self.hs // 2, 1))

    def store(self, plane, table, rows):
        if len(rows) == 0:
            return
        t = np.arange(len(rows))
        b = torch.tensor(np.array(table)[t // self.B], device="cuda")
        self.view(plane)[b, torch.tensor(t % self.B, device="cuda")] = rows

    def run(self, weight=None, prefix=None, stream=None):
        if prefix is None:
            n = gms.gms_kv_attention_workspace(self.desc, self.layout, self.attn, weight)
        else:
            n = gms.gms_kv_attention_shared_workspace(self.desc, self.layout, self.attn, prefix)
        # the workspace's bits before the call must not matter
        self.ws = torch.full((max(n, 1) + 256,), 0xFF, dtype=torch.uint8, device="cuda")
        self.attn.set_workspace(self.ws[:max(n, 1)])
        if prefix is None:
            gms.gms_kv_attention(self.desc, self.layout, self.attn, weight, stream)
        else:
            gms.gms_kv_attention_shared(self.desc, self.layout, self.attn, prefix, stream)
        torch.cuda.synchronize()
        assert int(self.status.item()) == 0
        assert bool((self.ws[max(n, 1):] == 0xFF).all()), "the workspace was written beyond its size"
        assert bool((self.ofull[0] == 3).all()) and bool((self.ofull[-1] == 3).all()) and bool((self.ofull[:, self.H:] == 3).all())
        assert bool((self.lfull[0] == 77).all()) and bool((self.lfull[-1] == 77).all())

    def make_prefix(self):
        gs = self.groups
        self.gs = torch.tensor(gs, dtype=torch.int32, device="cuda")
        self.pl = torch.tensor(self.prefix_lens, dtype=torch.int32, device="cuda")
        rows = [self.cu_h[b] - self.cu_h[a] for a, b in zip(gs, gs[1:])]
        return gms.kv_prefix(group_start=self.gs, prefix_lens=self.pl, prefix_table=self.prefix, max_prefix=max(self.prefix_lens),
                             max_group_q=max(rows))

    def visible(self, s):
        """[queries, tokens] of sequence s, without the prefix."""
        n, a = self.kv_lens[s], self.q_lens[s]
        pos = n - a + torch.arange(a, device="cuda")[:, None]
        t = torch.arange(n, device="cuda")[None, :]
        vis = t <= pos
        if self.window:
            vis &= (t > pos - self.window) | (t < self.sinks)
        for j, b in enumerate(self.table_h[s]):
            if not 0 <= b < self.n_blocks:
                vis[:, j * self.B:(j + 1) * self.B] = False
        return vis

    def reference(self):
        """Per sequence: out, its allowed error, lse, its allowed error, weight sums and theirs (float64)."""
        res = []
        G = self.H // self.C
        for s, (a, n) in enumerate(zip(self.q_lens, self.kv_lens)):
            K, V, vis = self.K[s].double(), self.V[s].double(), self.visible(s)
            if self.prefix_lens:
                for g, (lo, hi) in enumerate(zip(self.groups, self.groups[1:])):
                    if lo <= s < hi:
                        K, V = torch.cat([self.PK[g].double(), K]), torch.cat([self.PV[g].double(), V])
                        vis = torch.cat([torch.ones((a, self.prefix_lens[g]), dtype=torch.bool, device="cuda"), vis], 1)
            Q = self.q[self.cu_h[s]:self.cu_h[s + 1]].double()
            out = torch.zeros((a, self.H, self.D), dtype=torch.float64, device="cuda")
            otol, lse = torch.zeros_like(out), torch.full((a, self.H), -math.inf, dtype=torch.float64, device="cuda")
            ltol = torch.zeros_like(lse)
            wsum = torch.zeros((self.C, K.shape[0]), dtype=torch.float64, device="cuda")
            wtol = torch.zeros_like(wsum)
            for h in range(self.H if K.shape[0] and a else 0):
                c = h // G
                k, v = K[:, c], V[:, c]
                x = (Q[:, h] @ torch.where(torch.isfinite(k), k, 0.0).T) * self.scale
                mag = (Q[:, h].abs() @ torch.where(torch.isfinite(k), k, 0.0).abs().T) * abs(self.scale)
                x = torch.where(vis, x, -math.inf)
                has = vis.any(1)
                m = torch.where(has, x.amax(1), 0.0)
                e = torch.exp(x - m[:, None])
                l = e.sum(1)
                p = torch.where(has[:, None], e / l.clamp_min(1e-300)[:, None], 0.0)
                nvis = vis.sum(1).double()
                dx = torch.where(vis, (self.D + 8) * 2.0 ** -24 * mag + 2.0 ** -22 * (x.abs() + m.abs()[:, None]), 0.0)
                dxm = dx.amax(1)
                rel = 2 * dxm + 2.0 ** -21 + nvis * 2.0 ** -24
                u = U[self.dtype]
                # what a query does not see contributes nothing, whatever it holds
                mix = torch.zeros((a, self.D), dtype=torch.float64, device="cuda")
                amix = torch.zeros_like(mix)
                vf = torch.where(torch.isfinite(v), v, 0.0)
                mix, amix = p @ vf, p @ vf.abs()
                bad = ~torch.isfinite(v)
                if bool(bad.any()):
                    for t in torch.nonzero(bad.any(1)).flatten().tolist():
                        mix = torch.where(vis[:, t:t + 1] & bad[t], math.nan, mix)
                out[:, h] = mix
                otol[:, h] = (amix * (rel + u + nvis * 2.0 ** -24)[:, None] + u * mix.abs().nan_to_num() + 1e-30
                              + (nvis * 2.0 ** -25)[:, None] * vf.abs().amax() * (self.dtype == torch.float16))
                lse[:, h] = torch.where(has, m + torch.log(l.clamp_min(1e-300)), -math.inf)
                ltol[:, h] = dxm + nvis * 2.0 ** -24 + 2.0 ** -20 + 2.0 ** -22 * m.abs()
                wsum[c] += p.sum(0)
                wtol[c] += (p * (2 * rel)[:, None]).sum(0)
            res.append((out, otol, lse, ltol, wsum, wtol))
        return res

    def check(self, ref=None):
        for s, (out, otol, lse, ltol, _, _) in enumerate(ref or self.reference()):
            got = self.out[self.cu_h[s]:self.cu_h[s + 1]].double()
            nan = torch.isnan(out)
            assert bool((~torch.isfinite(got) == nan).all()), f"sequence {s}: non-finite values differ"
            err = torch.where(nan, 0.0, (got - out).abs())
            over = err - torch.where(nan, 0.0, otol)
            assert not bool((over > 0).any()), f"sequence {s}: out off by {float(err.max())} (allowed there {float(otol.flatten()[over.argmax()])})"
            if self.lse is not None:
                gl = self.lse[self.cu_h[s]:self.cu_h[s + 1]].double()
                empty = lse == -math.inf
                assert bool((gl[empty] == -math.inf).all()) and bool((got[empty] == 0).all())
                assert not bool(((gl - lse).abs()[~empty] > ltol[~empty]).any()), f"sequence {s}: lse"
