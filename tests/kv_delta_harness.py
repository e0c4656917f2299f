"""Problems and the 64-bit reference of gms_kv_delta.

The reference goes row by row, in float64, all heads of a sequence at once.  How far a result may be off (Frobenius norms over
a head, m the largest norm that the state and the terms that make it up reach):

  states: a row of the row-by-row kernel makes D + 16 roundings of 2^-24 relative of at most m; with keys of length at most 1,
          strengths at most 2 and gates at most 1 an error that is there does not grow (|I - b k k^T| <= 1), so errors add up:
          rows (D + 16) 2^-24 m.  A chunk of 64 tokens takes its products in two 16-bit terms (2^-16 relative each, five of them on
          the way into a state, and its decays in 32 bits): 8 2^-16 m more a chunk, times the norm of the inverse of I + A,
          which stands for the same recursion and does not grow either, but whose columns add up: sqrt(64).
  out:    an element is scale times a product of a row of length |q| with a column of the state: scale |q| (that column's error),
          and where a term enters as one 16-bit number, 2 u scale |q| (m_v + sum_j |d_jv| |k_j|), m_v the column's norm; the last
          rounding u |out| (f16: and 2^-25).
"""
from __future__ import annotations

import math

import numpy as np
import torch

from paper_2609_25451_b200 import gms

BF16, F16 = torch.bfloat16, torch.float16
U = {BF16: 2.0 ** -8, F16: 2.0 ** -11}


class Delta:
    def __init__(self, seed, *, lens=(5,), H=4, K=2, D=128, dtype=BF16, per=2, unit=True, fresh=(), gates=True, betas=True, in_place=False, fused=True,
                 plane=0, pad_rows=0, scale=None, decay=1.0, decode=False, beta_scale=1.0, same_source=False, max_q=None, gap=0, key_noise=1.0,
                 state_scale=0.3):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.__dict__.update(lens=list(lens), H=H, K=K, D=D, dtype=dtype, unit=unit, in_place=in_place, per=per, eps=1e-6, plane=plane)
        S, T = len(lens), sum(lens)
        self.S, self.T = S, T
        self.max_q = max([1] + list(lens)) if max_q is None else max_q
        self.max_q = min(self.max_q, T + pad_rows)

        def rand(*shape):
            return torch.randn(shape, device="cuda", generator=g)

        rows = T + pad_rows
        common = rand(1, K, D)

        def keyed(x):  # key_noise below 1: keys that are nearly alike
            return common + key_noise * x if key_noise < 1 else x

        q, k, v = rand(rows, K, D), keyed(rand(rows, K, D)), rand(rows, H, D)
        if not unit:
            q, k = q / q.norm(dim=-1, keepdim=True), k / k.norm(dim=-1, keepdim=True) * 0.99
        if fused:
            qkv = torch.cat([x.reshape(rows, -1) for x in (q, k, v)], 1).to(dtype)
            self.q, self.k, self.v = (x.view(rows, -1, D) for x in qkv.split([K * D, K * D, H * D], 1))
        else:
            def spread(x):
                y = torch.full((x.shape[1] + 1, rows + 2, D + 8), 9.0, dtype=dtype, device="cuda")
                y[:x.shape[1], 1:rows + 1, :D] = x.transpose(0, 1).to(dtype)
                return y[:x.shape[1], 1:rows + 1, :D].transpose(0, 1)
            self.q, self.k, self.v = spread(q), spread(k), spread(v)
        wide = torch.full((rows, H + 3), 50.0, device="cuda")
        wide[:, :H] = -decay * torch.rand((H,), device="cuda", generator=g) * torch.nn.functional.softplus(rand(rows, H) - 1)
        self.g = wide[:, :H] if gates else None
        self.beta = beta_scale * torch.sigmoid(rand(rows, H)) if betas else None
        self.out_full = torch.full((rows + 2, H + 1, D), 3.0, dtype=dtype, device="cuda")
        self.out = self.out_full[1:rows + 1, :H]
        self.cu_h = [0] + np.cumsum(lens).tolist()
        self.cu = None if decode else torch.tensor(self.cu_h, dtype=torch.int32, device="cuda")
        n = (H + per - 1) // per
        self.n = n
        self.block_bytes = per * D * D * 4
        self.stride = self.block_bytes + gap
        self.n_blocks = 2 * S * n + 3
        self.raw = rand((plane + 1) * self.n_blocks * self.stride // 4) * state_scale
        self.plane_stride = self.n_blocks * self.stride
        ids = rng.permutation(self.n_blocks)
        self.src_h = ids[:S * n].reshape(S, n).copy()
        if same_source:
            self.src_h[:] = self.src_h[:1]
        self.dst_h = self.src_h.copy() if in_place else ids[S * n:2 * S * n].reshape(S, n).copy()
        self.fresh = [s in fresh for s in range(S)]
        self.past = torch.tensor([0 if f else 7 for f in self.fresh], dtype=torch.int32, device="cuda") if fresh else None
        self.status = torch.zeros(1, dtype=torch.int64, device="cuda")
        self.scale = 1.0 / math.sqrt(D) if scale is None else scale
        self.desc = gms.KvPool(base=self.raw.data_ptr(), plane_stride=self.plane_stride, block_stride=self.stride, n_planes=plane + 1,
                               n_blocks=self.n_blocks, block_bytes=self.block_bytes)
        self.state = gms.KvState(plane=plane, n_heads=H, head_dim=D)
        self.make()

    def make(self):
        self.src = torch.from_numpy(self.src_h.astype(np.int32)).cuda()
        self.dst = self.src if self.in_place else torch.from_numpy(self.dst_h.astype(np.int32)).cuda()
        self.args = gms.kv_delta_args(q=self.q, k=self.k, v=self.v, out=self.out, g=self.g, beta=self.beta, cu_q=self.cu, max_q=self.max_q,
                                      past_lens=self.past, src_table=self.src, dst_table=self.dst, scale=self.scale,
                                      unit_eps=self.eps if self.unit else None, status=self.status)
        need = gms.gms_kv_delta_workspace(self.desc, self.state, self.args)
        self.ws = torch.full((max(need, 256),), 0xFF, dtype=torch.uint8, device="cuda")  # its bits before the call must not matter
        self.args.set_workspace(self.ws)

    def run(self, stream=None):
        torch.cuda.synchronize()
        gms.gms_kv_delta(self.desc, self.state, self.args, stream)
        torch.cuda.synchronize()

    def place(self, raw, table, s, h):
        """The [D, D] view of a head's state, or None in a hole."""
        i = int(table[s][h // self.per])
        if not 0 <= i < self.n_blocks:
            return None
        at = (self.plane * self.plane_stride + i * self.stride) // 4 + h % self.per * self.D * self.D
        return raw[at:at + self.D * self.D].view(self.D, self.D)

    def reference(self, raw):
        """Per sequence: rows processed, outputs [rows, H, D], state [H, D, D], bounds of both; from the pool as it was."""
        H, K, D = self.H, self.K, self.D
        res = []
        for s, n in enumerate(self.lens):
            n = min(n, self.max_q)
            r = slice(self.cu_h[s], self.cu_h[s] + n)
            q, k = (x[r].double().repeat_interleave(H // K, 1) for x in (self.q, self.k))
            if self.unit:
                q, k = (x / ((x * x).sum(-1, keepdim=True) + self.eps).sqrt() for x in (q, k))
            v = self.v[r].double()
            g = self.g[r].double() if self.g is not None else torch.zeros(n, H, dtype=torch.float64, device="cuda")
            b = self.beta[r].double() if self.beta is not None else torch.ones(n, H, dtype=torch.float64, device="cuda")
            S = torch.zeros(H, D, D, dtype=torch.float64, device="cuda")
            for h in range(H):
                x = None if self.fresh[s] else self.place(raw, self.src_h, s, h)
                if x is not None:
                    S[h] = x.double()
            out = torch.zeros(n, H, D, dtype=torch.float64, device="cuda")
            top = S.flatten(1).norm(dim=1)               # largest norm of a head's state and of what goes into it
            col = S.norm(dim=1)                          # the same of its columns
            rough = torch.zeros(n, H, D, dtype=torch.float64, device="cuda")
            spent = torch.zeros(H, D, dtype=torch.float64, device="cuda")
            chunk = 64
            for t in range(n):
                if t % chunk == 0:
                    start, spent = S.norm(dim=1), torch.zeros_like(spent)
                S = S * g[t].exp()[:, None, None]
                d = b[t][:, None] * (v[t] - (k[t][:, :, None] * S).sum(1))
                S = S + k[t][:, :, None] * d[:, None, :]
                out[t] = self.scale * (q[t][:, :, None] * S).sum(1)
                spent = spent + d.abs() * k[t].norm(dim=-1)[:, None]
                rough[t] = abs(self.scale) * q[t].norm(dim=-1)[:, None] * (start + spent)
                top = torch.maximum(top, torch.maximum(S.flatten(1).norm(dim=1), spent.norm(dim=1) + v[t].norm(dim=1) * b[t].abs()))
                col = torch.maximum(col, torch.maximum(S.norm(dim=1), spent))
            chunks = (n + chunk - 1) // chunk if n > 1 else 0
            e = n * (D + 16) * 2.0 ** -24 + chunks * 64 * 2.0 ** -16
            u = U[self.dtype]
            qn = q.norm(dim=-1)[:, :, None] if n else torch.zeros(0, H, 1, device="cuda")
            bound = u * out.abs() + 2 * u * rough * (n > 1) + abs(self.scale) * qn * e * top[None, :, None] + (2.0 ** -25 if self.dtype == F16 else 0)
            res.append((n, out, S, bound, e * top))
        return res

    def check(self, stream=None, run=True):
        before = self.raw.clone()
        if run:
            self.run(stream)
        ref = self.reference(before)
        after = before.clone()
        out_after = torch.full_like(self.out_full, 3.0)
        holes = False
        for s, (n, out, S, bound, e) in enumerate(ref):
            r = slice(self.cu_h[s], self.cu_h[s] + n)
            got = self.out[r]
            assert torch.isfinite(got.float()).all()
            assert ((got.double() - out).abs() <= bound).all(), (s, ((got.double() - out).abs() / bound).max())
            out_after[1 + r.start:1 + r.stop, :self.H] = got
            for h in range(self.H):
                holes |= not self.fresh[s] and self.place(self.raw, self.src_h, s, h) is None
                x = self.place(self.raw, self.dst_h, s, h)
                if x is None:
                    holes = True
                    continue
                err = (x.double() - S[h]).norm()
                assert err <= e[h], (s, h, float(err), float(e[h]))
                self.place(after, self.dst_h, s, h).copy_(x)
        assert torch.equal(after, self.raw)            # nothing but these states was written
        assert torch.equal(out_after, self.out_full)
        assert int(self.status) == (gms.DEV_HOLE if holes else 0)
