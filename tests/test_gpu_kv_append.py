"""gms_kv_append against the formulas in 64 bits.

How far a value may be off: x is exact in 32 bits; the mean of squares has D + 2 roundings, the reciprocal root, the weight's
sum and three products a few more: (D / 2 + 12) 2^-24 relative of the normed value; the angle is reduced in 64 bits and off by
at most 2^-24 of a half turn afterwards, cosine and sine by 2^-22 in all, the two products and their sum by 3 2^-24: together
(|a| + |b|) (D / 2 + 40) 2^-24; then one rounding, u = eps / 2 of the type (f16 below 2^-14: 2^-25 absolute).
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2609_25451_b200 import gms  # noqa: E402

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


class Append:
    def __init__(self, seed, *, rows=5, H=8, C=2, D=128, B=16, dtype=BF16, wdtype=None, order="token", rotary=None, pairs=gms.PAIR_HALVES, axes=1,
                 norm="qk", offset=0.0, eps=1e-6, rope_scale=1.0, live=None, far=5000, fused=True, what="qkv", bad_slots=(), gap=0, base=10000.0,
                 in_place=False, planes=(0, 1), head_major=False, scale=2.0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        rng = np.random.default_rng(seed)
        R = D if rotary is None else rotary
        self.__dict__.update(rows=rows, H=H, C=C, D=D, B=B, dtype=dtype, order=order, R=R, pairs=pairs, offset=offset, eps=eps, rope_scale=rope_scale,
                             live=rows if live is None else live, what=what, in_place=in_place, planes=planes)

        def rand(*shape):
            return torch.randn(shape, device="cuda", generator=g) * scale

        if fused:
            qkv = rand(rows, (H + 2 * C) * D).to(dtype)
            self.q, self.k, self.v = (x.view(rows, -1, D) for x in qkv.split([H * D, C * D, C * D], 1))
        else:  # heads outside rows, gaps
            self.q, self.k, self.v = (rand(n + 1, rows + 2, D + 8).to(dtype)[:n, 1:rows + 1, :D].transpose(0, 1) for n in (H, C, C))
        self.q0 = self.q.clone()
        self.out_full = torch.full((rows + 2, H + 1, D), 3.0, dtype=dtype, device="cuda")
        self.q_out = None if in_place else self.out_full[1:rows + 1, :H]
        n_blocks = (rows + B - 1) // B + 4
        if order == "token":
            hs, ts = D * 2 + gap, C * (D * 2 + gap)
        else:
            ts, hs = D * 2 + gap, B * (D * 2 + gap)
        used = (B - 1) * ts + (C - 1) * hs + D * 2
        bb = (used + 4095) // 4096 * 4096
        self.stride, self.hs, self.ts, self.n_blocks = bb + 64, hs, ts, n_blocks
        n_planes = max(planes) + 1
        self.raw = torch.randint(0, 256, (n_planes * n_blocks * self.stride,), dtype=torch.uint8, device="cuda", generator=g)
        self.plane_stride = n_blocks * self.stride
        slots = rng.permutation(n_blocks * B)[:rows].astype(np.int64)
        for i, x in bad_slots:
            slots[i] = x
        self.slots = torch.from_numpy(slots).cuda()
        self.positions = torch.from_numpy(rng.integers(0, far + 1, (axes, rows)).astype(np.int32)).cuda()
        self.freq = torch.tensor([base ** (-2.0 * j / max(R, 1)) for j in range(R // 2)], dtype=torch.float64).float().cuda() if R else None
        self.axis_h = rng.integers(0, axes + (2 if axes > 1 else 0), R // 2).astype(np.uint8) if axes > 1 else np.zeros(R // 2, np.uint8)
        self.axes = torch.from_numpy(self.axis_h).cuda() if axes > 1 and R else None
        wdtype = wdtype or dtype
        self.qw, self.kw = ((1.0 - offset + 0.3 * torch.randn(D, device="cuda", generator=g)).to(wdtype) if c in norm else None for c in "qk")
        self.n_rows = None if live is None else torch.tensor([live], dtype=torch.int32, device="cuda")
        self.desc = gms.KvPool(base=self.raw.data_ptr(), plane_stride=self.plane_stride, block_stride=self.stride, n_planes=n_planes,
                               n_blocks=n_blocks, block_bytes=bb)
        self.layout = gms.KvLayout(k_plane=planes[0], v_plane=planes[1], n_kv_heads=C, head_dim=D, block_tokens=B,
                                   dtype=gms.DTYPE_BF16 if dtype == BF16 else gms.DTYPE_F16, token_stride=ts, head_stride=hs)
        kv = "k" in what
        self.args = gms.kv_append_args(q=self.q if "q" in what else None, k=self.k if kv else None, v=self.v if kv else None,
                                       q_out=self.q_out if "q" in what else None, slots=self.slots if kv else None,
                                       positions=(self.positions if axes > 1 else self.positions[0]) if R else None, inv_freq=self.freq,
                                       axes=self.axes, n_rows=self.n_rows, q_weight=self.qw, k_weight=self.kw, pairs=pairs, weight_offset=offset,
                                       eps=eps, rope_scale=rope_scale)

    def view(self, raw, plane):
        return torch.as_strided(raw[plane * self.plane_stride:].view(self.dtype), (self.n_blocks, self.B, self.C, self.D),
                                (self.stride // 2, self.ts // 2, self.hs // 2, 1))

    def want(self, x, w):
        """Values in 64 bits and how far off they may be, for the rows that are there."""
        R, D = self.R, self.D
        y = x[:self.live].double()
        if w is not None:
            y = y * (((y * y).mean(-1, keepdim=True) + self.eps) ** -0.5) * (w.double() + self.offset)
        mag = y.abs()
        if R:
            n_axes = self.positions.shape[0]
            axis = torch.from_numpy(np.minimum(self.axis_h, n_axes - 1).astype(np.int64)).cuda()
            angle = self.positions[:, :self.live].double()[axis].T * self.freq.double()
            c, s = torch.cos(angle)[:, None] * self.rope_scale, torch.sin(angle)[:, None] * self.rope_scale
            i0 = torch.arange(R // 2, device="cuda") if self.pairs == gms.PAIR_HALVES else torch.arange(0, R, 2, device="cuda")
            i1 = i0 + R // 2 if self.pairs == gms.PAIR_HALVES else i0 + 1
            a, b = y[..., i0], y[..., i1]
            both = (a.abs() + b.abs()) * max(abs(self.rope_scale), 1.0)
            mag = mag.clone()
            mag[..., i0], mag[..., i1] = both, both
            y = y.clone()
            y[..., i0], y[..., i1] = a * c - b * s, b * c + a * s
        u = torch.finfo(self.dtype).eps / 2
        bound = u * y.abs() + mag * (D / 2 + 40) * 2.0 ** -24 * (1 + u) + (2.0 ** -25 if self.dtype == F16 else 0.0)
        return y, bound

    def check(self, stream=None):
        before = self.raw.clone()
        torch.cuda.synchronize()
        gms.gms_kv_append(self.desc, self.layout, self.args, stream)
        torch.cuda.synchronize()
        n = self.live
        if "q" in self.what:
            y, bound = self.want(self.q0, self.qw)
            got = (self.q if self.in_place else self.q_out)
            assert ((got[:n].double() - y).abs() <= bound).all()
            if self.in_place:
                assert torch.equal(got[n:], self.q0[n:])
            else:
                assert (self.out_full[0] == 3).all() and (self.out_full[n + 1:] == 3).all() and (self.out_full[:, self.H:] == 3).all()
        else:
            assert (self.out_full == 3).all()
        after = before.clone()
        if "k" in self.what and n:
            slot = self.slots[:n]
            ok = (slot >= 0) & (slot < self.n_blocks * self.B)
            blk, tok = slot[ok] // self.B, slot[ok] % self.B
            y, bound = self.want(self.k, self.kw)
            got = self.view(self.raw, self.planes[0])[blk, tok]
            assert ((got.double() - y[ok]).abs() <= bound[ok]).all()
            self.view(after, self.planes[0])[blk, tok] = got
            self.view(after, self.planes[1])[blk, tok] = self.v[:n][ok]
        assert torch.equal(self.raw, after)  # values exact, everything else as it was


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("pairs", [gms.PAIR_HALVES, gms.PAIR_NEIGHBOURS])
@pytest.mark.parametrize("rotary", [0, 8, 24, 64, None])
def test_types_and_rotations(dtype, D, pairs, rotary):
    Append(1, dtype=dtype, D=D, pairs=pairs, rotary=rotary, rows=37).check()


@pytest.mark.parametrize("rows", [1, 2, 3, 16, 63, 257, 1000])
@pytest.mark.parametrize("H,C", [(1, 1), (8, 1), (32, 8), (5, 5), (7, 7), (20, 4)])
def test_rows_and_heads(rows, H, C):
    Append(rows + H, rows=rows, H=H, C=C, D=64, B=32 if C < 8 else 16).check()


@pytest.mark.parametrize("wdtype", [BF16, F16, F32])
@pytest.mark.parametrize("norm", ["", "q", "k", "qk"])
def test_weights(wdtype, norm):
    Append(3, wdtype=wdtype, norm=norm, offset=1.0, rows=20).check()
    Append(4, wdtype=wdtype, norm=norm, offset=0.0, rows=20, D=64, eps=0.5).check()


@pytest.mark.parametrize("kw", [dict(order="head", B=32), dict(order="head", gap=16), dict(gap=32), dict(fused=False), dict(in_place=True),
                                dict(in_place=True, fused=False), dict(planes=(3, 1)), dict(B=1024, C=1, H=4, D=64), dict(rope_scale=1.3),
                                dict(rope_scale=-0.5)])
def test_layouts_and_strides(kw):
    Append(7, rows=45, **kw).check()


@pytest.mark.parametrize("axes", [2, 3, 8])
@pytest.mark.parametrize("pairs", [gms.PAIR_HALVES, gms.PAIR_NEIGHBOURS])
def test_axes(axes, pairs):
    Append(9, rows=33, axes=axes, pairs=pairs, rotary=96).check()


@pytest.mark.parametrize("far", [100, 10**6, 2**31 - 2])
def test_far_positions(far):
    Append(11, rows=300, far=far, base=1e6, norm="").check()


def test_negative_positions():
    a = Append(12, rows=40)
    a.positions.neg_()
    a.check()


@pytest.mark.parametrize("what", ["q", "kv"])
def test_queries_or_keys_alone(what):
    Append(13, rows=21, what=what).check()


@pytest.mark.parametrize("live", [0, 1, 20, 40, 99])
def test_rows_that_are_not_there(live):
    a = Append(14, rows=40, live=live)
    a.live = min(live, 40)
    a.check()


def test_slots_outside_the_pool():
    Append(15, rows=30, bad_slots=[(0, -1), (3, -2**62), (5, 10**9), (8, 2**62), (29, -1)]).check()


def test_negative_number_of_rows():
    a = Append(16, rows=4, live=0)
    a.n_rows.fill_(-3)
    a.check()


def test_nothing_to_do():
    a = Append(17, rows=3)
    a.args.rows = 0
    a.live = 0
    gms.gms_kv_append(a.desc, a.layout, a.args)
    torch.cuda.synchronize()
    assert (a.out_full == 3).all()


def test_values_that_are_not_finite_stay_in_their_rows():
    a = Append(18, rows=12, H=4, C=2)
    clean = Append(18, rows=12, H=4, C=2)
    a.q[3, 1, 7], a.k[5, 0, 0], a.v[6, 1, 2] = float("nan"), float("inf"), float("nan")
    for x in (a, clean):
        gms.gms_kv_append(x.desc, x.layout, x.args)
    torch.cuda.synchronize()
    assert torch.isnan(a.q_out[3, 1]).any()
    a.q_out[3, 1] = clean.q_out[3, 1]
    assert torch.equal(a.q_out, clean.q_out)
    for i, (row, head) in enumerate(((5, 0), (6, 1))):
        blk, tok = int(a.slots[row]) // a.B, int(a.slots[row]) % a.B
        assert not torch.isfinite(a.view(a.raw, i)[blk, tok, head].float()).all()
        a.view(a.raw, i)[blk, tok, head] = clean.view(clean.raw, i)[blk, tok, head]
    assert torch.equal(a.raw, clean.raw)


def test_zero_rows_have_no_norm_to_divide_by():
    a = Append(19, rows=8)
    a.q.zero_()
    a.q0.zero_()
    a.k.zero_()
    a.check()


def test_other_stream_and_graph():
    a = Append(20, rows=50)
    s = torch.cuda.Stream()
    a.check(s)
    b = Append(21, rows=50)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        gms.gms_kv_append(b.desc, b.layout, b.args)
    for seed in (1, 2):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        for x in (b.q, b.k, b.v):
            x.copy_(torch.randn(x.shape, device="cuda", generator=g))
        b.q0 = b.q.clone()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        y, bound = b.want(b.q0, b.qw)
        assert ((b.q_out.double() - y).abs() <= bound).all()
        y, bound = b.want(b.k, b.kw)
        assert ((b.view(b.raw, 0)[b.slots // b.B, b.slots % b.B].double() - y).abs() <= bound).all()
        assert torch.equal(b.view(b.raw, 1)[b.slots // b.B, b.slots % b.B], b.v)


def test_pool_beyond_32_bits():
    """A block more than 4 GiB into a plane, the values' plane behind it."""
    D, C, B = 128, 8, 16
    bb = B * C * D * 2
    n_blocks = (5 << 30) // bb
    raw = torch.zeros(2 * n_blocks * bb // 2, dtype=BF16, device="cuda")
    desc = gms.KvPool(base=raw.data_ptr(), plane_stride=n_blocks * bb, block_stride=bb, n_planes=2, n_blocks=n_blocks, block_bytes=bb)
    lay = gms.KvLayout(k_plane=0, v_plane=1, n_kv_heads=C, head_dim=D, block_tokens=B, dtype=gms.DTYPE_BF16, token_stride=C * D * 2, head_stride=D * 2)
    k, v = (torch.randn(3, C, D, device="cuda").to(BF16) for _ in range(2))
    slots = torch.tensor([n_blocks * B - 1, 7, (n_blocks - 1) * B], dtype=torch.int64, device="cuda")
    gms.gms_kv_append(desc, lay, gms.kv_append_args(k=k, v=v, slots=slots))
    torch.cuda.synchronize()
    pool = raw.view(2, n_blocks * B, C, D)
    assert torch.equal(pool[0, slots], k) and torch.equal(pool[1, slots], v)
    pool[:, slots] = 0
    assert not raw.any()
