"""gms_kv_evict against a sort: exact positions, weights, lengths and moved bytes."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2609_25451_b200 import gms  # noqa: E402


def expected_kept(w, budget, sinks, recent):
    n = len(w)
    if n <= budget:
        return list(range(n))
    mid = list(range(sinks, n - recent))
    order = sorted(mid, key=lambda t: (1, 0.0, t) if math.isnan(w[t]) else (0, -w[t], t))
    return sorted(list(range(sinks)) + order[:budget - sinks - recent] + list(range(n - recent, n)))


def run_evict(seed, *, layers=2, C=2, D=64, B=32, order="token", lens=(100, 7, 0, 333), budget=64, sinks=4, recent=9, max_len=None,
              make=None, with_out=True, layer_planes=2, planes=(0, 1), n_planes=None, w_pad=0, bad=False, gap=0, stream=None):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
    S = len(lens)
    max_len = max(lens) if max_len is None else max_len
    hs, ts = (D * 2, C * D * 2) if order == "token" else (B * D * 2, D * 2)
    bb = B * C * D * 2
    assert bb % 4096 == 0
    stride = bb + gap
    need = [(n + B - 1) // B for n in lens]
    dneed = [(min(n, budget) + B - 1) // B for n in lens]
    n_blocks = sum(need) + sum(dneed) + 2
    n_planes = n_planes or max(planes) + 1 + (layers - 1) * layer_planes
    raw = torch.randint(0, 256, (n_planes * n_blocks * stride,), dtype=torch.uint8, device="cuda", generator=g)
    before = raw.clone()
    ids = list(rng.permutation(n_blocks))
    src_h = [[int(ids.pop()) for _ in range(k)] for k in need]
    dst_h = [[int(ids.pop()) for _ in range(k)] for k in dneed]

    def table(rows):
        width = max([1] + [len(r) for r in rows])
        return torch.tensor([r + [-1] * (width - len(r)) for r in rows], dtype=torch.int32, device="cuda").view(S, width)

    if bad:
        src_h[3][1] = -4
        dst_h[0][1] = n_blocks
    w = torch.exp(torch.randn((layers, S, C, max_len + w_pad), device="cuda", generator=g) * 3)
    if make is not None:
        make(w)
    wo = torch.full((layers, S, C, max(budget, 1) + 5), -3.0, device="cuda")
    kept = torch.full((layers, S, C, budget), -99, dtype=torch.int32, device="cuda")
    lens_out = torch.full((S,), -1, dtype=torch.int32, device="cuda")
    desc = gms.KvPool(base=raw.data_ptr(), plane_stride=n_blocks * stride, block_stride=stride, n_planes=n_planes, n_blocks=n_blocks, block_bytes=bb)
    lay = gms.KvLayout(k_plane=planes[0], v_plane=planes[1], n_kv_heads=C, head_dim=D, block_tokens=B, dtype=gms.DTYPE_BF16,
                       token_stride=ts, head_stride=hs)
    args = gms.kv_evict_args(weights=w, weights_out=wo if with_out else None, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"),
                             lens_out=lens_out if with_out else None, src_table=table(src_h), dst_table=table(dst_h), kept=kept,
                             max_len=max_len, budget=budget, sinks=sinks, recent=recent, layer_planes=layer_planes)
    torch.cuda.synchronize()
    gms.gms_kv_evict(desc, lay, args, stream)
    torch.cuda.synchronize()
    want = before.view(n_planes, n_blocks, stride).cpu().numpy().copy()
    old = want.copy()
    wh, kh, woh = w.cpu().numpy(), kept.cpu().numpy(), wo.cpu().numpy()
    row = D * 2
    for l in range(layers):
        for s, n in enumerate(lens):
            n = min(n, max_len)
            for c in range(C):
                keep = expected_kept(wh[l, s, c, :n].tolist(), budget, sinks, recent)
                assert kh[l, s, c].tolist() == keep + [-1] * (budget - len(keep)), (l, s, c)
                if with_out:
                    assert np.array_equal(woh[l, s, c, :len(keep)].view(np.uint32), wh[l, s, c, keep].view(np.uint32) if keep else
                                          np.zeros(0, np.uint32))
                    assert (woh[l, s, c, len(keep):] == -3).all()
                for j, t in enumerate(keep):
                    a, b = src_h[s][t // B], dst_h[s][j // B]
                    if not 0 <= a < n_blocks or not 0 <= b < n_blocks:
                        continue
                    for p in planes:
                        f, to = t % B * ts + c * hs, j % B * ts + c * hs
                        want[p + l * layer_planes, b, to:to + row] = old[p + l * layer_planes, a, f:f + row]
    assert np.array_equal(raw.view(n_planes, n_blocks, stride).cpu().numpy(), want)
    if with_out:
        assert lens_out.tolist() == [min(n, budget) for n in lens]


@pytest.mark.parametrize("order,D,B,C", [("token", 64, 32, 2), ("head", 128, 16, 1), ("token", 128, 16, 8), ("head", 64, 1024, 1)])
@pytest.mark.parametrize("budget,sinks,recent", [(64, 4, 9), (13, 4, 9), (1, 0, 0), (50, 0, 50), (50, 50, 0), (332, 1, 1), (333, 0, 0), (1000, 3, 3)])
def test_kept_tokens(order, D, B, C, budget, sinks, recent):
    run_evict(1, order=order, D=D, B=B, C=C, budget=budget, sinks=sinks, recent=recent)


def ties(w):
    w.copy_((w * 2).round() / 2)
    w[..., ::3] = 0.0
    w[..., 1::7] = -0.0


def odd_values(w):
    w[..., ::5] = math.nan
    w[..., 1::5] = math.inf
    w[..., 2::5] = -math.inf
    w[..., 3::10] = -1.5
    w[..., 4::10] = 1e-42


def all_equal(w):
    w.fill_(0.25)


def all_nan(w):
    w.fill_(math.nan)


@pytest.mark.parametrize("make", [ties, odd_values, all_equal, all_nan])
@pytest.mark.parametrize("budget", [40, 101, 250])
def test_ties_and_odd_values(make, budget):
    run_evict(2, make=make, budget=budget, lens=(300, 299, 513, 41))


def test_nothing_else_is_touched():
    run_evict(3, with_out=False, gap=32)
    run_evict(4, bad=True)                       # ids outside the pool: those rows are not copied
    run_evict(5, planes=(2, 0), layer_planes=1, layers=2)   # planes 2,3 and 0,1
    run_evict(6, max_len=200, lens=(100, 200, 3, 150), w_pad=7)
    run_evict(7, lens=(0, 0), budget=5, sinks=0, recent=0, max_len=10)
    run_evict(8, lens=(10, 20), budget=0, sinks=0, recent=0)
    run_evict(9, stream=torch.cuda.Stream())


def test_long_rows():
    run_evict(10, layers=1, C=1, D=64, B=64, lens=(20011, 12345), budget=3001, sinks=4, recent=100)
    run_evict(11, layers=1, C=1, D=64, B=64, lens=(70001,), budget=65000, sinks=4, recent=100, make=ties)
