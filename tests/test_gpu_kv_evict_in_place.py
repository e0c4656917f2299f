"""gms_kv_evict with the lengths updated in place (lens_out = lens), with far more rows than the GPU holds at once."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2609_25451_b200 import gms  # noqa: E402


@pytest.mark.parametrize("layers,lens,budget,sinks,recent", [(32, (700, 300, 64, 1000, 65), 64, 4, 9), (48, (2000, 1999, 11, 500), 300, 0, 300),
                                                            (4, (12000, 9000), 100, 1, 1), (40, (90, 33, 10, 0), 0, 0, 0)])
def test_lengths_in_place(layers, lens, budget, sinks, recent):
    C, D, B = 8, 64, 16
    S, n_max = len(lens), max(lens)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    need, dneed = [(n + B - 1) // B for n in lens], [(min(n, budget) + B - 1) // B for n in lens]
    n_blocks = sum(need) + sum(dneed) + 1
    ids = list(np.random.default_rng(1).permutation(n_blocks))

    def table(counts):
        rows = [[int(ids.pop()) for _ in range(k)] for k in counts]
        width = max([1] + counts)
        return rows, torch.tensor([r + [-1] * (width - len(r)) for r in rows], dtype=torch.int32, device="cuda")

    src_h, src = table(need)
    dst_h, dst = table(dneed)
    pool = torch.randint(-30000, 30000, (2 * layers, n_blocks, B, C, D), dtype=torch.int16, device="cuda", generator=g)
    start = pool.clone()
    w = torch.rand((layers, S, C, n_max), device="cuda", generator=g)
    desc = gms.KvPool(base=pool.data_ptr(), plane_stride=pool.stride(0) * 2, block_stride=pool.stride(1) * 2, n_planes=2 * layers, n_blocks=n_blocks,
                      block_bytes=B * C * D * 2)
    lay = gms.KvLayout(k_plane=0, v_plane=1, n_kv_heads=C, head_dim=D, block_tokens=B, dtype=gms.DTYPE_BF16, token_stride=C * D * 2, head_stride=D * 2)
    for _ in range(3):
        pool.copy_(start)
        kept = torch.full((layers, S, C, budget), -9, dtype=torch.int32, device="cuda")
        length = torch.tensor(lens, dtype=torch.int32, device="cuda")
        gms.gms_kv_evict(desc, lay, gms.kv_evict_args(weights=w, lens=length, lens_out=length, src_table=src, dst_table=dst, kept=kept, max_len=n_max,
                                                      budget=budget, sinks=sinks, recent=recent))
        torch.cuda.synchronize()
        assert length.tolist() == [min(n, budget) for n in lens]
        for s, n in enumerate(lens):
            k = min(n, budget)
            if k == n:
                want = torch.arange(n, device="cuda").expand(layers, C, n)
            else:
                key = w[:, s, :, :n].clone()
                key[..., :sinks] = key[..., n - recent:] = 2.0
                want = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :k].sort(-1).values
            assert torch.equal(kept[:, s, :, :k].long(), want) and bool((kept[:, s, :, k:] == -1).all())
            if k == 0:
                continue
            a = torch.tensor(src_h[s], device="cuda")[want // B]
            j = torch.arange(k, device="cuda")
            b = torch.tensor(dst_h[s], device="cuda")[j // B].expand_as(want)
            h = torch.arange(C, device="cuda")[None, :, None].expand_as(want)
            for plane in (0, 1):
                p = (2 * torch.arange(layers, device="cuda") + plane)[:, None, None].expand_as(want)
                assert torch.equal(pool[p, b, (j % B).expand_as(want), h], start[p, a, want % B, h])
