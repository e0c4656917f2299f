"""gms_kv_evict over tables with holes: a kept token whose rows cannot be copied is reported, others are not."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2609_25451_b200 import gms  # noqa: E402


@pytest.mark.parametrize("src_hole,dst_hole,told", [(None, None, False), (-1, None, True), (40, None, True), (None, 2**31 - 1, True), ("unkept", None, False)])
def test_status(src_hole, dst_hole, told):
    C, D, B, n, budget = 2, 128, 16, 200, 40
    pool = torch.randint(-30000, 30000, (2, 32, B, C, D), dtype=torch.int16, device="cuda")
    start = pool.clone()
    w = torch.ones((1, 1, C, n), device="cuda")
    w[..., 64:80] = 0.0                                     # block 4 is never chosen
    w[..., 16:32] = 2.0                                     # block 1 always is
    src = list(range(13))
    dst = [20, 21, 22]
    if src_hole == "unkept":
        src[4] = -1
    elif src_hole is not None:
        src[1] = src_hole
    if dst_hole is not None:
        dst[2] = dst_hole
    desc = gms.KvPool(base=pool.data_ptr(), plane_stride=pool.stride(0) * 2, block_stride=pool.stride(1) * 2, n_planes=2, n_blocks=32,
                      block_bytes=B * C * D * 2)
    lay = gms.KvLayout(k_plane=0, v_plane=1, n_kv_heads=C, head_dim=D, block_tokens=B, dtype=gms.DTYPE_BF16, token_stride=C * D * 2, head_stride=D * 2)
    kept = torch.empty((1, 1, C, budget), dtype=torch.int32, device="cuda")
    status = torch.full((1,), 8, dtype=torch.int64, device="cuda")
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    args = gms.kv_evict_args(weights=w, lens=ints([n]), src_table=ints([src]), dst_table=ints([dst]), kept=kept, max_len=n, budget=budget, sinks=4,
                             recent=4, status=status)
    gms.gms_kv_evict(desc, lay, args)
    torch.cuda.synchronize()
    assert int(status.item()) == 8 | (gms.DEV_HOLE if told else 0)
    want = list(range(4)) + list(range(4, 20)) + list(range(20, 32)) + [32, 33, 34, 35] + list(range(196, 200))
    assert kept[0, 0, 0].tolist() == want == kept[0, 0, 1].tolist()
    for j, t in enumerate(want):
        a, b = src[t // B], dst[j // B]
        if 0 <= a < 32 and 0 <= b < 32:
            assert torch.equal(pool[:, b, j % B], start[:, a, t % B])
        elif 0 <= b < 32:
            assert torch.equal(pool[:, b, j % B], start[:, b, j % B])
