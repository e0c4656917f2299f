"""gms_kv_attention and gms_kv_attention_shared against a 64-bit reference, at the lengths, masks, layouts and bit
patterns where they can go wrong.  Tolerances are derived in kv_attn_harness."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2609_25451_b200 import gms  # noqa: E402

if torch.cuda.is_available():
    from kv_attn_harness import Problem  # noqa: E402

BF, HF = "bf16", "f16"


def dt(name):
    return torch.bfloat16 if name == BF else torch.float16


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("heads,kv_heads,dim,block,order", [
    (8, 2, 128, 16, "token"), (8, 1, 128, 16, "head"), (4, 4, 64, 32, "head"), (6, 2, 64, 64, "token"), (3, 1, 64, 1024, "token"),
    (32, 8, 128, 16, "token"), (16, 1, 64, 128, "token"), (40, 2, 128, 32, "head"), (5, 5, 64, 16, "token"), (17, 1, 128, 16, "token"),
    (64, 1, 64, 32, "token"), (130, 1, 128, 16, "token")])
def test_one_query_a_sequence(dtype, heads, kv_heads, dim, block, order):
    lens = [1, 2, 15, 16, 17, 0, 31, 127, 128, 129, 300, 1025]
    p = Problem(1, dtype=dt(dtype), heads=heads, kv_heads=kv_heads, dim=dim, block=block, order=order, q_lens=[1] * len(lens),
                kv_lens=lens, decode=True)
    p.run()
    p.check()


@pytest.mark.parametrize("dim,dtype", [(64, BF), (128, HF)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (5, 1), (16, 16), (64, 4), (100, 0), (1000, 20), (2**32 - 1, 2**32 - 1)])
@pytest.mark.parametrize("q", [1, 3, 70])
def test_window_and_sinks(dim, dtype, window, sinks, q):
    lens = [q, q + 1, 33 + q, 200 + q, 517 + q]
    p = Problem(2, dtype=dt(dtype), heads=4, kv_heads=2, dim=dim, block=32, q_lens=[q] * len(lens), kv_lens=lens, window=window, sinks=sinks)
    p.run()
    p.check()


@pytest.mark.parametrize("dtype,dim,heads,kv_heads", [(BF, 128, 8, 2), (HF, 64, 8, 8), (BF, 64, 12, 4), (HF, 128, 32, 1)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 2)])
def test_ragged_queries(dtype, dim, heads, kv_heads, window, sinks):
    kv = [0, 5, 300, 64, 1, 700, 128, 129, 333]
    q = [0, 5, 1, 17, 1, 200, 128, 0, 65]
    p = Problem(3, dtype=dt(dtype), heads=heads, kv_heads=kv_heads, dim=dim, block=32, q_lens=q, kv_lens=kv, window=window, sinks=sinks,
                q_pad=3, pad_block=64, plane_gap=4096)
    p.run()
    p.check()


def test_more_queries_than_tokens_leave_rows_empty():
    p = Problem(4, q_lens=[7, 3, 2], kv_lens=[4, 0, 2], heads=4, kv_heads=2)
    p.run()
    p.check()
    assert bool((p.lse[:3] == -math.inf).all()) and bool((p.out[:3] == 0).all())


@pytest.mark.parametrize("q", [1, 2, 40])
def test_holes_in_the_table(q):
    p = Problem(5, q_lens=[q, q, q], kv_lens=[100, 260, 48], heads=8, kv_heads=2,
                holes=[(0, 0, -1), (0, 3, 2**31 - 1), (1, 7, -2**31), (1, 8, 10**6), (1, 16, -1), (2, 0, -1), (2, 1, -1), (2, 2, -1)])
    p.run()
    p.check()


@pytest.mark.parametrize("q", [1, 4, 150])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_what_is_not_seen_cannot_reach_the_output(q, dtype):
    """NaN and infinities in every place that no query sees, and at tokens that only later queries see."""
    def poison(p):
        for s, n in enumerate(p.kv_lens):
            none = ~p.visible(s).any(0)
            vals = torch.tensor([math.nan, math.inf, -math.inf], dtype=p.dtype, device="cuda")
            for x in (p.K[s], p.V[s]):
                x[none] = vals[torch.arange(int(none.sum()), device="cuda") % 3][:, None, None]
        p.V[1][-1, :, 5] = math.inf      # the newest token: seen by the last query alone
        p.V[2][-1] = math.nan

    p = Problem(6, dtype=dt(dtype), heads=8, kv_heads=2, q_lens=[q] * 3, kv_lens=[q + 400, q + 333, q + 90], window=50, sinks=3, poison=poison)
    p.run()
    p.check()


def test_large_logits_and_a_growing_maximum():
    def poison(p):
        p.K[0] *= torch.linspace(0.1, 12, p.kv_lens[0], device="cuda")[:, None, None].to(p.dtype)
        p.K[1] *= torch.linspace(12, 0.1, p.kv_lens[1], device="cuda")[:, None, None].to(p.dtype)

    for q in (1, 130):
        p = Problem(7, heads=4, kv_heads=2, q_lens=[q, q], kv_lens=[600, 601], poison=poison, q_scale=4.0)
        p.run()
        p.check()


def test_infinite_logits():
    """A key that gives +infinity makes NaN of the queries that see it (as the formula does), -infinity counts nothing."""
    p = Problem(8, heads=4, kv_heads=1, q_lens=[2], kv_lens=[50], dim=64, block=32)
    p.q[:, :, 0] = 1.0
    p.K[0][10, :, 0] = -math.inf
    p.store(p.kp, p.table_h[0], p.K[0])
    p.run()
    assert bool(torch.isfinite(p.out).all())
    keep = [t for t in range(50) if t != 10]
    x = (p.q[1, 0].double() @ p.K[0][keep, 0].double().T) * p.scale
    assert abs(float(p.lse[1, 0]) - float(torch.logsumexp(x, 0))) < 1e-4
    p.K[0][49, :, 0] = math.inf
    p.store(p.kp, p.table_h[0], p.K[0])
    p.run()
    assert bool(torch.isfinite(p.out[0]).all()) and not bool(torch.isfinite(p.out[1]).any())


def test_strides_planes_and_no_lse():
    for order in ("token", "head"):
        p = Problem(9, order=order, heads=8, kv_heads=2, dim=64, block=32, head_gap=48, pad_block=16, plane_gap=16, planes=(3, 1),
                    q_lens=[1, 1, 30], kv_lens=[77, 400, 90], q_pad=5, lse=False, max_extra=100, table_pad=50)
        p.run()
        p.check()


def test_on_another_stream_and_in_a_graph():
    p = Problem(10, q_lens=[1, 1], kv_lens=[500, 33], decode=True)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    p.run(stream=st)
    p.check()
    want = p.out.clone()
    p.out.fill_(0)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            gms.gms_kv_attention(p.desc, p.layout, p.attn)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(p.out, want)


@pytest.mark.parametrize("q_lens", [(1, 1, 1, 1), (3, 1, 90, 7)])
def test_equal_calls_give_equal_bits(q_lens):
    p = Problem(11, q_lens=q_lens, kv_lens=(9000, 300, 4000, 77), heads=8, kv_heads=2)
    w = torch.zeros((4, 2, 9000), device="cuda")
    p.run(gms.kv_weights(None, w))
    a, b, c = p.out.clone(), p.lse.clone(), w.clone()
    for _ in range(3):
        p.run(gms.kv_weights(None, w))
        assert torch.equal(a, p.out) and torch.equal(b, p.lse) and torch.equal(c, w)


@pytest.mark.parametrize("dtype,dim,heads,kv_heads", [(BF, 128, 8, 2), (HF, 64, 16, 4), (HF, 128, 20, 1)])
@pytest.mark.parametrize("q_lens,window,sinks,lse", [((1, 1, 1, 1), 0, 0, True), ((1, 1, 1, 1), 40, 2, False), ((4, 0, 3, 1), 0, 0, False),
                                                     ((33, 1, 70, 2), 0, 0, True), ((33, 1, 70, 2), 25, 3, False)])
def test_accumulated_weights(dtype, dim, heads, kv_heads, q_lens, window, sinks, lse):
    kv = (300, 7, 129, 2)
    p = Problem(12, dtype=dt(dtype), dim=dim, heads=heads, kv_heads=kv_heads, block=32, q_lens=q_lens, kv_lens=kv, window=window, sinks=sinks,
                lse=lse, holes=[(0, 2, -1)])
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    w_in = torch.rand((4, kv_heads, 310), device="cuda", generator=g)
    w_out = torch.full_like(w_in, -5.0)
    p.run(gms.kv_weights(w_in, w_out, decay=0.75))
    ref = p.reference()
    p.check(ref)
    for s, n in enumerate(kv):
        want = 0.75 * w_in[s, :, :n].double() + ref[s][4]
        tol = ref[s][5] + 2.0 ** -23 * (q_lens[s] * heads + 2) * want
        assert not bool(((w_out[s, :, :n].double() - want).abs() > tol).any())
        assert bool((w_out[s, :, n:] == -5).all())
    # in place, and from nothing
    both = w_in.clone()
    p.run(gms.kv_weights(both, both, decay=0.75))
    for s, n in enumerate(kv):
        assert torch.equal(both[s, :, :n], w_out[s, :, :n]) and torch.equal(both[s, :, n:], w_in[s, :, n:])
    p.run(gms.kv_weights(None, both))
    assert not bool(((both[0, :, :300].double() - ref[0][4]).abs() > ref[0][5] + 1e-6 * ref[0][4]).any())


@pytest.mark.parametrize("dtype,dim,heads,kv_heads,block,order", [(BF, 128, 8, 1, 16, "token"), (HF, 64, 16, 4, 32, "head"), (BF, 128, 32, 8, 16, "token")])
@pytest.mark.parametrize("q_lens,kv_lens,prefix,groups", [
    ((1, 1, 1), (1, 40, 17), (129,), (0, 3)), ((1,) * 9, (5, 1, 0, 77, 200, 16, 3, 2, 1), (300, 0, 1000), (0, 3, 4, 9)),
    ((2, 1, 3, 0, 1, 40), (2, 9, 300, 4, 1, 41), (64, 513), (0, 5, 6)), ((1,) * 40, tuple(range(40)), (700,), (0, 40)),
    ((1, 1, 1, 1), (9, 9, 9, 9), (33, 55), (0, 0, 4))])
def test_shared_prefix(dtype, dim, heads, kv_heads, block, order, q_lens, kv_lens, prefix, groups):
    p = Problem(13, dtype=dt(dtype), dim=dim, heads=heads, kv_heads=kv_heads, block=block, order=order, q_lens=q_lens, kv_lens=kv_lens,
                prefix_lens=prefix, groups=list(groups))
    p.run(prefix=p.make_prefix())
    p.check()


def test_shared_equals_the_same_tokens_unshared():
    p = Problem(14, heads=8, kv_heads=2, q_lens=(1,) * 20, kv_lens=tuple(range(1, 21)), prefix_lens=(257,), groups=[0, 20])
    p.run(prefix=p.make_prefix())
    p.check()
    # a group of one whose "prefix" is empty is plain attention
    q = Problem(14, heads=8, kv_heads=2, q_lens=(1,) * 20, kv_lens=tuple(range(1, 21)), prefix_lens=(0,), groups=[0, 20])
    q.run(prefix=q.make_prefix())
    q.check()
    a = q.out.clone()
    q.run()
    assert float((a.double() - q.out.double()).abs().max()) <= 2.0 ** -7


def test_offsets_beyond_32_bits():
    """A pool of more than 4 GiB a plane, its last blocks in use."""
    B, C, D = 16, 8, 128
    n_blocks = 135000                       # 4.4 GB a plane
    pool = torch.empty((2, n_blocks, B, C, D), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    n = 100
    ids = [n_blocks - 1 - 3 * j for j in range(7)]
    for b in ids:
        pool[:, b] = torch.randn((2, B, C, D), device="cuda", generator=g).to(torch.bfloat16)
    q = torch.randn((1, 8, D), device="cuda", generator=g).to(torch.bfloat16)
    out, lse = torch.empty_like(q), torch.empty((1, 8), device="cuda")
    desc = gms.KvPool(base=pool.data_ptr(), plane_stride=pool.stride(0) * 2, block_stride=pool.stride(1) * 2, n_planes=2, n_blocks=n_blocks,
                      block_bytes=B * C * D * 2)
    lay = gms.KvLayout(k_plane=0, v_plane=1, n_kv_heads=C, head_dim=D, block_tokens=B, dtype=gms.DTYPE_BF16, token_stride=C * D * 2,
                       head_stride=D * 2)
    a = gms.kv_attn(q=q, out=out, lse=lse, kv_lens=torch.tensor([n], dtype=torch.int32, device="cuda"),
                    block_table=torch.tensor([ids], dtype=torch.int32, device="cuda"), max_kv=n, scale=0.1)
    a.set_workspace(torch.empty(max(1, gms.gms_kv_attention_workspace(desc, lay, a)), dtype=torch.uint8, device="cuda"))
    gms.gms_kv_attention(desc, lay, a)
    rows = pool[:, ids].reshape(2, -1, C, D)[:, :n].double()
    x = torch.einsum("hd,thd->ht", q[0].double(), rows[0]) * 0.1
    want = torch.einsum("ht,thd->hd", torch.softmax(x, 1), rows[1])
    assert float((out[0].double() - want).abs().max()) < 2.0 ** -7
    assert float((lse[0].double() - torch.logsumexp(x, 1)).abs().max()) < 1e-4


def test_a_long_cache():
    p = Problem(15, heads=8, kv_heads=1, dim=128, q_lens=(1, 1, 2), kv_lens=(70001, 3, 40000), block=64)
    p.run()
    p.check()


def test_empty_calls():
    p = Problem(16, q_lens=(1,), kv_lens=(5,))
    p.attn.n_seq, p.attn.total_q, p.attn.max_q = 0, 0, 0
    before = p.out.clone()
    gms.gms_kv_attention(p.desc, p.layout, p.attn)
    torch.cuda.synchronize()
    assert torch.equal(before, p.out)
    # no queries at all, but weights that decay
    q = Problem(17, q_lens=(0, 0), kv_lens=(5, 20))
    w = torch.ones((2, 2, 20), device="cuda")
    q.run(gms.kv_weights(w, w, decay=0.5))
    assert bool((w[0, :, :5] == 0.5).all()) and bool((w[0, :, 5:] == 1).all()) and bool((w[1] == 0.5).all())


@pytest.mark.parametrize("dtype,dim,window", [(BF, 128, 0), (HF, 64, 9000)])
def test_weights_of_a_long_cache(dtype, dim, window):
    """Many chunks of tokens a CTA, more query rows than it holds at once, and few."""
    for q_lens, kv_lens in (((33, 70), (20001, 3000)), ((9, 0), (30011, 77))):
        p = Problem(18, dtype=dt(dtype), dim=dim, heads=24, kv_heads=8, block=16, q_lens=q_lens, kv_lens=kv_lens, window=window, sinks=5)
        w = torch.zeros((2, 8, max(kv_lens)), device="cuda")
        p.run(gms.kv_weights(None, w))
        ref = p.reference()
        p.check(ref)
        for s, n in enumerate(kv_lens):
            want = ref[s][4]
            assert not bool(((w[s, :, :n].double() - want).abs() > ref[s][5] + 2.0 ** -23 * (q_lens[s] * 24 + 2) * want).any())


def test_behind_a_call_that_is_still_writing():
    """The kernels may be scheduled before their predecessor in the stream has drained; they must not read what it has yet to
    write.  A restore of the pool's blocks (which lets its successors start early) goes directly before the attention."""
    p = Problem(19, heads=8, kv_heads=2, q_lens=(1,) * 24, kv_lens=(3000,) * 24)
    ids = torch.tensor(sum(p.table_h, []), dtype=torch.int32, device="cuda")
    n_sel, per = len(ids), p.block_bytes // 4096
    img = torch.empty((2, n_sel, p.block_bytes), dtype=torch.uint8, device="cuda")
    bd = torch.zeros(n_sel * 2 * per, dtype=torch.int64, device="cuda")
    st = torch.zeros(4, dtype=torch.int64, device="cuda")
    gms.gms_kv_capture(p.desc, img, n_sel * p.block_bytes, p.block_bytes, gms.SRC_DEVICE, ids, n_sel, bd, None, st)
    w = torch.zeros((24, 2, 3000), device="cuda")
    weight = gms.kv_weights(None, w)
    p.run(weight)
    ref = p.reference()
    p.check(ref)
    want, lse, weights = p.out.clone(), p.lse.clone(), w.clone()
    for _ in range(5):
        p.raw.fill_(0xFF)
        p.out.fill_(3)
        gms.gms_kv_restore(p.desc, img, n_sel * p.block_bytes, p.block_bytes, gms.SRC_DEVICE, ids, n_sel, bd, None, st)
        gms.gms_kv_attention(p.desc, p.layout, p.attn, weight)
        torch.cuda.synchronize()
        assert torch.equal(p.out, want) and torch.equal(p.lse, lse) and torch.equal(w, weights)


@pytest.mark.parametrize("seqs,n", [(1, 500), (2, 2000), (36, 40), (37, 130), (50, 513), (64, 17), (130, 900), (300, 12), (300, 100)])
@pytest.mark.parametrize("q", [1, 3])
def test_item_counts_around_what_the_gpu_holds(seqs, n, q):
    """A CTA an item or all tiles dealt out: both sides of the rule's borders, ragged lengths, empty sequences among them."""
    lens = [n] + [(7 * s * s + 3 * s) % n for s in range(1, seqs)]
    p = Problem(20, heads=32, kv_heads=8, q_lens=[min(q, max(m, 1)) for m in lens], kv_lens=lens, decode=q == 1)
    p.run()
    p.check()


@pytest.mark.parametrize("kv_lens,prefix", [((2500, 40), (3000,)), ((5000, 1), (17,)), ((30, 3000), (0,))])
def test_shared_prefix_with_long_suffixes(kv_lens, prefix):
    p = Problem(21, heads=8, kv_heads=2, q_lens=(1, 2), kv_lens=kv_lens, prefix_lens=prefix, groups=[0, 2])
    p.run(prefix=p.make_prefix())
    p.check()


@pytest.mark.parametrize("scale", [0.0, -0.05, 1.0])
@pytest.mark.parametrize("heads,kv_heads,q", [(8, 2, 1), (8, 2, 90), (12, 4, 60), (3, 3, 200)])
def test_scales(scale, heads, kv_heads, q):
    """Zero (the mean of what is seen), negative, and large; head groups that do and do not divide 128 rows."""
    p = Problem(22, heads=heads, kv_heads=kv_heads, q_lens=(q, q), kv_lens=(q + 150, q + 11), window=70, sinks=2)
    p.scale = p.attn.scale = scale
    w = torch.zeros((2, kv_heads, q + 150), device="cuda")
    p.run(gms.kv_weights(None, w))
    ref = p.reference()
    p.check(ref)
    for s, n in enumerate(p.kv_lens):
        assert not bool(((w[s, :, :n].double() - ref[s][4]).abs() > ref[s][5] + 2.0 ** -23 * (q * heads + 2) * ref[s][4]).any())
