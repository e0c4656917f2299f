"""What the attention and eviction calls refuse, before any device work (no GPU needed: addresses are made up)."""
import ctypes

import pytest

from paper_2609_25451_b200 import build as gms_build
from paper_2609_25451_b200 import gms

BASE = 0x7F0000000000


@pytest.fixture(scope="module", autouse=True)
def built():
    gms_build.build()


def pool(**kw):
    d = dict(base=BASE, plane_stride=32768 * 100, block_stride=32768, n_planes=4, n_blocks=100, block_bytes=32768)
    d.update(kw)
    return gms.KvPool(**d)


def layout(**kw):
    d = dict(k_plane=0, v_plane=1, n_kv_heads=8, head_dim=128, block_tokens=16, dtype=0, token_stride=2048, head_stride=256)
    d.update(kw)
    return gms.KvLayout(**d)


def attn(**kw):
    d = dict(q=BASE, out=BASE, lse=BASE, cu_q=BASE, kv_lens=BASE, block_table=BASE, workspace=BASE, workspace_bytes=1 << 40,
             q_token_stride=8192, q_head_stride=256, out_token_stride=8192, out_head_stride=256, table_stride=64, n_seq=3, n_heads=32,
             total_q=9, max_q=5, max_kv=1000, window=0, sinks=0, scale=0.1)
    d.update(kw)
    return gms.KvAttn(**d)


def weight(**kw):
    d = dict(in_=BASE, out=BASE, seq_stride=8000, head_stride=1000, decay=1.0)
    d.update(kw)
    return gms.KvWeight(**d)


def prefix(**kw):
    d = dict(group_start=BASE, prefix_lens=BASE, prefix_table=BASE, prefix_stride=10, n_groups=2, max_prefix=160, max_group_q=9)
    d.update(kw)
    return gms.KvPrefix(**d)


def evict(**kw):
    d = dict(weights=BASE, weights_out=BASE + 4, lens=BASE, lens_out=BASE, src_table=BASE, dst_table=BASE, kept=BASE, w_layer_stride=10**6,
             w_seq_stride=10**5, w_head_stride=10**4, o_layer_stride=10**6, o_seq_stride=10**5, o_head_stride=10**4, src_stride=64,
             dst_stride=8, n_layers=2, layer_planes=2, n_seq=3, max_len=1000, budget=100, sinks=4, recent=30)
    d.update(kw)
    return gms.KvEvictArgs(**d)


def status(fn, *args):
    try:
        fn(*args)
    except gms.GmsError as e:
        return e.status
    return gms.OK


POOL = [(dict(base=None), gms.ERR_NULL), (dict(base=BASE + 8), gms.ERR_ALIGN), (dict(plane_stride=32768 * 100 + 8), gms.ERR_ALIGN),
        (dict(block_bytes=5000), gms.ERR_ALIGN), (dict(block_bytes=0), gms.ERR_ALIGN), (dict(block_bytes=135168), gms.ERR_ARG),
        (dict(n_blocks=0), gms.ERR_ARG), (dict(block_stride=16384), gms.ERR_ARG), (dict(plane_stride=4096), gms.ERR_ARG),
        (dict(flags=2), gms.ERR_ARG), (dict(n_planes=1), gms.ERR_ARG)]
LAYOUT = [(dict(head_dim=96), gms.ERR_ARG), (dict(head_dim=0), gms.ERR_ARG), (dict(dtype=2), gms.ERR_ARG), (dict(n_kv_heads=0), gms.ERR_ARG),
          (dict(block_tokens=8), gms.ERR_ARG), (dict(block_tokens=24), gms.ERR_ARG), (dict(block_tokens=2048), gms.ERR_ARG),
          (dict(block_tokens=32), gms.ERR_ARG), (dict(k_plane=4), gms.ERR_ARG), (dict(v_plane=4), gms.ERR_ARG), (dict(v_plane=0), gms.ERR_ARG),
          (dict(token_stride=2040), gms.ERR_ALIGN), (dict(head_stride=8), gms.ERR_ALIGN), (dict(token_stride=1024), gms.ERR_ARG),
          (dict(head_stride=128), gms.ERR_ARG), (dict(token_stride=2064), gms.ERR_ARG)]
ATTN = [(dict(n_heads=12), gms.ERR_ARG), (dict(n_heads=0), gms.ERR_ARG), (dict(scale=float("inf")), gms.ERR_ARG),
        (dict(scale=float("nan")), gms.ERR_ARG), (dict(q=None), gms.ERR_NULL), (dict(out=None), gms.ERR_NULL), (dict(kv_lens=None), gms.ERR_NULL),
        (dict(block_table=None), gms.ERR_NULL), (dict(q=BASE + 8), gms.ERR_ALIGN), (dict(out=BASE + 4), gms.ERR_ALIGN),
        (dict(q_token_stride=8200), gms.ERR_ALIGN), (dict(out_head_stride=8), gms.ERR_ALIGN), (dict(lse=BASE + 2), gms.ERR_ALIGN),
        (dict(status=BASE + 4), gms.ERR_ALIGN), (dict(workspace=BASE + 16), gms.ERR_ALIGN), (dict(cu_q=None), gms.ERR_ARG),
        (dict(max_q=10), gms.ERR_ARG), (dict(max_kv=1025), gms.ERR_RANGE), (dict(max_kv=1 << 31), gms.ERR_ARG),
        (dict(total_q=1 << 28), gms.ERR_RANGE), (dict(table_stride=1 << 41), gms.ERR_RANGE)]


@pytest.mark.parametrize("kw,want", POOL)
def test_pool(kw, want):
    assert status(gms.gms_kv_attention, pool(**kw), layout(), attn()) == want
    assert status(gms.gms_kv_evict, pool(**kw), layout(), evict(n_layers=1)) == want


@pytest.mark.parametrize("kw,want", LAYOUT)
def test_layout(kw, want):
    assert status(gms.gms_kv_attention, pool(), layout(**kw), attn()) == want
    assert status(gms.gms_kv_evict, pool(), layout(**kw), evict()) == want


@pytest.mark.parametrize("kw,want", ATTN)
def test_attention(kw, want):
    assert status(gms.gms_kv_attention, pool(), layout(), attn(**kw)) == want
    assert status(gms.gms_kv_attention_shared, pool(), layout(), attn(**kw), prefix()) == want
    assert status(gms.gms_kv_attention_workspace, pool(), layout(), attn(**kw)) == want


@pytest.mark.parametrize("kw,want", [(dict(out=None), gms.ERR_NULL), (dict(out=BASE + 2), gms.ERR_ALIGN), (dict(decay=float("nan")), gms.ERR_ARG),
                                     (dict(reserved=1), gms.ERR_ARG)])
def test_weights(kw, want):
    assert status(gms.gms_kv_attention, pool(), layout(), attn(), weight(**kw)) == want


@pytest.mark.parametrize("kw,want", [(dict(group_start=None), gms.ERR_NULL), (dict(prefix_lens=None), gms.ERR_NULL),
                                     (dict(prefix_table=None), gms.ERR_NULL), (dict(prefix_lens=BASE + 1), gms.ERR_ALIGN),
                                     (dict(max_prefix=161), gms.ERR_RANGE), (dict(n_groups=4), gms.ERR_ARG), (dict(reserved=1), gms.ERR_ARG),
                                     (dict(max_group_q=10), gms.ERR_ARG)])
def test_prefix(kw, want):
    assert status(gms.gms_kv_attention_shared, pool(), layout(), attn(), prefix(**kw)) == want


def test_shared_takes_no_window():
    assert status(gms.gms_kv_attention_shared, pool(), layout(), attn(window=4), prefix()) == gms.ERR_ARG
    assert status(gms.gms_kv_attention_shared, pool(), layout(), attn(sinks=4), prefix()) == gms.ERR_ARG


@pytest.mark.parametrize("kw,want", [(dict(sinks=71), gms.ERR_ARG), (dict(sinks=2**32 - 1, recent=2), gms.ERR_ARG), (dict(layer_planes=0), gms.ERR_ARG),
                                     (dict(layer_planes=1), gms.ERR_ARG), (dict(n_layers=3), gms.ERR_ARG), (dict(weights=None), gms.ERR_NULL),
                                     (dict(kept=None), gms.ERR_NULL), (dict(lens=None), gms.ERR_NULL), (dict(src_table=None), gms.ERR_NULL),
                                     (dict(dst_table=None), gms.ERR_NULL), (dict(weights=BASE + 2), gms.ERR_ALIGN), (dict(src_stride=62), gms.ERR_RANGE),
                                     (dict(dst_stride=6), gms.ERR_RANGE), (dict(weights_out=BASE), gms.ERR_ARG), (dict(reserved=1), gms.ERR_ARG)])
def test_evict(kw, want):
    assert status(gms.gms_kv_evict, pool(), layout(), evict(**kw)) == want


def test_null_structures():
    for args in ((None, layout(), attn()), (pool(), None, attn()), (pool(), layout(), None)):
        assert status(gms.gms_kv_attention, *args) == gms.ERR_NULL
        assert status(gms.gms_kv_attention_shared, *args, prefix()) == gms.ERR_NULL
    assert status(gms.gms_kv_attention_shared, pool(), layout(), attn(), None) == gms.ERR_NULL
    assert status(gms.gms_kv_evict, pool(), layout(), None) == gms.ERR_NULL


def test_workspace_size_is_enforced():
    n = gms.gms_kv_attention_workspace(pool(), layout(), attn(lse=None), weight())
    assert n > 0
    assert status(gms.gms_kv_attention, pool(), layout(), attn(lse=None, workspace_bytes=n - 1), weight()) == gms.ERR_RANGE
    assert status(gms.gms_kv_attention, pool(), layout(), attn(lse=None, workspace=None), weight()) == gms.ERR_NULL


def test_struct_sizes_match_the_header(tmp_path):
    import os
    import subprocess

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "gms.h"\nint main(void) { printf("%zu %zu %zu %zu %zu\\n", sizeof(gms_kv_layout), '
                   'sizeof(gms_kv_attn), sizeof(gms_kv_weight), sizeof(gms_kv_prefix), sizeof(gms_kv_evict_args)); return 0; }\n')
    exe = str(tmp_path / "sizes")
    subprocess.check_call(["gcc", "-I", os.path.join(root, "include"), "-o", exe, str(src)])
    got = [int(x) for x in subprocess.check_output([exe]).split()]
    assert got == [ctypes.sizeof(t) for t in (gms.KvLayout, gms.KvAttn, gms.KvWeight, gms.KvPrefix, gms.KvEvictArgs)]
