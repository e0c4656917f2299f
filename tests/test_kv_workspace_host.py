"""One workspace, sized for the largest call, serves every smaller one (no GPU needed: addresses are made up)."""
import random

import pytest

from paper_2609_25451_b200 import build as gms_build
from paper_2609_25451_b200 import gms
from test_kv_operators_host import BASE, attn, layout, prefix, weight
from test_kv_operators_host import pool as small_pool


@pytest.fixture(scope="module", autouse=True)
def built():
    gms_build.build()


def pool():
    return small_pool(block_bytes=65536, block_stride=65536, plane_stride=100 * 65536)


def layout_of(kv_heads, dim):
    return layout(n_kv_heads=kv_heads, head_dim=dim, token_stride=kv_heads * dim * 2, head_stride=dim * 2)


def size(lay, heads, seqs, max_q, max_kv, total_q, w=None, window=0, lse=None, x=None):
    a = attn(n_heads=heads, n_seq=seqs, max_q=max_q, max_kv=max_kv, total_q=total_q, table_stride=1 << 20, window=window, lse=lse)
    if x is not None:
        return gms.gms_kv_attention_shared_workspace(pool(), lay, a, x)
    return gms.gms_kv_attention_workspace(pool(), lay, a, w)


def test_the_sizes_of_a_shrinking_batch():
    lay = layout_of(8, 128)
    for w in (None, weight()):
        sizes = [size(lay, 32, n, 1, 2048, n, w) for n in (256, 64, 48, 32, 16, 1)]
        assert sizes == sorted(sizes, reverse=True), sizes
        # more than 16 rows a KV head, then fewer
        sizes = [size(lay, 32, 4, q, 16000, 4 * q, w) for q in (300, 64, 5, 4, 3, 1)]
        assert sizes == sorted(sizes, reverse=True), sizes


@pytest.mark.parametrize("heads,kv_heads,dim", [(32, 8, 128), (8, 1, 64), (16, 16, 128), (24, 8, 64), (40, 1, 128)])
@pytest.mark.parametrize("kind", ["plain", "window", "weights", "weights and lse", "shared"])
def test_smaller_calls_never_take_more(heads, kv_heads, dim, kind):
    rng = random.Random(heads * 1000 + kv_heads)
    lay = layout_of(kv_heads, dim)
    w = weight() if kind.startswith("weights") else None
    window = 300 if kind == "window" else 0
    lse = BASE if kind != "weights" else None

    def log(hi):
        return max(1, min(hi, round(hi ** rng.random())))

    def of(seqs, max_q, max_kv, total_q, groups, most, rows):
        x = prefix(n_groups=min(groups, seqs), max_prefix=most, max_group_q=min(rows, total_q), prefix_stride=1 << 20) if kind == "shared" else None
        return size(lay, heads, seqs, min(max_q, total_q), max_kv, total_q, w, window, lse, x)

    for _ in range(400):
        big = (log(300), log(500), log(70000), 0, log(8), log(40000), 0)
        big = big[:3] + (big[0] * big[1],) + big[4:6] + (big[0] * big[1],)
        small = tuple(log(v) for v in big)
        assert of(*small) <= of(*big), (big, small)


def test_kept_logits_under_a_window():
    """4 bytes for each head and token in reach, whatever the longest sequence is."""
    lay = layout_of(8, 128)
    far = size(lay, 32, 256, 1, 1 << 20, 256, weight(), window=256)
    near = size(lay, 32, 256, 1, 1 << 12, 256, weight(), window=256)
    assert far == near and far < 256 * 32 * 400 * 4 + (32 << 20)
