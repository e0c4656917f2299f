"""What the binding's helpers refuse before an address reaches a kernel: tensors that are too small, strided or not on a GPU."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2609_25451_b200 import build as gms_build
from paper_2609_25451_b200 import gms
from test_kv_operators_host import layout, pool


@pytest.fixture(scope="module", autouse=True)
def built():
    gms_build.build()


@pytest.fixture
def on_gpu(monkeypatch):
    """Tensors of this process pass for a GPU's: all that follows is refused before any of them is read."""
    monkeypatch.setattr(torch.Tensor, "is_pinned", lambda self: True)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def attn(**kw):
    d = dict(q=torch.zeros((3, 32, 128), dtype=torch.bfloat16), out=torch.zeros((3, 32, 128), dtype=torch.bfloat16), kv_lens=i32(3), block_table=i32(3, 10),
             max_kv=160, scale=0.1)
    d.update(kw)
    return gms.kv_attn(**d)


def evict(**kw):
    d = dict(weights=torch.zeros((2, 3, 8, 100)), lens=i32(3), src_table=i32(3, 7), dst_table=i32(3, 2), kept=i32(2, 3, 8, 32), max_len=100, budget=32)
    d.update(kw)
    return gms.kv_evict_args(**d)


def test_host_memory_is_refused():
    with pytest.raises(ValueError, match="host memory"):
        attn()
    with pytest.raises(ValueError, match="host memory"):
        evict()
    with pytest.raises(ValueError, match="device memory"):
        gms.KvAttn().set_workspace(torch.zeros(1 << 10, dtype=torch.uint8))
    with pytest.raises(ValueError, match="host memory"):
        gms.kv_weights(None, torch.zeros((3, 8, 160)))
    with pytest.raises(ValueError, match="host memory"):
        gms.kv_prefix(group_start=i32(2), prefix_lens=i32(1), prefix_table=i32(1, 4), max_prefix=64, max_group_q=3)


@pytest.mark.parametrize("kw", [
    dict(kv_lens=torch.tensor(5, dtype=torch.int32).expand(3)),              # one word for all: the kernels read three
    dict(block_table=i32(3, 1).expand(3, 10)), dict(kv_lens=i32(6)[::2]), dict(kv_lens=torch.zeros(3, dtype=torch.int64)),
    dict(kv_lens=torch.zeros(3)), dict(lse=torch.zeros((3, 1)).expand(3, 32)), dict(cu_q=torch.tensor(0, dtype=torch.int32).expand(4)),
    dict(status=torch.zeros(1)), dict(q=torch.zeros((3, 32, 128))), dict(q=torch.zeros((3, 32, 256), dtype=torch.bfloat16)[:, :, ::2])])
def test_strides_and_types(on_gpu, kw):
    attn()
    with pytest.raises(ValueError):
        attn(**kw)


@pytest.mark.parametrize("lay,kw", [(layout(head_dim=64, token_stride=1024, head_stride=128), {}), (layout(dtype=gms.DTYPE_F16), {}), (layout(), dict(max_kv=161))])
def test_attention_against_the_layout(on_gpu, lay, kw):
    with pytest.raises(ValueError):
        gms.gms_kv_attention(pool(), lay, attn(**kw))


@pytest.mark.parametrize("shape", [(2, 8, 160), (3, 4, 160), (3, 8, 159)])
def test_weights_that_are_too_small(on_gpu, shape):
    with pytest.raises(ValueError):
        gms.gms_kv_attention(pool(), layout(), attn(), gms.kv_weights(None, torch.zeros(shape)))
    with pytest.raises(ValueError):
        gms.kv_weights(torch.zeros((3, 8, 160))[:, :, :100], torch.zeros((3, 8, 160)))


def test_a_prefix_table_that_is_too_short(on_gpu):
    x = gms.kv_prefix(group_start=i32(2), prefix_lens=i32(1), prefix_table=i32(1, 4), max_prefix=65, max_group_q=3)
    with pytest.raises(ValueError):
        gms.gms_kv_attention_shared(pool(), layout(), attn(), x)


@pytest.mark.parametrize("kw", [dict(max_len=101, src_table=i32(3, 9)), dict(weights_out=torch.zeros((2, 3, 8, 31))), dict(weights_out=torch.zeros((2, 3, 4, 32))),
                                dict(lens_out=i32(2)), dict(lens=torch.tensor(5, dtype=torch.int32).expand(3))])
def test_eviction(on_gpu, kw):
    evict()
    with pytest.raises(ValueError):
        evict(**kw)


@pytest.mark.parametrize("kw", [dict(src_table=i32(3, 6)), dict(dst_table=i32(3, 1)), dict(weights=torch.zeros((2, 3, 4, 100)), kept=i32(2, 3, 4, 32))])
def test_eviction_against_the_layout(on_gpu, kw):
    with pytest.raises(ValueError):
        gms.gms_kv_evict(pool(), layout(), evict(**kw))


def test_structures_made_by_hand_are_the_callers():
    a = gms.KvAttn(n_heads=3)
    assert a._made is None and ctypes.sizeof(a) > 0
