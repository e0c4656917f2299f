"""What the binding of gms_kv_plan, gms_kv_append and gms_kv_delta refuses of tensors on a GPU (made up here: no GPU needed)."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_25451_b200 import gms  # noqa: E402


class OnGpu:
    """A host tensor that says it is on a GPU."""

    is_cuda = True

    def __init__(self, t, index=0):
        self.t, self.device = t, torch.device("cuda", index)

    def __getattr__(self, name):
        return getattr(self.t, name)


def gpu(*shape, dtype=torch.int32, index=0):
    return OnGpu(torch.zeros(shape, dtype=dtype), index)


def delta(**kw):
    x = dict(dtype=torch.bfloat16)
    return gms.kv_delta_args(**{**dict(q=gpu(5, 2, 64, **x), k=gpu(5, 2, 64, **x), v=gpu(5, 4, 64, **x), out=gpu(5, 4, 64, **x), src_table=gpu(3, 2), scale=1.0), **kw})


def append(**kw):
    x = dict(dtype=torch.bfloat16)
    return gms.kv_append_args(**{**dict(q=gpu(5, 4, 64, **x), k=gpu(5, 2, 64, **x), v=gpu(5, 2, 64, **x), slots=gpu(5, dtype=torch.int64)), **kw})


def test_a_workspace_on_another_device_is_refused():
    here, there = gpu(1024, dtype=torch.uint8), gpu(1024, dtype=torch.uint8, index=1)
    a = delta(workspace=here)
    assert a.workspace == here.data_ptr() and a.workspace_bytes == 1024
    with pytest.raises(ValueError, match="device"):
        delta(workspace=there)
    with pytest.raises(ValueError, match="device"):
        a.set_workspace(there)
    assert a.workspace == here.data_ptr()
    with pytest.raises(ValueError):
        a.set_workspace(torch.zeros(1024, dtype=torch.uint8))
    byhand = gms.KvDeltaArgs()  # (of no tensors: any device)
    byhand.set_workspace(there)
    assert byhand.workspace == there.data_ptr()


def test_a_number_of_rows_is_a_word():
    """An empty tensor has no address, which would stand for every row."""
    cu = gpu(4)
    assert append(n_rows=OnGpu(cu.t[3:])).n_rows == cu.t[3:].data_ptr()
    assert append().n_rows is None
    with pytest.raises(ValueError, match="n_rows"):
        append(n_rows=OnGpu(cu.t[4:]))
