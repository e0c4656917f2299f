"""What gms_kv_plan, gms_kv_append and gms_kv_delta refuse, before any device work (no GPU needed: addresses are made up)."""
import ctypes
import os
import subprocess

import pytest

from paper_2609_25451_b200 import build as gms_build
from paper_2609_25451_b200 import gms

BASE = 0x7F0000000000
FAR = [BASE + (i << 32) for i in range(1, 20)]
N, A, R, G = gms.ERR_NULL, gms.ERR_ALIGN, gms.ERR_RANGE, gms.ERR_ARG


@pytest.fixture(scope="module", autouse=True)
def built():
    gms_build.build()


def status(fn, *args):
    try:
        fn(*args)
    except gms.GmsError as e:
        return e.status
    return gms.OK


def pool(**kw):
    d = dict(base=BASE, plane_stride=131072 * 100, block_stride=131072, n_planes=4, n_blocks=100, block_bytes=131072)
    d.update(kw)
    return gms.KvPool(**d)


def layout(**kw):
    d = dict(k_plane=0, v_plane=1, n_kv_heads=8, head_dim=128, block_tokens=16, dtype=0, token_stride=2048, head_stride=256)
    d.update(kw)
    return gms.KvLayout(**d)


def plan(**kw):
    d = dict(lens=FAR[0], new_lens=FAR[1], drop_lens=FAR[2], lens_out=FAR[3], block_table=FAR[4], free_ids=FAR[5], free_state=FAR[6],
             free_state_out=FAR[7], cu_q=FAR[8], slots=FAR[9], positions=FAR[10], status=FAR[11], table_stride=64, n_seq=5, total_rows=40,
             table_blocks=60, free_cap=100, n_blocks=100, block_tokens=16)
    d.update(kw)
    return gms.KvPlanArgs(**d)


def append(**kw):
    d = dict(q=FAR[0], k=FAR[1], v=FAR[2], q_out=FAR[3], slots=FAR[4], positions=FAR[5], n_rows=FAR[6], inv_freq=FAR[7], axes=FAR[8],
             q_weight=FAR[9], k_weight=FAR[10], q_token_stride=8192, q_head_stride=256, k_token_stride=2048, k_head_stride=256,
             v_token_stride=2048, v_head_stride=256, out_token_stride=8192, out_head_stride=256, positions_stride=40, rows=40, n_heads=32,
             rotary_dim=128, n_axes=3, pairs=0, weight_dtype=2, weight_offset=0.0, eps=1e-6, rope_scale=1.0)
    d.update(kw)
    return gms.KvAppendArgs(**d)


def state(**kw):
    d = dict(plane=1, n_heads=32, head_dim=128)
    d.update(kw)
    return gms.KvState(**d)


def delta(**kw):
    d = dict(q=FAR[0], k=FAR[1], v=FAR[2], out=FAR[3], g=FAR[4], beta=FAR[5], cu_q=FAR[6], past_lens=FAR[7], src_table=FAR[8], dst_table=FAR[9],
             workspace=FAR[10], workspace_bytes=1 << 40, q_token_stride=4096, q_head_stride=256, k_token_stride=4096, k_head_stride=256,
             v_token_stride=8192, v_head_stride=256, out_token_stride=8192, out_head_stride=256, g_stride=32, beta_stride=32, src_stride=16,
             dst_stride=16, n_seq=3, n_key_heads=16, total_q=9, max_q=5, dtype=0, unit_qk=1, unit_eps=1e-6, scale=0.1)
    d.update(kw)
    return gms.KvDeltaArgs(**d)


@pytest.mark.parametrize("kw,want", [
    (dict(block_tokens=8), G), (dict(block_tokens=24), G), (dict(block_tokens=2048), G), (dict(block_tokens=0), G), (dict(n_blocks=0), G),
    (dict(n_blocks=1 << 31), G), (dict(total_rows=1 << 31), G), (dict(n_seq=1 << 31), G), (dict(free_cap=1 << 31), G), (dict(table_blocks=65), R),
    (dict(table_stride=1 << 41), R), (dict(table_stride=1 << 30, table_blocks=(1 << 20) + 1), R), (dict(lens=FAR[0] + 2), A),
    (dict(slots=FAR[9] + 4), A), (dict(status=FAR[9] + 4), A), (dict(positions=FAR[9] + 1), A), (dict(lens=None), N), (dict(new_lens=None), N),
    (dict(lens_out=None), N), (dict(block_table=None), N), (dict(free_ids=None), N), (dict(free_state=None), N), (dict(free_state_out=None), N),
    (dict(cu_q=None), N), (dict(slots=None), N), (dict(lens_out=FAR[0] + 4), G), (dict(lens_out=FAR[1]), G), (dict(lens_out=FAR[2] + 16), G),
    (dict(free_state_out=FAR[6] + 4), G)])
def test_plan(kw, want):
    assert status(gms.gms_kv_plan, plan(**kw)) == want


@pytest.mark.parametrize("kw,want", [
    (dict(reserved=1), G), (dict(rotary_dim=12), G), (dict(rotary_dim=136), G), (dict(n_axes=0), G), (dict(n_axes=9), G), (dict(pairs=2), G),
    (dict(weight_dtype=3), G), (dict(weight_offset=float("nan")), G), (dict(eps=float("inf")), G), (dict(eps=-1.0), G), (dict(rope_scale=float("inf")), G),
    (dict(rows=1 << 31), G), (dict(q=None), N), (dict(n_heads=0), N), (dict(q_out=None), N), (dict(k=None), N), (dict(v=None), N), (dict(slots=None), N),
    (dict(positions=None), N), (dict(inv_freq=None), N), (dict(q=FAR[0] + 8), A), (dict(k_weight=FAR[0] + 8), A), (dict(k_token_stride=2056), A),
    (dict(slots=FAR[0] + 4), A), (dict(positions=FAR[0] + 2), A), (dict(n_rows=FAR[0] + 2), A), (dict(positions_stride=39), R),
    (dict(positions_stride=1 << 41), R), (dict(q_out=FAR[0], out_token_stride=16384), G), (dict(rows=(1 << 31) - 1, positions_stride=1 << 31), R)])
def test_append(kw, want):
    assert status(gms.gms_kv_append, pool(), layout(), append(**kw)) == want


@pytest.mark.parametrize("kw,want", [(dict(base=None), N), (dict(base=BASE + 8), A), (dict(n_planes=1), G)])
def test_append_pool(kw, want):
    assert status(gms.gms_kv_append, pool(**kw), layout(), append()) == want


@pytest.mark.parametrize("kw,want", [(dict(dtype=2), G), (dict(head_dim=96), G), (dict(token_stride=2040), A), (dict(v_plane=0), G)])
def test_append_layout(kw, want):
    assert status(gms.gms_kv_append, pool(), layout(**kw), append()) == want


@pytest.mark.parametrize("kw,want", [
    (dict(n_key_heads=0), G), (dict(n_key_heads=12), G), (dict(dtype=2), G), (dict(unit_qk=2), G), (dict(scale=float("nan")), G),
    (dict(unit_eps=float("inf")), G), (dict(unit_eps=-1.0), G), (dict(max_q=10), G), (dict(cu_q=None), G), (dict(total_q=1 << 31), G), (dict(q=None), N),
    (dict(k=None), N), (dict(v=None), N), (dict(out=None), N), (dict(src_table=None), N), (dict(dst_table=None), N), (dict(q=FAR[0] + 8), A),
    (dict(v_head_stride=264), A), (dict(g=FAR[0] + 2), A), (dict(status=FAR[0] + 4), A), (dict(workspace=FAR[0] + 128), A), (dict(src_stride=15), R),
    (dict(dst_stride=15), R), (dict(g_stride=31), R), (dict(beta_stride=8), R)])
def test_delta(kw, want):
    assert status(gms.gms_kv_delta, pool(), state(), delta(**kw)) == want
    assert status(gms.gms_kv_delta_workspace, pool(), state(), delta(**kw)) == want


@pytest.mark.parametrize("kw,want", [(dict(plane=4), G), (dict(n_heads=0), G), (dict(head_dim=96), G), (dict(reserved=1), G), (dict(n_heads=24), G)])
def test_delta_state(kw, want):
    assert status(gms.gms_kv_delta, pool(), state(**kw), delta()) == want


def test_delta_pool():
    assert status(gms.gms_kv_delta, pool(block_bytes=32768), state(), delta()) == G  # no room for a state of 64 KiB
    assert status(gms.gms_kv_delta, pool(block_bytes=65536), state(), delta()) == R  # one head a block: 32 blocks a row
    assert status(gms.gms_kv_delta, pool(base=None), state(), delta()) == N


def test_delta_workspace_size_is_enforced():
    need = gms.gms_kv_delta_workspace(pool(), state(), delta(total_q=9000, max_q=5000))
    if need:
        assert status(gms.gms_kv_delta, pool(), state(), delta(total_q=9000, max_q=5000, workspace_bytes=need - 1)) == R
        assert status(gms.gms_kv_delta, pool(), state(), delta(total_q=9000, max_q=5000, workspace=None)) == N
    sizes = [gms.gms_kv_delta_workspace(pool(), state(), delta(n_seq=s, total_q=t, max_q=m))
             for s, t, m in ((1, 1, 1), (1, 64, 64), (1, 65, 65), (2, 200, 101), (3, 9000, 5000), (64, 9000, 9000), (64, 9000, 200))]
    for (a, b) in ((0, 1), (1, 2), (2, 3), (3, 4), (4, 5), (6, 5)):  # no smaller call takes more
        assert sizes[a] <= sizes[b]


def test_null_structures():
    assert status(gms.gms_kv_plan, None) == N
    for args in ((None, layout(), append()), (pool(), None, append()), (pool(), layout(), None)):
        assert status(gms.gms_kv_append, *args) == N
    for args in ((None, state(), delta()), (pool(), None, delta()), (pool(), state(), None)):
        assert status(gms.gms_kv_delta, *args) == N
        assert status(gms.gms_kv_delta_workspace, *args) == N


def test_struct_sizes_match_the_header(tmp_path):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "gms.h"\nint main(void) { printf("%zu %zu %zu %zu\\n", sizeof(gms_kv_plan_args), '
                   'sizeof(gms_kv_append_args), sizeof(gms_kv_state), sizeof(gms_kv_delta_args)); return 0; }\n')
    exe = str(tmp_path / "sizes")
    subprocess.check_call(["gcc", "-I", os.path.join(root, "include"), "-o", exe, str(src)])
    got = [int(x) for x in subprocess.check_output([exe]).split()]
    assert got == [ctypes.sizeof(t) for t in (gms.KvPlanArgs, gms.KvAppendArgs, gms.KvState, gms.KvDeltaArgs)]


def test_binding_refuses_tensors_that_do_not_fit():
    torch = pytest.importorskip("torch")
    i32 = dict(dtype=torch.int32)
    ok = dict(n_blocks=4, block_tokens=16, lens=torch.zeros(3, **i32), new_lens=torch.zeros(3, **i32), block_table=torch.zeros(3, 2, **i32),
              free_ids=torch.zeros(4, **i32), free_state=torch.zeros(2, **i32), cu_q=torch.zeros(4, **i32), slots=torch.zeros(5, dtype=torch.int64))
    for bad in ({}, dict(new_lens=torch.zeros(2, **i32)), dict(cu_q=torch.zeros(3, **i32)), dict(free_state=torch.zeros(3, **i32)),
                dict(positions=torch.zeros(4, **i32)), dict(slots=torch.zeros(5, **i32)), dict(block_table=torch.zeros(2, 2, **i32))):
        with pytest.raises(ValueError):  # {}: pageable host memory
            gms.kv_plan_args(**{**ok, **bad})
    x = torch.zeros(5, 4, 64, dtype=torch.bfloat16)
    for bad in ({}, dict(q=x.half()), dict(v=x[:4]), dict(v=x[:, :2]), dict(k=None), dict(slots=None)):
        with pytest.raises(ValueError):
            gms.kv_append_args(**{**dict(q=x, k=x, v=x, slots=torch.zeros(5, dtype=torch.int64)), **bad})
    for bad in ({}, dict(q=x[:, :, :32]), dict(out=x[:, :2]), dict(g=torch.zeros(5, 3)), dict(cu_q=torch.zeros(1, **i32))):
        with pytest.raises(ValueError):
            gms.kv_delta_args(**{**dict(q=x, k=x, v=x, out=x, src_table=torch.zeros(3, 2, **i32), scale=1.0), **bad})


def test_tensors_of_another_device_are_refused(monkeypatch):
    torch = pytest.importorskip("torch")
    from types import SimpleNamespace

    def on(i):
        return SimpleNamespace(is_cuda=i is not None, device=SimpleNamespace(index=i))

    assert gms._one_device((on(1), None, on(1), on(None))) == 1 and gms._one_device((None, on(None))) is None
    with pytest.raises(ValueError):
        gms._one_device((on(0), on(1)))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for args, call in ((plan(), gms.gms_kv_plan), (append(), lambda a: gms.gms_kv_append(pool(), layout(), a)),
                       (delta(), lambda a: gms.gms_kv_delta(pool(), state(), a))):
        args._device = 1
        with pytest.raises(ValueError):
            call(args)
