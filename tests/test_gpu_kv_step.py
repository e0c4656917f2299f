"""The operators of an engine's step together: plan, append, attention and the delta rule on one batch that goes on for some steps, each
stage against 64-bit arithmetic on what the stage before has left; the example of such steps, with a failure in between."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2609_25451_b200 import gms  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF16 = torch.bfloat16


@pytest.mark.parametrize("kw", [{}, dict(layers=2, requests=1, steps=3, heads=2, kv_heads=1), dict(layers=3, requests=9, steps=5, heads=6, kv_heads=3)])
def test_example(kw):
    spec = importlib.util.spec_from_file_location("kv_step", os.path.join(ROOT, "examples", "kv_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    assert m.main(**kw, quiet=True) == kw.get("steps", 12) + 2


@pytest.mark.parametrize("D,order,window", [(64, "token", 0), (128, "head", 0), (64, "head", 20)])
def test_steps(D, order, window):
    S, H, C, B, room = 5, 8, 4, 32, 160
    g = torch.Generator(device="cuda")
    g.manual_seed(D + window)
    bb, n_blocks = B * C * D * 2, S * room // B
    pool = torch.randint(0, 256, (2 * n_blocks * bb,), dtype=torch.uint8, device="cuda", generator=g)  # whatever bits
    ts, hs = (C * D * 2, D * 2) if order == "token" else (D * 2, B * D * 2)
    desc = gms.KvPool(base=pool.data_ptr(), plane_stride=n_blocks * bb, block_stride=bb, n_planes=2, n_blocks=n_blocks, block_bytes=bb)
    lay = gms.KvLayout(k_plane=0, v_plane=1, n_kv_heads=C, head_dim=D, block_tokens=B, dtype=gms.DTYPE_BF16, token_stride=ts, head_stride=hs)
    planes = torch.as_strided(pool.view(BF16), (2, n_blocks, B, C, D), (n_blocks * bb // 2, bb // 2, ts // 2, hs // 2, 1))
    per = 131072 // (4 * D * D)
    sn = (H + per - 1) // per
    states = torch.full((S * sn, per, D, D), float("nan"), device="cuda")
    sdesc = gms.KvPool(base=states.data_ptr(), plane_stride=0, block_stride=131072, n_planes=1, n_blocks=S * sn, block_bytes=131072)
    stable = torch.randperm(S * sn, device="cuda", generator=g).to(torch.int32).view(S, sn)
    i32 = dict(dtype=torch.int32, device="cuda")
    lens, table = torch.zeros(S, **i32), torch.full((S, room // B), -1, **i32)
    free, fs = torch.randperm(n_blocks, device="cuda", generator=g).to(torch.int32), torch.tensor([5, n_blocks], **i32)
    status = torch.zeros(1, dtype=torch.int64, device="cuda")
    freq = torch.tensor([1e4 ** (-2.0 * j / D) for j in range(D // 2)], device="cuda")
    wq, wk = (1 + 0.2 * torch.randn(D, device="cuda", generator=g) for _ in range(2))
    history = [[] for _ in range(S)]          # (key, value) rows as they were written
    past_state = torch.zeros(S, H, D, D, dtype=torch.float64, device="cuda")
    for new in ([40, 1, 0, 70, 33], [1, 1, 30, 1, 1], [1, 0, 1, 2, 1], [3, 3, 3, 3, 3], [1, 1, 1, 1, 1]):
        T, pad = sum(new), 3
        qkv = (torch.randn((T + pad, (H + 2 * C) * D), device="cuda", generator=g)).to(BF16)
        q, k, v = (x.view(T + pad, -1, D) for x in qkv.split([H * D, C * D, C * D], 1))
        cu, pos = torch.zeros(S + 1, **i32), torch.zeros(T + pad, **i32)
        slots = torch.zeros(T + pad, dtype=torch.int64, device="cuda")
        gms.gms_kv_plan(gms.kv_plan_args(n_blocks=n_blocks, block_tokens=B, lens=lens, new_lens=torch.tensor(new, **i32), block_table=table,
                                         free_ids=free, free_state=fs, cu_q=cu, slots=slots, positions=pos, status=status))
        q_out = torch.full((T + pad, H, D), 9.0, dtype=BF16, device="cuda")
        gms.gms_kv_append(desc, lay, gms.kv_append_args(q=q, k=k, v=v, q_out=q_out, slots=slots, n_rows=cu[S:], positions=pos, inv_freq=freq,
                                                        q_weight=wq, k_weight=wk))
        out = torch.full((T + pad, H, D), 7.0, dtype=BF16, device="cuda")
        a = gms.kv_attn(q=q_out, out=out, cu_q=cu, kv_lens=lens, block_table=table, max_q=max(new), max_kv=room, window=window, scale=D ** -0.5)
        a.set_workspace(torch.empty(gms.gms_kv_attention_workspace(desc, lay, a), dtype=torch.uint8, device="cuda"))
        gms.gms_kv_attention(desc, lay, a)
        # the recurrent layer on the same rows: keys of four heads for eight heads' values
        dv = torch.randn((T + pad, H, D), device="cuda", generator=g).to(BF16)
        gate, beta = -torch.rand((T + pad, H), device="cuda", generator=g), torch.rand((T + pad, H), device="cuda", generator=g)
        rec = torch.full((T + pad, H, D), 7.0, dtype=BF16, device="cuda")
        da = gms.kv_delta_args(q=k, k=k, v=dv, g=gate, beta=beta, out=rec, cu_q=cu, max_q=max(new), past_lens=lens - torch.tensor(new, **i32),
                               src_table=stable, scale=1.0, unit_eps=1e-6)
        da.set_workspace(torch.empty(max(256, gms.gms_kv_delta_workspace(sdesc, gms.KvState(plane=0, n_heads=H, head_dim=D), da)), dtype=torch.uint8,
                                     device="cuda"))
        gms.gms_kv_delta(sdesc, gms.KvState(plane=0, n_heads=H, head_dim=D), da)
        torch.cuda.synchronize()
        assert int(status) == 0 and cu.tolist() == [sum(new[:s]) for s in range(S + 1)]
        assert (q_out[T:] == 9).all() and (out[T:] == 7).all() and (rec[T:] == 7).all() and (slots[T:] == -1).all()
        lh = lens.tolist()
        for s in range(S):
            r = slice(sum(new[:s]), sum(new[:s]) + new[s])
            history[s] += [(planes[0, int(slots[i]) // B, int(slots[i]) % B].clone(), v[i].clone()) for i in range(r.start, r.stop)]
            assert lh[s] == len(history[s]) and pos[r].tolist() == list(range(lh[s] - new[s], lh[s]))
            # keys: the norm and the rotation in 64 bits
            x = k[r].double()
            x = x / ((x * x).mean(-1, keepdim=True) + 1e-6).sqrt() * wk.double()
            angle = pos[r].double()[:, None] * freq.double()
            c, sn_ = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
            x = torch.cat([x[..., :D // 2] * c - x[..., D // 2:] * sn_, x[..., D // 2:] * c + x[..., :D // 2] * sn_], -1)
            for i, (key, _) in enumerate(history[s][lh[s] - new[s]:]):
                assert ((key.double() - x[i]).abs() <= 2.0 ** -8 * x[i].abs() + 1e-4).all()
            if not lh[s]:
                continue
            # everything that was ever written is still there, where the table says
            for t, (key, value) in enumerate(history[s]):
                b = int(table[s, t // B])
                assert torch.equal(planes[0, b, t % B], key) and torch.equal(planes[1, b, t % B], value)
            if new[s]:
                K = torch.stack([h[0] for h in history[s]]).double().repeat_interleave(H // C, 1)
                V = torch.stack([h[1] for h in history[s]]).double().repeat_interleave(H // C, 1)
                z = torch.einsum("ihd,thd->hit", q_out[r].double(), K) * D ** -0.5
                p, t = pos[r][:, None], torch.arange(lh[s], device="cuda")[None, :]
                z = z.masked_fill((t > p) | ((t <= p - window) if window else torch.zeros_like(t > p)), -math.inf)
                want = torch.einsum("hit,thd->ihd", torch.softmax(z, -1), V)
                # weights and output rounded to bf16 once each: 2^-8 of the largest value's size twice
                assert ((out[r].double() - want).abs() <= 2.0 ** -7 * V.abs().max()).all()
            Sx = past_state[s]
            for i in range(r.start, r.stop):
                kk = k[i].double().repeat_interleave(H // C, 0)
                kk = kk / ((kk * kk).sum(-1, keepdim=True) + 1e-6).sqrt()
                Sx = Sx * gate[i].double().exp()[:, None, None]
                d = beta[i].double()[:, None] * (dv[i].double() - (kk[:, :, None] * Sx).sum(1))
                Sx = Sx + kk[:, :, None] * d[:, None, :]
                want = (kk[:, :, None] * Sx).sum(1)
                # two terms of 16 bits and one rounding; one term of 16 bits in chunks: 2 2^-8 of what a column can hold
                assert ((rec[i].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -7 * Sx.norm(dim=1).clamp(min=1.0) * 2).all()
            past_state[s] = Sx
            got = torch.stack([states[int(stable[s, h // per]), h % per] for h in range(H)]).double()
            if lh[s]:
                assert ((got - Sx).flatten(1).norm(dim=1) <= 1e-3 * Sx.flatten(1).norm(dim=1) + 1e-5).all()
