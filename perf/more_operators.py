"""What is measured of an engine step's operators on the state pool: cases, inputs, plain forms, exact values and floors.

The operators: ``plan`` (block tables and slot maps from request lengths), ``append`` (queries and keys normed and
rotated, keys and values written into paged blocks) and ``delta`` (the gated delta rule with its states in the pool).
With ``own`` true ``run`` makes the calls of the library, else it computes the same in elementary torch operations.
"""
import math
import random

import numpy as np
import torch

own = False

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------ cases
def _plan(name, **kw):
    c = {"name": name, "op": "plan", "block": 16, "seqs": 1, "len_max": 1, "len_min": 0, "new_max": 1, "new_min": 1, "leave": 0.0,
         "reject": 0, "pad": 0, "ragged": 1}
    c.update(kw)
    return c


def _append(name, **kw):
    c = {"name": name, "op": "append", "dtype": "bf16", "weights": "bf16", "heads": 32, "kv_heads": 8, "dim": 128, "block": 16,
         "order": "token", "rotary": 128, "pairs": "halves", "axes": 1, "norm": True, "offset": 0.0, "seqs": 1, "new_max": 1, "new_min": 1,
         "past_max": 0, "pad": 0, "ragged": 1}
    c.update(kw)
    return c


def _delta(name, **kw):
    c = {"name": name, "op": "delta", "dtype": "bf16", "heads": 32, "key_heads": 16, "dim": 128, "seqs": 1, "q_max": 1, "q_min": 1,
         "fresh": 0.0, "decay": 1.0, "unit": True, "ragged": 1}
    c.update(kw)
    return c


def listed():
    return [
        # one user's next token
        _plan("plan-decode-one", len_max=701, len_min=701),
        # a serving batch's next tokens, up to 4 a sequence with speculation of which some are taken back; rows padded to a graph's size
        _plan("plan-decode-batch", seqs=250, len_max=12001, len_min=300, new_max=4, reject=3, pad=24),
        # requests come and go: a third of the rows hold finished requests whose blocks go back, new prompts beside decoding ones
        _plan("plan-turnover", seqs=511, len_max=32768, len_min=17, new_max=601, new_min=1, leave=0.35),
        # one user's next token in one layer
        _append("append-decode-one", past_max=701),
        # a batch's next tokens on one rank of eight, heads-first blocks of 32, neighbouring pairs, no norms, fp16, padded
        _append("append-decode-rank", dtype="f16", heads=8, kv_heads=1, block=32, order="head", pairs="neighbours", norm=False, seqs=61,
                past_max=30000, pad=3),
        # a prompt of pictures and text: positions with three axes
        _append("append-three-axes", heads=16, kv_heads=4, axes=3, seqs=2, new_max=4001, new_min=2500),
        # a step's worth of prompts far into long documents, small heads of which half is rotated, weights stored as w - 1
        _append("append-prompts", weights="f32", heads=32, kv_heads=8, dim=64, rotary=32, offset=1.0, seqs=12, new_max=8192, new_min=100,
                past_max=900000),
        # one user's next token in one layer
        _delta("delta-decode-one"),
        # a batch's next tokens: every state is read and written
        _delta("delta-decode-batch", seqs=64),
        # speculation: up to 4 tokens a sequence, some sequences new
        _delta("delta-speculate", seqs=29, q_max=4, fresh=0.2),
        # a whole prompt
        _delta("delta-prompt", q_max=8192, q_min=8192, fresh=1.0),
        # chunked prefill mixed with decoding sequences, fp16, small heads, queries and keys used as they are
        _delta("delta-mixed", dtype="f16", heads=16, key_heads=16, dim=64, seqs=13, q_max=2001, fresh=0.5, unit=False),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    listed_work = {}
    for c in listed():
        w = work(c)
        m = listed_work.setdefault(c["op"], {"bytes": 0, "flops": 0})
        for k in m:
            m[k] = max(m[k], w[k])
    while True:
        op = rng.choice(["plan", "append", "append", "delta", "delta"])
        if op == "plan":
            n = _log_int(rng, 1, 32768)
            new = _log_int(rng, 1, 2048)
            c = _plan("", block=rng.choice([16, 32, 64, 128]), seqs=_log_int(rng, 1, 700), len_max=n, len_min=rng.randint(0, n), new_max=new,
                      new_min=rng.randint(0, new), leave=rng.choice([0.0, 0.2, 0.5]), reject=rng.choice([0, 0, 4]),
                      pad=rng.choice([0, 0, rng.randint(1, 300)]))
        elif op == "append":
            heads, kv_heads = rng.choice([(32, 8), (8, 1), (32, 32), (16, 4), (24, 8), (20, 4)])
            dim, axes = rng.choice([64, 128]), rng.choice([1, 1, 3])
            blocks = [b for b in (16, 32, 64) if b * kv_heads * dim * 2 % 4096 == 0 and b * kv_heads * dim * 2 <= 131072]
            if not blocks:
                continue
            new = _log_int(rng, 1, 8192)
            c = _append("", dtype=rng.choice(["bf16", "f16"]), weights=rng.choice(["bf16", "f32"]), heads=heads, kv_heads=kv_heads, dim=dim,
                        block=rng.choice(blocks), order=rng.choice(["token", "head"]), rotary=8 * rng.randint(1, dim // 8),
                        pairs=rng.choice(["halves", "neighbours"]), axes=axes, norm=rng.random() < 0.7, offset=rng.choice([0.0, 1.0]),
                        seqs=_log_int(rng, 1, 128), new_max=new, new_min=rng.randint(1, new), past_max=_log_int(rng, 1, 1000000),
                        pad=rng.choice([0, 0, rng.randint(1, 60)]))
        else:
            heads, key_heads = rng.choice([(32, 16), (16, 16), (4, 2), (8, 8), (24, 8), (6, 6)])
            q = rng.choice([1, 1, _log_int(rng, 2, 8192)])
            c = _delta("", dtype=rng.choice(["bf16", "bf16", "f16"]), heads=heads, key_heads=key_heads, dim=rng.choice([64, 128]),
                       seqs=_log_int(rng, 1, 96 if q < 64 else 16), q_max=q, q_min=rng.randint(1, q), fresh=rng.choice([0.0, 0.5, 1.0]),
                       decay=rng.choice([0.1, 1.0, 4.0]), unit=rng.random() < 0.7)
        c["ragged"] = rng.randrange(1 << 30)
        w = work(c)
        if all(w[k] <= listed_work[op][k] for k in w):
            del c["name"]
            return c


def _lens(c):
    """Ragged lengths: part of the case, not of the seed.  plan: (cached, dropped, new); append: (past, new); delta: (tokens, fresh)."""
    r = random.Random(c["ragged"])
    n = c["seqs"]
    if c["op"] == "plan":
        lens = [c["len_max"]] + [r.randint(c["len_min"], c["len_max"]) for _ in range(n - 1)]
        new = [c["new_max"]] + [r.randint(c["new_min"], c["new_max"]) for _ in range(n - 1)]
        drop = [r.randint(0, min(c["reject"], a)) for a in lens]
        for s in range(1, n):
            if r.random() < c["leave"]:  # a finished request: its row stays empty or takes a new prompt
                drop[s] = lens[s]
                new[s] = r.choice([0, new[s]])
            elif c["leave"]:
                new[s] = 1
        return lens, drop, new
    if c["op"] == "append":
        new = [c["new_max"]] + [r.randint(c["new_min"], c["new_max"]) for _ in range(n - 1)]
        return [r.randint(0, c["past_max"]) for _ in range(n)], new
    q = [c["q_max"]] + [r.randint(c["q_min"], c["q_max"]) for _ in range(n - 1)]
    return q, [r.random() < c["fresh"] for _ in range(n)]


def work(c):
    if c["op"] == "plan":
        lens, drop, new = _lens(c)
        B = c["block"]
        moved = sum(abs((a - d + m + B - 1) // B - (a + B - 1) // B) for a, d, m in zip(lens, drop, new))
        touched = sum(1 for a, d, m in zip(lens, drop, new) if m and (a - d) % B)
        # lengths in, lengths and offsets out, a slot and a position a row, ids that change hands, partly filled blocks looked up
        return {"bytes": 20 * c["seqs"] + 12 * (sum(new) + c["pad"]) + 8 * moved + 4 * touched, "flops": 0}
    if c["op"] == "append":
        t = sum(_lens(c)[1])
        rows, pairs = c["heads"] + c["kv_heads"], c["rotary"] // 2
        per = 4 * c["dim"] * (c["heads"] + 2 * c["kv_heads"]) + 8 + 4 * c["axes"]
        return {"bytes": t * per, "flops": t * rows * (6 * pairs + (4 * c["dim"] if c["norm"] else 0))}
    q, fresh = _lens(c)
    t, H, K, D = sum(q), c["heads"], c["key_heads"], c["dim"]
    states = 4 * H * D * D * (2 * len(q) - sum(fresh))
    return {"bytes": t * (2 * D * (2 * K + 2 * H) + 8 * H) + states, "flops": 6 * D * D * H * t}


# ------------------------------------------------------------------------------------------------ inputs
def prepare(c, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    st = {"case": c}
    {"plan": _prepare_plan, "append": _prepare_append, "delta": _prepare_delta}[c["op"]](st, c, gen, random.Random(seed))
    if own:
        {"plan": _own_plan, "append": _own_append, "delta": _own_delta}[c["op"]](st, c)
    return st


def _ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


def _prepare_plan(st, c, gen, rng):
    lens, drop, new = _lens(c)
    B, S = c["block"], c["seqs"]
    had = [(n + B - 1) // B for n in lens]
    want = [(a - d + m + B - 1) // B for a, d, m in zip(lens, drop, new)]
    take = sum(max(0, b - a) for a, b in zip(had, want))
    spare = take + 1 + c["ragged"] % 50
    n_blocks = sum(had) + spare + c["ragged"] % 9
    ids = np.random.default_rng(rng.randrange(1 << 62)).permutation(n_blocks).astype(np.int32)
    width = max(max(had), max(want)) + 1
    table = np.full((S, width), -1, np.int32)
    at = 0
    for s, k in enumerate(had):
        table[s, :k] = ids[at:at + k]
        at += k
    head = rng.randrange(n_blocks)  # the ring of free blocks begins anywhere
    ring = np.full(n_blocks, -1, np.int32)
    ring[(head + np.arange(spare)) % n_blocks] = ids[at:at + spare]
    rows = sum(new) + c["pad"]
    st.update(n_blocks=n_blocks, rows=rows, lens=_ints(lens), drop=_ints(drop), new=_ints(new), table=torch.from_numpy(table).cuda(),
              ring=torch.from_numpy(ring).cuda(), ring_state=_ints([head, spare]), ring_state_out=_ints([0, 0]),
              lens_out=_ints([0] * S), cu=_ints([0] * (S + 1)), slots=torch.zeros(rows, dtype=torch.int64, device="cuda"),
              positions=torch.zeros(rows, dtype=torch.int32, device="cuda"))


def _prepare_append(st, c, gen, rng):
    past, new = _lens(c)
    H, C, D, B, R, dt = c["heads"], c["kv_heads"], c["dim"], c["block"], c["rotary"], DT[c["dtype"]]
    T = sum(new) + c["pad"]
    blocks = [(p + n + B - 1) // B - p // B for p, n in zip(past, new)]
    ids = np.random.default_rng(rng.randrange(1 << 62)).permutation(sum(blocks) + 5)
    slots, where, at = [], [], 0
    for p, n, k in zip(past, new, blocks):
        pos = np.arange(p, p + n)
        slots.append(ids[at:at + k][pos // B - p // B] * B + pos % B)
        where.append(pos)
        at += k
    slots.append(np.full(c["pad"], -1))
    where = np.concatenate(where + [np.zeros(c["pad"], np.int64)])
    st["slots"] = torch.from_numpy(np.concatenate(slots).astype(np.int64)).cuda()
    if c["axes"] == 1:
        pos = where[None]
    else:  # frames of 24 x 32 patches, time, height and width
        pos = np.stack([where // 768, where // 32 % 24, where % 32])
    st["positions"] = torch.from_numpy(np.ascontiguousarray(pos).astype(np.int32)).cuda()
    st["rows"] = _ints([sum(new)])
    base = 10000.0 if c["past_max"] < 100000 else 1000000.0
    st["freq"] = torch.tensor([base ** (-2.0 * j / R) for j in range(R // 2)], dtype=torch.float64).float().cuda()
    st["axis"] = torch.tensor([j % 3 for j in range(R // 2)], dtype=torch.uint8, device="cuda") if c["axes"] > 1 else None
    # projections leave q, k and v side by side, one row a token
    qkv = torch.empty((T, (H + 2 * C) * D), dtype=dt, device="cuda")
    qkv.copy_(torch.randn(qkv.shape, device="cuda", generator=gen) * 2.0)
    st["q"], st["k"], st["v"] = (x.view(T, -1, D) for x in qkv.split([H * D, C * D, C * D], 1))
    st["q_out"] = torch.zeros((T, H, D), dtype=dt, device="cuda")
    for name in ("q_weight", "k_weight"):
        w = 1.0 - c["offset"] + 0.2 * torch.randn(D, device="cuda", generator=gen)
        st[name] = w.to(dt if c["weights"] == "bf16" else torch.float32) if c["norm"] else None
    shape = (sum(blocks) + 5, B, C, D) if c["order"] == "token" else (sum(blocks) + 5, C, B, D)
    st["pool"] = torch.zeros((2,) + shape, dtype=dt, device="cuda")


def _prepare_delta(st, c, gen, rng):
    q_lens, fresh = _lens(c)
    H, K, D, S, dt = c["heads"], c["key_heads"], c["dim"], c["seqs"], DT[c["dtype"]]
    T = sum(q_lens)
    cu = [0]
    for n in q_lens:
        cu.append(cu[-1] + n)
    st.update(q_lens=q_lens, fresh=fresh, cu_h=cu, cu=_ints(cu), past=_ints([0 if f else 100 for f in fresh]))

    def randn(*shape):
        return torch.randn(shape, device="cuda", generator=gen)

    qkv = torch.empty((T, (2 * K + H) * D), dtype=dt, device="cuda")
    qkv.copy_(randn(*qkv.shape))
    if not c["unit"]:  # the caller has made keys and queries unit vectors
        x = qkv[:, :2 * K * D].float().view(T, 2 * K, D)
        qkv[:, :2 * K * D] = (x / x.norm(dim=-1, keepdim=True)).view(T, -1).to(dt)
    st["q"], st["k"], st["v"] = (x.view(T, -1, D) for x in qkv.split([K * D, K * D, H * D], 1))
    # gates as models make them: -exp(a) softplus(x), strengths through a sigmoid
    st["g"] = -c["decay"] * torch.rand((H,), device="cuda", generator=gen) * torch.nn.functional.softplus(randn(T, H) - 2.0)
    st["beta"] = torch.sigmoid(randn(T, H))
    st["out"] = torch.zeros((T, H, D), dtype=dt, device="cuda")
    st["scale"] = 1.0 / math.sqrt(D)
    # two heads of 128 (eight of 64) a block of 128 KiB; states come from the first blocks and go to as many others
    per = 131072 // (4 * D * D)
    n = (H + per - 1) // per
    ids = list(range(S * n + 3))
    rng.shuffle(ids)
    st["src_h"] = [[ids.pop() for _ in range(n)] for _ in range(S)]
    st["n_src"] = S * n + 3
    st["dst_h"] = [[st["n_src"] + s * n + j for j in range(n)] for s in range(S)]
    st["src"], st["dst"] = _ints(st["src_h"]), _ints(st["dst_h"])
    st["pool"] = torch.zeros((st["n_src"] + S * n, per, D, D), device="cuda")
    st["pool"][:st["n_src"]] = randn(st["n_src"], per, D, D) * 0.3


def _own_plan(st, c):
    from paper_2609_25451_b200 import gms

    st["args"] = gms.kv_plan_args(n_blocks=st["n_blocks"], block_tokens=c["block"], lens=st["lens"], new_lens=st["new"],
                                  drop_lens=st["drop"], block_table=st["table"], free_ids=st["ring"],
                                  free_state=st["ring_state"], free_state_out=st["ring_state_out"], lens_out=st["lens_out"],
                                  cu_q=st["cu"], slots=st["slots"], positions=st["positions"])


def _own_append(st, c):
    from paper_2609_25451_b200 import gms

    pool, C, D, B = st["pool"], c["kv_heads"], c["dim"], c["block"]
    st["desc"] = gms.KvPool(base=pool.data_ptr(), plane_stride=pool.stride(0) * 2, block_stride=pool.stride(1) * 2, n_planes=2,
                            n_blocks=pool.shape[1], block_bytes=B * C * D * 2)
    tok, head = (C * D * 2, D * 2) if c["order"] == "token" else (D * 2, B * D * 2)
    st["layout"] = gms.KvLayout(k_plane=0, v_plane=1, n_kv_heads=C, head_dim=D, block_tokens=B,
                                dtype=gms.DTYPE_BF16 if c["dtype"] == "bf16" else gms.DTYPE_F16, token_stride=tok, head_stride=head)
    st["args"] = gms.kv_append_args(q=st["q"], k=st["k"], v=st["v"], q_out=st["q_out"], slots=st["slots"], n_rows=st["rows"],
                                    positions=st["positions"], inv_freq=st["freq"], axes=st["axis"],
                                    pairs=gms.PAIR_HALVES if c["pairs"] == "halves" else gms.PAIR_NEIGHBOURS,
                                    q_weight=st["q_weight"], k_weight=st["k_weight"], weight_offset=c["offset"], eps=1e-6)


def _own_delta(st, c):
    from paper_2609_25451_b200 import gms

    pool = st["pool"]
    st["desc"] = gms.KvPool(base=pool.data_ptr(), plane_stride=0, block_stride=131072, n_planes=1, n_blocks=pool.shape[0], block_bytes=131072)
    st["state"] = gms.KvState(plane=0, n_heads=c["heads"], head_dim=c["dim"])
    one_each = all(n == 1 for n in st["q_lens"])
    st["args"] = gms.kv_delta_args(q=st["q"], k=st["k"], v=st["v"], g=st["g"], beta=st["beta"], out=st["out"],
                                   cu_q=None if one_each else st["cu"], max_q=max(st["q_lens"]), past_lens=st["past"], src_table=st["src"],
                                   dst_table=st["dst"], scale=st["scale"], unit_eps=1e-6 if c["unit"] else None)
    nbytes = gms.gms_kv_delta_workspace(st["desc"], st["state"], st["args"])
    st["ws"] = torch.empty(max(nbytes, 16), dtype=torch.uint8, device="cuda")
    st["args"].set_workspace(st["ws"])


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    op = st["case"]["op"]
    if own:
        from paper_2609_25451_b200 import gms

        if op == "plan":
            gms.gms_kv_plan(st["args"])
        elif op == "append":
            gms.gms_kv_append(st["desc"], st["layout"], st["args"])
        else:
            gms.gms_kv_delta(st["desc"], st["state"], st["args"])
    else:
        {"plan": _plain_plan, "append": _plain_append, "delta": _plain_delta}[op](st)
    if op == "plan":
        return {k: st[k] for k in ("cu", "slots", "positions", "lens_out", "table", "ring", "ring_state_out")}
    if op == "append":
        return {"q": st["q_out"], "pool": st["pool"]}
    return {"out": st["out"], "states": st["pool"][st["n_src"]:]}


def _plain_plan(st):
    B, dev = st["case"]["block"], st["lens"].device
    lens, drop, new, table, ring = (st[k].long() for k in ("lens", "drop", "new", "table", "ring"))
    S, width, cap, rows = lens.numel(), table.shape[1], ring.numel(), st["rows"]
    head, count = st["ring_state"].long()
    base = (lens - drop).clamp(min=0)
    out = base + new
    cu = torch.zeros(S + 1, dtype=torch.long, device=dev)
    cu[1:] = new.cumsum(0)
    had, want = (lens + B - 1) // B, (out + B - 1) // B
    more = (want - had).clamp(min=0)
    rank = more.cumsum(0) - more
    col = torch.arange(width, device=dev)[None, :]
    fresh = (col >= had[:, None]) & (col < want[:, None])
    r = (rank - had)[:, None] + col
    ids = torch.where(r < count, ring[(head + r.clamp(min=0)) % cap], -1)
    freed = (col >= want[:, None]) & (col < had[:, None]) & (table >= 0) & (table < st["n_blocks"])
    back = torch.where(freed, freed.flatten().cumsum(0).view(S, width) - 1, 0)
    at = torch.where(freed, (head + count + back) % cap, cap)
    st["ring"].copy_(torch.cat([ring, ring[:1]]).scatter(0, at.flatten(), table.flatten())[:cap])
    table = torch.where(fresh, ids, table)
    st["table"].copy_(table)
    used = torch.minimum(more.sum(), count)
    st["ring_state_out"].copy_(torch.stack([(head + used) % cap, count - used + freed.sum()]))
    i = torch.arange(rows, device=dev)
    s = (i[:, None] >= cu[None, 1:]).sum(1) if S <= 64 else torch.searchsorted(cu[1:].contiguous(), i, right=True)
    live = s < S
    s = s.clamp(max=S - 1)
    pos = base[s] + i - cu[s]
    block = table[s, (pos // B).clamp(max=width - 1)]
    ok = live & (block >= 0) & (block < st["n_blocks"])
    st["slots"].copy_(torch.where(ok, block * B + pos % B, -1))
    st["positions"].copy_(torch.where(live, pos, 0))
    st["cu"].copy_(cu)
    st["lens_out"].copy_(out)


def _plain_append(st):
    c = st["case"]
    B, R = c["block"], c["rotary"]
    T = int(sum(_lens(c)[1]))
    where = st["positions"][:, :T].double()
    axis = st["axis"].long() if st["axis"] is not None else torch.zeros(R // 2, dtype=torch.long, device=where.device)
    angle = where[axis].T * st["freq"].double()  # far positions: 64 bits
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def turned(x, w):
        x = x[:T].float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * (w.float() + c["offset"])
        y = x.clone()
        if c["pairs"] == "halves":
            a, b = x[..., :R // 2], x[..., R // 2:R]
            y[..., :R // 2], y[..., R // 2:R] = a * cos - b * sin, b * cos + a * sin
        else:
            a, b = x[..., 0:R:2], x[..., 1:R:2]
            y[..., 0:R:2], y[..., 1:R:2] = a * cos - b * sin, b * cos + a * sin
        return y

    st["q_out"][:T] = turned(st["q"], st["q_weight"]).to(st["q_out"].dtype)
    block, at = st["slots"][:T] // B, st["slots"][:T] % B
    for plane, x in ((0, turned(st["k"], st["k_weight"]).to(st["pool"].dtype)), (1, st["v"][:T])):
        if c["order"] == "token":
            st["pool"][plane, block, at] = x
        else:
            st["pool"][plane, block, :, at] = x


def _plain_delta(st):
    """Token by token, all sequences that still have one at once (the longest first, so that they are a leading slice)."""
    c = st["case"]
    H, K, D, S = c["heads"], c["key_heads"], c["dim"], c["seqs"]
    order = sorted(range(S), key=lambda s: -st["q_lens"][s])
    dev = st["q"].device
    src = torch.tensor([st["src_h"][s] for s in order], device=dev)
    state = st["pool"][src].reshape(S, -1, D, D)[:, :H].contiguous()  # [sequence, head, key, value]
    state[torch.tensor([st["fresh"][s] for s in order], device=dev)] = 0.0
    q, k, v = (st[x].float() for x in "qkv")
    if c["unit"]:
        q = q * torch.rsqrt((q * q).sum(-1, keepdim=True) + 1e-6)
        k = k * torch.rsqrt((k * k).sum(-1, keepdim=True) + 1e-6)
    q = q.repeat_interleave(H // K, 1) * st["scale"]
    k = k.repeat_interleave(H // K, 1)
    gate = torch.exp(st["g"])
    first = torch.tensor([st["cu_h"][s] for s in order], device=dev)
    n = S
    for t in range(c["q_max"]):
        while st["q_lens"][order[n - 1]] <= t:
            n -= 1
        row = first[:n] + t
        s = state[:n]
        kt = k[row]
        s *= gate[row][:, :, None, None]
        d = (v[row] - torch.matmul(kt[:, :, None, :], s).squeeze(2)) * st["beta"][row][:, :, None]
        s += kt[:, :, :, None] * d[:, :, None, :]
        st["out"][row] = torch.matmul(q[row][:, :, None, :], s).squeeze(2).to(st["out"].dtype)
    dst = torch.tensor([st["dst_h"][s] for s in order], device=dev)
    per = st["pool"].shape[1]
    if dst.shape[1] * per != H:  # the last block of a sequence is not full
        state = torch.cat([state, state.new_zeros(S, dst.shape[1] * per - H, D, D)], 1)
    st["pool"][dst] = state.view(S, dst.shape[1], per, D, D)


# ------------------------------------------------------------------------------------------------ 64-bit values
def exact(c, seed):
    """From the definitions, in 64 bits, from the same inputs."""
    global own
    was, own = own, False
    try:
        st = prepare(c, seed)
    finally:
        own = was
    return {"plan": _exact_plan, "append": _exact_append, "delta": _exact_delta}[c["op"]](st)


def _exact_plan(st):
    """Sequence by sequence and row by row, on the host."""
    B, n_blocks = st["case"]["block"], st["n_blocks"]
    lens, drop, new, table, ring = (st[k].tolist() for k in ("lens", "drop", "new", "table", "ring"))
    head, count = st["ring_state"].tolist()
    cap = len(ring)
    free = [ring[(head + i) % cap] for i in range(count)]
    taken, back, cu, lens_out, slots, positions = 0, [], [0], [], [], []
    for s, row in enumerate(table):
        base = max(lens[s] - drop[s], 0)
        lens_out.append(base + new[s])
        cu.append(cu[-1] + new[s])
        had, want = -(-lens[s] // B), -(-lens_out[s] // B)
        for b in range(had, want):
            row[b] = free[taken] if taken < count else -1
            taken += 1
        back += [i for i in row[want:had] if 0 <= i < n_blocks]
        for p in range(base, base + new[s]):
            i = row[p // B]
            slots.append(i * B + p % B if 0 <= i < n_blocks else -1)
            positions.append(p)
    for i, b in enumerate(back):
        ring[(head + count + i) % cap] = b
    taken = min(taken, count)
    pad = st["rows"] - len(slots)
    return {"cu": _ints(cu), "slots": _ints(slots + [-1] * pad, torch.int64), "positions": _ints(positions + [0] * pad),
            "lens_out": _ints(lens_out), "table": _ints(table), "ring": _ints(ring),
            "ring_state_out": _ints([(head + taken) % cap, count - taken + len(back)])}


def _exact_append(st):
    """Pairs as complex numbers."""
    c = st["case"]
    R, B, D = c["rotary"], c["block"], c["dim"]
    T = sum(_lens(c)[1])
    pos = st["positions"].double()[:, :T]
    axis = [j % 3 if c["axes"] > 1 else 0 for j in range(R // 2)]
    turn = torch.polar(torch.ones(T, R // 2, dtype=torch.float64, device=pos.device),
                       torch.stack([pos[axis[j]] * st["freq"][j].double() for j in range(R // 2)], 1))
    pair = np.arange(R).reshape(2, R // 2).T if c["pairs"] == "halves" else np.arange(R).reshape(R // 2, 2)
    pair = torch.from_numpy(pair.copy()).to(pos.device)

    def turned(x, w):
        y = x[:T].double()
        if w is not None:
            y = y / ((y ** 2).sum(-1, keepdim=True) / D + 1e-6).sqrt() * (w.double() + c["offset"])
        z = torch.view_as_complex(y[:, :, pair].contiguous()) * turn[:, None]
        y[:, :, pair] = torch.view_as_real(z)
        return y

    q = torch.zeros(st["q_out"].shape, dtype=torch.float64, device=pos.device)
    q[:T] = turned(st["q"], st["q_weight"])
    pool = torch.zeros(st["pool"].shape, dtype=torch.float64, device=pos.device)
    flat = pool if c["order"] == "token" else pool.transpose(2, 3)  # [plane, block, token, head, dim]
    slot = st["slots"][:T]
    flat[0, slot // B, slot % B] = turned(st["k"], st["k_weight"])
    flat[1, slot // B, slot % B] = st["v"][:T].double()
    return {"q": q, "pool": pool}


def _exact_delta(st):
    """Runs of up to 32 tokens: what they add to a state solves a triangular system."""
    c = st["case"]
    H, K, D = c["heads"], c["key_heads"], c["dim"]
    per = st["pool"].shape[1]
    states = torch.zeros(st["pool"][st["n_src"]:].shape, dtype=torch.float64, device="cuda")
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    for s, n in enumerate(st["q_lens"]):
        r0 = st["cu_h"][s]
        heads = [j // (H // K) for j in range(H)]
        q, k = (st[x][r0:r0 + n].double()[:, heads].transpose(0, 1) for x in "qk")  # [head, token, dim]
        v, g, b = (st[x][r0:r0 + n].double().transpose(0, 1) for x in ("v", "g", "beta"))
        if c["unit"]:
            q, k = (x / ((x ** 2).sum(-1, keepdim=True) + 1e-6).sqrt() for x in (q, k))
        blocks = torch.tensor(st["src_h"][s], device="cuda")
        S = st["pool"][blocks].double().reshape(-1, D, D)[:H]
        if st["fresh"][s]:
            S = torch.zeros_like(S)
        for i in range(0, n, 32):
            qi, ki, vi, gi, bi = (x[:, i:i + 32] for x in (q, k, v, g, b))
            m = qi.shape[1]
            G = gi.cumsum(1)
            lower = torch.ones(m, m, dtype=torch.bool, device="cuda").tril()
            decay = torch.exp(torch.where(lower, G[:, :, None] - G[:, None, :], -math.inf))
            A = torch.eye(m, dtype=torch.float64, device="cuda") + bi[:, :, None] * torch.tril(ki @ ki.mT * decay, -1)
            rhs = bi[:, :, None] * (vi - G.exp()[:, :, None] * (ki @ S))
            d = torch.linalg.solve_triangular(A, rhs, upper=False, unitriangular=True)
            out[r0 + i:r0 + i + m] = (st["scale"] * (G.exp()[:, :, None] * (qi @ S) + (qi @ ki.mT * decay) @ d)).transpose(0, 1)
            last = G[:, -1:]
            S = last.exp()[:, :, None] * S + (ki * torch.exp(last - G)[:, :, None]).mT @ d
        dst = torch.tensor(st["dst_h"][s], device="cuda") - st["n_src"]
        full = torch.zeros((len(dst) * per, D, D), dtype=torch.float64, device="cuda")
        full[:H] = S
        states[dst] = full.view(len(dst), per, D, D)
    return {"out": out, "states": states}
