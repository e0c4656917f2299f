"""What is measured of the operators on the paged KV pool: cases, inputs, plain forms, exact values and floors.

The operators: ``attention`` (sliding window and sinks, through a block table), ``weights`` (the same, also
accumulating each token's attention weight), ``shared`` (a batch whose sequences share long prefixes) and
``evict`` (keep the heaviest tokens, move them into fresh blocks).  With ``own`` true ``run`` makes the calls
of the library, else it computes the same in elementary 32-bit torch operations.
"""
import math
import random

import numpy as np
import torch

own = False

DT = {"bf16": torch.bfloat16, "f16": torch.float16}


# ------------------------------------------------------------------------------------------------ cases
def _case(name, op, **kw):
    c = {"name": name, "op": op, "dtype": "bf16", "heads": 32, "kv_heads": 8, "dim": 128, "block": 16, "order": "token",
         "seqs": 1, "q_max": 1, "q_min": 1, "kv_max": 1, "kv_min": 1, "window": 0, "sinks": 0, "ragged": 1}
    c.update(kw)
    return c


def listed():
    return [
        # one user's next token with a short window: a call that is all latency
        _case("window-decode-one", "attention", kv_max=701, window=256, sinks=4),
        # a serving batch's next tokens, each seeing four sinks and the last 2,048 tokens of a ragged history
        _case("window-decode-batch", "attention", seqs=48, kv_max=12001, kv_min=300, window=2048, sinks=4),
        # next tokens over long full histories on one rank of eight (8 query heads on 1 KV head)
        _case("full-decode-long", "attention", heads=8, kv_heads=1, seqs=8, kv_max=65536, kv_min=20000),
        # a whole prompt under a sliding window, fp16
        _case("window-prefill", "attention", dtype="f16", q_max=8192, q_min=8192, kv_max=8192, kv_min=8192, window=1024, sinks=4),
        # chunked prefill mixed with a decoding sequence or two: new queries over cached tokens, everything visible
        _case("chunk-full", "attention", seqs=3, q_max=2048, q_min=1, kv_max=16384, kv_min=2500),
        # three requests behind one short system prompt, on one rank of eight
        _case("shared-small", "shared", heads=8, kv_heads=1, seqs=3, kv_max=40, prefix_max=129, prefix_min=129, groups=1),
        # a batch behind one 8k prompt, suffixes of different lengths
        _case("shared-batch", "shared", seqs=64, kv_max=512, prefix_max=8192, prefix_min=8192, groups=1),
        # two long prompts (documents), many short questions each, two tokens a step (speculation), heads-first blocks of 32, fp16
        _case("shared-two-documents", "shared", dtype="f16", block=32, order="head", seqs=48, q_max=2, q_min=1, kv_max=777, kv_min=2,
              prefix_max=32768, prefix_min=20001, groups=2),
        # next tokens of a batch, with the weights that eviction goes by
        _case("weights-decode", "weights", seqs=16, kv_max=8192, kv_min=1000),
        # a prompt's last 32 queries observed over all of it, small heads
        _case("weights-observe", "weights", dim=64, q_max=32, q_min=32, kv_max=16001, kv_min=16001),
        # one layer of one short sequence
        _case("evict-one", "evict", kv_max=601, layers=1, budget=256, sinks=4, recent=64),
        # every layer of a small batch from up to 8k tokens down to 2k
        _case("evict-all-layers", "evict", seqs=4, kv_max=8192, kv_min=3000, layers=32, budget=2048, sinks=4, recent=512),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    top = [work(c) for c in listed()]
    max_bytes, max_flops = max(t["bytes"] for t in top), max(t["flops"] for t in top)
    while True:
        op = rng.choice(["attention", "attention", "shared", "weights", "evict"])
        heads, kv_heads = rng.choice([(32, 8), (8, 1), (32, 32), (16, 4), (24, 8)])
        dim, order = rng.choice([64, 128]), rng.choice(["token", "head"])
        blocks = [b for b in (16, 32, 64) if b * kv_heads * dim * 2 % 4096 == 0 and b * kv_heads * dim * 2 <= 131072]
        if not blocks:
            continue
        c = _case("", op, dtype=rng.choice(["bf16", "f16"]), heads=heads, kv_heads=kv_heads, dim=dim, order=order,
                  block=rng.choice(blocks), ragged=rng.randrange(1 << 30))
        if op == "evict":
            n = _log_int(rng, 300, 8192)
            budget = rng.randint(n // 8 + 8, n)
            c.update(seqs=_log_int(rng, 1, 8), kv_max=n, kv_min=rng.randint(1, n), layers=_log_int(rng, 1, 32), budget=budget,
                     sinks=rng.randint(0, 4), recent=rng.randint(0, budget - 4))
        elif op == "shared":
            g = rng.choice([1, 1, 2, 3])
            p = _log_int(rng, 64, 32768)
            n = _log_int(rng, 3, 1024)
            c.update(seqs=max(g, _log_int(rng, 2, 96)), groups=g, prefix_max=p, prefix_min=rng.randint(p // 2, p), kv_max=n,
                     kv_min=rng.randint(1, n), q_max=rng.choice([1, 1, 2]))
        else:
            window = rng.choice([0, _log_int(rng, 64, 4096)])
            c.update(window=window, sinks=rng.randint(0, 8) if window else 0)
            if rng.random() < 0.5:  # next tokens of a batch
                n = _log_int(rng, 100, 65536)
                c.update(seqs=_log_int(rng, 1, 64), kv_max=n, kv_min=rng.randint(1, n))
            else:  # prompts and chunks
                n = _log_int(rng, 100, 16384)
                q = _log_int(rng, 2, min(n, 64) if op == "weights" else min(n, 8192))
                c.update(seqs=_log_int(rng, 1, 4), kv_max=n, kv_min=rng.randint(1, n), q_max=q, q_min=rng.randint(1, q))
        w = work(c)
        if 4 * c.get("layers", 1) * kv_heads * dim * (c["seqs"] * c["kv_max"] + c.get("groups", 0) * c.get("prefix_max", 0)) > 6 << 30:
            continue  # a pool that would fill the card
        if w["bytes"] <= max_bytes and w["flops"] <= max_flops:
            del c["name"]
            return c


def _lens(c):
    """Query and cached lengths of every sequence (and prefix lengths): part of the case, not of the seed."""
    r = random.Random(c["ragged"])
    kv = [c["kv_max"]] + [r.randint(c["kv_min"], c["kv_max"]) for _ in range(c["seqs"] - 1)]
    q = [c["q_max"]] + [r.randint(c["q_min"], c["q_max"]) for _ in range(c["seqs"] - 1)]
    q = [min(a, b) for a, b in zip(q, kv)]
    pre = []
    if c["op"] == "shared":
        pre = [c["prefix_max"]] + [r.randint(c["prefix_min"], c["prefix_max"]) for _ in range(c["groups"] - 1)]
    return q, kv, pre


def _group_start(c):
    return [c["seqs"] * g // c["groups"] for g in range(c["groups"] + 1)]


def work(c):
    q, kv, pre = _lens(c)
    H, C, D = c["heads"], c["kv_heads"], c["dim"]
    if c["op"] == "evict":
        kept = sum(min(n, c["budget"]) for n in kv)
        rows = c["layers"] * C
        return {"bytes": rows * (4 * sum(kv) + kept * (8 + 2 * 2 * 2 * D)), "flops": 0}
    keys = pairs = 0
    for a, n in zip(q, kv):
        first = n - a
        if c["window"]:
            lo = max(0, first - c["window"] + 1)
            keys += n - lo + min(lo, c["sinks"])
            for i in range(a):
                p = first + i
                b = max(0, p - c["window"] + 1)
                pairs += p + 1 - b + min(b, c["sinks"])
        else:
            keys += n
            pairs += a * first + a * (a + 1) // 2
    if c["op"] == "shared":
        gs = _group_start(c)
        for g, p in enumerate(pre):
            keys += p
            pairs += p * sum(q[gs[g]:gs[g + 1]])
    b = keys * C * D * 2 * 2 + sum(q) * H * (D * 2 * 2 + 4)
    f = 4 * D * H * pairs
    if c["op"] == "weights":
        b += 8 * C * sum(kv)
    return {"bytes": b, "flops": f}


# ------------------------------------------------------------------------------------------------ inputs
def prepare(c, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    rng = random.Random(seed)
    q, kv, pre = _lens(c)
    H, C, D, B, dt = c["heads"], c["kv_heads"], c["dim"], c["block"], DT[c["dtype"]]
    st = {"case": c, "q_lens": q, "kv_lens": kv, "prefix_lens": pre}

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=dev)

    # block tables over a shuffled pool, a few spare blocks in it
    need = [(n + B - 1) // B for n in kv]
    pneed = [(n + B - 1) // B for n in pre]
    n_src = sum(need) + sum(pneed) + 5
    ids = list(range(n_src))
    rng.shuffle(ids)

    def table(counts):
        rows = []
        for k in counts:
            rows.append([ids.pop() for _ in range(k)] + [0] * (max(counts) - k))
        return rows

    st["table_h"] = table(need)
    st["table"] = ints(st["table_h"])
    n_blocks, layers = n_src, 1
    if c["op"] == "evict":
        layers = c["layers"]
        per = (min(c["budget"], max(kv)) + B - 1) // B
        st["dst_h"] = [[n_src + s * per + j for j in range(per)] for s in range(c["seqs"])]
        st["dst"] = ints(st["dst_h"])
        n_blocks += per * c["seqs"]
    if pre:
        st["prefix_h"] = table(pneed)
        st["prefix"] = ints(st["prefix_h"])
        st["group_h"] = _group_start(c)
        st["group_start"] = ints(st["group_h"])
        st["prefix_lens_d"] = ints(pre)
    shape = (n_blocks, B, C, D) if c["order"] == "token" else (n_blocks, C, B, D)
    pool = torch.empty((2 * layers,) + shape, dtype=dt, device=dev)
    for p in range(2 * layers):  # keys and values of unit scale
        pool[p].copy_(torch.randn(shape, dtype=torch.float32, device=dev, generator=gen))
        pool[p, n_src:].zero_()
    st["pool"], st["n_blocks"], st["n_src"] = pool, n_blocks, n_src
    st["lens"] = ints(kv)
    S = c["seqs"]
    if c["op"] == "evict":
        # accumulated weights: heavy-tailed, the newest tokens not yet attended to (equal zeros)
        w = torch.exp(2.0 * torch.randn((layers, S, C, max(kv)), device=dev, generator=gen) - 4.0)
        w[torch.rand(w.shape, device=dev, generator=gen) < 0.2] = 0.0
        st["w"] = w
        n = min(c["budget"], max(kv))
        st["w_out"] = torch.zeros((layers, S, C, n), device=dev)
        st["kept"] = torch.full((layers, S, C, n), -1, dtype=torch.int32, device=dev)
        st["lens_out"] = torch.zeros(S, dtype=torch.int32, device=dev)
    else:
        T = sum(q)
        cu = [0]
        for a in q:
            cu.append(cu[-1] + a)
        st["cu_h"], st["cu"] = cu, ints(cu)
        # queries as a projection leaves them: beside the new keys and values, one row a token
        qkv = torch.empty((T, (H + 2 * C) * D), dtype=dt, device=dev)
        qkv.copy_(torch.randn(qkv.shape, device=dev, generator=gen) * 1.5)
        st["q"] = qkv[:, :H * D].view(T, H, D)
        st["out"] = torch.zeros((T, H, D), dtype=dt, device=dev)
        st["lse"] = torch.zeros((T, H), device=dev)
        st["scale"] = 1.0 / math.sqrt(D)
        if c["op"] == "weights":
            st["w"] = torch.rand((S, C, max(kv)), device=dev, generator=gen)
            st["w_out"] = torch.zeros((S, C, max(kv)), device=dev)
            st["decay"] = 0.95
    if own:
        _prepare_own(st)
    return st


def _prepare_own(st):
    from paper_2609_25451_b200 import gms

    c, pool = st["case"], st["pool"]
    C, D, B = c["kv_heads"], c["dim"], c["block"]
    st["desc"] = gms.KvPool(base=pool.data_ptr(), plane_stride=pool.stride(0) * 2, block_stride=pool.stride(1) * 2,
                            n_planes=pool.shape[0], n_blocks=st["n_blocks"], block_bytes=B * C * D * 2)
    tok, head = (C * D * 2, D * 2) if c["order"] == "token" else (D * 2, B * D * 2)
    st["layout"] = gms.KvLayout(k_plane=0, v_plane=1, n_kv_heads=C, head_dim=D, block_tokens=B,
                                dtype=gms.DTYPE_BF16 if c["dtype"] == "bf16" else gms.DTYPE_F16, token_stride=tok, head_stride=head)
    if c["op"] == "evict":
        st["args"] = gms.kv_evict_args(weights=st["w"], weights_out=st["w_out"], lens=st["lens"], lens_out=st["lens_out"],
                                       src_table=st["table"], dst_table=st["dst"], kept=st["kept"], max_len=max(st["kv_lens"]),
                                       budget=st["kept"].shape[3], sinks=c["sinks"], recent=c["recent"], layer_planes=2)
        return
    one_each = all(a == 1 for a in st["q_lens"])
    st["args"] = gms.kv_attn(q=st["q"], out=st["out"], lse=st["lse"], cu_q=None if one_each else st["cu"], kv_lens=st["lens"],
                             block_table=st["table"], max_q=max(st["q_lens"]), max_kv=max(st["kv_lens"]), window=c["window"],
                             sinks=c["sinks"], scale=st["scale"])
    extra = None
    if c["op"] == "weights":
        extra = gms.kv_weights(st["w"], st["w_out"], decay=st["decay"])
    if c["op"] == "shared":
        extra = gms.kv_prefix(group_start=st["group_start"], prefix_lens=st["prefix_lens_d"], prefix_table=st["prefix"],
                              max_prefix=max(st["prefix_lens"]),
                              max_group_q=max(st["cu_h"][b] - st["cu_h"][a] for a, b in zip(st["group_h"], st["group_h"][1:])))
    st["extra"] = extra
    if c["op"] == "shared":
        nbytes = gms.gms_kv_attention_shared_workspace(st["desc"], st["layout"], st["args"], extra)
    else:
        nbytes = gms.gms_kv_attention_workspace(st["desc"], st["layout"], st["args"], extra)
    st["ws"] = torch.empty(max(nbytes, 16), dtype=torch.uint8, device="cuda")
    st["args"].set_workspace(st["ws"])


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    op = st["case"]["op"]
    if own:
        from paper_2609_25451_b200 import gms

        if op == "evict":
            gms.gms_kv_evict(st["desc"], st["layout"], st["args"])
        elif op == "shared":
            gms.gms_kv_attention_shared(st["desc"], st["layout"], st["args"], st["extra"])
        else:
            gms.gms_kv_attention(st["desc"], st["layout"], st["args"], st["extra"])
    elif op == "evict":
        _plain_evict(st)
    else:
        _plain_attention(st)
    if op == "evict":
        return {"kept": st["kept"], "lens": st["lens_out"], "weights": st["w_out"], "pool": st["pool"][:, st["n_src"]:]}
    out = {"out": st["out"], "lse": st["lse"]}
    if op == "weights":
        out["weights"] = st["w_out"]
    return out


def _rows(st, plane, table_row, n):
    """Tokens 0..n of one table row as [kv_heads, n, dim] in 32 bits."""
    c = st["case"]
    B = c["block"]
    x = st["pool"][plane].index_select(0, table_row[:(n + B - 1) // B])
    if c["order"] == "head":
        x = x.transpose(1, 2)
    return x.reshape(-1, c["kv_heads"], c["dim"])[:n].float().transpose(0, 1)


def _plain_attention(st):
    c = st["case"]
    H, C, D = c["heads"], c["kv_heads"], c["dim"]
    G, dev = H // C, st["pool"].device
    for s, (a, n) in enumerate(zip(st["q_lens"], st["kv_lens"])):
        K, V, pre = _rows(st, 0, st["table"][s], n), _rows(st, 1, st["table"][s], n), 0
        if c["op"] == "shared":
            g = next(i for i in range(c["groups"]) if st["group_h"][i + 1] > s)
            pre = st["prefix_lens"][g]
            K = torch.cat([_rows(st, 0, st["prefix"][g], pre), K], 1)
            V = torch.cat([_rows(st, 1, st["prefix"][g], pre), V], 1)
        if c["op"] == "weights":
            st["w_out"][s, :, :n] = st["decay"] * st["w"][s, :, :n]
        step = max(1, min(a, (1 << 27) // (H * (n + pre))))
        t = torch.arange(n + pre, device=dev)
        for i0 in range(0, a, step):
            i1 = min(a, i0 + step)
            r0 = st["cu_h"][s] + i0
            Q = st["q"][r0:r0 + i1 - i0].float().view(i1 - i0, C, G, D).permute(1, 2, 0, 3).reshape(C, G * (i1 - i0), D)
            X = torch.matmul(Q, K.transpose(1, 2)) * st["scale"]
            pos = (pre + n - a + torch.arange(i0, i1, device=dev))[:, None]
            hide = t[None, :] > pos
            if c["window"]:
                hide |= (t[None, :] <= pos - c["window"]) & (t[None, :] >= c["sinks"])
            X = X.view(C, G, i1 - i0, n + pre).masked_fill_(hide, -math.inf)
            m = X.amax(-1, keepdim=True)
            E = torch.exp_(X.sub_(m))
            l = E.sum(-1, keepdim=True)
            E /= l
            O = torch.matmul(E.view(C, G * (i1 - i0), n + pre), V).view(C, G, i1 - i0, D)
            st["out"][r0:r0 + i1 - i0] = O.permute(2, 0, 1, 3).reshape(i1 - i0, H, D).to(st["out"].dtype)
            st["lse"][r0:r0 + i1 - i0] = (m + torch.log(l)).view(C, G, i1 - i0).permute(2, 0, 1).reshape(i1 - i0, H)
            if c["op"] == "weights":
                st["w_out"][s, :, :n] += E.sum((1, 2))


def _plain_evict(st):
    c = st["case"]
    B, C, D, L = c["block"], c["kv_heads"], c["dim"], c["layers"]
    dev = st["pool"].device
    budget = st["kept"].shape[3]
    for s, n in enumerate(st["kv_lens"]):
        k = min(n, budget)
        w = st["w"][:, s, :, :n]
        if k == n:
            kept = torch.arange(n, device=dev).expand(L, C, n)
        else:
            key = w.clone()
            key[:, :, :c["sinks"]] = math.inf
            key[:, :, n - c["recent"]:] = math.inf
            kept = torch.sort(key, dim=-1, descending=True, stable=True).indices[:, :, :k].sort(-1).values
        st["kept"][:, s, :, :k] = kept.int()
        st["w_out"][:, s, :, :k] = torch.gather(w, 2, kept)
        src = st["table"][s].long()[kept // B]
        dst = st["dst"][s].long()[torch.arange(k, device=dev) // B].expand(L, C, k)
        slot, to = kept % B, (torch.arange(k, device=dev) % B).expand(L, C, k)
        h = torch.arange(C, device=dev)[None, :, None].expand(L, C, k)
        for kv in range(2):
            p = (2 * torch.arange(L, device=dev) + kv)[:, None, None].expand(L, C, k)
            if c["order"] == "token":
                st["pool"][p, dst, to, h] = st["pool"][p, src, slot, h]
            else:
                st["pool"][p, dst, h, to] = st["pool"][p, src, h, slot]
    st["lens_out"].copy_(torch.clamp(st["lens"], max=budget))


# ------------------------------------------------------------------------------------------------ 64-bit values
def exact(c, seed):
    """The definition, query by query head in 64 bits, from the same inputs."""
    global own
    was, own = own, False
    try:
        st = prepare(c, seed)
    finally:
        own = was
    if c["op"] == "evict":
        return _exact_evict(st)
    H, C, D, B = c["heads"], c["kv_heads"], c["dim"], c["block"]
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device=st["out"].device)
    lse = torch.zeros(st["lse"].shape, dtype=torch.float64, device=out.device)
    res = {"out": out, "lse": lse}
    if c["op"] == "weights":
        res["weights"] = torch.zeros(st["w_out"].shape, dtype=torch.float64, device=out.device)
    planes = st["pool"].permute(0, 1, 3, 2, 4) if c["order"] == "token" else st["pool"]  # [2, blocks, heads, tokens, dim]
    for s in range(c["seqs"]):
        a, n = st["q_lens"][s], st["kv_lens"][s]
        where = [(st["table_h"][s][j // B], j % B) for j in range(n)]
        pre = 0
        if c["op"] == "shared":
            g = max(i for i in range(c["groups"]) if st["group_h"][i] <= s)
            pre = st["prefix_lens"][g]
            where = [(st["prefix_h"][g][j // B], j % B) for j in range(pre)] + where
        at = torch.tensor(where, device=out.device)
        r0 = st["cu_h"][s]
        for h in range(H):
            kv = planes[:, at[:, 0], h * C // H, at[:, 1]].double()
            for i0 in range(0, a, 4096):
                i1 = min(a, i0 + 4096)
                z = st["scale"] * (st["q"][r0 + i0:r0 + i1, h].double() @ kv[0].T)
                p = torch.arange(n - a + i0, n - a + i1, device=out.device)[:, None]
                j = torch.arange(-pre, n, device=out.device)[None, :]
                seen = j <= p
                if c["window"]:
                    seen &= (p - j < c["window"]) | (j < c["sinks"])
                z = torch.where(seen, z, -math.inf)
                z_lse = torch.logsumexp(z, 1)
                prob = torch.exp(z - z_lse[:, None])
                out[r0 + i0:r0 + i1, h] = prob @ kv[1]
                lse[r0 + i0:r0 + i1, h] = z_lse
                if c["op"] == "weights":
                    res["weights"][s, h * C // H, :n] += prob.sum(0)
        if c["op"] == "weights":
            res["weights"][s, :, :n] += st["decay"] * st["w"][s, :, :n].double()
    return res


def _exact_evict(st):
    c = st["case"]
    B, budget = c["block"], st["kept"].shape[3]
    kept, w_out = st["kept"].cpu(), st["w_out"].double()
    pool = st["pool"]
    lens = []
    wh = st["w"].double().cpu().numpy()
    for s, n in enumerate(st["kv_lens"]):
        k = min(n, budget)
        lens.append(k)
        for l in range(c["layers"]):
            for h in range(c["kv_heads"]):
                if k < n:
                    t = np.arange(c["sinks"], n - c["recent"])
                    mid = t[np.lexsort((t, -wh[l, s, h, c["sinks"]:n - c["recent"]]))][:k - c["sinks"] - c["recent"]]
                    keep = np.concatenate([np.arange(c["sinks"]), np.sort(mid), np.arange(n - c["recent"], n)])
                else:
                    keep = np.arange(n)
                kt = torch.from_numpy(keep)
                kept[l, s, h, :k] = kt.int()
                w_out[l, s, h, :k] = st["w"][l, s, h][kt.to(pool.device)].double()
                src = torch.from_numpy(np.array(st["table_h"][s])[keep // B]).to(pool.device)
                dst = torch.from_numpy(np.array(st["dst_h"][s])[np.arange(k) // B]).to(pool.device)
                fs, ts = (kt % B).to(pool.device), (torch.arange(k) % B).to(pool.device)
                for p in (2 * l, 2 * l + 1):
                    if c["order"] == "token":
                        pool[p, dst, ts, h] = pool[p, src, fs, h]
                    else:
                        pool[p, dst, h, ts] = pool[p, src, h, fs]
    return {"kept": kept.to(pool.device), "lens": torch.tensor(lens, dtype=torch.int32, device=pool.device), "weights": w_out,
            "pool": pool[:, st["n_src"]:]}
