"""KV state of a small batch through an engine failure and on: capture, restore, verify, then serve from the pool.

    python examples/kv_serving.py [--layers 4] [--sequences 6] [--prompt 700] [--steps 5]

One pool of paged KV blocks (16 tokens x kv heads x 128, bf16, a K and a V plane a layer) holds a prompt that all sequences
share and every sequence's own tokens.  The blocks in use are captured into a packed image with their digests, the pool is
lost, restored and checked in place; then the engine goes on with what lies in it:

  1. the sequences' next tokens attend to the shared prompt and to their own tokens (gms_kv_attention_shared);
  2. one sequence decodes some steps under a sliding window with sinks, adding up the attention weight of every token
     (gms_kv_attention with weights);
  3. its cache is cut down to the heaviest tokens (gms_kv_evict) and decoding goes on from fresh blocks;
  4. the blocks that it has left are captured again, next to nothing of the old ones.

The queries and keys are random (there is no model here); the printed errors compare with plain torch arithmetic.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_25451_b200 import gms  # noqa: E402

BLOCK, DIM = 16, 128


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def softmax_attention(q, k, v, scale, seen=None):
    """q [H, D], k and v [n, C, D] in 32 bits -> out [H, D], weight of each (kv head, token)."""
    H, C = q.shape[0], k.shape[1]
    x = torch.einsum("chd,tcd->cht", q.float().view(C, H // C, DIM), k.float()) * scale
    if seen is not None:
        x = x.masked_fill(~seen, -math.inf)
    p = torch.softmax(x, -1)
    return torch.einsum("cht,tcd->chd", p, v.float()).reshape(H, DIM), p.sum(1)


def main(layers=4, sequences=6, prompt=700, steps=5, heads=8, kv_heads=2, budget=256, window=128, sinks=4, quiet=False):
    torch.manual_seed(0)
    say = (lambda *a: None) if quiet else print
    n_planes, bb = 2 * layers, BLOCK * kv_heads * DIM * 2
    own = [20 + 37 * s for s in range(sequences)]                     # tokens of each sequence after the prompt
    blocks = lambda n: (n + BLOCK - 1) // BLOCK                       # noqa: E731
    n_blocks = blocks(prompt) + sum(blocks(n + steps) for n in own) + blocks(prompt + steps) + blocks(budget) + 8
    free = torch.randperm(n_blocks).tolist()
    take = lambda k: [free.pop() for _ in range(k)]                   # noqa: E731
    pool = torch.zeros((n_planes, n_blocks, BLOCK, kv_heads, DIM), dtype=torch.bfloat16, device="cuda")
    desc = gms.KvPool(base=pool.data_ptr(), plane_stride=n_blocks * bb, block_stride=bb, n_planes=n_planes, n_blocks=n_blocks, block_bytes=bb)

    def layout(layer):
        return gms.KvLayout(k_plane=2 * layer, v_plane=2 * layer + 1, n_kv_heads=kv_heads, head_dim=DIM, block_tokens=BLOCK,
                            dtype=gms.DTYPE_BF16, token_stride=kv_heads * DIM * 2, head_stride=DIM * 2)

    def fill(table, first, n):
        t = torch.arange(first, first + n, device="cuda")
        rows = torch.randn((n_planes, n, kv_heads, DIM), device="cuda").to(pool.dtype)
        pool[:, int32(table).long()[t // BLOCK], t % BLOCK] = rows

    def rows_of(plane, table, n):
        return pool[plane, int32(table[:blocks(n)]).long()].reshape(-1, kv_heads, DIM)[:n]

    prompt_table = take(blocks(prompt))
    fill(prompt_table, 0, prompt)
    tables = [take(blocks(n + steps)) for n in own]
    for t, n in zip(tables, own):
        fill(t, 0, n)
    alone = take(blocks(prompt + steps))                              # one more sequence, with a history of its own
    fill(alone, 0, prompt)

    # ---- the engine goes down: what is in use is captured with digests, lost, put back and checked where it lies
    used = prompt_table + sum((t[:blocks(n)] for t, n in zip(tables, own)), []) + alone[:blocks(prompt)]
    ids, n_sel, per = int32(used), len(used), bb // 4096
    image = torch.empty((n_planes, n_sel, bb), dtype=torch.uint8, device="cuda")
    digests = [torch.zeros(n_sel * n_planes * per, dtype=torch.int64, device="cuda") for _ in range(2)]
    status = torch.zeros(4, dtype=torch.int64, device="cuda")
    gms.gms_kv_capture(desc, image, n_sel * bb, bb, gms.SRC_DEVICE, ids, n_sel, digests[0], None, status)
    before = pool.clone()
    pool.fill_(float("nan"))
    gms.gms_kv_restore(desc, image, n_sel * bb, bb, gms.SRC_DEVICE, ids, n_sel, None, None, status)
    gms.gms_kv_digest(desc, ids, n_sel, digests[1], None, status)
    count = torch.ones(1, dtype=torch.int64, device="cuda")
    scratch = torch.zeros(gms.kv_verify_scratch_words(digests[0].numel()), dtype=torch.int32, device="cuda")
    gms.gms_kv_verify(desc, ids, n_sel, digests[1], digests[0], None, 0, count, scratch)
    assert int(count) == 0 and torch.equal(pool[:, ids.long()], before[:, ids.long()])
    say(f"{n_sel} of {n_blocks} blocks restored and verified")

    # ---- 1. every sequence's next token, behind the shared prompt, layer by layer
    scale = 1 / math.sqrt(DIM)
    width = max(len(t) for t in tables)
    table = int32([t + [-1] * (width - len(t)) for t in tables])
    q = torch.randn((layers, sequences, heads, DIM), device="cuda").to(pool.dtype)
    out, lens = torch.empty_like(q), int32(own)
    prefix = gms.kv_prefix(group_start=int32([0, sequences]), prefix_lens=int32([prompt]), prefix_table=int32([prompt_table]),
                           max_prefix=prompt, max_group_q=sequences)
    worst = 0.0
    ws = None
    for l in range(layers):
        a = gms.kv_attn(q=q[l], out=out[l], kv_lens=lens, block_table=table, max_kv=max(own), scale=scale)
        if ws is None:
            ws = torch.empty(gms.gms_kv_attention_shared_workspace(desc, layout(l), a, prefix), dtype=torch.uint8, device="cuda")
        a.set_workspace(ws)
        gms.gms_kv_attention_shared(desc, layout(l), a, prefix)
        for s in range(sequences):
            k, v = (torch.cat([rows_of(2 * l + i, prompt_table, prompt), rows_of(2 * l + i, tables[s], own[s])]) for i in (0, 1))
            worst = max(worst, float((out[l, s].float() - softmax_attention(q[l, s], k, v, scale)[0]).abs().max()))
    say(f"shared prompt of {prompt}: {sequences} sequences x {layers} layers, largest error {worst:.4f}")
    assert worst < 0.02

    # ---- 2. one sequence decodes under a window, its tokens' weights are added up
    weights = torch.zeros((layers, 1, kv_heads, prompt + steps), device="cuda")
    table1 = int32([alone])
    q1, o1 = (torch.empty((1, heads, DIM), dtype=pool.dtype, device="cuda") for _ in range(2))
    ws1, worst = None, 0.0
    for step in range(steps):
        n = prompt + step + 1
        fill(alone, n - 1, 1)                                         # the token's keys and values, as the projections leave them
        for l in range(layers):
            q1.normal_()
            a = gms.kv_attn(q=q1, out=o1, kv_lens=int32([n]), block_table=table1, max_kv=prompt + steps, window=window, sinks=sinks, scale=scale)
            w = gms.kv_weights(weights[l], weights[l])
            if ws1 is None:
                ws1 = torch.empty(gms.gms_kv_attention_workspace(desc, layout(l), a, w), dtype=torch.uint8, device="cuda")
            a.set_workspace(ws1)
            was = weights[l].clone()
            gms.gms_kv_attention(desc, layout(l), a, w)
            t = torch.arange(n, device="cuda")
            want, p = softmax_attention(q1[0], rows_of(2 * l, alone, n), rows_of(2 * l + 1, alone, n), scale, (t > n - 1 - window) | (t < sinks))
            worst = max(worst, float((o1[0].float() - want).abs().max()))
            assert torch.allclose(weights[l, 0, :, :n], was[0, :, :n] + p, atol=1e-4)
    say(f"{steps} steps under a window of {window} with {sinks} sinks, largest error {worst:.4f}")
    assert worst < 0.02

    # ---- 3. eviction to the heaviest tokens, every layer and KV head its own; decoding goes on from fresh blocks
    n = prompt + steps
    fresh = take(blocks(budget))
    kept = torch.empty((layers, 1, kv_heads, budget), dtype=torch.int32, device="cuda")
    left, new_len = torch.zeros((layers, 1, kv_heads, budget), device="cuda"), int32([0])
    gms.gms_kv_evict(desc, layout(0), gms.kv_evict_args(weights=weights, weights_out=left, lens=int32([n]), lens_out=new_len, src_table=table1,
                                                        dst_table=int32([fresh]), kept=kept, max_len=n, budget=budget, sinks=sinks, recent=32))
    assert new_len.tolist() == [budget]
    free += alone
    worst = 0.0
    for l in range(layers):
        q1.normal_()
        a = gms.kv_attn(q=q1, out=o1, kv_lens=new_len, block_table=int32([fresh]), max_kv=budget, scale=scale)
        a.set_workspace(torch.empty(gms.gms_kv_attention_workspace(desc, layout(l), a), dtype=torch.uint8, device="cuda"))
        gms.gms_kv_attention(desc, layout(l), a)
        k, v = (torch.stack([rows_of(2 * l + i, alone, n)[kept[l, 0, c].long(), c] for c in range(kv_heads)], 1) for i in (0, 1))
        worst = max(worst, float((o1[0].float() - softmax_attention(q1[0], k, v, scale)[0]).abs().max()))
    share = float(left.sum() / weights.sum())
    say(f"{n} tokens cut to {budget}, {100 * share:.1f} % of the weight kept, largest error {worst:.4f}")
    assert worst < 0.02

    # ---- 4. what is left of it, captured again
    ids, n_sel = int32(fresh), len(fresh)
    gms.gms_kv_capture(desc, image, n_sel * bb, bb, gms.SRC_DEVICE, ids, n_sel, None, None, status)
    torch.cuda.synchronize()
    assert status[:2].tolist() == [0, 0]
    say(f"captured again: {n_sel} blocks instead of {blocks(n)}")
    return share


if __name__ == "__main__":
    p = argparse.ArgumentParser()
    for name, default in (("layers", 4), ("sequences", 6), ("prompt", 700), ("steps", 5)):
        p.add_argument(f"--{name}", type=int, default=default)
    main(**vars(p.parse_args()))
