"""Steps of an engine with attention layers and recurrent layers on state that outlives it.

    python examples/kv_step.py [--layers 4] [--requests 6] [--steps 12]

Layers take turns: attention over paged keys and values, and the gated delta rule, whose states lie in blocks of a pool of their own.
A step is: which blocks and slots its tokens go to (gms_kv_plan), then layer by layer either queries and keys normed and rotated, keys
and values into the pool (gms_kv_append) and attention over all of it (gms_kv_attention), or the recurrent rule (gms_kv_delta).

  1. prompts of different lengths in one step, then tokens one by one, that step captured into a CUDA graph and replayed: lengths and
     the ring of free blocks are on the device and go on by themselves;
  2. a request leaves and another takes its place: the same calls, without the graph;
  3. the engine goes down: the blocks in use of both pools are captured with digests, lost, restored and checked where they lie;
  4. decoding goes on.  The outputs are those, bit for bit, of a run to which nothing happened.

There is no model behind it: weights are random.
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


class Engine:
    def __init__(self, layers, requests, heads, kv_heads, room):
        g = torch.Generator(device="cuda")
        g.manual_seed(7)
        self.layers, self.n, self.H, self.C, self.room = layers, requests, heads, kv_heads, room
        self.hidden, self.gates = 256, (2 * heads + 7) // 8 * 8  # (rows of projections keep to 16 bytes)
        bf16 = torch.bfloat16

        def weight(i, o):
            return (torch.randn((i, o), device="cuda", generator=g) / math.sqrt(i)).to(bf16)

        self.w_in = [weight(self.hidden, (heads + 2 * kv_heads) * DIM if self.attends(l) else 3 * heads * DIM + self.gates) for l in range(layers)]
        self.w_out = [weight(heads * DIM, self.hidden) for _ in range(layers)]
        self.norms = [torch.ones(DIM, dtype=bf16, device="cuda") + 0.1 * torch.randn(DIM, device="cuda", generator=g).to(bf16) for _ in range(2 * layers)]
        self.inv_freq = torch.tensor([10000.0 ** (-2.0 * j / DIM) for j in range(DIM // 2)], dtype=torch.float32, device="cuda")
        n_attn, n_rec = (layers + 1) // 2, layers // 2
        # keys and values: a plane each an attention layer; states: a plane a recurrent layer, two heads a block of 128 KiB
        per_seq = room // BLOCK
        self.n_blocks, bb = requests * per_seq, BLOCK * kv_heads * DIM * 2
        self.pool = torch.zeros((2 * n_attn, self.n_blocks, BLOCK, kv_heads, DIM), dtype=bf16, device="cuda")
        self.kv = gms.KvPool(base=self.pool.data_ptr(), plane_stride=self.n_blocks * bb, block_stride=bb, n_planes=2 * n_attn, n_blocks=self.n_blocks,
                             block_bytes=bb)
        self.s_blocks = requests * ((heads + 1) // 2)
        self.states = torch.zeros((max(n_rec, 1), self.s_blocks, 2, DIM, DIM), device="cuda")
        self.rec = gms.KvPool(base=self.states.data_ptr(), plane_stride=self.s_blocks * 131072, block_stride=131072, n_planes=max(n_rec, 1),
                              n_blocks=self.s_blocks, block_bytes=131072)
        self.state_table = torch.randperm(self.s_blocks, device="cuda", generator=g).to(torch.int32).view(requests, -1)
        # the books: lengths, block tables, the ring of free blocks
        self.lens = int32([0] * requests)
        self.table = torch.full((requests, per_seq), -1, dtype=torch.int32, device="cuda")
        self.free = torch.randperm(self.n_blocks, device="cuda", generator=g).to(torch.int32)
        self.free_state = int32([0, self.n_blocks])
        self.status = torch.zeros(1, dtype=torch.int64, device="cuda")

    def attends(self, layer):
        return layer % 2 == 0

    def buffers(self, rows, max_q):
        """What a step of so many rows works in; made once for a graph."""
        b = {"x": torch.zeros((rows, self.hidden), dtype=torch.bfloat16, device="cuda"), "new": int32([0] * self.n), "drop": int32([0] * self.n),
             "cu": int32([0] * (self.n + 1)), "slots": torch.zeros(rows, dtype=torch.int64, device="cuda"), "positions": int32([0] * rows), "max_q": max_q,
             "q": torch.zeros((rows, self.H, DIM), dtype=torch.bfloat16, device="cuda"),
             "out": torch.zeros((rows, self.H, DIM), dtype=torch.bfloat16, device="cuda")}
        b["ws"] = None
        return b

    def step(self, b):
        rows, H, C = b["x"].shape[0], self.H, self.C
        gms.gms_kv_plan(gms.kv_plan_args(n_blocks=self.n_blocks, block_tokens=BLOCK, lens=self.lens, new_lens=b["new"], drop_lens=b["drop"],
                                         block_table=self.table, free_ids=self.free, free_state=self.free_state, cu_q=b["cu"], slots=b["slots"],
                                         positions=b["positions"], status=self.status))
        past = self.lens - b["new"]  # (the plan has counted the new tokens already)
        live = b["cu"][self.n:]
        x = b["x"]
        for l in range(self.layers):
            y = x @ self.w_in[l]
            if self.attends(l):
                q, k, v = (t.view(rows, -1, DIM) for t in y.split([H * DIM, C * DIM, C * DIM], 1))
                layout = gms.KvLayout(k_plane=l, v_plane=l + 1, n_kv_heads=C, head_dim=DIM, block_tokens=BLOCK, dtype=gms.DTYPE_BF16,
                                      token_stride=C * DIM * 2, head_stride=DIM * 2)
                gms.gms_kv_append(self.kv, layout, gms.kv_append_args(q=q, k=k, v=v, q_out=b["q"], slots=b["slots"], n_rows=live, positions=b["positions"],
                                                                      inv_freq=self.inv_freq, q_weight=self.norms[2 * l], k_weight=self.norms[2 * l + 1]))
                a = gms.kv_attn(q=b["q"], out=b["out"], cu_q=b["cu"], kv_lens=self.lens, block_table=self.table, max_q=b["max_q"], max_kv=self.room,
                                scale=DIM ** -0.5)
                need = gms.gms_kv_attention_workspace(self.kv, layout, a)
                call = lambda: gms.gms_kv_attention(self.kv, layout, a)  # noqa: E731
            else:
                q, k, v = (t.view(rows, H, DIM) for t in y[:, :3 * H * DIM].split([H * DIM] * 3, 1))
                gates = y[:, 3 * H * DIM:].float()
                g, beta = -torch.nn.functional.softplus(gates[:, :H]), torch.sigmoid(gates[:, H:2 * H])
                state = gms.KvState(plane=l // 2, n_heads=H, head_dim=DIM)
                a = gms.kv_delta_args(q=q, k=k, v=v, g=g, beta=beta, out=b["out"], cu_q=b["cu"], max_q=b["max_q"], past_lens=past,
                                      src_table=self.state_table, scale=DIM ** -0.5, unit_eps=1e-6)
                need = gms.gms_kv_delta_workspace(self.rec, state, a)
                call = lambda: gms.gms_kv_delta(self.rec, state, a)  # noqa: E731
            if b["ws"] is None or b["ws"].numel() < need:
                b["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
            a.set_workspace(b["ws"])
            call()
            x = x + b["out"].view(rows, -1) @ self.w_out[l]
        return x

    def lose_and_restore(self):
        """Both pools through a packed image: captured with digests, wiped, put back, checked in place; how many blocks there were."""
        count = 0
        tables = self.table.cpu()
        used = [int(i) for s, n in enumerate(self.lens.tolist()) for i in tables[s, :(n + BLOCK - 1) // BLOCK]]
        for pool, memory, ids in ((self.kv, self.pool, int32(used)), (self.rec, self.states, self.state_table.flatten().contiguous())):
            n, bb, planes = len(ids), pool.block_bytes, pool.n_planes
            image = torch.empty((planes, n, bb), dtype=torch.uint8, device="cuda")
            before, after = (torch.zeros(n * planes * (bb // 4096), dtype=torch.int64, device="cuda") for _ in range(2))
            status = torch.zeros(4, dtype=torch.int64, device="cuda")
            gms.gms_kv_capture(pool, image, n * bb, bb, gms.SRC_DEVICE, ids, n, before, None, status)
            memory.fill_(float("nan"))
            gms.gms_kv_restore(pool, image, n * bb, bb, gms.SRC_DEVICE, ids, n, None, None, status)
            gms.gms_kv_digest(pool, ids, n, after, None, status)
            bad = torch.ones(1, dtype=torch.int64, device="cuda")
            scratch = torch.zeros(gms.kv_verify_scratch_words(before.numel()), dtype=torch.int32, device="cuda")
            gms.gms_kv_verify(pool, ids, n, after, before, None, 0, bad, scratch)
            assert int(bad) == 0
            count += n * planes
        return count


def run(interrupt, layers, requests, steps, heads, kv_heads, say):
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    prompts = [3 + 41 * s % 97 for s in range(requests)]
    e = Engine(layers, requests, heads, kv_heads, room=((max(prompts) + 40 + steps + BLOCK - 1) // BLOCK) * BLOCK)
    outputs = []

    def tokens(b, new, drop=None):
        b["x"].copy_(torch.randn(b["x"].shape, device="cuda", generator=g))
        b["new"].copy_(int32(new))
        b["drop"].copy_(int32(drop or [0] * requests))

    # 1. prompts, then tokens one by one
    b = e.buffers(sum(prompts) + 5, max(prompts))  # five rows of padding
    tokens(b, prompts)
    outputs.append(e.step(b)[:sum(prompts)].clone())
    d = e.buffers(requests, 1)
    tokens(d, [1] * requests)
    state = [t.clone() for t in (e.lens, e.table, e.free, e.free_state, e.pool, e.states)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # once before it is captured, then everything back as it was
        e.step(d)
    torch.cuda.current_stream().wait_stream(side)
    for t, was in zip((e.lens, e.table, e.free, e.free_state, e.pool, e.states), state):
        t.copy_(was)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        last = e.step(d)

    def decode(count):
        for _ in range(count):
            tokens(d, [1] * requests)
            graph.replay()
            outputs.append(last.clone())

    decode(steps // 2)
    # 2. the first request leaves, another with a prompt of its own takes its row; the others go on
    lens = e.lens.tolist()
    new = [29] + [1] * (requests - 1)
    b = e.buffers(sum(new), max(new))
    tokens(b, new, [lens[0]] + [0] * (requests - 1))
    outputs.append(e.step(b).clone())
    # 3. the engine goes down
    if interrupt:
        n = e.lose_and_restore()
        say(f"{n} blocks of keys, values and states restored and verified")
    # 4. and on
    decode(steps - steps // 2)
    assert int(e.status) == 0
    assert e.lens.tolist() == [29 + steps - steps // 2] + [p + steps + 1 for p in prompts[1:]]
    assert int(e.free_state[1]) == e.n_blocks - sum((n + BLOCK - 1) // BLOCK for n in e.lens.tolist())
    return outputs


def main(layers=4, requests=6, steps=12, heads=4, kv_heads=2, quiet=False):
    say = (lambda *a: None) if quiet else print
    with_failure = run(True, layers, requests, steps, heads, kv_heads, say)
    without = run(False, layers, requests, steps, heads, kv_heads, say)
    assert all(torch.isfinite(x.float()).all() for x in without)
    same = sum(torch.equal(x, y) for x, y in zip(with_failure, without))
    say(f"{same} of {len(without)} steps are bit for bit those of a run without the failure")
    assert same == len(without)
    return same


if __name__ == "__main__":
    p = argparse.ArgumentParser()
    for name, default in (("layers", 4), ("requests", 6), ("steps", 12)):
        p.add_argument(f"--{name}", type=int, default=default)
    main(**vars(p.parse_args()))
