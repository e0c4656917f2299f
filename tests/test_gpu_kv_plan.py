"""gms_kv_plan against the rule written down row by row: every output exact, everything else untouched."""
import random

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2609_25451_b200 import gms  # noqa: E402

LIMIT = 1 << 30


def expected(lens, new, drop, table, ring, head, count, rows, B, n_blocks, blocks):
    """(lens_out, cu, slots, positions, table, ring, state, full)"""
    table, ring, cap = [list(r) for r in table], list(ring), len(ring)
    full, taken, back, cu, out = False, 0, [], [0], []
    slots, positions = [], []
    free = [ring[(head + i) % cap] for i in range(count)]
    for s in range(len(lens)):
        n = min(max(lens[s], 0), LIMIT)
        base = max(n - min(max(drop[s], 0), LIMIT), 0)
        m = min(max(new[s], 0), LIMIT)
        if cu[-1] + m > rows:
            full = True
            m = rows - cu[-1]
        cu.append(cu[-1] + m)
        out.append(base + m)
        had, need = min(-(-n // B), blocks), min(-(-(base + m) // B), blocks)
        for b in range(had, need):
            table[s][b] = free[taken] if taken < count else -1
            full |= taken >= count
            taken += 1
        back += [table[s][b] for b in range(need, had) if 0 <= table[s][b] < n_blocks]
        for p in range(base, base + m):
            i = table[s][p // B] if p // B < blocks else -1
            full |= p // B >= blocks
            slots.append(i * B + p % B if 0 <= i < n_blocks else -1)
            positions.append(p)
    taken = min(taken, count)
    room = cap - count
    full |= len(back) > room
    back = back[:room]
    for i, b in enumerate(back):
        ring[(head + count + i) % cap] = b
    pad = rows - len(slots)
    state = [(head + taken) % cap if cap else 0, count - taken + len(back)]
    return out, cu, slots + [-1] * pad, positions + [0] * pad, table, ring, state, full


def run(lens, new, drop=None, *, B=16, rows=None, spare=20, blocks=None, width=None, head=5, cap_extra=0, holes=(), in_place=False, seed=1,
        positions=True, short=0, stream=None, count=None, check=True):
    rng = np.random.default_rng(seed)
    S = len(lens)
    zero = [0] * S
    had = [-(-min(max(n, 0), LIMIT) // B) for n in lens]
    want = [-(-(max(n - d, 0) + m) // B) for n, d, m in zip(lens, drop or zero, [max(x, 0) for x in new])]
    blocks = max([1] + had + want) if blocks is None else blocks
    width = blocks + 2 if width is None else width
    have = sum(min(h, blocks) for h in had)
    n_blocks = have + spare
    ids = rng.permutation(n_blocks)
    table = np.full((max(S, 1), width), -9, np.int32)
    at = 0
    for s in range(S):
        k = min(had[s], blocks)
        table[s, :k] = ids[at:at + k]
        at += k
    for s, j, bad in holes:
        table[s, j] = bad
    cap = max(n_blocks + cap_extra - short, 1)
    head %= cap
    count = min(spare, cap) if count is None else count
    ring = np.full(cap, -5, np.int32)
    ring[(head + np.arange(count)) % cap] = ids[at:at + count]
    rows = sum(max(x, 0) for x in new) if rows is None else rows

    def dev(x, dtype=torch.int32):
        return torch.tensor(np.asarray(x), dtype=dtype, device="cuda")

    t = dict(lens=dev(lens).view(S), new_lens=dev(new).view(S), drop_lens=None if drop is None else dev(drop), free_ids=dev(ring),
             free_state=dev([head, count]))
    table_d = dev(table)[:S]
    guard = torch.full((rows + 2,), 777, dtype=torch.int64, device="cuda")
    guard_p = torch.full((rows + 2,), 777, dtype=torch.int32, device="cuda")
    cu = torch.full((S + 3,), 777, dtype=torch.int32, device="cuda")
    lens_out = None if in_place else torch.full((S,), 777, dtype=torch.int32, device="cuda")
    state_out = None if in_place else torch.full((2,), 777, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int64, device="cuda")
    args = gms.kv_plan_args(n_blocks=n_blocks, block_tokens=B, block_table=table_d[:, :blocks], lens_out=lens_out, free_state_out=state_out,
                            cu_q=cu[1:S + 2], slots=guard[1:rows + 1], positions=guard_p[1:rows + 1] if positions else None, status=status, **t)
    torch.cuda.synchronize()
    gms.gms_kv_plan(args, stream)
    torch.cuda.synchronize()
    if not check:
        return args, t, table_d, guard, cu, status
    e = expected(lens, new, drop or zero, table[:S].tolist(), ring.tolist(), head, count, rows, B, n_blocks, blocks)
    assert (t["lens"] if in_place else lens_out).tolist() == e[0]
    assert cu.tolist() == [777] + e[1] + [777]
    assert guard.tolist() == [777] + e[2] + [777]
    assert guard_p.tolist() == ([777] + e[3] + [777] if positions else [777] * (rows + 2))
    assert table_d.tolist() == e[4]
    assert t["free_ids"].tolist() == e[5]
    assert (t["free_state"] if in_place else state_out).tolist() == e[6]
    assert int(status) == (gms.DEV_FULL if e[7] else 0)
    if not in_place:
        assert t["lens"].tolist() == list(lens) and t["free_state"].tolist() == [head, count]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("lens,new,drop", [
    ([0], [1], None), ([16], [1], None), ([15], [1], None), ([701], [1], [0]), ([5], [0], [5]), ([5], [0], [9]), ([33], [0], [1]), ([33], [3], [2]),
    ([100, 0, 7, 64, 65], [1, 40, 0, 1, 1], [0, 0, 7, 30, 1]), ([-5, 10], [3, -2], [-1, 4]), ([40, 40], [0, 0], [40, 33])])
def test_small(lens, new, drop, in_place):
    run(lens, new, drop, in_place=in_place)


@pytest.mark.parametrize("S", [1, 3, 31, 33, 511, 513, 2047, 2049, 5000])
@pytest.mark.parametrize("B", [16, 64])
def test_many_sequences(S, B):
    r = random.Random(S * B)
    lens = [r.randint(0, 90) for _ in range(S)]
    drop = [r.choice([0, 0, r.randint(0, 90)]) for _ in range(S)]
    new = [r.choice([0, 1, 1, r.randint(0, 40)]) for _ in range(S)]
    run(lens, new, drop, B=B, spare=3 * S, rows=sum(new) + r.choice([0, 7]), in_place=S % 2 == 0, head=r.randint(0, 10**6))


@pytest.mark.parametrize("n", [1, 15, 16, 17, 4000, 8190, 30000, 100001])
def test_long_prompts(n):
    run([3, 40, 0], [n, 0, n // 3], [0, 40, 0], B=16, spare=n // 8 + 30, rows=n + n // 3 + 11)


def test_blocks_of_1024_tokens():
    run([1023, 1024, 1025, 5000], [1, 1, 2, 3000], [0, 1, 2, 0], B=1024)


@pytest.mark.parametrize("big", [1, 500])
def test_ring_runs_empty_and_wraps(big):
    lens = [20, 0, 100, 30] * big
    run(lens, [40, 17, 0, 1] * big, [0, 0, 100, 0] * big, spare=3 * big, head=10**9 + 7)
    run(lens, [40, 17, 0, 1] * big, [0, 0, 100, 0] * big, spare=3 * big, count=0)


@pytest.mark.parametrize("big", [1, 800])
def test_ring_without_room_loses_blocks(big):
    run([100, 50] * big, [0, 0] * big, [100, 50] * big, spare=4, short=6 * big)


def test_holes_do_not_come_back():
    run([100, 50], [0, 30], [90, 0], holes=[(0, 3, -1), (0, 5, 10**6), (1, 3, -7)])


@pytest.mark.parametrize("rows", [0, 1, 5, 41, 9000])
def test_rows_are_cut_off(rows):
    run([3, 30, 0], [40, 0, 10000], None, rows=rows, spare=1000)


@pytest.mark.parametrize("big", [1, 400])
def test_tokens_beyond_the_table(big):
    run([30, 100, 64] * big, [40, 2, 1] * big, [0, 0, 20] * big, blocks=4, spare=9 * big)


def test_no_sequences():
    run([], [], rows=0)
    run([], [], rows=9000)


def test_no_ring_no_positions():
    run([3, 14], [2, 2], [0, 0], spare=0, positions=False)


def test_huge_lengths_are_cut():
    n = 2**31 - 1
    args, t, table, guard, cu, status = run([5, 3], [1, 1], blocks=3, check=False)
    t["lens"].fill_(n)
    t["new_lens"].fill_(n)
    gms.gms_kv_plan(args)
    torch.cuda.synchronize()
    assert cu.tolist()[1:4] == [0, 2, 2] and int(status) == gms.DEV_FULL and guard.tolist()[1:3] == [-1, -1]


@pytest.mark.parametrize("S", [3, 3000])
def test_replayed_step_by_step_in_place(S):
    """A captured step replayed: lengths and the ring go on from step to step; another stream."""
    steps, B = 40, 16
    r = random.Random(S)
    lens = [r.randint(0, 30) for _ in range(S)]
    n_blocks = S * 6
    ids = np.random.default_rng(S).permutation(n_blocks).astype(np.int32)
    table = np.full((S, 8), -9, np.int32)
    at = 0
    for s in range(S):
        k = -(-lens[s] // B)
        table[s, :k] = ids[at:at + k]
        at += k
    cap = n_blocks
    ring = np.full(cap, -5, np.int32)
    count, head = n_blocks - at, 3
    ring[(head + np.arange(count)) % cap] = ids[at:]
    dev = {k: torch.tensor(v, dtype=torch.int32, device="cuda") for k, v in
           dict(lens=lens, new=[1] * S, drop=[0] * S, table=table, ring=ring, state=[head, count], cu=[0] * (S + 1)).items()}
    slots, positions = torch.zeros(S + 2, dtype=torch.int64, device="cuda"), torch.zeros(S + 2, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int64, device="cuda")
    args = gms.kv_plan_args(n_blocks=n_blocks, block_tokens=B, lens=dev["lens"], new_lens=dev["new"], drop_lens=dev["drop"], block_table=dev["table"],
                            free_ids=dev["ring"], free_state=dev["state"], cu_q=dev["cu"], slots=slots, positions=positions, status=status)
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        gms.gms_kv_plan(args)
    state = [head, count]
    table, ring = table.tolist(), ring.tolist()
    for step in range(steps):
        new = [r.choice([0, 1, 1, 2]) if s % 7 else 0 for s in range(S)]
        drop = [r.choice([0, 0, 1, 60 if r.random() < 0.1 else 0]) for s in range(S)]
        dev["new"].copy_(torch.tensor(new))
        dev["drop"].copy_(torch.tensor(drop))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        lens, cu, sl, po, table, ring, state, full = expected(lens, new, drop, table, ring, *state, S + 2, B, n_blocks, 8)
        assert dev["lens"].tolist() == lens and dev["table"].tolist() == table and dev["ring"].tolist() == ring and dev["state"].tolist() == state
        assert slots.tolist() == sl and positions.tolist() == po and dev["cu"].tolist() == cu
        assert int(status) == (gms.DEV_FULL if full else int(status))


@pytest.mark.parametrize("extra", [-33, -1, 0, 1, 700])
@pytest.mark.parametrize("many", [1, 4096])
def test_around_the_most_blocks_that_are_fetched_at_once(extra, many):
    """One CTA of 16 warps, or a cluster of 256 (a short sequence each): 1,024 blocks a warp."""
    most = 1024 * (16 if many == 1 else 256) + extra
    lens = [16 * (most // many)] * many
    lens[many // 2] += 16 * (most % many)
    run(lens + [20, 3], [0] * many + [1, 1], lens + [0, 0], holes=[(0, 1, -7)])
