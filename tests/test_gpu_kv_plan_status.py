"""gms_kv_plan's status word, cleared before every replayed step: set where a step had no room for something, untouched where it had."""
import random

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2609_25451_b200 import gms  # noqa: E402
from test_gpu_kv_plan import expected  # noqa: E402


@pytest.mark.parametrize("S", [3, 3000])
@pytest.mark.parametrize("want", ["blocks", "rows", "table", "nothing"])
def test_every_step(S, want):
    steps, B, blocks = 30, 16, 8
    r = random.Random(S)
    n_blocks = max(S * 2 // 3, 2) if want == "blocks" else S * blocks
    rows = S if want == "rows" else 2 * S + 4
    lens, table, ring, state = [0] * S, [[-9] * blocks for _ in range(S)], np.random.default_rng(S).permutation(n_blocks).tolist(), [n_blocks // 3, n_blocks]
    dev = {k: torch.tensor(v, dtype=torch.int32, device="cuda") for k, v in
           dict(lens=lens, new=lens, drop=lens, table=table, ring=ring, state=state, cu=[0] * (S + 1)).items()}
    slots, status = torch.zeros(rows, dtype=torch.int64, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    args = gms.kv_plan_args(n_blocks=n_blocks, block_tokens=B, lens=dev["lens"], new_lens=dev["new"], drop_lens=dev["drop"], block_table=dev["table"],
                            free_ids=dev["ring"], free_state=dev["state"], cu_q=dev["cu"], slots=slots, status=status)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        gms.gms_kv_plan(args)
    seen = []
    for step in range(steps):
        often = step % 3 == 0  # steps that want much, and such that give it back
        new = [r.choice([0, 1, 2] if often else [0, 0, 1]) for _ in range(S)]
        drop = [0 if often else r.choice([0, 2, 40, 40]) for _ in range(S)]
        if want == "table" and often:
            new[S // 2] = min(rows - sum(new) + new[S // 2], 3)
            lens[S // 2] = blocks * B - 1 if step % 2 else blocks * B - 8
            for b in range(blocks):
                table[S // 2][b] = -1  # (holes: they take no blocks and give none back)
            dev["lens"].copy_(torch.tensor(lens))
            dev["table"].copy_(torch.tensor(table))
        dev["new"].copy_(torch.tensor(new))
        dev["drop"].copy_(torch.tensor(drop))
        status.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        lens, cu, sl, _, table, ring, state, full = expected(lens, new, drop, table, ring, *state, rows, B, n_blocks, blocks)
        assert int(status) == (gms.DEV_FULL if full else 0), step
        assert dev["lens"].tolist() == lens and dev["table"].tolist() == table and dev["ring"].tolist() == ring and dev["state"].tolist() == state
        assert slots.tolist() == sl and dev["cu"].tolist() == cu
        seen.append(full)
    assert not any(seen) if want == "nothing" else want != "nothing" and not all(seen)
