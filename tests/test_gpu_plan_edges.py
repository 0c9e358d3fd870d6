"""Plans of a step where buffers are shared, pages run out or sums are large, against the simulation of the header."""
import random

import pytest
import torch

from paper_2311_01305_b200 import aweq

from .test_gpu_plan import check, dev, made

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("order", [(2100, 64), (1025, 1024, 3), (64, 1500, 600)])
def test_plans_of_few_and_of_many_sequences_take_turns_on_one_workspace(order):
    """A workspace for the most sequences serves fewer: lengths, pages and the ring's counters are the simulation's step after step."""
    ws = aweq.workspace(aweq.aweq_kv_plan_workspace_bytes(max(order))).zero_()
    runs = []
    for n_seq in order:
        rng = random.Random(n_seq)
        held, sim, pool, table = made(rng, n_seq, 8, 12, 12 * n_seq + 3, 40, turn=5)
        into = aweq.StepPlan(n_seq, 3 * n_seq + 5000)           # (several thread blocks)
        into._ws = (ws.data_ptr(), ws.numel())
        runs.append([rng, held, sim, pool, table, into])
    for _ in range(3):
        for run in runs:
            rng, held, sim, pool, table, into = run
            change = [min(rng.choice([0, 1, 3, -rng.randint(0, h)]), 96 - h) for h in held]
            run[1] = check(sim, pool, table, into, held, change)["own_len"]


def test_a_thousand_sequences_that_give_back_more_than_there_is():
    """1024 rows of 2^22 pages each, all put back at once: the ring takes what it holds (the first row's, less what was free), once."""
    n_seq, pages = 1024, 1 << 22
    table = torch.zeros((n_seq, pages), dtype=torch.int32, device="cuda")
    table[0] = torch.arange(pages, device="cuda").to(torch.int32).flip(0)
    for free in (0, 5):
        pool, st = aweq.PagePool(pages, 1, state=dev([0, free], torch.int64)), aweq.new_status()
        held = dev([pages] * n_seq)
        into = pool.plan(table, held, -held, aweq.StepPlan(n_seq, 0), st=st)
        assert pool.state.tolist() == [0, pages] and not into.own_len.any()
        want = torch.cat([torch.arange(free), torch.arange(pages).flip(0)[:pages - free]]).to(torch.int32).cuda()
        assert torch.equal(pool.ring, want)
        assert aweq.read_out_of_range(st) == n_seq - (free == 0)
        assert (table[0] == -1).all() and (table[-1] == -1).all()
        table[0] = torch.arange(pages, device="cuda").to(torch.int32).flip(0)
