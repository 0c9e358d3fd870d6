"""Steps of drafted trees where something does not fit or is of another step: what can be answered is right, the rest is refused or counted."""
import pytest
import torch

from paper_2311_01305_b200 import aweq

from .test_gpu_drafting import D, FORMATS, PAGE, Recorded, Server, attended, check_output, drawn, i32, layer, make_block  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("prefix,pages", [(70, 5), (0, 4), (33, 3), (16, 1)])
def test_a_pool_that_runs_out(layer, fmt, prefix, pages):  # noqa: F811
    """Trees of up to 24 on a few pages.  Nodes that found a place are answered as if the tree ended there, so are whole trees; the step is
    counted; what is kept and given back by the lengths leaves a cache that the next step is right on."""
    rng = torch.Generator().manual_seed(7)
    n_seq, nodes, per_seq = 4, 24, 12
    tokens, rows, n_pages = layer[1], n_seq * nodes + 5, -(-prefix // PAGE) + pages
    block = make_block(layer, fmt, n_pages + 1, aweq.aweq_rope_table(D, 512))
    server = Server(block, layer, n_seq, nodes, rows, prefix, per_seq, torch.arange(n_pages, dtype=torch.int32, device="cuda"), Recorded)
    kept = [tokens[:prefix]] * n_seq
    short_once = False
    for _ in range(5):
        trees, call = drawn(rng, tokens, n_seq, nodes, rows)
        server.st.zero_()
        server.pool.plan(server.table, server.kept.own_len, call["n"], server.grown, first=prefix, parent=call["parent"], st=server.st)
        held, grown, slot = server.kept.own_len.tolist(), server.grown.own_len.tolist(), server.grown.slot.tolist()
        out = block.verify(call["x"], server.attend, server.table, server.grown, server.st)
        at, paths, short = 0, [], 0
        for b, (up, depth, sees, path) in enumerate(trees):
            placed = grown[b] - held[b]
            assert placed == sum(s >= 0 for s in slot[at:at + len(up)]) and 0 <= placed <= len(up)
            short += placed < len(up)
            paths.append([i for i in path if i < placed])
            if placed:
                old, x = kept[b].shape[0], call["x"][at:at + placed]
                pos = torch.cat([torch.arange(old), old + torch.tensor(depth[:placed])]).cuda()
                want, tol = attended(block, layer, torch.cat([kept[b], x]), pos,
                                     torch.cat([torch.ones(placed, old, dtype=torch.bool), sees[:placed, :placed]], 1).cuda())
                got = server.attend.seen[at:at + placed]
                assert ((got.double() - want).abs() <= tol).all()
                check_output(block, layer, got, out[at:at + placed])
                kept[b] = torch.cat([kept[b], x[torch.tensor(paths[b], dtype=torch.long, device="cuda")]])
            at += len(up)
        short_once |= short > 0
        # counted by the plan and by the attention
        assert aweq.read_out_of_range(server.st) == 2 * short
        aweq.aweq_kv_accept(block.cache, server.table, server.kept.own_len, i32([p + [0] * (nodes - len(p)) for p in paths]), i32([len(p) for p in paths]))
        back = [h + len(p) - g for h, p, g in zip(held, paths, grown)]
        server.pool.plan(server.table, server.grown.own_len, i32(back), server.kept)
        assert server.kept.own_len.tolist() == [k.shape[0] - prefix for k in kept]
    assert short_once and aweq.read_status(server.st)["wait_timeout"] == 0


def test_masks_of_another_step_are_refused(layer):  # noqa: F811
    """A plan that was last filled without parents has the masks of the step before, or none yet; with parents it serves again."""
    block = make_block(layer, "e8m0", 8)
    pool, table, held = aweq.PagePool(8, PAGE), i32([[-1] * 2, [-1] * 2]), i32([0, 0])
    plan, attend = aweq.StepPlan(2, 8, 4), block.drafts(2, 8, 4, max_own=32)
    x = layer[1][:8].contiguous()
    for _ in range(2):
        pool.plan(table, held, i32([3, 2]), plan)
        before = block.cache.k.clone()
        with pytest.raises(ValueError):
            block.verify(x, attend, table, plan)
        assert torch.equal(block.cache.k, before), "refused, but stored"
        pool.plan(table, plan.own_len, i32([-3, -2]), aweq.StepPlan(2, 0))
        pool.plan(table, held, i32([3, 2]), plan, parent=i32([-1, 0, 1, -1, 0, -1, -1, -1]))
        chain = block.verify(x, attend, table, plan)
        assert torch.isfinite(chain[:5]).all() and plan.mask[:5, 0].tolist() == [1, 3, 7, 1, 3]
        pool.plan(table, plan.own_len, i32([-3, -2]), aweq.StepPlan(2, 0))


@pytest.mark.parametrize("wrong", ["masks", "table"])
def test_what_is_refused_stores_nothing(layer, wrong):  # noqa: F811
    """Masks too narrow for the attention's trees, a table of other sequences: known before the first launch."""
    block = make_block(layer, "e8m0", 8)
    pool, table = aweq.PagePool(8, PAGE), i32([[-1] * 2, [-1] * 2])
    plan, attend = aweq.StepPlan(2, 8, 4), block.drafts(2, 8, 100 if wrong == "masks" else 4, max_own=32)
    pool.plan(table, i32([0, 0]), i32([3, 2]), plan, parent=i32([-1, 0, 1, -1, 0, -1, -1, -1]))
    with pytest.raises(ValueError):
        block.verify(layer[1][:8].contiguous(), attend, table[:1] if wrong == "table" else table, plan)
    assert not block.cache.k.any()


def test_no_rows_at_all(layer):  # noqa: F811
    """A plan without rows has no masks to be stale: nothing is answered, nothing stored."""
    block = make_block(layer, "e4m3", 8)
    plan, attend, table = aweq.StepPlan(2, 0, 4), block.drafts(2, 0, 4, max_own=32), i32([[-1] * 2, [-1] * 2])
    for parent in (None, i32([])):
        aweq.PagePool(8, PAGE).plan(table, i32([0, 0]), i32([0, 0]), plan, parent=parent)
        assert block.verify(layer[1][:0], attend, table, plan).shape == (0, block.o.C_out)
    assert not block.cache.k.any()
