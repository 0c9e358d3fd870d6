"""Pages, slots, positions and tree masks from request lengths, places given one by one, and accepted paths: each against a
step-by-step simulation in Python.  Everything here is whole numbers or copies: results are equal."""
import random

import pytest
import torch

from paper_2311_01305_b200 import aweq

pytestmark = pytest.mark.gpu


class Simulated:
    """The plan of the header, one sequence after another."""

    def __init__(self, page, table, ring, state):
        self.page, self.table, self.ring, self.state = page, [list(r) for r in table], list(ring), list(state)

    def plan(self, held, change, rows, first=0, parent=None, words=0):
        page, n, cap = self.page, len(self.ring), len(self.table[0]) * self.page
        bad, total = 0, 0
        taken, given = self.state
        free, given0 = given - taken, given
        own, start, seq, pos, slot, mask = [], [], [], [], [], []
        returned = []
        taken_now = 0
        for b, (h0, c0) in enumerate(zip(held, change)):
            h = min(max(h0, 0), cap)
            new, drop = min(max(c0, 0), cap - h), min(max(-c0, 0), h)
            wrong = h != h0 or new - drop != c0
            kept = min(new, rows - total)
            wrong |= kept != new
            new = kept
            have, after = -(-h // page), h + new - drop
            want = -(-after // page)
            pages = self.table[b]
            got = 0
            for p in range(have, want):
                if taken_now >= free:
                    break
                x = self.ring[(taken + taken_now) % n]
                taken_now += 1
                got += 1
                if not 0 <= x < n:
                    bad += 1
                    x = -1
                pages[p] = x
            if have + got < want:
                wrong = True
                taken_now = max(taken_now, free)
                after = min(after, (have + got) * page)
            for p in range(want, have):
                returned.append(pages[p])
                if len(returned) > n - free:
                    wrong = True
                pages[p] = -1
            start.append(total)
            own.append(after)
            for i in range(new):
                depth, bits = i, 0
                if parent is not None:
                    depth, at = 0, i
                    if i >= 64 * words:
                        bad += 1
                    else:
                        up = parent[total + i]
                        bad += up < -1 or up >= i
                        while True:
                            bits |= 1 << at
                            up = parent[total + at]
                            if up < 0 or up >= at:
                                break
                            at, depth = up, depth + 1
                seq.append(b)
                pos.append(first + h + depth)
                x = pages[(h + i) // page] if h + i < after else -1
                slot.append(x * page + (h + i) % page if 0 <= x < n else -1)
                mask.append([signed((bits >> (64 * w)) & (2 ** 64 - 1)) for w in range(words)])
            total += new
            bad += wrong
        for i, x in enumerate(returned[:n - free]):
            self.ring[(given0 + i) % n] = x
        self.state = [taken + min(taken_now, free), given0 + min(len(returned), n - free)]
        none = [-1] * (rows - total)
        return dict(own_len=own, start=start + [total], seq=seq + none, pos=pos + none, slot=slot + none,
                    mask=mask + [[0] * words for _ in none]), bad


def signed(x):
    return x - 2 ** 64 if x >= 2 ** 63 else x


def dev(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


def check(sim, pool, table, into, held, change, first=0, parent=None, st=None):
    st = aweq.new_status() if st is None else st
    words = 0 if parent is None else into.mask.shape[1]
    got = pool.plan(table, dev(held), dev(change), into, first, None if parent is None else dev(parent), st)
    want, bad = sim.plan(held, change, into.max_tokens, first, parent, words)
    for name in ("own_len", "start", "seq", "pos", "slot") + (("mask",) if words else ()):
        assert getattr(got, name).tolist() == want[name], name
    assert table.tolist() == sim.table and pool.ring.tolist() == sim.ring and pool.state.tolist() == sim.state
    assert aweq.read_out_of_range(st) == bad
    return want


def made(rng, n_seq, page, per_seq, n_pages, most_held, turn=0):
    held = [rng.randint(0, most_held) for _ in range(n_seq)]
    order = list(range(n_pages))
    rng.shuffle(order)
    table, at = [], 0
    for h in held:
        k = -(-h // page)
        table.append(order[at:at + k] + [-1] * (per_seq - k))
        at += k
    free = n_pages - at
    ring = [0] * n_pages
    for i in range(n_pages):
        ring[(turn + i) % n_pages] = order[at + i] if i < free else 0
    state = [turn, turn + free]
    sim, t = Simulated(page, table, ring, state), dev(table)
    return held, sim, aweq.PagePool(n_pages, page, ring=dev(ring), state=dev(state, torch.int64)), t


@pytest.mark.parametrize("n_seq,page,most_new,tree", [(1, 16, 1, False), (1, 1, 5, False), (3, 8, 40, True), (64, 16, 32, True), (256, 24, 7, False), (257, 16, 3, True),
                                                      (600, 64, 9, False), (1024, 16, 2, True), (1025, 16, 5, True), (2100, 8, 3, False), (5, 128, 3000, False),
                                                      (7, 16, 200, True)])
def test_steps_in_a_row(n_seq, page, most_new, tree):
    """Growing, shrinking and idle sequences, step after step on the same pages, around the end of the ring."""
    rng = random.Random(n_seq * 31 + page)
    per_seq = (150 + 3 * most_new) // page + 2
    n_pages = n_seq * per_seq + 3
    held, sim, pool, table = made(rng, n_seq, page, per_seq, n_pages, 150, turn=n_pages - 2)
    into = aweq.StepPlan(n_seq, (n_seq * most_new + 63) // 64 * 64 + 5, most_new if tree else 0)
    for step in range(4):
        change = [rng.choice([0, rng.randint(1, most_new), rng.randint(0, most_new), -rng.randint(0, h)]) if step < 3 else -h for h in held]
        change = [min(c, per_seq * page - h) for c, h in zip(change, held)]
        parent = None
        if tree:
            parent = []
            for c in change:
                parent += [rng.randint(max(-1, i - 9), i - 1) for i in range(max(c, 0))]
            parent += [rng.randint(-5, 99) for _ in range(into.max_tokens - len(parent))]         # rows that are no tokens: anything
        held = check(sim, pool, table, into, held, change, first=100 * step, parent=parent)["own_len"]
    assert held == [0] * n_seq and pool.state.tolist()[1] - pool.state.tolist()[0] == n_pages


def test_no_pages_left():
    rng = random.Random(5)
    held, sim, pool, table = made(rng, 6, 8, 20, 30, 20)
    into = aweq.StepPlan(6, 400)
    want = check(sim, pool, table, into, held, [50, 3, 60, 0, 40, 1])
    assert pool.state.tolist()[0] == pool.state.tolist()[1]
    assert any(s == -1 for s in want["slot"][:want["start"][-1]])
    held = want["own_len"]
    # nobody is left without what it holds, and what is given back serves the next
    check(sim, pool, table, into, held, [-h for h in held])
    check(sim, pool, table, into, [0] * 6, [9, 0, 1, 2, 3, 4])


@pytest.mark.parametrize("held,change,rows", [([-3, 500, 10], [4, 1, 2], 64), ([10, 10, 10], [-11, 2000, -2 ** 31], 64), ([0, 20, 5], [30, 30, 30], 50),
                                              ([0, 20, 5], [2 ** 31 - 1, 2 ** 31 - 1, 1], 16), ([64, 63, 0], [1, 1, 64], 66), ([2 ** 31 - 1, -2 ** 31, 1], [1, 1, 1], 8),
                                              ([5, 6, 7], [1, 1, 1], 0)])
def test_lengths_that_do_not_fit(held, change, rows):
    sane = [min(max(h, 0), 64) for h in held]
    table = [[3 * p + b if p < -(-s // 16) else -1 for p in range(4)] for b, s in enumerate(sane)]
    used = {x for r in table for x in r}
    free = [x for x in range(20) if x not in used]
    ring = free + [0] * (20 - len(free))
    sim, t = Simulated(16, table, ring, [0, len(free)]), dev(table)
    pool = aweq.PagePool(20, 16, ring=dev(ring), state=dev([0, len(free)], torch.int64))
    check(sim, pool, t, aweq.StepPlan(3, rows), held, change)


def test_bad_pages_in_the_ring_and_parents_that_are_none():
    table = [[-1] * 4 for _ in range(2)]
    ring = [5, 7, -1, 8, 2, 3, 4, 1]
    sim, t = Simulated(4, table, ring, [0, 8]), dev(table)
    pool = aweq.PagePool(8, 4, ring=dev(ring), state=dev([0, 8], torch.int64))
    parent = [-1, 0, 2, 9, 3, -7, 1, 6, 0, 1]
    check(sim, pool, t, aweq.StepPlan(2, 10, 64), [0, 0], [8, 2], parent=parent)


@pytest.mark.parametrize("state", [[-1, 5], [9, 3], [0, 9], [-2 ** 63, 2 ** 63 - 1]])
def test_a_ring_that_cannot_be(state):
    """Taken as empty: nobody gets a page, and what is given back starts it anew."""
    t, st = dev([[0, 1], [2, -1]]), aweq.new_status()
    pool = aweq.PagePool(8, 4, state=dev(state, torch.int64))
    into = pool.plan(t, dev([8, 4]), dev([-8, 1]), aweq.StepPlan(2, 4), st=st)
    assert into.own_len.tolist() == [0, 4] and into.slot.tolist() == [-1] * 4 and t.tolist() == [[-1, -1], [2, -1]]
    assert pool.state.tolist() == [0, 2] and pool.ring.tolist()[:2] == [0, 1] and aweq.read_out_of_range(st) == 2


def test_more_given_back_than_the_ring_holds():
    """Pages of two rows are the same: the ring is full before all are back."""
    t, st = dev([[0, 1, 2], [0, 1, 2]]), aweq.new_status()
    pool = aweq.PagePool(4, 4, ring=dev([3, 9, 9, 9]), state=dev([0, 1], torch.int64))
    pool.plan(t, dev([12, 12]), dev([-12, -12]), aweq.StepPlan(2, 0), st=st)
    assert pool.state.tolist() == [0, 4] and pool.ring.tolist() == [3, 0, 1, 2] and aweq.read_out_of_range(st) == 1


def test_trees_wider_than_the_words():
    table, ring = [[-1] * 10], list(range(16))
    sim, t = Simulated(16, table, ring, [0, 16]), dev(table)
    pool = aweq.PagePool(16, 16)
    into = aweq.StepPlan(1, 160, 128)
    check(sim, pool, t, into, [0], [140], parent=[i - 1 for i in range(160)])


def test_table_with_a_pitch_rows_around_it_stay():
    rng = random.Random(3)
    held, sim, pool, table = made(rng, 9, 16, 6, 80, 60)
    wide = torch.full((9, 11), 77, dtype=torch.int32, device="cuda")
    wide[:, 2:8] = table
    into = aweq.StepPlan(9, 128)
    check(sim, pool, wide[:, 2:8], into, held, [5, 0, -3, 20, 1, 1, 1, -2, 7] if min(held[2], held[7]) > 2 else [5, 0, 0, 20, 1, 1, 1, 0, 7])
    assert (wide[:, :2] == 77).all() and (wide[:, 8:] == 77).all()


def test_captured_step_replays():
    """A step of drafted tokens and one that gives all of them back, as a graph: after each replay lengths and number of pages are what they were."""
    rng = random.Random(8)
    held, sim, pool, table = made(rng, 40, 16, 8, 330, 90)
    grow, shrink = aweq.StepPlan(40, 1024, 24), aweq.StepPlan(40, 0)
    new = [rng.randint(0, 24) for _ in held]
    parent = [x for c in new for x in [i - 1 for i in range(c)]]
    parent += [-1] * (1024 - len(parent))
    h, c, back, up = dev(held), dev(new), dev([-x for x in new]), dev(parent)

    def step():
        pool.plan(table, h, c, grow, parent=up)
        pool.plan(table, grow.own_len, back, shrink)

    step()
    sim.plan(held, new, 1024, 0, parent, 1)
    sim.plan([a + b for a, b in zip(held, new)], [-x for x in new], 0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(5):
        graph.replay()
        want, _ = sim.plan(held, new, 1024, 0, parent, 1)
        sim.plan(want["own_len"], [-x for x in new], 0)
        assert grow.slot.tolist() == want["slot"] and grow.mask.tolist() == want["mask"] and shrink.own_len.tolist() == held
        assert table.tolist() == sim.table and pool.ring.tolist() == sim.ring and pool.state.tolist() == sim.state


@pytest.mark.parametrize("kw", [dict(own="held"), dict(parent=True), dict(short=True), dict(table=True), dict(ring=True), dict(state=True), dict(dtype=True)])
def test_plan_refusals_of_the_binding(kw):
    table, held = dev([[0, -1]]), dev([1])
    pool, into = aweq.PagePool(4, 4), aweq.StepPlan(1, 4)
    if "own" in kw:
        held = into.own_len                    # lengths are not rewritten in place
    if "table" in kw:
        table = table.to(torch.int64)
    with pytest.raises((ValueError, aweq.AweqError)):
        if "ring" in kw:
            aweq.PagePool(5, 4, ring=dev([1, 2]))
        if "state" in kw:
            aweq.PagePool(4, 4, state=dev([0, 4]))
        pool.plan(table, held.float() if "dtype" in kw else held, dev([1, 2]) if "short" in kw else dev([1]), into, parent=dev([-1] * 4) if "parent" in kw else None)


# ---------------------------------------------------------------------------- places given one by one
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n,heads,kv,d,rd,offset", [(1, 4, 2, 64, 64, 0), (37, 8, 2, 128, 64, 0), (37, 12, 12, 72, 24, 3), (300, 4, 1, 96, 0, 0)])
def test_append_by_slots_is_append(n, heads, kv, d, rd, offset, interleaved, dtype):
    """The same tokens at the same places and positions, found through a page table and given as slots."""
    g = torch.Generator(device="cuda").manual_seed(n)
    pools = [torch.randn((50, 8, kv, d), generator=g, device="cuda").to(dtype) for _ in range(2)]
    x = torch.randn((n, (heads + 2 * kv) * d + offset), generator=g, device="cuda").to(dtype)[:, offset:]
    q, k, v = (t.unflatten(1, (-1, d)) for t in x.split([heads * d, kv * d, kv * d], 1))
    order = torch.randperm(50, generator=g, device="cuda")[:40].to(torch.int32).view(1, 40)
    pos = torch.randperm(320, generator=g, device="cuda")[:n].to(torch.int32)
    table = aweq.aweq_rope_table(rd, 400) if rd else None
    a, b = ([p.clone() for p in pools] for _ in range(2))
    qa = aweq.aweq_kv_append(aweq.KVCache(*a), order, k, v, pos, seq=torch.zeros_like(pos), table=table, interleaved=interleaved, q=q, q_out=torch.empty((n, heads, d), dtype=dtype, device="cuda"))
    slot = order[0, (pos // 8).long()].long() * 8 + pos % 8
    qb = aweq.aweq_kv_append_slots(aweq.KVCache(*b), slot, k, v, pos, table=table, interleaved=interleaved, q=q, q_out=torch.empty((n, heads, d), dtype=dtype, device="cuda"))
    assert torch.equal(qa, qb) and torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    # no tokens, places outside, positions outside
    st = aweq.new_status()
    slot[:] = torch.where(torch.arange(n, device="cuda") % 3 == 0, -1, torch.where(torch.arange(n, device="cuda") % 3 == 1, 400, slot))
    bad = sum(i % 3 == 1 for i in range(n))
    c = [p.clone() for p in pools]
    qc = aweq.aweq_kv_append_slots(aweq.KVCache(*c), slot, k, v, pos, table=table, interleaved=interleaved, q=q, q_out=torch.empty((n, heads, d), dtype=dtype, device="cuda"), st=st)
    assert aweq.read_out_of_range(st) == bad
    assert (qc[::3] == 0).all() and torch.equal(qc[2::3], qa[2::3]) and torch.equal(qc[1::3], qa[1::3])
    want = [p.clone() for p in pools]
    for w, full in zip(want, a):
        w.view(400, kv, d)[slot[2::3]] = full.view(400, kv, d)[slot[2::3]]
    assert torch.equal(c[0], want[0]) and torch.equal(c[1], want[1])
    if rd:
        far = pos.clone()
        far[::2] = 400
        st = aweq.new_status()
        aweq.aweq_kv_append_slots(aweq.KVCache(*c), slot.clamp(0, 399), k, v, far, table=table, interleaved=interleaved, st=st)
        assert aweq.read_out_of_range(st) == (n + 1) // 2


# ---------------------------------------------------------------------------- accepted paths
def accepted(pool, page, table, base, path, count):
    out = pool.clone()
    flat, src = out.view(-1, *out.shape[2:]), pool.view(-1, *pool.shape[2:])
    for row, b, p, c in zip(table, base, path, count):
        for i in range(c):
            s, d = b + p[i], b + i
            flat[row[d // page] * page + d % page] = src[row[s // page] * page + s % page]
    return out


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n_seq,page,kv,d,nodes,most", [(1, 16, 1, 8, 2, 2), (3, 4, 2, 64, 30, 30), (40, 16, 8, 128, 64, 17), (5, 24, 3, 72, 100, 40), (2, 128, 12, 256, 16, 8)])
def test_accepted_paths(n_seq, page, kv, d, nodes, most, dtype):
    rng, g = random.Random(n_seq), torch.Generator(device="cuda").manual_seed(n_seq)
    base = [rng.randint(0, 70) for _ in range(n_seq)]
    per_seq = (70 + nodes) // page + 1
    order = list(range(n_seq * per_seq + 2))
    rng.shuffle(order)
    table = [order[b * per_seq:(b + 1) * per_seq] for b in range(n_seq)]
    path = [sorted(rng.sample(range(nodes), most)) for _ in range(n_seq)]
    count = [rng.randint(0, most) for _ in range(n_seq)]
    if n_seq > 2:
        path[0], count[0] = list(range(most)), most                                 # everything is where it belongs
        path[1], count[1] = list(range(nodes - most, nodes)), most                  # a run moves over itself
    pools = [torch.randn((len(order), page, kv, d), generator=g, device="cuda").to(dtype) for _ in range(2)]
    want = [accepted(p, page, table, base, path, count) for p in pools]
    st = aweq.new_status()
    aweq.aweq_kv_accept(aweq.KVCache(*pools), dev(table), dev(base), dev(path), dev(count), st)
    assert torch.equal(pools[0], want[0]) and torch.equal(pools[1], want[1]) and aweq.read_out_of_range(st) == 0


def test_accept_with_tokens_inside_heads_and_a_pitch():
    g = torch.Generator(device="cuda").manual_seed(1)
    pools = [torch.randn((6, 3, 8, 72), generator=g, device="cuda").half().permute(0, 2, 1, 3)[..., :64] for _ in range(2)]
    table, path = [[4, 1, 3]], [[1, 5, 9, 11]]
    want = [accepted(p.contiguous(), 8, table, [6], path, [4]) for p in pools]
    wide = torch.full((1, 9), -9, dtype=torch.int32, device="cuda")
    wide[:, :4] = dev(path)
    aweq.aweq_kv_accept(aweq.KVCache(*pools), dev(table), dev([6]), wide[:, :4], dev([4]))
    assert torch.equal(pools[0], want[0]) and torch.equal(pools[1], want[1])


@pytest.mark.parametrize("table,base,path,count,moved", [
    ([4, 1, 3], -1, [1, 2, 3], 3, 0), ([4, 1, 3], 25, [1, 2, 3], 3, 0), ([4, 1, 3], 2, [1, 4, 4], 3, 2), ([4, 1, 3], 2, [3, 2, 5], 3, 1), ([4, 1, 3], 2, [-1, 2, 5], 3, 0),
    ([4, 1, 3], 2, [1, 2, 5], 4, 3), ([4, 1, 3], 2, [1, 2, 5], -1, 0), ([4, 9, 3], 2, [1, 3, 7], 3, 2), ([4, -1, 3], 2, [1, 3, 7], 3, 2), ([4, 1, 3], 20, [1, 2, 5], 3, 2),
    ([4, 1, 3], 2 ** 31 - 1, [1, 2, 5], 3, 0), ([4, 1, 3], 20, [1, 2, 2 ** 31 - 1], 3, 2)])
def test_paths_that_do_not_fit(table, base, path, count, moved):
    """What comes before the fault is moved, the rest stays, and it is counted once."""
    g = torch.Generator(device="cuda").manual_seed(2)
    pools = [torch.randn((6, 8, 2, 64), generator=g, device="cuda").half() for _ in range(2)]
    want = [accepted(p, 8, [table], [base], [path], [moved]) for p in pools]
    st = aweq.new_status()
    aweq.aweq_kv_accept(aweq.KVCache(*pools), dev([table]), dev([base]), dev([path]), dev([count]), st)
    assert torch.equal(pools[0], want[0]) and torch.equal(pools[1], want[1]) and aweq.read_out_of_range(st) == 1
