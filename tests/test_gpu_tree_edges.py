"""Attention of drafted trees on starts, lengths and trees that are not as they should be: what is out of range is counted, what is
well formed keeps its outputs, and nothing is written outside the buffers."""
import pytest
import torch

from paper_2311_01305_b200 import aweq

from .test_gpu_tree import TINY, U16, Case, i32, words

pytestmark = pytest.mark.gpu


def guarded(case, starts, max_nodes=None):
    """The outputs for other starts, with scratch and output inside larger buffers that have to stay as they were; what was counted."""
    c, h, d = case, case.q.shape[1], case.q.shape[2]
    nodes, n_seq = max_nodes or c.max_nodes, len(c.counts)
    size = -(-aweq.aweq_tree_attention_workspace_bytes(c.cache, c.prefix, 2 ** 31 - 1, n_seq, c.rows, nodes, h) // 256) * 256
    ws, out = torch.full((size + (64 << 20),), 0xA5, dtype=torch.uint8, device="cuda"), torch.full((c.rows + 64, h, d), 9.0, dtype=c.dtype, device="cuda")
    assert ws.data_ptr() % 256 == 0
    st = aweq.new_status()
    aweq.aweq_tree_attention(c.q, c.cache, c.prefix_pages, c.prefix, c.table, c.own_len, starts, c.mask, 2 ** 31 - 1, nodes, d ** -0.5, out[:c.rows], ws[:size], st)
    assert (ws[size:] == 0xA5).all(), "write behind the scratch"
    assert (out[c.rows:] == 9).all() and aweq.read_status(st)["wait_timeout"] == 0
    return out[:c.rows], aweq.read_out_of_range(st)


def sequences(case, starts, max_nodes):
    """Each sequence's number of tokens, a start counting as the largest up to it, and those that have a start or length out of range."""
    starts, length = starts.cpu(), case.own_len.cpu()
    up = torch.cummax(starts.clamp(0, case.rows), 0).values
    nodes = up[1:] - up[:-1]
    cap = case.table.shape[1] * case.cache.page_size
    return nodes, (up[:-1] != starts[:-1]) | (up[1:] != starts[1:]) | (nodes > max_nodes) | (length > cap) | (length < nodes.clamp(max=max_nodes))


@pytest.mark.parametrize("h,kv", [(32, 8), (8, 1), (4, 4)])
@pytest.mark.parametrize("n_seq", [2, 16, 33, 64, 100])
@pytest.mark.parametrize("prefix", [0, 40])
def test_starts_that_go_up_and_down(n_seq, h, kv, prefix):
    """Every second sequence would have all rows: only the first has them, and its outputs are as they should be."""
    rows = 256
    case = Case([rows] + [0] * (n_seq - 1), [40 + 3 * b for b in range(n_seq)], h, kv, 64, prefix, 16, torch.float16)
    want = case.check()
    starts = i32(([0, rows] * (n_seq // 2 + 1))[:n_seq] + [rows])
    out, counted = guarded(case, starts)
    nodes, bad = sequences(case, starts, rows)
    assert nodes.tolist() == [rows] + [0] * (n_seq - 1) and torch.equal(out, want) and counted == int(bad.sum())


def test_one_start_below_the_one_before():
    counts, ctx = [5, 6, 7, 8], [30, 300, 50, 200]
    for seen_to in (3, 4, 0, -7):
        case = Case(counts, ctx, 8, 2, 64, 33, 16, torch.bfloat16, stale=False)
        want = case.check()
        starts = case.start.clone()
        starts[1] = 5
        starts[2] = seen_to                                     # ends the second before it starts
        out, counted = guarded(case, starts)
        # the second has no tokens, the third has the second's too: more than a tree may have
        assert counted == 2
        assert torch.equal(out[:5], want[:5]) and torch.equal(out[18:], want[18:])


@pytest.mark.parametrize("seed", range(12))
def test_starts_of_any_kind(seed):
    g = torch.Generator().manual_seed(seed)
    n_seq, rows = (3, 31, 32, 33, 64, 65)[seed % 6], 300
    ctx = torch.randint(0, 400, (n_seq,), generator=g).tolist()
    case = Case([rows // n_seq] * n_seq, ctx, 16, 4, 64, 70 * (seed % 2), 16, torch.float16, stale=False, extra=rows - rows // n_seq * n_seq, max_nodes=(256, 40)[seed % 2])
    starts = torch.randint(-50, rows + 100, (n_seq + 1,), generator=g)
    if seed % 3 == 0:
        starts[:] = torch.tensor([0, 256] * n_seq)[:n_seq + 1]
    if seed % 3 == 1:
        starts = starts.sort(descending=True).values
    case.own_len += torch.randint(0, 200, (n_seq,), generator=g).cuda().int() * (seed % 2)
    case.table.clamp_(min=0)
    _, bad = sequences(case, starts, case.max_nodes)
    _, counted = guarded(case, starts.int().cuda())
    assert counted == int(bad.sum())


def close(case, out, rows):
    """Rows of an output against the definition, with the tolerance of the tests of well-formed calls."""
    want, mag, reach = (x[rows] for x in case.reference())
    d, keys = case.q.shape[2], case.prefix + max(case.ctx) + max(case.counts)
    off = (reach * d * 2.0 ** -23 + 2.0 ** -20 + (keys / 16 + 64) * 2.0 ** -23)[..., None]
    u = U16[case.dtype]
    return bool(((out[rows].double() - want).abs() <= u * 1.001 * want.abs() + (u + 2 * off) * 1.01 * mag + TINY[case.dtype]).all())


@pytest.mark.parametrize("counts,most", [([9, 4, 12], 4), ([70, 3, 64], 64), ([200, 256, 130], 128), ([300, 2], 256), ([3000], 256)])
def test_the_first_nodes_of_trees_that_are_too_large(counts, most):
    """What they see is the keys before the tree and the nodes above them, which lie where the whole tree's keys begin."""
    g = torch.Generator().manual_seed(1)
    seen = torch.rand((sum(counts), max(256, *counts)), generator=g) < 0.1
    seen[:, most:] = False                                      # (what lies behind is beyond the mask's words)
    case = Case(counts, [100, 37, 0][:len(counts)], 8, 2, 64, 20, 16, torch.float16, stale=False, seen=seen.cuda(), max_nodes=max(counts))
    case.mask, case.max_nodes = words(case.seen[:, :256], 4), most
    out = torch.full_like(case.q, 9.0)
    st = aweq.new_status()
    case.attend()(case.q, case.table, case.own_len, case.start, case.mask, out, st=st)
    t = 0
    for n in counts:
        assert close(case, out, slice(t, t + min(n, most))) and (out[t + most:t + n] == 9).all()
        t += n
    assert aweq.read_out_of_range(st) == sum(n > most for n in counts)


@pytest.mark.parametrize("max_own", [0, 30, 41, 45, 60])
def test_keys_beyond_what_there_may_be(max_own):
    """Keys are what they are by their number: those from max_own on are nobody's, the others keep their part."""
    counts, ctx = [5, 6, 7], [40, 36, 20]
    case = Case(counts, ctx, 8, 2, 64, 33, 16, torch.float16, stale=False)
    st = aweq.new_status()
    out = case.attend(max_own)(case.q, case.table, case.own_len, case.start, case.mask, st=st)
    assert aweq.read_out_of_range(st) == sum(c + n > max_own for c, n in zip(ctx, counts))
    t = 0
    for b, n in enumerate(counts):
        case.seen[t:t + n, max(0, max_own - ctx[b]):] = False
        t += n
    case.ctx = [min(c, max_own) for c in ctx]
    # (the definition takes the nodes' keys from behind the context: where that is cut no node has a key)
    assert close(case, out, slice(0, t))


@pytest.mark.parametrize("counts,ctx,short", [([5, 24, 7], [40, 100, 20], [0, 12, 0]), ([5, 24, 7], [40, 100, 20], [5, 24, 1]), ([70, 3, 128], [0, 0, 300], [69, 3, 20]),
                                              ([40, 0, 40], [10, 90, 130], [0, 0, 60])])
def test_own_keys_that_end_before_the_last_node(counts, ctx, short):
    """With positions the nodes' keys begin where the sequence's held ones end, and those beyond its length are nobody's."""
    case = Case(counts, ctx, 8, 2, 64, 33, 16, torch.bfloat16, stale=False, extra=3)
    node = [i for n in counts for i in range(n)]
    base = [c for c, n in zip(ctx, counts) for _ in range(n)]
    pos = i32([1000 + b + (i * 7) % (i + 1) for b, i in zip(base, node)] + [-1] * 3)       # (depths: only a first node's is known, zero)
    attend, st = case.attend(), aweq.new_status()
    whole = attend(case.q, case.table, case.own_len, case.start, case.mask)
    total = sum(counts)
    assert torch.equal(attend(case.q, case.table, case.own_len, case.start, case.mask, st=st, pos=pos, first=1000)[:total], whole[:total])
    assert aweq.read_out_of_range(st) == 0
    case.own_len -= i32(short)
    out = attend(case.q, case.table, case.own_len, case.start, case.mask, st=st, pos=pos, first=1000)
    assert aweq.read_out_of_range(st) == sum(s > 0 and n > 0 for s, n in zip(short, counts))
    t = 0
    for b, n in enumerate(counts):
        case.seen[t:t + n, max(n - short[b], 0):] = False
        case.ctx[b] -= max(short[b] - n, 0)
        t += n
    assert close(case, out, slice(0, total))


@pytest.mark.parametrize("pos0,counted", [(-5, 1), (2 ** 31 - 1, 1), (-2 ** 31, 1), (900, 1), (1000 + 40, 0)])
def test_positions_out_of_range(pos0, counted):
    """Counted, and the other sequences' outputs are what they were."""
    case = Case([5, 6, 7], [30, 40, 20], 8, 2, 64, 33, 16, torch.float16, stale=False)
    pos = i32([1030] * 5 + [1040] * 6 + [1020] * 7)
    attend, st = case.attend(), aweq.new_status()
    want = attend(case.q, case.table, case.own_len, case.start, case.mask)
    pos[5] = pos0
    out = attend(case.q, case.table, case.own_len, case.start, case.mask, st=st, pos=pos, first=1000)
    assert aweq.read_out_of_range(st) == counted and torch.equal(out[:5], want[:5]) and torch.equal(out[11:], want[11:])


@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("page", [128, 50])
def test_two_thousand_million_keys(page, own):
    """Key numbers up to 2^31 - 2, pages over and over.  Queries of zeros and values of one: every sum of a thread block is a whole number of
    units below 2^24 of them, so exact, and a mean over some hundred parts is off by 2^-16 at most: one."""
    n = 2 ** 31 - 1
    k = torch.randn((4, page, 1, 8), device="cuda").half()
    cache = aweq.KVCache(k, torch.ones_like(k))
    pages = (torch.arange(-(-n // page), device="cuda") % 4).to(torch.int32)
    q, mask, st = torch.zeros((1, 1, 8), dtype=torch.float16, device="cuda"), torch.ones((1, 1), dtype=torch.int64, device="cuda"), aweq.new_status()
    table = pages.view(1, -1) if own else i32([[1]])
    attend = aweq.TreeAttention(cache, None if own else pages, 0 if own else n, 1, 1, 1, 1)
    out = attend(q, table, i32([n if own else 1]), i32([0, 1]), mask, st=st)
    assert (out == 1).all() and not st.any()


def test_items_that_take_longer_than_a_wait_may():
    """16 key heads over 2^31 - 1 keys, more than a tile of rows: a thread block that has the end of one item and the start of the next is at the
    first for seconds, and does not give up.  Nothing is said of the values: with ten million keys and more in a sum it is 2^31, 2^8 to its last bit,
    where a product is 2^7 (the header says how far sums go)."""
    n, page, rows = 2 ** 31 - 1, 128, 130
    k = torch.randn((4, page, 16, 8), device="cuda").half()
    cache, st = aweq.KVCache(k, torch.ones_like(k)), aweq.new_status()
    pages = (torch.arange(-(-n // page), device="cuda") % 4).to(torch.int32)
    attend = aweq.TreeAttention(cache, pages, n, 16, 1, rows, rows)
    out = attend(torch.zeros((rows, 16, 8), dtype=torch.float16, device="cuda"), i32([[1, 2]]), i32([rows]), i32([0, rows]),
                 torch.ones((rows, 3), dtype=torch.int64, device="cuda"), st=st)
    assert not st.any() and torch.isfinite(out).all()


@pytest.mark.parametrize("counts,h", [([5, 3], 4), ([90, 70], 4)])
@pytest.mark.parametrize("dtype,log2_size", [(torch.float16, e) for e in (4, 8, 9, 12, 13, 15)] + [(torch.bfloat16, e) for e in (8, 13, 16, 20, 24)])
def test_scores_far_beyond_the_exponents_resolution(counts, h, dtype, log2_size):
    """Queries and keys of plus and minus 2^e: scores are exact, and a few keys lead by so much that the softmax has nothing else (another
    key is 2 2^(2e) / 8 below, 64 at least).  Where several lead, in the prefix, before the tree and the node itself, the output is the mean
    of their values: a third is off by 2^-23, their sum by 2 2^-23, and it is rounded once."""
    ctx, d = [300, 41], 64
    case = Case(counts, ctx, h, h, d, 100, 16, dtype, stale=False, max_nodes=max(counts))
    g = torch.Generator(device="cuda").manual_seed(5)
    sign = lambda *s: torch.randint(0, 2, s, generator=g, device="cuda").mul_(2).sub_(1).to(dtype) * 2.0 ** log2_size  # noqa: E731
    case.cache.k.copy_(sign(*case.cache.k.shape))
    case.q.copy_(sign(1, h, d).expand(case.rows, h, d))
    mask = torch.zeros_like(case.mask)
    t = 0
    leads = []
    for b, n in enumerate(counts):
        for i in range(n):
            mask[t + i, i // 64] = (1 << i % 64) - (2 ** 64 if i % 64 == 63 else 0)
        leads.append([(case.prefix_pages[37 // 16], 37 % 16), (case.table[b, 29 // 16], 29 % 16)])
        t += n
    places = lambda b, n: [(case.table[b, (ctx[b] + i) // 16], (ctx[b] + i) % 16) for i in range(n)]  # noqa: E731
    k, v = case.cache.k, case.cache.v
    attend = case.attend()
    for which in range(1, 8):
        kept = k.clone()
        t, want = 0, []
        for b, n in enumerate(counts):
            here = [leads[b][j] for j in range(2) if which >> j & 1]
            for page, row in here:
                k[page.long(), row] = case.q[0]
            for page, row in places(b, n):
                k[page.long(), row] = case.q[0] if which & 4 else -case.q[0]
                parts = [v[p.long(), r].double() for p, r in here] + ([v[page.long(), row].double()] if which & 4 else [])
                want.append(sum(parts) / len(parts))
        out = attend(case.q, case.table, case.own_len, case.start, mask)
        want = torch.stack(want)
        worst = v.double().abs().max()
        assert ((out.double() - want).abs() <= U16[dtype] * want.abs() + 4 * 2.0 ** -23 * worst + TINY[dtype]).all(), which
        k.copy_(kept)
