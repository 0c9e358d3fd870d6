"""Attention of drafted trees against its definition in binary64.

Tolerance, with u = 2^-11 (fp16) or 2^-8 (bf16): a probability is off by its score's error (head_dim products added in binary32,
2^-23 each at worst), a few 2^-22 of the exponential and the rescalings, and by u where it is rounded for the product with v; the
output is their mean over |v|, rounded once to 16 bits (u of itself, 2^-25 for fp16 results below the normal range).
"""
import math

import pytest
import torch

from paper_2311_01305_b200 import aweq

pytestmark = pytest.mark.gpu

U16 = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}
DTYPES = [torch.float16, torch.bfloat16]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def make_cache(pages, page, kv, d, dtype, layout="tokens", seed=0):
    g = gen(seed + 100)
    if layout == "heads":
        pools = [torch.randn((pages, kv, page, d), generator=g, device="cuda").to(dtype).permute(0, 2, 1, 3) for _ in range(2)]
    elif layout == "joint":
        both = torch.randn((pages, page, 2, kv, d), generator=g, device="cuda").to(dtype)
        pools = [both[:, :, 0], both[:, :, 1]]
    else:
        pools = [torch.randn((pages, page, kv, d), generator=g, device="cuda").to(dtype) for _ in range(2)]
    return aweq.KVCache(*pools)


def ancestors(counts, seed):
    """[tokens, nodes] truth values of random trees, and every node's depth."""
    g = torch.Generator().manual_seed(seed)
    seen = torch.zeros((sum(counts), max(max(counts), 1)), dtype=torch.bool)
    t = 0
    for n in counts:
        for i in range(n):
            if i:
                up = max(0, i - int(torch.randint(1, 7, (1,), generator=g)))
                seen[t + i] = seen[t + up]
            seen[t + i, i] = True
        t += n
    return seen.cuda()


def words(seen, n):
    seen = torch.nn.functional.pad(seen.to(torch.int64), (0, n * 64 - seen.shape[1]))
    return (seen.unflatten(-1, (n, 64)) << torch.arange(64, device="cuda")).sum(-1).contiguous()


class Case:
    def __init__(self, counts, ctx, h, kv, d, prefix, page, dtype, layout="tokens", seed=3, spread=2.0, stale=True, max_nodes=None, seen=None, extra=0):
        g = gen(seed)
        n_seq, self.counts, self.ctx, self.prefix, self.dtype = len(counts), counts, ctx, prefix, dtype
        self.max_nodes = max_nodes or max(max(counts), 1)
        lens = [c + n for c, n in zip(ctx, counts)]
        per_seq, shared = max(1, -(-max(lens) // page)) + 1, -(-prefix // page)
        self.cache = make_cache(shared + n_seq * per_seq + 2, page, kv, d, dtype, layout, seed)
        order = torch.randperm(self.cache.n_pages, generator=g, device="cuda").to(torch.int32)
        self.prefix_pages, self.table = order[:shared].clone(), order[shared:shared + n_seq * per_seq].view(n_seq, per_seq).clone()
        if stale:
            # whatever lies behind the last key of a page or of a sequence must not be seen
            k, v = self.cache.k, self.cache.v
            if prefix % page:
                k[self.prefix_pages[-1].long(), prefix % page:] = math.nan
                v[self.prefix_pages[-1].long(), prefix % page:] = math.inf
            for b, n in enumerate(lens):
                used = -(-n // page)
                if n % page:
                    k[self.table[b, used - 1].long(), n % page:] = math.inf
                    v[self.table[b, used - 1].long(), n % page:] = math.nan
                self.table[b, used:] = -1
            for p in order[shared + n_seq * per_seq:].tolist():
                k[p], v[p] = math.nan, math.nan
        total = sum(counts)
        self.rows = total + extra
        self.q = (spread * torch.randn((self.rows, h, d), generator=g, device="cuda")).to(dtype)
        self.own_len, self.start = i32(lens), i32([sum(counts[:b]) for b in range(n_seq + 1)])
        self.seen = ancestors(counts, seed) if seen is None else seen
        mask = words(self.seen, -(-self.max_nodes // 64))
        self.mask = torch.cat([mask, mask.new_full((extra, mask.shape[1]), -1)])

    def attend(self, max_own=None, scale=None):
        return aweq.TreeAttention(self.cache, self.prefix_pages, self.prefix, self.q.shape[1], len(self.counts), self.rows, self.max_nodes, max_own, scale)

    def reference(self, scale=None):
        """(out, mean |v| under the probabilities, largest sum |q k| scale of a row), binary64."""
        kv, d, page, c = self.cache.n_kv_heads, self.cache.head_dim, self.cache.page_size, self.cache
        h = self.q.shape[1]
        scale = d ** -0.5 if scale is None else scale
        out = torch.zeros((self.rows, h, d), dtype=torch.float64, device="cuda")
        mag, reach = torch.zeros_like(out), torch.zeros((self.rows, h), dtype=torch.float64, device="cuda")
        pk, pv = (x[self.prefix_pages.long()].reshape(-1, kv, d)[:self.prefix].double() for x in (c.k, c.v))
        t = 0
        for b, n in enumerate(self.counts):
            if n == 0:
                continue
            total = self.ctx[b] + n
            ids = self.table[b, :-(-total // page)].long()
            keys, vals = (torch.cat([p, x[ids].reshape(-1, kv, d)[:total].double()]) for p, x in ((pk, c.k), (pv, c.v)))
            before = self.prefix + self.ctx[b]
            vis = torch.ones((n, before + n), dtype=torch.bool, device="cuda")
            vis[:, before:] = self.seen[t:t + n, :n]
            for j in range(h):
                kk, vv, q = keys[:, j // (h // kv)], vals[:, j // (h // kv)], self.q[t:t + n, j].double()
                kk, vv = kk.nan_to_num(0, 0, 0), torch.where(vis.any(0)[:, None], vv, 0.0)
                p = torch.softmax((q @ kk.t() * scale).masked_fill(~vis, -math.inf), -1)
                p = torch.where(vis.any(1)[:, None], p, 0.0)
                out[t:t + n, j], mag[t:t + n, j] = p @ vv, p @ vv.abs()
                reach[t:t + n, j] = ((q.abs() @ kk.abs().t()) * vis).max(1).values * abs(scale)
            t += n
        return out, mag, reach

    def check(self, max_own=None, scale=None):
        buf = torch.full((self.rows + 2,) + tuple(self.q.shape[1:]), 5.0, dtype=self.dtype, device="cuda")
        st = aweq.new_status()
        out = self.attend(max_own, scale)(self.q, self.table, self.own_len, self.start, self.mask, buf[1:-1], st=st)
        total = sum(self.counts)
        assert (buf[0] == 5).all() and (buf[1 + total:] == 5).all(), "write outside the output"
        assert aweq.read_out_of_range(st) == 0 and aweq.read_status(st)["wait_timeout"] == 0
        want, mag, reach = (x[:total] for x in self.reference(scale))
        d, keys = self.q.shape[2], self.prefix + max(self.ctx) + max(self.counts)
        off = (reach * d * 2.0 ** -23 + 2.0 ** -20 + (keys / 16 + 64) * 2.0 ** -23)[..., None]
        u = U16[self.dtype]
        tol = u * 1.001 * want.abs() + (u + 2 * off) * 1.01 * mag + TINY[self.dtype]
        err = (out[:total].double() - want).abs()
        assert torch.isfinite(out[:total]).all() and (err <= tol).all(), "error %.3g of what is allowed" % (err / tol.clamp(min=1e-300)).max().item()
        return out


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("h,kv,d", [(4, 4, 64), (8, 2, 128), (6, 1, 80), (16, 1, 128), (3, 3, 8), (5, 5, 96), (24, 1, 72), (40, 2, 64), (12, 4, 112)])
def test_head_shapes(h, kv, d, dtype):
    Case([1, 7, 20], [1, 40, 170], h, kv, d, 130, 16, dtype).check()


@pytest.mark.parametrize("prefix", [0, 1, 15, 16, 17, 127, 128, 129, 255, 1000, 4100])
@pytest.mark.parametrize("page", [16, 24])
def test_prefix_lengths(prefix, page):
    Case([3, 1, 5, 12, 2], [0, 1, 5, 64, 130], 4, 2, 64, prefix, page, torch.float16).check()


@pytest.mark.parametrize("layout", ["tokens", "heads", "joint"])
@pytest.mark.parametrize("page", [1, 7, 8, 24, 32, 40, 64, 100, 128, 192, 256])
def test_pages_and_layouts(page, layout):
    """Tiled copies and, where pages do not allow them, 16-byte ones."""
    Case([3, 30, 8, 1], [3, 300, 511, 129], 8, 4, 128, 200, page, torch.bfloat16, layout).check()


@pytest.mark.parametrize("layout", ["tokens", "heads", "joint"])
@pytest.mark.parametrize("page", [7, 24, 64, 100, 256])
def test_pages_and_layouts_with_two_tiles(page, layout):
    Case([70, 3, 90, 64], [511, 129, 300, 40], 8, 4, 128, 200, page, torch.float16, layout).check()


@pytest.mark.parametrize("ctx", [0, 1, 2, 15, 16, 17, 120, 127, 128, 129, 143, 144, 255, 256, 257, 640, 3000])
def test_contexts(ctx):
    """One tile of rows, whose units alternate, and two on the same keys."""
    Case([9], [ctx], 4, 2, 128, 0, 16, torch.bfloat16).check()
    Case([80, 70], [ctx, 2 * ctx], 4, 2, 128, 0, 16, torch.float16).check()


@pytest.mark.parametrize("counts,h,kv", [([1], 1, 1), ([32, 33, 31], 4, 1), ([64, 2, 63, 65], 8, 4), ([128], 2, 2), ([129, 127], 1, 1), ([200, 1, 256], 6, 2), ([100], 16, 1),
                                         ([16] * 9, 16, 2), ([0, 5, 0, 0, 40, 0], 8, 2), ([1] * 70, 4, 4), ([0] * 40 + [3], 4, 2)])
def test_row_tiles(counts, h, kv):
    ctx = [(37 * i * i + 100) % 700 for i in range(len(counts))]
    Case(counts, ctx, h, kv, 64, 77, 16, torch.bfloat16).check()
    Case(counts, ctx, h, kv, 128, 0, 32, torch.float16, max_nodes=256).check()


def test_many_sequences_and_a_long_context():
    Case([(i * 7) % 13 for i in range(150)], [(i * 131) % 400 for i in range(150)], 8, 2, 64, 300, 16, torch.bfloat16).check()
    Case([5, 20], [20000, 50], 8, 1, 128, 0, 64, torch.float16).check()
    Case([40], [30000], 8, 2, 128, 5000, 16, torch.bfloat16).check()


@pytest.mark.parametrize("nodes,d,ctx", [(16, 128, 6000), (16, 64, 6000), (64, 128, 2500)])
def test_first_calls_over_a_big_pool(nodes, d, ctx):
    """Pages all over a pool that nothing has looked at yet: tiles land in any order."""
    Case([nodes] * 32, [(i * 977) % ctx + ctx // 4 for i in range(32)], 32, 8, d, 0, 64, torch.bfloat16, stale=False).check()


@pytest.mark.parametrize("most,prefix", [(130, 0), (400, 130), (1100, 600)])
def test_many_short_items(most, prefix):
    """Several items to a CTA and units enough that an item counts for more than its own: cuts everywhere."""
    Case([1 + i % 5 for i in range(150)], [(i * 131) % most for i in range(150)], 16, 8, 64, prefix, 16, torch.float16).check()
    Case([1 + i % 40 for i in range(90)], [(i * 173) % most for i in range(90)], 32, 8, 128, prefix, 32, torch.bfloat16).check()


@pytest.mark.parametrize("most_nodes,h", [(40, 32), (30, 32), (5, 16)])
def test_the_same_answer_every_time(most_nodes, h):
    """Items of one and of two row tiles in turn, so that the sums of a CTA skip some of them; every run's output bit by bit."""
    case = Case([1 + i % most_nodes for i in range(90)], [(i * 173) % 1100 for i in range(90)], h, 8, 128, 600, 32, torch.bfloat16)
    want = case.check()
    attend, total = case.attend(), sum(case.counts)
    for _ in range(30):
        assert torch.equal(attend(case.q, case.table, case.own_len, case.start, case.mask)[:total], want[:total])


@pytest.mark.parametrize("scale", [0.0, -0.1, 1e-3, 3.0])
def test_scales(scale):
    Case([5, 40], [200, 333], 8, 2, 64, 100, 16, torch.float16, spread=1.0).check(scale=scale)


@pytest.mark.parametrize("dtype", DTYPES)
def test_maxima_that_rise_late_and_small_weights(dtype):
    """Keys far above all before them in the last units of a long context, and thousands of keys far below one: sums that are moved."""
    c = Case([12], [2000], 4, 2, 128, 0, 16, dtype, stale=False)
    pages = c.table[0].long()
    for tile, f in ((40, 2.0), (90, 5.0), (120, 9.0)):
        c.cache.k[pages[tile], 3] = (c.q[:, :2].float().mean(0) * f / 2).to(dtype)
    c.check()
    c = Case([9, 80], [4000, 1500], 4, 4, 64, 0, 16, dtype, spread=1.0, stale=False)
    c.cache.k.mul_(0.05)
    c.cache.k[c.table[:, 0].long(), 0] = (10.0 * c.q[0]).to(dtype) / 8
    c.check()


def test_masks_of_any_kind():
    """Nodes that see nothing of the tree, others' later nodes, everything, or not themselves; bits behind the last node."""
    g = torch.Generator().manual_seed(4)
    counts = [40, 70, 3]
    seen = torch.rand((sum(counts), 70), generator=g) < 0.3
    seen[0], seen[41], seen[5] = False, False, True
    seen[110:112] = False
    for ctx in ([100, 0, 0], [0, 0, 300]):
        c = Case(counts, ctx, 8, 2, 64, 0, 16, torch.bfloat16, seen=seen.cuda())
        out = c.check()
        for t, b in ((0, 0), (41, 1), (110, 2), (111, 2)):
            if ctx[b] == 0:
                assert (out[t] == 0).all()                     # a row without keys


def test_rows_without_any_key_are_zero():
    c = Case([3, 5], [0, 0], 4, 2, 64, 0, 16, torch.float16)
    c.mask.zero_()
    assert (c.attend()(c.q, c.table, c.own_len, c.start, c.mask) == 0).all()


def test_what_a_node_does_not_see_has_no_part():
    """Keys and values of other branches, and of other sequences, that are infinite or no numbers."""
    c = Case([20, 6], [77, 50], 4, 2, 128, 40, 16, torch.bfloat16)
    attend = c.attend()
    clean = attend(c.q, c.table, c.own_len, c.start, c.mask)
    page, row = c.table[0, (77 + 10) // 16].long(), (77 + 10) % 16
    c.cache.k[page, row, 0], c.cache.v[page, row] = math.inf, math.nan
    out = attend(c.q, c.table, c.own_len, c.start, c.mask)
    sees = c.seen[:, 10].clone()
    sees[20:] = False
    assert sees.any() and torch.equal(out[~sees], clean[~sees]) and torch.isnan(out[sees]).all()


def test_values_that_are_no_numbers_reach_those_that_see_them():
    c = Case([4, 4], [100, 300], 4, 2, 64, 20, 16, torch.float16)
    attend = c.attend()
    clean = attend(c.q, c.table, c.own_len, c.start, c.mask)
    c.cache.v[c.table[0, 3].long(), 2, 1] = math.inf
    c.q[6, 3] = math.nan
    out = attend(c.q, c.table, c.own_len, c.start, c.mask)
    hit = torch.zeros((8, 4), dtype=torch.bool, device="cuda")
    hit[:4, 2:] = True
    hit[6, 3] = True
    assert not torch.isfinite(out[hit]).any() and torch.equal(out[~hit], clean[~hit])
    # one key whose score is no number, alone in its part
    c = Case([4], [1], 2, 2, 64, 0, 16, torch.float16)
    c.cache.k[c.table[0, 0].long(), 0, 0, 5] = math.nan
    out = c.attend()(c.q, c.table, c.own_len, c.start, c.mask)
    assert torch.isnan(out[:, 0]).all() and torch.isfinite(out[:, 1]).all()
    # scores that are all minus infinity are no softmax
    c = Case([4], [20], 2, 2, 64, 0, 16, torch.float16, stale=False)
    c.cache.k.fill_(-math.inf)
    c.q.fill_(1.0)
    assert torch.isnan(c.attend()(c.q, c.table, c.own_len, c.start, c.mask)).all()


def test_rows_behind_the_last_sequence_and_max_own():
    Case([3, 9], [50, 60], 4, 2, 64, 30, 16, torch.bfloat16, extra=7).check(max_own=80)
    Case([0, 0], [5, 6], 4, 2, 64, 30, 16, torch.bfloat16, extra=4).check()


def test_lengths_starts_and_pages_out_of_range_are_counted():
    def run(change, want, counts=(5, 6, 7), ctx=(40, 50, 60), max_nodes=None, max_own=None):
        c = Case(list(counts), list(ctx), 4, 2, 64, 40, 16, torch.float16, stale=False, max_nodes=max_nodes)
        attend = c.attend(max_own)
        clean = attend(c.q, c.table, c.own_len, c.start, c.mask)
        keep = change(c)
        st = aweq.new_status()
        buf = torch.full_like(clean, 9.0)
        out = attend(c.q, c.table, c.own_len, c.start, c.mask, buf, st=st)
        assert aweq.read_out_of_range(st) == want and aweq.read_status(st)["wait_timeout"] == 0
        for b in keep:
            s = slice(int(sum(counts[:b])), int(sum(counts[:b + 1])))
            assert torch.equal(out[s], clean[s])
    run(lambda c: c.own_len.__setitem__(1, -5) or [0, 2], 1)
    run(lambda c: c.own_len.__setitem__(1, 4000) or [0, 2], 1)
    run(lambda c: c.own_len.__setitem__(1, 3) or [0, 2], 1)                    # fewer keys than nodes
    run(lambda c: c.own_len.__setitem__(2, 2 ** 31 - 1) or [0, 1], 1)
    run(lambda c: c.start.__setitem__(0, -3) or [1, 2], 1)
    run(lambda c: c.start.__setitem__(3, 1000) or [0, 1], 1)
    run(lambda c: c.table.__setitem__((1, 1), -1) or [0, 2], 1)
    run(lambda c: c.table.__setitem__((1, 3), 10 ** 6) or [0, 2], 1)           # keys 48 to 55: the last two before the nodes, and the nodes'
    run(lambda c: c.prefix_pages.__setitem__(1, 10 ** 6) or [], 1)
    run(lambda c: [0, 1, 2], 3, max_own=30)
    run(lambda c: [1], 2, counts=(9, 4, 9), max_nodes=4)


def test_strides_of_q_and_out():
    c = Case([3, 9], [50, 60], 4, 2, 64, 30, 16, torch.bfloat16)
    want = c.attend()(c.q, c.table, c.own_len, c.start, c.mask)
    qkv = torch.randn((12, 8 * 64), device="cuda").to(torch.bfloat16)
    qkv[:, :256] = c.q.flatten(1)
    wide = torch.zeros((12, 6, 64), dtype=torch.bfloat16, device="cuda")
    out = c.attend()(qkv[:, :256].unflatten(1, (4, 64)), c.table, c.own_len, c.start, c.mask, wide[:, 1:5])
    assert torch.equal(out, want) and (wide[:, 0] == 0).all() and (wide[:, 5] == 0).all()
    flat = aweq.aweq_tree_attention(c.q.flatten(1), c.cache, c.prefix_pages, 30, c.table, c.own_len, c.start, c.mask, 2 ** 31 - 1, c.max_nodes, 0.125,
                                    torch.empty_like(c.q).flatten(1), aweq.workspace(aweq.aweq_tree_attention_workspace_bytes(c.cache, 30, 2 ** 31 - 1, 2, 12, c.max_nodes, 4)))
    assert torch.equal(flat.view_as(want), want)


def test_on_another_stream_in_a_graph_and_again():
    """The same numbers every time: parts are joined in one order."""
    c = Case([30, 9, 64], [800, 90, 2500], 8, 2, 128, 500, 32, torch.bfloat16)
    attend, out = c.attend(), torch.empty_like(c.q)
    want = attend(c.q, c.table, c.own_len, c.start, c.mask)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        for _ in range(5):
            assert torch.equal(attend(c.q, c.table, c.own_len, c.start, c.mask), want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        attend(c.q, c.table, c.own_len, c.start, c.mask, out)
    for n in (2500, 1000, 2500):
        c.own_len[2] = n + 64
        out.zero_()
        graph.replay()
        assert torch.equal(out, c.attend()(c.q, c.table, c.own_len, c.start, c.mask))


@pytest.mark.parametrize("kw", [dict(table=1), dict(mask=1), dict(mask=2), dict(start=1), dict(lens=1), dict(q=1), dict(out=1), dict(pages=1), dict(nodes=1)])
def test_refusals_of_the_binding(kw):
    c = Case([3, 9], [50, 60], 4, 2, 64, 30, 16, torch.bfloat16)
    attend = c.attend()
    q, table, lens, start, mask, out = c.q, c.table, c.own_len, c.start, c.mask, torch.empty_like(c.q)
    with pytest.raises((ValueError, aweq.AweqError)):
        if "pages" in kw:
            attend.prefix_pages = attend.prefix_pages[:1]
        if "nodes" in kw:
            aweq.TreeAttention(c.cache, c.prefix_pages, 30, 4, 2, 12, 300)(q, table, lens, start, mask)
        attend(q[:11] if "q" in kw else q, table[:1] if "table" in kw else table, lens.long() if "lens" in kw else lens, start[:2] if "start" in kw else start,
               mask[:5] if kw.get("mask") == 1 else mask.int() if "mask" in kw else mask, out.half() if "out" in kw else out)
