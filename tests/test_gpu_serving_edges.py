"""Where the operators that run a calibrated layer could go wrong quietly: weights far below the row's largest,
channels beyond a grid's limit, codes that change after the layer was made, pools whose strides no tiled copy can
hold, scores of minus infinity, counts of bad entries, rows without a pitch, zero-points of 31 bits.  Tolerances
are those of ``test_gpu_serving`` (derived there); what a test adds to them is derived beside it."""
import math

import pytest
import torch

from paper_2311_01305_b200 import aweq

from .test_gpu_serving import (DTYPES, TINY, U16, attention_case, attention_check, attention_close, attention_reference, gen, linear_check,
                               linear_inputs, make_cache)

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------- weights far below the largest
# Rows and keys of a prefix for the kernel of few rows (page sizes that no tiled copy fits go there, whatever the rows) and
# for the tensor kernel; own keys of many sequences.
FEW, MANY, OWN = (dict(n_seq=50, heads=64, keys=4096, page=12), dict(n_seq=40, heads=16, keys=4100, page=16),
                  dict(n_seq=80, heads=16, keys=600, page=16, own=True))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("place", [0, 77, -1])
@pytest.mark.parametrize("log2_weight", [-12.3, -18.6, -23.5, -25])
@pytest.mark.parametrize("shape", [FEW, MANY, OWN], ids=["few", "many", "own"])
def test_attention_many_small_weights_beside_one_large(shape, log2_weight, place, dtype):
    """One key of weight 1 whose value is zero, hundreds to thousands of weight 2^-12 to 2^-25: the output is made of the small ones.

    The header allows fp16 probabilities to be off by 2^-32 of the largest each (beside u of themselves); values are below 2."""
    n_seq, h, n, page, own, d = shape["n_seq"], shape["heads"], shape["keys"], shape["page"], shape.get("own"), 64
    g = gen(31)
    each = -(-n // page)
    cache = make_cache(n_seq * each if own else each, page, h, d, dtype)
    listed = torch.arange(cache.n_pages, dtype=torch.int32, device="cuda").view(-1, each)
    k = torch.zeros(listed.shape + (page, h, d), device="cuda")
    v = 1.0 + torch.rand(k.shape, generator=g, device="cuda")
    k[..., 0] = log2_weight
    sink = place % n
    k[:, sink // page, sink % page], v[:, sink // page, sink % page] = 0.0, 0.0
    cache.k.copy_(k.view_as(cache.k))
    cache.v.copy_(v.view_as(cache.v))
    q = torch.zeros((n_seq, h, d), dtype=dtype, device="cuda")
    q[:, :, 0] = 1.0
    prefix, lens = (0, n) if own else (n, 0)
    pages = listed if own else torch.zeros((n_seq, 1), dtype=torch.int32, device="cuda")
    lens = torch.full((n_seq,), lens, dtype=torch.int32, device="cuda")
    attend = aweq.PrefixAttention(cache, listed[0], prefix, h, n_seq, 1, n, scale=math.log(2.0))
    out = attend(q, pages, lens)
    want, mag, reach = attention_reference(q, cache, listed[0], prefix, pages, lens, 1, attend.scale)
    off = (reach * d * 2.0 ** -23 + 2.0 ** -20 + (n / 16 + 64) * 2.0 ** -23)[..., None]
    tol = U16[dtype] * 1.001 * want.abs() + (U16[dtype] + 2 * off) * 1.01 * mag + TINY[dtype] + (n * 2.0 ** -32 * 2 if dtype is torch.float16 else 0)
    err = (out.double() - want).abs()
    assert (err <= tol).all(), "off by %.3g of the output" % (err / want.abs()).max().item()


# ---------------------------------------------------------------------------- large scores
@pytest.mark.parametrize("n_seq,heads", [(3, 4), (40, 16)])
@pytest.mark.parametrize("dtype,log2_size", [(torch.float16, e) for e in (8, 9, 12, 13, 15)] + [(torch.bfloat16, e) for e in (8, 9, 13, 16, 20, 24)])
def test_attention_of_scores_far_beyond_the_exponents_resolution(n_seq, heads, dtype, log2_size):
    """Queries and keys of plus and minus 2^e: scores are exact multiples of 2^(2e), and each row's own key leads by so much
    that the softmax has nothing else: the output is that key's value."""
    g, n, d, page = gen(17), 4100, 64, 16
    cache = make_cache(-(-n // page) + n_seq, page, heads, d, dtype)
    sign = lambda *s: torch.randint(0, 2, s, generator=g, device="cuda").mul_(2).sub_(1).to(dtype) * 2.0 ** log2_size  # noqa: E731
    cache.k.copy_(sign(*cache.k.shape))
    q = sign(n_seq, heads, d)
    pages = torch.arange(cache.n_pages, dtype=torch.int32, device="cuda")
    at = (torch.arange(n_seq, device="cuda") * 997 + 65) % n         # where each sequence's key lies in the prefix
    cache.k[at // page, at % page] = q
    attend = aweq.PrefixAttention(cache, pages[:-n_seq], n, heads, n_seq, 1, page)
    out = attend(q, pages[-n_seq:].view(-1, 1), torch.full((n_seq,), 5, dtype=torch.int32, device="cuda"))
    assert torch.equal(out, cache.v[at // page, at % page])


# ---------------------------------------------------------------------------- a layer is what it was made of
@pytest.mark.parametrize("n", [3, 300])
def test_linear_layer_keeps_its_weights_when_the_callers_change(n):
    """A calibrator that runs again writes its codes, Steps and zero-points in place."""
    i = linear_inputs(n, 256, 72, 15)
    layer = aweq.LinearW8A8(i["w"], i["ws"], i["wz"], i["b"])
    want = layer(i["x"], i["xs"], i["xz"])
    i["w"].copy_(255 - i["w"])
    i["ws"].mul_(3.0)
    i["wz"].add_(5)
    i["b"].add_(1.0)
    assert torch.equal(layer(i["x"], i["xs"], i["xz"]), want)
    linear_check(i, torch.float16)                                 # a layer made of them now


# ---------------------------------------------------------------------------- channels beyond a grid's limit
@pytest.mark.parametrize("n,k,o", [(1, 64, 65535 * 64 + 65), (17, 16, 65535 * 64 + 1), (3, 64, 65535 * 256 + 300)])
def test_linear_millions_of_channels(n, k, o):
    linear_check(linear_inputs(n, k, o, 6), torch.float16)


# ---------------------------------------------------------------------------- strides that no tiled copy can hold
@pytest.mark.parametrize("page_stride", [0, 1 << 40])
@pytest.mark.parametrize("n_seq", [2, 20, 40])
def test_attention_over_one_page_of_any_stride(n_seq, page_stride):
    """Everything in one page: its stride is never used, and may be more than a tiled copy can hold, or nothing.  Few rows and many
    rows take different kernels; both answer."""
    h, d, n = 16, 64, 4096
    cache = make_cache(1, n, h, d, torch.float16)
    cache.args.page_stride = page_stride
    zero = torch.zeros((n_seq, 1), dtype=torch.int32, device="cuda")
    lens = torch.full((n_seq,), 30, dtype=torch.int32, device="cuda")
    q = (2.0 * torch.randn((n_seq, h, d), generator=gen(9), device="cuda")).to(torch.float16)
    out = aweq.PrefixAttention(cache, zero[0], n - 7, h, n_seq, 1, 64)(q, zero, lens)
    cache.args.page_stride = n * h * d
    assert torch.isfinite(out).all()
    plain = aweq.PrefixAttention(cache, zero[0], n - 7, h, n_seq, 1, 64)(q, zero, lens)
    want, mag, reach = attention_reference(q, cache, zero[0], n - 7, zero, lens, 1, d ** -0.5)
    off = (reach * d * 2.0 ** -23 + 2.0 ** -20 + (n / 16 + 64) * 2.0 ** -23)[..., None]
    tol = U16[torch.float16] * 1.001 * want.abs() + (U16[torch.float16] + 2 * off) * 1.01 * mag + TINY[torch.float16]
    for got in (out, plain):
        assert ((got.double() - want).abs() <= tol).all()


# ---------------------------------------------------------------------------- scores of minus infinity
@pytest.mark.parametrize("n_seq,heads,prefix", [(3, 4, 70), (3, 4, 0), (40, 16, 4100)])
def test_attention_of_scores_that_are_all_minus_infinity(n_seq, heads, prefix):
    """The softmax of such a row is 0 / 0.  A row that sees no key stays zero."""
    q, cache, prefix_pages, pages, lens = attention_case(n_seq, 2, heads, heads, 64, prefix, [5] * n_seq, 16, torch.float16, stale=False)
    cache.k[..., 3] = -math.inf
    q[..., 3] = 1.0
    q[2, :, 3] = -1.0
    attend = aweq.PrefixAttention(cache, prefix_pages, prefix, heads, n_seq, 2)
    if prefix == 0:
        lens[2] = 1                                                # its first token sees nothing
    out = attend(q, pages, lens)
    nothing = torch.zeros(2 * n_seq, dtype=torch.bool, device="cuda")
    if prefix == 0:
        nothing[4] = True
    assert (out[nothing] == 0).all()
    assert torch.isnan(out[~nothing]).all()


# ---------------------------------------------------------------------------- the longest prefix
def test_attention_of_the_longest_prefix():
    """2^31 - 1 keys, most of them the same page: 24 keys to a page, five pages to a unit, so the last unit reaches past what 31 bits
    count.  The last seven keys outweigh all others; what lies behind them in their page is not a number."""
    n, page, d, n_seq = 2 ** 31 - 1, 24, 8, 33
    cache = make_cache(2, page, 1, d, torch.float16)
    cache.k.zero_()
    cache.k[1, :n % page, 0, 0], cache.k[1, n % page:], cache.v[1, n % page:] = 60.0, math.nan, math.nan
    pages = torch.zeros(-(-n // page), dtype=torch.int32, device="cuda")
    pages[-1] = 1
    q = torch.zeros((n_seq, 1, d), dtype=torch.float16, device="cuda")
    q[:, 0, 0] = 1.0
    lens = torch.zeros(n_seq, dtype=torch.int32, device="cuda")
    st = aweq.new_status()
    out = aweq.PrefixAttention(cache, pages, n, 1, n_seq, 1, 0, scale=1.0)(q, torch.zeros((n_seq, 1), dtype=torch.int32, device="cuda"), lens, st=st)
    assert aweq.read_out_of_range(st) == 0 and aweq.read_status(st)["wait_timeout"] == 0
    # exp(60) seven times beside 2^31 ones; the other keys' share is below 2^-55
    want = cache.v[1, :n % page, 0].double().mean(0)
    tol = U16[torch.float16] * (1.001 * want.abs() + 1.02 * cache.v[1, :n % page, 0].double().abs().mean(0)) + TINY[torch.float16]
    assert ((out[:, 0].double() - want).abs() <= tol + 2.0 ** -18).all()


# ---------------------------------------------------------------------------- zero-points of 31 bits
@pytest.mark.parametrize("n", [2, 100, 300])
@pytest.mark.parametrize("side", ["x", "w"])
def test_linear_sums_that_cancel_behind_large_zero_points(n, side):
    """One side's codes are all its zero-point, so the sum is zero whatever the other side's zero-point: the output is the
    bias, rounded once.  The parts of the sum reach 2^55 here, the sum's bound K reach(Zx) reach(Zw) stays below 2^62."""
    k, o = 65536, 40
    i = linear_inputs(n, k, o, 8)
    far = torch.tensor([2147483647, -2147483648, 2147483629, -2147483587], dtype=torch.int32, device="cuda")
    xz, wz = (i["xz"], i["wz"]) if side == "w" else (i["wz"], i["xz"])
    codes, steps = (i["w"], i["ws"]) if side == "w" else (i["x"], i["xs"])
    xz.copy_(far.repeat(xz.numel() // 4 + 1)[:xz.numel()])
    codes.fill_(255)
    wz.fill_(255)
    layer = aweq.LinearW8A8(i["w"], i["ws"], i["wz"], i["b"])
    out = layer(i["x"], i["xs"], i["xz"])
    assert torch.equal(out, i["b"].to(torch.float16).expand_as(out))


@pytest.mark.parametrize("n_seq,heads,prefix", [(3, 4, 70), (40, 16, 4100)])
def test_attention_with_a_scale_that_is_no_number(n_seq, heads, prefix):
    q, cache, prefix_pages, pages, lens = attention_case(n_seq, 1, heads, heads, 64, prefix, [5] * n_seq, 16, torch.float16)
    assert torch.isnan(aweq.PrefixAttention(cache, prefix_pages, prefix, heads, n_seq, scale=math.nan)(q, pages, lens)).all()
    lens.zero_()                                                   # by the prefix alone
    assert torch.isnan(aweq.PrefixAttention(cache, prefix_pages, prefix, heads, n_seq, scale=math.nan)(q, pages, lens)).all()


# ---------------------------------------------------------------------------- counts
def counted(attend, q, pages, lens):
    st = aweq.new_status()
    attend(q, pages, lens, st=st)
    assert aweq.read_status(st)["wait_timeout"] == 0
    return aweq.read_out_of_range(st)


@pytest.mark.parametrize("n_seq,h,kv,page,prefix", [(5, 4, 2, 16, 200), (5, 4, 2, 7, 200), (16, 16, 16, 16, 4100), (70, 4, 1, 12, 400),
                                                    (40, 16, 16, 16, 4100), (260, 16, 8, 128, 3700), (40, 14, 14, 256, 4096)])
def test_attention_counts_every_bad_entry_once(n_seq, h, kv, page, prefix):
    """A bad entry of the prefix's page list counts once, one of a sequence's pages once, a bad length once, whatever kernel meets it
    and however many heads, rows and keys lie behind it; entries behind the last key are not looked at."""
    q, cache, prefix_pages, pages, lens = attention_case(n_seq, 1, h, kv, 64, prefix, [(13 * b) % 60 + 1 for b in range(n_seq)], page,
                                                         torch.float16, stale=False)
    attend = aweq.PrefixAttention(cache, prefix_pages, prefix, h, n_seq, 1, 60)
    assert counted(attend, q, pages, lens) == 0
    for b in range(n_seq):
        pages[b, -(-int(lens[b]) // page):] = -1
    assert counted(attend, q, pages, lens) == 0
    attend.prefix_pages[0], attend.prefix_pages[-1] = -5, cache.n_pages
    assert counted(attend, q, pages, lens) == 2
    pages[3, 0], pages[4, 0] = cache.n_pages + 3, -2
    assert counted(attend, q, pages, lens) == 4
    lens[0], lens[1] = 61, -1
    # (the first sequence, of one key before, now reaches entries that were never given out)
    assert counted(attend, q, pages, lens) == 6 + -(-60 // page) - 1


@pytest.mark.parametrize("n_seq,prefix", [(3, 0), (3, 50), (40, 4100)])
def test_attention_counts_lengths_where_no_own_keys_are_allowed(n_seq, prefix):
    q, cache, prefix_pages, pages, lens = attention_case(n_seq, 1, 16, 16, 64, prefix, [3] * n_seq, 16, torch.float16, stale=False)
    attend = aweq.PrefixAttention(cache, prefix_pages, prefix, 16, n_seq, 1, max_own=0)
    assert counted(attend, q, pages, lens) == n_seq
    assert counted(attend, q, pages, torch.zeros_like(lens)) == 0


# ---------------------------------------------------------------------------- rows without a pitch
def test_one_row_has_no_pitch():
    """A single row cut from a matrix of any width."""
    i = linear_inputs(1, 64, 24, 2)
    layer = aweq.LinearW8A8(i["w"], i["ws"], i["wz"], i["b"])
    want = layer(i["x"], i["xs"], i["xz"])
    wide = torch.zeros((3, 101), dtype=torch.uint8, device="cuda")
    wide[:1, :64] = i["x"]
    assert torch.equal(layer(wide[:1, :64], i["xs"], i["xz"]), want)
    out = torch.empty_like(want)
    aweq.aweq_linear_w8a8(wide[:1, :64], i["xs"], i["xz"], aweq.PER_ROW, i["w"], i["ws"], i["wz"], layer.w_sum, aweq.PER_ROW, i["b"], out)
    assert torch.equal(out, want)
    q, cache, prefix_pages, pages, lens = attention_case(1, 1, 4, 2, 64, 40, [20], 16, torch.float16)
    attend = aweq.PrefixAttention(cache, prefix_pages, 40, 4, 1)
    want = attend(q, pages, lens)
    row, row_out = torch.zeros((2, 301), dtype=torch.float16, device="cuda"), torch.zeros((2, 259), dtype=torch.float16, device="cuda")
    row[:1, :256] = q.flatten(1)
    attend(row[:1, :256], pages, lens, row_out[:1, :256])
    assert torch.equal(row_out[:1, :256], want.flatten(1))
    # a pool of one page, of one token a page, of one head
    buf = torch.randn((1 << 16,), generator=gen(3), device="cuda").to(torch.float16)
    for shape, stride in [((1, 8, 2, 64), (1027, 128, 64, 1)), ((8, 1, 2, 64), (128, 3, 64, 1)), ((4, 8, 1, 64), (512, 64, 77, 1))]:
        odd = aweq.KVCache(buf.as_strided(shape, stride), buf.as_strided(shape, stride, 4096))
        even = aweq.KVCache(*(torch.empty(shape, dtype=torch.float16, device="cuda").copy_(t) for t in (odd.k, odd.v)))
        qq = torch.randn((1, 2, 64), generator=gen(4), device="cuda").to(torch.float16)
        table = torch.zeros((1, 8), dtype=torch.int32, device="cuda")
        one = torch.ones(1, dtype=torch.int32, device="cuda")
        outs = [aweq.PrefixAttention(c, None, 0, 2, 1)(qq, table, one) for c in (odd, even)]
        assert torch.equal(*outs)


def test_page_tables_of_overlapping_rows_are_refused():
    """One row for all sequences by a stride of zero: a table has a row for each."""
    q, cache, prefix_pages, pages, lens = attention_case(3, 1, 4, 2, 64, 0, [20, 20, 20], 16, torch.float16, stale=False)
    for table in (pages[:1].expand(3, -1), pages.flatten().as_strided((3, 3), (1, 1))):
        with pytest.raises(aweq.AweqError) as e:
            aweq.PrefixAttention(cache, None, 0, 4, 3)(q, table, lens)
        assert e.value.code == 3
        with pytest.raises(aweq.AweqError) as e:
            aweq.aweq_kv_append(cache, table, q[:, :2], q[:, :2], lens)
        assert e.value.code == 3


# ---------------------------------------------------------------------------- launches that follow one another
def test_attention_long_prefix_on_another_stream_and_in_a_graph():
    """The kernel of the own keys starts before the prefix's has ended: lengths, queries and pages that change from call to call, and
    calls that replay from a graph."""
    q, cache, prefix_pages, pages, lens = attention_case(40, 2, 16, 16, 64, 4100, [20 + b for b in range(40)], 16, torch.float16, stale=False)
    attend = aweq.PrefixAttention(cache, prefix_pages, 4100, 16, 40, 2)
    want = attend(q, pages, lens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = attend(q, pages, lens)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    out, graph = torch.zeros_like(want), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        attend(q, pages, lens, out)
    for step in range(5):
        lens.sub_(3)
        q.copy_(q.flip(0))
        pages.copy_(pages.flip(0))
        graph.replay()
        assert torch.equal(out, attend(q, pages, lens))


@pytest.mark.parametrize("n_seq,prefix", [(40, 4100), (20, 4100), (5, 100)])
def test_append_and_attention_in_a_row(n_seq, prefix):
    """Steps that are issued without waiting for one another give what the same steps give one by one: each reads the keys that
    the call before it has just stored, and queries that have just been turned."""
    h, d, page, steps = 16, 64, 16, 24
    q, cache, prefix_pages, pages, lens = attention_case(n_seq, 1, h, h, d, prefix, [steps] * n_seq, page, torch.float16, stale=False)
    table = aweq.aweq_rope_table(d, prefix + steps)
    attend = aweq.PrefixAttention(cache, prefix_pages, prefix, h, n_seq)
    g = gen(23)
    tokens = torch.randn((steps, 3, n_seq, h, d), generator=g, device="cuda").to(torch.float16)
    pos = [torch.full((n_seq,), prefix + t, dtype=torch.int32, device="cuda") for t in range(steps)]
    own = [torch.full((n_seq,), t + 1, dtype=torch.int32, device="cuda") for t in range(steps)]
    blank = cache.k.clone(), cache.v.clone()
    turned, runs = torch.empty_like(q), []
    for wait in (True, False):
        cache.k.copy_(blank[0])
        cache.v.copy_(blank[1])
        outs = [torch.empty_like(q) for _ in range(steps)]
        torch.cuda.synchronize()
        for t in range(steps):
            aweq.aweq_kv_append(cache, pages, tokens[t, 1], tokens[t, 2], pos[t], first=prefix, table=table, q=tokens[t, 0], q_out=turned)
            if wait:
                torch.cuda.synchronize()
            attend(turned, pages, own[t], outs[t])
            if wait:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        runs.append(torch.stack(outs))
    assert torch.equal(*runs)
    want, mag, reach = attention_reference(turned, cache, prefix_pages, prefix, pages, own[-1], 1, d ** -0.5)
    attention_close(runs[1][-1], want, mag, reach, prefix + steps, d, torch.float16)


@pytest.mark.parametrize("n_q", [128, 257, 500])
@pytest.mark.parametrize("h,kv,prefix", [(4, 4, 0), (8, 2, 130), (16, 16, 4100)])
def test_attention_of_prompts(n_q, h, kv, prefix):
    """All of a prompt's tokens at once, with and without something before them."""
    attention_check(2, n_q, h, kv, 64, prefix, [n_q, n_q + 19], 16, torch.float16)
