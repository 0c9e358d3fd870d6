"""Running a calibrated layer: the 8-bit product, the paged append with rotation and the attention
over a shared prefix, each against its definition in binary64.

Tolerances follow from the arithmetic the header states.  With u = 2^-11 (fp16) or 2^-8 (bf16) for the
one rounding to 16 bits and 2^-25 for fp16 results below the normal range:
  product    the sum is exact; its conversion, two multiplications and an addition in binary32 lose at
             most 4 * 2^-24 of the terms;
  rotation   cos and sin are rounded once, two products and a sum in binary32: 4 * 2^-24 (|x| + |y|);
  attention  a probability is off by its score's error (head_dim products added in binary32, 2^-23
             each at worst), a few 2^-22 of the exponential and the rescalings, and by u where it is
             rounded for the product with v; the output is their mean over |v|.
"""
import math

import numpy as np
import pytest
import torch

from paper_2311_01305_b200 import aweq

pytestmark = pytest.mark.gpu

U16 = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}
DTYPES = [torch.float16, torch.bfloat16]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def padded(rows, cols, ld, dtype, offset=0, fill=0):
    """A [rows x cols] view with row pitch ld that starts `offset` elements into a sentinel-filled buffer,
    and a check that nothing around the view has changed."""
    buf = torch.full((offset + rows * ld + 64,), fill, dtype=dtype, device="cuda")
    view = buf.as_strided((rows, cols), (ld, 1), offset)
    before = buf.clone()

    def check():
        after = buf.clone()
        after.as_strided((rows, cols), (ld, 1), offset).copy_(before.as_strided((rows, cols), (ld, 1), offset))
        assert torch.equal(after.view(torch.uint8), before.view(torch.uint8)), "write outside the output"
    return view, check


# ---------------------------------------------------------------------------- 8-bit product
def linear_inputs(n, k, o, seed, zp="inside", per_tensor=False, w_per_tensor=False, bias=True, ldx=None, ldw=None, hi=256):
    g = gen(seed)
    x = torch.empty((max(n, 1), ldx or k), dtype=torch.uint8, device="cuda")[:n, :k]
    w = torch.empty((o, ldw or k), dtype=torch.uint8, device="cuda")[:, :k]
    x.copy_(torch.randint(0, hi, (n, k), generator=g, device="cuda", dtype=torch.uint8))
    w.copy_(torch.randint(0, hi, (o, k), generator=g, device="cuda", dtype=torch.uint8))
    lo, top = {"inside": (0, 256), "wide": (-3000, 3000), "huge": (-1500000, 1500000)}[zp]
    nx, nw = (1 if per_tensor else n), (1 if w_per_tensor else o)
    return dict(x=x, w=w, xs=torch.rand(nx, generator=g, device="cuda") * 0.05 + 1e-3,
                ws=torch.rand(nw, generator=g, device="cuda") * 0.001 + 1e-5,
                xz=torch.randint(lo, top, (nx,), generator=g, device="cuda", dtype=torch.int32),
                wz=torch.randint(lo, top, (nw,), generator=g, device="cuda", dtype=torch.int32),
                b=torch.randn(o, generator=g, device="cuda") if bias else None)


def linear_reference(i):
    """(y, magnitude of the terms joined in binary32), binary64."""
    acc = (i["x"].double() - i["xz"].double()[:, None]) @ (i["w"].double() - i["wz"].double()[:, None]).t()
    y = acc * i["xs"].double()[:, None] * i["ws"].double()[None, :]
    b = torch.zeros((), dtype=torch.float64, device="cuda") if i["b"] is None else i["b"].double()
    return y + b, y.abs() + b.abs()


def linear_check(i, dtype, ldo=None, offset=0, layer=None):
    n, o = i["x"].shape[0], i["w"].shape[0]
    out, untouched = padded(n, o, ldo or o, dtype, offset, fill=77)
    layer = layer or aweq.LinearW8A8(i["w"], i["ws"], i["wz"], i["b"])
    st = aweq.new_status()
    assert layer(i["x"], i["xs"], i["xz"], out, st=st) is out
    untouched()
    assert aweq.read_status(st)["wait_timeout"] == 0
    y, mag = linear_reference(i)
    err = (out.double() - y).abs()
    tol = U16[dtype] * 1.001 * y.abs() + 4 * 2.0 ** -24 * mag + TINY[dtype]
    worst = (err / tol.clamp(min=1e-300)).max().item()
    assert torch.isfinite(out).all() and (err <= tol).all(), "error %.3g of what is allowed" % worst


LINEAR_SHAPES = [(1, 16, 1), (1, 768, 768), (2, 64, 16), (3, 48, 17), (8, 1040, 130), (9, 80, 33), (16, 4096, 40),
                 (17, 1040, 129), (32, 144, 64), (33, 128, 200), (48, 4096, 520), (64, 512, 64), (65, 400, 24),
                 (128, 256, 256), (129, 272, 257), (200, 768, 1000), (255, 5120, 96), (256, 128, 512), (300, 4096, 520),
                 (513, 1024, 777), (777, 16, 8), (1000, 144, 2304), (2049, 640, 1025), (31, 9216, 48), (5, 13824, 300)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,k,o", LINEAR_SHAPES)
def test_linear_shapes(n, k, o, dtype):
    linear_check(linear_inputs(n, k, o, n * 7 + k + o), dtype)


@pytest.mark.parametrize("n", [1, 2, 4, 7, 8, 12, 16, 24, 40, 63, 96, 127, 130, 192, 257, 384])
def test_linear_every_token_count_regime(n):
    linear_check(linear_inputs(n, 1536, 392, n), torch.float16)


@pytest.mark.parametrize("zp", ["inside", "wide", "huge"])
@pytest.mark.parametrize("n,k,o", [(3, 160, 40), (70, 4096, 72), (300, 1024, 264)])
def test_linear_zero_points_beyond_the_codes(n, k, o, zp):
    """Z far outside 0..255 (rows that do not contain zero): the sum leaves 32 bits."""
    linear_check(linear_inputs(n, k, o, 5, zp=zp), torch.bfloat16)


@pytest.mark.parametrize("per_tensor,w_per_tensor,bias", [(True, False, True), (False, True, False), (True, True, True)])
@pytest.mark.parametrize("n,k,o", [(1, 64, 8), (6, 256, 100), (140, 512, 300)])
def test_linear_single_pairs(n, k, o, per_tensor, w_per_tensor, bias):
    linear_check(linear_inputs(n, k, o, 9, per_tensor=per_tensor, w_per_tensor=w_per_tensor, bias=bias), torch.float16)


@pytest.mark.parametrize("n,k,o,ldx,ldw,ldo,offset", [(5, 96, 40, 112, 128, 56, 0), (5, 96, 40, 96, 96, 41, 1),
                                                      (130, 256, 250, 272, 256, 251, 3), (130, 256, 256, 256, 320, 264, 8),
                                                      (300, 128, 136, 144, 144, 139, 0)])
def test_linear_pitches_and_unaligned_outputs(n, k, o, ldx, ldw, ldo, offset):
    linear_check(linear_inputs(n, k, o, 13, ldx=ldx, ldw=ldw), torch.float16, ldo=ldo, offset=offset)


@pytest.mark.parametrize("n", [2, 24, 150])
@pytest.mark.parametrize("k", [32768, 36864, 40960, 65536])
def test_linear_longest_rows_all_codes_high(n, k):
    """All codes 255 and 254: S passes 2^31 (from 33026 on) and nearly 2^32; zero-points at both ends."""
    i = linear_inputs(n, k, 40, 3)
    i["x"].fill_(255)
    i["w"].fill_(255)
    i["x"][1::2] = 254
    i["xz"][:], i["wz"][:] = 0, 0
    i["xz"][1], i["wz"][3], i["wz"][4] = 255, 255, 128
    i["xs"].fill_(1e-3)
    i["ws"].fill_(1e-6)
    linear_check(i, torch.bfloat16)


def test_linear_layer_output_equals_the_definition_on_calibrated_codes():
    """Steps 4 and 6 of the calibration feed the product: y~ = dequant(Xq) dequant(Wq)^T + bias."""
    g = gen(21)
    X = torch.randn((96, 768), generator=g, device="cuda").to(torch.float16)
    W = (torch.randn((200, 768), generator=g, device="cuda") * 0.02).to(torch.float16)
    xq, xs, xz = torch.empty((96, 768), dtype=torch.uint8, device="cuda"), torch.empty(96, device="cuda"), torch.empty(96, dtype=torch.int32, device="cuda")
    wq, ws, wz = torch.empty((200, 768), dtype=torch.uint8, device="cuda"), torch.empty(200, device="cuda"), torch.empty(200, dtype=torch.int32, device="cuda")
    aweq.aweq_quant_act(X, None, 8, aweq.PER_ROW, None, xq, xs, xz)
    aweq.aweq_equalize_quantize(W, None, None, 8, aweq.PER_ROW, 0, wq, ws, wz)
    linear_check(dict(x=xq, w=wq, xs=xs, ws=ws, xz=xz, wz=wz, b=None), torch.float16)


def test_linear_no_tokens_and_row_sums():
    i = linear_inputs(0, 64, 24, 2)
    layer = aweq.LinearW8A8(i["w"], i["ws"], i["wz"], i["b"])
    assert torch.equal(layer.w_sum.long(), i["w"].long().sum(1))
    i["xs"], i["xz"] = torch.empty(0, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    assert layer(i["x"], i["xs"], i["xz"]).shape == (0, 24)
    wide = torch.randint(0, 256, (37, 40960), dtype=torch.uint8, device="cuda")
    assert torch.equal(aweq.aweq_code_sums(wide).long(), wide.long().sum(1))


def test_linear_infinite_step_stays_in_its_row_and_column():
    i = linear_inputs(20, 256, 48, 4)
    i["xs"][7], i["ws"][11] = math.inf, math.nan
    layer = aweq.LinearW8A8(i["w"], i["ws"], i["wz"], i["b"])
    out = layer(i["x"], i["xs"], i["xz"])
    y, _ = linear_reference(i)
    keep = torch.ones_like(y, dtype=torch.bool)
    keep[7], keep[:, 11] = False, False
    assert torch.isfinite(out[keep]).all()
    assert torch.isnan(out[:, 11]).all() and not torch.isfinite(out[7]).any()


@pytest.mark.parametrize("n", [1, 12, 50, 400])
def test_linear_repeats_bit_for_bit_on_another_stream_and_in_a_graph(n):
    i = linear_inputs(n, 2048, 328, 8)
    layer = aweq.LinearW8A8(i["w"], i["ws"], i["wz"], i["b"])
    want = layer(i["x"], i["xs"], i["xz"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = layer(i["x"], i["xs"], i["xz"])
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(want, got)
    out = torch.zeros_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(i["x"], i["xs"], i["xz"], out)
    i["x"].copy_(i["x"].flip(0))
    graph.replay()
    assert torch.equal(out, layer(i["x"], i["xs"], i["xz"]))


def test_linear_refusals():
    i = linear_inputs(4, 64, 24, 2)
    layer = aweq.LinearW8A8(i["w"], i["ws"], i["wz"], i["b"])
    with pytest.raises(ValueError):
        layer(i["x"][:, :48], i["xs"], i["xz"])
    with pytest.raises(ValueError):
        layer(i["x"], i["xs"][:3], i["xz"][:3])
    with pytest.raises(ValueError):
        layer(i["x"], i["xs"], i["xz"], torch.empty((4, 23), dtype=torch.float16, device="cuda"))
    with pytest.raises(TypeError):
        layer(i["x"], i["xs"], i["xz"], torch.empty((4, 24), device="cuda"))
    with pytest.raises(ValueError):
        layer(i["x"].cpu(), i["xs"], i["xz"])
    with pytest.raises(TypeError):
        aweq.LinearW8A8(i["w"].to(torch.int8), i["ws"], i["wz"])
    with pytest.raises(aweq.AweqError) as e:
        aweq.LinearW8A8(i["w"][:, :40].contiguous(), i["ws"], i["wz"])       # 40 is not a multiple of 16
    assert e.value.code == 2
    buf = torch.zeros(4 * 64 + 16, dtype=torch.uint8, device="cuda")
    with pytest.raises(aweq.AweqError) as e:
        layer(buf[8:8 + 256].view(4, 64), i["xs"], i["xz"])                  # base not 16-byte aligned
    assert e.value.code == 3


# ---------------------------------------------------------------------------- rotary tables
def frequencies(rd, theta=10000.0, scaling="none", factor=1.0, original_len=0.0, low=1.0, high=4.0):
    if scaling == "base":
        theta *= factor ** (rd / (rd - 2))
    f = theta ** (-np.arange(0, rd, 2) / rd)
    if scaling == "linear":
        f = f / factor
    if scaling == "bands":
        keep = np.clip((original_len * f / (2 * np.pi) - low) / (high - low), 0, 1)
        f = f * (keep + (1 - keep) / factor)
    return f


@pytest.mark.parametrize("kw", [dict(), dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0, theta=5e5),
                                dict(scaling="bands", factor=8.0, original_len=8192.0, low=1.0, high=4.0),
                                dict(scaling="bands", factor=32.0, original_len=4096.0, low=1.0, high=32.0, attention=1.25)])
@pytest.mark.parametrize("rd,n_pos", [(2, 3), (20, 100), (64, 4097), (128, 300000)])
def test_rope_table(rd, n_pos, kw):
    if kw.get("scaling") == "base" and rd < 4:
        with pytest.raises(aweq.AweqError):
            aweq.aweq_rope_table(rd, n_pos, **kw)
        return
    t = aweq.aweq_rope_table(rd, n_pos, **kw).double().cpu().numpy()
    kw = dict(kw)
    a = kw.pop("attention", 1.0)
    p = np.unique(np.linspace(0, n_pos - 1, 2000).astype(np.int64))
    angle = p[:, None] * frequencies(rd, **kw)[None, :]
    want = np.concatenate([np.cos(angle), np.sin(angle)], 1) * a
    # one rounding (2^-25 of values up to 1 or 2) plus the binary64 angle's own error, position * 2^-51
    assert np.abs(t[p] - want).max() <= a * 2.0 ** -24 + n_pos * 2.0 ** -50


# ---------------------------------------------------------------------------- append
def rotated(x, pos, table, interleaved):
    """binary64 rotation by the table's own entries: (result, |x| + |y| of each element's pair)."""
    y = x.double()
    mag = torch.zeros_like(y)
    if table is None:
        return y, mag
    rd = table.shape[1]
    cs = table.double()[pos.long().clamp(0, table.shape[0] - 1)][:, None, :]
    c, s = cs[..., :rd // 2], cs[..., rd // 2:]
    i = torch.arange(rd // 2, device="cuda")
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rd // 2)
    xa, xb = y[..., a].clone(), y[..., b].clone()
    y[..., a], y[..., b] = xa * c - xb * s, xa * s + xb * c
    mag[..., a] = mag[..., b] = xa.abs() + xb.abs()
    return y, mag


def close_rotation(got, want, mag, dtype):
    err = (got.double() - want).abs()
    tol = torch.where(mag > 0, U16[dtype] * 1.001 * want.abs() + 4 * 2.0 ** -24 * mag + TINY[dtype], torch.zeros_like(mag))
    assert (err <= tol).all(), "off by %.3g" % (err - tol).max().item()


def make_cache(n_pages, page, kv, d, dtype, layout="tokens", seed=0):
    g = gen(seed)
    if layout == "heads":                                          # tokens inside heads
        k = torch.randn((n_pages, kv, page, d), generator=g, device="cuda").to(dtype).transpose(1, 2)
        v = torch.randn((n_pages, kv, page, d), generator=g, device="cuda").to(dtype).transpose(1, 2)
    elif layout == "joint":                                        # keys and values of a page side by side
        kv_ = torch.randn((n_pages, 2, page, kv, d), generator=g, device="cuda").to(dtype)
        k, v = kv_[:, 0], kv_[:, 1]
    else:
        k = torch.randn((n_pages, page, kv, d), generator=g, device="cuda").to(dtype)
        v = torch.randn((n_pages, page, kv, d), generator=g, device="cuda").to(dtype)
    return aweq.KVCache(k, v)


def append_check(n_seq, new, h, kv, d, rd, interleaved, page, dtype, layout="tokens", first=0, before=0, offset=0, seed=1,
                 use_seq=True, in_place=False, with_q=True):
    """Tokens `first - before ..` of every sequence: those below `first` belong to the prefix."""
    g = gen(seed)
    per_seq = (new + page - 1) // page + 1
    cache = make_cache(n_seq * per_seq + 2, page, kv, d, dtype, layout, seed)
    pages = torch.randperm(cache.n_pages, generator=g, device="cuda")[:n_seq * per_seq].view(n_seq, per_seq).to(torch.int32)
    seq = torch.arange(n_seq, device="cuda", dtype=torch.int32).repeat_interleave(new)
    pos = (first - before + torch.arange(new, device="cuda", dtype=torch.int32)).repeat(n_seq)
    if use_seq:
        mix = torch.randperm(seq.numel(), generator=g, device="cuda")
        seq, pos = seq[mix].contiguous(), pos[mix].contiguous()
    n = seq.numel()
    width = (h + 2 * kv) * d
    store = torch.zeros(offset + n * (width + offset), dtype=dtype, device="cuda")
    qkv = store.as_strided((n, width), (width + offset, 1), offset)
    qkv.copy_(torch.randn((n, width), generator=g, device="cuda"))
    q, k, v = (t.unflatten(1, (-1, d)) for t in qkv.split([h * d, kv * d, kv * d], 1))
    table = aweq.aweq_rope_table(rd, first + new + 3) if rd else None
    want_k, want_v = cache.k.double(), cache.v.double()
    mag_k = torch.zeros_like(want_k)
    stored = pos.long() >= first
    at = pos.long()[stored] - first
    page_id = pages[seq.long()[stored], at // page].long()
    rk, mk = rotated(k, pos, table, interleaved)
    want_k[page_id, at % page], mag_k[page_id, at % page] = rk[stored], mk[stored]
    want_v[page_id, at % page] = v.double()[stored]
    want_q, mag_q = rotated(q, pos, table, interleaved)
    q_out = q if in_place else torch.full_like(q, 9.0, memory_format=torch.contiguous_format)
    st = aweq.new_status()
    aweq.aweq_kv_append(cache, pages, k, v, pos, seq=seq if use_seq else None, first=first, table=table,
                        interleaved=interleaved, q=q if with_q else None, q_out=q_out if with_q else None, st=st)
    assert aweq.read_out_of_range(st) == 0
    close_rotation(cache.k, want_k, mag_k, dtype)
    assert torch.equal(cache.v.double(), want_v)
    if with_q:
        close_rotation(q_out, want_q, mag_q, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("h,kv,d,rd", [(4, 4, 64, 64), (6, 2, 128, 128), (3, 1, 64, 32), (2, 2, 80, 20), (5, 5, 8, 2),
                                       (1, 1, 256, 256), (4, 2, 96, 0), (2, 1, 24, 10), (3, 3, 72, 8), (9, 3, 128, 16)])
def test_append_head_shapes(h, kv, d, rd, interleaved, dtype):
    append_check(3, 21, h, kv, d, rd, interleaved, 8, dtype)


@pytest.mark.parametrize("layout", ["tokens", "heads", "joint"])
@pytest.mark.parametrize("page", [1, 7, 16, 64])
def test_append_pages_and_layouts(page, layout):
    append_check(4, 33, 4, 2, 64, 64, False, page, torch.bfloat16, layout)
    append_check(2, 1, 4, 4, 128, 64, True, page, torch.float16, layout)


@pytest.mark.parametrize("n_seq,new", [(1, 1), (64, 1), (1, 1000), (257, 3)])
def test_append_batches(n_seq, new):
    append_check(n_seq, new, 8, 2, 128, 128, False, 16, torch.float16)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("offset", [1, 2, 4, 8])
def test_append_unaligned_rows(offset, interleaved):
    append_check(3, 9, 4, 2, 64, 32, interleaved, 16, torch.float16, offset=offset)


def test_append_one_token_per_sequence_without_seq_and_in_place():
    append_check(17, 1, 4, 4, 64, 64, False, 16, torch.float16, use_seq=False)
    append_check(5, 6, 4, 2, 64, 64, False, 16, torch.bfloat16, in_place=True)
    append_check(5, 6, 4, 2, 64, 64, True, 16, torch.bfloat16, in_place=True)
    append_check(5, 6, 4, 2, 64, 48, True, 16, torch.bfloat16, with_q=False)


def test_append_tokens_of_the_prefix_are_rotated_but_not_stored():
    append_check(3, 12, 4, 2, 64, 64, False, 8, torch.float16, first=100, before=5)


def test_append_far_positions():
    append_check(2, 40, 4, 2, 128, 128, False, 16, torch.bfloat16, first=131000)


def test_append_out_of_range_is_counted_and_harmless():
    cache = make_cache(6, 4, 2, 16, torch.float16)
    before_k, before_v = cache.k.clone(), cache.v.clone()
    table = aweq.aweq_rope_table(16, 50)
    k = torch.randn((8, 2, 16), device="cuda").to(torch.float16)
    pages = torch.tensor([[0, 1], [99, -1]], dtype=torch.int32, device="cuda")
    #       good, page beyond the row, page 99, page -1, sequence 5, sequence -1, position 50, position -1
    seq = torch.tensor([0, 0, 1, 1, 5, -1, 0, 0], dtype=torch.int32, device="cuda")
    pos = torch.tensor([3, 8, 1, 6, 2, 2, 50, -1], dtype=torch.int32, device="cuda")
    q_out = torch.full_like(k, 5.0)
    st = aweq.new_status()
    aweq.aweq_kv_append(cache, pages, k, k, pos, seq=seq, table=table, q=k, q_out=q_out, st=st)
    assert aweq.read_out_of_range(st) == 7
    want, mag = rotated(k, pos, table, False)
    close_rotation(q_out[:6], want[:6], mag[:6], torch.float16)
    assert (q_out[6:] == 0).all()
    close_rotation(cache.k[0, 3], want[0], mag[0], torch.float16)
    before_k[0, 3], before_v[0, 3] = cache.k[0, 3], k[0]
    assert torch.equal(cache.k, before_k) and torch.equal(cache.v, before_v)


def test_append_special_values_pass_through():
    cache = make_cache(2, 4, 1, 16, torch.float16)
    v = torch.zeros((2, 1, 16), dtype=torch.float16, device="cuda")
    v[0, 0, 3], v[0, 0, 5], v[1, 0, 9] = math.nan, math.inf, -math.inf
    pages = torch.tensor([[1]], dtype=torch.int32, device="cuda")
    pos = torch.tensor([0, 2], dtype=torch.int32, device="cuda")
    aweq.aweq_kv_append(cache, pages, torch.zeros_like(v), v, pos, seq=torch.zeros(2, dtype=torch.int32, device="cuda"))
    assert torch.equal(cache.v[1, [0, 2]].view(torch.int16), v.view(torch.int16))


def test_append_and_attention_refusals():
    cache = make_cache(4, 4, 2, 16, torch.float16)
    k = torch.zeros((3, 2, 16), dtype=torch.float16, device="cuda")
    pos = torch.zeros(3, dtype=torch.int32, device="cuda")
    pages = torch.zeros((3, 1), dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        aweq.aweq_kv_append(cache, pages, k.to(torch.bfloat16), k, pos)
    with pytest.raises(ValueError):
        aweq.aweq_kv_append(cache, pages, k, k[:2], pos)
    with pytest.raises(ValueError):
        aweq.aweq_kv_append(cache, pages, k, k, pos.long())
    with pytest.raises(ValueError):
        aweq.aweq_kv_append(cache, pages[:2], k, k, pos)
    with pytest.raises(ValueError):
        aweq.aweq_kv_append(cache, pages, k, k, pos, q=k[:, :, :8])
    with pytest.raises(aweq.AweqError):
        aweq.aweq_kv_append(cache, pages, k, k, pos, table=torch.zeros((4, 32), device="cuda"))     # 32 of 16
    with pytest.raises(ValueError):
        aweq.KVCache(cache.k, cache.v[:, :2])
    with pytest.raises(aweq.AweqError):
        aweq.aweq_kv_append(aweq.KVCache(cache.k[..., :12], cache.v[..., :12]), pages, k[..., :12].contiguous(),
                            k[..., :12].contiguous(), pos)
    lens = torch.ones(3, dtype=torch.int32, device="cuda")
    with pytest.raises(aweq.AweqError):
        aweq.PrefixAttention(cache, None, 0, 3, 3, 1, 4)(torch.zeros((3, 3, 16), dtype=torch.float16, device="cuda"), pages, lens)
    with pytest.raises(ValueError):
        aweq.PrefixAttention(cache, None, 0, 2, 3, 1, 4)(k, pages, lens.long())
    with pytest.raises(ValueError):
        aweq.PrefixAttention(cache, pages[:, 0][:1], 9, 2, 3, 1, 4)(k, pages, lens)                 # 3 pages are needed
    with pytest.raises(aweq.AweqError) as e:
        aweq.aweq_prefix_attention(k, cache, None, 0, pages, lens, 4, 1, 1.0, torch.empty_like(k),
                                   torch.empty(64, dtype=torch.uint8, device="cuda")[8:])
    assert e.value.code == 7


# ---------------------------------------------------------------------------- attention
def attention_reference(q, cache, prefix_pages, prefix, pages, lens, n_q, scale):
    """(out, mean |v| under the probabilities, largest sum |q k| scale of a row), binary64, one row at a time."""
    h, d, kv = q.shape[1], q.shape[2], cache.n_kv_heads
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    mag, reach = torch.zeros_like(out), torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda")
    pk = pv = torch.zeros((0, kv, d), dtype=torch.float64, device="cuda")
    if prefix:
        pk = cache.k[prefix_pages.long()].reshape(-1, kv, d)[:prefix].double()
        pv = cache.v[prefix_pages.long()].reshape(-1, kv, d)[:prefix].double()
    for b, n in enumerate(lens.tolist()):
        ids = pages[b, :-(-n // cache.page_size)].long()
        keys = torch.cat([pk, cache.k[ids].reshape(-1, kv, d)[:n].double()]).repeat_interleave(h // kv, 1)
        vals = torch.cat([pv, cache.v[ids].reshape(-1, kv, d)[:n].double()]).repeat_interleave(h // kv, 1)
        for i in range(n_q):
            t, own = b * n_q + i, max(0, n - (n_q - 1 - i))
            if prefix + own == 0:
                continue
            kk, vv = keys[:prefix + own], vals[:prefix + own]
            prod = kk * q[t].double()
            p = torch.softmax(prod.sum(-1) * scale, 0)[..., None]
            out[t], mag[t] = (p * vv).sum(0), (p * vv.abs()).sum(0)
            reach[t] = prod.abs().sum(-1).max(0).values * abs(scale)
    return out, mag, reach


def attention_case(n_seq, n_q, h, kv, d, prefix, lens, page, dtype, layout="tokens", seed=3, spread=2.0, stale=True):
    g = gen(seed)
    lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    per_seq = max(1, -(-int(lens.max()) // page)) + 1
    shared = -(-prefix // page)
    cache = make_cache(shared + n_seq * per_seq + 2, page, kv, d, dtype, layout, seed)
    order = torch.randperm(cache.n_pages, generator=g, device="cuda").to(torch.int32)
    prefix_pages, pages = order[:shared].clone(), order[shared:shared + n_seq * per_seq].view(n_seq, per_seq).clone()
    if stale:
        # whatever lies behind the last key of a page or of a sequence must not be seen
        if prefix % page:
            cache.k[prefix_pages[-1].long(), prefix % page:] = math.nan
            cache.v[prefix_pages[-1].long(), prefix % page:] = math.inf
        for b, n in enumerate(lens.tolist()):
            used = -(-n // page)
            if n % page:
                cache.k[pages[b, used - 1].long(), n % page:] = math.inf
                cache.v[pages[b, used - 1].long(), n % page:] = math.nan
            pages[b, used:] = -1
        for p in order[shared + n_seq * per_seq:].tolist():
            cache.k[p], cache.v[p] = math.nan, math.nan
    q = (spread * torch.randn((n_seq * n_q, h, d), generator=g, device="cuda")).to(dtype)
    return q, cache, prefix_pages, pages, lens


def attention_check(n_seq, n_q, h, kv, d, prefix, lens, page, dtype, layout="tokens", seed=3, spread=2.0, max_own=None, scale=None):
    q, cache, prefix_pages, pages, lens = attention_case(n_seq, n_q, h, kv, d, prefix, lens, page, dtype, layout, seed, spread)
    attend = aweq.PrefixAttention(cache, prefix_pages, prefix, h, n_seq, n_q, max_own, scale)
    out, st = torch.full_like(q, 7.0), aweq.new_status()
    attend(q, pages, lens, out, st)
    assert aweq.read_out_of_range(st) == 0 and aweq.read_status(st)["wait_timeout"] == 0
    attention_close(out, *attention_reference(q, cache, prefix_pages, prefix, pages, lens, n_q, attend.scale),
                    prefix + int(lens.max()), d, dtype)
    return q, cache, prefix_pages, pages, lens, attend, out


def attention_close(out, want, mag, reach, keys, d, dtype):
    rescalings = keys / 16 + 64
    off = (reach * d * 2.0 ** -23 + 2.0 ** -20 + rescalings * 2.0 ** -23)[..., None]
    tol = U16[dtype] * 1.001 * want.abs() + (U16[dtype] + 2 * off) * 1.01 * mag + TINY[dtype]
    err = (out.double() - want).abs()
    assert torch.isfinite(out).all() and (err <= tol).all(), "error %.3g of what is allowed" % (err / tol.clamp(min=1e-300)).max().item()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("h,kv,d", [(4, 4, 64), (8, 2, 128), (6, 1, 80), (16, 1, 128), (3, 3, 8), (5, 5, 96), (24, 1, 72), (40, 2, 64)])
def test_attention_head_shapes(h, kv, d, dtype):
    attention_check(3, 1, h, kv, d, 130, [1, 40, 17], 16, dtype)


@pytest.mark.parametrize("prefix", [0, 1, 15, 16, 17, 63, 64, 65, 127, 255, 1000, 4100])
@pytest.mark.parametrize("page", [16, 24])
def test_attention_prefix_lengths(prefix, page):
    attention_check(5, 1, 4, 2, 64, prefix, [0, 1, 5, 64, 130] if prefix else [1, 1, 5, 64, 130], page, torch.float16)


@pytest.mark.parametrize("layout", ["tokens", "heads", "joint"])
@pytest.mark.parametrize("page", [1, 7, 32, 128])
def test_attention_pages_and_layouts(page, layout):
    attention_check(4, 1, 8, 4, 128, 200, [3, 77, 128, 129], page, torch.bfloat16, layout)


@pytest.mark.parametrize("n_seq", [1, 2, 15, 16, 17, 33, 64, 65, 130])
@pytest.mark.parametrize("h,kv", [(2, 2), (8, 1)])
def test_attention_batches(n_seq, h, kv):
    attention_check(n_seq, 1, h, kv, 64, 300, [(7 * b) % 90 + 1 for b in range(n_seq)], 16, torch.float16)


@pytest.mark.parametrize("n_q", [2, 3, 5, 8, 17, 40])
@pytest.mark.parametrize("h,kv,prefix", [(4, 4, 70), (8, 2, 0), (6, 1, 513)])
def test_attention_several_tokens_per_sequence(n_q, h, kv, prefix):
    attention_check(3, n_q, h, kv, 64, prefix, [n_q, n_q + 50, n_q + 131], 16, torch.float16)


@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_rows_without_keys_are_zero(dtype):
    """No prefix, and fewer own keys than tokens: the first tokens see nothing."""
    q, cache, _, pages, lens, attend, out = attention_check(4, 3, 4, 2, 64, 0, [0, 1, 2, 9], 16, dtype)
    assert (out.view(4, 3, 4, 64)[0] == 0).all() and (out.view(4, 3, 4, 64)[1, :2] == 0).all()
    assert (out.view(4, 3, 4, 64)[2, 0] == 0).all() and (out.view(4, 3, 4, 64)[2, 1] != 0).any()
    attention_check(2, 1, 4, 2, 64, 40, [0, 0], 16, dtype)


def test_attention_long_own_keys_and_peaked_scores():
    attention_check(2, 1, 4, 2, 128, 77, [5000, 3], 64, torch.bfloat16)
    attention_check(3, 1, 4, 4, 64, 2000, [100, 200, 300], 16, torch.float16, spread=12.0)
    attention_check(3, 1, 4, 4, 64, 2000, [100, 200, 300], 16, torch.float16, spread=12.0, scale=-0.3)
    attention_check(3, 1, 4, 4, 64, 500, [100, 200, 300], 16, torch.float16, scale=0.0)


def test_attention_many_rows():
    """More rows per key head than any tile holds."""
    attention_check(70, 2, 16, 2, 128, 640, [(11 * b) % 60 + 2 for b in range(70)], 16, torch.bfloat16)


# A prefix of more than 32 rows per key head and three 128-key units for every SM goes to a kernel of its own.
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n_seq,n_q,h,kv,d,prefix,page", [
    (40, 1, 16, 16, 128, 4100, 16),     # one row tile, 40 of its 128 rows
    (33, 1, 16, 16, 64, 3585, 32),      # one row more than the other kernel takes; one key in the last unit
    (9, 2, 32, 4, 128, 7000, 16),       # 144 rows: two row tiles, the second of 16
    (130, 1, 8, 4, 128, 3700, 64),      # 260 rows: three tiles
    (35, 1, 15, 15, 72, 4000, 8),       # a head that is no multiple of 16
    (40, 1, 16, 16, 80, 3710, 24),      # 120 keys to a unit
    (50, 1, 12, 12, 96, 5000, 128),     # a page to a unit
    (36, 1, 14, 14, 8, 4096, 256),      # half a page to a unit, the smallest head
    (34, 1, 16, 16, 64, 4000, 192)])    # copies of 64 keys, units across pages
def test_attention_long_prefix(n_seq, n_q, h, kv, d, prefix, page, dtype):
    attention_check(n_seq, n_q, h, kv, d, prefix, [(7 * b) % 40 + n_q for b in range(n_seq)], page, dtype)


@pytest.mark.parametrize("layout", ["heads", "joint"])
def test_attention_long_prefix_layouts(layout):
    attention_check(40, 1, 16, 16, 128, 4100, [1 + b for b in range(40)], 16, torch.bfloat16, layout)


@pytest.mark.parametrize("page", [1, 12, 72, 136])
def test_attention_long_prefix_of_other_pages(page):
    """Page sizes that the tiled copies do not fit."""
    attention_check(40, 1, 16, 16, 64, 3000, [1 + b for b in range(40)], page, torch.float16)


@pytest.mark.parametrize("kw", [dict(spread=25.0), dict(spread=25.0, scale=-0.4), dict(scale=0.0), dict(spread=0.01)])
def test_attention_long_prefix_scores(kw):
    """Scores that climb far beyond a row's first maximum, a negative and a zero scale, no spread at all."""
    attention_check(40, 1, 16, 16, 128, 4100, [5] * 40, 16, torch.float16, **kw)


def test_attention_long_prefix_rising_maximum():
    """Keys that grow along the prefix: the reference maximum has to move many times."""
    q, cache, prefix_pages, pages, lens = attention_case(40, 1, 16, 16, 64, 4096, [3] * 40, 16, torch.bfloat16)
    grow = torch.linspace(0.05, 6.0, 4096, device="cuda").view(256, 16, 1, 1)
    cache.k[prefix_pages.long()] = (cache.k[prefix_pages.long()].float() * grow).to(torch.bfloat16)
    attend = aweq.PrefixAttention(cache, prefix_pages, 4096, 16, 40)
    attention_close(attend(q, pages, lens), *attention_reference(q, cache, prefix_pages, 4096, pages, lens, 1, attend.scale), 4100,
                    64, torch.bfloat16)


def test_attention_long_prefix_rows_are_independent():
    q, cache, prefix_pages, pages, lens = attention_case(40, 1, 16, 16, 64, 4100, [9] * 40, 16, torch.float16)
    attend = aweq.PrefixAttention(cache, prefix_pages, 4100, 16, 40)
    clean = attend(q, pages, lens)
    assert torch.equal(clean, attend(q, pages, lens))
    q[7, 3] = math.nan
    out = attend(q, pages, lens)
    assert torch.isnan(out[7, 3]).all()
    keep = torch.ones(40, 16, dtype=torch.bool, device="cuda")
    keep[7, 3] = False
    assert torch.equal(out[keep], clean[keep])
    # an infinite value reaches every row of its key head and no other
    cache.v[prefix_pages[100].long(), 3, 5, 11] = math.inf
    out = attend(q, pages, lens)
    assert torch.isinf(out[keep[:, 5].nonzero()[:, 0], 5, 11]).all()
    keep[:, 5] = False
    assert torch.equal(out[keep], clean[keep])


def test_attention_long_prefix_pages_out_of_range_are_counted():
    q, cache, prefix_pages, pages, lens = attention_case(40, 1, 16, 16, 64, 4100, [9] * 40, 16, torch.float16, stale=False)
    attend = aweq.PrefixAttention(cache, prefix_pages, 4100, 16, 40)
    attend.prefix_pages[3], attend.prefix_pages[200] = cache.n_pages, -1
    st = aweq.new_status()
    attend(q, pages, lens, st=st)
    assert aweq.read_out_of_range(st) >= 2 and aweq.read_status(st)["wait_timeout"] == 0


@pytest.mark.parametrize("d", [8, 40, 72, 80, 88, 104, 120])
def test_attention_many_items_of_odd_heads(d):
    """Many items to a CTA with heads that its tiles pad: what an item leaves behind must not reach the next one's padding."""
    lens = [(37 * b) % 150 for b in range(300)]
    attention_check(300, 1, 16, 16, d, 0, lens, 16, torch.bfloat16)
    attention_check(300, 1, 8, 8, d, 100, lens, 8, torch.float16)


def test_attention_many_short_sequences():
    """Many items of one or two units to a CTA, some sequences without keys, with and without a prefix."""
    lens = [(37 * b) % 200 for b in range(200)]
    attention_check(200, 1, 16, 16, 64, 0, lens, 16, torch.bfloat16)
    attention_check(200, 1, 16, 4, 128, 40, lens, 32, torch.float16)
    attention_check(200, 1, 8, 8, 128, 2500, lens, 16, torch.float16)


def test_attention_values_of_later_tokens_stay_out():
    """Infinities and NaN in the key and value of the last token: the earlier tokens do not see them."""
    q, cache, prefix_pages, pages, lens = attention_case(2, 4, 4, 2, 64, 33, [20, 65], 16, torch.float16)
    attend = aweq.PrefixAttention(cache, prefix_pages, 33, 4, 2, 4)
    clean = attend(q, pages, lens)
    for b, n in enumerate(lens.tolist()):
        cache.k[pages[b, (n - 1) // 16].long(), (n - 1) % 16] = math.inf
        cache.v[pages[b, (n - 1) // 16].long(), (n - 1) % 16] = math.nan
        cache.v[pages[b, (n - 2) // 16].long(), (n - 2) % 16, :, 5] = -math.inf
    out = attend(q, pages, lens).view(2, 4, 4, 64)
    assert torch.equal(out[:, :2], clean.view(2, 4, 4, 64)[:, :2])
    assert torch.isnan(out[:, 3]).all()
    assert torch.isinf(out[:, 2, :, 5]).all() and torch.equal(out[:, 2, :, 6:], clean.view(2, 4, 4, 64)[:, 2, :, 6:])


def test_attention_one_sequences_nan_stays_its_own():
    q, cache, prefix_pages, pages, lens = attention_case(6, 1, 4, 2, 64, 90, [20, 30, 5, 64, 1, 9], 16, torch.bfloat16)
    attend = aweq.PrefixAttention(cache, prefix_pages, 90, 4, 6)
    clean = attend(q, pages, lens)
    q[2] = math.nan
    cache.v[pages[4, 0].long(), 0] = math.inf
    out = attend(q, pages, lens)
    assert torch.isnan(out[2]).all() and not torch.isfinite(out[4]).any()
    keep = [0, 1, 3, 5]
    assert torch.equal(out[keep], clean[keep])


def test_attention_lengths_and_pages_out_of_range_are_counted():
    q, cache, prefix_pages, pages, lens = attention_case(4, 1, 2, 2, 64, 40, [20, 30, 5, 16], 16, torch.float16, stale=False)
    attend = aweq.PrefixAttention(cache, prefix_pages, 40, 2, 4, max_own=30)
    clean = attend(q, pages, lens)
    bad = torch.tensor([20, 31, -4, 16], dtype=torch.int32, device="cuda")       # the second is clamped to 30
    st = aweq.new_status()
    out = attend(q, pages, bad, st=st)
    assert aweq.read_out_of_range(st) >= 2
    assert torch.equal(out[[0, 1, 3]], clean[[0, 1, 3]])
    want = attend(q, pages, bad.clamp(min=0, max=30))
    assert torch.equal(out, want)
    pages[0, 0], pages[3, 0] = cache.n_pages, -7
    st = aweq.new_status()
    out = attend(q, pages, lens, st=st)
    assert aweq.read_out_of_range(st) >= 2 and torch.equal(out[[1, 2]], clean[[1, 2]])


def test_attention_strided_rows_another_stream_and_a_graph():
    q, cache, prefix_pages, pages, lens = attention_case(5, 2, 4, 2, 64, 100, [20, 30, 5, 64, 2], 16, torch.float16)
    attend = aweq.PrefixAttention(cache, prefix_pages, 100, 4, 5, 2)
    want = attend(q, pages, lens)
    wide = torch.zeros((10, 8 * 64), dtype=torch.float16, device="cuda")
    wide_out = torch.full((10, 6 * 64), 3.0, dtype=torch.float16, device="cuda")
    wide[:, 64:320] = q.flatten(1)
    attend(wide[:, 64:320], pages, lens, wide_out[:, 128:384])
    assert torch.equal(wide_out[:, 128:384], want.flatten(1))
    assert (wide_out[:, :128] == 3).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = attend(q, pages, lens)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    out, graph = torch.zeros_like(want), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        attend(q, pages, lens, out)
    lens.fill_(2)
    graph.replay()
    assert torch.equal(out, attend(q, pages, lens))


def test_offsets_beyond_32_bits():
    """A pool whose last pages lie more than 2^31 elements (and 2^32 bytes) in."""
    n_pages, page, kv, d = 33000, 64, 8, 128
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB free")
    k = torch.empty((n_pages, page, kv, d), dtype=torch.float16, device="cuda")
    cache = aweq.KVCache(k, torch.empty_like(k))
    g = gen(5)
    prefix_pages = torch.tensor([32999, 7], dtype=torch.int32, device="cuda")
    pages = torch.tensor([[32998, 32990], [32767, 0]], dtype=torch.int32, device="cuda")
    for p in prefix_pages.tolist():
        cache.k[p] = torch.randn((page, kv, d), generator=g, device="cuda").to(torch.float16)
        cache.v[p] = torch.randn((page, kv, d), generator=g, device="cuda").to(torch.float16)
    new = torch.randn((140, kv, d), generator=g, device="cuda").to(torch.float16)
    seq = torch.tensor([0] * 70 + [1] * 70, dtype=torch.int32, device="cuda")
    pos = torch.arange(70, dtype=torch.int32, device="cuda").repeat(2)
    aweq.aweq_kv_append(cache, pages, new, new, pos, seq=seq)
    assert torch.equal(cache.v[32998], new[:64]) and torch.equal(cache.k[32990, :6], new[64:70])
    lens = torch.tensor([70, 70], dtype=torch.int32, device="cuda")
    q = torch.randn((2, kv, d), generator=g, device="cuda").to(torch.float16)
    attend = aweq.PrefixAttention(cache, prefix_pages, 100, kv, 2)
    attention_close(attend(q, pages, lens), *attention_reference(q, cache, prefix_pages, 100, pages, lens, 1, attend.scale), 170,
                    d, torch.float16)
