"""Microscaled 4-bit floating point: quantisation, what it stands for, and the layer on it.

Codes and scales are compared bit by bit with the header's formulas in binary32, and what they stand for with
the nearest values in binary64.  The layer is compared with the binary64 product of what codes and scales stand
for: with operands whose partial sums are exact in binary32 the output has to be that product rounded once;
else a sum of K terms in binary32 loses at most K 2^-23 of the terms' magnitudes, the steps and the bias
4 * 2^-24, and the rounding to 16 bits half a step.
"""
import pytest
import torch

from paper_2311_01305_b200 import aweq

pytestmark = pytest.mark.gpu

U16 = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}
DTYPES = [torch.float16, torch.bfloat16]
FORMATS = ["e8m0", "e4m3"]
BLOCK = {"e8m0": 32, "e4m3": 16}
LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def activations(rows, cols, dtype, seed):
    g = gen(seed)
    x = torch.randn((rows, cols), generator=g, device="cuda") * torch.exp(2.0 * torch.randn(cols, generator=g, device="cuda"))
    return x.to(dtype), torch.exp(0.5 * torch.randn(cols, generator=g, device="cuda"))


def levels(dtype=torch.float32):
    return torch.tensor(LEVELS + [-v for v in LEVELS], dtype=dtype, device="cuda")


def elements(codes):
    """e2m1 values of packed codes, [rows x cols]."""
    return levels()[torch.stack([codes & 15, codes >> 4], -1).flatten(1).long()]


def scale_bytes(scales, rows, cols, fmt):
    """The scale bytes [rows x blocks] out of their tiles."""
    tiles = -(-cols // 256) * (2 if fmt == "e8m0" else 4)
    r, k = torch.arange(rows, device="cuda")[:, None], torch.arange(cols // BLOCK[fmt], device="cuda")[None, :]
    return scales[((r // 128) * tiles + k // 4) * 512 + 16 * (r % 32) + 4 * (r % 128 // 32) + k % 4]


def formulas(x, scale, fmt):
    """(elements, scale bytes, row steps) of the header's formulas in binary32."""
    v = x.float() if scale is None else x.float() * scale
    v = v.unflatten(1, (-1, BLOCK[fmt]))
    top = v.abs().amax(-1)
    if fmt == "e8m0":
        e = torch.where(top > 0, torch.frexp(top).exponent - 3, -127).clamp(min=-127)
        y, byte, row = torch.ldexp(v, -e[..., None]), (e + 127).to(torch.uint8), None
    else:
        row = top.amax(-1) * (torch.ones((), device="cuda") / torch.full((), 2688.0, device="cuda"))
        byte = (top / (6.0 * row)[:, None]).nan_to_num(0.0).to(torch.float8_e4m3fn)
        step = byte.float() * row[:, None]
        y = torch.where(step[..., None] >= 2.0 ** -126, v * (1.0 / step)[..., None], 0.0)
        byte = torch.where(step >= 2.0 ** -126, byte.view(torch.uint8), 0)
    grid = levels()[:8]
    mid = (grid[1:] + grid[:-1]) / 2
    lo, hi = torch.bucketize(y.abs(), mid), torch.bucketize(y.abs(), mid, right=True)
    return torch.copysign(grid[torch.where(hi % 2 == 0, hi, lo)], y).flatten(1), byte, row


def steps(byte, row, fmt):
    """What the scales of [rows x blocks] stand for, binary64."""
    s = torch.exp2(byte.double() - 127) if fmt == "e8m0" else byte.view(torch.float8_e4m3fn).double() * row.double()[:, None]
    return s


def stands_for(q):
    byte = scale_bytes(q.scales, q.rows, q.cols, q.fmt)
    return (elements(q.codes).double().unflatten(1, (-1, BLOCK[q.fmt])) * steps(byte, q.row_step, q.fmt)[..., None]).flatten(1)


def quantised(x, scale, fmt, **kw):
    return aweq.MX4(x.shape[0], x.shape[1], fmt).quantise(x, scale, **kw)


SHAPES = [(1, 32), (1, 768), (2, 64), (3, 96), (7, 224), (16, 5120), (33, 288), (127, 256), (128, 512), (129, 544), (300, 4096), (5, 11008),
          (4, 16384), (3, 16416), (3, 36864), (2, 65536), (1000, 160)]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_codes_and_scales(rows, cols, dtype, fmt):
    x, m = activations(rows, cols, dtype, rows + cols)
    for scale in (m, None):
        q = quantised(x, scale, fmt)
        elem, byte, row = formulas(x, scale, fmt)
        assert torch.equal(scale_bytes(q.scales, rows, cols, fmt), byte)
        assert torch.equal(elements(q.codes), elem)
        if row is not None:
            assert torch.equal(q.row_step, row)
        # columns up to a whole group of 256: zero scales
        pad = scale_bytes(q.scales, rows, -(-cols // 256) * 256, fmt)[:, cols // BLOCK[fmt]:]
        assert (pad == 0).all()
        for out_dtype in DTYPES:
            v = q.values(dtype=out_dtype)
            want = elem.unflatten(1, (-1, BLOCK[fmt])) * (torch.exp2(byte.float() - 127) if fmt == "e8m0" else byte.view(torch.float8_e4m3fn).float())[..., None]
            want = want.flatten(1) if row is None else want.flatten(1) * row[:, None]
            assert torch.equal(v, want.to(out_dtype))


@pytest.mark.parametrize("fmt", FORMATS)
def test_nearest_value(fmt):
    """Every element is within half a step of the grid of its block (the top of the grid: what saturates)."""
    x, m = activations(64, 2048, torch.bfloat16, 3)
    q = quantised(x, m, fmt)
    v = x.double() * m.double()
    step = steps(scale_bytes(q.scales, 64, 2048, fmt), q.row_step, fmt).repeat_interleave(BLOCK[fmt], 1)
    a = v.abs() / step
    half = torch.where(a <= 2, 0.25, torch.where(a <= 4, 0.5, torch.where(a <= 6, 1.0, a - 6)))
    err = (stands_for(q) - v).abs() / step
    assert (err <= half + 1e-5).all() and a.max() < 8


@pytest.mark.parametrize("fmt", FORMATS)
def test_ties_zeros_and_the_ends_of_the_range(fmt):
    # ties: multiples of a half step of a block whose largest is 6 (and of a row whose scales are 1, 448 in the first block)
    x = torch.zeros((4, 64), device="cuda")
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], device="cuda")
    x[0, 32:40], x[0, 40:48] = ties, -ties
    if fmt == "e4m3":
        x[0, 0] = 2688.0
        x[0, 48:56] = ties * 2
    x[2] = 1e-38
    x[3, 0], x[3, 32] = 3e38, 1e-30
    x = x.to(torch.bfloat16)
    q = quantised(x, None, fmt)
    elem, byte, row = formulas(x, None, fmt)
    assert torch.equal(elements(q.codes), elem) and torch.equal(scale_bytes(q.scales, 4, 64, fmt), byte)
    assert torch.equal(elements(q.codes)[0, 32:40], torch.tensor([0, 1, 1, 2, 2, 4, 4, 6.0], device="cuda"))
    assert (q.values()[1] == 0).all() and torch.isfinite(q.values()).all()
    if fmt == "e8m0":
        assert scale_bytes(q.scales, 4, 64, fmt)[1].eq(0).all()


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("fmt", FORMATS)
def test_blocks_that_are_no_numbers(fmt, bad):
    x, _ = activations(5, 320, torch.float16, 9)
    x.clamp_(-100, 100)
    good = quantised(x, None, fmt).values()
    x[1, 70] = bad
    st = aweq.new_status()
    q = quantised(x, None, fmt, st=st)
    hit = torch.zeros((5, 320), dtype=torch.bool, device="cuda")
    if fmt == "e8m0":
        hit[1, 64:96] = True
    else:
        hit[1] = True
    v = q.values()
    assert torch.isnan(v[hit]).all() and torch.equal(v[~hit], good[~hit])
    assert aweq.read_status(st)["nonfinite"] == 1
    # and in a product: every output of that token, no other
    w, _ = activations(48, 320, torch.float16, 10)
    for n in (5, 300):
        xs = torch.cat([x, x[2:3].expand(n - 5, -1)]).contiguous()
        y = aweq.LinearMX4(w, fmt)(quantised(xs, None, fmt))
        assert torch.isnan(y[1]).all() and torch.isfinite(y[[i for i in range(n) if i != 1]]).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_bias_correction_sums(fmt):
    """Row sums of (value - v) mu in binary32: K additions of terms that carry three roundings."""
    w, s = activations(130, 1056, torch.bfloat16, 21)
    mu = torch.randn(1056, generator=gen(2), device="cuda")
    eps = torch.empty(130, device="cuda")
    q = quantised(w, s, fmt, mu=mu, epsmu=eps)
    v = (w.float() * s).double()
    term = (stands_for(q) - v) * mu.double()
    tol = 1056 * 2.0 ** -24 * term.abs().sum(1) + 4 * 2.0 ** -24 * (v * mu.double()).abs().sum(1)
    assert ((eps.double() - term.sum(1)).abs() <= tol).all()
    again = torch.empty_like(eps)
    quantised(w, s, fmt, mu=mu, epsmu=again)
    assert torch.equal(again, eps)
    bias = torch.randn(130, generator=gen(3), device="cuda")
    assert torch.equal(aweq.LinearMX4(w, fmt, s, bias, mu).bias, bias - eps) and torch.equal(aweq.LinearMX4(w, fmt, s, None, mu).bias, -eps)


def exact_operand(rows, cols, fmt, seed):
    """16-bit rows that quantise without a rounding and whose products have few bits."""
    g = gen(seed)
    blocks = cols // BLOCK[fmt]
    e = levels()[torch.randint(0, 16, (rows, blocks, BLOCK[fmt]), generator=g, device="cuda")]
    e[:, :, 0] = 6.0
    if fmt == "e8m0":
        s = torch.exp2(torch.randint(0, 2, (rows, blocks), generator=g, device="cuda").float() - 3)
    else:
        s = 64.0 * torch.randint(1, 8, (rows, blocks), generator=g, device="cuda").float()
        s[torch.arange(rows, device="cuda"), torch.arange(rows, device="cuda") % blocks] = 448.0
        s = s * 2.0 ** -9
    return (e * s[..., None]).flatten(1)


LINEAR_SHAPES = [(1, 32, 1), (1, 768, 768), (2, 64, 16), (3, 96, 17), (8, 1056, 130), (9, 160, 33), (16, 2048, 40), (17, 1056, 129), (32, 288, 64),
                 (33, 128, 200), (48, 2048, 520), (64, 512, 64), (65, 416, 24), (100, 256, 1000), (128, 256, 256), (129, 544, 257), (200, 768, 1000),
                 (255, 2048, 96), (256, 128, 512), (257, 1024, 520), (300, 2048, 520), (513, 1024, 777), (777, 32, 8), (1000, 288, 2304),
                 (2049, 640, 1025), (700, 768, 4104)]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,k,o", LINEAR_SHAPES)
def test_products_that_are_exact(n, k, o, dtype, fmt):
    """Partial sums are multiples of a unit and below 2^24 of it: any order gives the same, and the output is it, rounded once."""
    x, w = exact_operand(n, k, fmt, n + k), exact_operand(o, k, fmt, o)
    layer, xq, st = aweq.LinearMX4(w.to(dtype), fmt), quantised(x.to(dtype), None, fmt), aweq.new_status()
    assert torch.equal(stands_for(xq), x.double()) and torch.equal(stands_for(layer.weight), w.double())
    y = layer(xq, dtype=dtype, st=st)
    want = x.double() @ w.double().t()
    assert torch.equal(y, want.to(dtype)) and aweq.read_status(st)["wait_timeout"] == 0


def layer_check(n, k, o, dtype, fmt, bias, ldo=None, offset=0, seed=0):
    x, rinv = activations(n, k, dtype, seed + 1)
    w, s = activations(o, k, dtype, seed + 2)
    b = torch.randn(o, generator=gen(seed), device="cuda") if bias else None
    layer, xq = aweq.LinearMX4(w, fmt, s, b), quantised(x, rinv, fmt)
    buf = torch.full((offset + n * (ldo or o) + 64,), 7.0, dtype=dtype, device="cuda")
    out = buf.as_strided((n, o), (ldo or o, 1), offset)
    assert layer(xq, out) is out
    xv, wv = stands_for(xq), stands_for(layer.weight)
    y, mag = xv @ wv.t(), xv.abs() @ wv.abs().t()
    bd = torch.zeros((), dtype=torch.float64, device="cuda") if b is None else b.double()
    tol = U16[dtype] * 1.001 * (y + bd).abs() + k * 2.0 ** -23 * mag + 4 * 2.0 ** -24 * (mag + bd.abs()) + TINY[dtype]
    big = (y + bd).abs() > (65000 if dtype == torch.float16 else 1e38)
    assert ((out.double() - y - bd).abs() <= tol)[~big].all()
    buf.as_strided((n, o), (ldo or o, 1), offset).fill_(7.0)
    assert (buf == 7.0).all(), "write outside the output"


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n,k,o", [(1, 4096, 4096), (5, 13824, 300), (24, 4096, 4104), (100, 5120, 640), (256, 9216, 256), (400, 5120, 1536), (31, 36864, 48)])
def test_layers(n, k, o, fmt):
    layer_check(n, k, o, torch.bfloat16, fmt, True)
    layer_check(n, k, o, torch.float16, fmt, False, seed=5)


@pytest.mark.parametrize("n,k,o,ldo,offset", [(5, 96, 40, 56, 0), (5, 96, 40, 41, 1), (130, 256, 250, 251, 3), (300, 256, 250, 251, 3), (300, 256, 256, 264, 8),
                                              (300, 128, 136, 139, 0), (20, 64, 131, 132, 4)])
def test_pitches_and_unaligned_outputs(n, k, o, ldo, offset):
    layer_check(n, k, o, torch.float16, "e8m0", True, ldo, offset)


def test_inputs_with_a_pitch_and_scales_left_alone():
    x, m = activations(40, 640, torch.float16, 4)
    q, whole = quantised(x[:, 64:576], m[64:576].contiguous(), "e8m0"), quantised(x[:, 64:576].contiguous(), m[64:576].contiguous(), "e8m0")
    assert torch.equal(q.codes, whole.codes)
    q = aweq.MX4(40, 640, "e4m3")
    q.scales.fill_(0xAB)
    q.quantise(x, m)
    rows = torch.zeros(128, dtype=torch.bool, device="cuda")
    rows[:40] = True
    left = scale_bytes(q.scales, 128, 768, "e4m3")[~rows]
    assert (left == 0xAB).all()


@pytest.mark.parametrize("ldo,offset", [(104, 0), (112, 8), (112, 16), (96, 8)])
@pytest.mark.parametrize("fmt", FORMATS)
def test_values_into_a_pitch(fmt, ldo, offset):
    """Rows that start on a sector, and such as only start on 16 bytes: the same values, and nothing around them."""
    x, s = activations(37, 96, torch.bfloat16, 61)
    q = quantised(x, s, fmt)
    buf = torch.full((38 * ldo + offset,), 7.0, dtype=torch.bfloat16, device="cuda")
    out = buf[offset:].as_strided((37, 96), (ldo, 1))
    want = q.values()
    q.values(out)
    assert torch.equal(out, want)
    out.fill_(7.0)
    assert (buf == 7).all()


def test_no_tokens():
    layer = aweq.LinearMX4(torch.ones((8, 32), dtype=torch.float16, device="cuda"), "e8m0")
    assert layer(aweq.MX4(0, 32, "e8m0")).shape == (0, 8)


@pytest.mark.parametrize("fmt", FORMATS)
def test_on_another_stream_and_in_a_graph(fmt):
    x, rinv = activations(40, 1024, torch.float16, 1)
    w, s = activations(512, 1024, torch.float16, 2)
    layer, xq, out = aweq.LinearMX4(w, fmt, s), aweq.MX4(40, 1024, fmt), torch.empty((40, 512), dtype=torch.float16, device="cuda")
    want = layer(xq.quantise(x, rinv)).clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        assert torch.equal(layer(xq.quantise(x, rinv), out), want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(xq.quantise(x, rinv), out)
    y, _ = activations(40, 1024, torch.float16, 7)
    for v in (x, y, x):
        x_now = v.clone()
        x.copy_(x_now)
        out.zero_()
        graph.replay()
        assert torch.equal(out, layer(quantised(x_now, rinv, fmt)))


def test_layer_keeps_what_it_was_made_of():
    w, s = activations(64, 128, torch.float16, 2)
    b = torch.randn(64, device="cuda")
    layer = aweq.LinearMX4(w, "e8m0", s, b)
    xq = quantised(w, s, "e8m0")
    want = layer(xq)
    w.zero_(), s.zero_(), b.zero_()
    assert torch.equal(layer(xq), want)


@pytest.mark.parametrize("call", [
    lambda x, q, l: q.quantise(x[:, :96]), lambda x, q, l: q.quantise(x[:3]), lambda x, q, l: q.quantise(x, torch.ones(64, device="cuda")),
    lambda x, q, l: q.quantise(x.t().contiguous().t()), lambda x, q, l: l(aweq.MX4(4, 96)), lambda x, q, l: l(aweq.MX4(4, 128, "e4m3")),
    lambda x, q, l: l(q, torch.empty((4, 9), dtype=torch.float16, device="cuda")), lambda x, q, l: l(q, torch.empty((8, 4), dtype=torch.float16, device="cuda").t()),
    lambda x, q, l: aweq.MX4(4, 48), lambda x, q, l: aweq.MX4(4, 64, "e5m2"), lambda x, q, l: q.quantise(x, mu=torch.ones(128, device="cuda", dtype=torch.float64)),
    lambda x, q, l: q.values(torch.empty((4, 64), dtype=torch.float16, device="cuda")), lambda x, q, l: q.quantise(x.cpu())])
def test_refusals_of_the_binding(call):
    x = torch.ones((4, 128), dtype=torch.float16, device="cuda")
    with pytest.raises(ValueError):
        call(x, aweq.MX4(4, 128), aweq.LinearMX4(torch.ones((8, 128), dtype=torch.float16, device="cuda")))
    with pytest.raises(TypeError):
        aweq.MX4(4, 128).quantise(x.float())
