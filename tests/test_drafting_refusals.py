"""What the entry points for 4-bit products, step plans, accepted paths and drafted trees refuse: host-side validation, no CUDA
call (the addresses below are never dereferenced)."""
import ctypes

import pytest

from paper_2311_01305_b200 import aweq

P = 0x10000                       # a 16- and 256-byte aligned address
OK, NULL, SHAPE, ALIGN, DTYPE, WORKSPACE, UNSUPPORTED = 0, 1, 2, 3, 4, 7, 9
lib = aweq._lib


def quant(**kw):
    a = dict(X=P, dt=0, rows=4, cols=64, ld=64, scale=None, fmt=1, codes=P, scales=P, row_step=P, mu=None, epsmu=None, st=None, stream=None)
    a.update(kw)
    return lib.aweq_quant_mx4(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(X=None), NULL), (dict(codes=None), NULL), (dict(scales=None), NULL), (dict(row_step=None), NULL), (dict(mu=P), NULL), (dict(epsmu=P), NULL),
    (dict(dt=2), DTYPE), (dict(fmt=2), UNSUPPORTED), (dict(fmt=-1), UNSUPPORTED), (dict(rows=-1), SHAPE), (dict(rows=1 << 31), SHAPE), (dict(cols=0), SHAPE),
    (dict(cols=48, ld=48), SHAPE), (dict(cols=65568, ld=65568), SHAPE), (dict(ld=32), ALIGN), (dict(ld=68), ALIGN), (dict(X=P + 8), ALIGN),
    (dict(codes=P + 8), ALIGN), (dict(scales=P + 4), ALIGN), (dict(scale=P + 4), ALIGN), (dict(row_step=P + 2), ALIGN), (dict(mu=P + 8, epsmu=P), ALIGN),
    (dict(mu=P, epsmu=P + 2), ALIGN), (dict(rows=0), OK), (dict(rows=0, X=None, codes=None, scales=None, row_step=None), OK)])
def test_quantiser_refusals(kw, code):
    assert quant(**kw) == code


def dequant(**kw):
    a = dict(codes=P, scales=P, row_step=P, fmt=1, rows=4, cols=64, out=P, dt=0, ldo=64, stream=None)
    a.update(kw)
    return lib.aweq_dequant_mx4(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(codes=None), NULL), (dict(scales=None), NULL), (dict(row_step=None), NULL), (dict(out=None), NULL), (dict(dt=3), DTYPE), (dict(fmt=7), UNSUPPORTED),
    (dict(rows=-1), SHAPE), (dict(cols=40), SHAPE), (dict(ldo=60), ALIGN), (dict(ldo=68), ALIGN), (dict(out=P + 2), ALIGN), (dict(codes=P + 1), ALIGN),
    (dict(rows=0, out=None), OK)])
def test_dequantiser_refusals(kw, code):
    assert dequant(**kw) == code


def linear(**kw):
    a = dict(Xq=P, xs=P, xt=P, Wq=P, ws=P, wt=P, fmt=1, bias=None, N=4, C_in=64, C_out=8, out=P, dt=0, ldo=8, st=None, stream=None)
    a.update(kw)
    return lib.aweq_linear_mx4(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(Xq=None), NULL), (dict(xs=None), NULL), (dict(xt=None), NULL), (dict(Wq=None), NULL), (dict(ws=None), NULL), (dict(wt=None), NULL),
    (dict(out=None), NULL), (dict(dt=2), DTYPE), (dict(fmt=2), UNSUPPORTED), (dict(N=-1), SHAPE), (dict(N=1 << 31), SHAPE), (dict(C_out=0), SHAPE),
    (dict(C_out=(1 << 30) + 1), SHAPE), (dict(C_in=0), SHAPE), (dict(C_in=48), SHAPE), (dict(C_in=65568), SHAPE), (dict(C_out=1 << 30, C_in=65536), SHAPE),
    (dict(Xq=P + 8), ALIGN), (dict(Wq=P + 4), ALIGN), (dict(xs=P + 8), ALIGN), (dict(ws=P + 8), ALIGN), (dict(xt=P + 2), ALIGN), (dict(wt=P + 1), ALIGN),
    (dict(bias=P + 2), ALIGN), (dict(out=P + 1), ALIGN), (dict(ldo=7), ALIGN), (dict(N=0), OK), (dict(N=0, Xq=None, xs=None, xt=None, out=None), OK)])
def test_linear_refusals(kw, code):
    assert linear(**kw) == code


@pytest.mark.parametrize("rows,cols,fmt,want", [
    (1, 32, 0, 1024), (128, 256, 0, 1024), (129, 256, 0, 2048), (1, 288, 0, 2048), (1, 16, 0, 0), (-1, 32, 0, 0), (1, 32, 3, 0), (0, 32, 1, 0),
    (1, 32, 1, 2048), (128, 256, 1, 2048), (300, 512, 1, 3 * 4096)])
def test_bytes_of_scales(rows, cols, fmt, want):
    """Tiles of 512 bytes, two (blocks of 32) or four (of 16) for 128 rows of 256 columns."""
    assert int(lib.aweq_mx4_scale_bytes(rows, cols, fmt)) == want


def cache(**kw):
    a = dict(k=P, v=P, dt=0, page_size=16, n_kv_heads=2, head_dim=64, n_pages=10, page_stride=2048, token_stride=128, head_stride=64)
    a.update(kw)
    return ctypes.byref(aweq.KvCacheArgs(*a.values()))


CACHES = [(dict(k=None), NULL), (dict(v=None), NULL), (dict(dt=5), DTYPE), (dict(page_size=0), SHAPE), (dict(n_kv_heads=0), SHAPE),
          (dict(head_dim=60), SHAPE), (dict(head_dim=0), SHAPE), (dict(head_dim=264), SHAPE), (dict(n_pages=0), SHAPE), (dict(k=P + 8), ALIGN),
          (dict(token_stride=130), ALIGN), (dict(head_stride=32), ALIGN), (dict(page_stride=-2048), ALIGN)]


def append(c=None, **kw):
    a = dict(cache=c or cache(), slot=P, k=P, ldk=128, v=P, ldv=128, pos=P, n=4, rope=P, n_pos=100, rd=64, inter=0, q=None, ldq=0, heads=0,
             q_out=None, ldqo=0, st=None, stream=None)
    a.update(kw)
    return lib.aweq_kv_append_slots(*a.values())


@pytest.mark.parametrize("kw,code", CACHES)
def test_append_refuses_caches(kw, code):
    assert append(cache(**kw)) == code


@pytest.mark.parametrize("kw,code", [
    (dict(slot=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(pos=None), NULL), (dict(slot=P + 4), ALIGN), (dict(ldk=120), ALIGN),
    (dict(ldv=0), ALIGN), (dict(k=P + 1), ALIGN), (dict(pos=P + 2), ALIGN), (dict(n=-1), SHAPE), (dict(n=1 << 31), SHAPE), (dict(rd=66), SHAPE),
    (dict(rd=7), SHAPE), (dict(n_pos=0), SHAPE), (dict(q=P), NULL), (dict(q_out=P), NULL), (dict(q=P, q_out=P, heads=0, ldq=256, ldqo=256), SHAPE),
    (dict(q=P, q_out=P, heads=4, ldq=255, ldqo=256), ALIGN), (dict(n=0), OK), (dict(n=0, slot=None, k=None, v=None, pos=None), OK)])
def test_append_refusals(kw, code):
    assert append(**kw) == code


def plan(**kw):
    a = dict(table=P, n_seq=4, pps=3, ld=3, page=16, ring=P, state=P, n_pages=10, held=P, change=P, first=0, rows=64, own=P + 256, start=P, seq=P,
             pos=P, slot=P, parent=P, mask=P, words=1, ws=P, ws_bytes=1 << 40, st=None, stream=None)
    a.update(kw)
    return lib.aweq_kv_plan(*a.values())


@pytest.mark.parametrize("kw,code", [
    *((dict([(n, None)]), NULL) for n in ("table", "ring", "state", "held", "change", "own", "start", "seq", "pos", "slot", "parent", "mask")),
    (dict(n_seq=0), SHAPE), (dict(n_seq=1 << 31), SHAPE), (dict(pps=0), SHAPE), (dict(page=0), SHAPE), (dict(page=(1 << 20) + 1), SHAPE), (dict(n_pages=0), SHAPE),
    (dict(n_pages=(1 << 22) + 1), SHAPE), (dict(first=-1), SHAPE), (dict(first=0x7fffffff), SHAPE), (dict(pps=1 << 20, ld=1 << 20, page=1 << 12), SHAPE),
    (dict(rows=-1), SHAPE), (dict(rows=0x7fffffff), SHAPE), (dict(words=0), SHAPE), (dict(words=5), SHAPE), (dict(ld=2), ALIGN), (dict(table=P + 2), ALIGN),
    (dict(state=P + 4), ALIGN), (dict(own=P), ALIGN), (dict(own=P, held=P + 64), ALIGN), (dict(seq=P + 4), ALIGN), (dict(pos=P + 8), ALIGN),
    (dict(slot=P + 8), ALIGN), (dict(mask=P + 8), ALIGN), (dict(ws=None), WORKSPACE), (dict(ws=P + 16), WORKSPACE), (dict(ws_bytes=0), WORKSPACE)])
def test_plan_refusals(kw, code):
    assert plan(**kw) == code


def accept(c=None, **kw):
    a = dict(cache=c or cache(), table=P, n_seq=4, pps=3, ld=3, base=P, path=P, ldp=8, most=8, n=P, st=None, stream=None)
    a.update(kw)
    return lib.aweq_kv_accept(*a.values())


@pytest.mark.parametrize("kw,code", CACHES)
def test_accept_refuses_caches(kw, code):
    assert accept(cache(**kw)) == code


@pytest.mark.parametrize("kw,code", [
    (dict(table=None), NULL), (dict(base=None), NULL), (dict(path=None), NULL), (dict(n=None), NULL), (dict(n_seq=-1), SHAPE), (dict(n_seq=1 << 31), SHAPE),
    (dict(pps=0), SHAPE), (dict(most=-1), SHAPE), (dict(ld=2), ALIGN), (dict(ldp=7), ALIGN), (dict(path=P + 2), ALIGN), (dict(base=P + 1), ALIGN),
    (dict(n_seq=0), OK), (dict(most=0, path=None), OK)])
def test_accept_refusals(kw, code):
    assert accept(**kw) == code


def attention(c=None, **kw):
    a = dict(q=P, ldq=256, cache=c or cache(), prefix_pages=P, prefix=20, table=P, pps=3, ld=3, lens=P, start=P, mask=P, words=1, max_own=40, n_seq=2,
             rows=9, nodes=8, heads=4, scale=1.0, out=P, ldo=256, ws=P, ws_bytes=1 << 40, st=None, stream=None)
    a.update(kw)
    return lib.aweq_tree_attention(*a.values())


@pytest.mark.parametrize("kw,code", CACHES + [(dict(head_dim=136, token_stride=272, head_stride=136), SHAPE)])
def test_attention_refuses_caches(kw, code):
    assert attention(cache(**kw)) == code


@pytest.mark.parametrize("kw,code", [
    *((dict([(n, None)]), NULL) for n in ("q", "out", "lens", "start", "mask", "prefix_pages", "table")),
    (dict(prefix=-1), SHAPE), (dict(max_own=-1), SHAPE), (dict(rows=-1), SHAPE), (dict(nodes=0), SHAPE), (dict(nodes=257, words=4), SHAPE),
    (dict(nodes=65), SHAPE), (dict(words=5), SHAPE), (dict(words=0), SHAPE), (dict(heads=3), SHAPE), (dict(heads=0), SHAPE), (dict(n_seq=-1), SHAPE),
    (dict(n_seq=(1 << 24) + 1), SHAPE), (dict(rows=1 << 30), SHAPE), (dict(pps=0), SHAPE), (dict(ldq=252), ALIGN), (dict(ldq=248), ALIGN), (dict(ldo=260), ALIGN),
    (dict(q=P + 8), ALIGN), (dict(out=P + 2), ALIGN), (dict(ld=2), ALIGN), (dict(mask=P + 4), ALIGN), (dict(start=P + 2), ALIGN), (dict(ws=None), WORKSPACE),
    (dict(ws=P + 16), WORKSPACE), (dict(ws_bytes=0), WORKSPACE), (dict(n_seq=0), OK), (dict(rows=0), OK), (dict(rows=0, q=None, out=None), OK)])
def test_attention_refusals(kw, code):
    assert attention(**kw) == code


def test_workspaces_of_what_is_refused():
    assert aweq.aweq_kv_plan_workspace_bytes(-1) == 0 and aweq.aweq_kv_plan_workspace_bytes(1) > 0
    size = lambda prefix=0, own=64, n_seq=2, rows=8, nodes=8, heads=4: int(  # noqa: E731
        lib.aweq_tree_attention_workspace_bytes(cache(), prefix, own, n_seq, rows, nodes, heads))
    assert size() > 0 and size(nodes=257) == 0 and size(heads=3) == 0 and size(prefix=-1) == 0 and size(n_seq=0) == 0
