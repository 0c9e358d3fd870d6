"""What the entry points that run a calibrated layer refuse: host-side validation, no CUDA call (the
addresses below are never dereferenced)."""
import ctypes

import pytest

from paper_2311_01305_b200 import aweq

P = 0x10000                       # a 16- and 256-byte aligned address
OK, NULL, SHAPE, ALIGN, DTYPE, WORKSPACE, UNSUPPORTED = 0, 1, 2, 3, 4, 7, 9
lib = aweq._lib


def linear(**kw):
    a = dict(Xq=P, ldx=64, xs=P, xz=P, xg=1, Wq=P, ldw=64, ws=P, wz=P, wsum=P, wg=1, bias=None, N=4, C_in=64, C_out=8, out=P,
             dt=0, ldo=8, st=None, stream=None)
    a.update(kw)
    return lib.aweq_linear_w8a8(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(Xq=None), NULL), (dict(xs=None), NULL), (dict(xz=None), NULL), (dict(Wq=None), NULL), (dict(ws=None), NULL),
    (dict(wz=None), NULL), (dict(wsum=None), NULL), (dict(out=None), NULL), (dict(dt=2), DTYPE), (dict(xg=2), UNSUPPORTED),
    (dict(wg=2), UNSUPPORTED), (dict(N=-1), SHAPE), (dict(N=1 << 31), SHAPE), (dict(C_out=0), SHAPE),
    (dict(C_out=(1 << 30) + 1), SHAPE), (dict(C_in=0), SHAPE), (dict(C_in=56), SHAPE), (dict(C_in=65552, ldx=65552, ldw=65552), SHAPE),
    (dict(ldx=48), ALIGN), (dict(ldx=72), ALIGN), (dict(ldw=56), ALIGN), (dict(Xq=P + 8), ALIGN), (dict(Wq=P + 4), ALIGN),
    (dict(ldo=7), ALIGN), (dict(out=P + 1), ALIGN), (dict(xs=P + 2), ALIGN), (dict(bias=P + 1), ALIGN),
    (dict(N=0), OK), (dict(N=0, Xq=None, xs=None, xz=None, out=None), OK)])
def test_linear_refusals(kw, code):
    assert linear(**kw) == code


@pytest.mark.parametrize("args,code", [((None, 4, 64, 64, P), NULL), ((P, 4, 64, 64, None), NULL), ((P, 0, 64, 64, P), SHAPE),
                                       ((P, 4, 65552, 65552, P), SHAPE), ((P, 4, 40, 48, P), SHAPE), ((P, 4, 64, 48, P), ALIGN),
                                       ((P + 2, 4, 64, 64, P), ALIGN)])
def test_code_sums_refusals(args, code):
    assert lib.aweq_code_sums(*args, None) == code


def rope(**kw):
    a = dict(rotary_dim=64, scaling=0, theta=1e4, factor=1.0, original_len=4096.0, low=1.0, high=4.0, attention=1.0)
    n_pos, table = kw.pop("n_pos", 16), kw.pop("table", P)
    a.update(kw)
    return lib.aweq_rope_table(ctypes.byref(aweq.RopeSpec(*a.values())), n_pos, table, None)


@pytest.mark.parametrize("kw,code", [(dict(table=None), NULL), (dict(n_pos=0), SHAPE), (dict(rotary_dim=0), SHAPE), (dict(rotary_dim=7), SHAPE),
                                     (dict(rotary_dim=258), SHAPE), (dict(scaling=4), UNSUPPORTED), (dict(theta=0.0), UNSUPPORTED),
                                     (dict(theta=float("nan")), UNSUPPORTED), (dict(attention=-1.0), UNSUPPORTED),
                                     (dict(scaling=1, factor=0.0), UNSUPPORTED), (dict(scaling=2, rotary_dim=2), SHAPE),
                                     (dict(scaling=3, high=1.0), UNSUPPORTED), (dict(scaling=3, original_len=0.0), UNSUPPORTED)])
def test_rope_table_refusals(kw, code):
    assert rope(**kw) == code


def cache(**kw):
    a = dict(k=P, v=P, dt=0, page_size=16, n_kv_heads=2, head_dim=64, n_pages=10, page_stride=2048, token_stride=128, head_stride=64)
    a.update(kw)
    return ctypes.byref(aweq.KvCacheArgs(*a.values()))


CACHES = [(dict(k=None), NULL), (dict(v=None), NULL), (dict(dt=5), DTYPE), (dict(page_size=0), SHAPE), (dict(n_kv_heads=0), SHAPE),
          (dict(head_dim=60), SHAPE), (dict(head_dim=0), SHAPE), (dict(head_dim=264), SHAPE), (dict(n_pages=0), SHAPE), (dict(k=P + 8), ALIGN),
          (dict(token_stride=130), ALIGN), (dict(head_stride=32), ALIGN), (dict(page_stride=-2048), ALIGN)]


def append(c=None, **kw):
    a = dict(cache=c or cache(), table=P, n_seq=4, pps=3, ld=3, k=P, ldk=128, v=P, ldv=128, pos=P, seq=None, first=0, n=4, rope=P,
             n_pos=100, rd=64, inter=0, q=None, ldq=0, heads=0, q_out=None, ldqo=0, st=None, stream=None)
    a.update(kw)
    return lib.aweq_kv_append(*a.values())


@pytest.mark.parametrize("kw,code", CACHES)
def test_append_refuses_caches(kw, code):
    assert append(cache(**kw)) == code


@pytest.mark.parametrize("kw,code", [
    (dict(table=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(pos=None), NULL), (dict(n_seq=0), SHAPE), (dict(pps=0), SHAPE),
    (dict(ld=2), ALIGN), (dict(ldk=120), ALIGN), (dict(ldv=0), ALIGN), (dict(k=P + 1), ALIGN), (dict(pos=P + 2), ALIGN), (dict(first=-1), SHAPE),
    (dict(n=-1), SHAPE), (dict(rd=66), SHAPE), (dict(rd=7), SHAPE), (dict(n_pos=0), SHAPE), (dict(q=P), NULL), (dict(q_out=P), NULL),
    (dict(q=P, q_out=P, heads=0, ldq=256, ldqo=256), SHAPE), (dict(q=P, q_out=P, heads=4, ldq=255, ldqo=256), ALIGN),
    (dict(n=5), SHAPE), (dict(n=0), OK)])
def test_append_refusals(kw, code):
    """Without seq every token needs a sequence of its own: five tokens for four sequences are refused."""
    assert append(**kw) == code


def attention(c=None, **kw):
    a = dict(q=P, ldq=256, cache=c or cache(), prefix_pages=P, prefix=20, table=P, pps=3, ld=3, lens=P, max_own=40, n_seq=2, n_q=1, heads=4,
             scale=1.0, out=P, ldo=256, ws=P, ws_bytes=1 << 40, st=None, stream=None)
    a.update(kw)
    return lib.aweq_prefix_attention(*a.values())


@pytest.mark.parametrize("kw,code", CACHES + [(dict(head_dim=136, token_stride=272, head_stride=136), SHAPE)])
def test_attention_refuses_caches(kw, code):
    assert attention(cache(**kw)) == code


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), NULL), (dict(out=None), NULL), (dict(lens=None), NULL), (dict(prefix_pages=None), NULL), (dict(table=None), NULL),
    (dict(prefix=-1), SHAPE), (dict(max_own=-1), SHAPE), (dict(n_q=0), SHAPE), (dict(heads=3), SHAPE), (dict(heads=0), SHAPE),
    (dict(n_seq=-1), SHAPE), (dict(ldq=252), ALIGN), (dict(ldo=248), ALIGN), (dict(q=P + 8), ALIGN), (dict(out=P + 2), ALIGN), (dict(ld=2), ALIGN),
    (dict(ws=None), WORKSPACE), (dict(ws=P + 16), WORKSPACE), (dict(ws_bytes=0), WORKSPACE), (dict(n_seq=0), OK)])
def test_attention_refusals(kw, code):
    assert attention(**kw) == code
