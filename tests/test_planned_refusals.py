"""What the attention of drafted trees on a plan refuses, and a plan beyond what its loops count: host-side validation, no CUDA call (the
addresses are never dereferenced)."""
import pytest

from paper_2311_01305_b200 import aweq

from .test_drafting_refusals import ALIGN, CACHES, NULL, OK, P, SHAPE, WORKSPACE, cache, plan


def planned(c=None, **kw):
    a = dict(q=P, ldq=256, cache=c or cache(), prefix_pages=P, prefix=20, table=P, pps=3, ld=3, lens=P, start=P, pos=P, first=0, mask=P, words=1,
             max_own=40, n_seq=2, rows=9, nodes=8, heads=4, scale=1.0, out=P, ldo=256, ws=P, ws_bytes=1 << 40, st=None, stream=None)
    a.update(kw)
    return aweq._lib.aweq_tree_attention_planned(*a.values())


@pytest.mark.parametrize("kw,code", CACHES)
def test_refuses_caches(kw, code):
    assert planned(cache(**kw)) == code


@pytest.mark.parametrize("kw,code", [
    *((dict([(n, None)]), NULL) for n in ("q", "out", "lens", "start", "pos", "mask", "prefix_pages", "table")),
    (dict(first=-1), SHAPE), (dict(first=1 << 31), SHAPE), (dict(nodes=257, words=4), SHAPE), (dict(words=0), SHAPE), (dict(rows=-1), SHAPE),
    (dict(pos=P + 2), ALIGN), (dict(mask=P + 4), ALIGN), (dict(ldq=252), ALIGN), (dict(ws=None), WORKSPACE), (dict(ws_bytes=0), WORKSPACE),
    (dict(n_seq=0), OK), (dict(rows=0), OK), (dict(rows=0, q=None, out=None, pos=None), OK)])
def test_refusals(kw, code):
    assert planned(**kw) == code


@pytest.mark.parametrize("n_seq,code", [((1 << 30) + 1, SHAPE), ((1 << 31) - 1, SHAPE)])
def test_a_plan_of_more_sequences_than_its_loops_count(n_seq, code):
    assert plan(n_seq=n_seq) == code and aweq.aweq_kv_plan_workspace_bytes(n_seq) == 0
