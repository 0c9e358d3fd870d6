"""A step of serving with drafted trees and 4-bit layers, as cases that can be timed and compared.

Five operators: microscaled 4-bit quantisation (``quant``), a linear layer on such codes from 16-bit
activations (``linear``), pages, slots, positions and tree masks from request lengths (``plan``),
attention of drafted trees over a paged cache (``tree``), and the move of an accepted path's keys and
values to their places (``accept``).  ``run`` computes a case in elementary torch operations in binary32,
or, where ``own`` is true, through this package.  ``exact`` evaluates the definitions in binary64.
"""
from __future__ import annotations

import math

import torch

own = False

_DEV = "cuda"
_DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
_BLOCK = {"e8m0": 32, "e4m3": 16}


def listed():
    return [
        # the activations of sixteen decoding sequences before LLaMA-13B's q/k/v: nothing but latency
        dict(name="quant_16x5120_e8m0", op="quant", dtype="f16", rows=16, cols=5120, fmt="e8m0"),
        # a weight matrix: LLaMA-7B's up projection, small blocks with a scale per row
        dict(name="quant_11008x4096_e4m3", op="quant", dtype="bf16", rows=11008, cols=4096, fmt="e4m3"),
        # one token through an OPT-125M projection
        dict(name="linear_1x768x768_e8m0", op="linear", dtype="f16", n=1, c_in=768, c_out=768, fmt="e8m0", bias=True),
        # 24 drafted tokens through the joint q/k/v projection of a LLaMA-7B layer
        dict(name="linear_24x4096x12288_e4m3", op="linear", dtype="bf16", n=24, c_in=4096, c_out=12288, fmt="e4m3", bias=False),
        # a batch of prompts through LLaMA-13B's gate, a few tokens more than whole tiles
        dict(name="linear_4099x5120x13824_e8m0", op="linear", dtype="bf16", n=4099, c_in=5120, c_out=13824, fmt="e8m0", bias=True),
        # 64 sequences with a drafted tree each: pages and masks for the step, then the rejected tokens' pages back
        dict(name="plan_64_trees", op="plan", n_seq=64, max_new=32, max_held=1500, page=16, first=512, tree=True),
        # 512 prompts admitted at once, and let go again
        dict(name="plan_512_prompts", op="plan", n_seq=512, max_new=4096, max_held=64, page=64, first=0, tree=False),
        # a few small trees after a short instruction, OPT-125M heads
        dict(name="tree_4x8_short", op="tree", dtype="f16", n_seq=4, nodes=8, n_heads=12, n_kv=12, head_dim=64, prefix=257,
             max_own=90, page=16),
        # ragged trees of a mid-sized batch, shared key heads, a common system prompt
        dict(name="tree_16x24_chat", op="tree", dtype="bf16", n_seq=16, nodes=24, n_heads=32, n_kv=8, head_dim=128, prefix=512,
             max_own=2100, page=32),
        # wide trees over long contexts, no common prefix
        dict(name="tree_32x64_long", op="tree", dtype="bf16", n_seq=32, nodes=64, n_heads=32, n_kv=8, head_dim=128, prefix=0,
             max_own=8192, page=64),
        # short accepted paths of a handful of sequences, OPT-125M heads
        dict(name="accept_8_short", op="accept", dtype="f16", n_seq=8, nodes=16, path=5, n_kv=12, head_dim=64, page=16, max_held=100),
        # a large batch, long accepted paths
        dict(name="accept_256_long", op="accept", dtype="bf16", n_seq=256, nodes=64, path=16, n_kv=8, head_dim=128, page=64,
             max_held=200),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quant", "linear", "linear", "plan", "tree", "tree", "accept"])
    dtype, fmt = rng.choice(["f16", "bf16"]), rng.choice(["e8m0", "e4m3"])
    page = rng.choice([8, 16, 16, 24, 32, 64, 128])
    if op == "quant":
        while True:
            rows, cols = _log_int(rng, 1, 16384), 32 * _log_int(rng, 1, 1152)
            if rows * cols <= 96 * 1024 * 1024:
                return dict(op=op, dtype=dtype, rows=rows, cols=cols, fmt=fmt)
    if op == "linear":
        while True:
            n, c_in, c_out = _log_int(rng, 1, 8192), 32 * _log_int(rng, 2, 1152), _log_int(rng, 48, 16384)
            if n * c_in * c_out <= 4099 * 5120 * 13824 and c_in * c_out <= 160 * 1024 * 1024:
                return dict(op=op, dtype=dtype, n=n, c_in=c_in, c_out=c_out, fmt=fmt, bias=rng.random() < 0.6)
    if op == "plan":
        tree = rng.random() < 0.5
        n_seq = _log_int(rng, 1, 1024)
        max_new = rng.randint(2, 96) if tree else _log_int(rng, 1, max(2, 1500000 // n_seq if n_seq > 360 else 4096))
        return dict(op=op, n_seq=n_seq, max_new=max_new, max_held=_log_int(rng, 16, 4096), page=page,
                    first=rng.choice([0, 0, 100, 2048]), tree=tree)
    n_heads, n_kv = rng.choice([(12, 12), (16, 16), (32, 32), (40, 40), (32, 8), (40, 8), (24, 3), (16, 1)])
    head_dim = rng.choice([64, 80, 96, 128, 128])
    if op == "accept":
        while True:
            n_seq, nodes = _log_int(rng, 1, 512), rng.randint(2, 96)
            path, max_held = rng.randint(1, min(nodes, 24)), _log_int(rng, 4, 1000)
            if n_seq * (max_held + nodes + page) * n_kv * head_dim <= 128 * 1024 * 1024:
                return dict(op=op, dtype=dtype, n_seq=n_seq, nodes=nodes, path=path, n_kv=n_kv, head_dim=head_dim, page=page,
                            max_held=max_held)
    while True:
        n_seq, nodes = _log_int(rng, 1, 64), rng.randint(2, 96)
        prefix = 0 if rng.random() < 0.4 else _log_int(rng, 16, 8192)
        max_own = nodes + _log_int(rng, 1, 8192)
        rows = n_seq * nodes * n_heads
        if rows * (max_own + prefix) <= 32 * 64 * 32 * 8192 and n_seq * max_own * n_kv * head_dim <= 256 * 1024 * 1024:
            return dict(op=op, dtype=dtype, n_seq=n_seq, nodes=nodes, n_heads=n_heads, n_kv=n_kv, head_dim=head_dim, prefix=prefix,
                        max_own=max_own, page=page)


# ---------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device=_DEV).manual_seed(int(seed) * 7919 + 23)


def _uneven(n, most):
    """n numbers between half of the most and the most, the same for every seed."""
    return [most - (most * i // (2 * n)) for i in range(n)]


def _activations(g, n, c, dt):
    """16-bit activations with outlier channels, and 1/s of an equalised layer."""
    x = torch.randn((n, c), generator=g, device=_DEV)
    x.mul_(1.0 + 0.5 * torch.rand(c, generator=g, device=_DEV)).add_(0.3 * torch.randn(c, generator=g, device=_DEV))
    out = torch.randint(0, c, (max(1, c // 512),), generator=g, device=_DEV)
    x[:, out] *= 20.0
    rinv = 0.6 + 0.9 * torch.rand(c, generator=g, device=_DEV)
    rinv[out] *= 0.2
    return x.to(dt), rinv


def _quant_inputs(case, seed):
    g = _gen(seed)
    x, m = _activations(g, case["rows"], case["cols"], _DTYPES[case["dtype"]])
    return dict(x=x, m=m)


def _linear_inputs(case, seed):
    g = _gen(seed)
    dt = _DTYPES[case["dtype"]]
    x, rinv = _activations(g, case["n"], case["c_in"], dt)
    w = torch.randn((case["c_out"], case["c_in"]), generator=g, device=_DEV).mul_(0.02).to(dt)
    return dict(x=x, rinv=rinv, w=w, s=1.0 / rinv, bias=0.1 * torch.randn(case["c_out"], generator=g, device=_DEV) if case["bias"] else None)


def _parents(g, start, total):
    """Trees: a node's parent is one of the eight before it (its number within the sequence), of the first node none."""
    n = torch.arange(total, device=_DEV)
    at = n - start[torch.searchsorted(start, n, right=True) - 1]
    back = torch.randint(1, 9, (total,), generator=g, device=_DEV)
    return torch.where(at == 0, torch.full_like(at, -1), (at - back).clamp(min=0))


def _pages(g, used, per_seq, n_pages):
    """A table [sequences, per_seq] with ``used`` pages each (-1 behind them) and the other pages in a row."""
    order = torch.randperm(n_pages, generator=g, device=_DEV).to(torch.int32)
    col = torch.arange(per_seq, device=_DEV)
    begin = torch.cumsum(used, 0) - used
    table = order[(begin[:, None] + col).clamp(max=n_pages - 1)]
    table[col >= used[:, None]] = -1
    return table.contiguous(), order.roll(-int(used.sum()))


def _plan_inputs(case, seed):
    g = _gen(seed)
    n_seq, page = case["n_seq"], case["page"]
    new = torch.tensor(_uneven(n_seq, case["max_new"]), device=_DEV)[torch.randperm(n_seq, generator=g, device=_DEV)]
    held = torch.randint(0, case["max_held"] + 1, (n_seq,), generator=g, device=_DEV)
    per_seq = (case["max_held"] + case["max_new"]) // page + 1
    n_pages = n_seq * per_seq
    used = (held + page - 1) // page
    table, ring = _pages(g, used, per_seq, n_pages)
    total = sum(_uneven(n_seq, case["max_new"]))
    # the rows a captured step would have: the tokens, and some that are none
    rows = (total + 63) // 64 * 64
    start = torch.cat([new.new_zeros(1), torch.cumsum(new, 0)])
    parent = torch.full((rows,), -1, device=_DEV)
    parent[:total] = _parents(g, start, total)
    turn = int(torch.randint(0, n_pages, (1,), generator=g, device=_DEV))
    return dict(table=table, ring=ring.roll(turn).contiguous(), state=torch.tensor([turn, turn + n_pages - int(used.sum())], device=_DEV),
                held=held.to(torch.int32), change=new.to(torch.int32), back=(-new).to(torch.int32), rows=rows,
                parent=parent.to(torch.int32) if case["tree"] else None, words=(case["max_new"] + 63) // 64)


def _ancestors(parent, start, n_seq, nodes):
    """[sequences, nodes, nodes] truth values: node j is node i itself or above it."""
    t = torch.arange(parent.numel(), device=_DEV)
    b = torch.searchsorted(start, t, right=True) - 1
    up = torch.zeros((n_seq, nodes, nodes), device=_DEV)
    up[b, t - start[b], parent.clamp(min=0)] = (parent >= 0).float()
    # sums of powers of the parent relation: zero exactly where there is no way up
    return torch.linalg.matrix_power(torch.eye(nodes, device=_DEV) + up, 128) > 0


def _words(seen, words):
    """Truth values [..., nodes] as 64-bit words, node j in bit j % 64 of word j / 64."""
    seen = torch.nn.functional.pad(seen.to(torch.int64), (0, words * 64 - seen.shape[-1]))
    return (seen.unflatten(-1, (words, 64)) << torch.arange(64, device=_DEV)).sum(-1)


def _tree_inputs(case, seed):
    g = _gen(seed)
    dt = _DTYPES[case["dtype"]]
    n_seq, kv, d, page, nodes = case["n_seq"], case["n_kv"], case["head_dim"], case["page"], case["nodes"]
    new = torch.tensor(_uneven(n_seq, nodes), device=_DEV)[torch.randperm(n_seq, generator=g, device=_DEV)]
    start = torch.cat([new.new_zeros(1), torch.cumsum(new, 0)])
    total = sum(_uneven(n_seq, nodes))
    parent = _parents(g, start, total)
    b = torch.searchsorted(start, torch.arange(total, device=_DEV), right=True) - 1
    mask = _words(_ancestors(parent, start, n_seq, nodes), (nodes + 63) // 64)[b, torch.arange(total, device=_DEV) - start[b]]
    most = case["max_own"] - nodes
    own_len = new + torch.randint(most // 4, most + 1, (n_seq,), generator=g, device=_DEV)
    per_seq, shared = -(-case["max_own"] // page), -(-case["prefix"] // page)
    n_pages = shared + n_seq * per_seq + 1
    table, order = _pages(g, (own_len + page - 1) // page, per_seq, n_pages)
    k = torch.randn((n_pages, page, kv, d), generator=g, device=_DEV)
    k *= 0.5 + torch.rand(d, generator=g, device=_DEV)                                     # channels of unlike size
    q = 2.0 * torch.randn((total, case["n_heads"], d), generator=g, device=_DEV)
    return dict(q=q.to(dt), k=k.to(dt), v=torch.randn((n_pages, page, kv, d), generator=g, device=_DEV).to(dt), page_table=table,
                prefix_pages=order[:shared].clone(), own_len=own_len.to(torch.int32), start=start.to(torch.int32), mask=mask.contiguous())


def _accept_inputs(case, seed):
    g = _gen(seed)
    dt = _DTYPES[case["dtype"]]
    n_seq, page, nodes, kv, d = case["n_seq"], case["page"], case["nodes"], case["n_kv"], case["head_dim"]
    base = torch.randint(0, case["max_held"] + 1, (n_seq,), generator=g, device=_DEV)
    per_seq = (case["max_held"] + nodes) // page + 1
    n_pages = n_seq * per_seq + 2
    table, _ = _pages(g, (base + nodes + page - 1) // page, per_seq, n_pages)
    # paths: ascending nodes, from the first on
    path = torch.rand((n_seq, nodes), generator=g, device=_DEV).argsort(1)[:, :case["path"]].sort(1).values
    path[:, 0] = 0
    n_path = torch.randint(1, case["path"] + 1, (n_seq,), generator=g, device=_DEV)
    return dict(k=torch.randn((n_pages, page, kv, d), generator=g, device=_DEV).to(dt), v=torch.randn((n_pages, page, kv, d), generator=g, device=_DEV).to(dt),
                page_table=table, base=base.to(torch.int32), path=path.to(torch.int32).contiguous(), n_path=n_path.to(torch.int32))


_INPUTS = {"quant": _quant_inputs, "linear": _linear_inputs, "plan": _plan_inputs, "tree": _tree_inputs, "accept": _accept_inputs}


def prepare(case, seed):
    s = _INPUTS[case["op"]](case, seed)
    s["case"] = case
    op = case["op"]
    if op == "linear":
        s["out"] = torch.empty((case["n"], case["c_out"]), dtype=_DTYPES[case["dtype"]], device=_DEV)
    if op == "quant":
        s["out"] = torch.empty_like(s["x"])
    if op == "tree":
        s["out"] = torch.empty_like(s["q"])
    if own:
        from paper_2311_01305_b200 import aweq
        if op == "quant":
            s["xq"] = aweq.MX4(case["rows"], case["cols"], case["fmt"])
        if op == "linear":
            s["layer"] = aweq.LinearMX4(s["w"], case["fmt"], s["s"], s["bias"])
            s["xq"] = aweq.MX4(case["n"], case["c_in"], case["fmt"])
        if op == "plan":
            s["pool"] = aweq.PagePool(s["ring"].numel(), case["page"], ring=s["ring"], state=s["state"])
            s["grow"] = aweq.StepPlan(case["n_seq"], s["rows"], case["max_new"] if case["tree"] else 0)
            s["shrink"] = aweq.StepPlan(case["n_seq"], 0)
        if op in ("tree", "accept"):
            s["cache"] = aweq.KVCache(s["k"], s["v"])
        if op == "tree":
            s["attend"] = aweq.TreeAttention(s["cache"], s["prefix_pages"], case["prefix"], case["n_heads"], case["n_seq"],
                                             s["q"].shape[0], case["nodes"], case["max_own"])
    elif op == "linear":
        # the layer's weights as they are held: elements (in halves), block scales, row scales
        s["w_elem"], s["w_scale"], s["w_row"] = _plain_quantised(s["w"], s["s"], case["fmt"])
        s["w_elem"] = (s["w_elem"] * 2).to(torch.int8)
    return s


# ---------------------------------------------------------------------------- the passes
def _plain_e2m1(y):
    """Nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with its sign, ties to the one whose code is even."""
    a = y.abs()
    low = (a > 0.25).float() + (a >= 0.75).float() + (a > 1.25).float() + (a >= 1.75).float()     # steps of a half, up to 2
    return torch.copysign(0.5 * low + (a > 2.5).float() + (a >= 3.5).float() + 2.0 * (a > 5.0).float(), y)


def _plain_quantised(x, m, fmt):
    """(elements, block scales, row scales) of x times m."""
    v = (x.float() * m).unflatten(1, (-1, _BLOCK[fmt]))
    top = v.abs().amax(-1)
    if fmt == "e8m0":
        e = (torch.frexp(top).exponent - 3).clamp(-127, 127)
        e = torch.where(top > 0, e, -127)
        elem = _plain_e2m1(v * torch.exp2(-e.float())[..., None])
        return elem.flatten(1), torch.exp2(e.float()), None
    row = top.amax(-1) / 2688.0
    t = top / (6.0 * row)[:, None]
    ulp = torch.exp2((torch.frexp(t).exponent - 4).clamp(min=-9).float())
    scale = torch.where(row[:, None] > 0, torch.round(t / ulp) * ulp, 0.0)
    step = scale * row[:, None]
    elem = torch.where(step[..., None] > 0, _plain_e2m1(v * (1.0 / step)[..., None]), 0.0)
    return elem.flatten(1), scale, row


def _plain_values(elem, scale, row, fmt):
    v = (elem.unflatten(1, (-1, _BLOCK[fmt])) * scale[..., None]).flatten(1)
    return v if row is None else v * row[:, None]


def _plain_quant(s):
    fmt = s["case"]["fmt"]
    return _plain_values(*_plain_quantised(s["x"], s["m"], fmt), fmt).to(s["x"].dtype)


def _plain_linear(s):
    fmt = s["case"]["fmt"]
    x = _plain_values(*_plain_quantised(s["x"], s["rinv"], fmt), fmt)
    w = _plain_values(s["w_elem"].float() * 0.5, s["w_scale"], s["w_row"], fmt)
    y = x @ w.t()
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(s["out"].dtype)


def _plain_step(s, change, rows):
    """Lengths and pages after ``change``, and the slots of the new tokens.  Rewrites table, ring and state."""
    case, table, ring, state = s["case"], s["table"], s["ring"], s["state"]
    page, n_pages, col = case["page"], ring.numel(), torch.arange(table.shape[1], device=_DEV)
    held = s["held"].long() if change is s["change"] else s["held"].long() + s["change"].long()
    after = held + change.long()
    have, want = (held + page - 1) // page, (after + page - 1) // page
    more, less = (want - have).clamp(min=0), (have - want).clamp(min=0)
    take, give = torch.cumsum(more, 0) - more, torch.cumsum(less, 0) - less
    fresh = (col >= have[:, None]) & (col < want[:, None])
    gone = (col >= want[:, None]) & (col < have[:, None])
    from_ring = ring[(state[0] + take[:, None] + col - have[:, None]) % n_pages]
    to_ring = (state[1] + give[:, None] + col - want[:, None]) % n_pages
    # pages given back: everything else is written to a place behind the ring that is cut off again
    ring.copy_(torch.cat([ring, ring[:1]]).scatter(0, torch.where(gone, to_ring, n_pages).flatten(), table.flatten())[:n_pages])
    table.copy_(torch.where(fresh, from_ring, torch.where(gone, -1, table)))
    state.copy_(state + torch.stack([more.sum(), less.sum()]))
    new = change.long().clamp(min=0)
    start = torch.cat([new.new_zeros(1), torch.cumsum(new, 0)])
    t = torch.arange(rows, device=_DEV)
    b = (torch.searchsorted(start, t, right=True) - 1).clamp(max=case["n_seq"] - 1)
    there = t < start[-1]
    at = t - start[b]
    key = torch.where(there, held[b] + at, 0)
    slot = torch.where(there, table[b, key // page].long() * page + key % page, -1)
    seq = torch.where(there, b, -1).to(torch.int32)
    return after.to(torch.int32), start.to(torch.int32), seq, there, held[b], at, slot


def _plain_plan(s):
    case = s["case"]
    own_len, start, seq, there, before, at, slot = _plain_step(s, s["change"], s["rows"])
    depth, mask = at, None
    if case["tree"]:
        # rows that are no token count as nodes of one more sequence
        total = sum(_uneven(case["n_seq"], case["max_new"]))
        seen = _ancestors(s["parent"][:total].long(), start.long(), case["n_seq"], case["max_new"])
        seen = seen[seq.clamp(min=0).long(), torch.where(there, at, 0)] & there[:, None]
        depth = seen.sum(-1) - 1
        mask = _words(seen, s["words"])
    pos = torch.where(there, case["first"] + before + depth, -1).to(torch.int32)
    after = _plain_step(s, s["back"], 0)[0]
    return [own_len, start, seq, pos, slot, mask, after, s["table"], s["ring"], s["state"]]


def _plain_tree(s):
    case = s["case"]
    b, n, h, kv, d, p = (case[x] for x in ("n_seq", "nodes", "n_heads", "n_kv", "head_dim", "prefix"))
    start, own_len = s["start"].long(), s["own_len"].long()
    count = start[1:] - start[:-1]
    node = torch.arange(n, device=_DEV)
    at = (start[:-1, None] + node).clamp(max=s["q"].shape[0] - 1)              # row of every node (one of another where there is none)
    q = s["q"][at].float().view(b, n, kv, h // kv, d) * (1.0 / math.sqrt(d))
    own_k = s["k"][s["page_table"].clamp(min=0).long()].flatten(1, 2).float()
    own_v = s["v"][s["page_table"].clamp(min=0).long()].flatten(1, 2).float()
    pre_k = s["k"][s["prefix_pages"].long()].flatten(0, 1)[:p].float()
    pre_v = s["v"][s["prefix_pages"].long()].flatten(0, 1)[:p].float()
    sp = torch.einsum("bikgd,pkd->bikgp", q, pre_k)
    so = torch.einsum("bikgd,bjkd->bikgj", q, own_k)
    key = torch.arange(so.shape[-1], device=_DEV)
    j = key[None, :] - (own_len - count)[:, None]                              # the key's node, below zero: before the tree
    jc = j.clamp(0, s["mask"].shape[1] * 64 - 1)
    words = s["mask"][at].gather(2, (jc // 64)[:, None, :].expand(b, n, -1))
    seen = (j < 0)[:, None] | (((words >> (jc % 64)[:, None, :]) & 1) != 0)
    seen &= (key[None, :] < own_len[:, None])[:, None]
    so = so.masked_fill(~seen[:, :, None, None, :], float("-inf"))
    top = torch.cat([sp, so], -1).amax(-1, keepdim=True)
    ep, eo = torch.exp(sp - top), torch.exp(so - top)
    total = ep.sum(-1, keepdim=True) + eo.sum(-1, keepdim=True)
    out = torch.einsum("bikgp,pkd->bikgd", ep, pre_v) + torch.einsum("bikgj,bjkd->bikgd", eo, own_v)
    return (out / total).reshape(b, n, h, d)[node < count[:, None]].to(s["q"].dtype)


def _plain_accept(s):
    page = s["case"]["page"]
    i = torch.arange(s["path"].shape[1], device=_DEV)
    on = i < s["n_path"][:, None]
    src, dst = s["base"][:, None] + s["path"], s["base"][:, None] + i
    src, dst = ((s["page_table"].gather(1, (x // page).long()).long() * page + x % page)[on] for x in (src, dst))
    k, v = (s[x].view(-1, *s[x].shape[2:]) for x in ("k", "v"))
    k[dst], v[dst] = k[src], v[src]
    return [s["k"], s["v"]]


def run(s):
    case = s["case"]
    if not own:
        return {"quant": _plain_quant, "linear": _plain_linear, "plan": _plain_plan, "tree": _plain_tree, "accept": _plain_accept}[case["op"]](s)
    from paper_2311_01305_b200 import aweq
    if case["op"] == "quant":
        return s["xq"].quantise(s["x"], s["m"]).values(s["out"])
    if case["op"] == "linear":
        return s["layer"](s["xq"].quantise(s["x"], s["rinv"]), s["out"])
    if case["op"] == "plan":
        p = s["pool"].plan(s["table"], s["held"], s["change"], s["grow"], first=case["first"], parent=s["parent"])
        after = s["pool"].plan(s["table"], p.own_len, s["back"], s["shrink"]).own_len
        return [p.own_len, p.start, p.seq, p.pos, p.slot, p.mask, after, s["table"], s["ring"], s["state"]]
    if case["op"] == "accept":
        aweq.aweq_kv_accept(s["cache"], s["page_table"], s["base"], s["path"], s["n_path"])
        return [s["k"], s["v"]]
    return s["attend"](s["q"], s["page_table"], s["own_len"], s["start"], s["mask"], s["out"])


# ---------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    op = case["op"]
    if op == "quant":
        n = case["rows"] * case["cols"]
        return {"bytes": 4 * n + 4 * case["cols"], "flops": 4 * n}
    if op == "linear":
        n, i, o, blk = case["n"], case["c_in"], case["c_out"], _BLOCK[case["fmt"]]
        rows = 0 if case["fmt"] == "e8m0" else 4 * o
        return {"bytes": int(2 * n * i + 4 * i + o * i / 2 + o * i / blk + rows + 2 * n * o + (4 * o if case["bias"] else 0)), "flops": 2 * n * i * o}
    if op == "plan":
        n, total = case["n_seq"], sum(_uneven(case["n_seq"], case["max_new"]))
        pages = total / case["page"]
        mask = (4 + 8 * ((case["max_new"] + 63) // 64)) * total if case["tree"] else 0
        return {"bytes": int(16 * total + mask + 4 * 8 * n + 4 * 4 * pages), "flops": int(4 * total)}
    if op == "accept":
        moved = sum(range(1, case["path"] + 1)) / case["path"] * case["n_seq"]
        return {"bytes": int(moved * (case["n_kv"] * case["head_dim"] * 8 + 4) + 8 * case["n_seq"]), "flops": int(moved)}
    h, kv, d, p = case["n_heads"], case["n_kv"], case["head_dim"], case["prefix"]
    total = sum(_uneven(case["n_seq"], case["nodes"]))
    own_len = total / case["n_seq"] + (case["max_own"] - case["nodes"]) * 0.625
    keys = p + case["n_seq"] * own_len
    return {"bytes": int(keys * kv * d * 4 + total * (h * d * 4 + 8) + keys / case["page"] * 4), "flops": int(4 * total * h * d * (p + own_len))}


# ---------------------------------------------------------------------------- the definitions in binary64
def _exact_values(x, m, fmt):
    """Every element of x times m replaced by what its code and scales stand for, in binary64."""
    v = x.double() * m.double()
    size = _BLOCK[fmt]
    blocks = v.view(-1, size)
    top = blocks.abs().max(1, keepdim=True).values
    if fmt == "e8m0":
        step = 2.0 ** (torch.floor(torch.log2(top.clamp(min=2.0 ** -149))) - 2.0).clamp(min=-127.0)
    else:
        row = (v.abs().max(1).values / 2688.0).repeat_interleave(v.shape[1] // size)[:, None]
        t = top / (6.0 * row)
        grid = torch.arange(0, 128, device=_DEV, dtype=torch.uint8)[:127].view(torch.float8_e4m3fn).double()
        near = torch.bucketize(t, (grid[1:] + grid[:-1]) / 2)                     # (a tie: down; it would take an unlikely one)
        step = grid[near] * row
    levels = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=_DEV)
    y = torch.where(step > 0, blocks.abs() / step, 0.0)
    mid = (levels[1:] + levels[:-1]) / 2
    up, down = torch.bucketize(y, mid, right=True), torch.bucketize(y, mid)
    code = torch.where(up % 2 == 0, up, down)                                      # a tie goes to the even code
    return (torch.sign(blocks) * levels[code] * step).view(v.shape)


def exact(case, seed):
    if case["op"] == "plan":
        return None
    s = _INPUTS[case["op"]](case, seed)
    if case["op"] == "quant":
        return _exact_values(s["x"], s["m"], case["fmt"])
    if case["op"] == "linear":
        y = _exact_values(s["x"], s["rinv"], case["fmt"]) @ _exact_values(s["w"], s["s"], case["fmt"]).T
        return y if s["bias"] is None else y + s["bias"].double()
    size = case["page"]
    if case["op"] == "accept":
        pools = [s["k"].double(), s["v"].double()]
        table, base, path, count = (s[x].tolist() for x in ("page_table", "base", "path", "n_path"))
        where = [(pg[(b0 + p[i]) // size], (b0 + p[i]) % size, pg[(b0 + i) // size], (b0 + i) % size)
                 for pg, b0, p, c in zip(table, base, path, count) for i in range(c)]
        sp, sr, dp, dr = torch.tensor(where, device=_DEV).T
        return [pool.index_put((dp, dr), pool[sp, sr]) for pool in pools]
    # one sequence after another: its keys in a row, a softmax over those that each node sees
    h, kv, d = case["n_heads"], case["n_kv"], case["head_dim"]
    out = torch.empty((s["q"].shape[0], h, d), dtype=torch.float64, device=_DEV)
    start, lens = s["start"].tolist(), s["own_len"].tolist()
    pk, pv = (s[x][s["prefix_pages"].long()].reshape(-1, kv, d)[:case["prefix"]].double() for x in ("k", "v"))
    for b, n in enumerate(lens):
        pages = s["page_table"][b, :-(-n // size)].long()
        keys, vals = (torch.cat([p, s[x][pages].reshape(-1, kv, d)[:n].double()]) for p, x in ((pk, "k"), (pv, "v")))
        r0, r1 = start[b], start[b + 1]
        before = case["prefix"] + n - (r1 - r0)
        bits = torch.stack([(s["mask"][r0:r1, j // 64] >> (j % 64)) & 1 for j in range(r1 - r0)], 1)
        for g in range(kv):
            q = s["q"][r0:r1, g * (h // kv):(g + 1) * (h // kv)].double()
            score = torch.einsum("ihd,jd->ihj", q, keys[:, g]) / math.sqrt(d)
            score[:, :, before:] = torch.where(bits[:, None] != 0, score[:, :, before:], -math.inf)
            out[r0:r1, g * (h // kv):(g + 1) * (h // kv)] = torch.softmax(score, -1) @ vals[:, g]
    return out
