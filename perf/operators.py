"""The operators of a calibrated decoder layer at work, as cases that can be timed and compared.

Three operators: the product of 8-bit codes with a (Step, zero-point) pair per token and per output
channel (``linear``), the appending of keys and values to a paged cache with the position rotation
applied on the way (``append``), and attention over that cache for a batch whose sequences share a
prefix (``attention``).  ``run`` computes a case in elementary torch operations in binary32, or,
where ``own`` is true, through this package.  ``exact`` evaluates the definitions in binary64.
"""
from __future__ import annotations

import math

import torch

own = False

_DEV = "cuda"
_DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # one token through an OPT-125M projection: nothing but latency
        dict(name="linear_1x768x768", op="linear", dtype="f16", n=1, c_in=768, c_out=768, act="token", bias=True),
        # sixteen sequences decoding through the joint q/k/v projection of a LLaMA-7B layer
        dict(name="linear_16x4096x12288", op="linear", dtype="f16", n=16, c_in=4096, c_out=12288, act="token", bias=True),
        # a ragged chunk of prompt tokens through LLaMA-13B's gate; one static activation range
        dict(name="linear_201x5120x13824", op="linear", dtype="bf16", n=201, c_in=5120, c_out=13824, act="tensor", bias=False),
        # a prompt through LLaMA-7B's up projection
        dict(name="linear_2048x4096x11008", op="linear", dtype="bf16", n=2048, c_in=4096, c_out=11008, act="token", bias=True),
        # a batch of prompts through OPT-66B's fc2: the longest rows the quantisers produce in a model
        dict(name="linear_4099x36864x9216", op="linear", dtype="f16", n=4099, c_in=36864, c_out=9216, act="token", bias=True),
        # one decoding step of 64 sequences, LLaMA-7B heads, positions after a shared prefix
        dict(name="append_64_decode", op="append", dtype="bf16", n_seq=64, max_new=1, n_heads=32, n_kv=32, head_dim=128,
             rotary_dim=128, interleaved=False, scaling="none", factor=1.0, n_pos=4096, first=2048, page=16),
        # ragged chunks of seven prompts, small heads rotated in part, interleaved pairs, odd page size
        dict(name="append_7_ragged", op="append", dtype="f16", n_seq=7, max_new=611, n_heads=12, n_kv=12, head_dim=64,
             rotary_dim=32, interleaved=True, scaling="linear", factor=2.0, n_pos=4096, first=0, page=24),
        # long prompts, shared key heads, positions far beyond the trained range (frequencies scaled by bands)
        dict(name="append_4_long", op="append", dtype="bf16", n_seq=4, max_new=8192, n_heads=40, n_kv=8, head_dim=128,
             rotary_dim=128, interleaved=False, scaling="bands", factor=8.0, n_pos=131072, first=65536, page=64),
        # a handful of continuations of a short instruction, OPT-125M heads
        dict(name="attn_4_short", op="attention", dtype="f16", n_seq=4, n_q=1, n_heads=12, n_kv=12, head_dim=64,
             prefix=257, max_own=60, page=16),
        # few-shot scoring: 32 questions after one set of worked examples, LLaMA-7B heads
        dict(name="attn_32_fewshot", op="attention", dtype="f16", n_seq=32, n_q=1, n_heads=32, n_kv=32, head_dim=128,
             prefix=2048, max_own=300, page=16),
        # five tokens of each sequence at once (drafted tokens being verified), ragged prefix
        dict(name="attn_8x5_draft", op="attention", dtype="bf16", n_seq=8, n_q=5, n_heads=32, n_kv=8, head_dim=128,
             prefix=4097, max_own=1000, page=32),
        # many users of one long document, shared key heads
        dict(name="attn_96_long", op="attention", dtype="bf16", n_seq=96, n_q=1, n_heads=32, n_kv=8, head_dim=128,
             prefix=32779, max_own=700, page=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "append", "attention"])
    dtype = rng.choice(["f16", "bf16"])
    if op == "linear":
        while True:
            n = _log_int(rng, 1, 8192)
            c_in = 16 * _log_int(rng, 4, 2304)
            c_out = _log_int(rng, 48, 16384)
            if n * c_in * c_out <= 4099 * 36864 * 9216 // 2:
                return dict(op=op, dtype=dtype, n=n, c_in=c_in, c_out=c_out, act=rng.choice(["token", "token", "tensor"]),
                            bias=rng.random() < 0.7)
    n_heads, n_kv = rng.choice([(12, 12), (16, 16), (32, 32), (40, 40), (32, 8), (40, 8), (24, 3), (16, 1)])
    head_dim = rng.choice([64, 80, 96, 128, 128])
    page = rng.choice([8, 16, 16, 24, 32, 64, 128])
    if op == "append":
        n_seq = _log_int(rng, 1, 128)
        max_new = 1 if rng.random() < 0.5 else _log_int(rng, 2, 32768 // n_seq)
        rotary_dim = rng.choice([head_dim, head_dim, head_dim // 2, 0])
        scaling = rng.choice(["none", "linear", "base", "bands"]) if rotary_dim else "none"
        n_pos = rng.choice([4096, 16384, 131072])
        n_pos = max(n_pos, 2 * max_new)
        return dict(op=op, dtype=dtype, n_seq=n_seq, max_new=max_new, n_heads=n_heads, n_kv=n_kv, head_dim=head_dim,
                    rotary_dim=rotary_dim, interleaved=rng.random() < 0.4, scaling=scaling,
                    factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0]), n_pos=n_pos,
                    first=rng.randrange(0, n_pos - max_new), page=page)
    while True:
        n_seq = _log_int(rng, 1, 128)
        n_q = 1 if rng.random() < 0.7 else rng.randint(2, 8)
        prefix = 0 if rng.random() < 0.05 else _log_int(rng, 16, 32768)
        max_own = _log_int(rng, max(n_q, 2), 2048)
        rows = n_seq * n_q * n_heads
        if rows * prefix <= 96 * 32 * 32779 and n_seq * max_own * n_kv * head_dim <= 128 * 1024 * 1024:
            return dict(op=op, dtype=dtype, n_seq=n_seq, n_q=n_q, n_heads=n_heads, n_kv=n_kv, head_dim=head_dim,
                        prefix=prefix, max_own=max_own, page=page)


# ---------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device=_DEV).manual_seed(int(seed) * 7919 + 11)


def _codes(v):
    """Asymmetric 8-bit codes of every row: (codes, Step, zero-point)."""
    lo, hi = v.amin(1), v.amax(1)
    step = (hi - lo) / 255.0
    zp = -torch.round(lo / step)
    q = (torch.round(v / step[:, None]) + zp[:, None]).clamp_(0, 255)
    return q.to(torch.uint8), step, zp.to(torch.int32)


def _linear_inputs(case, seed):
    g = _gen(seed)
    n, c_in, c_out = case["n"], case["c_in"], case["c_out"]
    x = torch.randn((n, c_in), generator=g, device=_DEV)
    x.mul_(1.0 + 0.5 * torch.rand(c_in, generator=g, device=_DEV)).add_(0.3 * torch.randn(c_in, generator=g, device=_DEV))
    x[:, torch.randint(0, c_in, (max(1, c_in // 512),), generator=g, device=_DEV)] *= 8.0     # outlier channels
    if case["act"] == "token":
        xq, x_step, x_zp = _codes(x)
    else:
        xq, x_step, x_zp = _codes(x.reshape(1, -1))
        xq = xq.reshape(n, c_in)
    wq, w_step, w_zp = _codes(torch.randn((c_out, c_in), generator=g, device=_DEV).mul_(0.02))
    bias = 0.1 * torch.randn(c_out, generator=g, device=_DEV) if case["bias"] else None
    return dict(xq=xq, x_step=x_step, x_zp=x_zp, wq=wq, w_step=w_step, w_zp=w_zp, bias=bias)


def _frequencies(case):
    """Rotation frequencies (binary64, radians per position) of a case, scaled for long contexts."""
    rd, factor = case["rotary_dim"], case["factor"]
    theta = 10000.0
    if case["scaling"] == "base":
        theta *= factor ** (rd / (rd - 2))
    freq = theta ** (-torch.arange(0, rd, 2, dtype=torch.float64, device=_DEV) / rd)
    if case["scaling"] == "linear":
        freq = freq / factor
    if case["scaling"] == "bands":
        # more than 4 turns within the trained 8192 positions: kept; fewer than 1: divided by the factor
        keep = ((8192.0 * freq / (2 * math.pi) - 1.0) / 3.0).clamp(0.0, 1.0)
        freq = freq * (keep + (1.0 - keep) / factor)
    return freq


def _new_tokens(case):
    """Tokens that a case brings for each of its sequences: uneven, between half of the most and the most."""
    most = case["max_new"]
    return [most - (most * i // (2 * case["n_seq"])) for i in range(case["n_seq"])]


def _append_inputs(case, seed):
    g = _gen(seed)
    dt = _DTYPES[case["dtype"]]
    n_seq, h, kv, d, page = case["n_seq"], case["n_heads"], case["n_kv"], case["head_dim"], case["page"]
    new = torch.tensor(_new_tokens(case), device=_DEV)[torch.randperm(n_seq, generator=g, device=_DEV)]
    seq = torch.repeat_interleave(torch.arange(n_seq, device=_DEV), new)
    begin = torch.cumsum(new, 0) - new
    spare = case["n_pos"] - case["first"] - case["max_new"]
    held = torch.randint(0, min(spare, 200) + 1, (n_seq,), generator=g, device=_DEV)       # tokens each sequence has already
    at = held[seq] + torch.arange(seq.numel(), device=_DEV) - begin[seq]
    tokens = seq.numel()
    per_seq = (case["max_new"] + min(spare, 200)) // page + 1
    n_pages = n_seq * per_seq + 3
    table = torch.randperm(n_pages, generator=g, device=_DEV)[:n_seq * per_seq].reshape(n_seq, per_seq).to(torch.int32)
    qkv = torch.randn((tokens, (h + 2 * kv) * d), generator=g, device=_DEV).to(dt)
    s = dict(qkv=qkv, seq=seq.to(torch.int32), pos=(case["first"] + at).to(torch.int32), page_table=table,
             k=torch.randn((n_pages, page, kv, d), generator=g, device=_DEV).to(dt),
             v=torch.randn((n_pages, page, kv, d), generator=g, device=_DEV).to(dt))
    s["q"], s["k_new"], s["v_new"] = (t.unflatten(1, (-1, d)) for t in qkv.split([h * d, kv * d, kv * d], 1))
    return s


def _attention_inputs(case, seed):
    g = _gen(seed)
    dt = _DTYPES[case["dtype"]]
    n_seq, kv, d, page = case["n_seq"], case["n_kv"], case["head_dim"], case["page"]
    per_seq = -(-case["max_own"] // page)
    shared = -(-case["prefix"] // page)
    n_pages = shared + n_seq * per_seq + 1
    order = torch.randperm(n_pages, generator=g, device=_DEV).to(torch.int32)
    own_len = torch.randint(max(case["n_q"], case["max_own"] // 4), case["max_own"] + 1, (n_seq,), generator=g, device=_DEV)
    table = order[shared:shared + n_seq * per_seq].reshape(n_seq, per_seq).clone()
    used = (own_len + page - 1) // page
    table[torch.arange(per_seq, device=_DEV)[None, :] >= used[:, None]] = -1               # pages not given out yet
    k = torch.randn((n_pages, page, kv, d), generator=g, device=_DEV)
    k *= 0.5 + torch.rand(d, generator=g, device=_DEV)                                     # channels of unlike size
    # queries that resemble keys somewhat: a softmax that is neither flat nor a single peak
    q = 2.0 * torch.randn((n_seq * case["n_q"], case["n_heads"], d), generator=g, device=_DEV)
    return dict(q=q.to(dt), k=k.to(dt), v=torch.randn((n_pages, page, kv, d), generator=g, device=_DEV).to(dt),
                prefix_pages=order[:shared].clone(), page_table=table, own_len=own_len.to(torch.int32))


_INPUTS = {"linear": _linear_inputs, "append": _append_inputs, "attention": _attention_inputs}


def prepare(case, seed):
    s = _INPUTS[case["op"]](case, seed)
    s["case"] = case
    dt = _DTYPES[case["dtype"]]
    if case["op"] == "linear":
        s["out"] = torch.empty((case["n"], case["c_out"]), dtype=dt, device=_DEV)
    if case["op"] == "append":
        s["table"] = None
        if case["rotary_dim"]:
            angle = torch.arange(case["n_pos"], dtype=torch.float64, device=_DEV)[:, None] * _frequencies(case)[None, :]
            s["table"] = torch.cat([angle.cos(), angle.sin()], 1).to(torch.float32)
        s["q_out"] = torch.empty_like(s["q"], memory_format=torch.contiguous_format)
    if case["op"] == "attention":
        s["out"] = torch.empty_like(s["q"])
    if own:
        from paper_2311_01305_b200 import aweq
        if case["op"] == "linear":
            s["layer"] = aweq.LinearW8A8(s["wq"], s["w_step"], s["w_zp"], s["bias"])
        else:
            s["cache"] = aweq.KVCache(s["k"], s["v"])
        if case["op"] == "attention":
            s["attend"] = aweq.PrefixAttention(s["cache"], s["prefix_pages"], case["prefix"], case["n_heads"], case["n_seq"],
                                               case["n_q"], case["max_own"])
    return s


# ---------------------------------------------------------------------------- the passes
def _plain_linear(s):
    x = (s["xq"].float() - s["x_zp"].float()[:, None]) * s["x_step"][:, None]
    w = (s["wq"].float() - s["w_zp"].float()[:, None]) * s["w_step"][:, None]
    y = x @ w.t()
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(s["out"].dtype)


def _plain_rotate(x, s):
    case = s["case"]
    rd = case["rotary_dim"]
    if not rd:
        return x
    cs = s["table"][s["pos"].long()]
    c, n = cs[:, None, :rd // 2], cs[:, None, rd // 2:]
    f = x.float()
    if case["interleaved"]:
        a, b = f[..., 0:rd:2], f[..., 1:rd:2]
        turned = torch.stack([a * c - b * n, a * n + b * c], -1).flatten(-2)
    else:
        a, b = f[..., :rd // 2], f[..., rd // 2:rd]
        turned = torch.cat([a * c - b * n, a * n + b * c], -1)
    return torch.cat([turned, f[..., rd:]], -1).to(x.dtype)


def _plain_append(s):
    case = s["case"]
    at = s["pos"].long() - case["first"]
    page = s["page_table"][s["seq"].long(), at // case["page"]].long()
    row = at % case["page"]
    s["k"][page, row] = _plain_rotate(s["k_new"], s)
    s["v"][page, row] = s["v_new"]
    return [_plain_rotate(s["q"], s), s["k"], s["v"]]


def _plain_attention(s):
    case = s["case"]
    b, n_q, h, kv, d, p = (case[x] for x in ("n_seq", "n_q", "n_heads", "n_kv", "head_dim", "prefix"))
    q = s["q"].float().view(b, n_q, kv, h // kv, d) * (1.0 / math.sqrt(d))
    own_k = s["k"][s["page_table"].clamp(min=0).long()].flatten(1, 2).float()
    own_v = s["v"][s["page_table"].clamp(min=0).long()].flatten(1, 2).float()
    pre_k = s["k"][s["prefix_pages"].long()].flatten(0, 1)[:p].float()
    pre_v = s["v"][s["prefix_pages"].long()].flatten(0, 1)[:p].float()
    sp = torch.einsum("bikgd,pkd->bikgp", q, pre_k)
    so = torch.einsum("bikgd,bjkd->bikgj", q, own_k)
    last = s["own_len"][:, None] - (n_q - 1) + torch.arange(n_q, device=q.device)[None, :]     # own keys seen by token i
    seen = torch.arange(so.shape[-1], device=q.device)[None, None, :] < last[:, :, None]
    so = so.masked_fill(~seen[:, :, None, None, :], float("-inf"))
    top = torch.cat([sp, so], -1).amax(-1, keepdim=True)
    ep, eo = torch.exp(sp - top), torch.exp(so - top)
    total = ep.sum(-1, keepdim=True) + eo.sum(-1, keepdim=True)
    out = torch.einsum("bikgp,pkd->bikgd", ep, pre_v) + torch.einsum("bikgj,bjkd->bikgd", eo, own_v)
    return (out / total).reshape(b * n_q, h, d).to(s["q"].dtype)


def run(s):
    case = s["case"]
    if not own:
        return {"linear": _plain_linear, "append": _plain_append, "attention": _plain_attention}[case["op"]](s)
    from paper_2311_01305_b200 import aweq
    if case["op"] == "linear":
        return s["layer"](s["xq"], s["x_step"], s["x_zp"], s["out"])
    if case["op"] == "append":
        aweq.aweq_kv_append(s["cache"], s["page_table"], s["k_new"], s["v_new"], s["pos"], seq=s["seq"], first=case["first"],
                            table=s["table"], interleaved=case["interleaved"], q=s["q"], q_out=s["q_out"])
        return [s["q_out"], s["k"], s["v"]]
    return s["attend"](s["q"], s["page_table"], s["own_len"], s["out"])


# ---------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "linear":
        n, i, o = case["n"], case["c_in"], case["c_out"]
        pairs = n if case["act"] == "token" else 1
        return {"bytes": n * i + o * i + 2 * n * o + 8 * (pairs + o) + (4 * o if case["bias"] else 0), "flops": 2 * n * i * o}
    h, kv, d = case["n_heads"], case["n_kv"], case["head_dim"]
    if case["op"] == "append":
        tokens = sum(_new_tokens(case))
        rows = min(tokens, case["n_pos"])
        return {"bytes": int(tokens * ((h + 2 * kv) * d * 4 + 8) + rows * case["rotary_dim"] * 4 + tokens / case["page"] * 4),
                "flops": int(tokens * (h + kv) * case["rotary_dim"] * 3)}
    b, n_q, p = case["n_seq"], case["n_q"], case["prefix"]
    own_len = (max(n_q, case["max_own"] // 4) + case["max_own"]) / 2
    return {"bytes": int((p + b * own_len) * kv * d * 4 + b * n_q * h * d * 4 + (p + b * own_len) / case["page"] * 4 + 4 * b),
            "flops": int(4 * b * n_q * h * d * (p + own_len))}


# ---------------------------------------------------------------------------- the definitions in binary64
def exact(case, seed):
    s = _INPUTS[case["op"]](case, seed)
    if case["op"] == "linear":
        # integers first (sums of products of codes are exact in binary64), then the two Steps
        acc = (s["xq"].double() - s["x_zp"].double().view(-1, 1)) @ (s["wq"].double() - s["w_zp"].double().view(-1, 1)).T
        acc = acc * s["x_step"].double().view(-1, 1) * s["w_step"].double()
        return acc if s["bias"] is None else acc + s["bias"].double()
    if case["op"] == "append":
        rd = case["rotary_dim"]

        def rotated(x):
            # (a + ib) e^{i pos f} of every pair
            y = x.double()
            if rd:
                turn = torch.polar(torch.ones((), dtype=torch.float64, device=_DEV),
                                   s["pos"].double()[:, None, None] * _frequencies(case))
                order = torch.arange(rd, device=_DEV).view(-1, 2) if case["interleaved"] else torch.arange(rd, device=_DEV).view(2, -1).T
                z = torch.complex(y[..., order[:, 0]], y[..., order[:, 1]]) * turn
                y[..., order[:, 0]], y[..., order[:, 1]] = z.real, z.imag
            return y

        k, v = s["k"].double(), s["v"].double()
        size = case["page"]
        lin = s["page_table"].long().gather(0, s["seq"].long()[:, None].expand(-1, s["page_table"].shape[1]))
        at = s["pos"].long() - case["first"]
        slot = lin.gather(1, (at // size)[:, None])[:, 0] * size + at % size
        k.view(-1, *k.shape[2:]).index_copy_(0, slot, rotated(s["k_new"]))
        v.view(-1, *v.shape[2:]).index_copy_(0, slot, s["v_new"].double())
        return [rotated(s["q"]), k, v]
    # one sequence after another: its keys in a row, an ordinary softmax over them
    n_q, h, kv, d = case["n_q"], case["n_heads"], case["n_kv"], case["head_dim"]
    out = torch.empty((case["n_seq"] * n_q, h, d), dtype=torch.float64, device=_DEV)
    lens = s["own_len"].tolist()
    pk = s["k"][s["prefix_pages"].long()].reshape(-1, kv, d)[:case["prefix"]].double()
    pv = s["v"][s["prefix_pages"].long()].reshape(-1, kv, d)[:case["prefix"]].double()
    for b, n in enumerate(lens):
        pages = s["page_table"][b, :-(-n // case["page"])].long()
        keys = torch.cat([pk, s["k"][pages].reshape(-1, kv, d)[:n].double()]).repeat_interleave(h // kv, 1)
        vals = torch.cat([pv, s["v"][pages].reshape(-1, kv, d)[:n].double()]).repeat_interleave(h // kv, 1)
        for i in range(n_q):
            upto = keys.shape[0] - (n_q - 1 - i)
            score = (keys[:upto] * s["q"][b * n_q + i].double()).sum(-1) / math.sqrt(d)
            out[b * n_q + i] = (torch.softmax(score, 0)[..., None] * vals[:upto]).sum(0)
    return out
