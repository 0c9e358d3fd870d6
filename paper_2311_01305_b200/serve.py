"""Running the attention half of a calibrated decoder layer.

``AttentionBlock`` takes what ``calibrate.LayerCalibrator`` left for the inputs ``attn_in`` and
``o_in`` (1/s, the 8-bit codes of q, k, v and o with their Step / zero-point pairs, the corrected biases)
and answers with them: per call one per-token quantisation and one joint product for q, k and v,
one launch that rotates queries and keys and stores keys and values in their pages, the attention
over the shared prefix and each sequence's own keys, one quantisation and one product for o.
With ``fmt`` both products run in microscaled 4-bit floating point instead, on weights quantised with the
calibration's s.  ``verify`` is the same for trees of drafted tokens, whose places, positions and masks a
``StepPlan`` has.  Buffer management and call order only.

``python -m paper_2311_01305_b200.serve`` calibrates a layer of OPT-125M's widths on synthetic inputs,
fills a prefix, lets sixteen sequences continue it token by token, and says how far the outputs are
from the 16-bit layer and what a step takes; then lets them continue it by drafted trees, with 4-bit products.
"""
from __future__ import annotations

from typing import Dict, List, Optional, Sequence

import torch

from . import aweq, calibrate, synth


def joint_linear(cal: calibrate.LayerCalibrator, names: Sequence[str]) -> aweq.LinearW8A8:
    """The calibrated linears ``names``, which share an input, as one product (channels one after the other)."""
    outs = [cal.out[n] for n in names]
    return aweq.LinearW8A8(torch.cat([o["codes"] for o in outs]), torch.cat([o["step"] for o in outs]),
                           torch.cat([o["zp"] for o in outs]), torch.cat([o["bias_f32"] for o in outs]), copy=False)


def joint_linear_mx4(cal: calibrate.LayerCalibrator, names: Sequence[str], W: Dict[str, torch.Tensor], fmt: str,
                     bias: Optional[Dict[str, torch.Tensor]] = None) -> aweq.LinearMX4:
    """The linears ``names``, which share an input, in 4 bits as one product: the 16-bit weights ``W`` equalised by the calibration's
    s, the biases (of those that have one) corrected for the mean of the rounding."""
    inp = cal.out[next(l.input for l in cal.wl.linears if l.name == names[0])]
    b = None
    if bias is not None and any(bias.get(n) is not None for n in names):
        b = torch.cat([torch.zeros(W[n].shape[0], device=W[n].device) if bias.get(n) is None else bias[n].float() for n in names])
    return aweq.LinearMX4(torch.cat([W[n] for n in names]), fmt, inp["s"] if cal.equalized else None, b, inp["mu_hat"])


class _Scratch:
    """What lies between the calls of a block, for up to ``rows`` tokens; ``of(n)``: its first n rows."""

    def __init__(self, block: "AttentionBlock", rows: int):
        dev, self.rows, self.n = block.cache.k.device, rows, -1
        u8 = lambda c: (torch.empty((rows, c), dtype=torch.uint8, device=dev), torch.empty(rows, dtype=torch.float32, device=dev),  # noqa: E731
                        torch.empty(rows, dtype=torch.int32, device=dev))
        codes = (lambda c: aweq.MX4(rows, c, block.fmt, dev)) if block.fmt else u8  # noqa: E731
        self.x, self.o = codes(block.qkv.C_in), codes(block.o.C_in)
        h, kv, d = block.n_heads, block.n_kv, block.head_dim
        self.widths, self.d = [h * d, kv * d, kv * d], d
        self.qkv = torch.empty((rows, block.qkv.C_out), dtype=block.dtype, device=dev)
        self.q, self.attended = (torch.empty((rows, h, d), dtype=block.dtype, device=dev) for _ in range(2))

    def of(self, n: int):
        if n != self.n:
            x, o = (u.first(n) if isinstance(u, aweq.MX4) else tuple(t[:n] for t in u) for u in (self.x, self.o))
            qkv, q, attended = self.qkv[:n], self.q[:n], self.attended[:n]
            self.views = x, o, qkv, [t.unflatten(1, (-1, self.d)) for t in qkv.split(self.widths, 1)], q, attended, attended.flatten(1)
            self.n = n
        return self.views


class AttentionBlock:
    """``cal``: a calibrator that has run, of a workload with 8-bit row-wise weights and activation
    quantisation; what it left is copied.  ``pages`` / ``page_size``: the cache it makes (16-bit, in the workload's type).
    ``fmt``: one of ``aweq.MX4_FORMATS``; the products then run in 4 bits, on the 16-bit weights ``W`` (and ``bias``) that the
    calibrator had, of any workload, and of the calibration s, 1/s and E[x/s] are used.

    Several streams or threads may call a block at a time, each with an attention of its own (``attention``) and pages that the
    others do not write.  The block keeps one set of buffers for each that did, for the most tokens it had."""

    def __init__(self, cal: calibrate.LayerCalibrator, n_heads: int, pages: int, page_size: int = 16, rope: Optional[torch.Tensor] = None,
                 interleaved: bool = False, fmt: Optional[str] = None, W: Optional[Dict[str, torch.Tensor]] = None,
                 bias: Optional[Dict[str, torch.Tensor]] = None):
        wl = cal.wl
        if fmt is None and not (wl.act_quant and cal.bits == 8 and wl.w_gran == "row"):
            raise ValueError("the block runs W8A8 layers with row-wise weights")
        if fmt is not None and (fmt not in aweq.MX4_FORMATS or W is None):
            raise ValueError("fmt is one of %s, with the 16-bit weights W" % sorted(aweq.MX4_FORMATS))
        width = {l.name: l.c_out for l in wl.linears}
        self.n_heads, self.head_dim = n_heads, width["q"] // n_heads
        self.n_kv = width["k"] // self.head_dim
        self.dtype, dev = synth.torch_dtype(wl.dtype), cal.ws.device
        self.fmt = fmt
        self.qkv, self.o = (joint_linear(cal, n) if fmt is None else joint_linear_mx4(cal, n, W, fmt, bias) for n in (("q", "k", "v"), ("o",)))
        self.rinv = {i: cal.out[i]["rinv"].clone() if cal.equalized else None for i in ("attn_in", "o_in")}
        shape = (pages, page_size, self.n_kv, self.head_dim)
        self.cache = aweq.KVCache(torch.zeros(shape, dtype=self.dtype, device=dev), torch.zeros(shape, dtype=self.dtype, device=dev))
        self.rope, self.interleaved = rope, interleaved
        self._idle: Dict[int, List[_Scratch]] = {}          # by stream

    def _quantised(self, x: torch.Tensor, rinv, into):
        if self.fmt:
            return (into.quantise(x, rinv),)
        aweq.aweq_quant_act(x, rinv, 8, aweq.PER_ROW, None, *into)
        return into

    def attention(self, n_seq: int, n_q: int = 1, prefix_pages: Optional[torch.Tensor] = None, prefix_len: int = 0,
                  max_own: Optional[int] = None) -> aweq.PrefixAttention:
        """The attention of one batch shape (holds its scratch)."""
        return aweq.PrefixAttention(self.cache, prefix_pages, prefix_len, self.n_heads, n_seq, n_q, max_own)

    def drafts(self, n_seq: int, max_tokens: int, max_nodes: int, prefix_pages: Optional[torch.Tensor] = None, prefix_len: int = 0,
               max_own: Optional[int] = None) -> aweq.TreeAttention:
        """The attention of drafted trees, up to ``max_nodes`` tokens for each of ``n_seq`` sequences, ``max_tokens`` in all (holds
        its scratch)."""
        return aweq.TreeAttention(self.cache, prefix_pages, prefix_len, self.n_heads, n_seq, max_tokens, max_nodes, max_own)

    def __call__(self, x: torch.Tensor, attend: aweq.PrefixAttention, page_table: torch.Tensor, own_len: torch.Tensor, pos: torch.Tensor,
                 seq: torch.Tensor, st: Optional[torch.Tensor] = None) -> torch.Tensor:
        """``x`` [n_seq * n_q, C_in], the block's input of every new token, sequence by sequence; ``pos`` their positions
        (a shared prefix counts), ``seq`` their sequences, ``own_len`` each sequence's own keys, these included."""
        if x.dim() != 2 or x.shape != (attend.n_seq * attend.n_q, self.qkv.C_in) or attend.cache is not self.cache:
            raise ValueError("x must be [%d x %d], with an attention of this block" % (attend.n_seq * attend.n_q, self.qkv.C_in))

        def step(q, k, v, q_turned, attended):
            aweq.aweq_kv_append(self.cache, page_table, k, v, pos, seq=seq, first=attend.prefix_len, table=self.rope,
                                interleaved=self.interleaved, q=q, q_out=q_turned, st=st)
            attend(q_turned, page_table, own_len, attended, st=st)
        return self._run(x, step, st)

    def verify(self, x: torch.Tensor, attend: aweq.TreeAttention, page_table: torch.Tensor, plan: aweq.StepPlan,
               st: Optional[torch.Tensor] = None) -> torch.Tensor:
        """``x`` [max_tokens, C_in], the block's input of the nodes in the order of ``plan``, which ``PagePool.plan`` has filled with
        the trees and with ``first`` = the prefix's length; the rows behind the last node are padding, their outputs anything, as are those of
        nodes that found no page (slot below zero; counted in ``st``).  A path of nodes is then kept with ``aweq.aweq_kv_accept``, and the
        rest given back with a plan whose changes are below zero (what is held less what is kept: ``plan.own_len`` says what is held)."""
        if (not isinstance(attend, aweq.TreeAttention) or attend.cache is not self.cache or plan.mask is None or plan.trees is False
                or plan.n_seq != attend.n_seq or plan.max_tokens != attend.max_tokens or 64 * plan.words < attend.max_nodes
                or page_table.shape[0] != plan.n_seq or x.dim() != 2 or x.shape != (plan.max_tokens, self.qkv.C_in)):
            raise ValueError("x must be [%d x %d], with a plan filled with trees and an attention of this block for as many rows and sequences" % (
                plan.max_tokens, self.qkv.C_in))

        def step(q, k, v, q_turned, attended):
            aweq.aweq_kv_append_slots(self.cache, plan.slot, k, v, plan.pos, table=self.rope, interleaved=self.interleaved, q=q, q_out=q_turned,
                                      st=st)
            # (node 0's key by its position: own_len ends before the last node where the pool ran out)
            where = {} if plan.first is None else dict(pos=plan.pos, first=plan.first)
            attend(q_turned, page_table, plan.own_len, plan.start, plan.mask, attended, st=st, **where)
        return self._run(x, step, st)

    def _run(self, x: torch.Tensor, step, st: Optional[torch.Tensor]) -> torch.Tensor:
        # A set of the current stream that no other thread is using, or a new one; a call's work is in the stream when it gives its
        # set back.  A graph that is being captured keeps its own.
        capturing = torch.cuda.is_current_stream_capturing()
        idle = self._idle.setdefault(torch.cuda.current_stream(x.device).cuda_stream, [])
        try:
            scratch = None if capturing else idle.pop()
        except IndexError:
            scratch = None
        if scratch is None or scratch.rows < x.shape[0]:
            scratch = _Scratch(self, x.shape[0])
        for_x, for_o, qkv, (q, k, v), q_turned, attended, attended_rows = scratch.of(x.shape[0])
        self.qkv(*self._quantised(x, self.rinv["attn_in"], for_x), qkv, st=st)
        step(q, k, v, q_turned, attended)
        out = self.o(*self._quantised(attended_rows, self.rinv["o_in"], for_o), dtype=self.dtype, st=st)
        if not capturing:
            idle.append(scratch)
        return out


def _rotate(rope, y, pos):
    d, cs = y.shape[-1], rope[pos][:, None]
    c, s, a, b = cs[..., :d // 2], cs[..., d // 2:], y[..., :d // 2], y[..., d // 2:]
    return torch.cat([a * c - b * s, a * s + b * c], -1)


def _layer16(z, W, rope, n_heads, pos, hidden):
    """The 16-bit layer in binary32 on one sequence's tokens; ``hidden``: the (token, key) pairs that are not seen."""
    from torch.nn.functional import linear
    z = z.float()
    q, k, v = (linear(z, W[n].float()).unflatten(1, (n_heads, -1)) for n in ("q", "k", "v"))
    score = torch.einsum("ihd,jhd->hij", _rotate(rope, q, pos), _rotate(rope, k, pos)) * q.shape[-1] ** -0.5
    p = torch.softmax(score.masked_fill(hidden, float("-inf")), -1)
    return linear(torch.einsum("hij,jhd->ihd", p, v).flatten(1), W["o"].float())


def main(n_seq: int = 16, prefix: int = 500, steps: int = 8) -> float:
    wl = synth.workloads(1.0 / 128)["opt125m_model_w8a8"]
    X, W = synth.generate(wl, "cuda")
    cal = calibrate.LayerCalibrator(wl, 8, X, W)
    cal.run()
    n_heads, d, page = 12, 64, 16
    rope = aweq.aweq_rope_table(d, 4096)
    shared, own = -(-prefix // page), -(-steps // page)
    block = AttentionBlock(cal, n_heads, shared + n_seq * own, page, rope)
    order = torch.randperm(shared + n_seq * own, device="cuda").to(torch.int32)
    prefix_pages, table = order[:shared], order[shared:].view(n_seq, own)
    tokens = X["attn_in"][:prefix + n_seq * steps]

    # the prefix: one sequence whose pages become everybody's
    i32 = dict(dtype=torch.int32, device="cuda")
    first = block(tokens[:prefix], block.attention(1, prefix, max_own=prefix), prefix_pages.view(1, -1), torch.tensor([prefix], **i32),
                  torch.arange(prefix, **i32), torch.zeros(prefix, **i32))
    attend = block.attention(n_seq, 1, prefix_pages, prefix, own * page)
    seq, outs = torch.arange(n_seq, **i32), []
    x = tokens[prefix:].view(n_seq, steps, -1)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for t in range(steps):
        if t == 1:
            begin.record()
        outs.append(block(x[:, t].contiguous(), attend, table, torch.full((n_seq,), t + 1, **i32), torch.full((n_seq,), prefix + t, **i32), seq))
    end.record()
    torch.cuda.synchronize()

    # the 16-bit layer in binary32: every sequence by itself
    worst = 0.0
    for b in range(n_seq):
        z = torch.cat([tokens[:prefix], x[b]])
        pos = torch.arange(z.shape[0], device="cuda")
        y = _layer16(z, W, rope, n_heads, pos, pos[None, None] > pos[None, :, None])
        got = torch.cat([first, torch.stack([o[b] for o in outs])]).float()
        worst = max(worst, ((got - y).norm() / y.norm()).item())
    print("%d sequences after a prefix of %d tokens, %d steps: at most %.3f off the 16-bit layer (2-norm), %.0f us a step" % (
        n_seq, prefix, steps, worst, begin.elapsed_time(end) * 1e3 / (steps - 1)))
    return worst


def drafting(n_seq: int = 16, prefix: int = 500, steps: int = 8, nodes: int = 24, fmt: str = "e4m3") -> float:
    wl = synth.workloads(1.0 / 128)["opt125m_model_w8a8"]
    X, W = synth.generate(wl, "cuda")
    cal = calibrate.LayerCalibrator(wl, 8, X, W)
    cal.run()
    n_heads, d, page = 12, 64, 16
    rope = aweq.aweq_rope_table(d, 4096)
    own = nodes * (steps + 1)
    per_seq, shared = -(-own // page), -(-prefix // page)
    block = AttentionBlock(cal, n_heads, shared + n_seq * per_seq, page, rope, fmt=fmt, W=W)
    i32 = dict(dtype=torch.int32, device="cuda")

    # the prefix takes the first pages of the pool, the sequences' tables are empty
    ring = torch.randperm(shared + n_seq * per_seq, device="cuda").to(torch.int32)
    prefix_pages = ring[:shared].clone()
    pool = aweq.PagePool(ring.numel(), page, ring=ring, state=torch.tensor([shared, ring.numel()], device="cuda"))
    table, rows = torch.full((n_seq, per_seq), -1, **i32), n_seq * nodes
    tokens = X["attn_in"]
    block(tokens[:prefix], block.attention(1, prefix, max_own=prefix), prefix_pages.view(1, -1), torch.tensor([prefix], **i32),
          torch.arange(prefix, **i32), torch.zeros(prefix, **i32))

    # The drafts: trees of different sizes, and of each the path from a root to some node, which a model's choice would be in earnest.
    g = torch.Generator().manual_seed(1)
    draw = lambda n: int(torch.randint(0, n, (1,), generator=g))  # noqa: E731
    drafts = []
    for _ in range(steps):
        parents = [[draw(i + 1) - 1 for i in range(1 + draw(nodes))] for _ in range(n_seq)]
        paths = []
        for up in parents:
            path = [draw(len(up))]
            while up[path[0]] >= 0:
                path.insert(0, up[path[0]])
            paths.append(path)
        n = [len(up) for up in parents]
        flat = sum(parents, [])
        drafts.append((parents, paths, torch.tensor(n, **i32), torch.tensor(flat + [-1] * (rows - len(flat)), **i32),
                       torch.tensor([p + [0] * (nodes - len(p)) for p in paths], **i32), torch.tensor([len(p) for p in paths], **i32),
                       torch.tensor([len(p) - m for p, m in zip(paths, n)], **i32), tokens[prefix + torch.randint(0, tokens.shape[0] - prefix, (rows,), generator=g)]))
    attend = block.drafts(n_seq, rows, nodes, prefix_pages, prefix, own)
    grown, kept = aweq.StepPlan(n_seq, rows, nodes), aweq.StepPlan(n_seq, 0)
    kept.own_len.zero_()
    held, outs, st = kept.own_len, [], aweq.new_status()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for t, (_, _, n, parent, path, n_path, change, x) in enumerate(drafts):
        if t == 1:
            begin.record()
        pool.plan(table, held, n, grown, first=prefix, parent=parent, st=st)
        outs.append(block.verify(x, attend, table, grown, st))
        aweq.aweq_kv_accept(block.cache, table, held, path, n_path, st)
        pool.plan(table, grown.own_len, change, kept, st=st)
    end.record()
    torch.cuda.synchronize()
    if aweq.read_out_of_range(st) or aweq.read_status(st)["wait_timeout"]:
        raise RuntimeError("a step did not fit: %s, %d out of range" % (aweq.read_status(st), aweq.read_out_of_range(st)))

    # the 16-bit layer in binary32: every sequence's tree behind what it has kept
    worst, accepted, mine = 0.0, 0, [tokens[:prefix]] * n_seq
    for out, (parents, paths, *_, x) in zip(outs, drafts):
        at, square, total = 0, 0.0, 0.0
        for b, (up, path) in enumerate(zip(parents, paths)):
            own_x, old = x[at:at + len(up)], mine[b].shape[0]
            sees, depth = torch.zeros(len(up), old + len(up), dtype=torch.bool), []
            for i, u in enumerate(up):
                sees[i] = sees[i] | (sees[u] if u >= 0 else torch.arange(sees.shape[1]) < old)
                sees[i, old + i] = True
                depth.append(depth[u] + 1 if u >= 0 else 0)
            pos = torch.cat([torch.arange(old), old + torch.tensor(depth)])
            hidden = torch.cat([torch.ones(old, old + len(up), dtype=torch.bool).triu(1), ~sees])
            y = _layer16(torch.cat([mine[b], own_x]), W, rope, n_heads, pos.cuda(), hidden.cuda())[old:]
            square += float((out[at:at + len(up)].float() - y).norm() ** 2)
            total += float(y.norm() ** 2)
            mine[b] = torch.cat([mine[b], own_x[torch.tensor(path, device="cuda")]])
            accepted += len(path)
            at += len(up)
        worst = max(worst, (square / total) ** 0.5)
    print("%d sequences, trees of up to %d drafted tokens, %d steps in 4 bits (%s): %d tokens kept, at most %.3f off the 16-bit layer (2-norm), %.0f us a step" % (
        n_seq, nodes, steps, fmt, accepted, worst, begin.elapsed_time(end) * 1e3 / max(steps - 1, 1)))
    return worst


if __name__ == "__main__":
    main()
    drafting()
