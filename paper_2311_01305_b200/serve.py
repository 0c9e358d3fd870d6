"""Running the attention half of a calibrated W8A8 decoder layer.

``AttentionBlock`` takes what ``calibrate.LayerCalibrator`` left for the inputs ``attn_in`` and
``o_in`` (1/s, the 8-bit codes of q, k, v and o with their Step / zero-point pairs, the corrected biases)
and answers with them: per call one per-token quantisation and one joint product for q, k and v,
one launch that rotates queries and keys and stores keys and values in their pages, the attention
over the shared prefix and each sequence's own keys, one quantisation and one product for o.
Buffer management and call order only.

``python -m paper_2311_01305_b200.serve`` calibrates a layer of OPT-125M's widths on synthetic inputs,
fills a prefix, lets sixteen sequences continue it token by token, and says how far the outputs are
from the 16-bit layer and what a step takes.
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


class _Scratch:
    """What lies between the calls of a block, for up to ``rows`` tokens; ``of(n)``: its first n rows."""

    def __init__(self, block: "AttentionBlock", rows: int):
        dev, self.rows, self.n = block.cache.k.device, rows, -1
        u8 = lambda c: (torch.empty((rows, c), dtype=torch.uint8, device=dev), torch.empty(rows, dtype=torch.float32, device=dev),  # noqa: E731
                        torch.empty(rows, dtype=torch.int32, device=dev))
        self.x, self.o = u8(block.qkv.C_in), u8(block.o.C_in)
        h, kv, d = block.n_heads, block.n_kv, block.head_dim
        self.widths, self.d = [h * d, kv * d, kv * d], d
        self.qkv = torch.empty((rows, block.qkv.C_out), dtype=block.dtype, device=dev)
        self.q, self.attended = (torch.empty((rows, h, d), dtype=block.dtype, device=dev) for _ in range(2))

    def of(self, n: int):
        if n != self.n:
            x, o = (tuple(t[:n] for t in u) for u in (self.x, self.o))
            qkv, q, attended = self.qkv[:n], self.q[:n], self.attended[:n]
            self.views = x, o, qkv, [t.unflatten(1, (-1, self.d)) for t in qkv.split(self.widths, 1)], q, attended, attended.flatten(1)
            self.n = n
        return self.views


class AttentionBlock:
    """``cal``: a calibrator that has run, of a workload with 8-bit row-wise weights and activation
    quantisation; what it left is copied.  ``pages`` / ``page_size``: the cache it makes (16-bit, in the workload's type).

    Several streams or threads may call a block at a time, each with an attention of its own (``attention``) and pages that the
    others do not write.  The block keeps one set of buffers for each that did, for the most tokens it had."""

    def __init__(self, cal: calibrate.LayerCalibrator, n_heads: int, pages: int, page_size: int = 16, rope: Optional[torch.Tensor] = None,
                 interleaved: bool = False):
        wl = cal.wl
        if not (wl.act_quant and cal.bits == 8 and wl.w_gran == "row"):
            raise ValueError("the block runs W8A8 layers with row-wise weights")
        width = {l.name: l.c_out for l in wl.linears}
        self.n_heads, self.head_dim = n_heads, width["q"] // n_heads
        self.n_kv = width["k"] // self.head_dim
        self.dtype, dev = synth.torch_dtype(wl.dtype), cal.ws.device
        self.qkv, self.o = joint_linear(cal, ("q", "k", "v")), joint_linear(cal, ("o",))
        self.rinv = {i: cal.out[i]["rinv"].clone() if cal.equalized else None for i in ("attn_in", "o_in")}
        shape = (pages, page_size, self.n_kv, self.head_dim)
        self.cache = aweq.KVCache(torch.zeros(shape, dtype=self.dtype, device=dev), torch.zeros(shape, dtype=self.dtype, device=dev))
        self.rope, self.interleaved = rope, interleaved
        self._idle: Dict[int, List[_Scratch]] = {}          # by stream

    def _quantised(self, x: torch.Tensor, rinv, into):
        aweq.aweq_quant_act(x, rinv, 8, aweq.PER_ROW, None, *into)
        return into

    def attention(self, n_seq: int, n_q: int = 1, prefix_pages: Optional[torch.Tensor] = None, prefix_len: int = 0,
                  max_own: Optional[int] = None) -> aweq.PrefixAttention:
        """The attention of one batch shape (holds its scratch)."""
        return aweq.PrefixAttention(self.cache, prefix_pages, prefix_len, self.n_heads, n_seq, n_q, max_own)

    def __call__(self, x: torch.Tensor, attend: aweq.PrefixAttention, page_table: torch.Tensor, own_len: torch.Tensor, pos: torch.Tensor,
                 seq: torch.Tensor, st: Optional[torch.Tensor] = None) -> torch.Tensor:
        """``x`` [n_seq * n_q, C_in], the block's input of every new token, sequence by sequence; ``pos`` their positions
        (a shared prefix counts), ``seq`` their sequences, ``own_len`` each sequence's own keys, these included."""
        if x.dim() != 2 or x.shape != (attend.n_seq * attend.n_q, self.qkv.C_in) or attend.cache is not self.cache:
            raise ValueError("x must be [%d x %d], with an attention of this block" % (attend.n_seq * attend.n_q, self.qkv.C_in))
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
        aweq.aweq_kv_append(self.cache, page_table, k, v, pos, seq=seq, first=attend.prefix_len, table=self.rope,
                            interleaved=self.interleaved, q=q, q_out=q_turned, st=st)
        attend(q_turned, page_table, own_len, attended, st=st)
        out = self.o(*self._quantised(attended_rows, self.rinv["o_in"], for_o), dtype=self.dtype, st=st)
        if not capturing:
            idle.append(scratch)
        return out


def main(n_seq: int = 16, prefix: int = 500, steps: int = 8) -> float:
    from torch.nn.functional import linear
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
    def rotate(y, pos):
        cs = rope[pos][:, None]
        c, s, a, b = cs[..., :d // 2], cs[..., d // 2:], y[..., :d // 2], y[..., d // 2:]
        return torch.cat([a * c - b * s, a * s + b * c], -1)
    worst = 0.0
    for b in range(n_seq):
        z = torch.cat([tokens[:prefix], x[b]]).float()
        q, k, v = (linear(z, W[n].float()).view(-1, n_heads, d) for n in ("q", "k", "v"))
        pos = torch.arange(z.shape[0], device="cuda")
        score = torch.einsum("ihd,jhd->hij", rotate(q, pos), rotate(k, pos)) * d ** -0.5
        p = torch.softmax(score.masked_fill(pos[None, None] > pos[None, :, None], float("-inf")), -1)
        y = linear(torch.einsum("hij,jhd->ihd", p, v).flatten(1), W["o"].float())
        got = torch.cat([first, torch.stack([o[b] for o in outs])]).float()
        worst = max(worst, ((got - y).norm() / y.norm()).item())
    print("%d sequences after a prefix of %d tokens, %d steps: at most %.3f off the 16-bit layer (2-norm), %.0f us a step" % (
        n_seq, prefix, steps, worst, begin.elapsed_time(end) * 1e3 / (steps - 1)))
    return worst


if __name__ == "__main__":
    main()
