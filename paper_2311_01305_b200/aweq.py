"""Thin Python binding of the C-ABI CUDA library ``libaweq.so``.

Every function here has the name and the argument order of the C entry point
declared in ``include/aweq.h`` and does argument marshalling only: tensors
become device pointers, the current PyTorch CUDA stream becomes the ``stream``
argument, scratch memory is a ``torch.uint8`` tensor.  All arithmetic of the
AWEQ calibration pass (arXiv 2311.01305) runs in the library's kernels; there
is no Python or CPU fallback, and importing this module fails loudly when the
library has not been built (``python -m paper_2311_01305_b200.build``).
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libaweq.so")
if not os.path.exists(LIB_PATH):
    raise ImportError(
        "libaweq.so is missing: build the CUDA library first with "
        "`python -m paper_2311_01305_b200.build` (needs nvcc; no GPU required to build)")
_lib = ctypes.CDLL(LIB_PATH)

OK = 0
F16, BF16 = 0, 1
PER_TENSOR, PER_ROW, PER_GROUP = 0, 1, 2
OP_STATS, OP_WRANGE, OP_EQUALIZE_QUANTIZE, OP_BIAS_CORRECT, OP_QUANT_ACT = 1, 2, 4, 5, 6
FLAG_NO_EQUALIZE, FLAG_NO_BIAS_CORRECT = 1, 2
FLAG_PHASE_REDUCE, FLAG_PHASE_QUANT, FLAG_PHASE_ACT = 4, 8, 16
FLAG_ABSMAX_CRITERION = 32
FLAG_MERGED_STATS = 64
ROPE_SCALINGS = {"none": 0, "linear": 1, "base": 2, "bands": 3}

_vp, _ll, _i, _sz = ctypes.c_void_p, ctypes.c_longlong, ctypes.c_int, ctypes.c_size_t


class DevStatus(ctypes.Structure):
    _fields_ = [("nonfinite", ctypes.c_ulonglong), ("zero_range", ctypes.c_ulonglong),
                ("wait_timeout", ctypes.c_ulonglong), ("out_of_range", ctypes.c_ulonglong)]


class LayerArgs(ctypes.Structure):
    _fields_ = [
        ("X", _vp), ("dt", _i), ("N", _ll), ("C_in", _ll), ("ldx", _ll),
        ("n_w", _i), ("W", ctypes.POINTER(_vp)), ("C_out", ctypes.POINTER(_ll)), ("ldw", ctypes.POINTER(_ll)),
        ("bits", _i), ("gran", _i), ("group", _i),
        ("bias_in", ctypes.POINTER(_vp)), ("bias_out", ctypes.POINTER(_vp)), ("bias_out_f32", ctypes.POINTER(_vp)),
        ("codes", ctypes.POINTER(_vp)), ("step", ctypes.POINTER(_vp)), ("zp", ctypes.POINTER(_vp)),
        ("epsmu", ctypes.POINTER(_vp)),
        ("xmin", _vp), ("xmax", _vp), ("xmean", _vp), ("wmin", _vp), ("wmax", _vp), ("s", _vp), ("rinv", _vp),
        ("mu_hat", _vp), ("pX", _vp), ("pW", _vp), ("scalars", _vp),
        ("Xq", _vp), ("act_step", _vp), ("act_zp", _vp), ("act_bits", _i), ("flags", _i),
        ("ev_stats_begin", _vp), ("ev_stats_end", _vp), ("ev_act_begin", _vp), ("ev_act_end", _vp),
        ("stat_negmin_max", _vp), ("stat_sum_count", _vp),
    ]


class RopeSpec(ctypes.Structure):
    _fields_ = [("rotary_dim", _i), ("scaling", _i), ("theta", ctypes.c_double), ("factor", ctypes.c_double),
                ("original_len", ctypes.c_double), ("low", ctypes.c_double), ("high", ctypes.c_double),
                ("attention", ctypes.c_double)]


class KvCacheArgs(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("dt", _i), ("page_size", _i), ("n_kv_heads", _i), ("head_dim", _i),
                ("n_pages", _ll), ("page_stride", _ll), ("token_stride", _ll), ("head_stride", _ll)]


_lib.aweq_strerror.restype = ctypes.c_char_p
_lib.aweq_strerror.argtypes = [_i]
_lib.aweq_last_cuda_error.restype = ctypes.c_char_p
_lib.aweq_version.restype = _i
_lib.aweq_launch_count.restype = ctypes.c_ulonglong
_lib.aweq_workspace_bytes.restype = _sz
_lib.aweq_workspace_bytes.argtypes = [_i, _ll, _ll, _i, _i, _i]
_lib.aweq_stats.argtypes = [_vp, _i, _ll, _ll, _ll, _vp, _vp, _vp, _vp, _vp, _i, _vp, _sz, _vp, _vp]
_lib.aweq_stats_static.argtypes = [_vp, _i, _ll, _ll, _ll, _vp, _vp, _vp, _vp, _vp]
_lib.aweq_stats_static.restype = _i
_lib.aweq_wrange.argtypes = [_vp, _i, _ll, _ll, _ll, _vp, _vp, _i, _vp, _sz, _vp, _vp]
_lib.aweq_factors.argtypes = [_vp, _vp, _vp, _vp, _vp, _ll, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]
_lib.aweq_factors_absmax.argtypes = [_vp, _vp, _vp, _vp, _vp, _ll, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]
_lib.aweq_factors_absmax.restype = _i
_lib.aweq_equalize_quantize.argtypes = [_vp, _i, _ll, _ll, _ll, _vp, _vp, _i, _i, _i, _vp, _vp, _vp, _vp, _vp, _sz,
                                        _vp, _vp]
_lib.aweq_bias_correct.argtypes = [_vp, _vp, _i, _vp, _vp, _vp, _vp, _vp, _ll, _ll, _ll, _i, _i, _i, _vp, _vp, _vp,
                                   _i, _vp, _vp]
_lib.aweq_quant_act.argtypes = [_vp, _i, _ll, _ll, _ll, _vp, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp]
_lib.aweq_layer_pass_workspace_bytes.restype = _sz
_lib.aweq_layer_pass_workspace_bytes.argtypes = [ctypes.POINTER(LayerArgs)]
_lib.aweq_layer_pass_fuses_ranges.restype = ctypes.c_int
_lib.aweq_layer_pass_fuses_ranges.argtypes = [ctypes.POINTER(LayerArgs)]
_lib.aweq_layer_pass.argtypes = [ctypes.POINTER(LayerArgs), _vp, _sz, _vp, _vp]
_lib.aweq_plan_query.argtypes = [_i, _ll, _ll, ctypes.POINTER(_ll * 8)]
_lib.aweq_plan_query.restype = _i
_lib.aweq_relabel_signed.argtypes = [_vp, _ll, _vp, _vp, _ll, _vp, _vp]
_lib.aweq_relabel_signed.restype = _i
_lib.aweq_fold_scale.argtypes = [_vp, _i, _ll, _ll, _ll, _vp, _vp, _ll, _vp]
_lib.aweq_fold_scale.restype = _i
_lib.aweq_forward_check_workspace_bytes.restype = _sz
_lib.aweq_forward_check_workspace_bytes.argtypes = [_ll, _ll, _ll]
_lib.aweq_forward_check.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i, _vp, _ll, _ll, _ll, _vp, _vp, _vp,
                                    _sz, _vp]
_lib.aweq_forward_check_weights_workspace_bytes.restype = _sz
_lib.aweq_forward_check_weights_workspace_bytes.argtypes = [_ll, _ll, _ll]
_lib.aweq_forward_check_weights.argtypes = [_vp, _vp, _vp, _i, _i, _i, _vp, _vp, _vp, _vp, _i, _vp, _ll, _ll, _ll, _vp, _vp,
                                            _vp, _sz, _vp]
_lib.aweq_forward_check_weights.restype = _i
_lib.aweq_code_sums.argtypes = [_vp, _ll, _ll, _ll, _vp, _vp]
_lib.aweq_code_sums.restype = _i
_lib.aweq_linear_w8a8.argtypes = [_vp, _ll, _vp, _vp, _i, _vp, _ll, _vp, _vp, _vp, _i, _vp, _ll, _ll, _ll, _vp, _i, _ll, _vp,
                                  _vp]
_lib.aweq_linear_w8a8.restype = _i
_lib.aweq_rope_table.argtypes = [ctypes.POINTER(RopeSpec), _ll, _vp, _vp]
_lib.aweq_rope_table.restype = _i
_lib.aweq_kv_append.argtypes = [ctypes.POINTER(KvCacheArgs), _vp, _ll, _ll, _ll, _vp, _ll, _vp, _ll, _vp, _vp, _ll, _ll, _vp,
                                _ll, _i, _i, _vp, _ll, _i, _vp, _ll, _vp, _vp]
_lib.aweq_kv_append.restype = _i
_lib.aweq_prefix_attention_workspace_bytes.argtypes = [ctypes.POINTER(KvCacheArgs), _ll, _ll, _ll, _i, _i]
_lib.aweq_prefix_attention_workspace_bytes.restype = _sz
_lib.aweq_prefix_attention.argtypes = [_vp, _ll, ctypes.POINTER(KvCacheArgs), _vp, _ll, _vp, _ll, _ll, _vp, _ll, _ll, _i, _i,
                                       ctypes.c_float, _vp, _ll, _vp, _sz, _vp, _vp]
_lib.aweq_prefix_attention.restype = _i
for _f in ("aweq_stats", "aweq_wrange", "aweq_factors", "aweq_equalize_quantize", "aweq_bias_correct",
           "aweq_quant_act", "aweq_layer_pass", "aweq_forward_check"):
    getattr(_lib, _f).restype = _i


class AweqError(RuntimeError):
    def __init__(self, code: int):
        self.code = code
        msg = _lib.aweq_strerror(code).decode()
        if code == 8:
            msg += ": " + _lib.aweq_last_cuda_error().decode()
        super().__init__("aweq status %d: %s" % (code, msg))


def _check(code: int) -> None:
    if code != OK:
        raise AweqError(code)


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("device tensors only (there is no CPU path)")
    return t.data_ptr()


def _stream() -> int:
    # the raw handle of the current stream (torch.cuda.current_stream() builds an object: 3 us a call)
    return _raw_stream(_current_device())


# (not a public name: a torch without it serves the slow way)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)
_current_device = torch.cuda.current_device


def dtype_tag(t: torch.Tensor) -> int:
    if t.dtype == torch.float16:
        return F16
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError("16-bit tensors must be float16 or bfloat16, got %s" % t.dtype)


def _ld(t: torch.Tensor) -> int:
    if t.dim() != 2 or t.stride(1) != 1:
        raise ValueError("matrices must be 2-D with a contiguous innermost dimension")
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def strerror(code: int) -> str:
    return _lib.aweq_strerror(code).decode()


def version() -> int:
    return int(_lib.aweq_version())


def launch_count() -> int:
    return int(_lib.aweq_launch_count())


def workspace_bytes(op: int, rows: int, cols: int, bits: int = 0, gran: int = 0, group: int = 0) -> int:
    return int(_lib.aweq_workspace_bytes(op, rows, cols, bits, gran, group))


def workspace(nbytes: int, device="cuda") -> torch.Tensor:
    """A 256-byte aligned scratch tensor of at least ``nbytes`` bytes."""
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def new_status(device="cuda") -> torch.Tensor:
    """A zeroed device status block (4 x uint64 viewed as int64)."""
    return torch.zeros(4, dtype=torch.int64, device=device)


def read_status(st: torch.Tensor) -> dict:
    """The three counters that the calibration calls write (``read_out_of_range`` has the fourth)."""
    v = st.cpu().tolist()
    return {"nonfinite": v[0], "zero_range": v[1], "wait_timeout": v[2]}


def read_out_of_range(st: torch.Tensor) -> int:
    """The fourth counter of a status block: positions, lengths, sequence or page numbers that
    pointed outside their table or pool (``aweq_kv_append``, ``aweq_prefix_attention``)."""
    return int(st[3])


def aweq_stats(X, xmin, xmax, xmean, xsum=None, count=None, accumulate=False, ws=None, st=None, N=None):
    n = X.shape[0] if N is None else N
    _check(_lib.aweq_stats(_ptr(X), dtype_tag(X), n, X.shape[1], _ld(X), _ptr(xmin), _ptr(xmax), _ptr(xmean),
                           _ptr(xsum), _ptr(count), int(accumulate), _ptr(ws), 0 if ws is None else ws.numel(),
                           _ptr(st), _stream()))


def aweq_stats_static(X, xmin, xmax, xmean, st=None):
    """Step 1 with the library's built-in scratch: for callers that cannot allocate
    device memory (no ``ws`` argument; C_in <= 16384).  Same results as aweq_stats."""
    _check(_lib.aweq_stats_static(_ptr(X), dtype_tag(X), X.shape[0], X.shape[1], _ld(X), _ptr(xmin), _ptr(xmax),
                                  _ptr(xmean), _ptr(st), _stream()))


def aweq_wrange(W, wmin, wmax, accumulate=False, ws=None, st=None):
    _check(_lib.aweq_wrange(_ptr(W), dtype_tag(W), W.shape[0], W.shape[1], _ld(W), _ptr(wmin), _ptr(wmax),
                            int(accumulate), _ptr(ws), 0 if ws is None else ws.numel(), _ptr(st), _stream()))


def aweq_factors(xmin, xmax, xmean, wmin, wmax, s, rinv, mu_hat, pX=None, pW=None, scalars=None, st=None):
    _check(_lib.aweq_factors(_ptr(xmin), _ptr(xmax), _ptr(xmean), _ptr(wmin), _ptr(wmax), xmin.numel(), _ptr(s),
                             _ptr(rinv), _ptr(mu_hat), _ptr(pX), _ptr(pW), _ptr(scalars), _ptr(st), _stream()))


def aweq_factors_absmax(xmin, xmax, xmean, wmin, wmax, s, rinv, mu_hat, pX=None, pW=None, scalars=None, st=None):
    _check(_lib.aweq_factors_absmax(_ptr(xmin), _ptr(xmax), _ptr(xmean), _ptr(wmin), _ptr(wmax), xmin.numel(), _ptr(s),
                                    _ptr(rinv), _ptr(mu_hat), _ptr(pX), _ptr(pW), _ptr(scalars), _ptr(st), _stream()))


def aweq_equalize_quantize(W, s, mu_hat, bits, gran, group, codes, step, zp, epsmu=None, ws=None, st=None):
    _check(_lib.aweq_equalize_quantize(_ptr(W), dtype_tag(W), W.shape[0], W.shape[1], _ld(W), _ptr(s), _ptr(mu_hat),
                                       bits, gran, group, _ptr(codes), _ptr(step), _ptr(zp), _ptr(epsmu), _ptr(ws),
                                       0 if ws is None else ws.numel(), _ptr(st), _stream()))


def aweq_bias_correct(epsmu, W, s, codes, step, zp, mu_hat, bits, gran, group, bias_in, bias_out, bias_out_f32,
                      bias_dt, C_out=None, st=None):
    if W is not None:
        c_out, c_in, ld, dt = W.shape[0], W.shape[1], _ld(W), dtype_tag(W)
    else:
        c_out, c_in, ld, dt = (epsmu.numel() if C_out is None else C_out), 8, 8, bias_dt
    _check(_lib.aweq_bias_correct(_ptr(epsmu), _ptr(W), dt, _ptr(s), _ptr(codes), _ptr(step), _ptr(zp), _ptr(mu_hat),
                                  c_out, c_in, ld, bits, gran, group, _ptr(bias_in), _ptr(bias_out),
                                  _ptr(bias_out_f32), bias_dt, _ptr(st), _stream()))


def aweq_quant_act(X, rinv, bits, gran, tensor_lo_hi, Xq, step, zp, st=None):
    _check(_lib.aweq_quant_act(_ptr(X), dtype_tag(X), X.shape[0], X.shape[1], _ld(X), _ptr(rinv), bits, gran,
                               _ptr(tensor_lo_hi), _ptr(Xq), _ptr(step), _ptr(zp), _ptr(st), _stream()))


def aweq_plan_query(op: int, rows: int, cols: int):
    """Launch geometry for an operation on a rows x cols matrix as a tuple of 8 integers
    (see ``include/aweq.h``); host logic only."""
    plan = (_ll * 8)()
    _check(_lib.aweq_plan_query(op, rows, cols, ctypes.byref(plan)))
    return tuple(plan)


def aweq_relabel_signed(codes, out=None, zp=None, zp_out=None):
    """8-bit codes q -> q - 128 (an ``int8`` view of the result is the signed code) and zero-points
    Z -> Z - 128; in place when ``out`` / ``zp_out`` are None."""
    out = codes if out is None else out
    if zp is not None and zp_out is None:
        zp_out = zp
    _check(_lib.aweq_relabel_signed(_ptr(codes), codes.numel(), _ptr(out), _ptr(zp), 0 if zp is None else zp.numel(),
                                    _ptr(zp_out), _stream()))
    return out, zp_out


def aweq_fold_scale(P, rinv, out=None):
    """Scale row r of a 16-bit matrix (or element r of a vector) by ``rinv[r]``; in place when
    ``out`` is None."""
    out = P if out is None else out
    if P.dim() == 1:
        rows, cols, ld, ld_out = P.shape[0], 1, P.stride(0), out.stride(0)
    else:
        rows, cols, ld, ld_out = P.shape[0], P.shape[1], _ld(P), _ld(out)
    _check(_lib.aweq_fold_scale(_ptr(P), dtype_tag(P), rows, cols, ld, _ptr(rinv), _ptr(out), ld_out, _stream()))
    return out


def forward_check_workspace_bytes(N: int, C_in: int, C_out: int) -> int:
    return int(_lib.aweq_forward_check_workspace_bytes(N, C_in, C_out))


def aweq_forward_check(Xq, act_step, act_zp, Wq, w_step, w_zp, bias_q, X, W, bias, mean_err, sums, ws=None):
    """Mean output error per output channel and sums of squares of the quantised layer
    against the 16-bit layer (argument marshalling only; see ``include/aweq.h``)."""
    N, C_in = X.shape
    C_out = W.shape[0]
    if not (X.is_contiguous() and W.is_contiguous() and Xq.is_contiguous() and Wq.is_contiguous()):
        raise ValueError("aweq_forward_check takes contiguous matrices")
    if ws is None:
        ws = workspace(forward_check_workspace_bytes(N, C_in, C_out), X.device)
    _check(_lib.aweq_forward_check(_ptr(Xq), _ptr(act_step), _ptr(act_zp), _ptr(Wq), _ptr(w_step), _ptr(w_zp),
                                   _ptr(bias_q), _ptr(X), _ptr(W), dtype_tag(X), _ptr(bias), N, C_in, C_out,
                                   _ptr(mean_err), _ptr(sums), _ptr(ws), ws.numel(), _stream()))
    return ws


def forward_check_weights_workspace_bytes(N: int, C_in: int, C_out: int) -> int:
    return int(_lib.aweq_forward_check_weights_workspace_bytes(N, C_in, C_out))


def aweq_forward_check_weights(codes, step, zp, bits, gran, group, rinv, bias_q, X, W, bias, mean_err, sums, ws=None):
    """Forward check of a weight-only layer (argument marshalling only; see ``include/aweq.h``)."""
    N, C_in = X.shape
    C_out = W.shape[0]
    if not (X.is_contiguous() and W.is_contiguous() and codes.is_contiguous()):
        raise ValueError("aweq_forward_check_weights takes contiguous matrices")
    if ws is None:
        ws = workspace(forward_check_weights_workspace_bytes(N, C_in, C_out), X.device)
    _check(_lib.aweq_forward_check_weights(_ptr(codes), _ptr(step), _ptr(zp), bits, gran, group, _ptr(rinv), _ptr(bias_q),
                                           _ptr(X), _ptr(W), dtype_tag(X), _ptr(bias), N, C_in, C_out, _ptr(mean_err),
                                           _ptr(sums), _ptr(ws), ws.numel(), _stream()))
    return ws


def _parr(tensors: Optional[Sequence[Optional[torch.Tensor]]], n: int):
    if tensors is None:
        return None
    arr = (_vp * n)()
    for i, t in enumerate(tensors):
        arr[i] = _ptr(t)
    return arr


class LayerPass:
    """Marshals the arguments of ``aweq_layer_pass`` once so that the call can be
    repeated cheaply; keeps the tensors alive."""

    def __init__(self, X, Ws, bits, gran, group, codes, step, zp, epsmu, bias_in, bias_out, bias_out_f32,
                 xmin, xmax, xmean, wmin, wmax, s, rinv, mu_hat, pX=None, pW=None, scalars=None,
                 Xq=None, act_step=None, act_zp=None, act_bits=8, flags=0, stat_negmin_max=None, stat_sum_count=None):
        n = len(Ws)
        self._keep = (X, Ws, codes, step, zp, epsmu, bias_in, bias_out, bias_out_f32, xmin, xmax, xmean, wmin, wmax,
                      s, rinv, mu_hat, pX, pW, scalars, Xq, act_step, act_zp, stat_negmin_max, stat_sum_count)
        a = LayerArgs()
        a.X, a.dt, a.N, a.C_in, a.ldx = _ptr(X), dtype_tag(X), X.shape[0], X.shape[1], _ld(X)
        a.n_w = n
        self._arrs = dict(
            W=_parr(Ws, n), C_out=(_ll * n)(*[w.shape[0] for w in Ws]), ldw=(_ll * n)(*[_ld(w) for w in Ws]),
            bias_in=_parr(bias_in, n), bias_out=_parr(bias_out, n), bias_out_f32=_parr(bias_out_f32, n),
            codes=_parr(codes, n), step=_parr(step, n), zp=_parr(zp, n), epsmu=_parr(epsmu, n))
        for k, v in self._arrs.items():
            if v is not None:
                setattr(a, k, v)
        a.bits, a.gran, a.group = bits, gran, group
        for k, v in dict(xmin=xmin, xmax=xmax, xmean=xmean, wmin=wmin, wmax=wmax, s=s, rinv=rinv, mu_hat=mu_hat,
                         pX=pX, pW=pW, scalars=scalars, Xq=Xq, act_step=act_step, act_zp=act_zp,
                         stat_negmin_max=stat_negmin_max, stat_sum_count=stat_sum_count).items():
            setattr(a, k, _ptr(v))
        a.act_bits, a.flags = act_bits, flags
        self.args = a
        self.ws_bytes = int(_lib.aweq_layer_pass_workspace_bytes(ctypes.byref(a)))
        # steps 1 and 2 in one launch (the hooks around step 1 then cover the weight ranges too)
        self.fused_ranges = bool(_lib.aweq_layer_pass_fuses_ranges(ctypes.byref(a)))
        self.weight_bytes = sum(w.numel() * w.element_size() for w in Ws)

    def set_events(self, stats=None, act=None) -> None:
        """Profiling hooks: pairs of recorded-once ``torch.cuda.Event(enable_timing=True)``
        (or None) that the library records around step 1 and step 6."""
        def h(e):
            return None if e is None else e.cuda_event
        self._events = (stats, act)
        self.args.ev_stats_begin, self.args.ev_stats_end = (h(stats[0]), h(stats[1])) if stats else (None, None)
        self.args.ev_act_begin, self.args.ev_act_end = (h(act[0]), h(act[1])) if act else (None, None)

    def __call__(self, ws: torch.Tensor, st: Optional[torch.Tensor] = None, phases: int = 0) -> None:
        """``phases``: 0 = the whole pass, or a mask of ``FLAG_PHASE_*`` (see ``include/aweq.h``)."""
        base = self.args.flags & ~(FLAG_PHASE_REDUCE | FLAG_PHASE_QUANT | FLAG_PHASE_ACT)
        self.args.flags = base | phases
        try:
            _check(_lib.aweq_layer_pass(ctypes.byref(self.args), _ptr(ws), ws.numel(), _ptr(st), _stream()))
        finally:
            self.args.flags = base


def aweq_layer_pass(lp: LayerPass, ws: torch.Tensor, st: Optional[torch.Tensor] = None) -> None:
    lp(ws, st)


# ---------------------------------------------------------------- running a calibrated layer
def _want(t: Optional[torch.Tensor], dtype, n: int, what: str) -> None:
    """The library cannot see a tensor's type or length: they are checked here."""
    if t is not None and (t.dtype != dtype or t.numel() < n or not t.is_contiguous()):
        raise ValueError("%s must be a contiguous %s tensor of at least %d elements" % (what, dtype, n))


def _pitch(t: torch.Tensor) -> int:
    """Row pitch of a matrix; one row has none of its own (its stride may be anything)."""
    _ld(t)
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _want_codes(t: torch.Tensor, what: str) -> None:
    if t.dtype != torch.uint8:
        raise TypeError("%s must be uint8 codes, got %s" % (what, t.dtype))


def aweq_code_sums(codes, sums=None):
    """Row sums of an 8-bit code matrix (int32)."""
    _want_codes(codes, "codes")
    if sums is None:
        sums = torch.empty(codes.shape[0], dtype=torch.int32, device=codes.device)
    _want(sums, torch.int32, codes.shape[0], "sums")
    _check(_lib.aweq_code_sums(_ptr(codes), codes.shape[0], codes.shape[1], _pitch(codes), _ptr(sums), _stream()))
    return sums


def aweq_linear_w8a8(Xq, act_step, act_zp, act_gran, Wq, w_step, w_zp, w_sum, w_gran, bias, out, st=None):
    """The calibrated W8A8 layer on step-6 codes (argument marshalling only; see ``include/aweq.h``).
    ``LinearW8A8`` marshals the weight's arguments once for repeated calls."""
    N, C_in = Xq.shape
    C_out = Wq.shape[0]
    _want_codes(Xq, "Xq")
    _want_codes(Wq, "Wq")
    if Wq.shape[1] != C_in or out.shape[0] != N or out.shape[1] != C_out:
        raise ValueError("shapes do not match: Xq %s, Wq %s, out %s" % (tuple(Xq.shape), tuple(Wq.shape), tuple(out.shape)))
    pairs, w_pairs = (N if act_gran == PER_ROW else 1), (C_out if w_gran == PER_ROW else 1)
    _want(act_step, torch.float32, pairs, "act_step")
    _want(act_zp, torch.int32, pairs, "act_zp")
    _want(w_step, torch.float32, w_pairs, "w_step")
    _want(w_zp, torch.int32, w_pairs, "w_zp")
    _want(w_sum, torch.int32, C_out, "w_sum")
    _want(bias, torch.float32, C_out, "bias")
    _check(_lib.aweq_linear_w8a8(_ptr(Xq), _pitch(Xq), _ptr(act_step), _ptr(act_zp), act_gran, _ptr(Wq), _pitch(Wq), _ptr(w_step),
                                 _ptr(w_zp), _ptr(w_sum), w_gran, _ptr(bias), N, C_in, C_out, _ptr(out), dtype_tag(out),
                                 _pitch(out), _ptr(st), _stream()))
    return out


class LinearW8A8:
    """A calibrated 8-bit linear layer ready to run: holds the step-4 codes (one pair per output channel,
    or a single pair), the corrected binary32 bias and the codes' row sums (formed here, once), and
    marshals them once.  Calling it with step-6 codes and their pairs (one per token, or a single
    pair) writes the 16-bit output on the current stream.

    The layer is what its arguments are now: it copies them, so that a calibration that runs again into the
    same tensors changes the next layer and not this one.  ``copy=False`` keeps the tensors themselves, for a
    caller that writes none of them as long as the layer lives (new codes would meet old row sums)."""

    def __init__(self, codes, step, zp, bias=None, copy=True):
        _want_codes(codes, "codes")
        ld = _pitch(codes)
        self.C_out, self.C_in = codes.shape
        gran = PER_TENSOR if step.numel() == 1 and self.C_out != 1 else PER_ROW
        pairs = self.C_out if gran == PER_ROW else 1
        _want(step, torch.float32, pairs, "step")
        _want(zp, torch.int32, pairs, "zp")
        _want(bias, torch.float32, self.C_out, "bias")
        if copy:
            ld = self.C_in
            codes, step, zp, bias = (None if t is None else t.clone(memory_format=torch.contiguous_format) for t in (codes, step, zp, bias))
        self.codes, self.step, self.zp, self.bias = codes, step, zp, bias
        self.w_sum = aweq_code_sums(codes)
        self._weight = (_ptr(codes), ld, _ptr(step), _ptr(zp), _ptr(self.w_sum), gran, _ptr(bias))

    def __call__(self, Xq, act_step, act_zp, out=None, dtype=torch.float16, st=None):
        n, c = Xq.shape
        if out is None:
            out = torch.empty((n, self.C_out), dtype=dtype, device=Xq.device)
        ldx, one = Xq.stride()
        ldo, out_one = out.stride()
        pairs = act_step.numel()
        # every check a few tenths of a microsecond: a decoding step calls this once per projection
        if (c != self.C_in or Xq.dtype is not torch.uint8 or one != 1 or out_one != 1 or out.shape != (n, self.C_out)
                or act_step.dtype is not torch.float32 or act_zp.dtype is not torch.int32 or act_zp.numel() != pairs
                or (pairs != n and pairs != 1) or not (act_step.is_contiguous() and act_zp.is_contiguous())
                or not (Xq.is_cuda and out.is_cuda and act_step.is_cuda and act_zp.is_cuda)):
            raise ValueError("device tensors: Xq [N x %d] uint8, act_step / act_zp float32 / int32 of N or one element, "
                             "out [N x %d], rows contiguous" % (self.C_in, self.C_out))
        if n == 1:                                                      # (see _pitch)
            ldx, ldo = c, self.C_out
        rc = _lib.aweq_linear_w8a8(Xq.data_ptr(), ldx, act_step.data_ptr(), act_zp.data_ptr(), PER_ROW if pairs == n else PER_TENSOR,
                                   *self._weight, n, c, self.C_out, out.data_ptr(), dtype_tag(out), ldo, _ptr(st), _stream())
        if rc:
            raise AweqError(rc)
        return out


def aweq_rope_table(rotary_dim, n_pos, theta=10000.0, scaling="none", factor=1.0, original_len=0.0, low=1.0, high=4.0,
                    attention=1.0, table=None, device="cuda"):
    """cos and sin of every position below ``n_pos``: float32 [n_pos x rotary_dim] for
    ``aweq_kv_append``.  ``scaling``: "none", "linear", "base" or "bands" (see ``include/aweq.h``)."""
    if scaling not in ROPE_SCALINGS:
        raise ValueError("scaling must be one of %s" % sorted(ROPE_SCALINGS))
    if table is None:
        table = torch.empty((n_pos, rotary_dim), dtype=torch.float32, device=device)
    _want(table, torch.float32, n_pos * rotary_dim, "table")
    spec = RopeSpec(rotary_dim, ROPE_SCALINGS[scaling], theta, factor, original_len, low, high, attention)
    _check(_lib.aweq_rope_table(ctypes.byref(spec), n_pos, _ptr(table), _stream()))
    return table


class KVCache:
    """A paged cache: two pools [n_pages, page_size, n_kv_heads, head_dim] with the same strides and a
    contiguous innermost dimension (a permuted view serves pools that keep tokens inside heads)."""

    def __init__(self, k, v):
        if k.dim() != 4 or k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype or k.stride(3) != 1:
            raise ValueError("k and v must be alike: [n_pages, page_size, n_kv_heads, head_dim], innermost contiguous")
        self.k, self.v = k, v
        self.n_pages, self.page_size, self.n_kv_heads, self.head_dim = k.shape
        self.dtype = k.dtype
        # a dimension of one element has no stride of its own
        stride = [self.head_dim if k.shape[i] == 1 else k.stride(i) for i in range(3)]
        self.args = KvCacheArgs(_ptr(k), _ptr(v), dtype_tag(k), self.page_size, self.n_kv_heads, self.head_dim, self.n_pages,
                                *stride)
        self.ref = ctypes.byref(self.args)


def _heads(t: torch.Tensor, n: int, n_heads: int, head_dim: int, dtype, what: str) -> int:
    """Row pitch of [n, heads, head_dim] (or [n, heads * head_dim]) on the device with contiguous rows."""
    stride = t.stride()
    if t.shape == (n, n_heads, head_dim):
        ok = stride[2] == 1 and (n_heads == 1 or stride[1] == head_dim)
    else:
        ok = t.shape == (n, n_heads * head_dim) and stride[1] == 1
    if not ok or t.dtype is not dtype or not t.is_cuda:
        raise ValueError("%s must be a %s device tensor [%d, %d, %d] with contiguous rows" % (what, dtype, n, n_heads, head_dim))
    return stride[0] if n > 1 else n_heads * head_dim


def _int32_rows(t: torch.Tensor, n: int, what: str) -> int:
    """Pointer of a contiguous int32 device tensor of n elements."""
    if t.dtype is not torch.int32 or t.numel() != n or not t.is_contiguous() or not t.is_cuda:
        raise ValueError("%s must be a contiguous int32 device tensor of %d elements" % (what, n))
    return t.data_ptr()


def _int32_table(t: torch.Tensor, what: str):
    """(pointer, rows, columns, pitch) of an int32 device matrix with contiguous rows."""
    if t.dtype is not torch.int32 or t.dim() != 2 or not t.is_cuda:
        raise ValueError("%s must be an int32 device matrix" % what)
    (rows, cols), (ld, one) = t.shape, t.stride()
    if cols > 1 and one != 1:
        raise ValueError("%s must have contiguous rows" % what)
    return t.data_ptr(), rows, cols, ld if rows > 1 else cols


def aweq_kv_append(cache, page_table, k, v, pos, seq=None, first=0, table=None, interleaved=False, q=None, q_out=None,
                   st=None):
    """Store keys and values of new tokens in their pages, keys (and ``q`` into ``q_out``) turned by
    their positions on the way (argument marshalling only; see ``include/aweq.h``).  Without ``q_out`` the
    queries are turned in place.  Returns where they are."""
    d, kv, dt, n = cache.head_dim, cache.n_kv_heads, cache.dtype, k.shape[0]
    ldk, ldv = _heads(k, n, kv, d, dt, "k"), _heads(v, n, kv, d, dt, "v")
    pages, n_seq, per_seq, ld_table = _int32_table(page_table, "page_table")
    if seq is None and n_seq < n:
        raise ValueError("without seq, page_table has a row per token")
    n_pos = rd = 0
    if table is not None:
        n_pos, rd = table.shape
        if table.dtype is not torch.float32 or not table.is_contiguous():
            raise ValueError("table must be contiguous float32 [positions, rotary_dim]")
    ldq = ldo = heads = 0
    if q is not None:
        heads = q.shape[1] if q.dim() == 3 else q.shape[1] // d
        q_out = q if q_out is None else q_out
        ldq, ldo = _heads(q, n, heads, d, dt, "q"), _heads(q_out, n, heads, d, dt, "q_out")
    rc = _lib.aweq_kv_append(cache.ref, pages, n_seq, per_seq, ld_table, k.data_ptr(), ldk, v.data_ptr(), ldv,
                             _int32_rows(pos, n, "pos"), None if seq is None else _int32_rows(seq, n, "seq"), first, n, _ptr(table),
                             n_pos, rd, 1 if interleaved else 0, _ptr(q), ldq, heads, _ptr(q_out), ldo, _ptr(st), _stream())
    if rc:
        raise AweqError(rc)
    return q_out


def aweq_prefix_attention_workspace_bytes(cache, prefix_len, max_own, n_seq, n_q, n_heads) -> int:
    return int(_lib.aweq_prefix_attention_workspace_bytes(cache.ref, prefix_len, max_own, n_seq, n_q, n_heads))


def aweq_prefix_attention(q, cache, prefix_pages, prefix_len, page_table, own_len, max_own, n_q, scale, out, ws, st=None):
    """Attention over a shared prefix and each sequence's own keys (argument marshalling only; see
    ``include/aweq.h``).  ``q``, ``out``: [n_seq * n_q, n_heads, head_dim]."""
    n_seq, d, dt = own_len.numel(), cache.head_dim, cache.dtype
    n_heads = q.shape[1] if q.dim() == 3 else q.shape[1] // d
    ldq, ldo = _heads(q, n_seq * n_q, n_heads, d, dt, "q"), _heads(out, n_seq * n_q, n_heads, d, dt, "out")
    pages, rows, per_seq, ld_table = _int32_table(page_table, "page_table")
    if rows != n_seq:
        raise ValueError("page_table has a row per sequence")
    if prefix_len:
        _want(prefix_pages, torch.int32, -(-prefix_len // cache.page_size), "prefix_pages")
    rc = _lib.aweq_prefix_attention(q.data_ptr(), ldq, cache.ref, _ptr(prefix_pages), prefix_len, pages, per_seq, ld_table,
                                    _int32_rows(own_len, n_seq, "own_len"), max_own, n_seq, n_q, n_heads, scale, out.data_ptr(), ldo,
                                    _ptr(ws), ws.numel(), _ptr(st), _stream())
    if rc:
        raise AweqError(rc)
    return out


class PrefixAttention:
    """``aweq_prefix_attention`` for one batch shape: holds the prefix's page list and the scratch.  One
    object serves one stream at a time (its calls share the scratch)."""

    def __init__(self, cache, prefix_pages, prefix_len, n_heads, n_seq, n_q=1, max_own=None, scale=None):
        self.cache, self.prefix_pages, self.prefix_len = cache, prefix_pages, int(prefix_len)
        self.n_heads, self.n_seq, self.n_q = n_heads, n_seq, n_q
        self.max_own = 0x7fffffff if max_own is None else int(max_own)
        self.scale = cache.head_dim ** -0.5 if scale is None else float(scale)
        if self.prefix_len:
            _want(prefix_pages, torch.int32, -(-self.prefix_len // cache.page_size), "prefix_pages")
        nbytes = aweq_prefix_attention_workspace_bytes(cache, self.prefix_len, self.max_own, n_seq, n_q, n_heads)
        self.ws = workspace(nbytes, cache.k.device)
        self._fixed = (cache.ref, _ptr(prefix_pages) if self.prefix_len else None, self.prefix_len)
        self._batch = (self.max_own, n_seq, n_q, n_heads, self.scale)
        self._scratch = (self.ws.data_ptr(), self.ws.numel())

    def __call__(self, q, page_table, own_len, out=None, st=None):
        out = torch.empty_like(q, memory_format=torch.contiguous_format) if out is None else out
        n, h, c = self.n_seq * self.n_q, self.n_heads, self.cache
        ldq, ldo = _heads(q, n, h, c.head_dim, c.dtype, "q"), _heads(out, n, h, c.head_dim, c.dtype, "out")
        pages, rows, per_seq, ld_table = _int32_table(page_table, "page_table")
        if rows != self.n_seq:
            raise ValueError("page_table has a row per sequence")
        rc = _lib.aweq_prefix_attention(q.data_ptr(), ldq, *self._fixed, pages, per_seq, ld_table,
                                        _int32_rows(own_len, self.n_seq, "own_len"), *self._batch, out.data_ptr(), ldo, *self._scratch,
                                        _ptr(st), _stream())
        if rc:
            raise AweqError(rc)
        return out
