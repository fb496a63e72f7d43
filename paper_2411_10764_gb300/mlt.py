"""Python binding of libmlt (ctypes): argument marshalling only.

Every step of screening runs in the CUDA library; this module only turns
torch tensors / numpy arrays into pointers and sizes, passes the current
CUDA stream, and raises MltError on a non-zero status.  There is no CPU
fallback: if libmlt.so cannot be built or loaded, the calls raise.
"""
from __future__ import annotations

import ctypes as C
import os
import re
import struct
import threading
from array import array

import numpy as np

from . import _build

MLT_MODEL_V, MLT_MODEL_P, MLT_MODEL_A = 0, 1, 2
STATUS = {0: "MLT_OK", -1: "MLT_EINVAL", -2: "MLT_ENOMODEL", -3: "MLT_ECUDA", -4: "MLT_ENOMEM",
          -5: "MLT_ETIMEOUT"}

NODE_DTYPE = np.dtype(
    [("feature", "<i4"), ("value", "<f4"), ("default_left", "u1"), ("pad", "u1", (3,))]
)
OP_DTYPE = np.dtype([("op", "<i4"), ("a", "<i4"), ("b", "<i4"), ("c", "<f4")])

MLT_F32, MLT_BF16, MLT_F16 = 0, 1, 2


class SampleRule(C.Structure):
    """mlt_sample_rule"""
    _fields_ = [("temperature", C.c_float), ("top_k", C.c_int32), ("top_p", C.c_float), ("min_p", C.c_float)]


class ScanArgs(C.Structure):
    """mlt_scan_args"""
    _fields_ = ([(k, C.c_int32) for k in ("dtype", "batch", "dim", "states", "groups", "taps")]
                + [("length", C.c_int64)]
                + [(k, C.c_void_p) for k in ("x", "dt", "z", "B", "C")]
                + [(f"{k}_{s}", C.c_int64) for k in ("x", "dt", "z", "B", "C") for s in ("batch", "step")]
                + [(k, C.c_void_p) for k in ("A", "skip", "dt_bias", "conv_w", "conv_b", "lengths", "state",
                                             "conv_state", "y")]
                + [("y_batch", C.c_int64), ("y_step", C.c_int64), ("state_out", C.c_void_p),
                   ("conv_state_out", C.c_void_p)])


class ScanGrads(C.Structure):
    """mlt_scan_grads"""
    _fields_ = ([("gy", C.c_void_p), ("gy_batch", C.c_int64), ("gy_step", C.c_int64)]
                + [(k, C.c_void_p) for k in ("g_state_out", "x", "dt", "z", "B", "C", "A", "skip", "dt_bias", "conv_w",
                                             "conv_b", "state", "conv_state")])



class NormArgs(C.Structure):
    """mlt_norm_args"""
    _fields_ = ([(k, C.c_int32) for k in ("dtype", "y_dtype", "w_dtype", "dim")] + [("rows", C.c_int64)]
                + [(k, C.c_void_p) for k in ("x", "residual", "weight", "bias")]
                + [("x_stride", C.c_int64), ("residual_stride", C.c_int64), ("y", C.c_void_p), ("total", C.c_void_p),
                   ("y_stride", C.c_int64), ("total_stride", C.c_int64), ("stats", C.c_void_p), ("eps", C.c_float)])


class NormGrads(C.Structure):
    """mlt_norm_grads"""
    _fields_ = [("gy", C.c_void_p), ("g_total", C.c_void_p), ("gy_stride", C.c_int64), ("g_total_stride", C.c_int64),
                ("gx", C.c_void_p), ("gx_stride", C.c_int64), ("gweight", C.c_void_p), ("gbias", C.c_void_p)]


class AdamWRule(C.Structure):
    """mlt_adamw_rule"""
    _fields_ = ([(k, C.c_double) for k in ("beta1", "beta2", "eps")] + [("step", C.c_int64)]
                + [(k, C.c_void_p) for k in ("step_device", "lr", "grad_scale")]
                + [("bits", C.c_int32), ("seed", C.c_uint32)])


class BeamArgs(C.Structure):
    """mlt_beam_args"""
    _fields_ = ([(k, C.c_int32) for k in ("dtype", "batch", "beams", "n", "m", "normalised")]
                + [("eos", C.c_int64), ("scores", C.c_void_p), ("batch_stride", C.c_int64), ("beam_stride", C.c_int64)]
                + [(k, C.c_void_p) for k in ("logp", "done", "out_parent", "out_token", "out_logp", "out_done")])


class BeamState(C.Structure):
    """mlt_beam_state"""
    _fields_ = [("data", C.c_void_p), ("row_bytes", C.c_int64), ("row_stride", C.c_int64)]


HEADER = os.path.join(_build.ROOT, "include", "mlt.h")


class MltError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"{STATUS.get(code, code)}: {message}")
        self.code = code


_lib = None
_lock = threading.Lock()


def library_path() -> str:
    return _build.LIB_PATH


def lib(build_if_missing: bool = True):
    """Load libmlt.so (building it first when missing or stale)."""
    global _lib
    with _lock:
        if _lib is not None:
            return _lib
        if build_if_missing:
            _build.build()
        if not os.path.exists(_build.LIB_PATH):
            raise RuntimeError(f"libmlt.so missing at {_build.LIB_PATH}")
        L = C.CDLL(_build.LIB_PATH)
        P, i32, i64, f32 = C.c_void_p, C.c_int, C.c_int64, C.c_float
        sig = {
            "mlt_set_num_features": [i32],
            "mlt_load_ensemble": [i32, P, i32, i32],
            "mlt_load_ensemble_f16": [i32, P, i32, i32],
            "mlt_screen_host_batches": [P, i64, P, i64, f32, i32, P, P, P],
            "mlt_selftest_wait_timeout": [P, i64],
            "mlt_selftest_walk_timeout": [i32, i64],
            "mlt_selftest_ordinal_timeout": [i64],
            "mlt_selftest_sample_timeout": [i64],
            "mlt_selftest_poison_state": [i32, C.c_uint32],
            "mlt_free_ensemble": [i32],
            "mlt_validity_cut": [f32, P],
            "mlt_screen": [P, P, i64, f32, i32, P, P, P],
            "mlt_screen_host": [P, P, i64, f32, i32, P, P, P],
            "mlt_decode_knobs": [P, P, P, i32, P, i32, i64, i64, P, P],
            "mlt_screen_decoded": [P, P, P, i32, P, i64, i64, f32, i32, P, P, P],
            "mlt_sync_status": [P],
            "mlt_last_survivor_count": [P, P],
            "mlt_profile_phases": [i32],
            "mlt_phase_times": [P, i32, P],
            "mlt_tune_walk": [i32, i32, i32, i32, i32, i32],
            "mlt_walk_shape": [i32, i64, i32, P],
            "mlt_ordinal_shape": [i32, i64, i32, P],
            "mlt_tune_head_levels": [i32],
            "mlt_tune_fused_small": [i32],
            "mlt_tune_decode_jit": [i64],
            "mlt_tune_ordinal": [i32],
            "mlt_decode_jit_available": [],
            "mlt_walk_peak": [P, i32, P, i64, i32, P, P],
            "mlt_screen_noalloc": [P, P, i64, f32, i32, P, P, P],
            "mlt_rerank": [P, P, i64, P, i32, i32, P, P],
            "mlt_merge_topk": [P, P, P, i64, i32, P],
            "mlt_screen_until": [P, P, i64, i64, i64, f32, i32, P, P, P, P],
            "mlt_screen_until_decoded": [P, P, P, i32, P, i64, i64, i64, i64, f32, i32, P, P, P, P],
            "mlt_sample": [P, P, i32, i64, i64, i64, P, i64, P, P, i32, P, C.c_size_t, P, P],
            "mlt_sample_workspace": [i32, i64, i64, i32, P],
            "mlt_embed": [P, P, i32, i64, i32, i64, P, i32, i64, f32, P, i32, i64],
            "mlt_embed_grad": [P, P, i32, i64, P, i32, i64, i64, i32, f32, P, C.c_size_t, P, i32, i64],
            "mlt_embed_grad_workspace": [i64, i64, i32, P],
            "mlt_scan": [P, P, P, C.c_size_t],
            "mlt_scan_workspace": [P, P],
            "mlt_scan_grad": [P, P, P, P, C.c_size_t],
            "mlt_scan_grad_workspace": [P, P],
            "mlt_layer_norm": [P, P],
            "mlt_layer_norm_grad": [P, P, P, P, C.c_size_t],
            "mlt_layer_norm_grad_workspace": [i64, i32, P],
            "mlt_adamw": [P, P, i32, P, P, P, P, P],
            "mlt_adamw_blocks": [P, i32, P],
            "mlt_beam_step": [P, P, P, C.c_size_t],
            "mlt_beam_step_workspace": [P, P],
            "mlt_beam_reorder": [P, P, i32, i32, P, i32],
            "mlt_sa_step": [P, P, P, i32, P, P, P, P, P, P, i64, f32, f32, P, P, P],
        }
        for name, args in sig.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = i32
        L.mlt_kernel_launches.argtypes = []
        L.mlt_kernel_launches.restype = i64
        L.mlt_decode_jit_calls.argtypes = []
        L.mlt_decode_jit_calls.restype = i64
        L.mlt_last_error.argtypes = []
        L.mlt_last_error.restype = C.c_char_p
        _lib = L
        return L


def declared_symbols() -> list[str]:
    """Every function the C header declares."""
    text = open(HEADER).read()
    return sorted(set(re.findall(r"^\s*(?:const\s+)?\w+\s*\*?\s*(mlt_\w+)\s*\(", text, re.M)))


def _check(rc: int):
    if rc != 0:
        msg = lib().mlt_last_error()
        raise MltError(rc, msg.decode() if msg else "")


def _stream_ptr(stream=None):
    import torch

    s = torch.cuda.current_stream() if stream is None else stream
    return C.c_void_p(s.cuda_stream)


def _dptr(t):
    return C.c_void_p(0 if t is None else t.data_ptr())


# ---------------------------------------------------------------------------
# Model management
# ---------------------------------------------------------------------------

def set_num_features(F: int) -> None:
    _check(lib().mlt_set_num_features(int(F)))


def load_ensemble(model_id: int, nodes: np.ndarray, n_trees: int, depth: int) -> None:
    nodes = np.ascontiguousarray(nodes)
    if nodes.dtype.itemsize != 12:
        raise ValueError("nodes must use the 12-byte slot layout")
    if nodes.size != n_trees * ((2 << depth) - 1):
        raise ValueError("node array size does not match n_trees and depth")
    _check(lib().mlt_load_ensemble(int(model_id), nodes.ctypes.data, int(n_trees), int(depth)))


def load_ensemble_f16(model_id: int, nodes: np.ndarray, n_trees: int, depth: int) -> None:
    """Load model V or P as half tables (binary16 thresholds, leaves and
    staged features: changes results, see mlt_load_ensemble_f16)."""
    nodes = np.ascontiguousarray(nodes)
    if nodes.dtype.itemsize != 12:
        raise ValueError("nodes must use the 12-byte slot layout")
    if nodes.size != n_trees * ((2 << depth) - 1):
        raise ValueError("node array size does not match n_trees and depth")
    _check(lib().mlt_load_ensemble_f16(int(model_id), nodes.ctypes.data, int(n_trees), int(depth)))


def free_ensemble(model_id: int) -> None:
    _check(lib().mlt_free_ensemble(int(model_id)))


def validity_cut(thr: float) -> float:
    out = C.c_float()
    _check(lib().mlt_validity_cut(C.c_float(thr), C.byref(out)))
    return out.value


# ---------------------------------------------------------------------------
# Screening
# ---------------------------------------------------------------------------

def _outputs(n, k, device, out_pvalid, out_perf, out_topk):
    import torch

    if out_pvalid is None:
        out_pvalid = torch.empty(n, dtype=torch.float32, device=device)
    if out_perf is None:
        out_perf = torch.empty(n, dtype=torch.float32, device=device)
    if out_topk is None:
        out_topk = torch.empty(k, dtype=torch.int64, device=device)
    return out_pvalid, out_perf, out_topk


def screen(feats, thr: float, k: int, out_pvalid=None, out_perf=None, out_topk=None, stream=None):
    """Screen a [n][F] fp32 CUDA tensor: returns (pvalid, perf, topk) tensors."""
    import torch

    if not (isinstance(feats, torch.Tensor) and feats.is_cuda and feats.dtype == torch.float32):
        raise TypeError("feats must be a float32 CUDA tensor")
    if not feats.is_contiguous() or feats.dim() != 2:
        raise ValueError("feats must be a contiguous [n][F] tensor")
    n = feats.shape[0]
    pv, pf, tk = _outputs(n, k, feats.device, out_pvalid, out_perf, out_topk)
    _check(lib().mlt_screen(_stream_ptr(stream), _dptr(feats), n, C.c_float(thr), int(k),
                            _dptr(pv), _dptr(pf), _dptr(tk)))
    return pv, pf, tk


def screen_noalloc(feats, thr: float, k: int, out_pvalid=None, out_perf=None, out_topk=None,
                   stream=None):
    """mlt_screen_noalloc: like screen(), with the library's fixed scratch
    (n <= 262,144; overlapping calls race)."""
    import torch

    if not (isinstance(feats, torch.Tensor) and feats.is_cuda and feats.dtype == torch.float32):
        raise TypeError("feats must be a float32 CUDA tensor")
    n = feats.shape[0]
    pv, pf, tk = _outputs(n, k, feats.device, out_pvalid, out_perf, out_topk)
    _check(lib().mlt_screen_noalloc(_stream_ptr(stream), _dptr(feats), n, C.c_float(thr), int(k),
                                    _dptr(pv), _dptr(pf), _dptr(tk)))
    return pv, pf, tk


def screen_until(feats, batch: int, target: int, thr: float, k: int, with_outputs=True, stream=None):
    """Batched accumulation over the rows of `feats`: returns (pvalid, perf,
    topk, stats) with stats = [consumed, kept, batches] (CUDA tensors)."""
    import torch

    n = feats.shape[0]
    pv = torch.empty(n, dtype=torch.float32, device=feats.device) if with_outputs else None
    pf = torch.empty(n, dtype=torch.float32, device=feats.device) if with_outputs else None
    tk = torch.empty(int(k), dtype=torch.int64, device=feats.device)
    stats = torch.empty(3, dtype=torch.int64, device=feats.device)
    _check(lib().mlt_screen_until(_stream_ptr(stream), _dptr(feats), n, int(batch), int(target), C.c_float(thr),
                                  int(k), _dptr(pv), _dptr(pf), _dptr(tk), _dptr(stats)))
    return pv, pf, tk, stats


def screen_until_decoded(radices, option_values, program, first_index: int, n_total: int, batch: int,
                         target: int, thr: float, k: int, device="cuda", with_outputs=True, stream=None):
    """Batched accumulation over a decoded knob space."""
    import torch

    r, ov, prog = _decoder_args(radices, option_values, program)
    pv = torch.empty(n_total, dtype=torch.float32, device=device) if with_outputs else None
    pf = torch.empty(n_total, dtype=torch.float32, device=device) if with_outputs else None
    tk = torch.empty(int(k), dtype=torch.int64, device=device)
    stats = torch.empty(3, dtype=torch.int64, device=device)
    _check(lib().mlt_screen_until_decoded(_stream_ptr(stream), r.ctypes.data, ov.ctypes.data, r.size,
                                          prog.ctypes.data, int(first_index), int(n_total), int(batch),
                                          int(target), C.c_float(thr), int(k), _dptr(pv), _dptr(pf),
                                          _dptr(tk), _dptr(stats)))
    return pv, pf, tk, stats


def sa_step(radices, option_values, program, parent, parent_score, knob_draw, digit_draw, log_u,
            temperature: float, thr: float, stream=None):
    """One explorer proposal step over the chains in `parent` (CUDA tensors:
    int64, float32, uint32-as-int32, int32, float32): returns (next,
    next_score, accepted) CUDA tensors."""
    import torch

    r, ov, prog = _decoder_args(radices, option_values, program)
    m = parent.numel()
    nxt = torch.empty(m, dtype=torch.int64, device=parent.device)
    nsc = torch.empty(m, dtype=torch.float32, device=parent.device)
    acc = torch.empty(m, dtype=torch.int32, device=parent.device)
    _check(lib().mlt_sa_step(_stream_ptr(stream), r.ctypes.data, ov.ctypes.data, r.size, prog.ctypes.data,
                             _dptr(parent), _dptr(parent_score), _dptr(knob_draw), _dptr(digit_draw), _dptr(log_u),
                             m, C.c_float(temperature), C.c_float(thr), _dptr(nxt), _dptr(nsc), _dptr(acc)))
    return nxt, nsc, acc


def rerank(feats, cand, n_final: int, out_score=None, out_final=None, stream=None):
    """Model A's rerank of candidate indices `cand` (CUDA int64 tensor) whose
    rows are in `feats`: returns (scores [m], final [n_final])."""
    import torch

    if not (isinstance(cand, torch.Tensor) and cand.is_cuda and cand.dtype == torch.int64):
        raise TypeError("cand must be an int64 CUDA tensor")
    m = cand.numel()
    if out_score is None:
        out_score = torch.empty(m, dtype=torch.float32, device=cand.device)
    if out_final is None:
        out_final = torch.empty(int(n_final), dtype=torch.int64, device=cand.device)
    _check(lib().mlt_rerank(_stream_ptr(stream), _dptr(feats), feats.shape[0], _dptr(cand), m, int(n_final),
                            _dptr(out_score), _dptr(out_final)))
    return out_score, out_final


def merge_topk(scores, indices, k: int, out=None, stream=None):
    """mlt_merge_topk: the k best (score, global index) pairs (CUDA fp32 and
    int64 tensors of equal length; a negative index is an empty slot) by
    (score desc, index asc), -1 padded: returns a CUDA int64 tensor [k]."""
    import torch

    for t, dt in ((scores, torch.float32), (indices, torch.int64)):
        if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dt and t.is_contiguous()):
            raise TypeError("scores / indices must be contiguous float32 / int64 CUDA tensors")
    m = indices.numel()
    if scores.numel() != m:
        raise ValueError("scores and indices differ in length")
    if out is None:
        out = torch.empty(int(k), dtype=torch.int64, device=indices.device)
    _check(lib().mlt_merge_topk(_stream_ptr(stream), _dptr(scores), _dptr(indices), m, int(k), _dptr(out)))
    return out


# ---------------------------------------------------------------------------
# Sequence-model operators
# ---------------------------------------------------------------------------

# These calls are short: a small draw or lookup takes the GPU about 5 us, so the checks
# here go by attributes that cost next to nothing.

_torch = None
_DTYPES: dict = {}
_raw_stream = None
_current_device = None


def _setup():
    """The library and, once, what the calls below need of torch."""
    global _torch, _raw_stream, _current_device
    if _torch is None:
        import torch

        _DTYPES.update({torch.float32: MLT_F32, torch.bfloat16: MLT_BF16, torch.float16: MLT_F16})
        # the handle of the current stream without building a Stream object
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda device: torch.cuda.current_stream(device).cuda_stream)
        _current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
        _torch = torch
    return _lib or lib()


def _stream_of(t):
    return _raw_stream(t.get_device())


def _on(stream, call, *args):
    """call(*args) with `stream` as the current one.  Workspace, copies and new outputs are then
    of that stream's memory, which no work still queued elsewhere uses; and the
    tensors given are kept until its work is done."""
    with _torch.cuda.stream(stream):
        for t in args:
            for one in t if isinstance(t, (tuple, list)) else (t,):
                if isinstance(one, _torch.Tensor) and one.is_cuda:
                    one.record_stream(stream)
        return call(*args)


def _dtype_code(t) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"float32, bfloat16 or float16 wanted, got {t.dtype}")
    return code


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


# ctypes passes the low 32 bits of larger numbers; the library refuses those it does see
_INT_MAX = 0x7FFFFFFF


def _cuda(t, name: str, dtype=None):
    if not (isinstance(t, _torch.Tensor) and t.is_cuda and (dtype is None or t.dtype == dtype)):
        raise TypeError(f"{name} must be a CUDA tensor" + (f" of {dtype}" if dtype is not None else ""))
    return t


def _rows(t, name: str) -> int:
    """Elements between the rows of a matrix whose columns are adjacent."""
    if t.dim() != 2:
        raise ValueError(f"{name} must have two dimensions")
    stride, column = t.stride()
    if column != 1 and t.shape[1] > 1:
        raise ValueError(f"{name} must have adjacent columns")
    return stride


def _like(t):
    """A contiguous tensor of t's shape and type (half the time of new_empty)."""
    return _torch.empty_like(t, memory_format=_torch.contiguous_format)


_ws_bytes: dict = {}


def _workspace(key, query, device):
    """Device memory for one call (torch's allocator reuses it in the order of
    the current stream); the sizes that the library asks for are
    remembered by the call's sizes."""
    n = _ws_bytes.get(key)
    if n is None:
        out = C.c_size_t()
        _check(query(out))
        if len(_ws_bytes) > 4096:
            _ws_bytes.clear()
        n = _ws_bytes[key] = out.value
    if n == 0:
        return None, 0
    return _torch.empty(n, dtype=_torch.uint8, device=device), n


def sample_rules(temperature, top_k=0, top_p=1.0, min_p=0.0, rows: int | None = None, device="cuda"):
    """mlt_sample_rule records for mlt.sample's `rules`: an int32 CUDA tensor
    [rows][4].  Each argument is a number or one value a row."""
    import torch

    top_k = torch.as_tensor(top_k, dtype=torch.int64, device=device).clamp(-1, _INT_MAX)
    cols = [torch.as_tensor(v, dtype=dt, device=device) for v, dt in
            ((temperature, torch.float32), (top_k, torch.int32), (top_p, torch.float32), (min_p, torch.float32))]
    if rows is None:
        rows = max([c.numel() for c in cols if c.dim() > 0], default=1)
    cols = [c.expand(rows).contiguous().view(torch.int32) for c in cols]
    return torch.stack(cols, 1).contiguous()


def sample(scores, noise, temperature: float = 1.0, top_k: int = 0, top_p: float = 1.0, min_p: float = 0.0,
           m: int = 1, rules=None, out=None, stream=None):
    """mlt_sample: m different entries of every row of `scores` ([rows][n], or
    [n] for one row) drawn with the given noise (fp32, same shape; Gumbel
    numbers -ln(-ln u)).  `rules` (sample_rules) gives every row its own
    cuts instead of the four numbers.  Returns (index [rows][m] int64, -1
    past the last kept entry, logprob [rows][m] fp32)."""
    L = _setup()
    if stream is not None:
        return _on(stream, sample, scores, noise, temperature, top_k, top_p, min_p, m, rules, out)
    torch = _torch
    _cuda(scores, "scores")
    _cuda(noise, "noise", torch.float32)
    code = _dtype_code(scores)
    one = scores.dim() == 1
    if one:
        scores, noise = scores[None], noise[None] if noise.dim() == 1 else noise
    if noise.shape != scores.shape:
        raise ValueError("scores and noise differ in shape")
    stride, noise_stride = _rows(scores, "scores"), _rows(noise, "noise")
    rows, n = scores.shape
    m = int(m)
    _need(m <= _INT_MAX, "m must lie in [1, 2048]")
    rule = each = None
    if rules is None:
        if not 0 <= top_k <= _INT_MAX:
            top_k = 0  # all
        rule = C.byref(SampleRule(temperature, top_k, top_p, min_p))
    else:
        _cuda(rules, "rules", torch.int32)
        if rules.shape != (rows, 4) or not rules.is_contiguous():
            raise ValueError("rules must be a contiguous int32 tensor [rows][4]")
        each = rules.data_ptr()
    device = scores.device
    if out is None:
        index = torch.empty(rows, m, dtype=torch.int64, device=device)
        logprob = torch.empty(rows, m, dtype=torch.float32, device=device)
    else:
        index, logprob = out
        for t, dt in ((index, torch.int64), (logprob, torch.float32)):
            _cuda(t, "out", dt)
            _need(t.is_contiguous() and t.numel() == rows * m, "out must be contiguous [rows][m] tensors")
    ws, n_ws = _workspace(("sample", code, rows, n, m),
                          lambda b: L.mlt_sample_workspace(code, rows, n, m, C.byref(b)), device)
    rc = L.mlt_sample(_stream_of(scores), scores.data_ptr(), code, rows, n, stride, noise.data_ptr(),
                      noise_stride, rule, each, m, None if ws is None else ws.data_ptr(), n_ws, index.data_ptr(),
                      logprob.data_ptr())
    if rc:
        _check(rc)
    return (index[0], logprob[0]) if one and out is None else (index, logprob)


def _ids(ids):
    _cuda(ids, "ids")
    dtype = ids.dtype
    if dtype != _torch.int64 and dtype != _torch.int32:
        raise TypeError("ids must be int32 or int64")
    if not ids.is_contiguous():
        raise ValueError("ids must be contiguous")
    return 1 if dtype == _torch.int64 else 0


def embed(ids, table, scale: float = 1.0, out_dtype=None, out=None, stream=None):
    """mlt_embed: scale * table[ids], rounded once to `out_dtype` (default: the
    table's); ids of any shape, negative ones give zeros."""
    L = _setup()
    if stream is not None:
        return _on(stream, embed, ids, table, scale, out_dtype, out)
    ids_64 = _ids(ids)
    _cuda(table, "table")
    code, stride = _dtype_code(table), _rows(table, "table")
    vocab, dim = table.shape
    _need(dim <= _INT_MAX, "dim must lie in [1, 2^20]")
    if out is None:
        out = _torch.empty(*ids.shape, dim, dtype=out_dtype or table.dtype, device=table.device)
        out_stride = dim
    else:
        _cuda(out, "out")
        _need(tuple(out.shape) == (*ids.shape, dim), "out must have the shape of ids and one more dimension, dim")
        flat = out if out.dim() == 2 else out.view(-1, dim)
        out_stride = _rows(flat, "out")
    rc = L.mlt_embed(_stream_of(table), table.data_ptr(), code, vocab, dim, stride, ids.data_ptr(), ids_64,
                     ids.numel(), scale, out.data_ptr(), _dtype_code(out), out_stride)
    if rc:
        _check(rc)
    return out


def embed_grad(ids, grad_out, vocab: int, scale: float = 1.0, out_dtype=None, out=None, stream=None):
    """mlt_embed_grad: the gradient [vocab][dim] of embed's table from that of
    its output; the same from call to call."""
    L = _setup()
    if stream is not None:
        return _on(stream, embed_grad, ids, grad_out, vocab, scale, out_dtype, out)
    ids_64 = _ids(ids)
    _cuda(grad_out, "grad_out")
    dim = grad_out.shape[-1]
    _need(tuple(grad_out.shape[:-1]) == tuple(ids.shape), "grad_out must have the shape of ids and one more dimension")
    flat = grad_out if grad_out.dim() == 2 else grad_out.reshape(-1, dim)
    code, stride = _dtype_code(flat), _rows(flat, "grad_out")
    vocab, tokens = int(vocab), ids.numel()
    _need(dim <= _INT_MAX, "dim must lie in [1, 2^20]")
    if out is None:
        out = _torch.empty(vocab, dim, dtype=out_dtype or grad_out.dtype, device=grad_out.device)
    else:
        _cuda(out, "out")
        _need(tuple(out.shape) == (vocab, dim), "out must be [vocab][dim]")
    ws, n_ws = _workspace(("embed_grad", tokens, vocab, dim),
                          lambda b: L.mlt_embed_grad_workspace(tokens, vocab, dim, C.byref(b)), out.device)
    _check(L.mlt_embed_grad(_stream_of(out), flat.data_ptr(), code, stride, ids.data_ptr(), ids_64, tokens, vocab,
                            dim, scale, None if ws is None else ws.data_ptr(), n_ws, out.data_ptr(), _dtype_code(out),
                            _rows(out, "out")))
    return out


def _wide(t, name, dtype, shape):
    """(address, batch stride, step stride) of a [batch][length]... input."""
    if t is None:
        return None, 0, 0
    if not t.is_cuda or t.dtype != dtype:
        raise TypeError(f"{name} must be a CUDA tensor of x's type")
    if t.shape != shape:
        raise ValueError(f"{name} must have the shape {shape}")
    s = t.stride()
    if s[-1] != 1 and shape[-1] > 1 and t.numel() > 0:
        raise ValueError(f"the channels of {name} must be adjacent")
    return t.data_ptr(), s[0], s[1]


def _plain(t, name, dtype, shape):
    """Address of a contiguous input, or None."""
    if t is None:
        return None
    if not t.is_cuda or t.dtype != dtype:
        raise TypeError(f"{name} must be a CUDA tensor of {dtype}")
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous, of the shape {shape}")
    return t.data_ptr()


def _scan_args(x, dt, B, Cm, A, z, skip, dt_bias, conv_w, conv_b, lengths, state, conv_state):
    _cuda(x, "x")
    dtype, f32 = x.dtype, _torch.float32
    if x.dim() != 3:
        raise ValueError("x must be [batch][length][dim]")
    b, L, d = x.shape
    if B.dim() == 3:
        B = B.unsqueeze(2)
    if Cm.dim() == 3:
        Cm = Cm.unsqueeze(2)
    if B.dim() != 4:
        raise ValueError("B must be [batch][length][groups][states]")
    g, n = B.shape[2:]
    taps = 0 if conv_w is None else conv_w.shape[1]
    _need(b <= _INT_MAX and d <= _INT_MAX, "batch must lie in [0, 65535], dim in [1, 2^20]")
    wide, narrow = (b, L, d), (b, L, g, n)
    xp, xb, xs = _wide(x, "x", dtype, wide)
    dp, db, ds = _wide(dt, "dt", dtype, wide)
    zp, zb, zs = _wide(z, "z", dtype, wide)
    Bp, Bb, Bs = _wide(B, "B", dtype, narrow)
    Cp, Cb, Cs = _wide(Cm, "C", dtype, narrow)
    if g > 1 and B.numel() > 0 and (B.stride(2) != n or Cm.stride(2) != n):
        raise ValueError("the groups of B and C must be adjacent")
    return ScanArgs(_dtype_code(x), b, d, n, g, taps, L, xp, dp, zp, Bp, Cp, xb, xs, db, ds, zb, zs, Bb, Bs, Cb, Cs,
                    _plain(A, "A", f32, (d, n)), _plain(skip, "skip", f32, (d,)),
                    _plain(dt_bias, "dt_bias", f32, (d,)), _plain(conv_w, "conv_w", f32, (d, taps)),
                    _plain(conv_b, "conv_b", f32, (d,)), _plain(lengths, "lengths", _torch.int32, (b,)),
                    _plain(state, "state", f32, (b, d, n)),
                    _plain(conv_state, "conv_state", dtype, (b, max(0, taps - 1), d)))


def scan(x, dt, B, C_, A, z=None, skip=None, dt_bias=None, conv_w=None, conv_b=None, lengths=None, state=None,
         conv_state=None, out=None, state_out=None, conv_state_out=None, stream=None):
    """mlt_scan: selective scan with its short causal convolution.  x, dt, z
    [batch][length][dim]; B, C_ [batch][length][groups][states] (or without
    the groups dimension); the rest fp32 (see mlt_scan in include/mlt.h).
    Returns (y, state, conv_state), the last None with fewer than two taps.
    For single tokens (length 1) pass state_out=state and
    conv_state_out=conv_state to update them in place."""
    lb = _setup()
    if stream is not None:
        return _on(stream, scan, x, dt, B, C_, A, z, skip, dt_bias, conv_w, conv_b, lengths, state, conv_state, out,
                   state_out, conv_state_out)
    torch = _torch
    a = _scan_args(x, dt, B, C_, A, z, skip, dt_bias, conv_w, conv_b, lengths, state, conv_state)
    b, L, d = x.shape
    y = _like(x) if out is None else out
    if out is not None:
        _need(tuple(y.shape) == (b, L, d) and y.dtype == x.dtype and y.is_cuda and (d == 1 or y.stride(2) == 1),
              "out must be like x, its channels adjacent")
    n, taps = a.states, a.taps
    if state_out is None:
        state_out = _like(state) if state is not None else torch.empty(b, d, n, dtype=torch.float32, device=x.device)
        a.state_out = state_out.data_ptr()
    else:
        a.state_out = _plain(state_out, "state_out", torch.float32, (b, d, n))
    if taps < 2:
        conv_state_out = None
    else:
        if conv_state_out is None:
            conv_state_out = (_like(conv_state) if conv_state is not None
                              else torch.empty(b, taps - 1, d, dtype=x.dtype, device=x.device))
        a.conv_state_out = _plain(conv_state_out, "conv_state_out", x.dtype, (b, taps - 1, d))
    a.y = y.data_ptr()
    a.y_batch, a.y_step, _ = y.stride()
    ws, n_ws = _workspace(("scan", b, L, d, n, a.groups), lambda q: lb.mlt_scan_workspace(C.byref(a), C.byref(q)),
                          x.device)
    rc = lb.mlt_scan(_stream_of(x), C.byref(a), None if ws is None else ws.data_ptr(), n_ws)
    if rc:
        _check(rc)
    return y, state_out, conv_state_out


def scan_grad(gy, x, dt, B, C_, A, z=None, skip=None, dt_bias=None, conv_w=None, conv_b=None, lengths=None, state=None,
              conv_state=None, g_state=None, stream=None):
    """mlt_scan_grad: the gradients of scan's inputs from those of y (`gy`) and
    of the returned state (`g_state`, or None).  Returns a dict by the names of
    the arguments (C_'s as "C"); None for inputs that were not given."""
    lb = _setup()
    if stream is not None:
        return _on(stream, scan_grad, gy, x, dt, B, C_, A, z, skip, dt_bias, conv_w, conv_b, lengths, state, conv_state,
                   g_state)
    torch = _torch
    a = _scan_args(x, dt, B, C_, A, z, skip, dt_bias, conv_w, conv_b, lengths, state, conv_state)
    q = ScanGrads()
    q.gy, q.gy_batch, q.gy_step = _wide(gy, "gy", x.dtype, x.shape)
    q.g_state_out = _plain(g_state, "g_state", torch.float32, (a.batch, a.dim, a.states))
    g = {}
    for name, t in (("x", x), ("dt", dt), ("z", z), ("B", B), ("C", C_), ("A", A), ("skip", skip),
                    ("dt_bias", dt_bias), ("conv_w", conv_w), ("conv_b", conv_b), ("state", state),
                    ("conv_state", conv_state)):
        if t is None:
            g[name] = None
            continue
        g[name] = new = _like(t)
        if new.numel() > 0:
            setattr(q, name, new.data_ptr())
    ws, n_ws = _workspace(("scan_grad", *x.shape, a.states, a.groups),
                          lambda w: lb.mlt_scan_grad_workspace(C.byref(a), C.byref(w)), x.device)
    rc = lb.mlt_scan_grad(_stream_of(x), C.byref(a), C.byref(q), None if ws is None else ws.data_ptr(), n_ws)
    if rc:
        _check(rc)
    return g


def _flat(t, name: str, dim: int, dtype=None):
    """(tensor [rows][dim], elements between its rows); a copy where t's rows lie at no one distance."""
    _cuda(t, name, dtype)
    if t.dim() != 2:
        t = t.reshape(-1, dim)
    stride, column = t.stride()
    if column != 1 and dim > 1 and t.numel() > 0:
        raise ValueError(f"{name} must have adjacent columns")
    return t, stride


def _flat_out(t, name: str, like, dtype):
    """The same for an output of like's shape, which may not be copied."""
    _cuda(t, name, dtype)
    _need(t.shape == like.shape, f"{name} must have x's shape")
    dim = t.shape[-1]
    flat = t if t.dim() == 2 else t.view(-1, dim)
    return flat.data_ptr(), _rows(flat, name)


def _one_device(first, *others):
    """That all tensors lie on first's device, and it is the current one; its number."""
    d = first.get_device()
    for t in others:
        if t is not None and t.get_device() != d:
            raise ValueError("all tensors must lie on one CUDA device")
    if _current_device() != d:
        raise ValueError(f"the tensors lie on device {d}, which is not the current one (torch.cuda.set_device)")
    return d


def _norm_weights(weight, bias, dim):
    """(type code, address, address) of vectors of dim values; their device is looked at elsewhere."""
    code, w, b = MLT_F32, None, None
    if weight is not None:
        code, w = _dtype_code(weight), weight.data_ptr()
        if weight.shape != (dim,) or (dim > 1 and weight.stride(0) != 1):
            raise ValueError(f"weight must be contiguous, of the shape ({dim},)")
    if bias is not None:
        b = bias.data_ptr()
        if bias.shape != (dim,) or (dim > 1 and bias.stride(0) != 1):
            raise ValueError(f"bias must be contiguous, of the shape ({dim},)")
        if weight is None:
            code = _dtype_code(bias)
        elif bias.dtype != weight.dtype:
            raise TypeError("weight and bias must be of one type")
    return code, w, b


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, residual=None, out_dtype=None, out=None, total_out=None,
               stream=None):
    """mlt_layer_norm over the last dimension of x, after adding `residual` (x's
    shape and type) where one is given.  Returns (y, total, stats): y in
    `out_dtype` (x's type, or a narrower one where x is fp32), the sum (x itself without a residual)
    and fp32 [...][2] of mean and 1 / deviation, which layer_norm_grad takes.  `out` and
    `total_out` receive y and total and may be x or residual themselves."""
    L = _setup()
    if stream is not None:
        return _on(stream, layer_norm, x, weight, bias, eps, residual, out_dtype, out, total_out)
    _cuda(x, "x")
    _need(x.dim() > 0, "x must have a last dimension")
    code, dim = _dtype_code(x), x.shape[-1]
    _need(1 <= dim <= _INT_MAX, "dim must lie in [1, 2^20]")
    flat, stride = _flat(x, "x", dim)
    w_code, w, b = _norm_weights(weight, bias, dim)
    r, r_stride = None, 0
    if residual is not None:
        if residual.shape != x.shape:
            raise ValueError("residual must have x's shape")
        r, r_stride = _flat(residual, "residual", dim, x.dtype)
    if out is None:
        y = _like(x) if out_dtype is None or out_dtype is x.dtype else _torch.empty(x.shape, dtype=out_dtype, device=x.device)
        at, y_stride = y.data_ptr(), dim
    else:
        y = out
        at, y_stride = _flat_out(out, "out", x, out_dtype)
    total, t_at, t_stride = x, None, 0
    if residual is None:
        _need(total_out is None, "total_out needs a residual")
    elif total_out is None:
        total = _like(x)
        t_at, t_stride = total.data_ptr(), dim
    else:
        total = total_out
        t_at, t_stride = _flat_out(total, "total_out", x, x.dtype)
    stats = _torch.empty((*x.shape[:-1], 2), dtype=_torch.float32, device=x.device)
    d = _one_device(x, weight, bias, residual, y, total)
    a = NormArgs(code, _dtype_code(y), w_code, dim, flat.shape[0], flat.data_ptr(), None if r is None else r.data_ptr(), w, b,
                 stride, r_stride, at, t_at, y_stride, t_stride, stats.data_ptr(), eps)
    rc = L.mlt_layer_norm(_raw_stream(d), C.byref(a))
    if rc:
        _check(rc)
    return y, total, stats


def layer_norm_grad(gy, x, stats, weight=None, bias=None, g_total=None, out=None, stream=None):
    """mlt_layer_norm_grad: the gradients of layer_norm's inputs from those of y (`gy`) and of
    total (`g_total`, or None).  `x` is what was normed: the total where a residual was added.
    Returns a dict: "x" (x's type, also the residual's gradient), "weight" and
    "bias" (their types; None where they were not given).  `out` receives "x" and may be x, g_total, or
    gy where the types are the same."""
    L = _setup()
    if stream is not None:
        return _on(stream, layer_norm_grad, gy, x, stats, weight, bias, g_total, out)
    _cuda(x, "x")
    _need(x.dim() > 0, "x must have a last dimension")
    code, dim = _dtype_code(x), x.shape[-1]
    _need(1 <= dim <= _INT_MAX, "dim must lie in [1, 2^20]")
    flat, stride = _flat(x, "x", dim)
    rows = flat.shape[0]
    for t, name in ((gy, "gy"), (g_total, "g_total")):
        _need(t is None or t.shape == x.shape, f"{name} must have x's shape")
    gy, gy_stride = _flat(gy, "gy", dim)
    t, t_stride = (None, 0) if g_total is None else _flat(g_total, "g_total", dim, x.dtype)
    w_code, w, b = _norm_weights(weight, bias, dim)
    s = _plain(stats, "stats", _torch.float32, (*x.shape[:-1], 2))
    if out is None:
        gx = _like(x)
        at, x_stride = gx.data_ptr(), dim
    else:
        gx = out
        at, x_stride = _flat_out(out, "out", x, x.dtype)
    g = {"x": gx, "weight": None, "bias": None}
    if weight is not None:
        g["weight"] = _like(weight)
    if bias is not None:
        g["bias"] = _like(bias)
    d = _one_device(x, gy, stats, weight, bias, g_total, out)
    a = NormArgs(code, _dtype_code(gy), w_code, dim, rows, flat.data_ptr(), None, w, b, stride, 0, None, None, 0, 0, s, 0.0)
    q = NormGrads(gy.data_ptr(), None if t is None else t.data_ptr(), gy_stride, t_stride, at, x_stride,
                  None if weight is None else g["weight"].data_ptr(), None if bias is None else g["bias"].data_ptr())
    ws, n_ws = (None, 0) if weight is None and bias is None else _workspace(
        ("layer_norm_grad", rows, dim), lambda o: L.mlt_layer_norm_grad_workspace(rows, dim, C.byref(o)), x.device)
    rc = L.mlt_layer_norm_grad(_raw_stream(d), C.byref(a), C.byref(q), None if ws is None else ws.data_ptr(), n_ws)
    if rc:
        _check(rc)
    return g


ADAMW_BLOCK = 256


class AdamWState(tuple):
    """The moments of adamw's tensors: flat tensors m, v, m_scale and v_scale (the scales None with
    moments in 32 bits); each parameter's part begins at a multiple of ADAMW_BLOCK
    elements.  32 bits: m and v fp32; 8 bits: m float8_e4m3fn, v float8_e5m2, and a moment
    is its value times its block's scale."""

    def __new__(cls, m, v, m_scale=None, v_scale=None):
        return super().__new__(cls, (m, v, m_scale, v_scale))

    m, v, m_scale, v_scale = (property(lambda self, k=k: self[k]) for k in range(4))

    @property
    def bits(self) -> int:
        return 32 if self[2] is None else 8


def adamw_state(params, bits: int = 32) -> AdamWState:
    """Moments of zero for adamw over `params` (a list of tensors), in 32 or 8 bits."""
    import torch

    _need(bits in (8, 32), "bits must be 8 or 32")
    blocks = sum(-(-p.numel() // ADAMW_BLOCK) for p in params)
    device = params[0].device if len(params) else "cuda"
    new = lambda n, dt: torch.zeros(n, dtype=dt, device=device)  # noqa: E731
    if bits == 32:
        return AdamWState(*(new(blocks * ADAMW_BLOCK, torch.float32) for _ in range(2)))
    return AdamWState(*(new(blocks * ADAMW_BLOCK, torch.uint8).view(dt) for dt in (torch.float8_e4m3fn, torch.float8_e5m2)),
                      *(new(blocks, torch.float32) for _ in range(2)))


_rate_words: dict = {}


def _rate_word(lr: float, decay: float) -> int:
    """lr and weight_decay of an mlt_adamw_tensor as one 64-bit word."""
    word = _rate_words.get((lr, decay))
    if word is None:
        if len(_rate_words) > 4096:
            _rate_words.clear()
        word = _rate_words[lr, decay] = struct.unpack("<q", struct.pack("<ff", lr, decay))[0]
    return word


def _per_tensor(value, count: int, name: str):
    if isinstance(value, (list, tuple)):
        _need(len(value) == count, f"{name} must have a value for each tensor")
        return value
    return [value] * count


def _adamw_rows(params, grads, copies, rates, decays, device):
    """mlt_adamw_tensor records of a few tensors as 64-bit words, the blocks of their moments, and what has
    to live until the launch."""
    words, blocks, kept = [], 0, []
    for p, g, rate, decay, copy in zip(params, grads, rates, decays, copies or [None] * len(params)):
        n = p.numel()
        blocks += -(-n // ADAMW_BLOCK)
        if g is None:
            words += (0, 0, 0, n, 0, 0)
            continue
        if p.get_device() != device or g.get_device() != device:
            raise ValueError("parameters, gradients, copies and moments must lie on one CUDA device")
        if not p.is_contiguous():
            raise ValueError("parameters and copies must be contiguous")
        if g.shape != p.shape:
            raise ValueError("a gradient and a copy must have their parameter's shape")
        if not g.is_contiguous():
            g = g.contiguous()
            kept.append(g)
        kinds, to = _dtype_code(p) | _dtype_code(g) << 16, 0
        if copy is not None:
            kinds |= _dtype_code(copy) << 32
            if copy.shape != p.shape or copy.get_device() != device:
                raise ValueError("a copy must be of its parameter's shape and device")
            if not copy.is_contiguous():
                raise ValueError("parameters and copies must be contiguous")
            to = copy.data_ptr()
        words += (p.data_ptr(), g.data_ptr(), to, n, kinds, _rate_words.get((rate, decay)) or _rate_word(rate, decay))
    return array("q", words), blocks, kept


def _adamw_columns(params, grads, copies, rates, decays, device):
    """The same for many tensors, column by column."""
    Tensor, count = _torch.Tensor, len(params)
    sizes = array("q", map(Tensor.numel, params))
    have = [k for k, g in enumerate(grads) if g is not None]
    if len(have) < count:  # the others' rows hold a size alone
        params, grads, copies, rates, decays = (q if q is None else [q[k] for k in have]
                                                for q in (params, grads, copies, rates, decays))
    bare = () if copies is None else [k for k, c in enumerate(copies) if c is None]
    if bare:  # the parameter stands in, and has no address below
        copies = [p if c is None else c for p, c in zip(params, copies)]
    given = [params, grads] if copies is None else [params, grads, copies]
    for some in given:
        if any(d != device for d in map(Tensor.get_device, some)):
            raise ValueError("parameters, gradients, copies and moments must lie on one CUDA device")
    if not all(map(Tensor.is_contiguous, params)) or not (copies is None or all(map(Tensor.is_contiguous, copies))):
        raise ValueError("parameters and copies must be contiguous")
    shapes = [p.shape for p in params]
    if any([t.shape for t in some] != shapes for some in given[1:]):
        raise ValueError("a gradient and a copy must have their parameter's shape")
    if not all(map(Tensor.is_contiguous, grads)):
        grads = given[1] = [g.contiguous() for g in grads]
    kinds, mixed = 0, None
    for k, some in enumerate(given):
        types = {t.dtype for t in some}
        if not types <= _DTYPES.keys():
            raise TypeError(f"float32, bfloat16 or float16 wanted, got {(types - _DTYPES.keys()).pop()}")
        if len(types) == 1:
            kinds += _DTYPES[types.pop()] << 16 * k
        elif types:
            mixed = [x + (_DTYPES[t.dtype] << 16 * k) for x, t in zip(mixed or [0] * len(some), some)]
    words = list(map(_rate_words.get, zip(rates, decays)))
    if None in words:
        words = [_rate_word(a, b) for a, b in zip(rates, decays)]
    columns = [array("q", map(Tensor.data_ptr, some)) for some in given] + [None] * (3 - len(given))
    for k in bare:
        columns[2][k] = 0
    columns += [sizes, array("q", [kinds] * len(have) if mixed is None else [x + kinds for x in mixed]), array("q", words)]
    table = array("q", bytes(48 * count))
    for k, column in enumerate(columns):
        if column is None:
            continue
        if len(column) < count:
            whole = array("q", bytes(8 * count))
            for i, x in zip(have, column):
                whole[i] = x
            column = whole
        table[k::6] = column
    blocks = int((-(-np.frombuffer(sizes, np.int64) // ADAMW_BLOCK)).sum()) if count else 0
    return table, blocks, given


def adamw(params, grads, state: AdamWState, step, lr=1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay=0.0,
          copies=None, grad_scale=None, seed: int = 0, lr_scale=1.0, stream=None) -> None:
    """mlt_adamw: one AdamW step over the tensors of `params`, in place, with `state` (adamw_state
    of the same list).  `grads`: a tensor of the parameter's shape for each, any of the three types, or
    None: that one is left as it is.  `step` counts from 1: a number or an int64 CUDA
    tensor of one value; `lr`: a number, a list of one for each tensor or an fp32 CUDA tensor of one
    value (tensors are read when the step runs, so a captured one may be replayed with others).
    `lr_scale` multiplies it; `weight_decay`, `lr_scale`: a number or a list.  `copies`: None, or a list that has
    for each parameter a tensor of its shape, which receives it in its own type, or None.  `grad_scale`: an
    fp32 CUDA tensor of one value that multiplies the gradients.  `seed`: of the rounding of moments in
    8 bits, 32 bits of it."""
    L = _setup()
    if stream is not None:
        return _on(stream, adamw, params, grads, state, step, lr, betas, eps, weight_decay, copies, grad_scale, seed,
                   lr_scale)
    torch = _torch
    count = len(params)
    _need(len(grads) == count and (copies is None or len(copies) == count),
          "grads and copies must have an entry for each parameter")
    m, v, ms, vs = state
    bits = 32 if ms is None else 8
    _need((ms is None) == (vs is None), "state must have both scales or none")
    f32 = torch.float32
    for t, dt in ((m, f32 if bits == 32 else torch.float8_e4m3fn), (v, f32 if bits == 32 else torch.float8_e5m2), (ms, f32),
                  (vs, f32)):
        if t is not None:
            _cuda(t, "moments", dt)
            _need(t.is_contiguous(), "moments must be contiguous")
    scalars = []
    for t, dt, name in ((step, torch.int64, "step"), (lr, f32, "lr"), (grad_scale, f32, "grad_scale")):
        if t is not None and (isinstance(t, torch.Tensor) or name == "grad_scale"):
            _cuda(t, name, dt)
            _need(t.numel() == 1, f"{name} must have one value")
            scalars.append(t.data_ptr())
        else:
            scalars.append(None)
    rates = _per_tensor(1.0 if scalars[1] is not None else lr, count, "lr")
    decays = _per_tensor(weight_decay, count, "weight_decay")
    if isinstance(lr_scale, (list, tuple)) or lr_scale != 1.0:
        rates = [a * b for a, b in zip(rates, _per_tensor(lr_scale, count, "lr_scale"))]
    device = m.get_device()
    table, blocks, kept = (_adamw_rows if count <= 32 else _adamw_columns)(params, grads, copies, rates, decays, device)
    _need(m.numel() == v.numel() == blocks * ADAMW_BLOCK and (ms is None or ms.numel() == vs.numel() == blocks),
          "the moments are of other parameters")
    _one_device(m, v, ms, vs, *[t for t in (step, lr, grad_scale) if isinstance(t, torch.Tensor)])
    rule = AdamWRule(betas[0], betas[1], eps, 0 if scalars[0] is not None else int(step), *scalars, bits, seed & 0xFFFFFFFF)
    rc = L.mlt_adamw(_raw_stream(device), table.buffer_info()[0], count, C.byref(rule), m.data_ptr(), v.data_ptr(),
                     None if ms is None else ms.data_ptr(), None if vs is None else vs.data_ptr())
    if rc:
        _check(rc)


def beam_step(scores, logp, m: int, done=None, eos: int = -1, normalised: bool = False, stream=None):
    """mlt_beam_step: the m best continuations of every item's beams.  `scores` [batch][beams][n]
    (or [beams][n] for one item), `logp` fp32 [batch][beams], `done` bool or uint8 of the same
    shape.  Returns (parent, token, logp, done): int64, int64, fp32 and bool
    [batch][m]; -1, -1, -infinity and False past the last continuation."""
    L = _setup()
    if stream is not None:
        return _on(stream, beam_step, scores, logp, m, done, eos, normalised)
    torch = _torch
    _cuda(scores, "scores")
    code = _dtype_code(scores)
    one = scores.dim() == 2
    if one:
        scores, logp = scores[None], logp[None]
        done = None if done is None else done[None]
    _need(scores.dim() == 3, "scores must be [batch][beams][n]")
    batch, beams, n = scores.shape
    m, eos = int(m), int(eos)
    _need(max(batch, beams, n, m) <= _INT_MAX, "batch, beams, n or m too large")
    strides = scores.stride()
    if strides[2] != 1 and n > 1 and scores.numel() > 0:
        raise ValueError("the scores of a beam must be adjacent")
    lp = _plain(logp, "logp", torch.float32, (batch, beams))
    d = None if done is None else _plain(done, "done", torch.uint8 if done.dtype == torch.uint8 else torch.bool, (batch, beams))
    device = scores.device
    size = (batch, m)
    parent = torch.empty(size, dtype=torch.int64, device=device)
    token = torch.empty(size, dtype=torch.int64, device=device)
    out = torch.empty(size, dtype=torch.float32, device=device)
    ended = torch.empty(size, dtype=torch.bool, device=device)
    on = _one_device(scores, logp, done)
    a = BeamArgs(code, batch, beams, n, m, 1 if normalised else 0, eos, scores.data_ptr(), strides[0], strides[1], lp, d,
                 parent.data_ptr(), token.data_ptr(), out.data_ptr(), ended.data_ptr())
    ws, n_ws = _workspace(("beam", code, batch, beams, n, m), lambda q: L.mlt_beam_step_workspace(C.byref(a), C.byref(q)),
                          device)
    rc = L.mlt_beam_step(_raw_stream(on), C.byref(a), None if ws is None else ws.data_ptr(), n_ws)
    if rc:
        _check(rc)
    return (parent[0], token[0], out[0], ended[0]) if one else (parent, token, out, ended)


def beam_reorder(parent, *tensors, stream=None) -> None:
    """mlt_beam_reorder: puts the rows of beams' states into the order that `parent` (int64
    [batch][beams], or [beams] for one item) gives, in place: row w of an item becomes what row
    parent[w] was; a negative parent leaves the row.  `tensors`: of any type,
    [batch * beams][...] or [batch][beams][...], the elements of a row adjacent."""
    L = _setup()
    if stream is not None:
        return _on(stream, beam_reorder, parent, *tensors)
    _cuda(parent, "parent", _torch.int64)
    _need(parent.dim() in (1, 2) and parent.is_contiguous(), "parent must be a contiguous int64 tensor [batch][beams]")
    batch, beams = (1, *parent.shape) if parent.dim() == 1 else parent.shape
    rows = batch * beams
    _need(batch <= _INT_MAX and beams <= _INT_MAX, "batch must lie in [0, 65535], beams in [1, 1024]")
    words = []
    on = _one_device(parent, *tensors)
    for t in tensors:
        shape = t.shape
        if len(shape) == 0 or (shape[0] != rows and tuple(shape[:2]) != (batch, beams)):
            raise ValueError("states must be [batch * beams][...] or [batch][beams][...]")
        n = t.numel()
        if n == 0:
            continue
        size = t.element_size()
        if t.is_contiguous():
            words += (t.data_ptr(), n * size // rows, n * size // rows)
            continue
        try:
            flat = t.view(rows, -1)
        except RuntimeError:
            raise ValueError("the elements of a state's row must be adjacent, its rows at one distance") from None
        stride, column = flat.stride()
        _need(column == 1 or flat.shape[1] == 1, "the elements of a state's row must be adjacent")
        words += (t.data_ptr(), flat.shape[1] * size, stride * size)
    moves = array("q", words)  # mlt_beam_state records
    rc = L.mlt_beam_reorder(_raw_stream(on), parent.data_ptr(), batch, beams, moves.buffer_info()[0], len(words) // 3)
    if rc:
        _check(rc)


def screen_host(feats: np.ndarray, thr: float, k: int, out=None, stream=None):
    """Screen a host [n][F] float32 array (copies in and out inside the call).

    `out` may be a (pvalid, perf, topk) triple of host arrays (for example
    pinned torch tensors' numpy views) to fill in place."""
    feats = np.ascontiguousarray(feats, dtype=np.float32)
    n = feats.shape[0]
    if out is None:
        out = (np.empty(n, np.float32), np.empty(n, np.float32), np.empty(k, np.int64))
    pv, pf, tk = out
    _check(lib().mlt_screen_host(_stream_ptr(stream), feats.ctypes.data, n, C.c_float(thr), int(k),
                                 pv.ctypes.data, pf.ctypes.data, tk.ctypes.data))
    return pv, pf, tk


def screen_host_batches(feats, thr: float, k: int, outs=None, stream=None):
    """Screen a list of host batches (each [n][F] fp32, page-locked for
    overlap) with the pipelined host entry point.  `outs`: a list of
    (pvalid, perf, topk) host arrays per batch (pvalid / perf may be None);
    allocated if omitted.  Returns the list."""
    feats = [np.asarray(f) for f in feats]
    nb = len(feats)
    n = feats[0].shape[0] if nb else 0
    for f in feats:
        if f.dtype != np.float32 or not f.flags.c_contiguous or f.shape[0] != n:
            raise ValueError("batches must be C-contiguous fp32 arrays of equal length")
    if outs is None:
        outs = [(np.empty(n, np.float32), np.empty(n, np.float32), np.empty(k, np.int64)) for _ in range(nb)]
    arr = lambda xs: (C.c_void_p * max(1, nb))(*[None if x is None else x.ctypes.data for x in xs])
    fp = arr(feats)
    pv = arr([o[0] for o in outs])
    pf = arr([o[1] for o in outs])
    tk = arr([o[2] for o in outs])
    _check(lib().mlt_screen_host_batches(_stream_ptr(stream), nb, fp, int(n), C.c_float(thr), int(k), pv, pf, tk))
    return outs


def _decoder_args(radices, option_values, program):
    r = np.ascontiguousarray(radices, dtype=np.int32)
    ov = np.ascontiguousarray(option_values, dtype=np.float32)
    prog = np.ascontiguousarray(program)
    if prog.dtype.itemsize != 16:
        raise ValueError("program must use the 16-byte op layout")
    return r, ov, prog


def decode_knobs(radices, option_values, program, first_index: int, n: int, device="cuda",
                 want_knobs=True, want_feats=True, stream=None):
    """(knobs [n][K] uint8, feats [n][F] fp32) CUDA tensors (None if not wanted)."""
    import torch

    r, ov, prog = _decoder_args(radices, option_values, program)
    knobs = torch.empty((n, r.size), dtype=torch.uint8, device=device) if want_knobs else None
    feats = torch.empty((n, prog.size), dtype=torch.float32, device=device) if want_feats else None
    _check(lib().mlt_decode_knobs(_stream_ptr(stream), r.ctypes.data, ov.ctypes.data, r.size,
                                  prog.ctypes.data, prog.size, int(first_index), int(n),
                                  _dptr(knobs), _dptr(feats)))
    return knobs, feats


def screen_decoded(radices, option_values, program, first_index: int, n: int, thr: float, k: int,
                   device="cuda", out_pvalid=None, out_perf=None, out_topk=None, stream=None):
    """Screen candidates first_index .. first_index+n-1 of a knob space."""
    r, ov, prog = _decoder_args(radices, option_values, program)
    pv, pf, tk = _outputs(n, k, device, out_pvalid, out_perf, out_topk)
    _check(lib().mlt_screen_decoded(_stream_ptr(stream), r.ctypes.data, ov.ctypes.data, r.size,
                                    prog.ctypes.data, int(first_index), int(n), C.c_float(thr),
                                    int(k), _dptr(pv), _dptr(pf), _dptr(tk)))
    return pv, pf, tk


def sync_status(stream=None) -> None:
    _check(lib().mlt_sync_status(_stream_ptr(stream)))


def selftest_wait_timeout(limit_ns: int, stream=None) -> None:
    """Launch the failure-detection self-test (a device wait that runs out);
    the next sync_status raises MltError with MLT_ETIMEOUT."""
    _check(lib().mlt_selftest_wait_timeout(_stream_ptr(stream), int(limit_ns)))


def selftest_walk_timeout(cta: int, limit_ns: int) -> None:
    """Arm the in-path self-test: the next screening call's V pass (full
    table) makes CTA `cta` give up waiting for its first tree chunk after
    limit_ns; the next sync_status raises MltError with MLT_ETIMEOUT."""
    _check(lib().mlt_selftest_walk_timeout(int(cta), int(limit_ns)))


def selftest_ordinal_timeout(limit_ns: int) -> None:
    """Arm a one-shot: CTA 0 of the next kernel that writes ordinals waits
    limit_ns on a barrier nothing completes."""
    _check(lib().mlt_selftest_ordinal_timeout(int(limit_ns)))


def selftest_sample_timeout(limit_ns: int) -> None:
    """Arm a one-shot: in the next draw from long rows one CTA of each row stays away and the
    others' waits give up after limit_ns; the row draws nothing."""
    _check(lib().mlt_selftest_sample_timeout(int(limit_ns)))


def selftest_poison_state(value: int, static_scratch: bool = False) -> None:
    """Write `value` into the selection state's counters (as a call that
    stopped part-way could leave them); the next call must not notice."""
    _check(lib().mlt_selftest_poison_state(1 if static_scratch else 0, C.c_uint32(value)))


def walk_peak(feats, rounds: int, model_id: int = MLT_MODEL_V, out_sums=None, stream=None):
    """mlt_walk_peak: walk the first trees of a full-table model, held in
    shared memory, `rounds` times for every row of `feats` (a [n][F] fp32
    CUDA tensor).  Returns (sums, visits): the per-row fp32 leaf sums and the
    node visits of the launch (time it with events on `stream`)."""
    import torch

    if not (isinstance(feats, torch.Tensor) and feats.is_cuda and feats.dtype == torch.float32):
        raise TypeError("feats must be a float32 CUDA tensor")
    if not feats.is_contiguous() or feats.dim() != 2:
        raise ValueError("feats must be a contiguous [n][F] tensor")
    n = feats.shape[0]
    if out_sums is None:
        out_sums = torch.empty(n, dtype=torch.float32, device=feats.device)
    visits = C.c_int64()
    _check(lib().mlt_walk_peak(_stream_ptr(stream), int(model_id), _dptr(feats), n, int(rounds), _dptr(out_sums),
                               C.byref(visits)))
    return out_sums, int(visits.value)


def last_survivor_count(stream=None) -> int:
    out = C.c_int64()
    _check(lib().mlt_last_survivor_count(_stream_ptr(stream), C.byref(out)))
    return int(out.value)


PHASES = ("v_pass", "compaction", "p_pass", "topk")


def profile_phases(enable: bool) -> None:
    _check(lib().mlt_profile_phases(1 if enable else 0))


def phase_times():
    """({phase: summed ms}, recorded calls) since profiling was enabled."""
    out = (C.c_float * 4)()
    calls = C.c_int64()
    _check(lib().mlt_phase_times(out, 4, C.byref(calls)))
    return dict(zip(PHASES, [float(v) for v in out])), int(calls.value)


def tune_walk(model_id: int, candidates: int = 0, splits: int = 0, group: int = 0, chunk_trees: int = 0,
              nbuf: int = 0) -> None:
    """Fix (or with zeros, release) the tree walk's launch shape for one model."""
    _check(lib().mlt_tune_walk(int(model_id), int(candidates), int(splits), int(group), int(chunk_trees),
                               int(nbuf)))


def tune_fused_small(max_n: int) -> None:
    """Batches up to max_n candidates (0 .. 8192) screen in one launch when
    their models allow it; 0 turns the single-launch path off."""
    _check(lib().mlt_tune_fused_small(int(max_n)))


def walk_shape(model_id: int, n: int, p_pass: bool = False) -> dict:
    """The launch shape the fp32 (or binary16) walk over model_id's trees would
    use for a screening call of n candidates (P pass: planned for about n/2)
    that is not walked in ordinal form."""
    out = np.zeros(7, dtype=np.int32)
    _check(lib().mlt_walk_shape(int(model_id), int(n), 1 if p_pass else 0, out.ctypes.data))
    kinds = {0: "full", 1: "compact", 2: "half", 3: "split"}
    return {"candidates": int(out[0]), "splits": int(out[1]), "group": int(out[2]), "chunk_trees": int(out[3]),
            "nbuf": int(out[4]), "resident": int(out[5]), "table": kinds.get(int(out[6]), str(int(out[6])))}


def ordinal_shape(model_id: int, n: int, p_pass: bool = False) -> dict | None:
    """The same for the walk in ordinal form; None where such a pass would be
    walked in fp32 form."""
    out = np.zeros(6, dtype=np.int32)
    _check(lib().mlt_ordinal_shape(int(model_id), int(n), 1 if p_pass else 0, out.ctypes.data))
    if out[0] == 0:
        return None
    names = ("candidates", "splits", "group", "chunk_trees", "nbuf", "resident")
    return dict({k: int(v) for k, v in zip(names, out)}, table="ordinal")


def tune_decode_jit(min_n: int) -> None:
    """Decoded batches of at least min_n candidates build their rows with
    the feature program compiled at run time (NVRTC); 0 keeps every decoded
    batch on the interpreted program."""
    _check(lib().mlt_tune_decode_jit(int(min_n)))


def tune_ordinal(mode: int) -> None:
    """Walk rows in ordinal form (same results): 1 where the library expects
    it to be faster (the default), 2 wherever a model has that form, 0 never."""
    _check(lib().mlt_tune_ordinal(int(mode)))


def decode_jit_available() -> bool:
    """Whether NVRTC and the CUDA driver library load in this process."""
    return bool(lib().mlt_decode_jit_available())


def decode_jit_calls() -> int:
    """Screening calls so far that ran the compiled feature program."""
    return int(lib().mlt_decode_jit_calls())


def tune_head_levels(levels: int) -> None:
    """Table format of deep (depth > 10) V and P models loaded afterwards:
    6 or 7 head levels in shared memory (split table), or 0 (compact)."""
    _check(lib().mlt_tune_head_levels(int(levels)))


def kernel_launches() -> int:
    return int(lib().mlt_kernel_launches())


def load_workload_models(w, half: bool = False) -> None:
    """Set F and load the workload's V and P ensembles (as half tables if
    `half`)."""
    set_num_features(w.cfg.F if w.feats is None else w.feats.shape[1])
    load = load_ensemble_f16 if half else load_ensemble
    load(MLT_MODEL_V, w.v.nodes, w.v.n_trees, w.v.depth)
    load(MLT_MODEL_P, w.p.nodes, w.p.n_trees, w.p.depth)
