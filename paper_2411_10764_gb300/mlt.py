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
import threading

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


def _setup():
    """The library and, once, what the calls below need of torch."""
    global _torch, _raw_stream
    if _torch is None:
        import torch

        _DTYPES.update({torch.float32: MLT_F32, torch.bfloat16: MLT_BF16, torch.float16: MLT_F16})
        # the handle of the current stream without building a Stream object
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda device: torch.cuda.current_stream(device).cuda_stream)
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
            for one in t if isinstance(t, tuple) else (t,):
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
