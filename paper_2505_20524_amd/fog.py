"""Thin ctypes binding over libfog.so: the same calls as include/fog.h, argument marshalling only.

Tensors are torch CUDA tensors used purely as device buffers (`data_ptr()`); every step of the
path runs in the library's HIP kernels.  There is no CPU fallback: if the library has not been
built, `load()` raises.
"""
import ctypes
import os

import torch

E4M3, E5M2 = 0, 1
NT, NN, TN = 0, 1, 2
VECTOR, TILE = 0, 1          # fog_block: how an operand's block scales lie
BF16, F32 = 0, 1             # fog_real
STATES_F32, STATES_FP8 = 0, 1    # fog_states
HALF, INTERLEAVED = 0, 1     # fog_rope_layout
ROPE_JOBS_MAX, ROPE_DIM_MAX = 8, 1008      # FOG_ROPE_JOBS_MAX, FOG_ROPE_DIM_MAX of the header
CAST_BATCH_MAX = 32          # FOG_CAST_BATCH_MAX of the header

_LIB = None
_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfog.so")

_c = ctypes
_P, _I64, _I, _F, _D, _SZ = _c.c_void_p, _c.c_int64, _c.c_int, _c.c_float, _c.c_double, _c.c_size_t

SIGNATURES = {
    "fog_status_string": (_c.c_char_p, [_I]),
    "fog_version": (_I, []),
    "fog_amax": (_I, [_P, _I64, _P, _P]),
    "fog_scale": (_I, [_P, _I, _I, _P, _P, _P]),
    "fog_scale_delayed": (_I, [_P, _I, _P, _I, _I, _P, _P, _P]),
    "fog_quantize": (_I, [_P, _I64, _I64, _I64, _I, _P, _P, _I64, _P, _I64, _P, _P]),
    "fog_quantize_jit": (_I, [_P, _I64, _I64, _I64, _I, _I, _P, _I64, _P, _I64, _P, _P, _P, _P, _SZ, _P]),
    "fog_quantize_jit_workspace": (_SZ, []),
    "fog_quantize_jit_batch": (_I, [_P, _I, _P, _SZ, _P]),
    "fog_quantize_jit_batch_workspace": (_SZ, [_I]),
    "fog_quantize_delayed": (_I, [_P, _I64, _I64, _I64, _I, _I, _P, _I, _I64, _P, _SZ, _P, _I64, _P, _I64, _P, _P, _P, _P]),
    "fog_quantize_delayed_batch": (_I, [_P, _I, _I64, _P]),
    "fog_quantize_delayed_state": (_SZ, []),
    "fog_delayed_amax": (_I, [_P, _I64, _P, _P]),
    "fog_rmsnorm_quantize": (_I, [_P, _I64, _I64, _I64, _F, _I, _P, _P, _I64, _P, _P]),
    "fog_rope_quantize": (_I, [_P, _I, _I, _I, _I, _I, _I, _P, _I64, _P, _I, _I64, _P, _SZ, _P]),
    "fog_rope_grad": (_I, [_P, _I, _I, _I, _I, _I, _I, _P, _I64, _P, _I, _I64, _P, _SZ, _P]),
    "fog_rope_workspace": (_SZ, []),
    "fog_rope_table": (_I, [_P, _I64, _I64, _I, _P, _P]),
    "fog_xielu_quantize": (_I, [_P, _I64, _I64, _I64, _F, _F, _I, _P, _P, _I64, _P, _P]),
    "fog_gelu_quantize": (_I, [_P, _I64, _I64, _I64, _I, _P, _P, _I64, _P, _P]),
    "fog_tanh_quantize": (_I, [_P, _I64, _I64, _I64, _F, _I, _P, _P, _I64, _P, _P]),
    "fog_postnorm_residual_quantize": (_I, [_P, _I64, _P, _I64, _I64, _I64, _P, _I, _P, _P, _I64, _P, _I64, _P, _P]),
    "fog_postnorm_residual_grad": (_I, [_P, _I64, _P, _I64, _P, _I64, _I64, _I64, _P, _I, _P, _P, _I64, _P, _I64, _P, _I64, _P, _P, _I, _P, _SZ, _P]),
    "fog_postnorm_residual_grad_workspace": (_SZ, [_I64, _I64]),
    "fog_xielu_grad": (_I, [_P, _I64, _P, _I64, _I64, _I64, _F, _F, _I, _P, _P, _I64, _P, _I64, _P, _P, _I, _P, _SZ, _P]),
    "fog_gelu_grad": (_I, [_P, _I64, _P, _I64, _I64, _I64, _I, _P, _P, _I64, _P, _I64, _P, _P, _SZ, _P]),
    "fog_tanh_grad": (_I, [_P, _I64, _P, _I64, _I64, _I64, _F, _I, _P, _P, _I64, _P, _I64, _P, _P, _I, _P, _SZ, _P]),
    "fog_act_grad_workspace": (_SZ, []),
    "fog_kurtosis": (_I, [_P, _I64, _I64, _I64, _P, _P, _P]),
    "fog_fp8_gemm": (_I, [_I, _I64, _I64, _I64, _P, _I, _I64, _P, _P, _I, _I64, _P, _P, _I64, _P, _SZ, _P]),
    "fog_fp8_gemm_workspace": (_SZ, [_I, _I64, _I64, _I64]),
    "fog_quantize_block": (_I, [_P, _I64, _I64, _I64, _I, _I, _P, _I64, _P, _I64, _P, _I64, _P, _I64, _P]),
    "fog_quantize_tile": (_I, [_P, _I64, _I64, _I64, _I, _I, _P, _I64, _P, _I64, _P]),
    "fog_fp8_gemm_block": (_I, [_I, _I64, _I64, _I64, _P, _I, _I64, _I, _P, _I64, _P, _I, _I64, _I, _P, _I64, _P, _I64, _P, _SZ, _P]),
    "fog_fp8_gemm_block_workspace": (_SZ, [_I, _I64, _I64, _I64]),
    "fog_embed_quantize": (_I, [_P, _I, _I64, _P, _I64, _I64, _I64, _F, _I, _P, _P, _I64, _P, _I64, _P, _P]),
    "fog_embed_grad": (_I, [_P, _I, _I64, _P, _I64, _I64, _I64, _F, _I, _P, _I64, _I, _P, _SZ, _P]),
    "fog_embed_grad_workspace": (_SZ, [_I64, _I64, _I64]),
    "fog_grad_sumsq": (_I, [_P, _I, _P, _P, _SZ, _P]),
    "fog_grad_sumsq_workspace": (_SZ, [_I]),
    "fog_grad_clip": (_I, [_P, _I, _P, _F, _P, _P]),
    "fog_adamw": (_I, [_P, _I, _I, _D, _P, _D, _D, _D, _I64, _P, _c.c_uint64, _P, _F, _P]),
    "fog_fp8_attn_fwd": (_I, [_I, _I, _I, _I, _I, _F, _I, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _SZ, _P]),
    "fog_fp8_attn_bwd": (_I, [_I, _I, _I, _I, _I, _F, _I, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P,
                              _P, _P, _P, _P, _P, _SZ, _P]),
    "fog_fp8_attn_workspace": (_SZ, [_I, _I, _I, _I, _I, _I]),
    "fog_fp8_attn_bwd_static": (_I, [_I, _I, _I, _I, _I, _F, _I, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P,
                                     _P, _P, _P, _P, _P]),
}
ATTN_BWD_STATIC_MAX_ROWS = 524288      # FOG_ATTN_BWD_STATIC_MAX_ROWS of the header


# measurement helpers of the benchmark (include/fog_probe.h): not part of the hot path
PROBE_SIGNATURES = {
    "fog_probe_mfma_rate": (_I, [_P, _I, _P, _SZ, _c.POINTER(_c.c_double), _c.POINTER(_c.c_double), _P]),
    "fog_probe_attention_loop": (_I, [_I, _I, _I, _P, _SZ, _c.POINTER(_c.c_double), _P]),
    "fog_probe_mfma_coissue": (_I, [_I, _I, _I, _I, _P, _SZ, _c.POINTER(_c.c_double), _P]),
    "fog_probe_mfma_cross_wave": (_I, [_I, _I, _I, _I, _P, _SZ, _c.POINTER(_c.c_double), _c.POINTER(_c.c_double), _P]),
    "fog_probe_cast_plan": (_I, [_I64, _I64, _I, _I, _c.POINTER(_I)]),
    "fog_probe_quantize_held": (_I, [_P, _I, _P, _SZ, _I64, _P]),
    "fog_probe_quantize_held_transpose": (_I, [_P, _I64, _I64, _I64, _I, _I, _P, _I64, _P, _I64, _P, _P, _P, _P, _SZ, _I64, _P]),
    "fog_probe_gemm_plan": (_I, [_I, _I64, _I64, _I64, _I, _I] + [_c.POINTER(_I)] * 5),
    "fog_probe_gemm_products_only": (_I, [_I64, _I64, _I64, _P, _I64, _P, _I64, _P, _P, _P, _I64, _P]),
}


class FogError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        msg = load().fog_status_string(code).decode()
        super().__init__("%s failed: %s (status %d)" % (where, msg, code))


def load():
    """Loads libfog.so (built by __graft_entry__.build()); raises if it is missing."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libfog.so is not built: run `python __graft_entry__.py` (hipcc, gfx950) first; "
                               "there is no fallback path")
        lib = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in list(SIGNATURES.items()) + list(PROBE_SIGNATURES.items()):
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _LIB = lib
    return _LIB


def _ptr(t):
    return None if t is None else t.data_ptr()


# The current stream's handle without building a torch.cuda.Stream object around it: 0.5 us a call instead of 3.1 us, on calls
# whose kernels take 5 us.  (Builds of torch without the getter take the object.)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
# The same for the current device, 0.05 us instead of 0.2 (tensors on a device have initialised it).
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _check(code, where):
    if code != 0:
        raise FogError(code, where)


def amax(x, out, stream=None):
    _check(load().fog_amax(_ptr(x), x.numel(), _ptr(out), _stream(stream)), "fog_amax")


def scale(amax_t, fmt, scale_out, scale_inv_out, margin=0, stream=None):
    _check(load().fog_scale(_ptr(amax_t), fmt, margin, _ptr(scale_out), _ptr(scale_inv_out), _stream(stream)), "fog_scale")


def scale_delayed(history, new_amax, fmt, scale_out, scale_inv_out, margin=0, stream=None):
    _check(load().fog_scale_delayed(_ptr(history), history.numel(), _ptr(new_amax), fmt, margin, _ptr(scale_out),
                                    _ptr(scale_inv_out), _stream(stream)), "fog_scale_delayed")


def quantize(x, fmt, scale_t, q=None, qT=None, amax_out=None, stream=None):
    rows, cols = x.shape
    _check(load().fog_quantize(_ptr(x), rows, cols, x.stride(0), fmt, _ptr(scale_t),
                               _ptr(q), q.stride(0) if q is not None else 0,
                               _ptr(qT), qT.stride(0) if qT is not None else 0,
                               _ptr(amax_out), _stream(stream)), "fog_quantize")


def quantize_jit(x, fmt, amax_out, scale_out, scale_inv_out, workspace, q=None, qT=None, margin=0, stream=None):
    rows, cols = x.shape
    _check(load().fog_quantize_jit(_ptr(x), rows, cols, x.stride(0), fmt, margin,
                                   _ptr(q), q.stride(0) if q is not None else 0,
                                   _ptr(qT), qT.stride(0) if qT is not None else 0,
                                   _ptr(amax_out), _ptr(scale_out), _ptr(scale_inv_out),
                                   _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           "fog_quantize_jit")


def quantize_jit_workspace():
    return load().fog_quantize_jit_workspace()


class CastJob(ctypes.Structure):
    """Mirror of fog_cast_job."""
    _fields_ = [("x_bf16", _P), ("rows", _I64), ("cols", _I64), ("fmt", _I), ("margin", _I), ("q", _P), ("amax", _P),
                ("scale", _P), ("scale_inv", _P)]


def make_cast_jobs(items, margin=0):
    """items: (x, fmt, q, amax, scale, scale_inv) tuples of contiguous tensors -> ctypes array for quantize_jit_batch."""
    arr = (CastJob * len(items))()
    for job, (x, fmt, q, amax_t, scale_t, sinv_t) in zip(arr, items):
        rows, cols = x.shape
        job.x_bf16, job.rows, job.cols, job.fmt, job.margin = _ptr(x), rows, cols, fmt, margin
        job.q, job.amax, job.scale, job.scale_inv = _ptr(q), _ptr(amax_t), _ptr(scale_t), _ptr(sinv_t)
    return arr


def quantize_jit_batch(jobs, workspace, stream=None):
    """jobs: the array make_cast_jobs returns (it can be built once and reused while the tensors stay in place)."""
    _check(load().fog_quantize_jit_batch(ctypes.cast(jobs, _P), len(jobs), _ptr(workspace),
                                         workspace.numel() * workspace.element_size(), _stream(stream)), "fog_quantize_jit_batch")


def quantize_jit_batch_workspace(count):
    return load().fog_quantize_jit_batch_workspace(count)


def quantize_delayed(x, fmt, history, step, state, scale_out, scale_inv_out=None, q=None, qT=None, amax_prev=None, margin=0,
                     stream=None):
    rows, cols = x.shape
    _check(load().fog_quantize_delayed(_ptr(x), rows, cols, x.stride(0), fmt, margin, _ptr(history), history.numel(), step,
                                       _ptr(state), state.numel() * state.element_size(),
                                       _ptr(q), q.stride(0) if q is not None else 0,
                                       _ptr(qT), qT.stride(0) if qT is not None else 0,
                                       _ptr(amax_prev), _ptr(scale_out), _ptr(scale_inv_out), _stream(stream)),
           "fog_quantize_delayed")


class DelayedJob(ctypes.Structure):
    """Mirror of fog_delayed_job."""
    _fields_ = [("x_bf16", _P), ("rows", _I64), ("cols", _I64), ("fmt", _I), ("margin", _I), ("history", _P), ("history_len", _I),
                ("state", _P), ("state_bytes", _SZ), ("q", _P), ("amax_prev", _P), ("scale", _P), ("scale_inv", _P)]


def make_delayed_jobs(items, margin=0):
    """items: (x, fmt, q, history, state, amax_prev, scale, scale_inv) tuples of contiguous tensors (amax_prev and
    scale_inv may be None) -> ctypes array for quantize_delayed_batch."""
    arr = (DelayedJob * len(items))()
    for job, (x, fmt, q, history, state, amax_prev, scale_t, sinv_t) in zip(arr, items):
        rows, cols = x.shape
        job.x_bf16, job.rows, job.cols, job.fmt, job.margin = _ptr(x), rows, cols, fmt, margin
        job.history, job.history_len = _ptr(history), history.numel()
        job.state, job.state_bytes = _ptr(state), state.numel() * state.element_size()
        job.q, job.amax_prev, job.scale, job.scale_inv = _ptr(q), _ptr(amax_prev), _ptr(scale_t), _ptr(sinv_t)
    return arr


def quantize_delayed_batch(jobs, step, stream=None):
    """jobs: the array make_delayed_jobs returns (built once, reused while the tensors stay in place); step: the call number."""
    _check(load().fog_quantize_delayed_batch(ctypes.cast(jobs, _P), len(jobs), step, _stream(stream)), "fog_quantize_delayed_batch")


def quantize_delayed_state():
    return load().fog_quantize_delayed_state()


def delayed_amax(state, step, amax_out, stream=None):
    _check(load().fog_delayed_amax(_ptr(state), step, _ptr(amax_out), _stream(stream)), "fog_delayed_amax")


def rmsnorm_quantize(x, fmt, scale_t, q, gain=1.0, amax_out=None, stream=None):
    rows, cols = x.shape
    _check(load().fog_rmsnorm_quantize(_ptr(x), rows, cols, x.stride(0), gain, fmt, _ptr(scale_t), _ptr(q),
                                       q.stride(0) if q is not None else 0, _ptr(amax_out), _stream(stream)),
           "fog_rmsnorm_quantize")


class RopeScaling(ctypes.Structure):
    """Mirror of fog_rope_scaling."""
    _fields_ = [(k, _D) for k in ("base", "factor", "low", "high", "original", "amplitude")]


def rope_table(table, base=10000.0, first=0, factor=1.0, low=1.0, high=4.0, original=0.0, amplitude=1.0, stream=None):
    """table [positions, rot]: cosines, then sines, of the pairs at positions first, first + 1, ...; factor, low, high, original: frequencies scaled for long contexts."""
    positions, rot = table.shape
    if table.dtype != torch.float32 or not table.is_contiguous():
        raise ValueError("table: a contiguous float32 matrix is needed, got %s with strides %s" % (table.dtype, table.stride()))
    scaling = RopeScaling(base, factor, low, high, original, amplitude)
    _check(load().fog_rope_table(_c.byref(scaling), first, positions, rot, _ptr(table), _here(stream, table)), "fog_rope_table")


class Heads(ctypes.Structure):
    """Mirror of fog_heads."""
    _fields_ = [("p", _P), ("batch", _I64), ("token", _I64), ("head", _I64)]


class RopeJob(ctypes.Structure):
    """Mirror of fog_rope_job."""
    _fields_ = [("x", Heads), ("q", Heads), ("heads", _I), ("rotate", _I), ("gain", _F), ("fmt", _I), ("scale", _P), ("amax", _P)]


class RopeGradJob(ctypes.Structure):
    """Mirror of fog_rope_grad_job."""
    _fields_ = [("dy", Heads), ("x", Heads), ("dx", Heads), ("q", Heads), ("heads", _I), ("rotate", _I), ("gain", _F), ("fmt", _I), ("scale", _P), ("amax", _P)]


def _rope_jobs(kind, items, names, fmt):
    arr = (kind * len(items))()
    arr.tensors, arr.shape = [], None           # the array keeps the tensors alive
    for job, item in zip(arr, items):
        given = {k: item.get(k) for k in names}
        B, S, heads, D = given[names[0]].shape
        job.fmt = item.get("fmt", fmt)
        for k, t in given.items():
            if t is None:
                continue
            types = _codes(job.fmt) if k == "q" else _HALVES
            if tuple(t.shape) != (B, S, heads, D) or t.dtype not in types or (D > 1 and t.stride(3) != 1):
                raise ValueError("%s: a [%d, %d, %d, %d] tensor of one of %s with contiguous vectors is needed, got %s of %s with strides %s"
                                 % (k, B, S, heads, D, types, tuple(t.shape), t.dtype, t.stride()))
            setattr(job, k, Heads(_ptr(t), t.stride(0), t.stride(1), t.stride(2)))
            arr.tensors.append(t)
        if arr.shape not in (None, (B, S, D)):
            raise ValueError("tensors of one batch, length and head size are needed, got %s beside %s" % ((B, S, D), arr.shape))
        arr.shape = (B, S, D)
        job.heads, job.rotate, job.gain = heads, int(item.get("rotate", True)), item.get("gain", 0.0)
        for k in ("scale", "amax"):
            _floats(item.get(k), k)
            setattr(job, k, _ptr(item.get(k)))
            arr.tensors += [item[k]] if item.get(k) is not None else []
    arr.devices = {t.get_device() for t in arr.tensors}
    return arr


def make_rope_jobs(items):
    """items: dicts of a tensor's x (bfloat16 [B, S, heads, D], any strides between vectors), q (codes, the same shape, any strides), scale, and where they are
    wanted amax, rotate (True if missing), gain (0: no norm) and fmt (E4M3) -> ctypes array for rope_quantize (built once, reused while the tensors stay in place)."""
    if any(item.get("q") is None for item in items):
        raise ValueError("q: the codes' tensor is needed")
    return _rope_jobs(RopeJob, items, ("x", "q"), E4M3)


def make_rope_grad_jobs(items):
    """items: dicts of dy (bfloat16 [B, S, heads, D]), x (the forward's, where gain is above 0), dx and / or q with its scale, amax, rotate, gain, fmt (E5M2)
    -> ctypes array for rope_grad."""
    return _rope_jobs(RopeGradJob, items, ("dy", "x", "dx", "q"), E5M2)


def _rope(name, jobs, table, workspace, layout, positions, offset, stream):
    rows, rot = (0, 0) if table is None else table.shape
    if table is None and any(job.rotate for job in jobs):
        raise ValueError("a table is needed: without one, nothing is turned (rotate=False)")
    if table is not None and (table.dtype != torch.float32 or not table.is_contiguous()):
        raise ValueError("table: a contiguous float32 matrix is needed, got %s with strides %s" % (table.dtype, table.stride()))
    B, S, D = jobs.shape or (0, 0, rot)
    pos, size = None, 0
    if positions is not None:
        pos, size, count = _ids(positions)
        if count != B * S:
            raise ValueError("positions: one for each of the %d x %d tokens is needed, got %d" % (B, S, count))
    _jobs_here(jobs)
    _check(getattr(load(), name)(jobs, len(jobs), B, S, D, rot, layout, _ptr(table), rows, pos, size, offset, _ptr(workspace), _room(workspace),
                                 _here(stream, table, positions, workspace)), name)


def rope_quantize(jobs, table, workspace=None, layout=HALF, positions=None, offset=0, stream=None):
    """QK norm, rotary positions and FP8 cast of the jobs' tensors.  table: [positions, rot] of rope_table; positions: an int32 or int64 row of the table for
    every token, [B, S], or None for offset + s; workspace: rope_workspace() bytes, where a job has an amax."""
    _rope("fog_rope_quantize", jobs, table, workspace, layout, positions, offset, stream)


def rope_grad(jobs, table, workspace=None, layout=HALF, positions=None, offset=0, stream=None):
    """The gradients of rope_quantize's tensors from those of its results (table, layout, positions and offset as there)."""
    _rope("fog_rope_grad", jobs, table, workspace, layout, positions, offset, stream)


def rope_workspace():
    return load().fog_rope_workspace()


def xielu_quantize(x, alpha_p, alpha_n, fmt, scale_t, q, amax_out=None, stream=None):
    rows, cols = x.shape
    _check(load().fog_xielu_quantize(_ptr(x), rows, cols, x.stride(0), alpha_p, alpha_n, fmt, _ptr(scale_t), _ptr(q),
                                     q.stride(0) if q is not None else 0, _ptr(amax_out), _stream(stream)),
           "fog_xielu_quantize")


def gelu_quantize(x, fmt, scale_t, q, amax_out=None, stream=None):
    rows, cols = x.shape
    _check(load().fog_gelu_quantize(_ptr(x), rows, cols, x.stride(0), fmt, _ptr(scale_t), _ptr(q),
                                    q.stride(0) if q is not None else 0, _ptr(amax_out), _stream(stream)), "fog_gelu_quantize")


def tanh_quantize(x, alpha, fmt, scale_t, q, amax_out=None, stream=None):
    rows, cols = x.shape
    _check(load().fog_tanh_quantize(_ptr(x), rows, cols, x.stride(0), alpha, fmt, _ptr(scale_t), _ptr(q),
                                    q.stride(0) if q is not None else 0, _ptr(amax_out), _stream(stream)), "fog_tanh_quantize")


def postnorm_residual_quantize(x, y, gamma, fmt, scale_t, xnew, q=None, amax_out=None, stream=None):
    rows, cols = y.shape
    _check(load().fog_postnorm_residual_quantize(_ptr(x), x.stride(0), _ptr(y), y.stride(0), rows, cols, _ptr(gamma), fmt,
                                                 _ptr(scale_t), _ptr(xnew), xnew.stride(0), _ptr(q),
                                                 q.stride(0) if q is not None else 0, _ptr(amax_out), _stream(stream)),
           "fog_postnorm_residual_quantize")


def kurtosis(x, out, amax_out=None, stream=None):
    rows, cols = x.shape
    _check(load().fog_kurtosis(_ptr(x), rows, cols, x.stride(0), _ptr(out), _ptr(amax_out), _stream(stream)), "fog_kurtosis")


def fp8_gemm(layout, M, N, K, A, fmt_a, sinv_a, B, fmt_b, sinv_b, C, workspace=None, stream=None):
    ws = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(load().fog_fp8_gemm(layout, M, N, K, _ptr(A), fmt_a, A.stride(0), _ptr(sinv_a),
                               _ptr(B), fmt_b, B.stride(0), _ptr(sinv_b), _ptr(C), C.stride(0),
                               _ptr(workspace), ws, _stream(stream)), "fog_fp8_gemm")


def fp8_gemm_workspace(layout, M, N, K):
    return load().fog_fp8_gemm_workspace(layout, M, N, K)


BLOCK = 128                  # elements of a block scale


# what a tensor may be that the calls read or write as scale bytes, as codes of a format, as bfloat16, as binary32
_BYTES = (torch.uint8, torch.int8)
_CODES = {E4M3: _BYTES + (torch.float8_e4m3fn,), E5M2: _BYTES + (torch.float8_e5m2,)}
_HALVES = (torch.bfloat16, torch.int16)
_WORDS = (torch.float32,)


def _matrix(t, what, rows, cols, types):
    """The leading dimension of a matrix of at least rows x cols; refuses a tensor that the pointer and leading dimension of the call would
    misdescribe.  (Half a microsecond: calls that take five have up to five matrices.)"""
    if t.dim() == 2:
        r, c = t.shape
        ld, step = t.stride()
        if r >= rows and c >= cols and (step == 1 or c == 1) and t.dtype in types:
            return ld if ld >= cols or r > 1 else cols
    raise ValueError("%s: a [%d, %d] matrix of one of %s with contiguous rows is needed, got %s of %s with strides %s"
                     % (what, rows, cols, types, tuple(t.shape), t.dtype, t.stride()))


def _floats(t, what, dtype=torch.float32):
    if t is not None and (t.dtype != dtype or t.numel() < 1):
        raise ValueError("%s: a %s tensor is needed, got %s of %s" % (what, dtype, tuple(t.shape), t.dtype))


def _here(stream, *tensors):
    """The handle of the stream, after a look at where the tensors are: a kernel is launched on the current device and would fault on
    host memory or on another device's."""
    dev = _current_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError("a tensor on %s: the call runs on the current device, cuda:%d" % (t.device, dev))
    if stream is None:
        return _raw_stream(dev) if _raw_stream is not None else torch.cuda.current_stream().cuda_stream
    if stream.device_index != dev:
        raise ValueError("a stream of cuda:%d: the call runs on the current device, cuda:%d" % (stream.device_index, dev))
    return stream.cuda_stream


def _room(workspace):
    """Bytes of a workspace, which lie in one piece."""
    if workspace is None:
        return 0
    if not workspace.is_contiguous():
        raise ValueError("workspace: a contiguous tensor is needed, got strides %s" % (workspace.stride(),))
    return workspace.numel() * workspace.element_size()


def _codes(fmt):
    return _CODES.get(fmt, _BYTES)       # the call itself refuses a format that is none


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def quantize_block(x, fmt, q_row=None, s_row=None, q_col=None, s_col=None, margin=0, stream=None):
    """Casts with a scale for each block of 128 along the rows (q_row, s_row), along the columns (q_col, s_col), or both in one pass."""
    rows, cols = x.shape
    ldx = _matrix(x, "x", rows, cols, _HALVES)
    ld = [0, 0, 0, 0]
    codes = _codes(fmt)
    if q_row is not None:
        ld[0] = _matrix(q_row, "q_row", rows, cols, codes)
    if s_row is not None:
        ld[1] = _matrix(s_row, "s_row", _blocks(cols), rows, _BYTES)
    if q_col is not None:
        ld[2] = _matrix(q_col, "q_col", rows, cols, codes)
    if s_col is not None:
        ld[3] = _matrix(s_col, "s_col", _blocks(rows), cols, _BYTES)
    _check(load().fog_quantize_block(_ptr(x), rows, cols, ldx, fmt, margin, _ptr(q_row), ld[0], _ptr(s_row), ld[1],
                                     _ptr(q_col), ld[2], _ptr(s_col), ld[3], _here(stream, x, q_row, s_row, q_col, s_col)), "fog_quantize_block")


def quantize_tile(x, fmt, q, s, margin=0, stream=None):
    """The cast with a scale for each tile of 128 x 128."""
    rows, cols = x.shape
    _check(load().fog_quantize_tile(_ptr(x), rows, cols, _matrix(x, "x", rows, cols, _HALVES), fmt, margin, _ptr(q), _matrix(q, "q", rows, cols, _codes(fmt)),
                                    _ptr(s), _matrix(s, "s", _blocks(rows), _blocks(cols), _BYTES), _here(stream, x, q, s)), "fog_quantize_tile")


def fp8_gemm_block(layout, M, N, K, A, fmt_a, block_a, s_a, B, fmt_b, block_b, s_b, C, workspace=None, stream=None):
    """fp8_gemm on operands with a scale for each block of 128 contraction indices; block_a, block_b: VECTOR or TILE."""
    a_rows, a_cols = (K, M) if layout == TN else (M, K)
    b_rows, b_cols = (N, K) if layout == NT else (K, N)
    lda, ldb = _matrix(A, "A", a_rows, a_cols, _codes(fmt_a)), _matrix(B, "B", b_rows, b_cols, _codes(fmt_b))
    lds_a = _matrix(s_a, "s_a", _blocks(a_rows), _blocks(a_cols), _BYTES) if block_a == TILE else _matrix(s_a, "s_a", _blocks(K), M, _BYTES)
    lds_b = _matrix(s_b, "s_b", _blocks(b_rows), _blocks(b_cols), _BYTES) if block_b == TILE else _matrix(s_b, "s_b", _blocks(K), N, _BYTES)
    _check(load().fog_fp8_gemm_block(layout, M, N, K, _ptr(A), fmt_a, lda, block_a, _ptr(s_a), lds_a, _ptr(B), fmt_b, ldb, block_b, _ptr(s_b), lds_b,
                                     _ptr(C), _matrix(C, "C", M, N, _HALVES), _ptr(workspace), _room(workspace), _here(stream, A, s_a, B, s_b, C, workspace)), "fog_fp8_gemm_block")


def fp8_gemm_block_workspace(layout, M, N, K):
    return load().fog_fp8_gemm_block_workspace(layout, M, N, K)


def _ids(tokens):
    """Tokens as the calls take them: a contiguous vector of 4- or 8-byte integers."""
    if tokens.dtype not in (torch.int32, torch.int64) or not tokens.is_contiguous():
        raise ValueError("tokens: contiguous int32 or int64 ids are needed, got %s with strides %s" % (tokens.dtype, tokens.stride()))
    return tokens.data_ptr(), tokens.element_size(), tokens.numel()


def embed_quantize(tokens, table, factor, fmt, scale_t, x, q=None, amax_out=None, stream=None):
    """x = bf16(factor * table[tokens]) with its FP8 cast and abs-max; tokens outside the table give rows of zeros."""
    ids, size, count = _ids(tokens)
    vocab, cols = table.shape
    _floats(scale_t, "scale_t")
    _floats(amax_out, "amax_out")
    _check(load().fog_embed_quantize(ids, size, count, _ptr(table), vocab, cols, _matrix(table, "table", vocab, cols, _HALVES), factor, fmt, _ptr(scale_t),
                                     _ptr(x), _matrix(x, "x", count, cols, _HALVES), _ptr(q), _matrix(q, "q", count, cols, _codes(fmt)) if q is not None else 0,
                                     _ptr(amax_out), _here(stream, tokens, table, scale_t, x, q, amax_out)), "fog_embed_quantize")


def embed_grad(tokens, dx, factor, dE, workspace, accumulate=False, stream=None):
    """dE[v] = factor * sum of dx[t] over the tokens t with id v (binary32 or bf16 dE, overwritten or added to)."""
    ids, size, count = _ids(tokens)
    vocab, cols = dE.shape
    kind = F32 if dE.dtype == torch.float32 else BF16
    _check(load().fog_embed_grad(ids, size, count, _ptr(dx), _matrix(dx, "dx", count, cols, _HALVES), vocab, cols, factor, kind, _ptr(dE),
                                 _matrix(dE, "dE", vocab, cols, _WORDS if kind == F32 else _HALVES), int(accumulate),
                                 _ptr(workspace), _room(workspace), _here(stream, tokens, dx, dE, workspace)), "fog_embed_grad")


def embed_grad_workspace(count, vocab, cols):
    return load().fog_embed_grad_workspace(count, vocab, cols)


class GradJob(ctypes.Structure):
    """Mirror of fog_grad_job."""
    _fields_ = [("g", _P), ("out", _P), ("n", _I64), ("type", _I)]


def make_grad_jobs(items):
    """items: gradients, or (gradient, clipped gradient) pairs, contiguous and in binary32 or 2-byte bfloat16 -> ctypes array for grad_sumsq
    and grad_clip (built once, reused while the tensors stay in place).  A gradient by itself is clipped in place."""
    arr = (GradJob * len(items))()
    arr.tensors = []           # the array keeps them alive
    for job, item in zip(arr, items):
        g, out = item if isinstance(item, (tuple, list)) else (item, item)
        for t in (g, out):
            if not t.is_contiguous() or t.dtype not in _WORDS + _HALVES or t.dtype != g.dtype or t.numel() != g.numel():
                raise ValueError("contiguous float32 or bfloat16 gradients are needed, with results of their size and type")
        job.g, job.out, job.n, job.type = _ptr(g), _ptr(out), g.numel(), F32 if g.dtype == torch.float32 else BF16
        arr.tensors += [g, out]
    arr.devices = {t.get_device() for t in arr.tensors}
    return arr


def _jobs_here(jobs):
    dev = _current_device()
    if jobs.devices - {dev}:
        raise ValueError("gradients on devices %s (-1: the host): the call runs on the current device, cuda:%d" % (sorted(jobs.devices), dev))


def grad_sumsq(jobs, sumsq, workspace, stream=None):
    """sumsq (one float64): the sum of the squares of all gradients."""
    _floats(sumsq, "sumsq", torch.float64)
    _jobs_here(jobs)
    _check(load().fog_grad_sumsq(jobs, len(jobs), _ptr(sumsq), _ptr(workspace), _room(workspace),
                                 _here(stream, sumsq, workspace)), "fog_grad_sumsq")


def grad_sumsq_workspace(count):
    return load().fog_grad_sumsq_workspace(count)


def grad_clip(jobs, sumsq, max_norm, norm=None, stream=None):
    """out = g * min(1, max_norm / sqrt(sumsq)) for every job; norm: receives sqrt(sumsq)."""
    _floats(sumsq, "sumsq", torch.float64)
    _floats(norm, "norm")
    _jobs_here(jobs)
    _check(load().fog_grad_clip(jobs, len(jobs), _ptr(sumsq), max_norm, _ptr(norm), _here(stream, sumsq, norm)), "fog_grad_clip")


def _vector(t, what, n):
    """Pointer of a contiguous vector of n floats that may be missing."""
    if t is None:
        return None
    if t.dtype != torch.float32 or t.numel() != n or not t.is_contiguous():
        raise ValueError("%s: %d contiguous float32 numbers are needed, got %s of %s with strides %s" % (what, n, tuple(t.shape), t.dtype, t.stride()))
    return t.data_ptr()


def _some(t, what, rows, cols, types):
    """Pointer and leading dimension of a matrix that may be missing."""
    if t is None:
        return None, 0
    if t.shape == (rows, cols) and t.dtype in types:          # (the usual case at half the cost)
        ld, step = t.stride()
        if step == 1 and ld >= cols:
            return t.data_ptr(), ld
    return t.data_ptr(), _matrix(t, what, rows, cols, types)


def postnorm_residual_grad(dres, y, gamma, fmt, scale_t, dgamma, workspace, dbranch=None, dstream=None, dy=None, q=None, amax_out=None, accumulate=False, stream=None):
    """The way back through postnorm_residual_quantize: dstream = dres + dbranch, the gradient dy of y and / or its codes q, their abs-max, and the gains' gradient dgamma
    (None for none; accumulate: added to)."""
    rows, cols = y.shape
    _floats(scale_t, "scale_t")
    _floats(amax_out, "amax_out")
    where = _here(stream, dres, y, gamma, scale_t, dgamma, workspace, dbranch, dstream, dy, q, amax_out)
    _check(load().fog_postnorm_residual_grad(*_some(dres, "dres", rows, cols, _HALVES), *_some(dbranch, "dbranch", rows, cols, _HALVES), *_some(y, "y", rows, cols, _HALVES),
                                             rows, cols, _vector(gamma, "gamma", cols), fmt, _ptr(scale_t), *_some(dstream, "dstream", rows, cols, _HALVES),
                                             *_some(dy, "dy", rows, cols, _HALVES), *_some(q, "q", rows, cols, _codes(fmt)), _ptr(amax_out),
                                             _vector(dgamma, "dgamma", cols), int(accumulate), _ptr(workspace), _room(workspace), where), "fog_postnorm_residual_grad")


def postnorm_residual_grad_workspace(rows, cols):
    return load().fog_postnorm_residual_grad_workspace(rows, cols)


def _act_grad(name, x, dy, alpha, params, fmt, scale_t, workspace, dx, q, amax_out, dalpha, accumulate, stream):
    rows, cols = x.shape
    _floats(scale_t, "scale_t")
    _floats(amax_out, "amax_out")
    where = _here(stream, x, dy, scale_t, workspace, dx, q, amax_out, dalpha)
    own = (_vector(dalpha, "dalpha", params), int(accumulate)) if params else ()
    _check(getattr(load(), name)(*_some(x, "x", rows, cols, _HALVES), *_some(dy, "dy", rows, cols, _HALVES), rows, cols, *alpha, fmt, _ptr(scale_t),
                                 *_some(dx, "dx", rows, cols, _HALVES), *_some(q, "q", rows, cols, _codes(fmt)), _ptr(amax_out), *own, _ptr(workspace), _room(workspace),
                                 where), name)


def xielu_grad(x, dy, alpha_p, alpha_n, fmt, scale_t, workspace, dx=None, q=None, amax_out=None, dalpha=None, accumulate=False, stream=None):
    """The way back through xielu_quantize: dx and / or its codes q, their abs-max, and dalpha, two floats for alpha_p and alpha_n (accumulate: added to)."""
    _act_grad("fog_xielu_grad", x, dy, (alpha_p, alpha_n), 2, fmt, scale_t, workspace, dx, q, amax_out, dalpha, accumulate, stream)


def gelu_grad(x, dy, fmt, scale_t, workspace, dx=None, q=None, amax_out=None, stream=None):
    """The way back through gelu_quantize: dx and / or its codes q, and their abs-max."""
    _act_grad("fog_gelu_grad", x, dy, (), 0, fmt, scale_t, workspace, dx, q, amax_out, None, False, stream)


def tanh_grad(x, dy, alpha, fmt, scale_t, workspace, dx=None, q=None, amax_out=None, dalpha=None, accumulate=False, stream=None):
    """The way back through tanh_quantize: dx and / or its codes q, their abs-max, and dalpha, one float (accumulate: added to)."""
    _act_grad("fog_tanh_grad", x, dy, (alpha,), 1, fmt, scale_t, workspace, dx, q, amax_out, dalpha, accumulate, stream)


def act_grad_workspace():
    return load().fog_act_grad_workspace()


class AdamwJob(ctypes.Structure):
    """Mirror of fog_adamw_job."""
    _fields_ = [("p", _P), ("g", _P), ("master", _P), ("m", _P), ("v", _P), ("m_scale", _P), ("v_scale", _P), ("n", _I64), ("p_type", _I), ("g_type", _I),
                ("weight_decay", _F)]


def make_adamw_jobs(items):
    """items: dicts of a parameter's contiguous tensors p, g, m, v, where it has them master, m_scale and v_scale, and its weight_decay (0 if
    missing) -> ctypes array for adamw (built once, reused while the tensors stay in place).  Moments in float32, or codes with scale bytes."""
    arr = (AdamwJob * len(items))()
    arr.tensors, arr.states = [], None          # the array keeps them alive
    for job, item in zip(arr, items):
        t = {k: item.get(k) for k in ("p", "g", "master", "m", "v", "m_scale", "v_scale")}
        if t["p"] is None or t["m"] is None:
            raise ValueError("a parameter p and its states m and v are needed")
        n, states = t["p"].numel(), STATES_F32 if t["m"].dtype == torch.float32 else STATES_FP8
        fp8, blocks = states == STATES_FP8, _blocks(n)
        want = {"p": (_WORDS + _HALVES, n), "g": (_WORDS + _HALVES, n), "master": (_WORDS, n), "m": (_codes(E4M3) if fp8 else _WORDS, n),
                "v": (_codes(E5M2) if fp8 else _WORDS, n), "m_scale": (_BYTES, blocks), "v_scale": (_BYTES, blocks)}
        for k, (types, size) in want.items():
            if t[k] is None and (k == "master" or (k in ("m_scale", "v_scale") and not fp8)):
                continue
            if t[k] is None or not t[k].is_contiguous() or t[k].dtype not in types or t[k].numel() != size:
                raise ValueError("%s: a contiguous tensor of %d elements of one of %s is needed" % (k, size, types))
        if arr.states not in (None, states):
            raise ValueError("states of one kind are needed for all tensors of a call")
        arr.states = states
        job.p, job.g, job.master, job.m, job.v = _ptr(t["p"]), _ptr(t["g"]), _ptr(t["master"]), _ptr(t["m"]), _ptr(t["v"])
        job.m_scale, job.v_scale, job.n = _ptr(t["m_scale"]) if fp8 else None, _ptr(t["v_scale"]) if fp8 else None, n
        job.p_type, job.g_type = (F32 if t[k].dtype == torch.float32 else BF16 for k in ("p", "g"))
        job.weight_decay = item.get("weight_decay", 0.0)
        arr.tensors += [x for x in t.values() if x is not None]
    arr.devices = {t.get_device() for t in arr.tensors}
    return arr


def adamw(jobs, lr, step, beta1=0.9, beta2=0.95, eps=1e-8, seed=0, sumsq=None, max_norm=1.0, stream=None):
    """One AdamW step.  lr, step: numbers, or one float32 and one int64 in device memory (for a step that is captured and replayed); sumsq: the sum of
    squares from grad_sumsq, by which the gradients are clipped to max_norm on their way, None for no clipping."""
    lr_dev, step_dev = (t if isinstance(t, torch.Tensor) else None for t in (lr, step))
    _floats(sumsq, "sumsq", torch.float64)
    _floats(lr_dev, "lr")
    _floats(step_dev, "step", torch.int64)
    _jobs_here(jobs)
    _check(load().fog_adamw(jobs, len(jobs), jobs.states or 0, 0.0 if lr_dev is not None else lr, _ptr(lr_dev), beta1, beta2, eps,
                            0 if step_dev is not None else step, _ptr(step_dev), seed, _ptr(sumsq), max_norm, _here(stream, lr_dev, step_dev, sumsq)), "fog_adamw")


def fp8_attn_fwd(B, H, S, D, softmax_scale, causal, Q, K, V, sinv_q, sinv_k, sinv_v, scale_p, O, lse,
                 amax_p=None, workspace=None, stream=None, H_kv=None):
    """H_kv: key/value heads (grouped-query attention); None means H (multi-head)."""
    ws = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(load().fog_fp8_attn_fwd(B, H, H if H_kv is None else H_kv, S, D, softmax_scale, int(causal), _ptr(Q), _ptr(K), _ptr(V),
                                   _ptr(sinv_q), _ptr(sinv_k), _ptr(sinv_v), _ptr(scale_p), _ptr(O), _ptr(lse),
                                   _ptr(amax_p), _ptr(workspace), ws, _stream(stream)), "fog_fp8_attn_fwd")


def fp8_attn_bwd(B, H, S, D, softmax_scale, causal, Q, K, V, sinv_q, sinv_k, sinv_v, O, dO, dO8, sinv_do,
                 lse, scale_p, scale_ds, dQ, dK, dV, amax_ds=None, workspace=None, stream=None, H_kv=None):
    ws = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(load().fog_fp8_attn_bwd(B, H, H if H_kv is None else H_kv, S, D, softmax_scale, int(causal), _ptr(Q), _ptr(K), _ptr(V),
                                   _ptr(sinv_q), _ptr(sinv_k), _ptr(sinv_v), _ptr(O), _ptr(dO), _ptr(dO8),
                                   _ptr(sinv_do), _ptr(lse), _ptr(scale_p), _ptr(scale_ds),
                                   _ptr(dQ), _ptr(dK), _ptr(dV), _ptr(amax_ds), _ptr(workspace), ws,
                                   _stream(stream)), "fog_fp8_attn_bwd")


def fp8_attn_bwd_static(B, H, S, D, softmax_scale, causal, Q, K, V, sinv_q, sinv_k, sinv_v, O, dO, dO8, sinv_do,
                        lse, scale_p, scale_ds, dQ, dK, dV, amax_ds=None, stream=None, H_kv=None):
    """fp8_attn_bwd without a workspace: the library's own device array serves (B * H * S <= ATTN_BWD_STATIC_MAX_ROWS)."""
    _check(load().fog_fp8_attn_bwd_static(B, H, H if H_kv is None else H_kv, S, D, softmax_scale, int(causal), _ptr(Q), _ptr(K),
                                          _ptr(V), _ptr(sinv_q), _ptr(sinv_k), _ptr(sinv_v), _ptr(O), _ptr(dO), _ptr(dO8),
                                          _ptr(sinv_do), _ptr(lse), _ptr(scale_p), _ptr(scale_ds),
                                          _ptr(dQ), _ptr(dK), _ptr(dV), _ptr(amax_ds), _stream(stream)), "fog_fp8_attn_bwd_static")


def fp8_attn_workspace(B, H, S, D, is_bwd, H_kv=None):
    return load().fog_fp8_attn_workspace(B, H, H if H_kv is None else H_kv, S, D, int(is_bwd))


def probe_mfma_rate(operand_bytes, iters, sink, stream=None):
    """(TFLOP/s, GHz) of a register-resident FP8 matrix-instruction loop on the given 64 KB of operand codes (fog_probe.h)."""
    tf, ghz = _c.c_double(0.0), _c.c_double(0.0)
    _check(load().fog_probe_mfma_rate(_ptr(operand_bytes), iters, _ptr(sink), sink.numel() * sink.element_size(),
                                      _c.byref(tf), _c.byref(ghz), _stream(stream)), "fog_probe_mfma_rate")
    return tf.value, ghz.value


def probe_attention_loop(what, waves_per_simd, iters, sink, stream=None):
    """ns a SIMD spends per wave and key block in the memory-free attention inner loop (fog_probe.h); what: 0 all, 1 matrix
    instructions only, 2 softmax arithmetic only."""
    ns = _c.c_double(0.0)
    _check(load().fog_probe_attention_loop(what, waves_per_simd, iters, _ptr(sink), sink.numel() * sink.element_size(),
                                           _c.byref(ns), _stream(stream)), "fog_probe_attention_loop")
    return ns.value


def probe_mfma_coissue(op, vector_ops, with_mfma, iters, sink, stream=None):
    """Shader cycles per slot (one matrix instruction + vector_ops vector operations, order pinned), one wave per SIMD."""
    cyc = _c.c_double(0.0)
    _check(load().fog_probe_mfma_coissue(op, vector_ops, int(with_mfma), iters, _ptr(sink), sink.numel() * sink.element_size(),
                                         _c.byref(cyc), _stream(stream)), "fog_probe_mfma_coissue")
    return cyc.value


def probe_mfma_cross_wave(op, vector_ops, iters_matrix, iters_vector, sink, stream=None):
    """(cycles per matrix instruction of the matrix waves, cycles per group of vector_ops operations of the vector waves that
    share their SIMDs); a role with zero trips is absent."""
    cm, cv = _c.c_double(0.0), _c.c_double(0.0)
    _check(load().fog_probe_mfma_cross_wave(op, vector_ops, iters_matrix, iters_vector, _ptr(sink), sink.numel() * sink.element_size(),
                                            _c.byref(cm), _c.byref(cv), _stream(stream)), "fog_probe_mfma_cross_wave")
    return cm.value, cv.value


def probe_cast_plan(rows, cols, with_transpose=False, compute_units=0):
    """Whether quantize_jit casts such a tensor in one launch (fog_probe.h; no device needed)."""
    out = _I(0)
    _check(load().fog_probe_cast_plan(rows, cols, int(with_transpose), compute_units, _c.byref(out)), "fog_probe_cast_plan")
    return bool(out.value)


def probe_quantize_held(jobs, workspace, absent, stream=None):
    """quantize_jit_batch in its one-launch form whatever the sizes (fog_probe.h)."""
    _check(load().fog_probe_quantize_held(ctypes.cast(jobs, _P), len(jobs), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                          absent, _stream(stream)), "fog_probe_quantize_held")


def probe_quantize_held_transpose(x, fmt, amax_out, scale_out, scale_inv_out, workspace, absent, qT, q=None, margin=0, stream=None):
    """quantize_jit with a transposed copy in its one-launch form whatever the sizes (fog_probe.h)."""
    rows, cols = x.shape
    _check(load().fog_probe_quantize_held_transpose(_ptr(x), rows, cols, x.stride(0), fmt, margin,
                                                    _ptr(q), q.stride(0) if q is not None else 0, _ptr(qT), qT.stride(0),
                                                    _ptr(amax_out), _ptr(scale_out), _ptr(scale_inv_out),
                                                    _ptr(workspace), workspace.numel() * workspace.element_size(), absent, _stream(stream)),
           "fog_probe_quantize_held_transpose")


def probe_gemm_plan(layout, M, N, K, with_workspace=False, compute_units=0):
    """(tile_m, tile_n, workgroups per CU, splits, k_chunk) of the kernel that fp8_gemm takes (fog_probe.h; no device needed)."""
    out = [_I(0) for _ in range(5)]
    _check(load().fog_probe_gemm_plan(layout, M, N, K, int(with_workspace), compute_units, *[_c.byref(o) for o in out]), "fog_probe_gemm_plan")
    return tuple(o.value for o in out)


def probe_gemm_products_only(M, N, K, A, sinv_a, B, sinv_b, C, stream=None):
    """fog_fp8_gemm's NT product of E4M3 operands without any tile's epilogue (fog_probe.h); C is not written."""
    _check(load().fog_probe_gemm_products_only(M, N, K, _ptr(A), A.stride(0), _ptr(B), B.stride(0), _ptr(sinv_a), _ptr(sinv_b),
                                               _ptr(C), C.stride(0), _stream(stream)), "fog_probe_gemm_products_only")
