"""ctypes binding of liblogquant.so: argument marshalling only.

The functions carry the names of the C entry points declared in
include/logquant.h.  PyTorch appears only as the owner of device memory and of
the HIP stream; every step of the path runs in the library's kernels.  There is
no fallback: if the shared library is missing, importing this module fails.
"""
import collections
import ctypes as C
import os
from array import array

# PyTorch ships its own HIP runtime.  It has to be in the process before the library
# is loaded so that the library binds to that same runtime (matched by soname); two
# HIP runtimes in one process cannot both open the GPU.
import torch  # noqa: F401  (device memory and streams come from here as well)

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "liblogquant.so")

LQ_OK, LQ_ERR_NULL, LQ_ERR_SHAPE, LQ_ERR_UNSUPPORTED, LQ_ERR_CAPACITY, LQ_ERR_STATE, LQ_ERR_HIP = range(7)
LQ_F16, LQ_BF16 = 0, 1


class lq_config(C.Structure):
    _fields_ = [("B", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("d", C.c_int32),
                ("fp_budget", C.c_int32), ("group", C.c_int32), ("bits", C.c_int32),
                ("dtype", C.c_int32), ("q_capacity", C.c_int32)]


class lq_cache(C.Structure):
    _fields_ = [("k_fp", C.c_void_p * 2), ("v_fp", C.c_void_p * 2), ("pos_fp", C.c_void_p * 2),
                ("k_codes", C.c_void_p), ("v_codes", C.c_void_p),
                ("k_scale", C.c_void_p), ("k_zero", C.c_void_p),
                ("v_scale", C.c_void_p), ("v_zero", C.c_void_p),
                ("pos_q", C.c_void_p),
                ("cur", C.c_int32), ("n_fp", C.c_int32), ("n_q", C.c_int32)]


class lq_cache_seq(C.Structure):
    _fields_ = [("k_fp", C.c_void_p * 2), ("v_fp", C.c_void_p * 2), ("pos_fp", C.c_void_p * 2),
                ("k_codes", C.c_void_p), ("v_codes", C.c_void_p),
                ("k_scale", C.c_void_p), ("k_zero", C.c_void_p),
                ("v_scale", C.c_void_p), ("v_zero", C.c_void_p),
                ("pos_q", C.c_void_p),
                ("cur", C.POINTER(C.c_int32)), ("n_fp", C.POINTER(C.c_int32)), ("n_q", C.POINTER(C.c_int32)),
                ("seq_state", C.c_void_p)]


class lq_sizes(C.Structure):
    _fields_ = [(n, C.c_size_t) for n in ("k_fp", "v_fp", "pos_fp", "k_codes", "v_codes", "k_meta",
                                          "v_meta", "pos_q", "workspace")]


class lq_config8(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("B", "Hq", "Hkv", "d", "block", "dtype", "capacity")]


class lq_cache8(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail")] + [
        ("n", C.POINTER(C.c_int32)), ("seq_state", C.c_void_p)]


class lq_sizes8(C.Structure):
    _fields_ = [(n, C.c_size_t) for n in ("codes", "scale", "tail", "seq_state", "workspace")]


class lq_rope(C.Structure):
    _fields_ = [("dims", C.c_int32), ("interleaved", C.c_int32), ("factor", C.c_float), ("freq", C.c_void_p)]


class lq_scores(C.Structure):
    _fields_ = [("softcap", C.c_float), ("window", C.c_int32), ("slopes", C.c_void_p)]


class lq_config_paged(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("B", "Hq", "Hkv", "d", "page", "dtype", "n_pages", "max_pages", "weighted")]


class lq_cache_paged(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k_pages", "v_pages", "table", "weights")] + [
        (n, C.POINTER(C.c_int32)) for n in ("n", "cur", "pages")] + [("seq_state", C.c_void_p)]


class lq_sizes_paged(C.Structure):
    _fields_ = [(n, C.c_size_t) for n in ("pages", "table", "weights", "seq_state", "workspace")]


class lq_plan(C.Structure):
    _fields_ = [("blocks", C.c_int32), ("waves_per_block", C.c_int32), ("splits", C.c_int32),
                ("fp_waves", C.c_int32), ("bytes_read", C.c_int64)]


EXPORTS = ("logquant_sizes", "logquant_workspace_bytes", "logquant_workspace_init", "logquant_append", "logquant_compress",
           "logquant_prefill", "logquant_prefill_positions", "logquant_decode_attn", "logquant_decode_attn_static",
           "logquant_decode_step", "logquant_decode_plan",
           "logquant_seq_state_bytes", "logquant_prefill_seq", "logquant_append_seq", "logquant_compress_seq",
           "logquant_decode_attn_seq", "logquant_decode_step_seq", "logquant_decode_plan_seq",
           "logquant_sizes8", "logquant_workspace_init8", "logquant_append8", "logquant_read8",
           "logquant_decode_attn8", "logquant_decode_step8",
           "logquant_rope_frequencies", "logquant_rotate",
           "logquant_sizes_paged", "logquant_workspace_init_paged", "logquant_append_paged", "logquant_decode_attn_paged",
           "logquant_decode_step_paged", "logquant_evict_paged",
           "logquant_read_probe", "logquant_status_string")

if not os.path.exists(LIB_PATH):
    raise ImportError("liblogquant.so is not built: run `python -m paper_2503_19950_amd.build` "
                      "(there is no fallback path)")
_lib = C.CDLL(LIB_PATH)

_lib.logquant_sizes.argtypes = [C.POINTER(lq_config), C.POINTER(lq_sizes)]
_lib.logquant_sizes.restype = C.c_int
_lib.logquant_workspace_bytes.argtypes = [C.POINTER(lq_config)]
_lib.logquant_workspace_bytes.restype = C.c_size_t
_lib.logquant_workspace_init.argtypes = [C.POINTER(lq_config), C.c_void_p, C.c_void_p]
_lib.logquant_workspace_init.restype = C.c_int
_lib.logquant_append.argtypes = [C.POINTER(lq_config), C.POINTER(lq_cache), C.c_void_p, C.c_void_p,
                                 C.c_int32, C.c_void_p]
_lib.logquant_append.restype = C.c_int
_lib.logquant_compress.argtypes = [C.POINTER(lq_config), C.POINTER(lq_cache), C.c_void_p, C.c_void_p]
_lib.logquant_compress.restype = C.c_int
_lib.logquant_prefill.argtypes = [C.POINTER(lq_config), C.POINTER(lq_cache), C.c_void_p, C.c_void_p, C.c_int32,
                                  C.c_void_p]
_lib.logquant_prefill.restype = C.c_int
_lib.logquant_prefill_positions.argtypes = [C.c_int32, C.c_int32, C.POINTER(C.c_int32), C.POINTER(C.c_int32),
                                            C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
_lib.logquant_prefill_positions.restype = C.c_int
_lib.logquant_decode_attn.argtypes = [C.POINTER(lq_config), C.POINTER(lq_cache), C.c_void_p, C.c_float,
                                      C.c_void_p, C.c_void_p, C.c_void_p]
_lib.logquant_decode_attn.restype = C.c_int
_lib.logquant_decode_attn_static.argtypes = [C.POINTER(lq_config), C.POINTER(lq_cache), C.c_void_p, C.c_float,
                                             C.c_void_p, C.c_void_p]
_lib.logquant_decode_attn_static.restype = C.c_int
_lib.logquant_decode_step.argtypes = [C.POINTER(lq_config), C.POINTER(lq_cache), C.c_void_p, C.c_void_p, C.c_void_p,
                                      C.c_float, C.c_void_p, C.c_void_p, C.c_void_p]
_lib.logquant_decode_step.restype = C.c_int
_lib.logquant_decode_plan.argtypes = [C.POINTER(lq_config), C.c_int32, C.c_int32, C.POINTER(lq_plan)]
_lib.logquant_decode_plan.restype = C.c_int
_I32P = C.POINTER(C.c_int32)
_lib.logquant_seq_state_bytes.argtypes = [C.POINTER(lq_config)]
_lib.logquant_seq_state_bytes.restype = C.c_size_t
_lib.logquant_prefill_seq.argtypes = [C.POINTER(lq_config), C.POINTER(lq_cache_seq), C.c_void_p, C.c_void_p, _I32P,
                                      C.c_int32, C.c_void_p]
_lib.logquant_prefill_seq.restype = C.c_int
_lib.logquant_append_seq.argtypes = [C.POINTER(lq_config), C.POINTER(lq_cache_seq), C.c_void_p, C.c_void_p, _I32P,
                                     C.c_void_p]
_lib.logquant_append_seq.restype = C.c_int
_lib.logquant_compress_seq.argtypes = [C.POINTER(lq_config), C.POINTER(lq_cache_seq), C.c_void_p]
_lib.logquant_compress_seq.restype = C.c_int
_lib.logquant_decode_attn_seq.argtypes = [C.POINTER(lq_config), C.POINTER(lq_cache_seq), C.c_void_p, C.c_float,
                                          C.c_void_p, C.c_void_p, C.c_void_p]
_lib.logquant_decode_attn_seq.restype = C.c_int
_lib.logquant_decode_step_seq.argtypes = [C.POINTER(lq_config), C.POINTER(lq_cache_seq), C.c_void_p, C.c_void_p,
                                          C.c_void_p, C.c_float, C.c_void_p, C.c_void_p, C.c_void_p]
_lib.logquant_decode_step_seq.restype = C.c_int
_lib.logquant_decode_plan_seq.argtypes = [C.POINTER(lq_config), _I32P, _I32P, C.POINTER(lq_plan)]
_lib.logquant_decode_plan_seq.restype = C.c_int
_lib.logquant_sizes8.argtypes = [C.POINTER(lq_config8), C.POINTER(lq_sizes8)]
_lib.logquant_sizes8.restype = C.c_int
_lib.logquant_workspace_init8.argtypes = [C.POINTER(lq_config8), C.c_void_p, C.c_void_p]
_lib.logquant_workspace_init8.restype = C.c_int
_lib.logquant_append8.argtypes = [C.POINTER(lq_config8), C.POINTER(lq_cache8), C.c_void_p, C.c_void_p, _I32P, C.c_int32,
                                  C.c_void_p]
_lib.logquant_append8.restype = C.c_int
_lib.logquant_read8.argtypes = [C.POINTER(lq_config8), C.POINTER(lq_cache8), C.c_int32, C.c_int32, C.c_void_p, C.c_void_p,
                                C.c_void_p]
_lib.logquant_read8.restype = C.c_int
_lib.logquant_decode_attn8.argtypes = [C.POINTER(lq_config8), C.POINTER(lq_cache8), C.c_void_p, C.c_float, C.c_void_p,
                                       C.c_void_p, C.c_void_p]
_lib.logquant_decode_attn8.restype = C.c_int
_lib.logquant_decode_step8.argtypes = [C.POINTER(lq_config8), C.POINTER(lq_cache8), C.c_void_p, C.c_void_p, C.c_void_p,
                                       C.c_float, C.c_void_p, C.c_void_p, C.c_void_p]
_lib.logquant_decode_step8.restype = C.c_int
_ROPEP, _CFGP, _CACHEP = C.POINTER(lq_rope), C.POINTER(lq_config_paged), C.POINTER(lq_cache_paged)
_lib.logquant_rope_frequencies.argtypes = [C.c_int32] + [C.c_double] * 5 + [C.POINTER(C.c_double)]
_lib.logquant_rope_frequencies.restype = C.c_int
_lib.logquant_rotate.argtypes = [_ROPEP] + [C.c_int32] * 6 + [C.c_void_p] * 6
_lib.logquant_rotate.restype = C.c_int
_lib.logquant_sizes_paged.argtypes = [_CFGP, C.POINTER(lq_sizes_paged)]
_lib.logquant_sizes_paged.restype = C.c_int
_lib.logquant_workspace_init_paged.argtypes = [_CFGP, C.c_void_p, C.c_void_p]
_lib.logquant_workspace_init_paged.restype = C.c_int
_lib.logquant_append_paged.argtypes = [_CFGP, _CACHEP, _ROPEP, C.c_void_p, C.c_void_p, C.c_void_p, _I32P, C.c_int32, C.c_void_p]
_lib.logquant_append_paged.restype = C.c_int
_lib.logquant_decode_attn_paged.argtypes = [_CFGP, _CACHEP, C.POINTER(lq_scores), C.c_void_p, C.c_float, C.c_void_p, C.c_void_p,
                                            C.c_void_p]
_lib.logquant_decode_attn_paged.restype = C.c_int
_lib.logquant_decode_step_paged.argtypes = [_CFGP, _CACHEP, _ROPEP, C.c_void_p, C.POINTER(lq_scores), C.c_void_p, C.c_void_p,
                                            C.c_void_p, C.c_float, C.c_void_p, C.c_void_p, C.c_void_p]
_lib.logquant_decode_step_paged.restype = C.c_int
_lib.logquant_evict_paged.argtypes = [_CFGP, _CACHEP, _I32P, C.c_int32, C.c_void_p, C.c_void_p]
_lib.logquant_evict_paged.restype = C.c_int
_lib.logquant_read_probe.argtypes = [C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
_lib.logquant_read_probe.restype = C.c_int
_lib.logquant_status_string.argtypes = [C.c_int]
_lib.logquant_status_string.restype = C.c_char_p


class LogQuantError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__("%s: %s" % (where, logquant_status_string(status)))


def _ptr(x):
    """Device (or null) pointer of a torch tensor / int / None."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _p(struct):
    return C.byref(struct) if struct is not None else None


def logquant_status_string(status):
    return _lib.logquant_status_string(int(status)).decode()


def logquant_sizes(cfg):
    out = lq_sizes()
    st = _lib.logquant_sizes(_p(cfg), C.byref(out))
    if st != LQ_OK:
        raise LogQuantError(st, "logquant_sizes")
    return out


def logquant_workspace_bytes(cfg):
    return int(_lib.logquant_workspace_bytes(_p(cfg)))


def logquant_workspace_init(cfg, workspace, stream=0):
    return _lib.logquant_workspace_init(_p(cfg), _ptr(workspace), stream)


def logquant_append(cfg, cache, k_new, v_new, n_new, stream=0):
    return _lib.logquant_append(_p(cfg), _p(cache), _ptr(k_new), _ptr(v_new), int(n_new), stream)


def logquant_compress(cfg, cache, workspace=None, stream=0):
    return _lib.logquant_compress(_p(cfg), _p(cache), _ptr(workspace), stream)


def logquant_prefill(cfg, cache, k, v, L, stream=0):
    return _lib.logquant_prefill(_p(cfg), _p(cache), _ptr(k), _ptr(v), int(L), stream)


def logquant_prefill_positions(W, L):
    """-> (status, pos_fp list, pos_q list); host arithmetic only."""
    n_fp, n_q = C.c_int32(0), C.c_int32(0)
    st = _lib.logquant_prefill_positions(int(W), int(L), None, C.byref(n_fp), None, C.byref(n_q))
    if st != LQ_OK:
        return st, None, None
    a = (C.c_int32 * max(1, n_fp.value))()
    q = (C.c_int32 * max(1, n_q.value))()
    st = _lib.logquant_prefill_positions(int(W), int(L), a, C.byref(n_fp), q, C.byref(n_q))
    return st, list(a[:n_fp.value]), list(q[:n_q.value])


def logquant_decode_attn(cfg, cache, q, softmax_scale, out, workspace, stream=0):
    return _lib.logquant_decode_attn(_p(cfg), _p(cache), _ptr(q), float(softmax_scale), _ptr(out),
                                     _ptr(workspace), stream)


def logquant_decode_attn_static(cfg, cache, q, softmax_scale, out, stream=0):
    return _lib.logquant_decode_attn_static(_p(cfg), _p(cache), _ptr(q), float(softmax_scale), _ptr(out), stream)


def logquant_decode_step(cfg, cache, k_new, v_new, q, softmax_scale, out, workspace, stream=0):
    return _lib.logquant_decode_step(_p(cfg), _p(cache), _ptr(k_new), _ptr(v_new), _ptr(q), float(softmax_scale),
                                     _ptr(out), _ptr(workspace), stream)


def logquant_decode_plan(cfg, n_fp, n_q):
    out = lq_plan()
    st = _lib.logquant_decode_plan(_p(cfg), int(n_fp), int(n_q), C.byref(out))
    if st != LQ_OK:
        raise LogQuantError(st, "logquant_decode_plan")
    return out


def _i32(values):
    """Host int32 array (or null) from a Python sequence.  (ctypes by itself would take numbers modulo 2^32.)"""
    if values is None:
        return None
    try:
        values = array("i", map(int, values))
        return (C.c_int32 * len(values)).from_buffer(values or bytearray(4))
    except OverflowError:
        raise ValueError("expected 32-bit numbers") from None


def logquant_seq_state_bytes(cfg):
    return int(_lib.logquant_seq_state_bytes(_p(cfg)))


def logquant_prefill_seq(cfg, cache, k, v, L, L_stride, stream=0):
    return _lib.logquant_prefill_seq(_p(cfg), _p(cache), _ptr(k), _ptr(v), _i32(L), int(L_stride), stream)


def logquant_append_seq(cfg, cache, k_new, v_new, active=None, stream=0):
    return _lib.logquant_append_seq(_p(cfg), _p(cache), _ptr(k_new), _ptr(v_new), _i32(active), stream)


def logquant_compress_seq(cfg, cache, stream=0):
    return _lib.logquant_compress_seq(_p(cfg), _p(cache), stream)


def logquant_decode_attn_seq(cfg, cache, q, softmax_scale, out, workspace, stream=0):
    return _lib.logquant_decode_attn_seq(_p(cfg), _p(cache), _ptr(q), float(softmax_scale), _ptr(out),
                                         _ptr(workspace), stream)


def logquant_decode_step_seq(cfg, cache, k_new, v_new, q, softmax_scale, out, workspace, stream=0):
    return _lib.logquant_decode_step_seq(_p(cfg), _p(cache), _ptr(k_new), _ptr(v_new), _ptr(q),
                                         float(softmax_scale), _ptr(out), _ptr(workspace), stream)


def logquant_decode_plan_seq(cfg, n_fp, n_q):
    out = lq_plan()
    st = _lib.logquant_decode_plan_seq(_p(cfg), _i32(n_fp), _i32(n_q), C.byref(out))
    if st != LQ_OK:
        raise LogQuantError(st, "logquant_decode_plan_seq")
    return out


def logquant_read_probe(buf, nbytes, sink, stream=0):
    return _lib.logquant_read_probe(_ptr(buf), int(nbytes), _ptr(sink), stream)


def logquant_sizes8(cfg):
    out = lq_sizes8()
    st = _lib.logquant_sizes8(_p(cfg), C.byref(out))
    if st != LQ_OK:
        raise LogQuantError(st, "logquant_sizes8")
    return out


def logquant_workspace_init8(cfg, workspace, stream=0):
    return _lib.logquant_workspace_init8(_p(cfg), _ptr(workspace), stream)


def logquant_append8(cfg, cache, k_new, v_new, n_new, n_max, stream=0):
    return _lib.logquant_append8(_p(cfg), _p(cache), _ptr(k_new), _ptr(v_new), _i32(n_new), int(n_max), stream)


def logquant_read8(cfg, cache, t0, n, k_out, v_out, stream=0):
    return _lib.logquant_read8(_p(cfg), _p(cache), int(t0), int(n), _ptr(k_out), _ptr(v_out), stream)


def logquant_decode_attn8(cfg, cache, q, softmax_scale, out, workspace, stream=0):
    return _lib.logquant_decode_attn8(_p(cfg), _p(cache), _ptr(q), float(softmax_scale), _ptr(out), _ptr(workspace), stream)


def logquant_decode_step8(cfg, cache, k_new, v_new, q, softmax_scale, out, workspace, stream=0):
    return _lib.logquant_decode_step8(_p(cfg), _p(cache), _ptr(k_new), _ptr(v_new), _ptr(q), float(softmax_scale),
                                      _ptr(out), _ptr(workspace), stream)


def logquant_rope_frequencies(dims, base=10000.0, stretch=1.0, original=0.0, slow=1.0, fast=32.0):
    """-> list of dims/2 radians per position; host arithmetic only."""
    freq = (C.c_double * max(1, dims // 2))()
    st = _lib.logquant_rope_frequencies(int(dims), base, stretch, original, slow, fast, freq)
    if st != LQ_OK:
        raise LogQuantError(st, "logquant_rope_frequencies")
    return list(freq)


def logquant_rotate(rope, B, L, Hq, Hkv, d, dtype, positions, q, q_out, k, k_out, stream=0):
    return _lib.logquant_rotate(_p(rope), B, L, Hq, Hkv, d, dtype, _ptr(positions), _ptr(q), _ptr(q_out), _ptr(k), _ptr(k_out), stream)


def logquant_sizes_paged(cfg):
    out = lq_sizes_paged()
    st = _lib.logquant_sizes_paged(_p(cfg), C.byref(out))
    if st != LQ_OK:
        raise LogQuantError(st, "logquant_sizes_paged")
    return out


def logquant_workspace_init_paged(cfg, workspace, stream=0):
    return _lib.logquant_workspace_init_paged(_p(cfg), _ptr(workspace), stream)


def logquant_append_paged(cfg, cache, rope, positions, k_new, v_new, n_new, n_max, stream=0):
    return _lib.logquant_append_paged(_p(cfg), _p(cache), _p(rope), _ptr(positions), _ptr(k_new), _ptr(v_new), _i32(n_new), int(n_max),
                                      stream)


def logquant_decode_attn_paged(cfg, cache, scores, q, softmax_scale, out, workspace, stream=0):
    return _lib.logquant_decode_attn_paged(_p(cfg), _p(cache), _p(scores), _ptr(q), float(softmax_scale), _ptr(out), _ptr(workspace),
                                           stream)


def logquant_decode_step_paged(cfg, cache, rope, positions, scores, k_new, v_new, q, softmax_scale, out, workspace, stream=0):
    return _lib.logquant_decode_step_paged(_p(cfg), _p(cache), _p(rope), _ptr(positions), _p(scores), _ptr(k_new), _ptr(v_new), _ptr(q),
                                           float(softmax_scale), _ptr(out), _ptr(workspace), stream)


def logquant_evict_paged(cfg, cache, keep, recent, workspace, stream=0):
    return _lib.logquant_evict_paged(_p(cfg), _p(cache), _i32(keep), int(recent), _ptr(workspace), stream)


def torch_dtype(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float16


def to_dev(x, dtype, device="cuda:0"):
    """float32 numpy array of exact T values -> device tensor of type T."""
    import numpy as np
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).to(device).to(torch_dtype(dtype))


def make_config(B, Hq, Hkv, d, fp_budget, group, dtype, q_capacity, bits=2):
    return lq_config(B, Hq, Hkv, d, fp_budget, group, bits, LQ_BF16 if dtype == "bf16" else LQ_F16,
                     q_capacity)


def make_config8(B, Hq, Hkv, d, block, dtype, capacity):
    return lq_config8(B, Hq, Hkv, d, block, LQ_BF16 if dtype == "bf16" else LQ_F16, capacity)


def make_config_paged(B, Hq, Hkv, d, page, dtype, n_pages, max_pages, weighted=False):
    return lq_config_paged(B, Hq, Hkv, d, page, LQ_BF16 if dtype == "bf16" else LQ_F16, n_pages, max_pages, int(weighted))


class DeviceCache:
    """Owner of the device buffers of one lq_cache (torch tensors) plus the
    workspace.  Only allocation and pointer bookkeeping happen here."""

    def __init__(self, cfg, device="cuda:0", poison=False):
        import torch
        self.torch = torch
        self.cfg = cfg
        self.device = torch.device(device)
        sz = logquant_sizes(cfg)
        self.sizes = sz

        def buf(nbytes):
            t = torch.empty(max(int(nbytes), 16), dtype=torch.uint8, device=self.device)
            t.fill_(0xFF if poison else 0)   # 0xFF..: NaN patterns in fp16/bf16
            return t

        self.k_fp = [buf(sz.k_fp), buf(sz.k_fp)]
        self.v_fp = [buf(sz.v_fp), buf(sz.v_fp)]
        self.pos_fp = [buf(sz.pos_fp), buf(sz.pos_fp)]
        self.k_codes, self.v_codes = buf(sz.k_codes), buf(sz.v_codes)
        self.k_scale, self.k_zero = buf(sz.k_meta), buf(sz.k_meta)
        self.v_scale, self.v_zero = buf(sz.v_meta), buf(sz.v_meta)
        self.pos_q = buf(sz.pos_q)
        self.workspace = buf(sz.workspace)
        c = lq_cache()
        for i in range(2):
            c.k_fp[i] = self.k_fp[i].data_ptr()
            c.v_fp[i] = self.v_fp[i].data_ptr()
            c.pos_fp[i] = self.pos_fp[i].data_ptr()
        c.k_codes, c.v_codes = self.k_codes.data_ptr(), self.v_codes.data_ptr()
        c.k_scale, c.k_zero = self.k_scale.data_ptr(), self.k_zero.data_ptr()
        c.v_scale, c.v_zero = self.v_scale.data_ptr(), self.v_zero.data_ptr()
        c.pos_q = self.pos_q.data_ptr()
        c.cur = c.n_fp = c.n_q = 0
        self.c = c
        self._check(logquant_workspace_init(cfg, self.workspace, self._stream()), "logquant_workspace_init")

    BUFFERS = ("k_codes", "v_codes", "k_scale", "k_zero", "v_scale", "v_zero", "pos_q")

    def clone(self):
        """A second cache with its own device buffers and the same contents/counts."""
        other = DeviceCache(self.cfg, device=self.device)
        for i in range(2):
            other.k_fp[i].copy_(self.k_fp[i])
            other.v_fp[i].copy_(self.v_fp[i])
            other.pos_fp[i].copy_(self.pos_fp[i])
        for name in self.BUFFERS:
            getattr(other, name).copy_(getattr(self, name))
        other.c.cur, other.c.n_fp, other.c.n_q = self.c.cur, self.c.n_fp, self.c.n_q
        return other

    def counts(self):
        return (self.c.cur, self.c.n_fp, self.c.n_q)

    def set_counts(self, counts):
        """Rewind the host-side counts (the device buffers are left as they are)."""
        self.c.cur, self.c.n_fp, self.c.n_q = counts

    @property
    def W(self):
        return self.cfg.fp_budget // 2

    def _stream(self):
        # the current stream's handle alone: as an attribute of a torch.cuda.Stream made for the purpose it was 1.9 of the
        # 7.3 us of a call.  A device of another type is refused, as by current_stream: its addresses are not the GPU's
        if self.device.type != "cuda":
            raise ValueError("Expected a cuda device, but got: %s" % self.device)
        i = self.device.index
        return self.torch._C._cuda_getCurrentRawStream(self.torch.cuda.current_device() if i is None else i)

    def _check(self, st, where):
        if st != LQ_OK:
            raise LogQuantError(st, where)

    def append(self, k_new, v_new):
        """k_new, v_new: [B][Hkv][n][d] tensors of the cache dtype, contiguous."""
        n = k_new.shape[2]
        assert k_new.is_contiguous() and v_new.is_contiguous()
        self._check(logquant_append(self.cfg, self.c, k_new, v_new, n, self._stream()), "logquant_append")

    def compress(self):
        self._check(logquant_compress(self.cfg, self.c, self.workspace, self._stream()), "logquant_compress")

    def prefill(self, K, V):
        """K, V: [B][Hkv][L][d] tensors of the cache dtype, contiguous; the cache must be empty."""
        assert K.is_contiguous() and V.is_contiguous()
        self._check(logquant_prefill(self.cfg, self.c, K, V, K.shape[2], self._stream()), "logquant_prefill")

    def stream_in(self, K, V):
        """Append [B][Hkv][n][d] rows with the eager trigger: compress whenever the
        fp region reaches 3W rows.  Returns the number of compress events."""
        n, i, ev, cap = K.shape[2], 0, 0, 3 * self.W
        while i < n:
            m = min(cap - self.c.n_fp, n - i)
            self.append(K[:, :, i:i + m].contiguous(), V[:, :, i:i + m].contiguous())
            i += m
            if self.c.n_fp == cap:
                self.compress()
                ev += 1
        return ev

    def decode_step(self, k_new, v_new, q, out=None, softmax_scale=0.0):
        """Append one token ([B][Hkv][1][d]) and attend, in one launch."""
        if out is None:
            out = self.torch.empty_like(q)
        assert k_new.is_contiguous() and v_new.is_contiguous()
        self._check(logquant_decode_step(self.cfg, self.c, k_new, v_new, q, softmax_scale, out, self.workspace,
                                         self._stream()), "logquant_decode_step")
        return out

    def decode_attn(self, q, out=None, softmax_scale=0.0):
        if out is None:
            out = self.torch.empty_like(q)
        self._check(logquant_decode_attn(self.cfg, self.c, q, softmax_scale, out, self.workspace,
                                         self._stream()), "logquant_decode_attn")
        return out


class DeviceCacheSeq(DeviceCache):
    """The same device buffers with per-sequence counts (lq_cache_seq): host arrays of B
    entries for cur / n_fp / n_q and the device scratch the calls pass them through."""

    def __init__(self, cfg, device="cuda:0", poison=False):
        super().__init__(cfg, device, poison)
        B = cfg.B
        self.cur, self.n_fp, self.n_q = ((C.c_int32 * B)() for _ in range(3))
        self.seq_state = self.torch.zeros(max(logquant_seq_state_bytes(cfg), 16), dtype=self.torch.uint8,
                                          device=self.device)
        cs = lq_cache_seq()
        for name, _ in lq_cache._fields_[:10]:
            setattr(cs, name, getattr(self.c, name))
        cs.cur = C.cast(self.cur, _I32P)
        cs.n_fp = C.cast(self.n_fp, _I32P)
        cs.n_q = C.cast(self.n_q, _I32P)
        cs.seq_state = self.seq_state.data_ptr()
        self.cs = cs

    def prefill_seq(self, K, V, L):
        assert K.is_contiguous() and V.is_contiguous()
        self._check(logquant_prefill_seq(self.cfg, self.cs, K, V, L, K.shape[2], self._stream()), "logquant_prefill_seq")

    def append_seq(self, k_new, v_new, active=None):
        assert k_new.is_contiguous() and v_new.is_contiguous()
        self._check(logquant_append_seq(self.cfg, self.cs, k_new, v_new, active, self._stream()), "logquant_append_seq")

    def compress_seq(self):
        self._check(logquant_compress_seq(self.cfg, self.cs, self._stream()), "logquant_compress_seq")

    def decode_attn_seq(self, q, out=None, softmax_scale=0.0):
        if out is None:
            out = self.torch.empty_like(q)
        self._check(logquant_decode_attn_seq(self.cfg, self.cs, q, softmax_scale, out, self.workspace,
                                             self._stream()), "logquant_decode_attn_seq")
        return out

    def decode_step_seq(self, k_new, v_new, q, out=None, softmax_scale=0.0):
        if out is None:
            out = self.torch.empty_like(q)
        assert k_new.is_contiguous() and v_new.is_contiguous()
        self._check(logquant_decode_step_seq(self.cfg, self.cs, k_new, v_new, q, softmax_scale, out, self.workspace,
                                             self._stream()), "logquant_decode_step_seq")
        return out

    def view(self, b):
        """Counts of sequence b as a (cur, n_fp, n_q) triple."""
        return (self.cur[b], self.n_fp[b], self.n_q[b])


class DeviceCache8:
    """Owner of the device buffers of one lq_cache8 (torch tensors), its counts and the workspace.  Tensors are refused
    (ValueError) unless they are of the cache's type, shape and device and contiguous.  A call goes to the current stream
    of the cache's device, whichever device is current."""

    BUFFERS = ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail")

    def __init__(self, cfg, device="cuda:0", poison=False):
        self.cfg = cfg
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError("Expected a cuda device, but got: %s" % self.device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.dtype = torch_dtype("bf16" if cfg.dtype == LQ_BF16 else "f16")
        self.sizes = logquant_sizes8(cfg)

        def buf(nbytes):
            return torch.full((int(nbytes),), 0xFF if poison else 0, dtype=torch.uint8, device=self.device)

        for name in self.BUFFERS:
            setattr(self, name, buf(getattr(self.sizes, name[2:])))
        self.seq_state, self.workspace = buf(self.sizes.seq_state), buf(self.sizes.workspace)
        self.n = (C.c_int32 * cfg.B)()
        self.c = lq_cache8(*[getattr(self, name).data_ptr() for name in self.BUFFERS], C.cast(self.n, _I32P),
                           self.seq_state.data_ptr())
        # what every call takes, made once (a decode call's host time 6.5 -> 5.1 us)
        self._index = self.device.index
        self._cfg, self._c, self._ws = C.byref(cfg), C.byref(self.c), self.workspace.data_ptr()
        self._q_shape, self._token = torch.Size((cfg.B, cfg.Hq, cfg.d)), torch.Size((cfg.B, cfg.Hkv, 1, cfg.d))
        self._call("logquant_workspace_init8", self._ws)

    def _call(self, name, *args):
        i = self._index
        f = getattr(_lib, name)
        if torch._C._cuda_getDevice() == i:
            st = f(self._cfg, *args, torch._C._cuda_getCurrentRawStream(i))
        else:
            with torch.cuda.device(i):
                st = f(self._cfg, *args, torch._C._cuda_getCurrentRawStream(i))
        if st != LQ_OK:
            raise LogQuantError(st, name)

    def _address(self, name, t, shape):
        if t.shape != shape or t.dtype is not self.dtype or t.get_device() != self._index or not t.is_contiguous():
            raise ValueError("%s: expected a contiguous %s tensor of shape %s on %s" % (name, self.dtype, tuple(shape), self.device))
        return t.data_ptr()

    def clone(self):
        """A second cache with its own device buffers and the same contents and counts."""
        other = DeviceCache8(self.cfg, self.device)
        for name in self.BUFFERS:
            getattr(other, name).copy_(getattr(self, name))
        other.set_counts(self.counts())
        return other

    def counts(self):
        return list(self.n)

    def set_counts(self, counts):
        """Set the host-side counts (the device buffers are left as they are)."""
        self.n[:] = counts

    def append(self, k_new, v_new, n_new=None):
        """k_new, v_new: [B][Hkv][n][d]; n_new: tokens that each row takes of them, 0..n (None: all)."""
        c = self.cfg
        n = k_new.shape[2] if k_new.dim() == 4 else 1
        shape = self._token if n == 1 else torch.Size((c.B, c.Hkv, n, c.d))
        k, v = self._address("k_new", k_new, shape), self._address("v_new", v_new, shape)
        if n_new is not None and len(n_new) != c.B:
            raise ValueError("n_new: expected %d counts" % c.B)
        self._call("logquant_append8", self._c, k, v, _i32(n_new), n)

    def read(self, t0, n, k_out=None, v_out=None):
        """Tokens t0 .. t0+n-1 as ([B][Hkv][n][d], [B][Hkv][n][d]) tensors of the cache type: the given ones, whose rows
        behind a sequence are left as they were, or new ones with zeros there."""
        c = self.cfg
        if n < 1 or t0 < 0 or t0 + n > c.capacity:       # (before room for it is made)
            raise LogQuantError(LQ_ERR_SHAPE, "logquant_read8")
        shape = torch.Size((c.B, c.Hkv, n, c.d))
        k_out, v_out = (torch.zeros(shape, dtype=self.dtype, device=self.device) if t is None else t for t in (k_out, v_out))
        self._call("logquant_read8", self._c, t0, n, self._address("k_out", k_out, shape), self._address("v_out", v_out, shape))
        return k_out, v_out

    def decode_attn(self, q, out=None, softmax_scale=0.0):
        """q: [B][Hq][d]; rows of the batch that hold no token give zeros."""
        if out is None:
            out = torch.empty_like(q)
        self._call("logquant_decode_attn8", self._c, self._address("q", q, self._q_shape), softmax_scale,
                   self._address("out", out, self._q_shape), self._ws)
        return out

    def decode_step(self, k_new, v_new, q, out=None, softmax_scale=0.0):
        """Append one token per row ([B][Hkv][1][d]) and attend."""
        if out is None:
            out = torch.empty_like(q)
        self._call("logquant_decode_step8", self._c, self._address("k_new", k_new, self._token), self._address("v_new", v_new, self._token),
                   self._address("q", q, self._q_shape), softmax_scale, self._address("out", out, self._q_shape), self._ws)
        return out


def _cuda(device):
    device = torch.device(device)
    if device.type != "cuda":
        raise ValueError("Expected a cuda device, but got: %s" % device)
    return torch.device("cuda", torch.cuda.current_device()) if device.index is None else device


def _tensor(name, t, shape, dtype, device):
    """Address of a tensor that is what a call takes."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device.index or not t.is_contiguous():
        raise ValueError("%s: expected a contiguous %s tensor of shape %s on %s" % (name, dtype, tuple(shape), device))
    return t.data_ptr()


def _on_device(index, f, *args):
    """An entry point on the current stream of device `index`, whichever device is current."""
    if torch._C._cuda_getDevice() == index:
        st = f(*args, torch._C._cuda_getCurrentRawStream(index))
    else:
        with torch.cuda.device(index):
            st = f(*args, torch._C._cuda_getCurrentRawStream(index))
    if st != LQ_OK:
        raise LogQuantError(st, f.__name__)


_rotate, _init_paged, _append_paged = _lib.logquant_rotate, _lib.logquant_workspace_init_paged, _lib.logquant_append_paged
_attn_paged, _step_paged, _evict_paged = _lib.logquant_decode_attn_paged, _lib.logquant_decode_step_paged, _lib.logquant_evict_paged


class Rope:
    """Rotary positions: frequencies (radians per position of every pair, as logquant_rope_frequencies gives them) on a
    device, which pairs they turn, and a factor on what is turned."""

    def __init__(self, freq, interleaved=False, factor=1.0, device="cuda:0"):
        self.device = _cuda(device)
        self.freq = torch.as_tensor(freq, dtype=torch.float64).to(self.device).contiguous()
        if self.freq.dim() != 1 or not len(self.freq):
            raise ValueError("freq: expected one frequency for every pair")
        self.index = self.device.index
        self.c = lq_rope(2 * len(self.freq), int(interleaved), factor, self.freq.data_ptr())
        self._c = C.byref(self.c)


def rotate(rope, positions=None, q=None, k=None, q_out=None, k_out=None):
    """q [B][Hq][L][d], or [B][Hq][d] for L = 1, and k [B][Hkv][L][d], either may be None, turned by positions ([B][L] int32,
    or [B]; None: 0 .. L-1): into the given tensors, which may be q and k themselves, or new ones.  -> (q_out, k_out).
    The call goes to the current stream of the rope's device."""
    x = q if q is not None else k
    if x is None:
        raise ValueError("rotate: no tensor")
    dtype, shape, device = x.dtype, x.shape, rope.device
    B, L, d = shape[0], shape[2] if len(shape) == 4 else 1, shape[-1]
    if len(shape) not in (3, 4) or (dtype is not torch.bfloat16 and dtype is not torch.float16):
        raise ValueError("rotate: expected fp16 or bf16 tensors of shape [B][H][L][d] or [B][H][d]")
    Hq = Hkv = 0
    at_q = at_q_out = at_k = at_k_out = at = None
    if q is not None:
        Hq = shape[1]
        at_q = _tensor("q", q, shape, dtype, device)
        if q_out is None:
            q_out = torch.empty_like(q)
        at_q_out = at_q if q_out is q else _tensor("q_out", q_out, shape, dtype, device)
    elif q_out is not None:
        raise ValueError("q_out without q")
    if k is not None:
        shape = k.shape
        if len(shape) not in (3, 4) or shape[0] != B or shape[-1] != d or (shape[2] if len(shape) == 4 else 1) != L:
            raise ValueError("k: expected [%d][Hkv][%d][%d]" % (B, L, d))
        Hkv = shape[1]
        at_k = _tensor("k", k, shape, dtype, device)
        if k_out is None:
            k_out = torch.empty_like(k)
        at_k_out = at_k if k_out is k else _tensor("k_out", k_out, shape, dtype, device)
    elif k_out is not None:
        raise ValueError("k_out without k")
    if positions is not None:
        at = _tensor("positions", positions, (B,) if L == 1 and positions.dim() == 1 else (B, L), torch.int32, device)
    _on_device(rope.index, _rotate, rope._c, B, L, Hq, Hkv, d, LQ_BF16 if dtype is torch.bfloat16 else LQ_F16, at, at_q, at_q_out, at_k,
               at_k_out)
    return q_out, k_out


class DeviceCachePaged:
    """Owner of the device buffers of one lq_cache_paged (torch tensors), its counts, tables and workspace, and of the pool's
    free pages.  Tensors are refused (ValueError) unless they are of the cache's type, shape and device and contiguous.  A call
    goes to the current stream of the cache's device, whichever device is current."""

    BUFFERS = ("k_pages", "v_pages", "table", "weights")
    INT_MAX = 2 ** 31 - 1                                         # more tokens than any row can have

    def __init__(self, cfg, device="cuda:0", poison=False):
        self.cfg = cfg
        self.device = _cuda(device)
        self.dtype = torch_dtype("bf16" if cfg.dtype == LQ_BF16 else "f16")
        self.sizes = logquant_sizes_paged(cfg)
        B = cfg.B

        def buf(nbytes):
            return torch.full((int(nbytes),), 0xFF if poison else 0, dtype=torch.uint8, device=self.device)

        self.k_pages, self.v_pages = buf(self.sizes.pages), buf(self.sizes.pages)
        self.table = torch.full((2, B, cfg.max_pages), -1, dtype=torch.int32, device=self.device)
        self.weights = buf(self.sizes.weights).view(torch.float32).view(2, B, cfg.Hkv, -1) if cfg.weighted else None
        self.seq_state, self.workspace = buf(self.sizes.seq_state), buf(self.sizes.workspace)
        self.n, self.cur, self.pages = (C.c_int32 * B)(), (C.c_int32 * B)(), (C.c_int32 * (2 * B))()
        self._at_n, self._at_cur = (memoryview(x).cast("B").cast("i") for x in (self.n, self.cur))
        self.ids = [[[] for _ in range(B)] for _ in range(2)]     # pages that the table names, by half and row
        self.free, self.uses = dict.fromkeys(range(cfg.n_pages - 1, -1, -1)), [0] * cfg.n_pages
        self.shared = 0                                           # pages that are named more than once
        self.gaps = set()                                         # halves of rows, half * B + row, that were evicted into
        self.c = lq_cache_paged(self.k_pages.data_ptr(), self.v_pages.data_ptr(), self.table.data_ptr(),
                                self.weights.data_ptr() if cfg.weighted else None, *(C.cast(x, _I32P) for x in (self.n, self.cur, self.pages)),
                                self.seq_state.data_ptr())
        # what every call takes, made once
        self._index = self.device.index
        self._cfg, self._c, self._ws = C.byref(cfg), C.byref(self.c), self.workspace.data_ptr()
        self._q_shape, self._token = torch.Size((B, cfg.Hq, cfg.d)), torch.Size((B, cfg.Hkv, 1, cfg.d))
        _on_device(self._index, _init_paged, self._cfg, self._ws)

    def clone(self):
        """A second cache with its own device buffers and the same contents, pages and counts."""
        other = DeviceCachePaged(self.cfg, self.device)
        for name in self.BUFFERS:
            if getattr(self, name) is not None:
                getattr(other, name).copy_(getattr(self, name))
        other.ids, other.uses, other.free = [[list(x) for x in half] for half in self.ids], list(self.uses), dict(self.free)
        other.shared = self.shared
        other.pages[:] = list(self.pages)
        other.set_counts(self.counts(), list(self.cur))
        other.gaps = set(self.gaps)
        return other

    # ---- pages
    def _name(self, half, b, ids, first):
        """The pages of a row's half are now `ids`, of which those before the first-th were its own.  -> what that makes of
        the table: places and pages."""
        before, self.ids[half][b] = self.ids[half][b], ids
        uses = self.uses
        for i in ids[first:]:
            uses[i] += 1
            if uses[i] == 1:
                self.free.pop(i, None)
            elif uses[i] == 2:
                self.shared += 1
        for i in before[first:]:
            uses[i] -= 1
            if not uses[i]:
                self.free[i] = None
            elif uses[i] == 1:
                self.shared -= 1
        row = half * self.cfg.B + b
        self.pages[row] = len(ids)
        if not ids:
            self.gaps.discard(row)
        at = row * self.cfg.max_pages
        return range(at + first, at + len(ids)), ids[first:]

    def _half(self, call, b, spare):
        """Which half of the table a row's pages, or its spare ones, are in."""
        if not 0 <= b < self.cfg.B:
            raise ValueError("%s: expected a row in 0 .. %d" % (call, self.cfg.B - 1))
        return self.cur[b] ^ int(bool(spare))

    def _no_recording(self, call):
        """Pages are named from the host, which a graph cannot record."""
        with torch.cuda.device(self.device):
            if torch.cuda.is_current_stream_capturing():
                raise LogQuantError(LQ_ERR_STATE, call)

    def _upload(self, names):
        places = [i for at, _ in names for i in at]
        if places:
            both = torch.tensor([places, [i for _, ids in names for i in ids]]).to(self.device)
            self.table.view(-1)[both[0]] = both[1].int()

    def set_pages(self, b, ids, spare=False):
        """The pages of row b's tokens, in order (`spare`: those that its next eviction moves to, which nothing else may
        name).  Pages that were named there before, and by nothing else, go back to the pool.  A row's spare pages, those that
        an eviction left among them, are refused unless some row still reads them."""
        self._no_recording("set_pages")
        ids = [int(i) for i in ids]
        if len(ids) > self.cfg.max_pages or any(not 0 <= i < self.cfg.n_pages for i in ids):
            raise ValueError("set_pages: expected up to %d pages in 0 .. %d" % (self.cfg.max_pages, self.cfg.n_pages - 1))
        half = self._half("set_pages", b, spare)
        if not spare and len(ids) * self.cfg.page < self.n[b]:
            raise ValueError("set_pages: row %d holds %d tokens" % (b, self.n[b]))
        if spare:
            mine = set(self.ids[half][b])
            if len(set(ids)) < len(ids) or any(self.uses[i] > (i in mine) for i in ids):
                raise ValueError("set_pages: a spare page is one that nothing else names")
        else:
            rows = range(self.cfg.B)
            left = set(ids).intersection(i for row in rows for i in self.ids[self.cur[row] ^ 1][row])
            if left and not left <= {i for row in rows for i in self.ids[self.cur[row]][row]}:
                raise ValueError("set_pages: a row's spare page is not another's (release(row, spare=True) gives it back)")
        self._upload([self._name(half, b, ids, 0)])

    def reserve(self, counts, spare=False):
        """Pages out of the pool for counts[b] tokens of every row (`spare`: for its next eviction).  LogQuantError
        (LQ_ERR_CAPACITY) if the pool or a row's table has too few, or (LQ_ERR_STATE) if any are to be taken while a graph is
        recorded; nothing is taken then."""
        if len(counts) != self.cfg.B:
            raise ValueError("reserve: expected %d counts" % self.cfg.B)
        self._take("reserve", [(b, int(count)) for b, count in enumerate(counts) if count > 0], spare)

    def _take(self, call, counts, spare):
        """reserve for the rows of `counts`, [(row, tokens)].  Spare pages that an eviction left and that another row names as
        well are given back first."""
        page, most, uses = self.cfg.page, self.cfg.max_pages, self.uses
        cur, other = self.cur[:], int(bool(spare))
        back, more, total = {}, [], 0                                    # back: spare pages that are given back, by row
        for b, count in counts:
            half = cur[b] ^ other
            ids = self.ids[half][b]
            need = -(-count // page)
            if need > most:
                raise LogQuantError(LQ_ERR_CAPACITY, call)
            if spare and self.shared and any(uses[i] > 1 for i in ids):
                back[b] = ids
            else:
                need -= len(ids)
            if need > 0:
                more.append((half, b, need))
                total += need
        room = len(self.free)
        if back:
            named = collections.Counter(i for ids in back.values() for i in ids)
            room += sum(uses[i] == times for i, times in named.items())
        if total > room:
            raise LogQuantError(LQ_ERR_CAPACITY, call)
        if more:
            self._no_recording(call)
        for b in back:
            self.release(b, spare=True)
        names = []
        for half, b, need in more:
            ids = self.ids[half][b]
            names.append(self._name(half, b, ids + [self.free.popitem()[0] for _ in range(need)], len(ids)))
        self._upload(names)

    def release(self, b, spare=False):
        """Row b gives its pages back and is empty (`spare`: gives back those that it has for its next eviction, or had
        before its last)."""
        half = self._half("release", b, spare)
        if not spare:
            self.n[b] = 0
        self._name(half, b, [], 0)

    # ---- counts
    def counts(self):
        return list(self.n)

    def set_counts(self, counts, cur=None):
        """Set the host-side counts (the device buffers are left as they are), and, where given, which half is every row's.  A
        row of 0 tokens begins anew."""
        try:                                                      # (ctypes by itself would take numbers modulo 2^32)
            counts = array("i", counts)
            if cur is not None:
                cur = array("i", cur)
                if len(counts) != self.cfg.B:
                    raise ValueError("set_counts: expected %d counts" % self.cfg.B)
                self._at_cur[:] = cur
            self._at_n[:] = counts
        except OverflowError:
            raise ValueError("set_counts: expected 32-bit numbers") from None
        if self.gaps:
            self.gaps.difference_update([self.cur[b] * self.cfg.B + b for b, n in enumerate(self.n) if not n])

    # ---- calls
    def _turn(self, rope, positions, n, n_new=None):
        if rope is None:
            if positions is not None:
                raise ValueError("positions without a rope")
            return None, None
        if rope.index != self._index:
            raise ValueError("rope: expected it on %s" % self.device)
        if positions is None:
            if self.gaps:
                for b in range(self.cfg.B):
                    if self.cur[b] * self.cfg.B + b in self.gaps and (n_new is None or n_new[b]):
                        raise ValueError("positions: row %d was evicted from, its tokens' places are not their positions" % b)
            return rope._c, None
        shape = (self.cfg.B,) if n == 1 and positions.dim() == 1 else (self.cfg.B, n)
        return rope._c, _tensor("positions", positions, shape, torch.int32, self.device)

    def _how(self, softcap, window, slopes):
        if not softcap and not window and slopes is None:
            return None
        at = None if slopes is None else _tensor("slopes", slopes, (self.cfg.Hq,), torch.float32, self.device)
        return C.byref(lq_scores(softcap, max(-1, min(window, self.INT_MAX)), at))

    def append(self, k_new, v_new, n_new=None, rope=None, positions=None):
        """k_new, v_new: [B][Hkv][n][d]; n_new: tokens that each row takes of them, 0..n (None: all).  With a rope, keys are
        turned by positions ([B][n] int32; None: the places of the tokens, refused for a row that was evicted from and takes
        any)."""
        c = self.cfg
        n = k_new.shape[2] if k_new.dim() == 4 else 1
        shape = self._token if n == 1 else torch.Size((c.B, c.Hkv, n, c.d))
        k, v = _tensor("k_new", k_new, shape, self.dtype, self.device), _tensor("v_new", v_new, shape, self.dtype, self.device)
        if n_new is not None and len(n_new) != c.B:
            raise ValueError("n_new: expected %d counts" % c.B)
        turn, at = self._turn(rope, positions, n, n_new)
        _on_device(self._index, _append_paged, self._cfg, self._c, turn, at, k, v, _i32(n_new), n)

    def decode_attn(self, q, out=None, softmax_scale=0.0, softcap=0.0, window=0, slopes=None):
        """q: [B][Hq][d]; rows of the batch that hold no token give zeros.  slopes: [Hq] fp32."""
        if out is None:
            out = torch.empty_like(q)
        _on_device(self._index, _attn_paged, self._cfg, self._c, self._how(softcap, window, slopes),
                   _tensor("q", q, self._q_shape, self.dtype, self.device), softmax_scale,
                   _tensor("out", out, self._q_shape, self.dtype, self.device), self._ws)
        return out

    def decode_step(self, k_new, v_new, q, out=None, softmax_scale=0.0, rope=None, positions=None, softcap=0.0, window=0, slopes=None):
        """Append one token per row ([B][Hkv][1][d]) and attend; with a rope, its key and the query are turned by positions
        ([B] int32; None: the places of the tokens, refused after an eviction)."""
        if out is None:
            out = torch.empty_like(q)
        turn, at = self._turn(rope, positions, 1)
        _on_device(self._index, _step_paged, self._cfg, self._c, turn, at, self._how(softcap, window, slopes),
                   _tensor("k_new", k_new, self._token, self.dtype, self.device), _tensor("v_new", v_new, self._token, self.dtype, self.device),
                   _tensor("q", q, self._q_shape, self.dtype, self.device), softmax_scale,
                   _tensor("out", out, self._q_shape, self.dtype, self.device), self._ws)
        return out

    def evict(self, keep, recent=0):
        """Rows with more than `keep` tokens (a number, or one for every row) keep the newest `recent` and the heaviest
        others, in pages that are taken from the pool if the row has too few spare ones.  The pages that it leaves are its
        spare ones (`release(b, spare=True)` gives them back).  A call that is refused (counts, a pool without room, pages to
        be taken while a graph is recorded) changes nothing."""
        B, n = self.cfg.B, self.n[:]
        keep = [int(keep)] * B if isinstance(keep, int) else [int(x) for x in keep]
        if len(keep) != B:
            raise ValueError("keep: expected %d counts" % B)
        recent = int(recent)
        # what the call refuses is refused before pages are taken: with every row's count to keep it only checks
        _on_device(self._index, _evict_paged, self._cfg, self._c, self.n, max(-1, min(recent, self.INT_MAX)), self._ws)
        if max(keep) > self.INT_MAX:
            keep = [min(x, self.INT_MAX) for x in keep]
        lose = [(b, x) for b, x in enumerate(keep) if n[b] > x]
        if min(keep) < 0 or any([recent > x for _, x in lose]):
            raise LogQuantError(LQ_ERR_SHAPE, _evict_paged.__name__)
        if not lose:
            return
        self._take("evict", lose, True)
        _on_device(self._index, _evict_paged, self._cfg, self._c, _i32(keep), recent, self._ws)
        cur = self.cur[:]
        self.gaps.update([cur[b] * B + b for b, _ in lose])
