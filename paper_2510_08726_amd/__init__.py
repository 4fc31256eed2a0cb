"""Fused attention for AMD Instinct MI355X (gfx950) — Python binding of libattn.so.

A thin layer over the C ABI declared in ``include/*.h``: the functions
below have the same names as the C entry points and only marshal arguments
(device pointers, sizes, the current HIP stream).  Every step of the
computation runs in the HIP kernels of ``libattn.so``; PyTorch only provides
device memory and streams.  There is no fallback: if the library is missing
or a call fails, an exception is raised.

A plainly valid call on the current stream is marshalled in C++
(``csrc/binding.cpp``, the ``_binding`` module), whose functions return None
for anything else: the call then goes through the checks below, which raise
the errors, and ctypes.
"""

import ctypes
import math
import os

import torch

__all__ = [
    "attn_fwd", "attn_fwd_mod", "attn_decode", "attn_decode_mod", "attn_decode_workspace_bytes",
    "attn_decode_num_splits", "attn_decode_noalloc", "peaks_hbm_read", "peaks_mfma", "peaks_mfma_waves",
    "peaks_mfma_operand_bytes", "norm_chunks", "norm_kernels", "norm_workspace_bytes", "norm_l2", "rmsnorm_rowmax", "attn_fwd_kernels", "attn_fwd_call_kernels",
    "attn_decode_kernels",
    "rope_frequencies", "rope_fwd", "rope_bwd", "kv4_page_bytes", "kv_slots", "kv4_append", "kv4_load",
    "attn_decode_kv4", "attn_decode_kv4_workspace_bytes",
    "attn_fwd_lse", "attn_bwd", "attn_bwd_workspace_bytes",
    "rmsnorm_add", "rmsnorm_add_quant", "quant8_load", "rmsnorm_add_bwd", "rmsnorm_add_bwd_workspace_bytes",
    "attn_status_string", "attn_last_hip_error", "library_path", "load_library", "AttnError",
    "ATTN_OK", "ATTN_ERR_NULL", "ATTN_ERR_SHAPE", "ATTN_ERR_UNSUPPORTED", "ATTN_ERR_WORKSPACE",
    "ATTN_ERR_HIP",
]

ATTN_OK = 0
ATTN_ERR_NULL = -1
ATTN_ERR_SHAPE = -2
ATTN_ERR_UNSUPPORTED = -3
ATTN_ERR_WORKSPACE = -4
ATTN_ERR_HIP = -5

ATTN_F16 = 0
ATTN_BF16 = 1
_DTYPE_CODE = {torch.float16: ATTN_F16, torch.bfloat16: ATTN_BF16}

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None
_BINDING = None


class AttnError(RuntimeError):
    """A call into libattn.so returned an error status."""

    def __init__(self, status, msg):
        super().__init__(msg)
        self.status = status


def library_path():
    return os.path.join(_HERE, "libattn.so")


def load_library():
    """Load (once) and return the ctypes handle of libattn.so; raises if absent."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = library_path()
    if not os.path.exists(path):
        raise RuntimeError(
            f"{path} is not built; run `python -c 'import __graft_entry__ as g; g.build()'` "
            "or `python paper_2510_08726_amd/build.py` first")
    lib = ctypes.CDLL(path)
    vp, ci, cf, cs = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
    lib.attn_fwd.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, cf, vp, ci, vp]
    lib.attn_fwd.restype = ci
    lib.attn_fwd_mod.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, cf, vp, cf, ci, ci, vp]
    lib.attn_fwd_mod.restype = ci
    lib.attn_fwd_split.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, cf, vp, cf, ci, vp, cs, ci, vp]
    lib.attn_fwd_split.restype = ci
    lib.attn_fwd_num_splits.argtypes = [ci, ci, ci, ci, ci, ci, ci, ci]
    lib.attn_fwd_num_splits.restype = ci
    lib.attn_fwd_workspace_bytes.argtypes = [ci, ci, ci, ci, ci]
    lib.attn_fwd_workspace_bytes.restype = cs
    lib.attn_decode.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, ci, cf, vp, ci, vp, cs, ci, vp]
    lib.attn_decode.restype = ci
    lib.attn_decode_mod.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, ci, cf, vp, cf, ci, vp, cs, ci, vp]
    lib.attn_decode_mod.restype = ci
    lib.attn_decode_workspace_bytes.argtypes = [ci, ci, ci, ci]
    lib.attn_decode_workspace_bytes.restype = cs
    lib.attn_decode_num_splits.argtypes = [ci, ci, ci, ci, ci]
    lib.attn_decode_num_splits.restype = ci
    lib.attn_decode_noalloc.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, ci, cf, vp, cf, ci, ci, vp]
    lib.attn_decode_noalloc.restype = ci
    lib.attn_fwd_kernels.argtypes = [ci, ci, ci, ci, cf, ci, ctypes.c_char_p, cs]
    lib.attn_fwd_kernels.restype = ci
    lib.attn_fwd_call_kernels.argtypes = [ci, ci, ci, ci, ci, ci, ci, ci, ci, cf, ci, ci, ctypes.c_char_p, cs]
    lib.attn_fwd_call_kernels.restype = ci
    lib.attn_decode_kernels.argtypes = [ci, ci, ci, ci, ci, cf, ctypes.c_char_p, cs]
    lib.attn_decode_kernels.restype = ci
    lib.norm_kernels.argtypes = [ci, ci, ci, ci, ctypes.c_char_p, cs]
    lib.norm_kernels.restype = ci
    lib.peaks_hbm_read.argtypes = [vp, cs, vp, vp]
    lib.peaks_hbm_read.restype = ci
    lib.peaks_hbm_read_sink_floats.argtypes = []
    lib.peaks_hbm_read_sink_floats.restype = ci
    lib.peaks_mfma.argtypes = [ci, ci, vp, vp, vp, vp]
    lib.peaks_mfma.restype = ci
    lib.peaks_mfma_waves.argtypes = []
    lib.peaks_mfma_waves.restype = ci
    lib.peaks_mfma_operand_bytes.argtypes = []
    lib.peaks_mfma_operand_bytes.restype = cs
    lib.norm_chunks.argtypes = [ci, ci, ci, ci]
    lib.norm_chunks.restype = ci
    lib.norm_workspace_bytes.argtypes = [ci, ci]
    lib.norm_workspace_bytes.restype = cs
    lib.norm_l2.argtypes = [vp, vp, ci, ci, ci, ci, vp, cs, vp]
    lib.norm_l2.restype = ci
    lib.rmsnorm_rowmax.argtypes = [vp, vp, vp, ci, ci, cf, ci, ci, vp, cs, vp]
    lib.rmsnorm_rowmax.restype = ci
    cd, cl = ctypes.c_double, ctypes.c_longlong
    lib.rope_frequencies.argtypes = [ci, cd, ci, cd, cd, cd, cd, vp]
    lib.rope_frequencies.restype = ci
    for f in (lib.rope_fwd, lib.rope_bwd):
        f.argtypes = [vp, vp, vp, ci, vp, vp, vp, ci, ci, ci, ci, vp, ci, cl, vp, ci, ci, cf, ci, vp]
        f.restype = ci
    lib.kv4_page_bytes.argtypes = [ci, ci]
    lib.kv4_page_bytes.restype = cs
    lib.kv_slots.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, ci, vp, vp, vp, vp, vp]
    lib.kv_slots.restype = ci
    lib.kv4_append.argtypes = [vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, vp]
    lib.kv4_append.restype = ci
    lib.kv4_load.argtypes = [vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, ci, vp]
    lib.kv4_load.restype = ci
    lib.attn_decode_kv4_workspace_bytes.argtypes = [ci, ci, ci, ci]
    lib.attn_decode_kv4_workspace_bytes.restype = cs
    lib.attn_decode_kv4.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, cf, vp, cf, ci, vp, cs, ci, vp]
    lib.attn_decode_kv4.restype = ci
    lib.attn_fwd_lse.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, cf, vp, cf, ci, ci, vp]
    lib.attn_fwd_lse.restype = ci
    lib.attn_bwd_workspace_bytes.argtypes = [ci] * 8
    lib.attn_bwd_workspace_bytes.restype = cs
    lib.attn_bwd.argtypes = [vp] * 10 + [ci] * 7 + [cf, vp, cf, ci, vp, cs, ci, vp]
    lib.attn_bwd.restype = ci
    lib.rmsnorm_add.argtypes = [vp] * 6 + [ci, ci, cd, cf, ci, ci, vp]
    lib.rmsnorm_add.restype = ci
    lib.rmsnorm_add_quant.argtypes = [vp] * 7 + [ci, ci, ci, ci, cd, cf, ci, ci, vp]
    lib.rmsnorm_add_quant.restype = ci
    lib.quant8_load.argtypes = [vp, vp, vp, ci, ci, ci, ci, ci, vp]
    lib.quant8_load.restype = ci
    lib.rmsnorm_add_bwd_workspace_bytes.argtypes = [ci, ci]
    lib.rmsnorm_add_bwd_workspace_bytes.restype = cs
    lib.rmsnorm_add_bwd.argtypes = [vp] * 8 + [ci, ci, cf, vp, cs, ci, ci, vp]
    lib.rmsnorm_add_bwd.restype = ci
    lib.attn_status_string.argtypes = [ci]
    lib.attn_status_string.restype = ctypes.c_char_p
    lib.attn_last_hip_error.argtypes = []
    lib.attn_last_hip_error.restype = ci
    _LIB = lib
    return lib


class _NotBuilt:
    """Stands for the _binding module where nothing is built: every call goes
    through the checks in Python and then load_library's error."""

    @staticmethod
    def _none(*args):
        return None

    attn_fwd = attn_decode = attn_decode_noalloc = norm_l2 = rmsnorm_rowmax = _none
    rope = kv_slots = kv4_append = kv4_load = attn_decode_kv4 = _none
    attn_fwd_lse = attn_bwd = rmsnorm_add = rmsnorm_add_quant = quant8_load = rmsnorm_add_bwd = _none


def _load_binding():
    """Load (once) the _binding module; raises if only libattn.so is built."""
    global _BINDING
    if not os.path.exists(library_path()):
        return _NotBuilt
    load_library()
    try:
        from . import _binding as b
    except ImportError as e:
        raise RuntimeError(
            f"{os.path.join(_HERE, '_binding.so')} is not built for this PyTorch; run "
            "`python -c 'import __graft_entry__ as g; g.build()'` first") from e
    _BINDING = b
    return b


def attn_status_string(status):
    return load_library().attn_status_string(int(status)).decode()


def attn_last_hip_error():
    return load_library().attn_last_hip_error()


def _check(rc):
    if rc != ATTN_OK:
        msg = attn_status_string(rc)
        if rc == ATTN_ERR_HIP:
            msg += f" (hipError_t {attn_last_hip_error()})"
        raise AttnError(rc, msg)


def _result(r):
    """What a _binding function returned: the output, or an error status (int)."""
    if type(r) is int:
        _check(r)
    return r


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _require(cond, msg):
    if not cond:
        raise ValueError(msg)


def _check_tensors(q, k, v, slopes):
    for name, t in (("q", q), ("k", k), ("v", v)):
        _require(t.is_cuda, f"{name} must be a GPU tensor")
        _require(t.is_contiguous(), f"{name} must be contiguous [B, H, L, D]")
        _require(t.dim() == 4, f"{name} must be 4-D [B, H, L, D]")
    _require(q.dtype == k.dtype == v.dtype, "q, k, v must share one dtype")
    _require(q.dtype in _DTYPE_CODE, "dtype must be float16 or bfloat16")
    _require(k.shape == v.shape, "k and v must have the same shape")
    if slopes is not None:
        _require(slopes.is_cuda and slopes.dtype == torch.float32 and slopes.is_contiguous(),
                 "alibi_slopes must be a contiguous float32 GPU tensor")
        _require(slopes.numel() == q.shape[1], "alibi_slopes needs one value per query head")


def _fwd_args(q, k, v, o, alibi_slopes):
    _check_tensors(q, k, v, alibi_slopes)
    B, Hq, Lq, D = q.shape
    _require(k.shape[0] == B and k.shape[3] == D, "k/v batch and head dim must match q")
    if o is None:
        o = torch.empty_like(q)
    _require(o.shape == q.shape and o.dtype == q.dtype and o.is_contiguous() and o.is_cuda,
             "o must be a contiguous GPU tensor shaped like q")
    return o


def _on_stream(t, stream):
    """The stream of a call, if PyTorch can allocate for it beside t, else None."""
    s = torch.cuda.current_stream() if stream is None else stream
    return s if isinstance(s, torch.cuda.Stream) and s.device == t.device else None


def _fwd_workspace(q, Hkv, Lk, causal, window, stream):
    """The workspace of a call whose keys are divided over workgroups, or None
    (one range): allocated in the pool of the stream that it is used on, so
    not where that stream is unknown to PyTorch or on another device."""
    B, Hq, Lq, D = q.shape
    lib = load_library()
    S = lib.attn_fwd_num_splits(B, Hq, Hkv, Lq, Lk, D, int(bool(causal)), int(window or 0))
    s = _on_stream(q, stream)
    if S <= 1 or s is None:
        return None
    try:
        with torch.cuda.stream(s):
            return torch.empty(lib.attn_fwd_workspace_bytes(B, Hq, Lq, D, S), dtype=torch.uint8, device=q.device)
    except torch.cuda.OutOfMemoryError:
        return None


def _workspace(t, nbytes, stream):
    """A workspace that a call drops when it returns, before its kernels have
    run: in the pool of their stream, where the next tenant of the memory runs
    after them.  (A stream of another kind, or of another device, has no such
    pool here: the caller of one keeps its workspace itself.)"""
    with torch.cuda.stream(_on_stream(t, stream)):
        return torch.empty(max(nbytes, 16), dtype=torch.uint8, device=t.device)


def attn_fwd(q, k, v, o=None, *, causal=False, scale=None, alibi_slopes=None, softcap=None,
             window=None, stream=None):
    """O = softmax(Q K^T * scale + bias) V by the fused prefill kernels.

    q [B, Hq, Lq, D], k and v [B, Hkv, Lk, D] (float16 or bfloat16, contiguous,
    on the GPU); ``o`` is written if given, else allocated.  ``scale``
    defaults to 1/sqrt(D).  ``softcap`` (cap > 0) and ``window`` (W >= 1) are
    the score modifiers of the C entry point ``attn_fwd_mod``.  Where the keys
    of few query rows are divided over workgroups (``attn_fwd_split``), the
    workspace is allocated here, and the call does without where memory has
    run out.  Returns ``o``.
    """
    r = (_BINDING or _load_binding()).attn_fwd(q, k, v, o, causal, scale, alibi_slopes, softcap, window, stream)
    if r is not None:
        return _result(r)
    o = _fwd_args(q, k, v, o, alibi_slopes)
    B, Hq, Lq, D = q.shape
    Hkv, Lk = k.shape[1], k.shape[2]
    sc = 1.0 / math.sqrt(D) if scale is None else float(scale)
    cap, win = float(softcap or 0.0), int(window or 0)
    ws = _fwd_workspace(q, Hkv, Lk, causal, win, stream)
    _check(load_library().attn_fwd_split(_ptr(q), _ptr(k), _ptr(v), _ptr(o), B, Hq, Hkv, Lq, Lk, D,
                                         int(bool(causal)), sc, _ptr(alibi_slopes), cap, win, _ptr(ws),
                                         0 if ws is None else ws.numel(), _DTYPE_CODE[q.dtype], _stream(stream)))
    return o


def attn_fwd_mod(q, k, v, o=None, *, causal=False, scale=None, alibi_slopes=None, softcap=None,
                 window=None, stream=None):
    """attn_fwd with the SoftCap modifier (``softcap``: None or cap > 0) and the
    causal sliding window (``window``: None or W >= 1 keys per row)."""
    return attn_fwd(q, k, v, o, causal=causal, scale=scale, alibi_slopes=alibi_slopes, softcap=softcap,
                    window=window, stream=stream)


def attn_decode_workspace_bytes(B, Hq, D, num_splits):
    return load_library().attn_decode_workspace_bytes(B, Hq, D, num_splits)


def attn_decode_num_splits(B, Hq, Hkv, Lk, D):
    return load_library().attn_decode_num_splits(B, Hq, Hkv, Lk, D)


def _decode_args(q, k, v, o, alibi_slopes, num_splits, workspace, stream):
    _check_tensors(q, k, v, alibi_slopes)
    B, Hq, Lq, D = q.shape
    _require(Lq == 1, "decode takes one query token (q.shape[2] == 1)")
    Hkv, Lk = k.shape[1], k.shape[2]
    _require(k.shape[0] == B and k.shape[3] == D, "k/v batch and head dim must match q")
    if o is None:
        o = torch.empty_like(q)
    _require(o.shape == q.shape and o.dtype == q.dtype and o.is_contiguous() and o.is_cuda,
             "o must be a contiguous GPU tensor shaped like q")
    lib = load_library()
    S = num_splits if num_splits else lib.attn_decode_num_splits(B, Hq, Hkv, Lk, D)
    need = lib.attn_decode_workspace_bytes(B, Hq, D, max(S, 1))
    if workspace is None:
        workspace = _workspace(q, need, stream)
    return o, workspace


def attn_decode(q, k, v, o=None, *, scale=None, alibi_slopes=None, softcap=None, num_splits=0,
                workspace=None, stream=None):
    """Single-token decode by split-k: q [B, Hq, 1, D] against k, v [B, Hkv, Lk, D].

    ``softcap``: None, or the cap > 0 of the SoftCap score modifier
    (cap * tanh(scale q.k / cap)); with it the call goes to ``attn_decode_mod``.
    ``num_splits`` = 0 lets the library choose.  ``workspace`` (uint8 GPU
    tensor) is allocated when not given.  Returns ``o`` [B, Hq, 1, D].
    """
    r = (_BINDING or _load_binding()).attn_decode(q, k, v, o, scale, alibi_slopes, softcap, num_splits, workspace, stream)
    if r is not None:
        return _result(r)
    if softcap:
        return attn_decode_mod(q, k, v, o, scale=scale, alibi_slopes=alibi_slopes, softcap=softcap,
                               num_splits=num_splits, workspace=workspace, stream=stream)
    o, workspace = _decode_args(q, k, v, o, alibi_slopes, num_splits, workspace, stream)
    B, Hq, _, D = q.shape
    Hkv, Lk = k.shape[1], k.shape[2]
    sc = 1.0 / math.sqrt(D) if scale is None else float(scale)
    _check(load_library().attn_decode(_ptr(q), _ptr(k), _ptr(v), _ptr(o), B, Hq, Hkv, Lk, D, sc,
                                      _ptr(alibi_slopes), int(num_splits), _ptr(workspace),
                                      workspace.numel() * workspace.element_size(), _DTYPE_CODE[q.dtype],
                                      _stream(stream)))
    return o


def attn_decode_mod(q, k, v, o=None, *, scale=None, alibi_slopes=None, softcap=None, num_splits=0,
                    workspace=None, stream=None):
    """attn_decode with the SoftCap score modifier (``softcap``: None or cap > 0)."""
    r = (_BINDING or _load_binding()).attn_decode(q, k, v, o, scale, alibi_slopes, softcap, num_splits, workspace, stream)
    if r is not None:
        return _result(r)
    o, workspace = _decode_args(q, k, v, o, alibi_slopes, num_splits, workspace, stream)
    B, Hq, _, D = q.shape
    Hkv, Lk = k.shape[1], k.shape[2]
    sc = 1.0 / math.sqrt(D) if scale is None else float(scale)
    _check(load_library().attn_decode_mod(_ptr(q), _ptr(k), _ptr(v), _ptr(o), B, Hq, Hkv, Lk, D, sc,
                                          _ptr(alibi_slopes), float(softcap or 0.0), int(num_splits),
                                          _ptr(workspace), workspace.numel() * workspace.element_size(),
                                          _DTYPE_CODE[q.dtype], _stream(stream)))
    return o


ATTN_DECODE_NOALLOC_BYTES = 16 << 20


def attn_decode_noalloc(q, k, v, o=None, *, scale=None, alibi_slopes=None, softcap=None, num_splits=0,
                        stream=None):
    """attn_decode_mod with the workspace in the library's static device array
    (no allocation inside the library; ``o`` is allocated here if not given).
    Calls that overlap on one GPU race on that array."""
    r = (_BINDING or _load_binding()).attn_decode_noalloc(q, k, v, o, scale, alibi_slopes, softcap, num_splits, stream)
    if r is not None:
        return _result(r)
    _check_tensors(q, k, v, alibi_slopes)
    B, Hq, Lq, D = q.shape
    _require(Lq == 1, "decode takes one query token (q.shape[2] == 1)")
    Hkv, Lk = k.shape[1], k.shape[2]
    _require(k.shape[0] == B and k.shape[3] == D, "k/v batch and head dim must match q")
    if o is None:
        o = torch.empty_like(q)
    _require(o.shape == q.shape and o.dtype == q.dtype and o.is_contiguous() and o.is_cuda,
             "o must be a contiguous GPU tensor shaped like q")
    sc = 1.0 / math.sqrt(D) if scale is None else float(scale)
    _check(load_library().attn_decode_noalloc(_ptr(q), _ptr(k), _ptr(v), _ptr(o), B, Hq, Hkv, Lk, D, sc,
                                              _ptr(alibi_slopes), float(softcap or 0.0), int(num_splits),
                                              _DTYPE_CODE[q.dtype], _stream(stream)))
    return o


def attn_fwd_kernels(D, dtype, causal, alibi, softcap=0.0, window=0):
    """Name of the kernel attn_fwd_mod launches for these arguments where the
    query rows give every compute unit work (host only)."""
    buf = ctypes.create_string_buffer(256)
    _check(load_library().attn_fwd_kernels(D, _DTYPE_CODE.get(dtype, dtype), int(bool(causal)), int(bool(alibi)),
                                           float(softcap or 0.0), int(window or 0), buf, 256))
    return buf.value.decode().split(";")


def attn_fwd_call_kernels(B, Hq, Hkv, Lq, Lk, D, dtype, causal, alibi, softcap=0.0, window=0, workspace=True):
    """Names of the kernels that attn_fwd launches for these sizes (host only;
    workspace=False: those of the C entry points without one)."""
    buf = ctypes.create_string_buffer(256)
    _check(load_library().attn_fwd_call_kernels(B, Hq, Hkv, Lq, Lk, D, _DTYPE_CODE.get(dtype, dtype),
                                                int(bool(causal)), int(bool(alibi)), float(softcap or 0.0),
                                                int(window or 0), int(bool(workspace)), buf, 256))
    return buf.value.decode().split(";")


def attn_decode_kernels(Hq, Hkv, D, dtype, alibi, softcap=0.0):
    """Names of the kernels attn_decode_mod launches for these arguments (host only)."""
    buf = ctypes.create_string_buffer(256)
    _check(load_library().attn_decode_kernels(Hq, Hkv, D, _DTYPE_CODE.get(dtype, dtype), int(bool(alibi)),
                                              float(softcap or 0.0), buf, 256))
    return buf.value.decode().split(";")


def peaks_hbm_read(buf, sink=None, stream=None):
    """Stream-read every byte of the GPU tensor ``buf`` once (peaks.h).  Returns ``sink``."""
    lib = load_library()
    if sink is None:
        sink = torch.empty(lib.peaks_hbm_read_sink_floats(), dtype=torch.float32, device=buf.device)
    _check(lib.peaks_hbm_read(_ptr(buf), buf.numel() * buf.element_size(), _ptr(sink), _stream(stream)))
    return sink


def peaks_mfma(dtype, iters, operands, sink=None, clocks=None, stream=None):
    """Run the MFMA loop of peaks.h; returns (sink, clocks) tensors."""
    lib = load_library()
    if sink is None:
        sink = torch.empty(lib.peaks_mfma_waves(), dtype=torch.float32, device=operands.device)
    if clocks is None:
        clocks = torch.zeros(2, dtype=torch.int64, device=operands.device)
    _check(lib.peaks_mfma(_DTYPE_CODE.get(dtype, dtype), int(iters), _ptr(operands), _ptr(sink), _ptr(clocks),
                          _stream(stream)))
    return sink, clocks


def peaks_mfma_waves():
    return load_library().peaks_mfma_waves()


def peaks_mfma_operand_bytes():
    return load_library().peaks_mfma_operand_bytes()


NORM_F16, NORM_BF16, NORM_F32 = 0, 1, 2
_NORM_CODE = {torch.float16: NORM_F16, torch.bfloat16: NORM_BF16, torch.float32: NORM_F32}


def norm_chunks(op, N, M, dtype):
    """Chunks per row that norm_l2 (op "l2") or rmsnorm_rowmax (op "rms") uses for chunks=0."""
    return load_library().norm_chunks(int(op == "rms"), N, M, _NORM_CODE[dtype])


def norm_kernels(op, M, dtype, chunks):
    """Names of the kernels norm_l2 (op "l2") or rmsnorm_rowmax (op "rms")
    launches for rows of M elements and `chunks` >= 1 chunks per row (host only)."""
    buf = ctypes.create_string_buffer(128)
    _check(load_library().norm_kernels(int(op == "rms"), int(M), _NORM_CODE.get(dtype, dtype), int(chunks), buf, 128))
    return buf.value.decode().split(";")


def norm_workspace_bytes(N, chunks):
    return load_library().norm_workspace_bytes(N, chunks)


def _norm_args(op, x, chunks, workspace, stream):
    _require(x.is_cuda and x.is_contiguous() and x.dim() == 2, "x must be a contiguous 2-D GPU tensor [N, M]")
    _require(x.dtype in _NORM_CODE, "x must be float16, bfloat16 or float32")
    N, M = x.shape
    lib = load_library()
    C = chunks or lib.norm_chunks(int(op == "rms"), N, M, _NORM_CODE[x.dtype])
    if workspace is None:
        workspace = _workspace(x, lib.norm_workspace_bytes(N, max(C, 1)), stream)
    return N, M, workspace


def norm_l2(x, out=None, *, chunks=0, workspace=None, stream=None):
    """Row L2 norms of x [N, M] (single pass, split over the row): out [N] float32."""
    r = (_BINDING or _load_binding()).norm_l2(x, out, chunks, workspace, stream)
    if r is not None:
        return _result(r)
    N, M, workspace = _norm_args("l2", x, chunks, workspace, stream)
    if out is None:
        out = torch.empty(N, dtype=torch.float32, device=x.device)
    _require(out.is_cuda and out.dtype == torch.float32 and out.numel() == N, "out must be float32 [N]")
    _check(load_library().norm_l2(_ptr(x), _ptr(out), N, M, _NORM_CODE[x.dtype], int(chunks), _ptr(workspace),
                                  workspace.numel() * workspace.element_size(), _stream(stream)))
    return out


def rmsnorm_rowmax(x, y=None, rowmax=None, *, eps=1e-6, chunks=0, workspace=None, stream=None):
    """y = x / sqrt(mean(x^2) + eps) (x's dtype) and rowmax [N] = max of each row of y (float32)."""
    r = (_BINDING or _load_binding()).rmsnorm_rowmax(x, y, rowmax, eps, chunks, workspace, stream)
    if r is not None:
        return _result(r)
    N, M, workspace = _norm_args("rms", x, chunks, workspace, stream)
    if y is None:
        y = torch.empty_like(x)
    if rowmax is None:
        rowmax = torch.empty(N, dtype=torch.float32, device=x.device)
    _require(y.shape == x.shape and y.dtype == x.dtype and y.is_contiguous() and y.is_cuda, "y must match x")
    _require(rowmax.is_cuda and rowmax.dtype == torch.float32 and rowmax.numel() == N, "rowmax must be float32 [N]")
    _check(load_library().rmsnorm_rowmax(_ptr(x), _ptr(y), _ptr(rowmax), N, M, float(eps), _NORM_CODE[x.dtype],
                                         int(chunks), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                         _stream(stream)))
    return y, rowmax


# Rotary positions, and the paged 4-bit cache with the decode that reads it.

_ROPE_SCALING = {None: 0, "linear": 1, "base": 2, "parts": 3}


def rope_frequencies(rotary_dim, base=10000.0, *, scaling=None, factor=1.0, original_length=0, slow=1.0, fast=32.0,
                     device=None):
    """Frequencies (radians per position, float64 [rotary_dim / 2]) for rope_fwd.

    ``scaling`` adapts them to contexts longer than the trained one by
    ``factor``: None, "linear" (positions interpolated), "base" (a larger
    base) or "parts" (pairs that make fewer than ``slow`` turns over
    ``original_length`` tokens are interpolated, those over ``fast`` are not,
    with a ramp between).
    """
    _require(scaling in _ROPE_SCALING, "scaling must be None, 'linear', 'base' or 'parts'")
    n = int(rotary_dim)
    _require(_fits(n), "rotary_dim must fit 32 bits")
    f = torch.empty(max(n // 2, 1), dtype=torch.float64)
    _check(load_library().rope_frequencies(n, float(base), _ROPE_SCALING[scaling], float(factor),
                                           float(original_length), float(slow), float(fast), _ptr(f)))
    return f if device is None else f.to(device)


_INT_MAX = (1 << 31) - 1


def _fits(*sizes):
    """Whether the C entry points' ints hold them (ctypes would cut them to 32 bits)."""
    return all(0 <= n <= _INT_MAX for n in sizes)


def _on_device(t, stream):
    """Stream and device of a call on t: t's device becomes the current one for
    the call, and a stream that is given has to be on it."""
    if stream is None:
        stream = torch.cuda.current_stream(t.device)
    _require(getattr(stream, "device", t.device) == t.device, "stream must be on the tensors' device")
    return stream


def _same_device(first, **tensors):
    _require(first.is_cuda, "tensors must be on the GPU")
    _require(_fits(*first.shape), "sizes must fit 32 bits")
    for name, t in tensors.items():
        _require(t.device == first.device, f"{name} must be on the same GPU as the other tensors")
        _require(_fits(*t.shape), f"{name}'s sizes must fit 32 bits")


def _ints(name, t, dtype, shape):
    _require(t.dtype == dtype and tuple(t.shape) == tuple(shape) and t.is_contiguous(),
             f"{name} must be a contiguous {str(dtype)[6:]} tensor of shape {list(shape)}")


def _strides(t):
    """Strides of batches, heads and tokens; 0 where there is one alone."""
    return (ctypes.c_longlong * 3)(*(s if n > 1 else 0 for s, n in zip(t.stride()[:3], t.shape)))


def _rows(name, t, shape=None):
    _require(t.dim() == 4, f"{name} must be 4-D [B, H, L, D]")
    _require(t.shape[3] == 1 or t.stride(3) == 1, f"{name} must have contiguous rows (the last dim)")
    _require(shape is None or tuple(t.shape) == tuple(shape), f"{name} must have shape {list(shape or [])}")


def _allocate(shape, like, stream, dtype=None):
    """An output, in the pool of the stream that it is written on."""
    if isinstance(stream, torch.cuda.Stream):
        with torch.cuda.stream(stream):
            return torch.empty(shape, dtype=dtype or like.dtype, device=like.device)
    return torch.empty(shape, dtype=dtype or like.dtype, device=like.device)


def _overlaps(a, b):
    """Whether the memory that two tensors span has a common part."""
    end = lambda t: t.data_ptr() + (1 + sum((n - 1) * s for n, s in zip(t.shape, t.stride()))) * t.element_size()  # noqa: E731
    return bool(a.numel() and b.numel()) and a.data_ptr() < end(b) and b.data_ptr() < end(a)


def _rope(bwd, q, k, positions, freqs, q_out, k_out, interleaved, magnitude, stream):
    r = (_BINDING or _load_binding()).rope(q, k, positions, freqs, q_out, k_out, interleaved, magnitude, bwd, stream)
    if r is not None:
        return _result(r)
    _rows("q", q)
    B, Hq, L, D = q.shape
    _require(q.dtype in _NORM_CODE, "dtype must be float16, bfloat16 or float32")
    _same_device(q, positions=positions, freqs=freqs)
    if k is None:
        _require(k_out is None, "k_out needs k")
    else:
        _rows("k", k)
        _same_device(q, k=k)
        _require(k.dtype == q.dtype and (k.shape[0], *k.shape[2:]) == (B, L, D),
                 "k must have q's dtype, batch, length and head dim")
    _require(freqs.dtype == torch.float64 and freqs.dim() == 1 and freqs.is_contiguous() and _fits(2 * freqs.numel()),
             "freqs must be a contiguous float64 tensor [rotary_dim / 2]")
    _require(positions.dtype in (torch.int32, torch.int64) and tuple(positions.shape) in ((B, L), (L,))
             and positions.is_contiguous(), "positions must be a contiguous int32 or int64 tensor [B, L] or [L]")
    stream = _on_device(q, stream)
    outs = []
    for name, x, o in (("q", q, q_out), ("k", k, k_out)):
        if o is None and x is not None:
            o = _allocate(x.shape, x, stream)
        elif o is not None:
            _same_device(q, **{name + "_out": o})
            _require(o.shape == x.shape and o.dtype == x.dtype and o.is_contiguous(),
                     f"{name}_out must be a contiguous tensor shaped like {name}")
        outs.append(o)
    for name, x, o, others in (("q", q, outs[0], (k, outs[1])), ("k", k, outs[1], (q, outs[0]))):
        if o is not None:
            others = [t for t in others if t is not None]
            if not (x.is_contiguous() and o.data_ptr() == x.data_ptr()):
                others.append(x)
            _require(not any(_overlaps(o, t) for t in others),
                     f"{name}_out may share memory with nothing, but be {name} itself if that is contiguous")
    lib = load_library()
    fn = lib.rope_bwd if bwd else lib.rope_fwd
    with torch.cuda.device(q.device):
        _check(fn(_ptr(q), _strides(q), _ptr(outs[0]), Hq, _ptr(k), None if k is None else _strides(k), _ptr(outs[1]),
                  0 if k is None else k.shape[1], B, L, D, _ptr(positions), positions.element_size() * 8,
                  L if positions.dim() == 2 else 0, _ptr(freqs), 2 * freqs.numel(), int(bool(interleaved)),
                  float(magnitude), _NORM_CODE[q.dtype], _stream(stream)))
    return outs[0], outs[1]


def rope_fwd(q, k, positions, freqs, q_out=None, k_out=None, *, interleaved=False, magnitude=1.0, stream=None):
    """Rotate q [B, Hq, L, D] and k [B, Hkv, L, D] (or None) by their positions.

    float16, bfloat16 or float32; strided views with contiguous rows are taken
    as they are (a projection's [B, L, H, D] transposed).  ``positions``: int32 or
    int64 [B, L] or [L]; ``freqs``: float64 [rotary_dim / 2] on the GPU
    (rope_frequencies); the first rotary_dim dims are rotated in pairs
    (i, i + rotary_dim / 2), or (2 i, 2 i + 1) if ``interleaved``, and the
    rest copied.  ``magnitude`` scales the rotated dims.  Outputs are contiguous;
    q_out may be q itself, and k_out k.  Nothing is recorded for autograd: a program
    that trains calls rope_bwd.  Returns (q_out, k_out).
    """
    return _rope(False, q, k, positions, freqs, q_out, k_out, interleaved, magnitude, stream)


def rope_bwd(dq, dk, positions, freqs, q_out=None, k_out=None, *, interleaved=False, magnitude=1.0, stream=None):
    """Gradients of rope_fwd's q and k from those of its outputs (the transposed
    rotation), with the same arguments."""
    return _rope(True, dq, dk, positions, freqs, q_out, k_out, interleaved, magnitude, stream)


def kv4_page_bytes(page, D):
    """Bytes of a page of `page` tokens of one head in the 4-bit cache (0 if not supported)."""
    return load_library().kv4_page_bytes(page, D) if _fits(page, D) else 0


def kv_slots(lens, counts, table, free_pages, page, L, *, slots=None, positions=None, new_lens=None, taken=None,
             stream=None):
    """Pages and slots of the new tokens of B requests, on the GPU.

    ``lens`` and ``counts`` (int32 [B]): tokens in the cache, and new ones (at
    most L of them are taken).  Pages that they need are taken off the front
    of ``free_pages`` (int32 [F]) request by request and written into ``table``
    (int32 [B, max_pages], in place).  Returns (slots [B, L] int64, -1 for no
    token; positions [B, L] int32; new_lens [B] int32; taken [1] int32, the number
    of pages taken); see kv4.h.
    """
    r = (_BINDING or _load_binding()).kv_slots(lens, counts, table, free_pages, page, L, slots, positions, new_lens,
                                               taken, stream)
    if r is not None:
        return _result(r)
    page, L = int(page), int(L)
    _require(lens.dim() == 1 and table.dim() == 2 and free_pages.dim() == 1,
             "lens must be [B], table [B, max_pages] and free_pages [F]")
    B, M = lens.shape[0], table.shape[1]
    _same_device(lens, counts=counts, table=table, free_pages=free_pages)
    _ints("lens", lens, torch.int32, (B,))
    _ints("counts", counts, torch.int32, (B,))
    _ints("table", table, torch.int32, (B, M))
    _ints("free_pages", free_pages, torch.int32, (free_pages.shape[0],))
    _require(L >= 1 and _fits(page, L), "page and L must be at least 1 and fit 32 bits")
    _require(not any(_overlaps(table, x) for x in (lens, counts, free_pages)),
             "table, which is written, must not share memory with the other tensors")
    stream = _on_device(lens, stream)
    outs = []
    for name, t, dtype, shape in (("slots", slots, torch.int64, (B, L)), ("positions", positions, torch.int32, (B, L)),
                                  ("new_lens", new_lens, torch.int32, (B,)), ("taken", taken, torch.int32, (1,))):
        if t is None:
            t = _allocate(shape, lens, stream, dtype)
        else:
            _same_device(lens, **{name: t})
            _ints(name, t, dtype, shape)
            _require(not any(_overlaps(t, x) for x in (lens, counts, table, free_pages, *outs)),
                     f"{name} must not share memory with the other tensors")
        outs.append(t)
    with torch.cuda.device(lens.device):
        _check(load_library().kv_slots(_ptr(lens), _ptr(counts), _ptr(table), _ptr(free_pages), free_pages.shape[0], B,
                                       M, page, L, *(_ptr(t) for t in outs), _stream(stream)))
    return tuple(outs)


def _cache_page(cache, D):
    """Tokens of a page of a cache [pages, Hkv, bytes] of head dim D."""
    _require(cache.dtype == torch.uint8 and cache.dim() == 3 and cache.is_contiguous(),
             "cache must be a contiguous uint8 tensor [pages, Hkv, kv4_page_bytes(page, D)]")
    _require(D in (64, 128), "head dim must be 64 or 128")
    page = cache.shape[2] * 16 // (17 * D)
    _require(page > 0 and kv4_page_bytes(page, D) == cache.shape[2],
             "the cache's rows must be kv4_page_bytes(page, D) of a power of two from 16 to 32768")
    return page


def kv4_append(k, v, cache, slots, *, stream=None):
    """Round k and v [B, Hkv, L, D] (float16 or bfloat16, rows contiguous) to 4
    bits and write them into ``cache`` (uint8 [pages, Hkv, kv4_page_bytes(page,
    D)]) at ``slots`` (int64 [B, L], distinct; others than 0 .. pages * page - 1
    are skipped).  The cache shares memory with no other operand.  Returns ``cache``."""
    r = (_BINDING or _load_binding()).kv4_append(k, v, cache, slots, stream)
    if r is not None:
        return _result(r)
    _rows("k", k)
    _rows("v", v, k.shape)
    B, H, L, D = k.shape
    _require(k.dtype == v.dtype and k.dtype in _DTYPE_CODE, "k and v must both be float16 or bfloat16")
    _same_device(k, v=v, cache=cache, slots=slots)
    page = _cache_page(cache, D)
    _require(cache.shape[1] == H, "cache and k must have the same number of heads")
    _ints("slots", slots, torch.int64, (B, L))
    stream = _on_device(k, stream)
    with torch.cuda.device(k.device):
        _check(load_library().kv4_append(_ptr(k), _strides(k), _ptr(v), _strides(v), _ptr(cache), _ptr(slots), B, H, L,
                                         D, cache.shape[0], page, _DTYPE_CODE[k.dtype], _stream(stream)))
    return cache


def _paged(cache, table, lens):
    _require(table.dim() == 2, "table must be [B, max_pages]")
    _same_device(cache, table=table, lens=lens)
    B, M = table.shape
    _ints("table", table, torch.int32, (B, M))
    _ints("lens", lens, torch.int32, (B,))
    return B, M


def kv4_load(cache, table, lens, L, D, dtype, k=None, v=None, *, starts=None, stream=None):
    """k and v [B, Hkv, L, D] of tokens starts[b] .. starts[b] + L - 1 (default:
    from token 0) of each sequence of a 4-bit cache, as held; zeros from
    token lens[b] on.  ``table`` int32 [B, max_pages], ``lens`` and
    ``starts`` int32 [B]; k and v, if given, share memory with nothing.  Returns
    (k, v), which attn_fwd takes: for requests of one length, as it sees every key."""
    r = (_BINDING or _load_binding()).kv4_load(cache, table, lens, L, D, dtype, k, v, starts, stream)
    if r is not None:
        return _result(r)
    L, D = int(L), int(D)
    _require(dtype in _DTYPE_CODE, "dtype must be float16 or bfloat16")
    page = _cache_page(cache, D)
    B, M = _paged(cache, table, lens)
    _require(L >= 1 and _fits(L), "L must be at least 1 and fit 32 bits")
    if starts is not None:
        _same_device(cache, starts=starts)
        _ints("starts", starts, torch.int32, (B,))
    stream = _on_device(cache, stream)
    outs = []
    for name, t in (("k", k), ("v", v)):
        shape = (B, cache.shape[1], L, D)
        if t is None:
            t = _allocate(shape, cache, stream, dtype)
        else:
            _same_device(cache, **{name: t})
            _require(tuple(t.shape) == shape and t.dtype == dtype and t.is_contiguous(),
                     f"{name} must be a contiguous {str(dtype)[6:]} tensor of shape {list(shape)}")
        outs.append(t)
    with torch.cuda.device(cache.device):
        _check(load_library().kv4_load(_ptr(cache), _ptr(table), _ptr(starts), _ptr(lens), _ptr(outs[0]),
                                       _ptr(outs[1]), B, cache.shape[1], L, D, cache.shape[0], page, M,
                                       _DTYPE_CODE[dtype], _stream(stream)))
    return outs[0], outs[1]


def attn_decode_kv4_workspace_bytes(B, Hq, Hkv, D):
    return load_library().attn_decode_kv4_workspace_bytes(B, Hq, Hkv, D) if _fits(B, Hq, Hkv, D) else 0


def attn_decode_kv4(q, cache, table, lens, o=None, *, scale=None, alibi_slopes=None, softcap=None, window=None,
                    workspace=None, stream=None):
    """Single-token decode against a 4-bit cache: q [B, Hq, 1, D] (float16 or
    bfloat16, what the cache was written from) is token lens[b] - 1 of its
    sequence and sees the tokens up to itself, or the last ``window`` of them.

    ``cache`` uint8 [pages, Hkv, kv4_page_bytes(page, D)], ``table`` int32 [B,
    max_pages], ``lens`` int32 [B].  ``scale`` defaults to 1/sqrt(D);
    ``alibi_slopes`` and ``softcap`` as for attn_decode.  ``workspace`` (uint8
    GPU tensor of attn_decode_kv4_workspace_bytes) is allocated when not given;
    neither it nor ``o`` may share memory with another operand, but ``o`` may be
    q itself.  Returns ``o`` [B, Hq, 1, D], 0 for a sequence that sees nothing.
    """
    r = (_BINDING or _load_binding()).attn_decode_kv4(q, cache, table, lens, o, scale, alibi_slopes, softcap, window,
                                                      workspace, stream)
    if r is not None:
        return _result(r)
    _require(q.dim() == 4 and q.is_contiguous() and q.shape[2] == 1, "q must be contiguous [B, Hq, 1, D]")
    _require(q.dtype in _DTYPE_CODE, "dtype must be float16 or bfloat16")
    B, Hq, _, D = q.shape
    _same_device(q, cache=cache)
    page = _cache_page(cache, D)
    _require(_paged(cache, table, lens)[0] == B, "table and lens must have one row for each of q's sequences")
    if alibi_slopes is not None:
        _same_device(q, alibi_slopes=alibi_slopes)
        _require(alibi_slopes.dtype == torch.float32 and alibi_slopes.is_contiguous() and alibi_slopes.numel() == Hq,
                 "alibi_slopes must be a contiguous float32 tensor with one value per query head")
    stream = _on_device(q, stream)
    if o is None:
        o = _allocate(q.shape, q, stream)
    _same_device(q, o=o)
    _require(o.shape == q.shape and o.dtype == q.dtype and o.is_contiguous(),
             "o must be a contiguous GPU tensor shaped like q")
    if workspace is None:
        _require(isinstance(stream, torch.cuda.Stream), "a stream of this kind needs a workspace of the caller's")
        with torch.cuda.device(q.device):            # whose compute units the size counts
            size = attn_decode_kv4_workspace_bytes(B, Hq, cache.shape[1], D)
        workspace = _allocate((max(size, 16),), q, stream, torch.uint8)
    _same_device(q, workspace=workspace)
    _require(workspace.is_contiguous(), "workspace must be contiguous")
    sc = 1.0 / math.sqrt(D) if scale is None else float(scale)
    win = min(int(window or 0), _INT_MAX)            # (that many see every token)
    _require(win >= 0, "window must be at least 1")
    with torch.cuda.device(q.device):
        _check(load_library().attn_decode_kv4(_ptr(q), _ptr(cache), _ptr(table), _ptr(lens), _ptr(o), B, Hq,
                                              cache.shape[1], D, cache.shape[0], page, table.shape[1], sc,
                                              _ptr(alibi_slopes), float(softcap or 0.0), win,
                                              _ptr(workspace), workspace.numel() * workspace.element_size(),
                                              _DTYPE_CODE[q.dtype], _stream(stream)))
    return o


# Attention in training: the forward pass with its rows' log-sum-exp, and the backward pass.

def _train_args(q, k, v, alibi_slopes):
    for name, t in (("q", q), ("k", k), ("v", v)):
        _require(t.dim() == 4 and t.is_contiguous(), f"{name} must be contiguous [B, H, L, D]")
    _same_device(q, k=k, v=v)
    _require(q.dtype == k.dtype == v.dtype and q.dtype in _DTYPE_CODE, "q, k, v must share one dtype, float16 or bfloat16")
    B, Hq, Lq, D = q.shape
    _require(k.shape == v.shape and k.shape[0] == B and k.shape[3] == D,
             "k and v must have the same shape, and q's batch and head dim")
    if alibi_slopes is not None:
        _same_device(q, alibi_slopes=alibi_slopes)
        _require(alibi_slopes.dtype == torch.float32 and alibi_slopes.is_contiguous() and alibi_slopes.numel() == Hq,
                 "alibi_slopes must be a contiguous float32 tensor with one value per query head")
    return B, Hq, k.shape[1], Lq, k.shape[2], D


def _train_mod(D, scale, softcap, window):
    win = min(int(window or 0), _INT_MAX)            # (that many see every key)
    _require(win >= 0, "window must be at least 1")
    return 1.0 / math.sqrt(D) if scale is None else float(scale), float(softcap or 0.0), win


def _given(name, t, like, stream, shape=None, dtype=None):
    """An output: allocated, or the one that the caller gave, which has to be laid out like it."""
    shape, dtype = tuple(like.shape) if shape is None else tuple(shape), dtype or like.dtype
    if t is None:
        return _allocate(shape, like, stream, dtype)
    _same_device(like, **{name: t})
    _require(tuple(t.shape) == shape and t.dtype == dtype and t.is_contiguous(),
             f"{name} must be a contiguous {str(dtype)[6:]} tensor of shape {list(shape)}")
    return t


def attn_fwd_lse(q, k, v, o=None, lse=None, *, causal=False, scale=None, alibi_slopes=None, softcap=None, window=None,
                 stream=None):
    """attn_fwd that also gives each row's log-sum-exp, for attn_bwd.

    q [B, Hq, Lq, D], k and v [B, Hkv, Lk, D] and the other arguments as for
    attn_fwd; ``softcap`` at most 1024.  ``lse`` [B, Hq, Lq] float32: log sum_j
    exp(s_ij) of the row's scores (scaled, capped, with the bias), -inf for a row
    that sees no key.  q, k, v and o are 16-byte aligned; neither output may share memory
    with another operand.
    Nothing is recorded for autograd: a program that trains calls attn_bwd.
    Returns (o, lse).
    """
    r = (_BINDING or _load_binding()).attn_fwd_lse(q, k, v, o, lse, causal, scale, alibi_slopes, softcap, window, stream)
    if r is not None:
        return _result(r)
    B, Hq, Hkv, Lq, Lk, D = _train_args(q, k, v, alibi_slopes)
    sc, cap, win = _train_mod(D, scale, softcap, window)
    stream = _on_device(q, stream)
    o = _given("o", o, q, stream)
    lse = _given("lse", lse, q, stream, (B, Hq, Lq), torch.float32)
    with torch.cuda.device(q.device):
        _check(load_library().attn_fwd_lse(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), B, Hq, Hkv, Lq, Lk, D,
                                           int(bool(causal)), sc, _ptr(alibi_slopes), cap, win, _DTYPE_CODE[q.dtype],
                                           _stream(stream)))
    return o, lse


def attn_bwd_workspace_bytes(B, Hq, Hkv, Lq, Lk, D, causal=False, window=None):
    sizes = (B, Hq, Hkv, Lq, Lk, D, min(int(window or 0), _INT_MAX))
    return load_library().attn_bwd_workspace_bytes(*sizes[:6], int(bool(causal)), sizes[6]) if _fits(*sizes) else 0


def attn_bwd(do, q, k, v, o, lse, dq=None, dk=None, dv=None, *, causal=False, scale=None, alibi_slopes=None,
             softcap=None, window=None, workspace=None, stream=None):
    """Gradients of attention's q, k and v from ``do``, that of its output.

    ``o`` and ``lse`` are attn_fwd_lse's of the same q, k, v and arguments; the
    probabilities are recomputed.  ``do`` [B, Hq, Lq, D] may be a strided view
    with contiguous rows (a [B, Lq, Hq, D] transposed), strides multiples of 8.
    dk and dv [B, Hkv, Lk, D] are summed over the query heads of each KV head; alibi_slopes get
    no gradient.  ``workspace`` (uint8 GPU tensor of attn_bwd_workspace_bytes) is
    allocated when not given; neither it nor an output may share memory with
    another operand.  Returns (dq, dk, dv).
    """
    r = (_BINDING or _load_binding()).attn_bwd(do, q, k, v, o, lse, dq, dk, dv, causal, scale, alibi_slopes, softcap, window,
                                               workspace, stream)
    if r is not None:
        return _result(r)
    B, Hq, Hkv, Lq, Lk, D = _train_args(q, k, v, alibi_slopes)
    sc, cap, win = _train_mod(D, scale, softcap, window)
    _same_device(q, do=do, o=o, lse=lse)
    _rows("do", do, q.shape)
    _require(do.dtype == q.dtype, "do must have q's dtype")
    _require(o.shape == q.shape and o.dtype == q.dtype and o.is_contiguous(), "o must be a contiguous tensor like q")
    _ints("lse", lse, torch.float32, (B, Hq, Lq))
    stream = _on_device(q, stream)
    dq, dk, dv = _given("dq", dq, q, stream), _given("dk", dk, k, stream), _given("dv", dv, v, stream)
    if workspace is None:
        _require(isinstance(stream, torch.cuda.Stream), "a stream of this kind needs a workspace of the caller's")
        with torch.cuda.device(q.device):            # whose compute units the size counts
            size = attn_bwd_workspace_bytes(B, Hq, Hkv, Lq, Lk, D, causal, win)
        workspace = _allocate((max(size, 16),), q, stream, torch.uint8)
    _same_device(q, workspace=workspace)
    _require(workspace.is_contiguous(), "workspace must be contiguous")
    with torch.cuda.device(q.device):
        _check(load_library().attn_bwd(_ptr(do), _strides(do), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(dq),
                                       _ptr(dk), _ptr(dv), B, Hq, Hkv, Lq, Lk, D, int(bool(causal)), sc,
                                       _ptr(alibi_slopes), cap, win, _ptr(workspace),
                                       workspace.numel() * workspace.element_size(), _DTYPE_CODE[q.dtype],
                                       _stream(stream)))
    return dq, dk, dv


# The norm between a model's layers.

_QUANT8_CODE = {torch.float8_e4m3fn: 0, torch.int8: 1}


def _norm_rows(name, x):
    """Rows and their length of x [..., M]."""
    _require(x.dim() >= 1 and x.is_contiguous(), f"{name} must be contiguous [..., M]")
    _require(x.dtype in _NORM_CODE, f"{name} must be float16, bfloat16 or float32")
    M = x.shape[-1]
    _require(M >= 1 and x.numel() >= 1, f"{name} must not be empty")
    N = x.numel() // M
    _same_device(x)
    _require(_fits(N, M), "sizes must fit 32 bits")
    return N, M


def _norm_inputs(x, residual, weight):
    N, M = _norm_rows("x", x)
    if residual is not None:
        _same_device(x, residual=residual)
        _require(residual.shape == x.shape and residual.is_contiguous() and residual.dtype in (x.dtype, torch.float32),
                 "residual must be a contiguous tensor shaped like x, of its dtype or float32")
    _norm_weight(x, weight, M)
    return N, M, x.dtype if residual is None else residual.dtype


def _norm_weight(x, weight, M):
    if weight is not None:
        _same_device(x, weight=weight)
        _ints("weight", weight, x.dtype, (M,))


def rmsnorm_add(x, residual=None, weight=None, y=None, h=None, rstd=None, *, eps=1e-6, weight_offset=0.0, stream=None):
    """h = x + residual, rstd = 1 / sqrt(mean(h^2) + eps), y = h rstd (weight + weight_offset).

    x [..., M] (float16, bfloat16 or float32, contiguous, M at most 32768),
    ``residual`` like x or in float32, ``weight`` [M] of x's dtype (None: ones, and no
    offset).  h has the residual's dtype, and is x itself without a residual; y has x's; ``rstd`` [...]
    is float32.  y may be x itself and h the residual; otherwise outputs share
    memory with nothing.  Nothing is recorded for autograd: a program that trains
    calls rmsnorm_add_bwd.  Returns (y, h, rstd).
    """
    r = (_BINDING or _load_binding()).rmsnorm_add(x, residual, weight, y, h, rstd, eps, weight_offset, stream)
    if r is not None:
        return _result(r)
    N, M, wide = _norm_inputs(x, residual, weight)
    _require(residual is not None or h is None, "h without a residual is x")
    stream = _on_device(x, stream)
    y = _given("y", y, x, stream)
    h = x if residual is None else _given("h", h, residual, stream)
    rstd = _given("rstd", rstd, x, stream, x.shape[:-1], torch.float32)
    with torch.cuda.device(x.device):
        _check(load_library().rmsnorm_add(_ptr(x), _ptr(residual), _ptr(weight), _ptr(y),
                                          None if residual is None else _ptr(h), _ptr(rstd), N, M, float(eps),
                                          float(weight_offset), _NORM_CODE[x.dtype], _NORM_CODE[wide], _stream(stream)))
    return y, h, rstd


def _quant_groups(M, group):
    group = int(group)
    _require(group in (0, 32, 64, 128, 256), "group must be 0 (the whole row), 32, 64, 128 or 256")
    return group, -(-M // group) if group else 1


def rmsnorm_add_quant(x, residual=None, weight=None, q=None, scales=None, h=None, rstd=None, *,
                      dtype=torch.float8_e4m3fn, group=0, eps=1e-6, weight_offset=0.0, stream=None):
    """rmsnorm_add with y in 8 bits: codes q [..., M] (``dtype``: float8_e4m3fn or int8)
    and scales [..., groups] (float32), y ~ q * scale.

    ``group`` elements share a scale: 0 for the whole row (one scale), or 32, 64, 128
    or 256 (the last one may be short).  The scale is the group's largest |y| over 448 or 127;
    y / scale is rounded to the nearest, ties to even.  Zeros have scale 0; a group with an infinity or NaN
    has scale NaN.  ``rstd`` [...] float32 is written if given.  h may be the residual
    itself; otherwise outputs share memory with nothing.  Returns (q, scales, h).
    """
    r = (_BINDING or _load_binding()).rmsnorm_add_quant(x, residual, weight, q, scales, h, rstd, dtype, group, eps,
                                                        weight_offset, stream)
    if r is not None:
        return _result(r)
    N, M, wide = _norm_inputs(x, residual, weight)
    _require(dtype in _QUANT8_CODE, "dtype must be float8_e4m3fn or int8")
    group, groups = _quant_groups(M, group)
    _require(residual is not None or h is None, "h without a residual is x")
    stream = _on_device(x, stream)
    q = _given("q", q, x, stream, dtype=dtype)
    scales = _given("scales", scales, x, stream, (*x.shape[:-1], groups), torch.float32)
    h = x if residual is None else _given("h", h, residual, stream)
    if rstd is not None:
        rstd = _given("rstd", rstd, x, stream, x.shape[:-1], torch.float32)
    with torch.cuda.device(x.device):
        _check(load_library().rmsnorm_add_quant(_ptr(x), _ptr(residual), _ptr(weight), _ptr(q), _ptr(scales),
                                                None if residual is None else _ptr(h), _ptr(rstd), N, M, group,
                                                _QUANT8_CODE[dtype], float(eps), float(weight_offset),
                                                _NORM_CODE[x.dtype], _NORM_CODE[wide], _stream(stream)))
    return q, scales, h


def quant8_load(q, scales, y=None, *, group=0, dtype=torch.bfloat16, stream=None):
    """What rows in 8 bits stand for: y [..., M] = q * scale, formed in 32 bits and
    rounded to ``dtype`` (float16, bfloat16 or float32).  q [..., M] float8_e4m3fn or int8, scales [..., groups]
    float32 and ``group`` as for rmsnorm_add_quant.  Returns y."""
    r = (_BINDING or _load_binding()).quant8_load(q, scales, y, group, dtype, stream)
    if r is not None:
        return _result(r)
    _require(q.dim() >= 1 and q.is_contiguous() and q.numel() >= 1, "q must be contiguous [..., M], not empty")
    _require(q.dtype in _QUANT8_CODE, "q must be float8_e4m3fn or int8")
    _require(dtype in _NORM_CODE, "dtype must be float16, bfloat16 or float32")
    M = q.shape[-1]
    group, groups = _quant_groups(M, group)
    _same_device(q, scales=scales)
    _ints("scales", scales, torch.float32, (*q.shape[:-1], groups))
    N = q.numel() // M
    _require(_fits(N, M), "sizes must fit 32 bits")
    stream = _on_device(q, stream)
    y = _given("y", y, q, stream, dtype=dtype)
    with torch.cuda.device(q.device):
        _check(load_library().quant8_load(_ptr(q), _ptr(scales), _ptr(y), N, M, group, _QUANT8_CODE[q.dtype],
                                          _NORM_CODE[dtype], _stream(stream)))
    return y


def rmsnorm_add_bwd_workspace_bytes(N, M):
    return load_library().rmsnorm_add_bwd_workspace_bytes(N, M) if _fits(N, M) else 0


def rmsnorm_add_bwd(dy, h, rstd, weight=None, dh=None, dx=None, dresidual=None, dweight=None, *, weight_offset=0.0,
                    workspace=None, stream=None):
    """Gradients of rmsnorm_add.

    ``dy`` [..., M] is the gradient of y, ``h`` and ``rstd`` what rmsnorm_add
    returned, ``dh`` (like h, or None) the gradient that reaches h past the norm, as a
    residual stream has one.  Returns (dx, dresidual, dweight): dx of dy's dtype;
    dresidual of h's, which is dx itself where they are one dtype; dweight [M] float32, None
    without a weight.  ``workspace`` (uint8 GPU tensor of rmsnorm_add_bwd_workspace_bytes(N, M)) is allocated
    when not given.  dx may be dy itself, or dh of its dtype, and dresidual dh; otherwise what is
    written shares memory with nothing.
    """
    r = (_BINDING or _load_binding()).rmsnorm_add_bwd(dy, h, rstd, weight, dh, dx, dresidual, dweight, weight_offset,
                                                      workspace, stream)
    if r is not None:
        return _result(r)
    N, M = _norm_rows("dy", dy)
    _same_device(dy, h=h, rstd=rstd)
    _require(h.shape == dy.shape and h.is_contiguous() and h.dtype in (dy.dtype, torch.float32),
             "h must be a contiguous tensor shaped like dy, of its dtype or float32")
    _ints("rstd", rstd, torch.float32, dy.shape[:-1])
    _norm_weight(dy, weight, M)
    if dh is not None:
        _same_device(dy, dh=dh)
        _ints("dh", dh, h.dtype, h.shape)
    same = h.dtype == dy.dtype
    _require(not same or dresidual is None, "dresidual of dx's dtype is dx")
    _require(weight is not None or dweight is None, "dweight needs a weight")
    stream = _on_device(dy, stream)
    dx = _given("dx", dx, dy, stream)
    if not same:
        dresidual = _given("dresidual", dresidual, h, stream)
    if weight is not None:
        dweight = _given("dweight", dweight, dy, stream, (M,), torch.float32)
        if workspace is None:
            _require(isinstance(stream, torch.cuda.Stream), "a stream of this kind needs a workspace of the caller's")
            workspace = _allocate((max(rmsnorm_add_bwd_workspace_bytes(N, M), 16),), dy, stream, torch.uint8)
    if workspace is not None:
        _same_device(dy, workspace=workspace)
        _require(workspace.is_contiguous(), "workspace must be contiguous")
    with torch.cuda.device(dy.device):
        _check(load_library().rmsnorm_add_bwd(_ptr(dy), _ptr(h), _ptr(rstd), _ptr(weight), _ptr(dh), _ptr(dx),
                                              None if same else _ptr(dresidual), _ptr(dweight), N, M,
                                              float(weight_offset), _ptr(workspace),
                                              0 if workspace is None else workspace.numel() * workspace.element_size(),
                                              _NORM_CODE[dy.dtype], _NORM_CODE[h.dtype], _stream(stream)))
    return dx, dx if same else dresidual, dweight


def norm_partials(workspace, N, chunks):
    """View a norm workspace as (r [N, chunks], t [N, chunks]) float32."""
    f = workspace.view(torch.float32)
    n = N * chunks
    return f[:n].view(N, chunks), f[n:2 * n].view(N, chunks)


def decode_partials(workspace, B, Hq, D, num_splits):
    """View the decode workspace as (o_l [B,Hq,S,D], max_l [B,Hq,S], sum_l [B,Hq,S]) fp32."""
    n = B * Hq * num_splits
    f = workspace.view(torch.float32)
    return (f[:n * D].view(B, Hq, num_splits, D), f[n * D:n * D + n].view(B, Hq, num_splits),
            f[n * D + n:n * D + 2 * n].view(B, Hq, num_splits))
