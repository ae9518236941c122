"""Python binding of ``libvd.so`` (argument marshalling only).

The names follow the C ABI in ``include/vd.h``.  Tensors are torch tensors on
the GPU: torch supplies device memory and the stream, every step of the pass
runs in the library's HIP kernels.  There is no fallback: if the library is
missing or a call is rejected, an exception is raised.

Cache tensors ``k`` and ``v`` are 5-D views ``[seq, layer, kv_head, slot,
head_dim]`` with any strides whose last one is 1 (a per-layer ``[seq, slot,
kv_head, head_dim]`` cache is ``x.permute(0, 2, 1, 3).unsqueeze(1)``).
Per-unit arrays are ``[seq, layer, kv_head, ...]`` contiguous, i.e. unit
``u = (s * layers + l) * kv_heads + h``.
"""
import array
import contextlib
import ctypes
import os
from typing import NamedTuple

import torch
from torch.autograd import forward_ad
from torch.utils._device import DeviceContext

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libvd.so")

VD_OK, VD_ERR_INVALID_ARG, VD_ERR_UNSUPPORTED, VD_ERR_WORKSPACE, VD_ERR_HIP = range(5)
VD_DTYPE_BF16, VD_DTYPE_F32 = 0, 1
VARIANTS = {"l2": 0, "dir": 1, "norm": 2, "key_l2": 3, "key_dir": 4, "key_norm": 5,
            "fastcaote": 6}
MAX_CAPACITY = 16384

EXPORTS = ("vd_score", "vd_select_topn", "vd_compact", "vd_evict_step",
           "vd_evict_step_workspace_size", "vd_evict_step_split",
           "vd_evict_step_split_size", "vd_status_string", "vd_stream_read",
           "vd_append", "vd_geometry", "vd_decode_attention_evict", "vd_decode_attention_workspace_size",
           "vd_decode_attention_evict_noalloc", "vd_decode_attention_noalloc_max_bytes",
           "vd_append_mx4", "vd_read_mx4", "vd_attention_mx4", "vd_attention_mx4_workspace_size",
           "vd_evict_step_mx4", "vd_qk_norm_rope")


class VdError(RuntimeError):
    def __init__(self, fn, status, msg):
        super().__init__(f"{fn}: {msg} (status {status})")
        self.status = status


class VdCacheDesc(ctypes.Structure):
    _fields_ = [
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
        ("dtype", ctypes.c_int32), ("num_seqs", ctypes.c_int32),
        ("num_layers", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
        ("num_q_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
        ("capacity", ctypes.c_int32),
        ("stride_seq", ctypes.c_int64), ("stride_layer", ctypes.c_int64),
        ("stride_head", ctypes.c_int64), ("stride_slot", ctypes.c_int64),
    ]


class VdMx4Cache(ctypes.Structure):
    _fields_ = [(x, ctypes.c_void_p) for x in ("k", "v", "k_scale", "v_scale")] + [
        (x, ctypes.c_int32) for x in ("num_seqs", "num_layers", "num_kv_heads", "num_q_heads", "head_dim", "capacity")] + [
        (x, ctypes.c_int64) for x in ("stride_seq", "stride_layer", "stride_head", "stride_slot",
                                      "scale_seq", "scale_layer", "scale_head", "scale_slot")]


_Strides4 = ctypes.c_int64 * 4


class VdRopeSide(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("out", ctypes.c_void_p), ("weight", ctypes.c_void_p),
                ("strides", _Strides4), ("out_strides", _Strides4),
                ("heads", ctypes.c_int32), ("out_dtype", ctypes.c_int32)]


class VdRopeArgs(ctypes.Structure):
    _fields_ = [("q", VdRopeSide), ("k", VdRopeSide), ("pos", ctypes.c_void_p), ("inv_freq", ctypes.c_void_p)] + [
        (x, ctypes.c_int32) for x in ("dtype", "weight_dtype", "num_seqs", "num_layers", "rows", "head_dim", "rotary",
                                      "interleaved")] + [("eps", ctypes.c_float)]


_lib = None


def load():
    """Loads ``libvd.so``; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                           "`python -m paper_2609_23314_amd.build`")
    lib = ctypes.CDLL(LIB_PATH)
    P, I32, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    D = ctypes.POINTER(VdCacheDesc)
    lib.vd_score.argtypes = [D, P, I32, P, P, P]
    lib.vd_select_topn.argtypes = [D, P, P, P, P, P]
    lib.vd_compact.argtypes = [D, P, P, P, P, P]
    lib.vd_evict_step.argtypes = [D, P, P, I32, P, P, P, P, P, SZ, P]
    lib.vd_evict_step_split.argtypes = lib.vd_evict_step.argtypes
    lib.vd_evict_step_split_size.argtypes = [D]
    lib.vd_evict_step_split_size.restype = ctypes.c_size_t
    for f in ("vd_score", "vd_select_topn", "vd_compact", "vd_evict_step", "vd_evict_step_split"):
        getattr(lib, f).restype = ctypes.c_int
    lib.vd_evict_step_workspace_size.argtypes = [D]
    lib.vd_evict_step_workspace_size.restype = ctypes.c_size_t
    lib.vd_status_string.argtypes = [ctypes.c_int]
    lib.vd_status_string.restype = ctypes.c_char_p
    lib.vd_stream_read.argtypes = [P, SZ, P, P]
    lib.vd_stream_read.restype = ctypes.c_int
    lib.vd_append.argtypes = [D, I32, I32, I32, P, P, P, P, P, I32, P]
    lib.vd_append.restype = ctypes.c_int
    lib.vd_geometry.argtypes = [D, P, P, P, P, P]
    lib.vd_geometry.restype = ctypes.c_int
    lib.vd_decode_attention_evict.argtypes = [D, P, ctypes.c_float, P, P, I32, P, P, P, P, SZ, P]
    lib.vd_decode_attention_evict.restype = ctypes.c_int
    lib.vd_decode_attention_workspace_size.argtypes = [D, I32]
    lib.vd_decode_attention_evict_noalloc.argtypes = [D, P, ctypes.c_float, P, P, I32, P, P, P, P]
    lib.vd_decode_attention_evict_noalloc.restype = ctypes.c_int
    lib.vd_decode_attention_noalloc_max_bytes.argtypes = []
    lib.vd_decode_attention_noalloc_max_bytes.restype = ctypes.c_size_t
    lib.vd_decode_attention_workspace_size.restype = ctypes.c_size_t
    M = ctypes.POINTER(VdMx4Cache)
    lib.vd_append_mx4.argtypes = [M, P, P, I32, I32, P, P, P, P, P, P, P]
    lib.vd_read_mx4.argtypes = [M, P, P, I32, I32, P, P, P, P, P]
    lib.vd_attention_mx4.argtypes = [M, I32, P, P, I32, P, ctypes.c_float, P, P, P, P, SZ, P]
    lib.vd_attention_mx4_workspace_size.argtypes = [M, I32, I32, I32]
    lib.vd_attention_mx4_workspace_size.restype = SZ
    lib.vd_evict_step_mx4.argtypes = [M, P, P, I32, P, P, P, P]
    lib.vd_qk_norm_rope.argtypes = [ctypes.POINTER(VdRopeArgs), P]
    for f in ("vd_append_mx4", "vd_read_mx4", "vd_attention_mx4", "vd_evict_step_mx4", "vd_qk_norm_rope"):
        getattr(lib, f).restype = ctypes.c_int
    _lib = lib
    return lib


def _check(fn, status):
    if status != VD_OK:
        raise VdError(fn, status, load().vd_status_string(status).decode())


def _dtype_code(t):
    if t.dtype == torch.bfloat16:
        return VD_DTYPE_BF16
    if t.dtype == torch.float32:
        return VD_DTYPE_F32
    raise TypeError(f"cache dtype must be bfloat16 or float32, got {t.dtype}")


def cache_desc(v, k=None, num_q_heads=None) -> VdCacheDesc:
    """Descriptor of a 5-D ``[seq, layer, kv_head, slot, head_dim]`` cache view."""
    shape, strides = v.shape, v.stride()
    if len(shape) != 5:
        raise ValueError("v must be a 5-D [seq, layer, kv_head, slot, head_dim] view")
    if strides[4] != 1:
        raise ValueError("the head_dim stride must be 1")
    if k is not None and (k.shape != shape or k.stride() != strides or k.dtype != v.dtype):
        raise ValueError("k must match v in shape, strides and dtype")
    S, L, H, C, Dh = shape
    return VdCacheDesc(None if k is None else k.data_ptr(), v.data_ptr(), _dtype_code(v), S, L, H,
                       H if num_q_heads is None else int(num_q_heads), Dh, C, *strides[:4])


# The host's work for a small pass takes longer than the GPU's (an append and a
# pass over one unit: 33 us against 10), so the few helpers that every call goes
# through keep to plain Python objects: a descriptor filled by its constructor, a
# list of ints as a C array rather than a tensor, the current stream's handle
# without a Stream object (append and pass of one unit 33 -> 24 us, of 32 units 33 -> 27).

def _host_i32(x, S, name):
    """One int32 per sequence as a host array (a ctypes one where x is a list or
    tuple of ints, else a tensor, which converts what torch converts)."""
    if type(x) in (list, tuple) and all(type(i) is int and -2 ** 31 <= i < 2 ** 31 for i in x):
        if len(x) != S:
            raise ValueError(f"{name} must have one entry per sequence ({S})")
        return (ctypes.c_int32 * S)(*x)
    t = torch.as_tensor(x, dtype=torch.int32).reshape(-1).cpu().contiguous()
    if t.numel() != S:
        raise ValueError(f"{name} must have one entry per sequence ({S})")
    return t


def _ptr(t):
    if t is None:
        return None
    return ctypes.addressof(t) if isinstance(t, ctypes.Array) else t.data_ptr()


def _stream(dev, stream):
    if stream is None and dev.type == "cuda" and dev.index is not None:
        return torch._C._cuda_getCurrentRawStream(dev.index)
    s = stream if stream is not None else torch.cuda.current_stream(dev)
    return s.cuda_stream


def _units(v):
    S, L, H = v.shape[:3]
    return S * L * H


def _need(t, name, dtype, numel, dev):
    if t.dtype != dtype or not t.is_contiguous() or t.numel() < numel or t.device != dev:
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of >= {numel} "
                         f"elements on {dev}")


def vd_score(v, n_valid, variant="l2", scores=None, mean_out=None, *, k=None,
             num_q_heads=None, stream=None):
    """Mean and scores of every unit; returns (scores [U, cap] f32, mean_out or None)."""
    U, C, Dh = _units(v), v.shape[3], v.shape[4]
    desc = cache_desc(v, k, num_q_heads)
    n_h = _host_i32(n_valid, v.shape[0], "n_valid")
    if scores is None:
        scores = torch.empty((U, C), dtype=torch.float32, device=v.device)
    _need(scores, "scores", torch.float32, U * C, v.device)
    if mean_out is not None:
        _need(mean_out, "mean_out", torch.float32, U * Dh, v.device)
    _check("vd_score", load().vd_score(ctypes.byref(desc), _ptr(n_h), VARIANTS[variant],
                                       _ptr(scores), _ptr(mean_out), _stream(v.device, stream)))
    return scores, mean_out


def vd_select_topn(v, scores, n_valid, budget, keep_mask=None, *, stream=None):
    """Keep mask (uint8 [U, cap]) of the N highest scores of every unit."""
    U, C = _units(v), v.shape[3]
    desc = cache_desc(v)
    n_h = _host_i32(n_valid, v.shape[0], "n_valid")
    b_h = _host_i32(budget, v.shape[0], "budget")
    _need(scores, "scores", torch.float32, U * C, v.device)
    if keep_mask is None:
        keep_mask = torch.empty((U, C), dtype=torch.uint8, device=v.device)
    _need(keep_mask, "keep_mask", torch.uint8, U * C, v.device)
    _check("vd_select_topn", load().vd_select_topn(ctypes.byref(desc), _ptr(scores), _ptr(n_h),
                                                   _ptr(b_h), _ptr(keep_mask),
                                                   _stream(v.device, stream)))
    return keep_mask


def vd_compact(k, v, keep_mask, n_valid, budget, pos=None, *, stream=None):
    """Slot-reuse gather of K, V (and pos) from a keep mask, in place."""
    U, C = _units(v), v.shape[3]
    desc = cache_desc(v, k)
    n_h = _host_i32(n_valid, v.shape[0], "n_valid")
    b_h = _host_i32(budget, v.shape[0], "budget")
    _need(keep_mask, "keep_mask", torch.uint8, U * C, v.device)
    if pos is not None:
        _need(pos, "pos", torch.int32, U * C, v.device)
    _check("vd_compact", load().vd_compact(ctypes.byref(desc), _ptr(keep_mask), _ptr(n_h),
                                           _ptr(b_h), _ptr(pos), _stream(v.device, stream)))


def vd_evict_step_workspace_size(v, k=None):
    desc = cache_desc(v, k)
    return int(load().vd_evict_step_workspace_size(ctypes.byref(desc)))


def vd_evict_step_split_size(v, k=None):
    """Bytes of scratch that ``vd_evict_step`` can use to split units; 0: none."""
    desc = cache_desc(v, k)
    return int(load().vd_evict_step_split_size(ctypes.byref(desc)))


def _call_scratch(size, dev, stream):
    """``size`` bytes of torch's allocator for one call on its stream, which are
    handed on in that stream's order once the call is queued (under torch's capture they
    come from the graph's own pool and live as long as the graph); None where
    there is no memory for them."""
    try:
        if stream is None:
            return torch.empty(size, dtype=torch.uint8, device=dev)
        at = stream
        if not isinstance(stream, torch.cuda.Stream):  # (torch would take the handle 0 as a wish for a new stream)
            handle = stream.cuda_stream
            at = torch.cuda.ExternalStream(handle, dev) if handle else torch.cuda.default_stream(dev)
        with torch.cuda.stream(at):
            return torch.empty(size, dtype=torch.uint8, device=dev)
    except torch.OutOfMemoryError:
        return None


def vd_evict_step(k, v, n_valid, budget, variant="l2", running_sum=None, pos=None,
                  scores_out=None, keep_out=None, workspace=None, *, num_q_heads=None,
                  stream=None, scratch=None):
    """One eviction pass over every unit, in place (see ``vd_evict_step`` in vd.h).
    With ``scratch`` (a uint8 tensor of ``vd_evict_step_split_size`` bytes, not
    shared by calls that overlap, or True: the call takes its own from torch) a
    pass over few units spreads each of them over several workgroups
    (``vd_evict_step_split`` in vd.h, which takes no ``workspace``)."""
    U, C, Dh = _units(v), v.shape[3], v.shape[4]
    desc = cache_desc(v, k, num_q_heads)
    n_h = _host_i32(n_valid, v.shape[0], "n_valid")
    b_h = _host_i32(budget, v.shape[0], "budget")
    if running_sum is not None:
        _need(running_sum, "running_sum", torch.float64, U * (Dh + 1), v.device)
    if pos is not None:
        _need(pos, "pos", torch.int32, U * C, v.device)
    if scores_out is not None:
        _need(scores_out, "scores_out", torch.float32, U * C, v.device)
    if keep_out is not None:
        _need(keep_out, "keep_out", torch.uint8, U * C, v.device)
    if scratch is True:
        size = load().vd_evict_step_split_size(ctypes.byref(desc))
        scratch = _call_scratch(size, v.device, stream) if size else None
    if scratch is not None:
        _need(scratch, "scratch", torch.uint8, 0, v.device)
        _check("vd_evict_step_split", load().vd_evict_step_split(
            ctypes.byref(desc), _ptr(n_h), _ptr(b_h), VARIANTS[variant], _ptr(running_sum),
            _ptr(pos), _ptr(scores_out), _ptr(keep_out), _ptr(scratch), scratch.numel(),
            _stream(v.device, stream)))
        return
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check("vd_evict_step", load().vd_evict_step(
        ctypes.byref(desc), _ptr(n_h), _ptr(b_h), VARIANTS[variant], _ptr(running_sum),
        _ptr(pos), _ptr(scores_out), _ptr(keep_out), _ptr(workspace), ws_bytes,
        _stream(v.device, stream)))


_Strides3 = ctypes.c_int64 * 3


_compiling, _tracing = torch.compiler.is_compiling, torch._C._is_tracing
_dispatch_modes, _function_modes = torch._C._len_torch_dispatch_stack, torch._C._len_torch_function_stack
_transform = torch._C._functorch.peek_interpreter_stack


def _torch_follows():
    """Whether torch itself follows what is done to tensors just now: a compile or a
    trace, a dispatch or function mode (other than a default device's), a functorch
    transform, a forward-mode level.  A kernel launched past torch would escape it."""
    return (_compiling() or _tracing() or _dispatch_modes() > 0 or forward_ad._current_level >= 0
            or _transform() is not None
            or (_function_modes() > 0 and
                any(type(m) is not DeviceContext for m in torch.overrides._get_current_function_mode_stack())))


def _append_strides(x, dtype, dev, L, H, D):
    """The strides of rows that the append kernel reads, else None."""
    if not (type(x) is torch.Tensor and x.dtype == dtype and x.device == dev):
        return None
    shape = x.shape
    if len(shape) != 4 or shape[0] != L or shape[1] != H or shape[3] != D or x.requires_grad or x.is_neg():
        return None
    strides = x.stride()
    return strides if strides[3] == 1 else None


def vd_append(k, v, seq, n_old, k_rows, v_rows, pos=None, pos0=0):
    """Rows [L, H, t, D] into slots [n_old, n_old + t) of sequence ``seq`` and
    their indices pos0 + r into ``pos``, on the current stream.  True if the
    library took the call; False, with nothing queued, for rows or caches that
    are not what its kernel reads (another dtype, device or layout, rows that
    overlap the cache) or while torch follows copies (a transform, a trace, a
    mode), which a caller then makes with torch."""
    if _torch_follows():
        return False
    if not (type(k) is torch.Tensor and type(v) is torch.Tensor and v.is_cuda):
        return False
    shape, strides, dtype, dev = v.shape, v.stride(), v.dtype, v.device
    if not (len(shape) == 5 and strides[4] == 1 and k.shape == shape and k.stride() == strides and k.dtype == dtype
            and k.device == dev and dtype in (torch.bfloat16, torch.float32)):
        return False
    if k.requires_grad or v.requires_grad or k.is_neg() or v.is_neg():
        return False
    if (k.is_inference() or v.is_inference() or (pos is not None and pos.is_inference())) and not torch.is_inference_mode_enabled():
        return False
    S, L, H, C, D = shape
    seq, n_old, pos0 = int(seq), int(n_old), int(pos0)
    ks, vs = _append_strides(k_rows, dtype, dev, L, H, D), _append_strides(v_rows, dtype, dev, L, H, D)
    if ks is None or vs is None:
        return False
    t = k_rows.shape[2]
    if not (v_rows.shape[2] == t and t > 0 and 0 <= seq < S and 0 <= n_old <= C and 0 <= pos0 < 2 ** 31):
        return False
    if pos is not None and not (type(pos) is torch.Tensor and pos.dtype == torch.int32 and pos.device == dev
                                and pos.shape == (S * L * H, C) and pos.is_contiguous()):
        return False
    if dev.index != torch._C._cuda_getDevice():
        return False
    desc = VdCacheDesc(k.data_ptr(), v.data_ptr(), VD_DTYPE_BF16 if dtype == torch.bfloat16 else VD_DTYPE_F32,
                       S, L, H, H, D, C, *strides[:4])
    st = load().vd_append(ctypes.byref(desc), seq, n_old, t, k_rows.data_ptr(), _Strides3(*ks[:3]),
                          v_rows.data_ptr(), _Strides3(*vs[:3]), None if pos is None else pos.data_ptr(), pos0,
                          torch._C._cuda_getCurrentRawStream(dev.index))
    if st in (VD_ERR_INVALID_ARG, VD_ERR_UNSUPPORTED):
        return False
    _check("vd_append", st)
    # torch's backward refuses tensors whose version moved since it saved them
    torch._C._increment_version((k, v) if pos is None else (k, v, pos))
    return True


def vd_geometry(k, v, n_valid, out=None, *, k_sum=None, v_sum=None, stream=None):
    """Key and value geometry of every unit (see ``vd_geometry`` in vd.h):
    float64 [U, 5] = sigma_K, sigma_V, mean ||k - k_bar||, mean ||v - v_bar||,
    bos-cosim.  k_sum / v_sum: optional float64 [U, D + 1] column sums and
    row counts (both or neither)."""
    U, Dh = _units(v), v.shape[4]
    if k is None:
        raise ValueError("vd_geometry needs k")
    desc = cache_desc(v, k)
    n_h = _host_i32(n_valid, v.shape[0], "n_valid")
    if out is None:
        out = torch.empty((U, 5), dtype=torch.float64, device=v.device)
    _need(out, "out", torch.float64, U * 5, v.device)
    for t, nm in ((k_sum, "k_sum"), (v_sum, "v_sum")):
        if t is not None:
            _need(t, nm, torch.float64, U * (Dh + 1), v.device)
    _check("vd_geometry", load().vd_geometry(ctypes.byref(desc), _ptr(n_h), _ptr(k_sum),
                                             _ptr(v_sum), _ptr(out), _stream(v.device, stream)))
    return out


def vd_decode_attention_workspace_size(k, v, num_q_heads, variant="l2"):
    desc = cache_desc(v, k, num_q_heads)
    return int(load().vd_decode_attention_workspace_size(ctypes.byref(desc), VARIANTS[variant]))


def _decode_args(k, v, q, n_valid, budget, running_sum, pos, out):
    if k is None:
        raise ValueError("the fused decode step needs k")
    S, L, H, C, Dh = v.shape
    if q.dim() != 4 or q.shape[0] != S or q.shape[1] != L or q.shape[3] != Dh:
        raise ValueError("q must be [S, L, Hq, D] matching the cache")
    U = _units(v)
    desc = cache_desc(v, k, q.shape[2])
    n_h = _host_i32(n_valid, S, "n_valid")
    b_h = _host_i32(budget, S, "budget")
    _need(q, "q", torch.float32, q.numel(), v.device)
    _need(running_sum, "running_sum", torch.float64, U * (Dh + 1), v.device)
    if pos is not None:
        _need(pos, "pos", torch.int32, U * C, v.device)
    if out is None:
        out = torch.empty(q.shape, dtype=torch.float32, device=v.device)
    _need(out, "out", torch.float32, q.numel(), v.device)
    return desc, n_h, b_h, out


def vd_decode_attention_evict(k, v, q, n_valid, budget, running_sum, scale=None, pos=None,
                              out=None, workspace=None, *, variant="l2", stream=None):
    """One decode step fused with its eviction (see ``vd_decode_attention_evict``
    in vd.h): q is float32 [S, L, Hq, D]; returns the attention output (float32,
    q's shape).  K, V, pos and the running sum are updated in place.  variant is
    "l2" (ValueDiff) or "fastcaote"."""
    desc, n_h, b_h, out = _decode_args(k, v, q, n_valid, budget, running_sum, pos, out)
    if workspace is None:
        ws_need = int(load().vd_decode_attention_workspace_size(ctypes.byref(desc), VARIANTS[variant]))
        workspace = torch.zeros(max(ws_need, 16), dtype=torch.uint8, device=v.device)
    ws_bytes = workspace.numel() * workspace.element_size()
    sc = float(v.shape[4]) ** -0.5 if scale is None else float(scale)
    _check("vd_decode_attention_evict", load().vd_decode_attention_evict(
        ctypes.byref(desc), _ptr(q), sc, _ptr(n_h), _ptr(b_h), VARIANTS[variant],
        _ptr(running_sum), _ptr(pos), _ptr(out), _ptr(workspace), ws_bytes,
        _stream(v.device, stream)))
    return out


def vd_decode_attention_evict_noalloc(k, v, q, n_valid, budget, running_sum, out, scale=None,
                                      pos=None, *, variant="l2", stream=None):
    """The fused decode step without a workspace (see
    ``vd_decode_attention_evict_noalloc`` in vd.h): the library's static device
    scratch holds the split partials.  ``out`` is required (float32, q's
    shape); nothing is allocated here."""
    if out is None:
        raise ValueError("out is required: the allocation-free call allocates nothing")
    desc, n_h, b_h, out = _decode_args(k, v, q, n_valid, budget, running_sum, pos, out)
    sc = float(v.shape[4]) ** -0.5 if scale is None else float(scale)
    _check("vd_decode_attention_evict_noalloc", load().vd_decode_attention_evict_noalloc(
        ctypes.byref(desc), _ptr(q), sc, _ptr(n_h), _ptr(b_h), VARIANTS[variant],
        _ptr(running_sum), _ptr(pos), _ptr(out), _stream(v.device, stream)))
    return out


def vd_decode_attention_noalloc_max_bytes():
    return int(load().vd_decode_attention_noalloc_max_bytes())


# ------------------------------------------------- a cache in 4 bits, and its rows

class Mx4Cache(NamedTuple):
    """A KV cache in 4 bits (see "A KV cache held in 4 bits" in vd.h): uint8
    codes [seq, layer, kv_head, slot, head_dim / 2] and scales [seq, layer,
    kv_head, slot, head_dim / 32], views of any strides whose last one is 1; k and
    v alike, k_scale and v_scale alike."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor

    @classmethod
    def zeros(cls, num_seqs, num_layers, num_kv_heads, capacity, head_dim, device="cuda"):
        shape = (num_seqs, num_layers, num_kv_heads, capacity)
        return cls(*(torch.zeros((*shape, head_dim // n), dtype=torch.uint8, device=device) for n in (2, 2, 32, 32)))

    def seq(self, s):
        """The cache of sequence ``s`` alone (a view)."""
        if not 0 <= s < self.k.shape[0]:
            raise IndexError(f"no sequence {s}")
        return Mx4Cache(*(x[s:s + 1] for x in self))


# As above: what every call goes through keeps to few and plain Python steps (the host's
# time for sixteen sequences' append and read-back 31 -> 24 us, for one layer's attention
# 18 -> 14, where the GPU takes 7 and 18).

def mx4_desc(cache, num_q_heads=None) -> VdMx4Cache:
    """Descriptor of an ``Mx4Cache``."""
    k, v, ks, vs = cache
    shape, sshape, strides, sstrides, dev = k.shape, ks.shape, k.stride(), ks.stride(), k.device
    if len(shape) != 5 or v.shape != shape or len(sshape) != 5 or vs.shape != sshape:
        raise ValueError("codes and scales must be 5-D [seq, layer, kv_head, slot, bytes] views, k and v alike")
    S, L, H, C, B = shape
    if sshape != (S, L, H, C, B // 16) or B % 16:
        raise ValueError("a row of head_dim channels has head_dim / 2 bytes of codes and head_dim / 32 of scales")
    if v.stride() != strides or vs.stride() != sstrides or strides[4] != 1 or (sstrides[4] != 1 and B > 16):
        raise ValueError("k and v must have the same strides, and the last one must be 1")
    if not (k.dtype == v.dtype == ks.dtype == vs.dtype == torch.uint8 and v.device == dev and ks.device == dev
            and vs.device == dev and k.is_cuda):
        raise ValueError("codes and scales must be uint8 tensors on one GPU")
    return VdMx4Cache(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), S, L, H,
                      H if num_q_heads is None else num_q_heads, 2 * B, C, *strides[:4], *sstrides[:4])


_grad_enabled = torch.is_grad_enabled


def _no_grad(name):
    """These calls have no backward: an input that asks for one is refused."""
    raise ValueError(f"{name} has no gradient: detach its inputs or call it under torch.no_grad()")


def _rows_view(x, name, shape, dtype, dev):
    """Pointer and strides of a 5-D [seq, layer, head, row, head_dim] view."""
    if x.shape != shape or x.dtype != dtype or x.device != dev or x.is_neg():
        raise ValueError(f"{name} must be a {dtype} tensor {list(shape)} on {dev}")
    strides = x.stride()
    if strides[4] != 1:
        raise ValueError(f"{name}: the head_dim stride must be 1")
    return x.data_ptr(), _Strides4(*strides[:4])


def _host_list(x, S, name):
    """``_host_i32`` for what mostly is a list of S ints; and its address."""
    if type(x) is list and len(x) == S:
        try:
            made = array.array("i", x)   # (checks types and range)
            return made, made.buffer_info()[0]
        except (TypeError, OverflowError):
            pass
    made = _host_i32(x, S, name)
    return made, _ptr(made)


_no_list = (None, None)
_nothing = contextlib.nullcontext()


def _on(dev, stream):
    """The device of the call's tensors made the current one, where it is not, and the
    caller's stream torch's, where it gives one: what the call allocates belongs to it."""
    if stream is None:
        return _nothing if torch._C._cuda_getDevice() == dev.index else torch.cuda.device(dev)
    if isinstance(stream, torch.cuda.Stream):
        return torch.cuda.stream(stream)
    handle = stream.cuda_stream
    return torch.cuda.stream(torch.cuda.ExternalStream(handle, dev) if handle else torch.cuda.default_stream(dev))


def _moved(*tensors):
    """torch's backward refuses tensors whose version moved since it saved them."""
    try:
        torch._C._increment_version(tensors)
    except RuntimeError:   # an inference tensor, which keeps no version
        torch._C._increment_version(tuple(t for t in tensors if not t.is_inference()))


def vd_append_mx4(cache, n_old, k_rows, v_rows, rows=None, pos=None, pos0=None, *, stream=None):
    """Rows [S, L, H, t, D] (bfloat16 or float32) into slots [n_old[s], n_old[s] +
    rows[s]) of every unit, in 4 bits (see ``vd_append_mx4`` in vd.h); rows: t
    each where None.  pos: int32 [U, capacity], given pos0[s] + r (pos0: n_old)."""
    if (k_rows.requires_grad or v_rows.requires_grad) and _grad_enabled():
        _no_grad("vd_append_mx4")
    desc = mx4_desc(cache)
    S, L, H, C, B = cache[0].shape
    dev, dtype, t = cache[0].device, k_rows.dtype, k_rows.shape[3] if k_rows.dim() == 5 else 0
    shape = (S, L, H, t, 2 * B)
    kp, ks = _rows_view(k_rows, "k_rows", shape, dtype, dev)
    vp, vs = _rows_view(v_rows, "v_rows", shape, dtype, dev)
    if pos is not None:
        _need(pos, "pos", torch.int32, S * L * H * C, dev)
    n_h, n_p = _host_list(n_old, S, "n_old")
    r_h, r_p = _no_list if rows is None else _host_list(rows, S, "rows")
    p_h, p_p = _no_list if pos0 is None else _host_list(pos0, S, "pos0")
    with _on(dev, stream):
        _check("vd_append_mx4", load().vd_append_mx4(
            ctypes.byref(desc), n_p, r_p, t, _dtype_code(k_rows), kp, ks, vp, vs, _ptr(pos), p_p,
            _stream(dev, stream)))
    if pos is None:
        _moved(*cache)
    else:
        _moved(*cache, pos)


def vd_read_mx4(cache, first, t, rows=None, k_out=None, v_out=None, *, dtype=torch.bfloat16, stream=None):
    """The values of slots [first[s], first[s] + rows[s]) of every unit (see
    ``vd_read_mx4`` in vd.h); returns (k, v), [S, L, H, t, D] of ``dtype`` or the
    given outputs.  rows: t each where None; others are left as they were."""
    desc = mx4_desc(cache)
    S, L, H, _, B = cache[0].shape
    dev, t = cache[0].device, int(t)
    shape = (S, L, H, t, 2 * B)
    n_h, n_p = _host_list(first, S, "first")
    r_h, r_p = _no_list if rows is None else _host_list(rows, S, "rows")
    with _on(dev, stream):
        if k_out is None:
            k_out = torch.empty(shape, dtype=dtype, device=dev)
        if v_out is None:
            v_out = torch.empty(shape, dtype=k_out.dtype, device=dev)
        if (k_out.requires_grad or v_out.requires_grad) and _grad_enabled():
            _no_grad("vd_read_mx4")
        kp, ks = _rows_view(k_out, "k_out", shape, k_out.dtype, dev)
        vp, vs = _rows_view(v_out, "v_out", shape, k_out.dtype, dev)
        _check("vd_read_mx4", load().vd_read_mx4(ctypes.byref(desc), n_p, r_p, t, _dtype_code(k_out),
                                                 kp, ks, vp, vs, _stream(dev, stream)))
    _moved(k_out, v_out)
    return k_out, v_out


def vd_attention_mx4_workspace_size(cache, num_q_heads, t, n=None, dtype=torch.bfloat16):
    """Bytes of workspace for ``t`` query rows a sequence over at most n cached
    tokens (None: the cache's capacity)."""
    desc = mx4_desc(cache, int(num_q_heads))
    code = VD_DTYPE_BF16 if dtype == torch.bfloat16 else VD_DTYPE_F32
    return int(load().vd_attention_mx4_workspace_size(ctypes.byref(desc), code, int(t), desc.capacity if n is None else int(n)))


def vd_attention_mx4(cache, q, n_valid, rows=None, scale=None, out=None, workspace=None, *, stream=None):
    """Attention of the newest tokens over a 4-bit cache (see ``vd_attention_mx4``
    in vd.h): q is [S, L, Hq, t, D], bfloat16 or float32, any strides whose last
    one is 1; returns the output, q's shape and type.  Query row i of rows[s] (t
    where None) sees the slots j < n_valid[s] - rows[s] + 1 + i.  Without a
    workspace the call takes its own from torch."""
    if q.dim() != 5:
        raise ValueError("q must be [S, L, Hq, t, D] matching the cache")
    if (q.requires_grad or (out is not None and out.requires_grad)) and _grad_enabled():
        _no_grad("vd_attention_mx4")
    S, L, _, _, B = cache[0].shape
    _, _, Hq, t, _ = q.shape
    desc = mx4_desc(cache, Hq)
    dev, dtype, shape = cache[0].device, q.dtype, (S, L, Hq, t, 2 * B)
    qp, qs = _rows_view(q, "q", shape, dtype, dev)
    code = _dtype_code(q)
    n_h, n_p = _host_list(n_valid, S, "n_valid")
    r_h, r_p = _no_list if rows is None else _host_list(rows, S, "rows")
    sc = (2.0 * B) ** -0.5 if scale is None else float(scale)
    lib = load()
    with _on(dev, stream):
        if out is None:
            out = torch.empty(shape, dtype=dtype, device=dev)
        if workspace is None:
            longest = int(max(n_h))
            size = lib.vd_attention_mx4_workspace_size(ctypes.byref(desc), code, t, min(max(longest, 0), desc.capacity))
            ws_p = None
            if size:
                workspace = torch.empty(size, dtype=torch.uint8, device=dev)
                ws_p = workspace.data_ptr()
        else:
            _need(workspace, "workspace", torch.uint8, 0, dev)
            ws_p, size = workspace.data_ptr(), workspace.numel()
        op, os_ = _rows_view(out, "out", shape, dtype, dev)
        _check("vd_attention_mx4", lib.vd_attention_mx4(
            ctypes.byref(desc), code, qp, qs, t, r_p, sc, n_p, op, os_, ws_p, size, _stream(dev, stream)))
    _moved(out)
    return out


def vd_evict_step_mx4(cache, n_valid, budget, variant="l2", pos=None, scores_out=None, keep_out=None, *, stream=None):
    """One eviction pass over every unit of a 4-bit cache, in place (see
    ``vd_evict_step_mx4`` in vd.h)."""
    desc = mx4_desc(cache)
    S, L, H, C, _ = cache[0].shape
    dev, U = cache[0].device, S * L * H
    n_h, n_p = _host_list(n_valid, S, "n_valid")
    b_h, b_p = _host_list(budget, S, "budget")
    if pos is not None:
        _need(pos, "pos", torch.int32, U * C, dev)
    if scores_out is not None:
        _need(scores_out, "scores_out", torch.float32, U * C, dev)
    if keep_out is not None:
        _need(keep_out, "keep_out", torch.uint8, U * C, dev)
    with _on(dev, stream):
        _check("vd_evict_step_mx4", load().vd_evict_step_mx4(
            ctypes.byref(desc), n_p, b_p, VARIANTS[variant], _ptr(pos), _ptr(scores_out), _ptr(keep_out),
            _stream(dev, stream)))
    _moved(*cache, *(x for x in (pos, scores_out, keep_out) if x is not None))


_no_side = VdRopeSide()


def _rope_side(x, out, weight, names, S, L, t, D, dev, w_dtype):
    shape, dtype = (S, L, x.shape[2], t, D), x.dtype
    xp, xs = _rows_view(x, names[0], shape, dtype, dev)
    out_dtype = out.dtype
    op, os_ = _rows_view(out, names[1], shape, out_dtype, dev)
    wp = None
    if weight is not None:
        if weight.dtype != w_dtype or weight.shape != (L, D) or weight.device != dev or not weight.is_contiguous():
            raise ValueError(f"{names[2]} must be a contiguous {w_dtype} tensor [{L}, {D}] on {dev}")
        wp = weight.data_ptr()
    return VdRopeSide(xp, op, wp, xs, os_, shape[2], _dtype_code(out))


def vd_qk_norm_rope(q, k, pos, inv_freq, q_weight=None, k_weight=None, q_out=None, k_out=None, *, eps=1e-6,
                    interleaved=False, stream=None):
    """Norm of each head's query and key rows and their rotation (see
    ``vd_qk_norm_rope`` in vd.h): q [S, L, Hq, t, D] and k [S, L, H, t, D],
    bfloat16 or float32, any strides whose last one is 1, either of them None; pos
    int32 [S, t]; inv_freq float32 [rotary / 2]; weights [L, D], None for no norm.
    Returns (q_out, k_out): new tensors of the inputs' type, or the given ones
    (either type; the input itself for a call in place, or the cache's own slots)."""
    some = k if q is None else q
    if some is None or some.dim() != 5:
        raise ValueError("q or k must be given, [S, L, heads, t, D]")
    for x in (q, k, q_weight, k_weight, q_out, k_out):
        if x is not None and x.requires_grad and _grad_enabled():
            _no_grad("vd_qk_norm_rope")
    S, L, _, t, D = some.shape
    dev, dtype = some.device, some.dtype
    if not some.is_cuda:
        raise ValueError("q and k must be on a GPU")
    if k is not None and q is not None and (k.dim() != 5 or k.dtype != dtype):
        raise ValueError("k must match q in type and device")
    if (q is None and (q_out is not None or q_weight is not None)) or (k is None and (k_out is not None or k_weight is not None)):
        raise ValueError("an output or a weight without its input")
    if pos.shape != (S, t):
        raise ValueError(f"pos must be [{S}, {t}]")
    _need(pos, "pos", torch.int32, 0, dev)
    _need(inv_freq, "inv_freq", torch.float32, 0, dev)
    w = k_weight if q_weight is None else q_weight
    w_dtype = dtype if w is None else w.dtype
    with _on(dev, stream):
        if q is not None and q_out is None:
            q_out = torch.empty(q.shape, dtype=dtype, device=dev)
        if k is not None and k_out is None:
            k_out = torch.empty(k.shape, dtype=dtype, device=dev)
        args = VdRopeArgs(
            _no_side if q is None else _rope_side(q, q_out, q_weight, ("q", "q_out", "q_weight"), S, L, t, D, dev, w_dtype),
            _no_side if k is None else _rope_side(k, k_out, k_weight, ("k", "k_out", "k_weight"), S, L, t, D, dev, w_dtype),
            pos.data_ptr(), inv_freq.data_ptr(), _dtype_code(some), VD_DTYPE_F32 if w is None else _dtype_code(w), S, L, t,
            D, 2 * inv_freq.numel(), 1 if interleaved else 0, eps)
        _check("vd_qk_norm_rope", load().vd_qk_norm_rope(ctypes.byref(args), _stream(dev, stream)))
    if q is None:
        _moved(k_out)
    elif k is None:
        _moved(q_out)
    else:
        _moved(q_out, k_out)
    return q_out, k_out


def vd_stream_read(buf, sink, *, stream=None):
    """One streaming read of the whole of ``buf`` (a measurement aid: the
    practical HBM read ceiling next to the pass); ``sink`` is a device int32
    tensor of at least one element."""
    if not buf.is_contiguous() or sink.dtype != torch.int32 or sink.device != buf.device:
        raise ValueError("buf must be contiguous and sink an int32 tensor on the same device")
    _check("vd_stream_read", load().vd_stream_read(_ptr(buf), buf.numel() * buf.element_size(),
                                                   _ptr(sink), _stream(buf.device, stream)))
