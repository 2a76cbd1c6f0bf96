"""ctypes binding of include/si.h.  Same names as the C entry points.

Tensors are torch tensors on a HIP device (torch is used for device memory
and streams only); descriptors are built from their shapes and data pointers.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, List, Optional, Sequence, Tuple

SI_F32, SI_BF16 = 0, 1
SI_BLOCK_TEMPORAL, SI_BLOCK_SPATIAL = 0, 1
SI_AXIS_F, SI_AXIS_HW = 2, 3

_HERE = os.path.dirname(os.path.abspath(__file__))


def library_path() -> str:
    return os.path.join(_HERE, "libsi.so")


class SiError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: si_status {status} ({si_status_str(status)})")


class _Tensor5(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("dtype", C.c_int32),
                ("B", C.c_int64), ("C", C.c_int64), ("F", C.c_int64), ("H", C.c_int64), ("W", C.c_int64)]


class _Context(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("dtype", C.c_int32),
                ("B", C.c_int64), ("M", C.c_int64), ("Cc", C.c_int64)]


WEIGHT_FIELDS = ("gn_g", "gn_b", "w_in", "b_in", "ln1_g", "ln1_b", "wq", "wk", "wv", "wo", "bo",
                 "ln2_g", "ln2_b", "wq2", "wk2", "wv2", "wo2", "bo2",
                 "ln3_g", "ln3_b", "w1", "b1", "w2", "b2", "w_out", "b_out")


class _Weights(C.Structure):
    _fields_ = ([("kind", C.c_int32), ("heads", C.c_int32), ("dim_head", C.c_int32), ("gn_groups", C.c_int32),
                 ("gn_eps", C.c_float), ("ln_eps", C.c_float), ("add_sin_pe", C.c_int32)]
                + [(n, C.c_void_p) for n in WEIGHT_FIELDS])


RES_WEIGHT_FIELDS = ("gn1_g", "gn1_b", "w_conv1", "b_conv1", "w_temb", "b_temb", "gn2_g", "gn2_b", "w_conv2", "b_conv2")


class _ResWeights(C.Structure):
    _fields_ = ([("gn_groups", C.c_int32), ("gn_eps", C.c_float), ("temb_dim", C.c_int32)]
                + [(n, C.c_void_p) for n in RES_WEIGHT_FIELDS]
                + [("c_out", C.c_int32), ("w_skip", C.c_void_p), ("b_skip", C.c_void_p)])


class _Heads(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("dtype", C.c_int32),
                ("B", C.c_int64), ("N", C.c_int64), ("heads", C.c_int64), ("dim_head", C.c_int64),
                ("stride_b", C.c_int64), ("stride_n", C.c_int64), ("stride_h", C.c_int64)]


class _Rope(C.Structure):
    _fields_ = [("extent", C.c_int64 * 3), ("pairs", C.c_int32 * 3), ("layout", C.c_int32), ("theta", C.c_double),
                ("origin", C.c_double * 3), ("step", C.c_double * 3), ("norm_eps", C.c_float),
                ("q_gain", C.c_void_p), ("k_gain", C.c_void_p)]


class _AttnOptions(C.Structure):
    _fields_ = [("rope", C.POINTER(_Rope)), ("q_block", C.c_int64), ("k_block", C.c_int64), ("keep", C.c_int64)]


class _Cache4(C.Structure):
    _fields_ = [("k_codes", C.c_void_p), ("k_scales", C.c_void_p), ("v_codes", C.c_void_p), ("v_scales", C.c_void_p),
                ("B", C.c_int64), ("heads", C.c_int64), ("capacity", C.c_int64), ("dim_head", C.c_int64)]


class _RehashCache(C.Structure):
    _fields_ = [("x_key", C.c_void_p), ("y_key", C.c_void_p), ("valid", C.c_int32)]


_lib = None


def lib() -> C.CDLL:
    """Loads libsi.so (built in-tree by paper_2411_01171_amd.build); raises if absent."""
    global _lib
    if _lib is not None:
        return _lib
    path = library_path()
    if not os.path.exists(path):
        raise FileNotFoundError(f"{path} not built: run `python -c 'import __graft_entry__ as g; g.build()'`")
    L = C.CDLL(path)
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    L.si_workspace_bytes.restype = sz
    L.si_workspace_bytes.argtypes = [C.POINTER(_Tensor5), C.POINTER(_Weights), C.POINTER(_Context), i32, i64]
    L.si_live_activation_bytes.restype = sz
    L.si_live_activation_bytes.argtypes = L.si_workspace_bytes.argtypes
    L.si_windows_in_flight.restype = i32
    L.si_windows_in_flight.argtypes = L.si_workspace_bytes.argtypes
    L.si_block_forward.restype = i32
    L.si_block_forward.argtypes = [C.POINTER(_Tensor5), C.POINTER(_Weights), C.POINTER(_Context), C.POINTER(_Tensor5),
                                   i32, i64, vp, sz, vp]
    L.si_block_forward_ex.restype = i32
    L.si_block_forward_ex.argtypes = L.si_block_forward.argtypes[:8] + [C.c_uint32, vp]
    L.si_block_forward_rehash.restype = i32
    L.si_block_forward_rehash.argtypes = L.si_block_forward.argtypes[:8] + [
        C.POINTER(_RehashCache), C.c_float, vp, C.POINTER(C.c_double), C.POINTER(i32)]
    L.si_resblock_workspace_bytes.restype = sz
    L.si_resblock_workspace_bytes.argtypes = [C.POINTER(_Tensor5), C.POINTER(_ResWeights), i64]
    L.si_resblock_live_activation_bytes.restype = sz
    L.si_resblock_live_activation_bytes.argtypes = L.si_resblock_workspace_bytes.argtypes
    L.si_resblock_forward.restype = i32
    L.si_resblock_forward.argtypes = [C.POINTER(_Tensor5), C.POINTER(_ResWeights), vp, C.POINTER(_Tensor5), i64, vp, sz, vp]
    L.si_resample_workspace_bytes.restype = sz
    L.si_resample_workspace_bytes.argtypes = [C.POINTER(_Tensor5), i32, i64]
    L.si_resample_forward.restype = i32
    L.si_resample_forward.argtypes = [C.POINTER(_Tensor5), i32, vp, vp, C.POINTER(_Tensor5), i64, vp, sz, vp]
    ph = C.POINTER(_Heads)
    L.si_rope_forward.restype = i32
    L.si_rope_forward.argtypes = [ph, ph, C.POINTER(_Rope), i64, ph, ph, vp]
    L.si_attn_block_words.restype = i64
    L.si_attn_block_words.argtypes = [i64, i64]
    L.si_attn_select_workspace_bytes.restype = sz
    L.si_attn_select_workspace_bytes.argtypes = [ph, ph, i64, i64]
    L.si_attn_select.restype = i32
    L.si_attn_select.argtypes = [ph, ph, i64, i64, i64, vp, vp, vp, vp, sz, vp]
    L.si_attn_sparse_workspace_bytes.restype = sz
    L.si_attn_sparse_workspace_bytes.argtypes = [ph, ph, i64, i64]
    L.si_attn_sparse_forward.restype = i32
    L.si_attn_sparse_forward.argtypes = [ph, ph, ph, i64, i64, C.c_float, vp, vp, vp, ph, vp, sz, vp]
    pc = C.POINTER(_Cache4)
    L.si_cache4_store.restype = i32
    L.si_cache4_store.argtypes = [ph, ph, vp, vp, pc, vp, vp]
    L.si_cache4_load.restype = i32
    L.si_cache4_load.argtypes = [pc, vp, vp, ph, ph, vp]
    L.si_cache4_attn_workspace_bytes.restype = sz
    L.si_cache4_attn_workspace_bytes.argtypes = [ph, pc, i32]
    L.si_cache4_attn_forward.restype = i32
    L.si_cache4_attn_forward.argtypes = [ph, pc, C.c_float, i64, vp, vp, vp, C.c_float, vp, ph, vp, sz, vp]
    L.si_cache4_evict_workspace_bytes.restype = sz
    L.si_cache4_evict_workspace_bytes.argtypes = [pc, i64]
    L.si_cache4_evict.restype = i32
    L.si_cache4_evict.argtypes = [pc, vp, vp, i64, i64, i64, pc, vp, vp, vp, vp, sz, vp]
    po = C.POINTER(_AttnOptions)
    L.si_block_attn_workspace_bytes.restype = sz
    L.si_block_attn_workspace_bytes.argtypes = L.si_workspace_bytes.argtypes[:3] + [po, i32, i64]
    L.si_block_forward_attn.restype = i32
    L.si_block_forward_attn.argtypes = L.si_block_forward.argtypes[:3] + [po, C.POINTER(_Tensor5), i32, i64, vp, sz, C.c_uint32, vp]
    L.si_rehash_scratch_bytes.restype = sz
    L.si_rehash_scratch_bytes.argtypes = [i64]
    L.si_rehash_check.restype = i32
    L.si_rehash_check.argtypes = [vp, vp, i64, i32, C.c_float, vp, vp, vp, vp]
    L.si_rehash_check_sync.restype = i32
    L.si_rehash_check_sync.argtypes = [vp, vp, i64, i32, C.c_float, vp, vp, vp,
                                       C.POINTER(C.c_double), C.POINTER(i32)]
    L.si_init_device.restype = i32
    L.si_init_device.argtypes = []
    L.si_rehash_check_static.restype = i32
    L.si_rehash_check_static.argtypes = [vp, vp, i64, i32, C.c_float, vp, vp, vp]
    L.si_key_step_search.restype = i32
    L.si_key_step_search.argtypes = [C.POINTER(C.c_float), i32, C.c_float, C.POINTER(i32)]
    L.si_stage_timing_enable.restype = None
    L.si_stage_timing_enable.argtypes = [i32]
    L.si_stage_timing_read.restype = i32
    L.si_stage_timing_read.argtypes = [C.POINTER(C.c_char_p), C.POINTER(C.c_double), C.POINTER(i64), i32]
    L.si_status_str.restype = C.c_char_p
    L.si_status_str.argtypes = [i32]
    L.si_abi_version.restype = i32
    L.si_abi_version.argtypes = []
    _lib = L
    return L


def si_status_str(status: int) -> str:
    return lib().si_status_str(int(status)).decode()


def si_abi_version() -> int:
    return int(lib().si_abi_version())


def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.float32:
        return SI_F32
    if t.dtype == torch.bfloat16:
        return SI_BF16
    return -1


def _tensor5(t) -> _Tensor5:
    if t.dim() != 5 or not t.is_contiguous():
        raise ValueError("feature must be a contiguous [B,C,F,H,W] tensor")
    B, Cc, F, H, W = t.shape
    return _Tensor5(t.data_ptr(), _dtype_code(t), B, Cc, F, H, W)


def _context(t) -> Optional[_Context]:
    if t is None:
        return None
    if t.dim() != 3 or not t.is_contiguous():
        raise ValueError("context must be a contiguous [B,M,Cc] tensor")
    return _Context(t.data_ptr(), _dtype_code(t), *t.shape)


class BlockWeights:
    """Holds the device tensors of one block and the matching C struct.

    `tensors` maps the field names of si_block_weights to torch tensors (or
    None); the tensors are kept alive by this object."""

    def __init__(self, kind: int, heads: int, dim_head: int, gn_groups: int, tensors: Dict[str, object],
                 gn_eps: float = 1e-6, ln_eps: float = 1e-5, add_sin_pe: bool = False):
        self.tensors = dict(tensors)
        s = _Weights()
        s.kind, s.heads, s.dim_head, s.gn_groups = kind, heads, dim_head, gn_groups
        s.gn_eps, s.ln_eps, s.add_sin_pe = gn_eps, ln_eps, int(bool(add_sin_pe))
        for name in WEIGHT_FIELDS:
            t = self.tensors.get(name)
            if t is not None and not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous")
            setattr(s, name, None if t is None else t.data_ptr())
        self.struct = s


def _stream_ptr(stream) -> Optional[int]:
    if stream is None:
        import torch
        stream = torch.cuda.current_stream()
    return getattr(stream, "cuda_stream", stream) or None


def _pctx(ctx):
    c = _context(ctx)
    return (C.byref(c) if c is not None else None), c


def si_workspace_bytes(x, weights: BlockWeights, ctx, axis: int, slice_len: int) -> int:
    xd = _tensor5(x)
    pc, _keep = _pctx(ctx)
    return int(lib().si_workspace_bytes(C.byref(xd), C.byref(weights.struct), pc, axis, slice_len))


def si_live_activation_bytes(x, weights: BlockWeights, ctx, axis: int, slice_len: int) -> int:
    xd = _tensor5(x)
    pc, _keep = _pctx(ctx)
    return int(lib().si_live_activation_bytes(C.byref(xd), C.byref(weights.struct), pc, axis, slice_len))


def si_windows_in_flight(x, weights: BlockWeights, ctx, axis: int, slice_len: int) -> int:
    xd = _tensor5(x)
    pc, _keep = _pctx(ctx)
    return int(lib().si_windows_in_flight(C.byref(xd), C.byref(weights.struct), pc, axis, slice_len))


SI_FWD_WEIGHTS_PACKED = 1


def si_block_forward(x, weights: BlockWeights, ctx, out, axis: int, slice_len: int, workspace, stream=None) -> None:
    """Enqueues the sliced block forward on `stream` (default: torch's current stream)."""
    xd, od = _tensor5(x), _tensor5(out)
    pc, _keep = _pctx(ctx)
    st = lib().si_block_forward(C.byref(xd), C.byref(weights.struct), pc, C.byref(od), axis, slice_len,
                                workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                _stream_ptr(stream))
    if st != 0:
        raise SiError(st, "si_block_forward")


def si_block_forward_ex(x, weights: BlockWeights, ctx, out, axis: int, slice_len: int, workspace, flags: int = 0,
                        stream=None) -> None:
    """si_block_forward with flags (SI_FWD_WEIGHTS_PACKED: the workspace still holds these weights re-laid-out)."""
    xd, od = _tensor5(x), _tensor5(out)
    pc, _keep = _pctx(ctx)
    st = lib().si_block_forward_ex(C.byref(xd), C.byref(weights.struct), pc, C.byref(od), axis, slice_len,
                                   workspace.data_ptr(), workspace.numel() * workspace.element_size(), flags,
                                   _stream_ptr(stream))
    if st != 0:
        raise SiError(st, "si_block_forward_ex")


class ResBlockWeights:
    """Device tensors of one Spatial ResBlock and the matching C struct (kept alive by this object)."""

    def __init__(self, gn_groups: int, tensors: Dict[str, object], gn_eps: float = 1e-6, temb_dim: int = 0, c_out: int = 0):
        self.tensors = dict(tensors)
        s = _ResWeights()
        s.gn_groups, s.gn_eps, s.temb_dim, s.c_out = gn_groups, gn_eps, temb_dim, c_out
        for name in RES_WEIGHT_FIELDS + ("w_skip", "b_skip"):
            t = self.tensors.get(name)
            if t is not None and not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous")
            setattr(s, name, None if t is None else t.data_ptr())
        self.struct = s


def si_resblock_workspace_bytes(x, weights: ResBlockWeights, slice_len: int) -> int:
    xd = _tensor5(x)
    return int(lib().si_resblock_workspace_bytes(C.byref(xd), C.byref(weights.struct), slice_len))


def si_resblock_live_activation_bytes(x, weights: ResBlockWeights, slice_len: int) -> int:
    xd = _tensor5(x)
    return int(lib().si_resblock_live_activation_bytes(C.byref(xd), C.byref(weights.struct), slice_len))


def si_resblock_forward(x, weights: ResBlockWeights, temb, out, slice_len: int, workspace, stream=None) -> None:
    """Enqueues the sliced Spatial ResBlock forward (frame windows of `slice_len`) on `stream`."""
    xd, od = _tensor5(x), _tensor5(out)
    if temb is not None and not temb.is_contiguous():
        raise ValueError("temb must be contiguous")
    st = lib().si_resblock_forward(C.byref(xd), C.byref(weights.struct), None if temb is None else temb.data_ptr(),
                                   C.byref(od), slice_len, workspace.data_ptr(),
                                   workspace.numel() * workspace.element_size(), _stream_ptr(stream))
    if st != 0:
        raise SiError(st, "si_resblock_forward")


SI_RESAMPLE_DOWN, SI_RESAMPLE_UP = 0, 1


def si_resample_workspace_bytes(x, kind: int, slice_len: int) -> int:
    xd = _tensor5(x)
    return int(lib().si_resample_workspace_bytes(C.byref(xd), kind, slice_len))


def si_resample_forward(x, kind: int, w_conv, b_conv, out, slice_len: int, workspace, stream=None) -> None:
    """Enqueues the sliced Spatial Down/UpSample (3x3 convolution, stride 2 / after nearest doubling)."""
    xd, od = _tensor5(x), _tensor5(out)
    if not w_conv.is_contiguous() or (b_conv is not None and not b_conv.is_contiguous()):
        raise ValueError("parameters must be contiguous")
    st = lib().si_resample_forward(C.byref(xd), kind, w_conv.data_ptr(), None if b_conv is None else b_conv.data_ptr(),
                                   C.byref(od), slice_len, workspace.data_ptr(),
                                   workspace.numel() * workspace.element_size(), _stream_ptr(stream))
    if st != 0:
        raise SiError(st, "si_resample_forward")


SI_ROPE_INTERLEAVED, SI_ROPE_HALVES = 0, 1


class Rope:
    """Rotary positions on the axes (frame, row, column) of a grid: si_rope.  Keeps the gains alive.

    norm_eps: None, or the heads are RMS-normalised (times q_gain / k_gain) before they turn."""

    def __init__(self, extent: Sequence[int], pairs: Sequence[int], *, theta: float = 1e4, layout: int = SI_ROPE_INTERLEAVED,
                 origin: Sequence[float] = (0.0, 0.0, 0.0), step: Sequence[float] = (1.0, 1.0, 1.0), norm_eps: Optional[float] = None,
                 q_gain=None, k_gain=None):
        self.gains = (q_gain, k_gain)
        s = _Rope()
        s.extent[:], s.pairs[:], s.origin[:], s.step[:] = list(extent), list(pairs), list(origin), list(step)
        s.layout, s.theta, s.norm_eps = layout, theta, -1.0 if norm_eps is None else norm_eps
        if norm_eps is not None and norm_eps < 0:
            raise ValueError("norm_eps must not be negative")
        for g in self.gains:
            if g is not None and (norm_eps is None or g.dim() != 1 or not g.is_contiguous()):
                raise ValueError("gains are contiguous [dim_head] tensors and need norm_eps")
        s.q_gain, s.k_gain = (None if g is None else g.data_ptr() for g in self.gains)
        self.struct = s


def _heads(t) -> _Heads:
    try:
        B, N, h, d = t.shape
    except ValueError:
        raise ValueError("heads must be a [B, N, heads, dim_head] tensor") from None
    sb, sn, sh, sc = t.stride()
    if sc != 1 and d > 1:
        raise ValueError("the channels of heads must be contiguous")
    return _Heads(t.data_ptr(), _dtype_code(t), B, N, h, d, sb, sn, sh)


def _call(name: str, stream, tensors, args) -> None:
    """Calls the entry point with `args` and a stream of the tensors' device (its current one unless given), on that device."""
    import torch
    index = tensors[0].get_device()  # -1: not on a GPU
    for t in tensors:
        if t is not None and t.get_device() != index:
            index = -1
    if index < 0:
        raise ValueError("all tensors must be on one GPU")
    if stream is None:
        st = torch._C._cuda_getCurrentRawStream(index) or None  # torch.cuda.current_stream(index).cuda_stream, without the object
    else:
        st = _stream_ptr(stream)
    fn = getattr(lib(), name)
    if index == torch._C._cuda_getDevice():  # torch.cuda.current_device(); torch has been initialised, a tensor is on the GPU
        status = fn(*args, st)
    else:
        with torch.cuda.device(index):
            status = fn(*args, st)
    if status != 0:
        raise SiError(status, name)


def _lengths(t, B: int) -> Optional[int]:
    if t is None:
        return None
    import torch
    if t.dtype != torch.int32 or t.dim() != 1 or t.shape[0] != B or not t.is_contiguous():
        raise ValueError("lengths must be a contiguous int32 tensor [B]")
    return t.data_ptr()


def _bitmap(t, q, k, q_block: int, k_block: int) -> Optional[int]:
    if t is None:
        return None
    import torch
    if q_block < 1 or k_block < 1:
        raise SiError(2, "key blocks")
    shape = (q.shape[0], k.shape[2], -(-q.shape[1] // q_block), -(-(-(-k.shape[1] // k_block)) // 32))
    if t.dtype != torch.int32 or tuple(t.shape) != shape or not t.is_contiguous():
        raise ValueError(f"blocks must be a contiguous int32 tensor {list(shape)}")
    return t.data_ptr()


def si_rope_forward(q, k, rope: Rope, q_out, k_out, first: int = 0, stream=None) -> None:
    """Rotates the heads of q [B,N,heads,dim_head] and k (or None) into q_out and k_out; token n is grid point first + n."""
    for g in rope.gains:
        if g is not None and (g.shape[0] != q.shape[3] or g.dtype != q.dtype):
            raise ValueError("gains must be [dim_head] in the operands' dtype")
    kd = None if k is None else C.byref(_heads(k))
    ko = None if k_out is None else C.byref(_heads(k_out))
    _call("si_rope_forward", stream, (q, k, q_out, k_out, *rope.gains),
          (C.byref(_heads(q)), kd, C.byref(rope.struct), first, C.byref(_heads(q_out)), ko))


def si_attn_block_words(n_keys: int, k_block: int) -> int:
    return int(lib().si_attn_block_words(n_keys, k_block))


def si_attn_select_workspace_bytes(q, k, q_block: int, k_block: int) -> int:
    qd, kd = _heads(q), _heads(k)
    return int(lib().si_attn_select_workspace_bytes(C.byref(qd), C.byref(kd), q_block, k_block))


def si_attn_select(q, k, q_block: int, k_block: int, keep: int, blocks, workspace, q_len=None, k_len=None, stream=None) -> None:
    """Writes the `keep` best key blocks of every run of q_block queries as bitmaps: blocks int32
    [B, k heads, runs, si_attn_block_words(N of k, k_block)]."""
    ql, kl, bits = _lengths(q_len, q.shape[0]), _lengths(k_len, q.shape[0]), _bitmap(blocks, q, k, q_block, k_block)
    _call("si_attn_select", stream, (q, k, blocks, workspace, q_len, k_len),
          (C.byref(_heads(q)), C.byref(_heads(k)), q_block, k_block, keep, ql, kl, bits, workspace.data_ptr(), workspace.nbytes))


def si_attn_sparse_workspace_bytes(q, k, q_block: int, k_block: int) -> int:
    qd, kd = _heads(q), _heads(k)
    return int(lib().si_attn_sparse_workspace_bytes(C.byref(qd), C.byref(kd), q_block, k_block))


def si_attn_sparse_forward(q, k, v, q_block: int, k_block: int, blocks, out, workspace, scale: Optional[float] = None, q_len=None,
                           k_len=None, stream=None) -> None:
    """Attention of runs of q_block queries over the key blocks in their bitmaps (blocks None: over every key).
    scale: 1/sqrt(dim_head) unless given."""
    ql, kl, bits = _lengths(q_len, q.shape[0]), _lengths(k_len, q.shape[0]), _bitmap(blocks, q, k, q_block, k_block)
    _call("si_attn_sparse_forward", stream, (q, k, v, blocks, out, workspace, q_len, k_len),
          (C.byref(_heads(q)), C.byref(_heads(k)), C.byref(_heads(v)), q_block, k_block, q.shape[3] ** -0.5 if scale is None else scale,
           ql, kl, bits, C.byref(_heads(out)), workspace.data_ptr(), workspace.nbytes))


class Cache4:
    """Keys and values in 4 bits: si_cache4 over uint8 tensors codes [B, heads, capacity, 16 G], scales [B, heads, capacity, S]."""

    def __init__(self, k_codes, k_scales, v_codes, v_scales, dim_head: int):
        import torch
        groups, room = self.row_bytes(dim_head)
        self.tensors = (k_codes, k_scales, v_codes, v_scales)
        for t, n in zip(self.tensors, (groups, room, groups, room)):
            if t.dtype != torch.uint8 or t.dim() != 4 or tuple(t.shape) != (*k_codes.shape[:3], n) or not t.is_contiguous():
                raise ValueError(f"codes and scales must be contiguous uint8 tensors [B, heads, capacity, {groups}] and [.., {room}]")
        self.k_codes, self.k_scales, self.v_codes, self.v_scales = self.tensors
        self.dim_head = dim_head
        self.shape = (*k_codes.shape[:3], dim_head)  # B, heads, capacity, dim_head
        self.slots = self.shape[:3]
        self.struct = _Cache4(*(t.data_ptr() for t in self.tensors), *self.shape)
        index = {t.get_device() for t in self.tensors}
        self.index = index.pop() if len(index) == 1 else -1  # the GPU that holds all of it

    def get_device(self) -> int:
        return self.index

    @staticmethod
    def row_bytes(dim_head: int) -> Tuple[int, int]:
        """Bytes of a token's codes and of its scales."""
        if dim_head < 8 or dim_head > 128 or dim_head % 8:
            raise ValueError("dim_head must be a multiple of 8, at most 128")
        groups = -(-dim_head // 32)
        return 16 * groups, (1, 2, 4, 4)[groups - 1]

    @classmethod
    def empty(cls, B: int, heads: int, capacity: int, dim_head: int, device="cuda") -> "Cache4":
        import torch
        codes, scales = cls.row_bytes(dim_head)
        return cls(*(torch.empty(B, heads, capacity, n, dtype=torch.uint8, device=device) for n in (codes, scales, codes, scales)), dim_head)


def _weights(t, cache: Cache4, what: str) -> Optional[int]:
    if t is None:
        return None
    import torch
    if t.dtype != torch.float32 or t.shape != cache.slots or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous float32 tensor {list(cache.slots)}")
    return t.data_ptr()


def si_cache4_store(k, v, cache: Cache4, first=None, length=None, weight=None, stream=None) -> None:
    """Stores the tokens of k and v [B,N,heads,dim_head] from slot first[b] on (int32 [B]; None: 0), length[b] of them (None: N).
    weight: zeroed at these slots."""
    B = cache.shape[0]
    args = (C.byref(_heads(k)), C.byref(_heads(v)), _lengths(first, B), _lengths(length, B), C.byref(cache.struct), _weights(weight, cache, "weight"))
    _call("si_cache4_store", stream, (k, v, cache, first, length, weight), args)


def si_cache4_load(cache: Cache4, k, v, first=None, length=None, stream=None) -> None:
    """Writes what slots first[b] + n stand for to the tokens of k and v."""
    B = cache.shape[0]
    args = (C.byref(cache.struct), _lengths(first, B), _lengths(length, B), C.byref(_heads(k)), C.byref(_heads(v)))
    _call("si_cache4_load", stream, (k, v, cache, first, length), args)


def si_cache4_attn_workspace_bytes(q, cache: Cache4, weights: bool = False) -> int:
    return int(lib().si_cache4_attn_workspace_bytes(C.byref(_heads(q)), C.byref(cache.struct), int(bool(weights))))


def si_cache4_attn_forward(q, cache: Cache4, out, workspace, scale: Optional[float] = None, q_len=None, k_len=None, run: int = 0,
                           weight_in=None, weight_out=None, decay: float = 1.0, stream=None) -> None:
    """Attention of q [B,N,heads,dim_head] over the first k_len[b] slots; run > 0: a query sees no later run of `run` queries.
    scale: 1/sqrt(dim_head) unless given.  weight_out = decay * weight_in + the softmax weight that every slot received."""
    B = cache.shape[0]
    args = (C.byref(_heads(q)), C.byref(cache.struct), q.shape[3] ** -0.5 if scale is None else scale, run, _lengths(q_len, B), _lengths(k_len, B),
            _weights(weight_in, cache, "weight_in"), decay, _weights(weight_out, cache, "weight_out"), C.byref(_heads(out)),
            workspace.data_ptr(), workspace.nbytes)
    _call("si_cache4_attn_forward", stream, (q, out, cache, workspace, q_len, k_len, weight_in, weight_out), args)


def si_cache4_evict_workspace_bytes(cache: Cache4, keep: int) -> int:
    return int(lib().si_cache4_evict_workspace_bytes(C.byref(cache.struct), keep))


def si_cache4_evict(cache: Cache4, weight, keep: int, out: Cache4, weight_out, kept, out_len, workspace, first: int = 0, last: int = 0,
                    k_len=None, stream=None) -> None:
    """Moves the `keep` slots that stay (the first `first`, the last `last`, and the largest weights between) to `out`, with their
    weights; kept int32 [B, heads, keep] receives the slots that they had, out_len int32 [B] how many there are."""
    import torch
    B, heads = cache.shape[:2]
    if kept.dtype != torch.int32 or tuple(kept.shape) != (B, heads, keep) or not kept.is_contiguous():
        raise ValueError(f"kept must be a contiguous int32 tensor {[B, heads, keep]}")
    args = (C.byref(cache.struct), _lengths(k_len, B), _weights(weight, cache, "weight"), keep, first, last, C.byref(out.struct),
            _weights(weight_out, out, "weight_out"), kept.data_ptr(), _lengths(out_len, B), workspace.data_ptr(), workspace.nbytes)
    _call("si_cache4_evict", stream, (weight, weight_out, cache, out, kept, out_len, workspace, k_len), args)


class AttnOptions:
    """Self-attention of si_block_forward_attn: rotary positions (a Rope or None) and, with keep > 0, the `keep` best blocks of
    k_block keys for every run of q_block queries."""

    def __init__(self, rope: Optional[Rope] = None, q_block: int = 128, k_block: int = 64, keep: int = 0):
        self.rope = rope
        self.struct = _AttnOptions(None if rope is None else C.pointer(rope.struct), q_block, k_block, keep)


def si_block_attn_workspace_bytes(x, weights: BlockWeights, ctx, attn: AttnOptions, axis: int, slice_len: int) -> int:
    xd = _tensor5(x)
    pc, _keep = _pctx(ctx)
    return int(lib().si_block_attn_workspace_bytes(C.byref(xd), C.byref(weights.struct), pc, C.byref(attn.struct), axis, slice_len))


def si_block_forward_attn(x, weights: BlockWeights, ctx, attn: AttnOptions, out, axis: int, slice_len: int, workspace, flags: int = 0,
                          stream=None) -> None:
    """si_block_forward_ex of a spatial block whose self-attention is the one that `attn` describes."""
    if attn.rope is not None:
        for g in attn.rope.gains:
            if g is not None and (g.shape[0] != weights.struct.dim_head or g.dtype != x.dtype or g.device != x.device):
                raise ValueError("gains must be [dim_head] in the feature's dtype, on its device")
    xd, od = _tensor5(x), _tensor5(out)
    pc, _keep = _pctx(ctx)
    st = lib().si_block_forward_attn(C.byref(xd), C.byref(weights.struct), pc, C.byref(attn.struct), C.byref(od), axis, slice_len,
                                     workspace.data_ptr(), workspace.numel() * workspace.element_size(), flags, _stream_ptr(stream))
    if st != 0:
        raise SiError(st, "si_block_forward_attn")


class RehashCache:
    """Anchor buffers of si_block_forward_rehash for one block (device tensors shaped like the feature)."""

    def __init__(self, like):
        import torch
        self.x_key = torch.empty_like(like)
        self.y_key = torch.empty_like(like)
        self.struct = _RehashCache(self.x_key.data_ptr(), self.y_key.data_ptr(), 0)

    @property
    def valid(self) -> bool:
        return bool(self.struct.valid)

    def reset(self) -> None:
        self.struct.valid = 0


def si_block_forward_rehash(x, weights: BlockWeights, ctx, out, axis: int, slice_len: int, workspace,
                            cache: RehashCache, gamma: float, stream=None) -> Tuple[bool, float]:
    """Step Rehash around the block, decided on its input.  Returns (reused, cos); waits for the stream
    when the cache holds an anchor."""
    xd, od = _tensor5(x), _tensor5(out)
    pc, _keep = _pctx(ctx)
    cos, reused = C.c_double(), C.c_int32()
    st = lib().si_block_forward_rehash(C.byref(xd), C.byref(weights.struct), pc, C.byref(od), axis, slice_len,
                                       workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                       C.byref(cache.struct), gamma, _stream_ptr(stream),
                                       C.byref(cos), C.byref(reused))
    if st != 0:
        raise SiError(st, "si_block_forward_rehash")
    return bool(reused.value), cos.value


def si_rehash_scratch_bytes(n: int) -> int:
    return int(lib().si_rehash_scratch_bytes(n))


def si_rehash_check(feat_t, feat_prev, thresh: float, cos_dev, decision_dev, scratch, stream=None) -> None:
    """Enqueues the similarity test; results land in cos_dev (float64[1] or None) and decision_dev (int32[1])."""
    if feat_t.numel() != feat_prev.numel() or feat_t.dtype != feat_prev.dtype:
        raise ValueError("features must have the same size and dtype")
    if not (feat_t.is_contiguous() and feat_prev.is_contiguous()):
        raise ValueError("features must be contiguous")
    st = lib().si_rehash_check(feat_t.data_ptr(), feat_prev.data_ptr(), feat_t.numel(), _dtype_code(feat_t),
                               thresh, None if cos_dev is None else cos_dev.data_ptr(), decision_dev.data_ptr(),
                               scratch.data_ptr(), _stream_ptr(stream))
    if st != 0:
        raise SiError(st, "si_rehash_check")


def si_init_device() -> None:
    st = lib().si_init_device()
    if st != 0:
        raise SiError(st, "si_init_device")


def si_rehash_check_static(feat_t, feat_prev, thresh: float, cos_dev, decision_dev, stream=None) -> None:
    """si_rehash_check without a scratch argument: the partial sums live in the library's device array."""
    if feat_t.numel() != feat_prev.numel() or feat_t.dtype != feat_prev.dtype:
        raise ValueError("features must have the same size and dtype")
    if not (feat_t.is_contiguous() and feat_prev.is_contiguous()):
        raise ValueError("features must be contiguous")
    st = lib().si_rehash_check_static(feat_t.data_ptr(), feat_prev.data_ptr(), feat_t.numel(), _dtype_code(feat_t),
                                      thresh, None if cos_dev is None else cos_dev.data_ptr(), decision_dev.data_ptr(),
                                      _stream_ptr(stream))
    if st != 0:
        raise SiError(st, "si_rehash_check_static")


def si_rehash_check_sync(feat_t, feat_prev, thresh: float, scratch, result_dev, stream=None) -> Tuple[float, int]:
    if feat_t.numel() != feat_prev.numel() or feat_t.dtype != feat_prev.dtype:
        raise ValueError("features must have the same size and dtype")
    cos, dec = C.c_double(), C.c_int32()
    st = lib().si_rehash_check_sync(feat_t.data_ptr(), feat_prev.data_ptr(), feat_t.numel(), _dtype_code(feat_t),
                                    thresh, scratch.data_ptr(), result_dev.data_ptr(), _stream_ptr(stream),
                                    C.byref(cos), C.byref(dec))
    if st != 0:
        raise SiError(st, "si_rehash_check_sync")
    return cos.value, dec.value


def si_key_step_search(S: Sequence[Sequence[float]], gamma: float) -> List[int]:
    """Algorithm 1 on a K x K similarity map (host)."""
    K = len(S)
    flat = (C.c_float * (K * K))(*[float(v) for row in S for v in row])
    G = (C.c_int32 * max(K, 1))()
    n = lib().si_key_step_search(flat, K, gamma, G)
    if n < 0:
        raise SiError(7, "si_key_step_search")
    return [int(G[i]) for i in range(n)]


def si_stage_timing_enable(on: bool) -> None:
    lib().si_stage_timing_enable(int(bool(on)))


def si_stage_timing_read() -> Dict[str, Tuple[float, int]]:
    """{stage: (total milliseconds, launches)} since the last read."""
    cap = 64
    names = (C.c_char_p * cap)()
    ms = (C.c_double * cap)()
    cnt = (C.c_int64 * cap)()
    n = lib().si_stage_timing_read(names, ms, cnt, cap)
    if n < 0:
        raise SiError(8, "si_stage_timing_read")
    return {names[i].decode(): (ms[i], int(cnt[i])) for i in range(min(n, cap)) if cnt[i] > 0}
