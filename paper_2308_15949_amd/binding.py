"""Thin binding of liblaud.so (ctypes; the token operators' calls through a small extension): argument marshalling only.

Every function below has the name and the meaning of the C entry point declared in
include/laud.h; tensors are torch CUDA tensors used purely as device memory, the
stream is torch's current stream.  There is no CPU fallback: if the library has not
been built, loading raises.
"""
from __future__ import annotations

import ctypes as C
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "liblaud.so")

F32, BF16, E4M3 = 0, 1, 2
NORM_RMS, NORM_LAYER = 0, 1
MOE_MAX_TOKENS = 1024
OP_MASK_GEN, OP_COMPACT, OP_GATHER, OP_DYN_BOTTLENECK, OP_CHANNEL_SKIP = range(5)
OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_HIP, ERR_SCRATCH_LIMIT = 0, -1, -2, -3, -4, -5
NOALLOC_SCRATCH_BYTES = 16 << 20

EXPORTS = ["laud_status_string", "laud_abi_version", "laud_workspace_size", "laud_mask_gen",
           "laud_layer_skip_compact", "laud_gather_patches", "laud_dyn_bottleneck",
           "laud_channel_skip_conv", "laud_masker_dyn_bottleneck", "laud_channel_masker", "laud_channel_masker_workspace", "laud_dyn_bottleneck_unfused",
           "laud_dyn_bottleneck_unfused_workspace", "laud_static_bottleneck", "laud_static_bottleneck_workspace",
           "laud_stem", "laud_stem3x3", "laud_stem_workspace", "laud_dyn_projection_bottleneck", "laud_dyn_projection_workspace",
           "laud_dyn_group_se_bottleneck", "laud_dyn_group_se_projection_bottleneck", "laud_stage_timing_enable", "laud_stage_timing_read", "laud_stage_name",
           "laud_init", "laud_dyn_bottleneck_noalloc", "laud_probe_mfma", "laud_probe_copy", "laud_probe_read",
           "laud_packed_weights_size", "laud_pack_weights",
           "laud_norm_residual", "laud_quantize_e4m3", "laud_matmul_e4m3_workspace", "laud_matmul_e4m3", "laud_moe_workspace",
           "laud_moe",
           "laud_attention", "laud_cache_write", "laud_cache_read", "laud_cache_attention_workspace", "laud_cache_attention"]
STAGE_COUNT = 13


class Fmap(C.Structure):
    _fields_ = [("N", C.c_int32), ("H", C.c_int32), ("W", C.c_int32), ("C", C.c_int32), ("dtype", C.c_int32)]


class Bottleneck(C.Structure):
    _fields_ = [("c_in", C.c_int32), ("c_mid", C.c_int32), ("c_out", C.c_int32),
                ("w1", C.c_void_p), ("w2", C.c_void_p), ("w3", C.c_void_p),
                ("s1", C.c_void_p), ("t1", C.c_void_p), ("s2", C.c_void_p), ("t2", C.c_void_p),
                ("s3", C.c_void_p), ("t3", C.c_void_p), ("relu_out", C.c_int32), ("packed", C.c_void_p)]


class GroupSE(C.Structure):
    _fields_ = [("group_width", C.c_int32), ("se_width", C.c_int32), ("w_se1", C.c_void_p), ("b_se1", C.c_void_p),
                ("w_se2", C.c_void_p), ("b_se2", C.c_void_p)]


class NormBlock(C.Structure):
    _fields_ = [("C", C.c_int32), ("dtype", C.c_int32), ("kind", C.c_int32), ("eps", C.c_float), ("post_w", C.c_void_p),
                ("post_b", C.c_void_p), ("pre_w", C.c_void_p), ("pre_b", C.c_void_p), ("alpha", C.c_float), ("beta", C.c_float)]


class MoeLayer(C.Structure):
    _fields_ = [("C", C.c_int32), ("F", C.c_int32), ("E", C.c_int32), ("top_k", C.c_int32), ("dtype", C.c_int32),
                ("w_dtype", C.c_int32), ("router", C.c_void_p), ("up", C.c_void_p), ("down", C.c_void_p), ("s_up", C.c_void_p),
                ("s_down", C.c_void_p), ("renormalise", C.c_int32), ("scale", C.c_float)]


class Heads(C.Structure):
    _fields_ = [("heads", C.c_int32), ("kv_heads", C.c_int32), ("D", C.c_int32), ("dtype", C.c_int32), ("causal", C.c_int32),
                ("scale", C.c_float)]


class Cache(C.Structure):
    _fields_ = [("pages", C.c_int32), ("page", C.c_int32), ("kv_heads", C.c_int32), ("D", C.c_int32), ("dtype", C.c_int32),
                ("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p)]
    device = None  # of its tensors (make_cache)


class Batch(C.Structure):
    _fields_ = [("B", C.c_int32), ("table_ld", C.c_int32), ("offsets", C.c_void_p), ("lens", C.c_void_p), ("table", C.c_void_p),
                ("prefix", C.c_void_p), ("prefix_len", C.c_int32)]
    device = None  # of its tensors (make_batch)


class LaudError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)}")


_lib = None


def load() -> C.CDLL:
    """Loads liblaud.so (once).  Raises if it has not been built: there is no fallback."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2308_15949_amd.build` "
                           "(there is no CPU fallback)")
    lib = C.CDLL(LIB_PATH)
    vp, i32, sz = C.c_void_p, C.c_int, C.c_size_t
    lib.laud_status_string.restype = C.c_char_p
    lib.laud_status_string.argtypes = [i32]
    lib.laud_abi_version.restype = i32
    lib.laud_abi_version.argtypes = []
    lib.laud_workspace_size.restype = sz
    lib.laud_workspace_size.argtypes = [i32, Fmap, C.POINTER(Bottleneck), i32]
    lib.laud_mask_gen.restype = i32
    lib.laud_mask_gen.argtypes = [vp, Fmap, i32, vp, C.c_float, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.laud_layer_skip_compact.restype = i32
    lib.laud_layer_skip_compact.argtypes = [vp, i32, vp, vp, vp, sz, vp]
    lib.laud_gather_patches.restype = i32
    lib.laud_gather_patches.argtypes = [vp, Fmap, i32, i32, vp, vp, vp, vp]
    lib.laud_dyn_bottleneck.restype = i32
    lib.laud_dyn_bottleneck.argtypes = [vp, Fmap, C.POINTER(Bottleneck), i32, vp, vp, vp, vp, sz, vp]
    lib.laud_probe_mfma.restype = i32
    lib.laud_probe_mfma.argtypes = [i32, i32, i32, C.POINTER(C.c_double), vp, vp]
    lib.laud_probe_read.restype = i32
    lib.laud_probe_read.argtypes = [vp, sz, vp, vp]
    lib.laud_probe_copy.restype = i32
    lib.laud_probe_copy.argtypes = [vp, vp, sz, vp]
    lib.laud_packed_weights_size.restype = sz
    lib.laud_packed_weights_size.argtypes = [C.POINTER(Bottleneck), i32]
    lib.laud_pack_weights.restype = i32
    lib.laud_pack_weights.argtypes = [C.POINTER(Bottleneck), i32, vp, vp]
    lib.laud_init.restype = i32
    lib.laud_init.argtypes = []
    lib.laud_dyn_bottleneck_noalloc.restype = i32
    lib.laud_dyn_bottleneck_noalloc.argtypes = [vp, Fmap, C.POINTER(Bottleneck), i32, vp, vp, vp, vp]
    lib.laud_dyn_group_se_bottleneck.restype = i32
    lib.laud_dyn_group_se_bottleneck.argtypes = [vp, Fmap, C.POINTER(Bottleneck), C.POINTER(GroupSE), i32, vp, vp, vp, vp,
                                                 sz, vp]
    lib.laud_channel_skip_conv.restype = i32
    lib.laud_channel_skip_conv.argtypes = [vp, Fmap, C.POINTER(Bottleneck), vp, i32, vp, vp, sz, vp]
    lib.laud_masker_dyn_bottleneck.restype = i32
    lib.laud_masker_dyn_bottleneck.argtypes = [vp, Fmap, C.POINTER(Bottleneck), i32, vp, C.c_float, vp, vp, vp, vp,
                                               vp, vp, vp, vp, sz, vp]
    lib.laud_dyn_bottleneck_unfused_workspace.restype = sz
    lib.laud_dyn_bottleneck_unfused_workspace.argtypes = [Fmap, C.POINTER(Bottleneck), i32]
    lib.laud_dyn_bottleneck_unfused.restype = i32
    lib.laud_dyn_bottleneck_unfused.argtypes = [vp, Fmap, C.POINTER(Bottleneck), i32, vp, vp, vp, vp, sz, vp]
    lib.laud_static_bottleneck_workspace.restype = sz
    lib.laud_static_bottleneck_workspace.argtypes = [Fmap, C.POINTER(Bottleneck), i32]
    lib.laud_static_bottleneck.restype = i32
    lib.laud_static_bottleneck.argtypes = [vp, Fmap, C.POINTER(Bottleneck), vp, vp, vp, i32, vp, vp, sz, vp]
    lib.laud_dyn_projection_workspace.restype = sz
    lib.laud_dyn_projection_workspace.argtypes = [Fmap, C.POINTER(Bottleneck), i32]
    lib.laud_dyn_projection_bottleneck.restype = i32
    lib.laud_dyn_projection_bottleneck.argtypes = [vp, Fmap, C.POINTER(Bottleneck), vp, vp, vp, i32, i32, vp, vp, vp, vp,
                                                   sz, vp]
    lib.laud_dyn_group_se_projection_bottleneck.restype = i32
    lib.laud_dyn_group_se_projection_bottleneck.argtypes = [vp, Fmap, C.POINTER(Bottleneck), C.POINTER(GroupSE), vp, vp, vp,
                                                            i32, i32, vp, vp, vp, vp, sz, vp]
    lib.laud_stem_workspace.restype = sz
    lib.laud_stem_workspace.argtypes = [i32, i32, i32, i32, i32]
    lib.laud_stem.restype = i32
    lib.laud_stem.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp, i32, vp, vp, sz, vp]
    lib.laud_stem3x3.restype = i32
    lib.laud_stem3x3.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp, i32, vp, vp]
    lib.laud_channel_masker_workspace.restype = sz
    lib.laud_channel_masker_workspace.argtypes = [Fmap]
    lib.laud_channel_masker.restype = i32
    lib.laud_channel_masker.argtypes = [vp, Fmap, vp, vp, i32, vp, vp, i32, vp, vp, vp, sz, vp]
    i64 = C.c_int64
    lib.laud_norm_residual.restype = i32
    lib.laud_norm_residual.argtypes = [C.POINTER(NormBlock), i32, vp, i64, vp, i64, vp, vp, i32, vp, i64, vp, i64, i32, vp, vp]
    lib.laud_quantize_e4m3.restype = i32
    lib.laud_quantize_e4m3.argtypes = [vp, i64, i32, i32, i32, i32, vp, i64, vp, vp]
    lib.laud_matmul_e4m3_workspace.restype = sz
    lib.laud_matmul_e4m3_workspace.argtypes = [i32, i32, i32]
    lib.laud_matmul_e4m3.restype = i32
    lib.laud_matmul_e4m3.argtypes = [vp, i64, vp, vp, i64, vp, i32, i32, i32, vp, i64, i32, vp, sz, vp]
    lib.laud_moe_workspace.restype = sz
    lib.laud_moe_workspace.argtypes = [C.POINTER(MoeLayer), i32]
    lib.laud_moe.restype = i32
    lib.laud_moe.argtypes = [C.POINTER(MoeLayer), i32, vp, i64, vp, vp, i64, vp, vp, vp, sz, vp]
    lib.laud_attention.restype = i32
    lib.laud_attention.argtypes = [C.POINTER(Heads), i32, vp, i32, vp, i64, vp, i64, vp, i64, vp, vp, i64, vp]
    lib.laud_cache_write.restype = lib.laud_cache_read.restype = i32
    lib.laud_cache_write.argtypes = lib.laud_cache_read.argtypes = [C.POINTER(Cache), C.POINTER(Batch), i32, vp, i64, vp, i64, i32, vp]
    lib.laud_cache_attention_workspace.restype = sz
    lib.laud_cache_attention_workspace.argtypes = [C.POINTER(Heads), C.POINTER(Cache), C.POINTER(Batch), i32]
    lib.laud_cache_attention.restype = i32
    lib.laud_cache_attention.argtypes = [C.POINTER(Heads), C.POINTER(Cache), C.POINTER(Batch), i32, vp, i64, vp, i64, vp, sz, vp]
    lib.laud_stage_timing_enable.restype = i32
    lib.laud_stage_timing_enable.argtypes = [i32]
    lib.laud_stage_timing_read.restype = i32
    lib.laud_stage_timing_read.argtypes = [C.POINTER(C.c_double), C.POINTER(C.c_int64)]
    lib.laud_stage_name.restype = C.c_char_p
    lib.laud_stage_name.argtypes = [i32]
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().laud_status_string(int(status)).decode()


def abi_version() -> int:
    return int(load().laud_abi_version())


# ----- marshalling helpers ---------------------------------------------------------------
# (A single image's block is a handful of launches of 4 us each, so the microseconds of the binding count: pointers go to
# ctypes as plain integers, and the stream comes from the raw getter instead of through a Stream object.)
def _ptr(t):
    """Device (or raw integer) pointer of a tensor; None -> NULL."""
    return t if t is None or isinstance(t, int) else t.data_ptr()


_raw_stream = None


def _stream():
    """torch's current stream on the current device, as an integer."""
    global _raw_stream
    if _raw_stream is None:
        import torch
        get_stream, get_device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
        if get_stream is not None and get_device is not None:
            torch.cuda.current_stream()  # initialises torch's device state, which the raw getters take for granted
            _raw_stream = lambda: get_stream(get_device())  # noqa: E731
        else:
            _raw_stream = lambda: torch.cuda.current_stream().cuda_stream  # noqa: E731
    return _raw_stream()


def _forget_raw_stream():
    global _raw_stream, _calls
    _raw_stream = _calls = None


# a forked child goes through torch once more, which refuses a device state that was initialised in the parent
os.register_at_fork(after_in_child=_forget_raw_stream)


def _check(status: int, where: str) -> None:
    if status != OK:
        raise LaudError(status, where)


def fmap_of(x, dtype: int | None = None) -> Fmap:
    """Fmap of an [N,H,W,C] tensor (float32 or bfloat16)."""
    import torch
    if dtype is None:
        dtype = BF16 if x.dtype == torch.bfloat16 else F32
    n, h, w, c = x.shape
    return Fmap(int(n), int(h), int(w), int(c), int(dtype))


def make_bottleneck(w1, w2, w3, s1, t1, s2, t2, s3, t3, relu_out: bool) -> Bottleneck:
    """Bottleneck descriptor over device tensors w1 [m,Cin], w2 [m,3,3,m], w3 [Cout,m] and
    float32 affine vectors.  The caller keeps the tensors alive."""
    return Bottleneck(int(w1.shape[1]), int(w1.shape[0]), int(w3.shape[0]),
                      w1.data_ptr(), w2.data_ptr(), w3.data_ptr(),
                      s1.data_ptr(), t1.data_ptr(), s2.data_ptr(), t2.data_ptr(),
                      s3.data_ptr(), t3.data_ptr(), 1 if relu_out else 0)


def packed_weights_size(p: Bottleneck, dtype: int) -> int:
    return int(load().laud_packed_weights_size(C.byref(p), int(dtype)))


def laud_pack_weights(p: Bottleneck, dtype: int, packed) -> None:
    """Re-orders the block's weights into `packed` (device memory of packed_weights_size bytes); the caller then sets
    p.packed = packed.data_ptr() and keeps the tensor alive."""
    _check(load().laud_pack_weights(C.byref(p), int(dtype), _ptr(packed), _stream()), "laud_pack_weights")


def workspace_size(op: int, fx: Fmap, p: Bottleneck | None, s_or_d: int) -> int:
    return int(load().laud_workspace_size(int(op), fx, C.byref(p) if p is not None else None, int(s_or_d)))


def _ws_args(ws):
    if ws is None:
        return None, 0
    return _ptr(ws), int(ws.numel() * ws.element_size())


# ----- entry points (same names as the C ABI) ---------------------------------------------
def laud_mask_gen(x, fx: Fmap, S: int, w, bias: float, keep, mask, idx, count, sample_offsets, logits, ws) -> None:
    wp, wb = _ws_args(ws)
    _check(load().laud_mask_gen(_ptr(x), fx, int(S), _ptr(w), float(bias), _ptr(keep), _ptr(mask), _ptr(idx),
                                _ptr(count), _ptr(sample_offsets), _ptr(logits), wp, wb, _stream()),
           "laud_mask_gen")


def laud_layer_skip_compact(keep, n: int, idx, count, ws) -> None:
    wp, wb = _ws_args(ws)
    _check(load().laud_layer_skip_compact(_ptr(keep), int(n), _ptr(idx), _ptr(count), wp, wb, _stream()),
           "laud_layer_skip_compact")


def laud_gather_patches(x, fx: Fmap, S: int, halo: int, idx, count, out) -> None:
    _check(load().laud_gather_patches(_ptr(x), fx, int(S), int(halo), _ptr(idx), _ptr(count), _ptr(out), _stream()),
           "laud_gather_patches")


def laud_dyn_bottleneck(x, fx: Fmap, p: Bottleneck, S: int, idx, count, out, ws) -> None:
    wp, wb = _ws_args(ws)
    _check(load().laud_dyn_bottleneck(_ptr(x), fx, C.byref(p), int(S), _ptr(idx), _ptr(count), _ptr(out),
                                      wp, wb, _stream()), "laud_dyn_bottleneck")


def laud_probe_mfma(dtype: int, iters: int, blocks: int, sink) -> float:
    """Enqueues the bare MFMA loop; returns the FLOPs of the launch."""
    fl = C.c_double(0.0)
    _check(load().laud_probe_mfma(int(dtype), int(iters), int(blocks), C.byref(fl), _ptr(sink), _stream()), "laud_probe_mfma")
    return float(fl.value)


def laud_probe_copy(src, dst, nbytes: int) -> None:
    _check(load().laud_probe_copy(_ptr(src), _ptr(dst), int(nbytes), _stream()), "laud_probe_copy")


def laud_probe_read(src, nbytes: int, sink) -> None:
    _check(load().laud_probe_read(_ptr(src), int(nbytes), _ptr(sink), _stream()), "laud_probe_read")


def laud_init() -> None:
    _check(load().laud_init(), "laud_init")


def laud_dyn_bottleneck_noalloc(x, fx: Fmap, p: Bottleneck, S: int, idx, count, out) -> None:
    _check(load().laud_dyn_bottleneck_noalloc(_ptr(x), fx, C.byref(p), int(S), _ptr(idx), _ptr(count), _ptr(out),
                                              _stream()), "laud_dyn_bottleneck_noalloc")


def make_group_se(group_width: int, w_se1=None, b_se1=None, w_se2=None, b_se2=None) -> GroupSE:
    """Descriptor of the group-convolution / SE extension over float32 device tensors (w_se1 [se_width, c_mid],
    w_se2 [c_mid, se_width]); without tensors: group convolution only.  The caller keeps the tensors alive."""
    if w_se1 is None:
        return GroupSE(int(group_width), 0, None, None, None, None)
    return GroupSE(int(group_width), int(w_se1.shape[0]), w_se1.data_ptr(), b_se1.data_ptr(), w_se2.data_ptr(),
                   b_se2.data_ptr())


def laud_dyn_group_se_bottleneck(x, fx: Fmap, p: Bottleneck, e: GroupSE, S: int, idx, count, out, ws) -> None:
    wp, wb = _ws_args(ws)
    _check(load().laud_dyn_group_se_bottleneck(_ptr(x), fx, C.byref(p), C.byref(e) if e is not None else None, int(S),
                                               _ptr(idx), _ptr(count), _ptr(out), wp, wb, _stream()),
           "laud_dyn_group_se_bottleneck")


def laud_channel_skip_conv(x, fx: Fmap, p: Bottleneck, cmask, D: int, out, ws) -> None:
    wp, wb = _ws_args(ws)
    _check(load().laud_channel_skip_conv(_ptr(x), fx, C.byref(p), _ptr(cmask), int(D), _ptr(out),
                                         wp, wb, _stream()), "laud_channel_skip_conv")


def laud_masker_dyn_bottleneck(x, fx: Fmap, p: Bottleneck, S: int, w, bias: float, keep, mask, idx, count,
                               sample_offsets, logits, out, ws) -> None:
    wp, wb = _ws_args(ws)
    _check(load().laud_masker_dyn_bottleneck(_ptr(x), fx, C.byref(p), int(S), _ptr(w), float(bias), _ptr(keep),
                                             _ptr(mask), _ptr(idx), _ptr(count), _ptr(sample_offsets), _ptr(logits),
                                             _ptr(out), wp, wb, _stream()), "laud_masker_dyn_bottleneck")


def dyn_bottleneck_unfused_workspace(fx: Fmap, p: Bottleneck, S: int) -> int:
    return int(load().laud_dyn_bottleneck_unfused_workspace(fx, C.byref(p), int(S)))


def laud_dyn_bottleneck_unfused(x, fx: Fmap, p: Bottleneck, S: int, idx, count, out, ws) -> None:
    wp, wb = _ws_args(ws)
    _check(load().laud_dyn_bottleneck_unfused(_ptr(x), fx, C.byref(p), int(S), _ptr(idx), _ptr(count), _ptr(out),
                                              wp, wb, _stream()), "laud_dyn_bottleneck_unfused")


def static_bottleneck_workspace(fx: Fmap, p: Bottleneck, stride: int) -> int:
    return int(load().laud_static_bottleneck_workspace(fx, C.byref(p), int(stride)))


def laud_static_bottleneck(x, fx: Fmap, p: Bottleneck, w_sc, s_sc, t_sc, stride: int, out, ws) -> None:
    wp, wb = _ws_args(ws)
    _check(load().laud_static_bottleneck(_ptr(x), fx, C.byref(p), _ptr(w_sc), _ptr(s_sc), _ptr(t_sc), int(stride),
                                         _ptr(out), wp, wb, _stream()), "laud_static_bottleneck")


def dyn_projection_workspace(fx: Fmap, p: Bottleneck, stride: int) -> int:
    return int(load().laud_dyn_projection_workspace(fx, C.byref(p), int(stride)))


def laud_dyn_projection_bottleneck(x, fx: Fmap, p: Bottleneck, w_sc, s_sc, t_sc, stride: int, S: int, idx, count,
                                   out, ws) -> None:
    wp, wb = _ws_args(ws)
    _check(load().laud_dyn_projection_bottleneck(_ptr(x), fx, C.byref(p), _ptr(w_sc), _ptr(s_sc), _ptr(t_sc),
                                                 int(stride), int(S), _ptr(idx), _ptr(count), _ptr(out), wp, wb,
                                                 _stream()), "laud_dyn_projection_bottleneck")


def laud_dyn_group_se_projection_bottleneck(x, fx: Fmap, p: Bottleneck, e: GroupSE, w_sc, s_sc, t_sc, stride: int, S: int,
                                            idx, count, out, ws) -> None:
    wp, wb = _ws_args(ws)
    _check(load().laud_dyn_group_se_projection_bottleneck(_ptr(x), fx, C.byref(p), C.byref(e) if e is not None else None,
                                                          _ptr(w_sc), _ptr(s_sc), _ptr(t_sc), int(stride), int(S),
                                                          _ptr(idx), _ptr(count), _ptr(out), wp, wb, _stream()),
           "laud_dyn_group_se_projection_bottleneck")


def stem_workspace(n: int, hin: int, win: int, c_out: int, dtype: int) -> int:
    return int(load().laud_stem_workspace(int(n), int(hin), int(win), int(c_out), int(dtype)))


def laud_stem(x, n: int, hin: int, win: int, dtype: int, w7, s, t, c_out: int, out, ws) -> None:
    wp, wb = _ws_args(ws)
    _check(load().laud_stem(_ptr(x), int(n), int(hin), int(win), int(dtype), _ptr(w7), _ptr(s), _ptr(t), int(c_out),
                            _ptr(out), wp, wb, _stream()), "laud_stem")


def laud_stem3x3(x, n: int, hin: int, win: int, dtype: int, w3, s, t, c_out: int, out) -> None:
    _check(load().laud_stem3x3(_ptr(x), int(n), int(hin), int(win), int(dtype), _ptr(w3), _ptr(s), _ptr(t), int(c_out),
                               _ptr(out), _stream()), "laud_stem3x3")


def channel_masker_workspace(fx: Fmap) -> int:
    return int(load().laud_channel_masker_workspace(fx))


def laud_channel_masker(x, fx: Fmap, wa, ba, hidden: int, wb, bb, D: int, cmask, logits2, ws) -> None:
    wp, wb_ = _ws_args(ws)
    _check(load().laud_channel_masker(_ptr(x), fx, _ptr(wa), _ptr(ba), int(hidden), _ptr(wb), _ptr(bb), int(D),
                                      _ptr(cmask), _ptr(logits2), wp, wb_, _stream()), "laud_channel_masker")


# ----- token operators --------------------------------------------------------------------------------------------------------
# (Their tensors come with strides and in three types, so their calls check device, type and shape: a tensor that does not fit raises
# LaudError like an argument the library refuses.  The calls go through _laud_torch.so, an extension that reads the tensors in C++:
# a call on a few rows is a launch of two or three microseconds, the same reading in Python and ctypes took five.)
FAST_PATH = os.path.join(HERE, "_laud_torch.so")
_calls = None


def _token_calls():
    """The extension, bound to the loaded library's entry points.  Raises if it has not been built: there is no other path."""
    global _calls
    lib = load()
    if not os.path.exists(FAST_PATH):
        raise RuntimeError(f"{FAST_PATH} is missing: build it with `python -m paper_2308_15949_amd.build`")
    import torch  # (loads the libraries that the extension is linked against)

    from . import _laud_torch
    if torch.cuda.is_available():
        torch.cuda.current_stream()  # initialises torch's device state, which the extension takes for granted
    _laud_torch.bind(*(C.cast(f, C.c_void_p).value for f in (lib.laud_norm_residual, lib.laud_quantize_e4m3, lib.laud_matmul_e4m3,
                                                              lib.laud_moe, lib.laud_attention, lib.laud_cache_write,
                                                              lib.laud_cache_read, lib.laud_cache_attention)))
    _calls = _laud_torch
    return _calls


def _bad(where: str):
    raise LaudError(ERR_INVALID_ARG, where)


def _int32(v, where: str) -> int:
    """A number that a descriptor holds in 32 bits (ctypes would cut it)."""
    v = int(v)
    if not -2 ** 31 <= v < 2 ** 31:
        _bad(where)
    return v


def _dtype_of(t) -> int:
    """laud_dtype of a tensor, -1 for other types."""
    import torch
    return {torch.float32: F32, torch.bfloat16: BF16, torch.float8_e4m3fn: E4M3}.get(t.dtype, -1)


def _dense(t, shape, code: int, where: str):
    """Pointer of a contiguous device tensor of that shape and type; None -> None."""
    if t is None:
        return None
    if not (t.is_cuda and t.shape == shape and _dtype_of(t) == code and t.is_contiguous()):
        _bad(where)
    return t.data_ptr()


def _blocks(n: int) -> int:
    return -(-n // 128)


def make_norm_block(c: int, dtype, kind: str, eps: float, post_w=None, post_b=None, pre_w=None, pre_b=None, alpha: float = 1.0,
                    beta: float = 1.0) -> NormBlock:
    """Descriptor of the norms after a block and before the next one over float32 device vectors [c]; dtype: torch's type of the
    rows, kind "rms" or "layer".  The caller keeps the tensors alive."""
    import torch
    where = "make_norm_block"
    if kind not in ("rms", "layer") or dtype not in (torch.float32, torch.bfloat16):
        _bad(where)
    v = [_dense(t, (c,), F32, where) for t in (post_w, post_b, pre_w, pre_b)]
    return NormBlock(int(c), BF16 if dtype == torch.bfloat16 else F32, NORM_LAYER if kind == "layer" else NORM_RMS, float(eps), *v,
                     float(alpha), float(beta))


def laud_norm_residual(p: NormBlock, x, y=None, keep=None, gate=None, rows_per_gate: int = 0, out=None, z=None, z_scale=None) -> None:
    """x, y, out, z [rows][C]; keep [rows] bytes; gate [ceil(rows / rows_per_gate) or more][C] float32; z float8_e4m3fn with
    z_scale [rows][ceil(C / 128)], or of x's type."""
    s = (_calls or _token_calls()).norm_residual(p, x, y, keep, gate, rows_per_gate, out, z, z_scale)
    if s:
        raise LaudError(s, "laud_norm_residual")


def laud_quantize_e4m3(x, q, scale, block_rows: int = 1) -> None:
    """x [rows][cols] float32 or bf16 -> q [rows][cols] float8_e4m3fn and scale [ceil(rows / block_rows)][ceil(cols / 128)]."""
    s = (_calls or _token_calls()).quantize(x, q, scale, block_rows)
    if s:
        raise LaudError(s, "laud_quantize_e4m3")


def matmul_e4m3_workspace(m: int, n: int, k: int) -> int:
    return int(load().laud_matmul_e4m3_workspace(int(m), int(n), int(k)))


def laud_matmul_e4m3(a, sa, b, sb, out, ws=None) -> None:
    """out [M][N] (float32 or bf16) = a [M][K] times b [N][K] transposed, both float8_e4m3fn with scales sa [M][ceil(K / 128)] and
    sb [ceil(N / 128)][ceil(K / 128)]."""
    s = (_calls or _token_calls()).matmul(a, sa, b, sb, out, ws)
    if s:
        raise LaudError(s, "laud_matmul_e4m3")


def make_moe(router, up, down, s_up=None, s_down=None, top_k: int = 1, renormalise: bool = False, scale: float = 1.0) -> MoeLayer:
    """Descriptor of a mixture-of-experts layer over device tensors router [E][C], up [E][2][F][C] (gate, up) and down [E][C][F];
    float8_e4m3fn weights come with s_up [E][2][ceil(F/128)][ceil(C/128)] and s_down [E][ceil(C/128)][ceil(F/128)].  The caller
    keeps the tensors alive."""
    where = "make_moe"
    if router.dim() != 2 or up.dim() != 4 or up.shape[1] != 2:
        _bad(where)
    (e, c), f = router.shape, up.shape[2]
    wd = _dtype_of(up)
    v = [_dense(router, (e, c), _dtype_of(router), where), _dense(up, (e, 2, f, c), wd, where), _dense(down, (e, c, f), wd, where)]
    s = [None, None]
    if wd == E4M3:
        if s_up is None or s_down is None:
            _bad(where)
        s = [_dense(s_up, (e, 2, _blocks(f), _blocks(c)), F32, where), _dense(s_down, (e, _blocks(c), _blocks(f)), F32, where)]
    return MoeLayer(int(c), int(f), int(e), int(top_k), _dtype_of(router), wd, *v, *s, 1 if renormalise else 0, float(scale))


def moe_workspace(p: MoeLayer, t: int) -> int:
    return int(load().laud_moe_workspace(C.byref(p), int(t)))


def laud_moe(p: MoeLayer, x, keep, out, experts, weights, ws) -> None:
    """x, out [T][C] of the router's type; keep [T] bytes or None; experts [T][top_k] int32 and weights [T][top_k] float32 receive
    the routing, each may be None."""
    s = (_calls or _token_calls()).moe(p, x, keep, out, experts, weights, ws)
    if s:
        raise LaudError(s, "laud_moe")


# ----- attention of a token block ------------------------------------------------------------------------------------------------
def make_heads(heads: int, kv_heads: int, d: int, dtype, causal: bool, scale: float | None = None) -> Heads:
    """Descriptor of an attention's heads; dtype: torch's type of the rows; scale None: 1 / sqrt(d)."""
    import torch
    if dtype not in (torch.float32, torch.bfloat16) or d <= 0:
        _bad("make_heads")
    heads, kv_heads, d = (_int32(n, "make_heads") for n in (heads, kv_heads, d))
    return Heads(heads, kv_heads, d, BF16 if dtype == torch.bfloat16 else F32, 1 if causal else 0,
                 float(d) ** -0.5 if scale is None else float(scale))


def _of_one_device(where: str, *tensors) -> None:
    if len({t.device for t in tensors if t is not None}) != 1:
        _bad(where)


def make_cache(k, v, k_scale=None, v_scale=None) -> Cache:
    """Descriptor of a paged cache over device tensors k, v [pages][kv_heads][page][D] (float32, bf16, or float8_e4m3fn with k_scale,
    v_scale [pages][kv_heads][page] float32), which it holds."""
    where = "make_cache"
    if k.dim() != 4 or _dtype_of(k) < 0 or (k_scale is None) != (v_scale is None) or (_dtype_of(k) == E4M3) != (k_scale is not None):
        _bad(where)
    pages, h, page, d = (int(n) for n in k.shape)
    _of_one_device(where, k, v, k_scale, v_scale)
    code = _dtype_of(k)
    c = Cache(pages, page, h, d, code, _dense(k, k.shape, code, where), _dense(v, k.shape, code, where),
              _dense(k_scale, (pages, h, page), F32, where), _dense(v_scale, (pages, h, page), F32, where))
    c.held, c.device = (k, v, k_scale, v_scale), k.get_device()
    return c


def _indices(t, dim: int, where: str):
    import torch
    if t is None:
        return None
    if not (t.is_cuda and t.dtype == torch.int32 and t.dim() == dim and t.is_contiguous()):
        _bad(where)
    return t.data_ptr()


def make_batch(offsets, lens, table, prefix=None, prefix_len: int = 0) -> Batch:
    """Descriptor of a batch over int32 device tensors: offsets [B + 1], lens [B], table [B][pages of the longest], and prefix [pages],
    those of the prefix_len tokens that come before every sequence's own.  It holds the tensors; their contents may change between calls."""
    where = "make_batch"
    prefix_len = _int32(prefix_len, where)
    v = [_indices(t, n, where) for t, n in ((offsets, 1), (lens, 1), (table, 2), (prefix, 1))]
    _of_one_device(where, offsets, lens, table, prefix)
    n = int(lens.shape[0])
    if offsets.shape[0] != n + 1 or table.shape[0] != n or (n and not table.shape[1]) or prefix_len < 0 or (prefix_len and prefix is None):
        _bad(where)
    b = Batch(_int32(n, where), _int32(table.shape[1], where), *v, prefix_len)
    b.held, b.device, b.prefix_pages = (offsets, lens, table, prefix), lens.get_device(), 0 if prefix is None else int(prefix.shape[0])
    return b


def _here(c: Cache, b: Batch, t, where: str) -> None:
    """Refuses descriptors over another device than the rows t (which the call checks against the current one)."""
    d = t.get_device()
    if c.device not in (None, d) or b.device not in (None, d):
        _bad(where)


def laud_attention(p: Heads, offsets, q, k, v, keep, out) -> None:
    """q, out [T][heads * D] and k, v [T][kv_heads * D] of one type, rows any distance apart; offsets [B + 1] int32; keep [T] bytes or
    None."""
    s = (_calls or _token_calls()).attention(p, offsets, q, k, v, keep, out)
    if s:
        raise LaudError(s, "laud_attention")


def laud_cache_write(c: Cache, b: Batch, k, v) -> None:
    """Rows k, v [T][kv_heads * D] to their places in the cache."""
    _here(c, b, k, "laud_cache_write")
    s = (_calls or _token_calls()).cache_write(c, b, k, v)
    if s:
        raise LaudError(s, "laud_cache_write")


def laud_cache_read(c: Cache, b: Batch, k, v) -> None:
    """Rows k, v [T][kv_heads * D] from their places in the cache."""
    _here(c, b, k, "laud_cache_read")
    s = (_calls or _token_calls()).cache_read(c, b, k, v)
    if s:
        raise LaudError(s, "laud_cache_read")


def cache_attention_workspace(p: Heads, c: Cache, b: Batch, t: int) -> int:
    return int(load().laud_cache_attention_workspace(C.byref(p), C.byref(c), C.byref(b), _int32(t, "cache_attention_workspace")))


def laud_cache_attention(p: Heads, c: Cache, b: Batch, q, out, ws=None) -> None:
    """q, out [T][heads * D]: new tokens over the cached ones of their sequences.  ws: cache_attention_workspace(p, c, b, T) bytes on the
    device (None where that is 0); calls that run at once need one each."""
    if b.prefix_len > getattr(b, "prefix_pages", b.prefix_len) * c.page:
        _bad("laud_cache_attention")
    _here(c, b, q, "laud_cache_attention")
    s = (_calls or _token_calls()).cache_attention(p, c, b, q, out, ws)
    if s:
        raise LaudError(s, "laud_cache_attention")


def laud_stage_timing_enable(on: bool) -> None:
    _check(load().laud_stage_timing_enable(1 if on else 0), "laud_stage_timing_enable")


def laud_stage_timing_read() -> dict[str, tuple[float, int]]:
    """{stage name: (total milliseconds, launches)} for the stages that ran since enabling."""
    ms = (C.c_double * STAGE_COUNT)()
    n = (C.c_int64 * STAGE_COUNT)()
    _check(load().laud_stage_timing_read(ms, n), "laud_stage_timing_read")
    return {load().laud_stage_name(i).decode(): (float(ms[i]), int(n[i])) for i in range(STAGE_COUNT) if n[i]}
