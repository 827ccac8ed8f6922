"""ctypes binding of libmoe_hip.so: argument marshalling only.

Every function here has the name and the argument order of the C entry point
declared in include/moe.h and does nothing but check tensor device, dtype and
contiguity, and pass raw device pointers plus the current HIP stream.  PyTorch
is used for device memory and streams only; every step of the layer runs in the
library's kernels.  There is no fallback: if the shared library is missing, or
a call returns a non-zero status, an exception is raised.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmoe_hip.so")

MOE_F32, MOE_BF16 = 0, 1
MOE_OK = 0
MOE_FLAG_PACKED_WEIGHTS = 1
MOE_FLAG_PACKED_GATE = 2
MOE_ROPE_HALF, MOE_ROPE_INTERLEAVED = 0, 1
MOE_ROPE_PLAIN, MOE_ROPE_LINEAR, MOE_ROPE_BY_PARTS = 0, 1, 2
MOE_CACHE_BF16, MOE_CACHE_FP8, MOE_CACHE_FP4 = 0, 1, 2
ENTRY_POINTS = ("moe_workspace_bytes", "moe_status_string", "moe_version", "moe_packed_weights_bytes",
                "moe_pack_weights", "moe_packed_gate_bytes", "moe_pack_gate", "moe_gate", "moe_gate_noalloc",
                "moe_gate_noalloc_bytes", "moe_gate_noalloc_max_bytes", "moe_dispatch",
                "moe_expert_ffn", "moe_expert_ffn_slice", "moe_expert_ffn_slice_reduce", "moe_combine", "moe_layer_forward", "moe_decode_block_workspace_bytes",
                "moe_decode_block_forward", "moe_rope_frequencies", "moe_rope", "moe_cache_bytes", "moe_cache_scale_bytes",
                "moe_cache_write", "moe_cache_read", "moe_tree_attention_workspace_bytes", "moe_tree_attention",
                "moe_draft_block_workspace_bytes", "moe_draft_block_forward", "moe_i8_weights_bytes", "moe_i8_quantize_weights", "moe_i8_pack_weights",
                "moe_i8_quantize_rows", "moe_i8_linear", "moe_i8_workspace_bytes", "moe_i8_expert_ffn", "moe_i8_layer_forward", "moe_profile_enable", "moe_profile_select",
                "moe_profile_stride", "moe_profile_calls",
                "moe_profile_stage_count", "moe_profile_stage_name", "moe_profile_elapsed")


class MoeShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("T", "d_model", "d_ffn", "E", "top_k", "capacity", "dtype", "residual", "flags")]


class MoeBlockShape(ctypes.Structure):
    _fields_ = [("n_heads", ctypes.c_int32), ("max_len", ctypes.c_int32)]


BLOCK_WEIGHT_FIELDS = ("ln1_gamma", "ln1_beta", "Wqkv", "bqkv", "Wo", "bo", "ln2_gamma", "ln2_beta", "Wg", "bg",
                       "W1", "b1", "W2", "b2", "Wd1", "bd1", "Wd2", "bd2")


class MoeBlockWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in BLOCK_WEIGHT_FIELDS]


class MoeRope(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("head_dim", "rot_dim", "layout", "dtype", "scaling")] + [("amplitude", ctypes.c_float)] + \
        [(n, ctypes.c_double) for n in ("base", "factor", "original_len", "low", "high")]


class MoeCacheShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_seq", "n_heads", "n_kv_heads", "head_dim", "max_len", "kind")]


class MoeI8Linear(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_rows", "K", "N", "out_dtype", "gelu")]


I8_WEIGHT_FIELDS = ("W1", "s1", "b1", "W2", "s2", "b2", "Wd1", "sd1", "bd1", "Wd2", "sd2", "bd2")


class MoeI8Weights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in I8_WEIGHT_FIELDS]


class MoeError(RuntimeError):
    def __init__(self, fn: str, status: int, text: str):
        super().__init__(f"{fn} failed: status {status} ({text})")
        self.status = status


_lib = None


def load_library() -> ctypes.CDLL:
    """Load libmoe_hip.so (built by ``python -m paper_2201_05596_amd.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run `python -m paper_2201_05596_amd.build`")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, st = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    sp = ctypes.POINTER(MoeShape)
    lib.moe_workspace_bytes.restype = st
    lib.moe_workspace_bytes.argtypes = [sp]
    lib.moe_status_string.restype = ctypes.c_char_p
    lib.moe_status_string.argtypes = [i32]
    lib.moe_version.restype = ctypes.c_char_p
    lib.moe_version.argtypes = []
    lib.moe_packed_weights_bytes.restype = st
    lib.moe_packed_weights_bytes.argtypes = [i32, i32, i32]
    lib.moe_pack_weights.restype = i32
    lib.moe_pack_weights.argtypes = [i32, i32, i32, vp, vp, vp]
    lib.moe_packed_gate_bytes.restype = st
    lib.moe_packed_gate_bytes.argtypes = [i32, i32]
    lib.moe_pack_gate.restype = i32
    lib.moe_pack_gate.argtypes = [i32, i32, vp, vp, vp]
    lib.moe_gate.restype = i32
    lib.moe_gate.argtypes = [sp] + [vp] * 9 + [vp, st, vp]
    lib.moe_gate_noalloc.restype = i32
    lib.moe_gate_noalloc.argtypes = [sp] + [vp] * 9 + [vp]
    lib.moe_gate_noalloc_bytes.restype = st
    lib.moe_gate_noalloc_bytes.argtypes = [sp]
    lib.moe_gate_noalloc_max_bytes.restype = st
    lib.moe_gate_noalloc_max_bytes.argtypes = []
    lib.moe_dispatch.restype = i32
    lib.moe_dispatch.argtypes = [sp] + [vp] * 4 + [vp]
    lib.moe_expert_ffn.restype = i32
    lib.moe_expert_ffn.argtypes = [sp] + [vp] * 7 + [vp, st, vp]
    lib.moe_expert_ffn_slice.restype = i32
    lib.moe_expert_ffn_slice.argtypes = [sp] + [vp] * 6 + [vp, st, vp]
    lib.moe_expert_ffn_slice_reduce.restype = i32
    lib.moe_expert_ffn_slice_reduce.argtypes = [sp, i32] + [vp] * 4 + [vp]
    lib.moe_combine.restype = i32
    lib.moe_combine.argtypes = [sp] + [vp] * 6 + [vp]
    lib.moe_layer_forward.restype = i32
    lib.moe_layer_forward.argtypes = [sp] + [vp] * 18 + [vp, st, vp]
    lib.moe_decode_block_workspace_bytes.restype = st
    lib.moe_decode_block_workspace_bytes.argtypes = [sp, ctypes.POINTER(MoeBlockShape)]
    lib.moe_decode_block_forward.restype = i32
    lib.moe_decode_block_forward.argtypes = [sp, ctypes.POINTER(MoeBlockShape), ctypes.POINTER(MoeBlockWeights)] + \
        [vp] * 8 + [vp, st, vp]
    rp, cp, i64 = ctypes.POINTER(MoeRope), ctypes.POINTER(MoeCacheShape), ctypes.c_int64
    lib.moe_rope_frequencies.restype = i32
    lib.moe_rope_frequencies.argtypes = [rp, vp]
    lib.moe_rope.restype = i32
    lib.moe_rope.argtypes = [rp, i32, i32, vp, i64, vp, vp, vp, i64, vp]
    lib.moe_cache_bytes.restype = st
    lib.moe_cache_bytes.argtypes = [cp]
    lib.moe_cache_scale_bytes.restype = st
    lib.moe_cache_scale_bytes.argtypes = [cp]
    lib.moe_cache_write.restype = i32
    lib.moe_cache_write.argtypes = [cp, i32, vp, i64, vp, i64] + [vp] * 7
    lib.moe_cache_read.restype = i32
    lib.moe_cache_read.argtypes = [cp, i32] + [vp] * 6 + [vp, i64, vp, i64, vp]
    lib.moe_tree_attention_workspace_bytes.restype = st
    lib.moe_tree_attention_workspace_bytes.argtypes = [cp, i32]
    lib.moe_tree_attention.restype = i32
    lib.moe_tree_attention.argtypes = [cp, i32] + [vp, i64] * 3 + [vp] * 7 + [vp, i64, vp, st, vp]
    lib.moe_draft_block_workspace_bytes.restype = st
    lib.moe_draft_block_workspace_bytes.argtypes = [sp, cp, i32]
    lib.moe_draft_block_forward.restype = i32
    lib.moe_draft_block_forward.argtypes = [sp, cp, i32, rp, ctypes.POINTER(MoeBlockWeights)] + [vp] * 14 + [vp, st, vp]
    lib.moe_i8_weights_bytes.restype = st
    lib.moe_i8_weights_bytes.argtypes = [i32] * 3
    lib.moe_i8_quantize_weights.restype = i32
    lib.moe_i8_quantize_weights.argtypes = [i32] * 3 + [vp] * 4
    lib.moe_i8_pack_weights.restype = i32
    lib.moe_i8_pack_weights.argtypes = [i32] * 3 + [vp] * 3
    lib.moe_i8_quantize_rows.restype = i32
    lib.moe_i8_quantize_rows.argtypes = [i32] * 3 + [vp, i64, vp, i64, vp, vp]
    lib.moe_i8_linear.restype = i32
    lib.moe_i8_linear.argtypes = [ctypes.POINTER(MoeI8Linear), vp, i64] + [vp] * 5 + [i64, vp]
    lib.moe_i8_workspace_bytes.restype = st
    lib.moe_i8_workspace_bytes.argtypes = [sp]
    wp = ctypes.POINTER(MoeI8Weights)
    lib.moe_i8_expert_ffn.restype = i32
    lib.moe_i8_expert_ffn.argtypes = [sp, wp] + [vp] * 4 + [st, vp]
    lib.moe_i8_layer_forward.restype = i32
    lib.moe_i8_layer_forward.argtypes = [sp, wp] + [vp] * 11 + [st, vp]
    lib.moe_profile_enable.restype = i32
    lib.moe_profile_enable.argtypes = [i32]
    lib.moe_profile_select.restype = i32
    lib.moe_profile_select.argtypes = [ctypes.c_uint]
    lib.moe_profile_stride.restype = i32
    lib.moe_profile_stride.argtypes = [i32]
    lib.moe_profile_calls.restype = i32
    lib.moe_profile_calls.argtypes = []
    lib.moe_profile_stage_count.restype = i32
    lib.moe_profile_stage_count.argtypes = []
    lib.moe_profile_stage_name.restype = ctypes.c_char_p
    lib.moe_profile_stage_name.argtypes = [i32]
    lib.moe_profile_elapsed.restype = i32
    lib.moe_profile_elapsed.argtypes = [i32, ctypes.POINTER(ctypes.c_float)]
    _lib = lib
    return lib


def make_shape(T: int, d_model: int, d_ffn: int, E: int, top_k: int, capacity: int, dtype, residual: bool = False,
               flags: int = 0) -> MoeShape:
    if isinstance(dtype, torch.dtype):
        dtype = {torch.float32: MOE_F32, torch.bfloat16: MOE_BF16}[dtype]
    elif isinstance(dtype, str):
        dtype = {"f32": MOE_F32, "bf16": MOE_BF16}[dtype]
    return MoeShape(T, d_model, d_ffn, E, top_k, capacity, int(dtype), int(bool(residual)), int(flags))


def _ptr(t: Optional[torch.Tensor], dtype: Optional[torch.dtype] = None, numel: Optional[int] = None,
         name: str = "tensor") -> Optional[int]:
    """Device address of a tensor argument after checking what the C ABI cannot: device, contiguity, dtype and, when
    `numel` is given, the element count (a buffer sized for another shape would be indexed out of bounds on the GPU)."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name}: device tensor required")
    if not t.is_contiguous():
        raise ValueError(f"{name}: contiguous tensor required")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name}: expected {dtype}, got {t.dtype}")
    if numel is not None and t.numel() != numel:
        raise ValueError(f"{name}: expected {numel} elements for this shape, got {t.numel()}")
    return t.data_ptr()


def _ws(shape, ws, need: Optional[int] = None):
    """(address, bytes) of a workspace tensor; `need`: the byte count the call requires (checked here as well)."""
    if ws is None:
        return None, 0
    nbytes = ws.numel() * ws.element_size()
    if need is not None and nbytes < need:
        raise ValueError(f"workspace: {nbytes} bytes, this shape needs {need}")
    return _ptr(ws, name="ws"), nbytes


def _w(shape, G: int, K: int, N: int) -> int:
    """Elements of an FFN weight array [G,K,N]: plain, or as moe_pack_weights lays it out."""
    if shape.flags & MOE_FLAG_PACKED_WEIGHTS:
        return G * ((K + 31) // 32) * ((N + 127) // 128) * 4096
    return G * K * N


def _wg(shape) -> int:
    """float32 elements of the gate weights: plain [d,E], or the buffer moe_pack_gate returns."""
    if shape.flags & MOE_FLAG_PACKED_GATE:
        return (_packed_gate_bytes(shape.d_model, shape.E) + 3) // 4
    return shape.d_model * shape.E


def _stream() -> int:
    # torch.cuda.current_stream().cuda_stream without the Stream object, whose making is 1 us of a call of 20
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _check(fn: str, status: int) -> None:
    if status != MOE_OK:
        raise MoeError(fn, status, load_library().moe_status_string(status).decode())


def _elem(shape: MoeShape) -> torch.dtype:
    return torch.float32 if shape.dtype == MOE_F32 else torch.bfloat16


def moe_workspace_bytes(shape: MoeShape) -> int:
    return int(load_library().moe_workspace_bytes(ctypes.byref(shape)))


# Byte counts that every call asks for, by the values they depend on (not by the object that holds them)
@functools.lru_cache(maxsize=256)
def _workspace_need(shape: bytes) -> int:
    return moe_workspace_bytes(MoeShape.from_buffer_copy(shape))


@functools.lru_cache(maxsize=256)
def _block_workspace_need(shape: bytes, block: bytes) -> int:
    return moe_decode_block_workspace_bytes(MoeShape.from_buffer_copy(shape), MoeBlockShape.from_buffer_copy(block))


@functools.lru_cache(maxsize=256)
def _packed_gate_bytes(d_model: int, E: int) -> int:
    return moe_packed_gate_bytes(d_model, E)


def moe_version() -> str:
    return load_library().moe_version().decode()


def alloc_workspace(shape: MoeShape, device="cuda") -> torch.Tensor:
    """Device memory for the `ws` argument (plumbing: torch owns the allocation)."""
    n = moe_workspace_bytes(shape)
    if n == 0:
        raise MoeError("moe_workspace_bytes", -1, "invalid shape")
    return torch.empty(n, dtype=torch.uint8, device=device)


def moe_packed_weights_bytes(G: int, K: int, N: int) -> int:
    return int(load_library().moe_packed_weights_bytes(int(G), int(K), int(N)))


def moe_pack_weights(W: torch.Tensor) -> torch.Tensor:
    """Packed copy of bf16 weights [G,K,N] (or [K,N]) for MOE_FLAG_PACKED_WEIGHTS; torch owns the new buffer."""
    G, K, N = (1, *W.shape) if W.dim() == 2 else W.shape
    nbytes = moe_packed_weights_bytes(G, K, N)
    if nbytes == 0:
        raise MoeError("moe_packed_weights_bytes", -2, "unsupported size")
    packed = torch.empty(nbytes // 2, dtype=torch.bfloat16, device=W.device)
    _check("moe_pack_weights", load_library().moe_pack_weights(G, K, N, _ptr(W, torch.bfloat16), _ptr(packed), _stream()))
    return packed


def moe_packed_gate_bytes(d_model: int, E: int) -> int:
    return int(load_library().moe_packed_gate_bytes(int(d_model), int(E)))


def moe_pack_gate(Wg: torch.Tensor) -> Optional[torch.Tensor]:
    """Packed copy of the float gate weights [d,E] for MOE_FLAG_PACKED_GATE, or None when the shape is not covered.
    The buffer is typed float32 only so that it passes where Wg is expected; its contents are bf16 triples."""
    d, E = Wg.shape
    nbytes = moe_packed_gate_bytes(d, E)
    if nbytes == 0:
        return None
    packed = torch.empty((nbytes + 3) // 4, dtype=torch.float32, device=Wg.device)
    _check("moe_pack_gate", load_library().moe_pack_gate(d, E, _ptr(Wg, torch.float32), _ptr(packed), _stream()))
    return packed


def _gate_args(shape, x, Wg, bg, logits, expert_idx, slot_idx, gate_w, expert_rows, slot_token):
    i32, f32 = torch.int32, torch.float32
    T, d, E, k, C = shape.T, shape.d_model, shape.E, shape.top_k, shape.capacity
    return (_ptr(x, _elem(shape) if x is not None else None, T * d, "x"),
            _ptr(Wg, f32, _wg(shape) if x is not None else None, "Wg"), _ptr(bg, f32, E, "bg"),
            _ptr(logits, f32, T * E, "logits"), _ptr(expert_idx, i32, T * k, "expert_idx"),
            _ptr(slot_idx, i32, T * k, "slot_idx"), _ptr(gate_w, f32, T * k, "gate_w"),
            _ptr(expert_rows, i32, E, "expert_rows"), _ptr(slot_token, i32, E * C, "slot_token"))


def moe_gate(shape, x, Wg, bg, logits, expert_idx, slot_idx, gate_w, expert_rows, slot_token, ws) -> None:
    wsp, wsn = _ws(shape, ws, _workspace_need(bytes(shape)))
    rc = load_library().moe_gate(ctypes.byref(shape), *_gate_args(shape, x, Wg, bg, logits, expert_idx, slot_idx, gate_w,
                                                                 expert_rows, slot_token), wsp, wsn, _stream())
    _check("moe_gate", rc)


def moe_gate_noalloc(shape, x, Wg, bg, logits, expert_idx, slot_idx, gate_w, expert_rows, slot_token) -> None:
    rc = load_library().moe_gate_noalloc(ctypes.byref(shape), *_gate_args(shape, x, Wg, bg, logits, expert_idx, slot_idx,
                                                                         gate_w, expert_rows, slot_token), _stream())
    _check("moe_gate_noalloc", rc)


def moe_gate_noalloc_bytes(shape: MoeShape) -> int:
    return int(load_library().moe_gate_noalloc_bytes(ctypes.byref(shape)))


def moe_gate_noalloc_max_bytes() -> int:
    return int(load_library().moe_gate_noalloc_max_bytes())


def moe_dispatch(shape, x, slot_token, expert_rows, xe) -> None:
    el = _elem(shape)
    T, d, E, C = shape.T, shape.d_model, shape.E, shape.capacity
    rc = load_library().moe_dispatch(ctypes.byref(shape), _ptr(x, el, T * d, "x"),
                                     _ptr(slot_token, torch.int32, E * C, "slot_token"),
                                     _ptr(expert_rows, torch.int32, E, "expert_rows"), _ptr(xe, el, E * C * d, "xe"), _stream())
    _check("moe_dispatch", rc)


def moe_expert_ffn(shape, xe, expert_rows, W1, b1, W2, b2, ye, ws) -> None:
    el = _elem(shape)
    d, f, E, C = shape.d_model, shape.d_ffn, shape.E, shape.capacity
    wsp, wsn = _ws(shape, ws, _workspace_need(bytes(shape)))
    rc = load_library().moe_expert_ffn(
        ctypes.byref(shape), _ptr(xe, el, E * C * d, "xe"), _ptr(expert_rows, torch.int32, E, "expert_rows"),
        _ptr(W1, el, _w(shape, E, d, f), "W1"), _ptr(b1, el, E * f, "b1"), _ptr(W2, el, _w(shape, E, f, d), "W2"),
        _ptr(b2, el, E * d, "b2"), _ptr(ye, el, E * C * d, "ye"), wsp, wsn, _stream())
    _check("moe_expert_ffn", rc)


def moe_expert_ffn_slice(shape, xe, expert_rows, W1s, b1s, W2s, ye_partial, ws) -> None:
    el = _elem(shape)
    d, f, E, C = shape.d_model, shape.d_ffn, shape.E, shape.capacity
    wsp, wsn = _ws(shape, ws, _workspace_need(bytes(shape)))
    rc = load_library().moe_expert_ffn_slice(
        ctypes.byref(shape), _ptr(xe, el, E * C * d, "xe"), _ptr(expert_rows, torch.int32, E, "expert_rows"),
        _ptr(W1s, el, _w(shape, E, d, f), "W1s"), _ptr(b1s, el, E * f, "b1s"), _ptr(W2s, el, _w(shape, E, f, d), "W2s"),
        _ptr(ye_partial, torch.float32, E * C * d, "ye_partial"), wsp, wsn, _stream())
    _check("moe_expert_ffn_slice", rc)


def moe_expert_ffn_slice_reduce(shape, n_slices, ye_partials, expert_rows, b2, ye) -> None:
    el = _elem(shape)
    d, E, C = shape.d_model, shape.E, shape.capacity
    rc = load_library().moe_expert_ffn_slice_reduce(
        ctypes.byref(shape), int(n_slices), _ptr(ye_partials, torch.float32, int(n_slices) * E * C * d, "ye_partials"),
        _ptr(expert_rows, torch.int32, E, "expert_rows"), _ptr(b2, el, E * d, "b2"), _ptr(ye, el, E * C * d, "ye"), _stream())
    _check("moe_expert_ffn_slice_reduce", rc)


def moe_combine(shape, ye, expert_idx, slot_idx, gate_w, addend, out) -> None:
    el = _elem(shape)
    T, d, E, k, C = shape.T, shape.d_model, shape.E, shape.top_k, shape.capacity
    rc = load_library().moe_combine(ctypes.byref(shape), _ptr(ye, el, E * C * d, "ye"),
                                    _ptr(expert_idx, torch.int32, T * k, "expert_idx"),
                                    _ptr(slot_idx, torch.int32, T * k, "slot_idx"), _ptr(gate_w, torch.float32, T * k, "gate_w"),
                                    _ptr(addend, el, T * d, "addend"), _ptr(out, el, T * d, "out"), _stream())
    _check("moe_combine", rc)


def _ffn_weight_args(shape, W1, b1, W2, b2, Wd1, bd1, Wd2, bd2):
    el = _elem(shape)
    d, f, E = shape.d_model, shape.d_ffn, shape.E
    return (_ptr(W1, el, _w(shape, E, d, f), "W1"), _ptr(b1, el, E * f, "b1"), _ptr(W2, el, _w(shape, E, f, d), "W2"),
            _ptr(b2, el, E * d, "b2"), _ptr(Wd1, el, _w(shape, 1, d, f), "Wd1"), _ptr(bd1, el, f, "bd1"),
            _ptr(Wd2, el, _w(shape, 1, f, d), "Wd2"), _ptr(bd2, el, d, "bd2"))


def moe_layer_forward(shape, x, Wg, bg, W1, b1, W2, b2, Wd1, bd1, Wd2, bd2, out,
                      logits_out, expert_idx_out, slot_idx_out, gate_w_out, expert_rows_out, slot_token_out, ws) -> None:
    el, i32, f32 = _elem(shape), torch.int32, torch.float32
    T, d, E, k, C = shape.T, shape.d_model, shape.E, shape.top_k, shape.capacity
    wsp, wsn = _ws(shape, ws, _workspace_need(bytes(shape)))
    rc = load_library().moe_layer_forward(
        ctypes.byref(shape), _ptr(x, el, T * d, "x"), _ptr(Wg, f32, _wg(shape), "Wg"), _ptr(bg, f32, E, "bg"),
        *_ffn_weight_args(shape, W1, b1, W2, b2, Wd1, bd1, Wd2, bd2), _ptr(out, el, T * d, "out"),
        _ptr(logits_out, f32, T * E, "logits_out"), _ptr(expert_idx_out, i32, T * k, "expert_idx_out"),
        _ptr(slot_idx_out, i32, T * k, "slot_idx_out"), _ptr(gate_w_out, f32, T * k, "gate_w_out"),
        _ptr(expert_rows_out, i32, E, "expert_rows_out"), _ptr(slot_token_out, i32, E * C, "slot_token_out"),
        wsp, wsn, _stream())
    _check("moe_layer_forward", rc)


def moe_decode_block_workspace_bytes(shape: MoeShape, block: MoeBlockShape) -> int:
    return int(load_library().moe_decode_block_workspace_bytes(ctypes.byref(shape), ctypes.byref(block)))


def _block_weights(shape, weights: dict, width: int) -> MoeBlockWeights:
    """width: columns of Wqkv."""
    el, f32 = _elem(shape), torch.float32
    d, f, E = shape.d_model, shape.d_ffn, shape.E
    sizes = {"ln1_gamma": (f32, d), "ln1_beta": (f32, d), "ln2_gamma": (f32, d), "ln2_beta": (f32, d),
             "Wqkv": (el, d * width), "bqkv": (el, width), "Wo": (el, d * d), "bo": (el, d),
             "Wg": (f32, _wg(shape)), "bg": (f32, E), "W1": (el, _w(shape, E, d, f)), "b1": (el, E * f),
             "W2": (el, _w(shape, E, f, d)), "b2": (el, E * d), "Wd1": (el, _w(shape, 1, d, f)), "bd1": (el, f),
             "Wd2": (el, _w(shape, 1, f, d)), "bd2": (el, d)}
    return MoeBlockWeights(**{n: _ptr(weights.get(n), sizes[n][0], sizes[n][1], n) for n in BLOCK_WEIGHT_FIELDS})


def moe_decode_block_forward(shape, block, weights: dict, x, k_cache, v_cache, pos, out, x1_out, moe_in_out, logits_out,
                             ws) -> None:
    """`weights`: name -> tensor (or None) for the fields of moe_block_weights_t."""
    el, f32 = _elem(shape), torch.float32
    T, d, E = shape.T, shape.d_model, shape.E
    cache = T * d * block.max_len                      # [T, H, max_len, d/H]
    w = _block_weights(shape, weights, 3 * d)
    wsp, wsn = _ws(shape, ws, _block_workspace_need(bytes(shape), bytes(block)))
    rc = load_library().moe_decode_block_forward(
        ctypes.byref(shape), ctypes.byref(block), ctypes.byref(w), _ptr(x, el, T * d, "x"),
        _ptr(k_cache, el, cache, "k_cache"), _ptr(v_cache, el, cache, "v_cache"), _ptr(pos, torch.int32, T, "pos"),
        _ptr(out, el, T * d, "out"), _ptr(x1_out, el, T * d, "x1_out"), _ptr(moe_in_out, el, T * d, "moe_in_out"),
        _ptr(logits_out, f32, T * E, "logits_out"), wsp, wsn, _stream())
    _check("moe_decode_block_forward", rc)


# ---- several new tokens per sequence ---------------------------------------------------------------------------

# A step makes several of these calls for a few microseconds of kernels each, so a tensor is looked at once, and what is wrong
# with it is worked out only for the error.

def _refuse(t, dtype, numel, name: str):
    device = torch._C._cuda_getDevice()
    if not t.is_cuda:
        raise ValueError(f"{name}: device tensor required")
    if t.get_device() != device:
        raise ValueError(f"{name}: on cuda:{t.get_device()}, the launch goes to the current device cuda:{device}")
    if t.dtype is not dtype:
        raise ValueError(f"{name}: expected {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: contiguous tensor required")
    raise ValueError(f"{name}: expected {numel} elements for this shape, got {t.numel()}")


def _at(t, device: int, dtype, numel: int, name: str):
    """Address of a contiguous tensor on the current device, or None."""
    if t is None:
        return None
    if t.get_device() != device or t.dtype is not dtype or t.numel() != numel or not t.is_contiguous():
        _refuse(t, dtype, numel, name)
    return t.data_ptr()


def _rows(t, device: int, dtype, rows: int, cols: int, name: str):
    """(address, distance between rows in elements) of [rows, cols], whose rows may be columns of wider ones."""
    if t.get_device() != device or t.dtype is not dtype:
        _refuse(t, dtype, rows * cols, name)
    if t.shape != (rows, cols):
        raise ValueError(f"{name}: expected shape {(rows, cols)}, got {tuple(t.shape)}")
    between, inside = t.stride()
    if inside != 1 and cols > 1:
        raise ValueError(f"{name}: the elements of a row have to be adjacent")
    return t.data_ptr(), between if rows > 1 else cols


def _workspace(ws, device: int, need: int):
    """(address, bytes) of a workspace tensor of any type; None where nothing is needed (the library then refuses the shape)."""
    nbytes = 0 if ws is None else ws.numel() * ws.element_size()
    if nbytes < need:
        raise ValueError(f"workspace: {nbytes} bytes, this shape needs {need}")
    return (None, 0) if ws is None else (_at(ws, device, ws.dtype, ws.numel(), "ws"), nbytes)


def make_rope(head_dim: int, rot_dim: int, layout, dtype, base: float = 10000.0, amplitude: float = 1.0, scaling="plain",
              factor: float = 1.0, original_len: float = 1.0, low: float = 1.0, high: float = 4.0) -> MoeRope:
    """layout: "half" or "interleaved"; scaling: "plain", "linear" or "by_parts" (or the MOE_ROPE_* numbers)."""
    if isinstance(layout, str):
        layout = {"half": MOE_ROPE_HALF, "interleaved": MOE_ROPE_INTERLEAVED}[layout]
    if isinstance(scaling, str):
        scaling = {"plain": MOE_ROPE_PLAIN, "linear": MOE_ROPE_LINEAR, "by_parts": MOE_ROPE_BY_PARTS}[scaling]
    if isinstance(dtype, torch.dtype):
        dtype = {torch.float32: MOE_F32, torch.bfloat16: MOE_BF16}[dtype]
    elif isinstance(dtype, str):
        dtype = {"f32": MOE_F32, "bf16": MOE_BF16}[dtype]
    return MoeRope(head_dim, rot_dim, int(layout), int(dtype), int(scaling), amplitude, base, factor, original_len, low, high)


def moe_rope_frequencies(rope: MoeRope, device="cuda") -> torch.Tensor:
    """Turns per position [rot_dim / 2], float64, on `device`: the `turns` of moe_rope."""
    host = torch.empty(max(rope.rot_dim, 2) // 2, dtype=torch.float64)
    _check("moe_rope_frequencies", load_library().moe_rope_frequencies(ctypes.byref(rope), host.data_ptr()))
    return host.to(device)


def moe_rope(rope: MoeRope, x, turns, pos, out) -> None:
    """x, out: [rows, heads * head_dim], columns of wider rows if need be; out may be x."""
    dtype = torch.float32 if rope.dtype == MOE_F32 else torch.bfloat16
    rows, cols = x.shape
    if rows == 0:
        return
    heads = cols // rope.head_dim if rope.head_dim > 0 else 1      # (no such head: the library refuses the shape)
    if rope.head_dim > 0 and (cols == 0 or cols % rope.head_dim):
        raise ValueError(f"x: {cols} columns are no heads of {rope.head_dim}")
    dev = torch._C._cuda_getDevice()
    xp, xs = _rows(x, dev, dtype, rows, cols, "x")
    op, os_ = _rows(out, dev, dtype, rows, cols, "out")
    rc = load_library().moe_rope(ctypes.byref(rope), rows, heads, xp, xs, _at(turns, dev, torch.float64, rope.rot_dim // 2, "turns"),
                                 _at(pos, dev, torch.int32, rows, "pos"), op, os_, torch._C._cuda_getCurrentRawStream(dev))
    _check("moe_rope", rc)


def make_cache_shape(n_seq: int, n_heads: int, n_kv_heads: int, head_dim: int, max_len: int, kind) -> MoeCacheShape:
    """kind: "bf16", "fp8" or "fp4" (or the MOE_CACHE_* numbers)."""
    if isinstance(kind, str):
        kind = {"bf16": MOE_CACHE_BF16, "fp8": MOE_CACHE_FP8, "fp4": MOE_CACHE_FP4}[kind]
    return MoeCacheShape(n_seq, n_heads, n_kv_heads, head_dim, max_len, int(kind))


def moe_cache_bytes(cache: MoeCacheShape) -> int:
    return int(load_library().moe_cache_bytes(ctypes.byref(cache)))


def moe_cache_scale_bytes(cache: MoeCacheShape) -> int:
    return int(load_library().moe_cache_scale_bytes(ctypes.byref(cache)))


def alloc_cache(cache: MoeCacheShape, device="cuda"):
    """(k_cache, v_cache, k_scale, v_scale): bf16, or uint8 with [n_seq, n_kv_heads, max_len, head_dim / 32] scales; scales None for bf16."""
    if moe_cache_bytes(cache) == 0:
        raise MoeError("moe_cache_bytes", -1, "invalid shape")
    B, G, L, dh = cache.n_seq, cache.n_kv_heads, cache.max_len, cache.head_dim
    if cache.kind == MOE_CACHE_BF16:
        return *(torch.zeros((B, G, L, dh), dtype=torch.bfloat16, device=device) for _ in "kv"), None, None
    cols = dh if cache.kind == MOE_CACHE_FP8 else dh // 2
    return *(torch.zeros((B, G, L, cols), dtype=torch.uint8, device=device) for _ in "kv"), \
        *(torch.zeros((B, G, L, dh // 32), dtype=torch.uint8, device=device) for _ in "kv")


def _cache_args(cache, device: int, k_cache, v_cache, k_scale, v_scale):
    kind, dh = cache.kind, cache.head_dim
    total = cache.n_seq * cache.n_kv_heads * cache.max_len
    if kind == MOE_CACHE_BF16:
        el, n = torch.bfloat16, total * dh
    else:
        el, n = torch.uint8, total * dh // (1 if kind == MOE_CACHE_FP8 else 2)
    x = total * (dh // 32)
    return (_at(k_cache, device, el, n, "k_cache"), _at(v_cache, device, el, n, "v_cache"), _at(k_scale, device, torch.uint8, x, "k_scale"),
            _at(v_scale, device, torch.uint8, x, "v_scale"))


def moe_cache_write(cache, k, v, seq, pos, k_cache, v_cache, k_scale, v_scale) -> None:
    """k, v: [rows, n_kv_heads * head_dim] bf16, columns of wider rows if need be; seq, pos: [rows] int32."""
    rows, cols = k.shape[0], cache.n_kv_heads * cache.head_dim
    if rows == 0:
        return
    dev, bf = torch._C._cuda_getDevice(), torch.bfloat16
    rc = load_library().moe_cache_write(
        ctypes.byref(cache), rows, *_rows(k, dev, bf, rows, cols, "k"), *_rows(v, dev, bf, rows, cols, "v"), _at(seq, dev, torch.int32, rows, "seq"),
        _at(pos, dev, torch.int32, rows, "pos"), *_cache_args(cache, dev, k_cache, v_cache, k_scale, v_scale), torch._C._cuda_getCurrentRawStream(dev))
    _check("moe_cache_write", rc)


def moe_cache_read(cache, k_cache, v_cache, k_scale, v_scale, seq, pos, k, v) -> None:
    """The reverse of moe_cache_write: fills the rows of k and v."""
    rows, cols = k.shape[0], cache.n_kv_heads * cache.head_dim
    if rows == 0:
        return
    dev, bf = torch._C._cuda_getDevice(), torch.bfloat16
    rc = load_library().moe_cache_read(
        ctypes.byref(cache), rows, *_cache_args(cache, dev, k_cache, v_cache, k_scale, v_scale), _at(seq, dev, torch.int32, rows, "seq"),
        _at(pos, dev, torch.int32, rows, "pos"), *_rows(k, dev, bf, rows, cols, "k"), *_rows(v, dev, bf, rows, cols, "v"),
        torch._C._cuda_getCurrentRawStream(dev))
    _check("moe_cache_read", rc)


def moe_tree_attention_workspace_bytes(cache: MoeCacheShape, n_draft: int) -> int:
    return int(load_library().moe_tree_attention_workspace_bytes(ctypes.byref(cache), int(n_draft)))


@functools.lru_cache(maxsize=256)
def _tree_workspace_need(cache: bytes, n_draft: int) -> int:
    return moe_tree_attention_workspace_bytes(MoeCacheShape.from_buffer_copy(cache), n_draft)


def moe_tree_attention(cache, n_draft: int, q, k, v, k_cache, v_cache, k_scale, v_scale, lens, counts, tree, out, ws) -> None:
    """q, out: [n_seq * n_draft, n_heads * head_dim], k, v: [n_seq * n_draft, n_kv_heads * head_dim] bf16, columns of wider rows if
    need be; counts and tree may be None."""
    bf, i32, dev = torch.bfloat16, torch.int32, torch._C._cuda_getDevice()
    B, dh = cache.n_seq, cache.head_dim
    T, qw, kw = B * n_draft, cache.n_heads * dh, cache.n_kv_heads * dh
    wp, nbytes = _workspace(ws, dev, _tree_workspace_need(bytes(cache), n_draft))
    rc = load_library().moe_tree_attention(
        ctypes.byref(cache), n_draft, *_rows(q, dev, bf, T, qw, "q"), *_rows(k, dev, bf, T, kw, "k"), *_rows(v, dev, bf, T, kw, "v"),
        *_cache_args(cache, dev, k_cache, v_cache, k_scale, v_scale), _at(lens, dev, i32, B, "lens"), _at(counts, dev, i32, B, "counts"),
        _at(tree, dev, i32, T * ((n_draft + 31) // 32), "tree"), *_rows(out, dev, bf, T, qw, "out"), wp, nbytes,
        torch._C._cuda_getCurrentRawStream(dev))
    _check("moe_tree_attention", rc)


def moe_draft_block_workspace_bytes(shape: MoeShape, cache: MoeCacheShape, n_draft: int) -> int:
    return int(load_library().moe_draft_block_workspace_bytes(ctypes.byref(shape), ctypes.byref(cache), int(n_draft)))


@functools.lru_cache(maxsize=256)
def _draft_workspace_need(shape: bytes, cache: bytes, n_draft: int) -> int:
    return moe_draft_block_workspace_bytes(MoeShape.from_buffer_copy(shape), MoeCacheShape.from_buffer_copy(cache), n_draft)


def moe_draft_block_forward(shape, cache, n_draft: int, rope, weights: dict, x, turns, pos, k_cache, v_cache, k_scale, v_scale, lens, tree, qkv, out,
                            x1_out, moe_in_out, logits_out, ws) -> None:
    """`weights` as in moe_decode_block_forward, with Wqkv [d, d + 2 n_kv_heads head_dim]; rope, turns and pos may be None."""
    el, f32, i32, dev = torch.bfloat16, torch.float32, torch.int32, torch._C._cuda_getDevice()
    T, d, E = shape.T, shape.d_model, shape.E
    width = d + 2 * cache.n_kv_heads * cache.head_dim
    w = _block_weights(shape, weights, width)
    wp, nbytes = _workspace(ws, dev, _draft_workspace_need(bytes(shape), bytes(cache), n_draft))
    rc = load_library().moe_draft_block_forward(
        ctypes.byref(shape), ctypes.byref(cache), n_draft, None if rope is None else ctypes.byref(rope), ctypes.byref(w), _at(x, dev, el, T * d, "x"),
        _at(turns, dev, torch.float64, 0 if rope is None else rope.rot_dim // 2, "turns"), _at(pos, dev, i32, T, "pos"),
        *_cache_args(cache, dev, k_cache, v_cache, k_scale, v_scale), _at(lens, dev, i32, cache.n_seq, "lens"),
        _at(tree, dev, i32, T * ((n_draft + 31) // 32), "tree"), _at(qkv, dev, el, T * width, "qkv"), _at(out, dev, el, T * d, "out"),
        _at(x1_out, dev, el, T * d, "x1_out"), _at(moe_in_out, dev, el, T * d, "moe_in_out"), _at(logits_out, dev, f32, T * E, "logits_out"),
        wp, nbytes, torch._C._cuda_getCurrentRawStream(dev))
    _check("moe_draft_block_forward", rc)


# ---- products in 8-bit integers ----------------------------------------------------------------------------------

# looked up once: a call's kernels take as long as its Python
_BF16, _F32, _INT8 = torch.bfloat16, torch.float32, torch.int8
_get_device, _get_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream

_MOST = (1 << 31) - 1          # ctypes passes what is left of a larger size in 32 bits


def moe_i8_weights_bytes(G: int, K: int, N: int) -> int:
    if not (0 < G <= _MOST and 0 < K <= _MOST and 0 < N <= _MOST):
        return 0
    return int(load_library().moe_i8_weights_bytes(int(G), int(K), int(N)))


def _i8_matrix(t: torch.Tensor, name: str):
    """(groups, K, N, empty buffer) for weights [G,K,N] or [K,N]."""
    if t.dim() not in (2, 3):
        raise ValueError(f"{name}: expected [K, N] or [G, K, N], got {tuple(t.shape)}")
    G, K, N = (1, *t.shape) if t.dim() == 2 else t.shape
    nbytes = moe_i8_weights_bytes(G, K, N)
    if nbytes == 0:
        raise MoeError("moe_i8_weights_bytes", -2, "unsupported size")
    return G, K, N, torch.empty(nbytes, dtype=torch.int8, device=t.device)


def moe_i8_quantize_weights(W: torch.Tensor):
    """(packed codes, scale [G,N] or [N]) of bf16 weights [G,K,N] or [K,N]; torch owns the new buffers."""
    G, K, N, packed = _i8_matrix(W, "W")
    scale = torch.empty(W.shape[:-2] + (N,), dtype=torch.float32, device=W.device)
    dev = _get_device()
    _check("moe_i8_quantize_weights", load_library().moe_i8_quantize_weights(
        G, K, N, _at(W, dev, torch.bfloat16, G * K * N, "W"), packed.data_ptr(), scale.data_ptr(), _get_stream(dev)))
    return packed, scale


def moe_i8_pack_weights(codes: torch.Tensor) -> torch.Tensor:
    """Packed copy of int8 codes [G,K,N] or [K,N]; torch owns the new buffer."""
    G, K, N, packed = _i8_matrix(codes, "codes")
    dev = _get_device()
    _check("moe_i8_pack_weights", load_library().moe_i8_pack_weights(
        G, K, N, _at(codes, dev, torch.int8, G * K * N, "codes"), packed.data_ptr(), _get_stream(dev)))
    return packed


def _i8_rows(t, device: int, dtype, rows: int, cols: int, name: str):
    """_rows, for [rows, cols or more] of which cols are read or written."""
    shape = t.shape
    if t.get_device() != device or t.dtype is not dtype:
        _refuse(t, dtype, rows * cols, name)
    if len(shape) != 2 or shape[0] != rows or shape[1] < cols:
        raise ValueError(f"{name}: expected {rows} rows of at least {cols}, got {tuple(shape)}")
    between, inside = t.stride()
    if inside != 1:
        raise ValueError(f"{name}: the elements of a row have to be adjacent")
    return t.data_ptr(), between if rows > 1 else cols


def moe_i8_quantize_rows(x, codes, scale) -> None:
    """x: [rows, cols] bf16 or float32, columns of wider rows if need be; codes: int8 [rows, at least cols rounded up to 64]."""
    rows, cols = x.shape
    if rows == 0:
        return
    dtype = x.dtype
    if dtype is not _BF16 and dtype is not _F32:
        raise ValueError(f"x: expected float32 or bfloat16, got {dtype}")
    if rows > _MOST or cols > _MOST:
        raise MoeError("moe_i8_quantize_rows", -2, "unsupported size")
    dev = _get_device()
    xp, xs = _rows(x, dev, dtype, rows, cols, "x")
    cp, cs = _i8_rows(codes, dev, _INT8, rows, (cols + 63) // 64 * 64, "codes")
    rc = load_library().moe_i8_quantize_rows(MOE_BF16 if dtype is _BF16 else MOE_F32, rows, cols, xp, xs, cp, cs, _at(scale, dev, _F32, rows, "scale"),
                                             _get_stream(dev))
    if rc:
        _check("moe_i8_quantize_rows", rc)


def make_i8_linear(n_rows: int, K: int, N: int, out_dtype, gelu: bool = False) -> MoeI8Linear:
    if isinstance(out_dtype, torch.dtype):
        out_dtype = {torch.float32: MOE_F32, torch.bfloat16: MOE_BF16}[out_dtype]
    elif isinstance(out_dtype, str):
        out_dtype = {"f32": MOE_F32, "bf16": MOE_BF16}[out_dtype]
    return MoeI8Linear(n_rows, K, N, int(out_dtype), int(bool(gelu)))


def moe_i8_linear(product: MoeI8Linear, codes, row_scale, W, col_scale, bias, out) -> None:
    """codes: int8 [n_rows, at least K rounded up to 64]; W, col_scale: as moe_i8_quantize_weights gave them; bias: bf16 or None."""
    rows, K, N = product.n_rows, product.K, product.N
    if rows == 0:
        return
    dev = _get_device()
    cp, cs = _i8_rows(codes, dev, _INT8, rows, (K + 63) // 64 * 64, "codes")
    op, os_ = _rows(out, dev, _F32 if product.out_dtype == MOE_F32 else _BF16, rows, N, "out")
    rc = load_library().moe_i8_linear(ctypes.byref(product), cp, cs, _at(row_scale, dev, _F32, rows, "row_scale"), _at(W, dev, _INT8, _i8_weights_need(1, K, N), "W"),
                                      _at(col_scale, dev, _F32, N, "col_scale"), _at(bias, dev, _BF16, N, "bias"), op, os_, _get_stream(dev))
    if rc:
        _check("moe_i8_linear", rc)


def moe_i8_workspace_bytes(shape: MoeShape) -> int:
    return int(load_library().moe_i8_workspace_bytes(ctypes.byref(shape)))


@functools.lru_cache(maxsize=256)
def _i8_weights_need(G: int, K: int, N: int) -> int:
    return moe_i8_weights_bytes(G, K, N)


@functools.lru_cache(maxsize=256)
def _i8_tensors(shape: bytes, dense: bool):
    """(name, dtype, elements) of a call's weights, the sizes of its other tensors and the bytes of its workspace."""
    s = MoeShape.from_buffer_copy(shape)
    T, d, f, E, k, C = s.T, s.d_model, s.d_ffn, s.E, s.top_k, s.capacity
    f32, i8, bf, up = torch.float32, torch.int8, torch.bfloat16, moe_i8_weights_bytes
    weights = [("W1", i8, up(E, d, f)), ("s1", f32, E * f), ("b1", bf, E * f), ("W2", i8, up(E, f, d)), ("s2", f32, E * d), ("b2", bf, E * d)]
    if dense:
        weights += [("Wd1", i8, up(1, d, f)), ("sd1", f32, f), ("bd1", bf, f), ("Wd2", i8, up(1, f, d)), ("sd2", f32, d), ("bd2", bf, d)]
    return tuple(weights), (T * d, _wg(s) if s.E > 0 and s.d_model > 0 else 0, E, T * E, T * k, E * C, E * C * d), moe_i8_workspace_bytes(s)


def _i8_weights(tensors, weights: dict, device: int) -> MoeI8Weights:
    at = []
    for name, dtype, numel in tensors:
        t = weights.get(name)
        if t is None:
            at.append(None)
            continue
        if t.get_device() != device or t.dtype is not dtype or t.numel() != numel or not t.is_contiguous():
            _refuse(t, dtype, numel, name)
        at.append(t.data_ptr())
    return MoeI8Weights(*at)


def moe_i8_expert_ffn(shape, weights: dict, xe, expert_rows, ye, ws) -> None:
    """`weights`: name -> tensor (or None) for the fields of moe_i8_weights_t."""
    bf, dev = torch.bfloat16, _get_device()
    tensors, sizes, need = _i8_tensors(bytes(shape), False)
    w = _i8_weights(tensors, weights, dev)
    wp, nbytes = _workspace(ws, dev, need)
    rc = load_library().moe_i8_expert_ffn(
        ctypes.byref(shape), ctypes.byref(w), _at(xe, dev, bf, sizes[6], "xe"), _at(expert_rows, dev, torch.int32, shape.E, "expert_rows"),
        _at(ye, dev, bf, sizes[6], "ye"), wp, nbytes, _get_stream(dev))
    _check("moe_i8_expert_ffn", rc)


def moe_i8_layer_forward(shape, weights: dict, x, Wg, bg, out, logits_out, expert_idx_out, slot_idx_out, gate_w_out, expert_rows_out,
                         slot_token_out, ws) -> None:
    """`weights` as in moe_i8_expert_ffn, with the dense branch's for residual layers."""
    bf, i32, f32, dev = torch.bfloat16, torch.int32, torch.float32, _get_device()
    tensors, (n, gate, E, logits, choices, slots, _), need = _i8_tensors(bytes(shape), True)
    w = _i8_weights(tensors, weights, dev)
    wp, nbytes = _workspace(ws, dev, need)
    rc = load_library().moe_i8_layer_forward(
        ctypes.byref(shape), ctypes.byref(w), _at(x, dev, bf, n, "x"), _at(Wg, dev, f32, gate, "Wg"), _at(bg, dev, f32, E, "bg"),
        _at(out, dev, bf, n, "out"), _at(logits_out, dev, f32, logits, "logits_out"), _at(expert_idx_out, dev, i32, choices, "expert_idx_out"),
        _at(slot_idx_out, dev, i32, choices, "slot_idx_out"), _at(gate_w_out, dev, f32, choices, "gate_w_out"),
        _at(expert_rows_out, dev, i32, E, "expert_rows_out"), _at(slot_token_out, dev, i32, slots, "slot_token_out"), wp, nbytes,
        _get_stream(dev))
    if rc:
        _check("moe_i8_layer_forward", rc)


def moe_profile_enable(max_calls: int) -> None:
    _check("moe_profile_enable", load_library().moe_profile_enable(int(max_calls)))


def moe_profile_select(stage_names=None) -> None:
    """Restrict stage timing to the named stages (None = all)."""
    names = moe_profile_stage_names()
    mask = 0xFFFFFFFF if stage_names is None else sum(1 << names.index(n) for n in stage_names)
    _check("moe_profile_select", load_library().moe_profile_select(mask))


def moe_profile_stride(every_nth_call: int) -> None:
    _check("moe_profile_stride", load_library().moe_profile_stride(int(every_nth_call)))


def moe_profile_calls() -> int:
    return int(load_library().moe_profile_calls())


def moe_profile_stage_names() -> list:
    lib = load_library()
    return [lib.moe_profile_stage_name(i).decode() for i in range(lib.moe_profile_stage_count())]


def moe_profile_elapsed(call: int) -> list:
    lib = load_library()
    n = lib.moe_profile_stage_count()
    buf = (ctypes.c_float * n)()
    _check("moe_profile_elapsed", lib.moe_profile_elapsed(int(call), buf))
    return list(buf)
