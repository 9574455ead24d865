"""ctypes binding of the operators around the attention (include/radial_layer.h): same names as the C ABI, argument marshalling only.
Tensors are torch CUDA tensors on the current device (others are refused); every step of the computation runs in the library's HIP kernels.
There is no fallback: a missing library or a failing call raises."""
from __future__ import annotations

import ctypes
import numbers
from ctypes import POINTER, byref, c_double, c_float, c_int32, c_int64, c_size_t, c_void_p

from . import binding
from .binding import RadialError, _check, _load_torch, _stream_ptr, radial_last_error, radial_tensor  # noqa: F401

RADIAL_BF16, RADIAL_F32 = 0, 1
RADIAL_NORM_NONE, RADIAL_NORM_LAYER, RADIAL_NORM_RMS = 0, 1, 2
RADIAL_ROPE_INTERLEAVED, RADIAL_ROPE_HALF = 0, 1
RADIAL_ROPE_SCALE_NONE, RADIAL_ROPE_SCALE_LINEAR, RADIAL_ROPE_SCALE_BASE, RADIAL_ROPE_SCALE_PARTS = 0, 1, 2, 3
RADIAL_GROUPS, RADIAL_BLOCKS = 0, 1

EXPORTS = (
    "radial_norm_fwd", "radial_norm_bwd_workspace", "radial_norm_bwd", "radial_rope_table_bytes", "radial_rope_table", "radial_rope_fwd",
    "radial_rope_bwd", "radial_quantize_groups_fp8", "radial_product_fp8",
)


class radial_rows(ctypes.Structure):
    _fields_ = [("ptr", c_void_p), ("stride_b", c_int64), ("stride_n", c_int64), ("type", c_int32)]


class radial_norm_params(ctypes.Structure):
    _fields_ = [("B", c_int32), ("N", c_int32), ("C", c_int32), ("group", c_int32), ("post", c_int32), ("pre", c_int32),
                ("eps", c_float), ("residual_scale", c_float), ("mod_stride", c_int64), ("dmod_stride", c_int64)]


class radial_rope_params(ctypes.Structure):
    _fields_ = [("axes", c_int32), ("size", c_int32 * 3), ("dims", c_int32 * 3), ("layout", c_int32), ("scaling", c_int32 * 3),
                ("original", c_int32 * 3), ("factor", c_double * 3), ("theta", c_double), ("fast", c_double), ("slow", c_double),
                ("magnitude", c_double)]


_lib = None
_types = None  # torch dtype -> RADIAL_ type
_f32 = _bf16 = _u8 = _i32 = None  # torch dtypes, set by load()
_device = None  # torch.cuda.current_device, set by load()


def load():
    """Loads libradial.so and declares the prototypes of radial_layer.h."""
    global _lib, _types, _f32, _bf16, _u8, _i32, _device
    if _lib is not None:
        return _lib
    lib = binding.load()
    rows, floats, heads = radial_rows, c_void_p, radial_tensor
    lib.radial_norm_fwd.argtypes = [POINTER(radial_norm_params), rows, rows] + [floats] * 5 + [rows, rows, c_void_p]
    lib.radial_norm_bwd_workspace.argtypes = [POINTER(radial_norm_params)]
    lib.radial_norm_bwd_workspace.restype = c_size_t
    lib.radial_norm_bwd.argtypes = [POINTER(radial_norm_params)] + [rows] * 4 + [floats] * 4 + [rows] * 2 + [floats] * 5 + [c_void_p, c_size_t, c_void_p]
    lib.radial_rope_table_bytes.argtypes = [POINTER(radial_rope_params)]
    lib.radial_rope_table_bytes.restype = c_size_t
    lib.radial_rope_table.argtypes = [POINTER(radial_rope_params), c_void_p, c_size_t, c_void_p]
    for fn in (lib.radial_rope_fwd, lib.radial_rope_bwd):
        fn.argtypes = [POINTER(radial_rope_params), c_void_p, c_size_t, c_int32, c_int32, c_int32, c_int32, heads, heads, c_int32, heads, heads, c_int32,
                       c_void_p, c_int32, c_void_p]
    lib.radial_quantize_groups_fp8.argtypes = [c_int32, c_int32, c_void_p, c_int32, c_int64, c_int32] + [c_void_p] * 5
    lib.radial_product_fp8.argtypes = [c_int32, c_int32, c_int32] + [c_void_p] * 4 + [c_int32, c_void_p, c_int64, c_void_p]
    for name in EXPORTS:
        fn = getattr(lib, name)
        if fn.restype is not c_size_t:
            fn.restype = ctypes.c_int
    torch = _load_torch()
    _types = {torch.bfloat16: RADIAL_BF16, torch.float32: RADIAL_F32}
    _f32, _bf16, _u8, _i32 = torch.float32, torch.bfloat16, torch.uint8, torch.int32
    _device = torch.cuda.current_device
    _lib = lib
    return lib


# ---- gated residual and norms ---------------------------------------------------------------

_NO_ROWS = radial_rows(None, 0, 0, RADIAL_BF16)


def _rows(t, name, shape, device) -> radial_rows:
    if t is None:
        return _NO_ROWS
    stride = t.stride()
    kind = _types.get(t.dtype)
    if kind is None or t.get_device() != device or t.shape != shape or (stride[2] != 1 and shape[2] > 1):
        raise ValueError(f"{name} must be a CUDA bf16 or float32 tensor {list(shape)} with unit stride in C")
    return radial_rows(t.data_ptr(), stride[0], stride[1], kind)


def _mods(B, G, C, device, **named):
    """Addresses of the conditioning tensors [B, G, C] that are given, and the elements between their rows: one stride for all of them, across
    batch entries too."""
    shape, found, out = (B, G, C), None, []
    for name, t in named.items():
        if t is None:
            out.append(None)
            continue
        stride = t.stride()
        if t.dtype is not _f32 or t.get_device() != device or t.shape != shape or (stride[2] != 1 and C > 1):
            raise ValueError(f"{name} must be a CUDA float32 tensor {[B, G, C]} with unit stride in C")
        step = stride[1] if G > 1 else stride[0] if B > 1 else C
        if G > 1 and B > 1 and stride[0] != G * step:
            raise ValueError(f"the rows of {name} must be evenly spaced over batch entries and groups")
        if found is not None and step != found:
            raise ValueError(f"{', '.join(n for n, x in named.items() if x is not None)} must have the same strides")
        found = step
        out.append(t.data_ptr())
    out.append(C if found is None else found)
    return out


def _too_large(what):
    raise ValueError(f"{what} must be below 2^31")  # ctypes would keep the low 32 bits


def _bytes(t, name, device):
    if t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous tensor on the current CUDA device")
    return t.data_ptr()


def _group(group, N) -> int:
    """Tokens that share a row of conditioning: all without `group`, and where it is larger."""
    return N if group is None or group > N else max(group, 0)


def _channels(t, name, C, device):
    if t is None:
        return None
    if t.dtype is not _f32 or t.get_device() != device or t.shape != (C,) or (C > 1 and t.stride()[0] != 1):
        raise ValueError(f"{name} must be a contiguous CUDA float32 tensor [C]")
    return t.data_ptr()


def radial_norm_fwd(x, r, z, *, y=None, gate=None, post_weight=None, weight=None, scale=None, shift=None, group=None, post=RADIAL_NORM_NONE,
                    pre=RADIAL_NORM_LAYER, residual_scale: float = 1.0, eps: float = 1e-6, stream=None):
    """r <- residual_scale x + gate N_post(y) post_weight and z <- N_pre(r) weight (1 + scale) + shift.

    x, r: residual stream [B, N, C]; y, z: branch in and out (bf16 or float32); r None without y, z None with pre = RADIAL_NORM_NONE.
    gate, scale, shift: float32 [B, ceil(N/group), C], a row for every `group` tokens (default: one for all); post_weight, weight: float32 [C]."""
    lib = _lib or load()
    shape, device = x.shape, _device()
    B, N, C = shape
    if (B * N | C) >> 31:
        _too_large("B*N and C")
    group = _group(group, N)
    gate, scale, shift, step = _mods(B, -(-N // max(group, 1)), C, device, gate=gate, scale=scale, shift=shift)
    p = radial_norm_params(B, N, C, group, post, pre, eps, residual_scale, step, step)
    _check(lib.radial_norm_fwd(byref(p), _rows(x, "x", shape, device), _rows(y, "y", shape, device), gate, _channels(post_weight, "post_weight", C, device),
                               _channels(weight, "weight", C, device), scale, shift, _rows(r, "r", shape, device), _rows(z, "z", shape, device), _stream_ptr(stream)))


def radial_norm_bwd_workspace(B: int, N: int, C: int, *, group=None, post=RADIAL_NORM_NONE, pre=RADIAL_NORM_LAYER) -> int:
    if (B | N | C) >> 31:
        _too_large("B, N and C")
    p = radial_norm_params(B, N, C, _group(group, N), post, pre, 1e-6, 1.0, C, C)
    return int((_lib or load()).radial_norm_bwd_workspace(byref(p)))


def radial_norm_bwd(r, dz, dx, workspace, *, dr=None, y=None, dy=None, gate=None, post_weight=None, weight=None, scale=None, dgate=None,
                    dscale=None, dshift=None, dpost_weight=None, dweight=None, group=None, post=RADIAL_NORM_NONE, pre=RADIAL_NORM_LAYER,
                    residual_scale: float = 1.0, eps: float = 1e-6, stream=None):
    """dx (and dy) <- gradients of radial_norm_fwd from dz and dr, with those of the conditioning and the weights that are given.

    r: the forward's r (its x without y), not read with pre = RADIAL_NORM_NONE; workspace: CUDA uint8 tensor of radial_norm_bwd_workspace bytes."""
    lib = _lib or load()
    shape, device = dx.shape, _device()
    B, N, C = shape
    if (B * N | C) >> 31:
        _too_large("B*N and C")
    group = _group(group, N)
    G = -(-N // max(group, 1))
    gate, scale, step = _mods(B, G, C, device, gate=gate, scale=scale)
    dgate, dscale, dshift, dstep = _mods(B, G, C, device, dgate=dgate, dscale=dscale, dshift=dshift)
    p = radial_norm_params(B, N, C, group, post, pre, eps, residual_scale, step, dstep)
    _check(lib.radial_norm_bwd(byref(p), _rows(r, "r", shape, device), _rows(y, "y", shape, device), _rows(dz, "dz", shape, device), _rows(dr, "dr", shape, device), gate,
                               _channels(post_weight, "post_weight", C, device), _channels(weight, "weight", C, device), scale, _rows(dx, "dx", shape, device),
                               _rows(dy, "dy", shape, device), dgate, dscale, dshift, _channels(dpost_weight, "dpost_weight", C, device),
                               _channels(dweight, "dweight", C, device), _bytes(workspace, "workspace", device),
                               workspace.numel() * workspace.element_size(),
                               _stream_ptr(stream)))


# ---- rotary positions -------------------------------------------------------------------------

_LAYOUTS = {"interleaved": RADIAL_ROPE_INTERLEAVED, "half": RADIAL_ROPE_HALF}
_SCALINGS = {"none": RADIAL_ROPE_SCALE_NONE, "linear": RADIAL_ROPE_SCALE_LINEAR, "base": RADIAL_ROPE_SCALE_BASE, "parts": RADIAL_ROPE_SCALE_PARTS}


def rope_params(sizes, dims, *, layout="interleaved", scaling="none", factor=1.0, original=0, theta: float = 1e4, fast: float = 32.0,
                slow: float = 1.0, magnitude: float = 1.0) -> radial_rope_params:
    """radial_rope_params for a grid of `sizes` positions whose axes turn `dims` dimensions of a head each.

    layout: "interleaved" or "half"; scaling: "none", "linear", "base" or "parts"; scaling, factor and original may be one value for all
    axes or one for each (only the frames of a longer video are scaled, for instance)."""
    axes = len(sizes)
    if not 1 <= axes <= 3 or len(dims) != axes:
        raise ValueError("sizes and dims need one entry for each of one to three axes")

    def of_axes(v, name):
        v = [v] * axes if isinstance(v, (str, numbers.Real)) else list(v)
        if len(v) != axes:
            raise ValueError(f"{name} needs one value, or one for each axis")
        return v

    p = radial_rope_params(axes=axes, theta=theta, fast=fast, slow=slow, magnitude=magnitude)
    if layout not in _LAYOUTS:
        raise ValueError(f"layout must be one of {', '.join(_LAYOUTS)}")
    p.layout = _LAYOUTS[layout]
    per_axis = zip(sizes, dims, of_axes(scaling, "scaling"), of_axes(factor, "factor"), of_axes(original, "original"))
    for i, (size, dim, how, by, before) in enumerate(per_axis):
        if max(size, dim, before) >> 31:
            _too_large("sizes, dims and original")
        if how not in _SCALINGS:
            raise ValueError(f"scaling must be one of {', '.join(_SCALINGS)}")
        p.size[i], p.dims[i], p.scaling[i], p.factor[i], p.original[i] = size, dim, _SCALINGS[how], by, before
    return p


def radial_rope_table_bytes(params: radial_rope_params) -> int:
    return int((_lib or load()).radial_rope_table_bytes(byref(params)))


def radial_rope_table(params: radial_rope_params, table, stream=None):
    """table (float32, radial_rope_table_bytes(params) bytes) <- the turns of every position."""
    lib = _lib or load()
    _check_table(table, _device())
    _check(lib.radial_rope_table(byref(params), table.data_ptr(), table.numel() * 4, _stream_ptr(stream)))


def _check_table(table, device):
    if table.dtype is not _f32 or table.get_device() != device or not table.is_contiguous():
        raise ValueError("table must be a contiguous CUDA float32 tensor")


_NO_HEADS = radial_tensor(None, 0, 0, 0)


def _heads(t, name, shape, dtype, device) -> radial_tensor:
    stride = t.stride()
    if t.dtype is not dtype or t.get_device() != device or t.shape != shape or stride[3] != 1:
        raise ValueError(f"{name} must be a CUDA tensor {list(shape)} of q's type with unit stride in D")
    return radial_tensor(t.data_ptr(), stride[0], stride[1], stride[2])


def _rope(call, names, params, table, q, q_out, k, k_out, positions, first, stream):
    shape, device = q.shape, _device()
    B, q_heads, N, D = shape
    if (B * N | D | q_heads) >> 31:
        _too_large("B*N, D and the heads")
    dtype = q.dtype
    kind = _types.get(dtype)
    if kind is None:
        raise ValueError(f"{names[0]} must be bf16 or float32")
    k_heads, k_in, k_to = 0, _NO_HEADS, _NO_HEADS
    if k is not None or k_out is not None:
        if k is None or k_out is None:
            raise ValueError(f"{names[2]} and {names[3]} go together")
        k_shape = k.shape
        k_heads = k_shape[1]
        if k_heads >> 31:
            _too_large("the heads")
        if k_shape != shape and k_shape != (B, k_heads, N, D):
            raise ValueError(f"{names[2]} must have {names[0]}'s shape but for the heads")
        k_in, k_to = _heads(k, names[2], k_shape, dtype, device), _heads(k_out, names[3], k_shape, dtype, device)
    at = None
    if positions is not None:
        if positions.dtype is not _i32 or positions.get_device() != device or not positions.is_contiguous() or positions.shape != (B, N):
            raise ValueError("positions must be a contiguous CUDA int32 tensor [B, N]")
        at = positions.data_ptr()
    elif first >= 1 << 31 or first < -1:
        raise ValueError("first must be below 2^31 and not negative")
    _check_table(table, device)
    _check(call(byref(params), table.data_ptr(), table.numel() * 4, B, N, D, q_heads, _heads(q, names[0], shape, dtype, device),
                _heads(q_out, names[1], shape, dtype, device), k_heads, k_in, k_to, kind, at, first, _stream_ptr(stream)))


def radial_rope_fwd(params: radial_rope_params, table, q, q_out, k=None, k_out=None, positions=None, first: int = 0, stream=None):
    """q_out, k_out <- q [B, H, N, D] and k [B, Hk, N, D] (bf16 or float32) turned to their tokens' positions on the grid.

    positions: int32 [B, N], index of each token on the grid (outside of it: copied as it is); default: first, first + 1, ..."""
    _rope((_lib or load()).radial_rope_fwd, ("q", "q_out", "k", "k_out"), params, table, q, q_out, k, k_out, positions, first, stream)


def radial_rope_bwd(params: radial_rope_params, table, dq_out, dq, dk_out=None, dk=None, positions=None, first: int = 0, stream=None):
    """dq, dk <- gradients of radial_rope_fwd's inputs from those of its outputs."""
    _rope((_lib or load()).radial_rope_bwd, ("dq_out", "dq", "dk_out", "dk"), params, table, dq_out, dq, dk_out, dk, positions, first, stream)


# ---- products in 8-bit floating point -----------------------------------------------------------

def _codes(codes, scales, name, rows, cols, scale_rows, device):
    if codes is None and scales is None:
        return None, None
    groups = -(-cols // 128)
    if codes is None or codes.dtype is not _u8 or codes.get_device() != device or not codes.is_contiguous() or codes.shape != (rows, groups * 128):
        raise ValueError(f"{name}codes must be a contiguous CUDA uint8 tensor {[rows, groups * 128]}")
    if scales is None or scales.dtype is not _f32 or scales.get_device() != device or not scales.is_contiguous() or scales.shape != (groups, scale_rows):
        raise ValueError(f"{name}scales must be a contiguous CUDA float32 tensor {[groups, scale_rows]}")
    return codes.data_ptr(), scales.data_ptr()


def radial_quantize_groups_fp8(x, codes=None, scales=None, codes_t=None, scales_t=None, grouping=RADIAL_GROUPS, stream=None):
    """E4M3 codes (uint8) and scales (float32) of x [rows, cols] (bf16 or float32) and, or, of its transpose.

    codes [rows, P], scales [P/128, rows] with P = cols rounded up to 128; codes_t [cols, Pt], scales_t [Pt/128, cols] likewise with rows.
    grouping = RADIAL_BLOCKS: one scale for 128 x 128, scales [P/128, ceil(rows/128)] and scales_t [Pt/128, ceil(cols/128)]."""
    lib = _lib or load()
    kind, shape, stride, device = _types.get(x.dtype), x.shape, x.stride(), _device()
    if kind is None or x.get_device() != device or len(shape) != 2 or (stride[1] != 1 and shape[1] > 1):
        raise ValueError("x must be a CUDA bf16 or float32 tensor [rows, cols] with unit stride in cols")
    rows, cols = shape
    if (rows | cols) >> 31:
        _too_large("rows and cols")
    blocks = grouping == RADIAL_BLOCKS
    c, s = _codes(codes, scales, "", rows, cols, -(-rows // 128) if blocks else rows, device)
    ct, st = _codes(codes_t, scales_t, "transposed ", cols, rows, -(-cols // 128) if blocks else cols, device)
    step = stride[0] if rows > 1 else max(cols, stride[0])
    _check(lib.radial_quantize_groups_fp8(rows, cols, x.data_ptr(), kind, step, grouping, c, s, ct, st, _stream_ptr(stream)))


def radial_product_fp8(a_codes, a_scales, b_codes, b_scales, out, stream=None):
    """out [M, N] (bf16) <- A B^T from the codes and scales of A [M, K] (groups) and B [N, K] (groups or blocks, by b_scales' shape)."""
    lib = _lib or load()
    shape, stride, device = out.shape, out.stride(), _device()
    if out.dtype is not _bf16 or out.get_device() != device or len(shape) != 2 or (stride[1] != 1 and shape[1] > 1):
        raise ValueError("out must be a CUDA bf16 tensor [M, N] with unit stride in N")
    M, N = shape
    K = a_codes.shape[-1]
    if (M | N | K) >> 31:
        _too_large("M, N and K")
    a, sa = _codes(a_codes, a_scales, "a_", M, K, M, device)
    blocks = b_scales.shape[-1] != N
    b, sb = _codes(b_codes, b_scales, "b_", N, K, -(-N // 128) if blocks else N, device)
    step = stride[0] if M > 1 else max(N, stride[0])
    _check(lib.radial_product_fp8(M, N, K, a, sa, b, sb, RADIAL_BLOCKS if blocks else RADIAL_GROUPS, out.data_ptr(), step, _stream_ptr(stream)))
