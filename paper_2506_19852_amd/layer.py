"""ctypes binding of the operators around the attention (include/radial_layer.h): same names as the C ABI, argument marshalling only.
Tensors are torch CUDA tensors on the current device (others are refused); every step of the computation runs in the library's HIP kernels.
There is no fallback: a missing library or a failing call raises."""
from __future__ import annotations

import ctypes
import numbers
import operator
from ctypes import POINTER, byref, c_double, c_float, c_int32, c_int64, c_size_t, c_uint64, c_void_p

from . import binding
from .binding import RadialError, _check, _load_torch, _stream_ptr, radial_last_error, radial_tensor  # noqa: F401

RADIAL_BF16, RADIAL_F32 = 0, 1
RADIAL_NORM_NONE, RADIAL_NORM_LAYER, RADIAL_NORM_RMS = 0, 1, 2
RADIAL_ROPE_INTERLEAVED, RADIAL_ROPE_HALF = 0, 1
RADIAL_ROPE_SCALE_NONE, RADIAL_ROPE_SCALE_LINEAR, RADIAL_ROPE_SCALE_BASE, RADIAL_ROPE_SCALE_PARTS = 0, 1, 2, 3
RADIAL_GROUPS, RADIAL_BLOCKS = 0, 1
RADIAL_ROUND_NEAREST, RADIAL_ROUND_RANDOM = 0, 1

EXPORTS = (
    "radial_norm_fwd", "radial_norm_bwd_workspace", "radial_norm_bwd", "radial_rope_table_bytes", "radial_rope_table", "radial_rope_fwd",
    "radial_rope_bwd", "radial_quantize_groups_fp8", "radial_product_fp8", "radial_quantize_rows_i8_workspace", "radial_quantize_rows_i8",
    "radial_product_i8", "radial_linear_i8_fwd_workspace", "radial_linear_i8_fwd", "radial_linear_i8_bwd_workspace", "radial_linear_i8_bwd",
    "radial_adamw_plan", "radial_adamw_table", "radial_grad_norm_workspace", "radial_grad_norm", "radial_adamw_step",
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


class radial_adamw_tensor(ctypes.Structure):
    _fields_ = [("weight", c_void_p), ("copy", c_void_p), ("grad", c_void_p), ("first", c_void_p), ("second", c_void_p), ("first_scales", c_void_p),
                ("second_scales", c_void_p), ("n", c_int64), ("weight_type", c_int32), ("grad_type", c_int32), ("decay", c_double)]


class radial_adamw_plan_info(ctypes.Structure):
    _fields_ = [("count", c_int32), ("pieces", c_int32), ("table_bytes", c_size_t)]


class radial_adamw_params(ctypes.Structure):
    _fields_ = [("lr", c_double), ("beta1", c_double), ("beta2", c_double), ("eps", c_double), ("step", c_int64), ("seed", c_uint64),
                ("rounding", c_int32), ("factor", c_void_p), ("lr_at", c_void_p), ("step_at", c_void_p)]


_lib = None
_types = None  # torch dtype -> RADIAL_ type
_f32 = _bf16 = _u8 = _i8 = _i32 = _i64 = None  # torch dtypes, set by load()
_device = None  # torch.cuda.current_device, set by load()


def load():
    """Loads libradial.so and declares the prototypes of radial_layer.h."""
    global _lib, _types, _f32, _bf16, _u8, _i8, _i32, _i64, _device
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
    sizes3, address, plan = [c_int32] * 3, c_void_p, POINTER(radial_adamw_plan_info)
    lib.radial_quantize_rows_i8_workspace.argtypes = [c_int32, c_int32]
    lib.radial_quantize_rows_i8.argtypes = [c_int32, c_int32, address, c_int32, c_int64] + [address] * 5 + [c_int32, address, c_size_t, address]
    lib.radial_product_i8.argtypes = sizes3 + [address] * 6 + [c_int32, c_int64, c_int32, address]
    lib.radial_linear_i8_fwd_workspace.argtypes = lib.radial_linear_i8_bwd_workspace.argtypes = sizes3
    lib.radial_linear_i8_fwd.argtypes = sizes3 + [address, c_int32, c_int64] + [address] * 4 + [c_int32, c_int64, address, c_size_t, address]
    lib.radial_linear_i8_bwd.argtypes = sizes3 + [address, c_int32, c_int64, address, c_int64, address, address, address, c_int32, c_int64, address, c_int32, c_int64,
                                                  address, c_int32, address, c_size_t, address]
    lib.radial_adamw_plan.argtypes = [POINTER(radial_adamw_tensor), c_int32, plan]
    lib.radial_adamw_table.argtypes = [POINTER(radial_adamw_tensor), plan, address, c_size_t, address]
    lib.radial_grad_norm_workspace.argtypes = [plan]
    lib.radial_grad_norm.argtypes = [plan, address, c_size_t, c_float, c_float, address, address, c_size_t, address]
    lib.radial_adamw_step.argtypes = [POINTER(radial_adamw_params), plan, address, c_size_t, address]
    for name in ("radial_quantize_rows_i8", "radial_linear_i8_fwd", "radial_linear_i8_bwd", "radial_grad_norm"):
        getattr(lib, name + "_workspace").restype = c_size_t
    for name in EXPORTS:
        fn = getattr(lib, name)
        if fn.restype is not c_size_t:
            fn.restype = ctypes.c_int
    torch = _load_torch()
    _types = {torch.bfloat16: RADIAL_BF16, torch.float32: RADIAL_F32}
    _f32, _bf16, _u8, _i8, _i32, _i64 = torch.float32, torch.bfloat16, torch.uint8, torch.int8, torch.int32, torch.int64
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


# ---- products in 8-bit integers -------------------------------------------------------------------

def _matrix(t, name, device, shape=None):
    """(address, type, elements from row to row) of a matrix."""
    kind, found, stride = _types.get(t.dtype), t.shape, t.stride()
    if kind is None or t.get_device() != device or len(found) != 2 or (shape is not None and found != shape) or (stride[1] != 1 and found[1] > 1):
        raise ValueError(f"{name} must be a CUDA bf16 or float32 tensor {'[rows, columns]' if shape is None else list(shape)} with unit stride in its rows")
    return t.data_ptr(), kind, stride[0] if found[0] > 1 else max(found[1], stride[0])


def _row_codes(codes, scales, name, rows, cols, device):
    if codes is None and scales is None:
        return None, None
    padded = -(-cols // 128) * 128
    if codes is None or codes.dtype is not _i8 or codes.get_device() != device or not codes.is_contiguous() or codes.shape != (rows, padded):
        raise ValueError(f"{name}codes must be a contiguous CUDA int8 tensor {[rows, padded]}")
    if scales is None:
        raise ValueError(f"{name}scales must be a contiguous CUDA float32 tensor {[rows]}")
    return codes.data_ptr(), _vector(scales, name + "scales", rows, device)


def _vector(t, name, length, device):
    if t is None:
        return None
    if t.dtype is not _f32 or t.get_device() != device or t.shape != (length,) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous CUDA float32 tensor {[length]}")
    return t.data_ptr()


def _sized(workspace, device):
    if workspace is None:
        return None, 0
    return _bytes(workspace, "workspace", device), workspace.numel() * workspace.element_size()


def radial_quantize_rows_i8_workspace(rows: int, cols: int) -> int:
    if (rows | cols) >> 31:
        _too_large("rows and cols")
    return int((_lib or load()).radial_quantize_rows_i8_workspace(rows, cols))


def radial_quantize_rows_i8(x, codes=None, scales=None, codes_t=None, scales_t=None, workspace=None, *, sums_t=None, accumulate: bool = False, stream=None):
    """Codes (int8) and scales (float32) of the rows of x [rows, cols] (bf16 or float32) and, or, of those of its transpose; sums_t [cols] <- its column sums.

    codes [rows, P], scales [rows] with P = cols rounded up to 128; codes_t [cols, Pt], scales_t [cols] likewise with rows.  workspace: CUDA uint8 tensor of
    radial_quantize_rows_i8_workspace bytes, needed for codes_t and sums_t; accumulate: sums_t is added to."""
    lib = _lib or load()
    device = _device()
    at, kind, step = _matrix(x, "x", device)
    rows, cols = x.shape
    if (rows | cols) >> 31:
        _too_large("rows and cols")
    c, s = _row_codes(codes, scales, "", rows, cols, device)
    ct, st = _row_codes(codes_t, scales_t, "transposed ", cols, rows, device)
    _check(lib.radial_quantize_rows_i8(rows, cols, at, kind, step, c, s, ct, st, _vector(sums_t, "sums_t", cols, device), bool(accumulate),
                                       *_sized(workspace, device), _stream_ptr(stream)))


def radial_product_i8(a_codes, a_scales, b_codes, b_scales, out, *, bias=None, accumulate: bool = False, stream=None):
    """out [M, N] (bf16 or float32) <- A B^T + bias from the codes and scales of A [M, K] and B [N, K]; accumulate: float32 out is added to."""
    lib = _lib or load()
    device = _device()
    at, kind, step = _matrix(out, "out", device)
    M, N = out.shape
    K = a_codes.shape[-1]
    if (M | N | K) >> 31:
        _too_large("M, N and K")
    a, sa = _row_codes(a_codes, a_scales, "a_", M, K, device)
    b, sb = _row_codes(b_codes, b_scales, "b_", N, K, device)
    _check(lib.radial_product_i8(M, N, K, a, sa, b, sb, _vector(bias, "bias", N, device), at, kind, step, bool(accumulate), _stream_ptr(stream)))


def _linear_workspace(call, M, N, K):
    if (M | N | K) >> 31:
        _too_large("M, N and K")
    return int(call(M, N, K))


def radial_linear_i8_fwd_workspace(M: int, N: int, K: int) -> int:
    return _linear_workspace((_lib or load()).radial_linear_i8_fwd_workspace, M, N, K)


def radial_linear_i8_bwd_workspace(M: int, N: int, K: int) -> int:
    return _linear_workspace((_lib or load()).radial_linear_i8_bwd_workspace, M, N, K)


def radial_linear_i8_fwd(x, w_codes, w_scales, y, workspace, *, bias=None, stream=None):
    """y [M, N] <- x W^T + bias: x [M, K] is quantised by rows and multiplied with the codes [N, P] and scales [N] of W.

    x, y: bf16 or float32; bias: float32 [N]; workspace: CUDA uint8 tensor of radial_linear_i8_fwd_workspace(M, N, K) bytes."""
    lib = _lib or load()
    device = _device()
    at, kind, step = _matrix(x, "x", device)
    M, K = x.shape
    N = y.shape[-1]
    if (M | N | K) >> 31:
        _too_large("M, N and K")
    to, y_kind, y_step = _matrix(y, "y", device, (M, N))
    w, sw = _row_codes(w_codes, w_scales, "w_", N, K, device)
    _check(lib.radial_linear_i8_fwd(M, N, K, at, kind, step, w, sw, _vector(bias, "bias", N, device), to, y_kind, y_step, *_sized(workspace, device),
                                    _stream_ptr(stream)))


def radial_linear_i8_bwd(dy, workspace, *, x=None, wt_codes=None, wt_scales=None, dx=None, dw=None, dbias=None, accumulate: bool = False, stream=None):
    """Gradients of radial_linear_i8_fwd from dy [M, N]: dx [M, K] <- dy W, dw [N, K] <- dy^T x, dbias [N] <- column sums of dy, those that are given.

    wt_codes [K, Pn], wt_scales [K]: of W transposed, for dx; x: the forward's, of dy's type, for dw; accumulate: dw (then float32) and dbias are added to;
    workspace: CUDA uint8 tensor of radial_linear_i8_bwd_workspace(M, N, K) bytes."""
    lib = _lib or load()
    device = _device()
    at, kind, step = _matrix(dy, "dy", device)
    M, N = dy.shape
    K = dx.shape[-1] if dx is not None else dw.shape[-1] if dw is not None else 1
    if (M | N | K) >> 31:
        _too_large("M, N and K")
    x_at = wt = swt = dx_at = dw_at = None
    x_step = dx_kind = dx_step = dw_kind = dw_step = 0
    if dx is not None:
        dx_at, dx_kind, dx_step = _matrix(dx, "dx", device, (M, K))
        wt, swt = _row_codes(wt_codes, wt_scales, "wt_", K, N, device)
    if dw is not None:
        if x is None:
            raise ValueError("dw needs x")
        x_at, x_kind, x_step = _matrix(x, "x", device, (M, K))
        if x_kind != kind:
            raise ValueError("x must be of dy's type")
        dw_at, dw_kind, dw_step = _matrix(dw, "dw", device, (N, K))
    _check(lib.radial_linear_i8_bwd(M, N, K, at, kind, step, x_at, x_step, wt, swt, dx_at, dx_kind, dx_step, dw_at, dw_kind, dw_step,
                                    _vector(dbias, "dbias", N, device), bool(accumulate), *_sized(workspace, device), _stream_ptr(stream)))


# ---- AdamW over many tensors ------------------------------------------------------------------------

_ROUNDINGS = {"nearest": RADIAL_ROUND_NEAREST, "random": RADIAL_ROUND_RANDOM}


def adamw_tensors(weights, grads, firsts, seconds, *, first_scales=None, second_scales=None, copies=None, decay=0.0):
    """The array of radial_adamw_tensor that radial_adamw_plan and radial_adamw_table take, from lists of contiguous CUDA tensors.

    weights, grads: bf16 or float32; firsts, seconds: float32 states, or uint8 codes with float32 first_scales and second_scales [ceil(n/128)]; copies:
    bf16, each gets its weight rounded (an entry may be None); decay: one number, or one for each tensor.  Nothing that a step writes may overlap another tensor.
    The array and the table made of it hold addresses: the caller keeps the tensors, and makes both again when one moves (gradients that are freed after each step do)."""
    _lib or load()
    device, count = _device(), len(weights)

    def of_tensors(v, name):
        v = [v] * count if v is None or isinstance(v, numbers.Real) else list(v)
        if len(v) != count:
            raise ValueError(f"{name} needs one entry for each of the weights")
        return v

    out = (radial_adamw_tensor * count)()
    spans = []   # (first byte, last byte, written, what) of all parts

    def part(t, what, n, types, written=True):
        if t is None or t.dtype not in types or t.get_device() != device or not t.is_contiguous() or t.numel() != n:
            raise ValueError(f"{what} must be a contiguous CUDA tensor of {n} values of {' or '.join(str(x) for x in types)}")
        at = t.data_ptr()
        if n:
            spans.append((at, at + n * t.element_size(), written, what))
        return at

    lists = [of_tensors(v, name) for v, name in ((grads, "grads"), (firsts, "firsts"), (seconds, "seconds"), (first_scales, "first_scales"),
                                                 (second_scales, "second_scales"), (copies, "copies"), (decay, "decay"))]
    for i, (w, g, m, v, ms, vs, copy, by) in enumerate(zip(weights, *lists)):
        n = w.numel() if w is not None else 0   # refused below
        e = out[i]
        e.n, e.weight_type, e.grad_type, e.decay = n, _types.get(getattr(w, "dtype", None), -1), _types.get(getattr(g, "dtype", None), -1), by
        e.weight = part(w, f"weight {i}", n, (_bf16, _f32))
        e.grad = part(g, f"gradient {i}", n, (_bf16, _f32), False)
        coded = ms is not None or vs is not None
        states = (_u8,) if coded else (_f32,)
        e.first, e.second = part(m, f"first state {i}", n, states), part(v, f"second state {i}", n, states)
        if coded:
            blocks = -(-n // 128)
            e.first_scales, e.second_scales = part(ms, f"first scales {i}", blocks, (_f32,)), part(vs, f"second scales {i}", blocks, (_f32,))
        if copy is not None:
            e.copy = part(copy, f"copy {i}", n, (_bf16,))
    end = written_end = 0   # of what begins before
    last = last_written = None
    for first, behind, written, what in sorted(spans, key=lambda span: span[:2]):
        if first < written_end or (written and first < end):
            raise ValueError(f"{what} overlaps {last_written if first < written_end else last}")
        if behind > end:
            end, last = behind, what
        if written and behind > written_end:
            written_end, last_written = behind, what
    return out


def radial_adamw_plan(tensors) -> radial_adamw_plan_info:
    """How many tensors, their pieces, and the bytes of their table."""
    plan = radial_adamw_plan_info()
    _check((_lib or load()).radial_adamw_plan(tensors, len(tensors), byref(plan)))
    return plan


def radial_adamw_table(tensors, plan: radial_adamw_plan_info, table, stream=None):
    """table (CUDA uint8 tensor of plan.table_bytes) <- the tensors' addresses and pieces, read by radial_grad_norm and radial_adamw_step."""
    lib = _lib or load()
    if len(tensors) != plan.count:
        raise ValueError("plan is not that of the tensors")
    _check(lib.radial_adamw_table(tensors, byref(plan), _bytes(table, "table", _device()), table.numel() * table.element_size(), _stream_ptr(stream)))


def radial_grad_norm_workspace(plan: radial_adamw_plan_info) -> int:
    return int((_lib or load()).radial_grad_norm_workspace(byref(plan)))


def radial_grad_norm(plan: radial_adamw_plan_info, table, norm, workspace, *, scale: float = 1.0, max_norm: float = float("inf"), stream=None):
    """norm (float32 [2]) <- scale |all gradients|, and the factor scale min(1, max_norm / norm[0]) that a step takes (NaN if a gradient is not finite).

    workspace: CUDA uint8 tensor of radial_grad_norm_workspace(plan) bytes."""
    lib = _lib or load()
    device = _device()
    _check(lib.radial_grad_norm(byref(plan), _bytes(table, "table", device), table.numel() * table.element_size(), scale, max_norm,
                                _vector(norm, "norm", 2, device), *_sized(workspace, device), _stream_ptr(stream)))


def _one(t, name, dtype, device):
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != device or t.numel() != 1:
        raise ValueError(f"{name} must be a CUDA {dtype} tensor of one value")
    return t.data_ptr()


def radial_adamw_step(plan: radial_adamw_plan_info, table, *, lr: float | None = None, step: int = 0, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                      factor=None, lr_at=None, step_at=None, rounding="nearest", seed: int = 0, stream=None):
    """One AdamW step over the table's tensors, in place.

    step: 1, 2, ..., or step_at, a CUDA int64 tensor of one value that is read when the step runs; lr, or lr_at (float32) likewise (one of them is needed); factor: radial_grad_norm's norm
    (float32 [2], of which the second value multiplies the gradients; while it is not finite nothing is changed); rounding: "nearest" or "random" (by seed and
    step), of states in 8 bits."""
    lib = _lib or load()
    device = _device()
    if rounding not in _ROUNDINGS:
        raise ValueError(f"rounding must be one of {', '.join(_ROUNDINGS)}")
    if lr is None:
        if lr_at is None:
            raise ValueError("lr or lr_at must be given")
        lr = 0.0
    seed, step = operator.index(seed), operator.index(step)
    if not 0 <= seed < 1 << 64 or step >> 63:
        raise ValueError("seed must be below 2^64 and step below 2^63, neither negative")
    by = _vector(factor, "factor", 2, device)
    p = radial_adamw_params(lr, beta1, beta2, eps, step, seed, _ROUNDINGS[rounding], by + 4 if by is not None else None, _one(lr_at, "lr_at", _f32, device),
                            _one(step_at, "step_at", _i64, device))
    _check(lib.radial_adamw_step(byref(p), byref(plan), _bytes(table, "table", device), table.numel() * table.element_size(), _stream_ptr(stream)))
