"""The operators of a tuning step on 8-bit integer products in numpy, from their definitions: codes of whole numbers with a scale for each row, AdamW with
states in 32 bits or in E4M3 codes.  Imports nothing from the product package."""
from __future__ import annotations

import numpy as np

from oracle import layer as ol

F32 = np.float32
BLOCK = 128


# ---- whole numbers ------------------------------------------------------------------------------

def quantize_rows(x):
    """(codes int8 [rows, P], scales float32 [rows]) of a float32 matrix."""
    rows, cols = x.shape
    a = np.abs(np.asarray(x, F32))
    fine = np.isfinite(a).all(1)
    amax = np.where(fine, np.where(np.isfinite(a), a, 0).max(1), 0).astype(F32)
    scale = np.maximum(amax / F32(127.0), F32(2.0 ** -126))
    assert scale.dtype == F32
    codes = np.zeros((rows, -(-cols // 128) * 128), np.int8)
    with np.errstate(invalid="ignore", over="ignore"):
        q = np.where(fine[:, None], np.asarray(x, F32) / scale[:, None], F32(0))
    codes[:, :cols] = np.rint(q).astype(np.int8)
    return codes, np.where(fine, scale, F32(np.nan))


def product(a, sa, b, sb, bias=None):
    """(A B^T + bias, size of what is scaled) from codes and scales, in float64 (whole numbers below 2^53 are exact)."""
    y = (a.astype(np.float64) @ b.astype(np.float64).T) * (sa.astype(np.float64)[:, None] * sb.astype(np.float64)[None])
    return y + (0.0 if bias is None else np.asarray(bias, np.float64)), np.abs(y)


# ---- AdamW --------------------------------------------------------------------------------------

def mixed(x):
    x = np.asarray(x, np.uint64) & np.uint64(0xFFFFFFFF)
    x = x ^ (x >> np.uint64(16))
    x = x * np.uint64(0x9E3779B1) & np.uint64(0xFFFFFFFF)
    x = x ^ (x >> np.uint64(15))
    x = x * np.uint64(0x6A09E667) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def random_bits(seed, step, tensor, n, first=0):
    """(bits of the first, of the second state) of n values of a tensor from `first` on, all on one side of each multiple of 2^32."""
    key = np.uint64(0)
    for word in (seed & 0xFFFFFFFF, seed >> 32, step & 0xFFFFFFFF, tensor) + ((first >> 32,) if first >> 32 else ()):
        key = mixed(key ^ np.uint64(word))
    h = mixed(key ^ (np.arange(n, dtype=np.uint64) + np.uint64(first & 0xFFFFFFFF)))
    return (h & np.uint64(0xFFFF)).astype(np.int64), (h >> np.uint64(16)).astype(np.int64)


def _blocks(v, fill=0):
    n = len(v)
    out = np.full((-(-n // BLOCK), BLOCK), fill, v.dtype)
    out.reshape(-1)[:n] = v
    return out


def encode(v, bits=None, positive=False):
    """(codes uint8 [n], scales float32 [blocks]) of float32 values, as float32 arithmetic gives them."""
    n = len(v)
    b = _blocks(np.asarray(v, F32))
    amax = np.where(np.isnan(b), 0, np.abs(b)).max(1).astype(F32)
    amax = np.where(amax < F32(2.0 ** -100), F32(0), amax)
    scale = (amax / F32(448)).astype(F32)
    with np.errstate(divide="ignore", invalid="ignore"):
        inverse = np.where(amax > 0, F32(448) / amax, F32(0)).astype(F32)
        y = (b * inverse[:, None]).astype(F32).reshape(-1)[:n]
    if bits is None:
        codes = ol.e4m3_codes(y)
    else:
        a = np.abs(y).astype(np.float64)
        step = np.exp2(np.maximum(np.frexp(a)[1] - 1, -6) - 3.0)
        below = np.minimum(np.floor(np.where(np.isnan(a), 0, a) / step + bits / 65536.0) * step, 448.0)
        codes = np.where(np.isnan(y), 0x7f, ol.e4m3_codes(below) | np.where(np.signbit(y), 128, 0)).astype(np.uint8)
    if positive:
        codes = np.where((y > 0) & (codes == 0), 1, codes).astype(np.uint8)
    return codes, scale


def decode(codes, scales, dtype=np.float64):
    return (ol.e4m3_values()[codes].astype(dtype) * np.repeat(scales.astype(dtype), BLOCK)[:len(codes)]).astype(dtype)


def moments(g, m, v, beta1, beta2):
    """(m, v) after a gradient; in the precision of the arrays."""
    t = g.dtype.type
    return m * t(beta1) + g * t(1.0 - beta1), v * t(beta2) + (g * g) * t(1.0 - beta2)


def update(w, m, v, lr, step, beta1, beta2, eps, decay):
    """The weights in float64, from the moments after the gradient."""
    m_hat, v_hat = m / (1.0 - beta1 ** step), v / (1.0 - beta2 ** step)
    return w * (1.0 - lr * decay) - lr * m_hat / (np.sqrt(v_hat) + eps)
