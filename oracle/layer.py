"""The operators of a transformer layer around the attention in float64 numpy, from their definitions: gated residual and norms with their
gradients, rotary positions, 8-bit codes with a scale for each 128 values.  Imports nothing from the product package."""
from __future__ import annotations

import math

import numpy as np

NONE, LAYER, RMS = 0, 1, 2


def norm(v, kind, eps):
    """(N(v), 1 / size) over the last axis."""
    if kind == NONE:
        return v, None
    mean = v.mean(-1, keepdims=True) if kind == LAYER else 0.0
    inverse = 1.0 / np.sqrt(((v - mean) ** 2).mean(-1, keepdims=True) + eps)
    return (v - mean) * inverse, inverse


def per_token(mod, N, group, missing):
    """Row n // group of mod [B, G, C] for each token n."""
    return missing if mod is None else np.asarray(mod, np.float64)[:, np.arange(N) // group]


def norm_fwd(x, y=None, gate=None, post_weight=None, weight=None, scale=None, shift=None, group=1, post=NONE, pre=LAYER, residual_scale=1.0, eps=1e-6):
    """(r, z); z None without a norm."""
    N = x.shape[1]
    r = x
    if y is not None:
        u, _ = norm(y, post, eps)
        r = residual_scale * x + per_token(gate, N, group, 1.0) * u * (1.0 if post_weight is None else post_weight)
    if pre == NONE:
        return r, None
    n, _ = norm(r, pre, eps)
    return r, n * (1.0 if weight is None else weight) * (1.0 + per_token(scale, N, group, 0.0)) + per_token(shift, N, group, 0.0)


def _through_norm(d, n, inverse, kind):
    if kind == NONE:
        return d
    flat = d.mean(-1, keepdims=True) if kind == LAYER else 0.0
    return inverse * (d - flat - n * (d * n).mean(-1, keepdims=True))


def _over_groups(v, group):
    N = v.shape[1]
    return np.stack([v[:, at:at + group].sum(1) for at in range(0, N, group)], 1)


def norm_bwd(r, dz=None, dr=None, y=None, gate=None, post_weight=None, weight=None, scale=None, group=1, post=NONE, pre=LAYER, residual_scale=1.0,
             eps=1e-6):
    """dict of dx, dy, dgate, dscale, dshift, dpost_weight, dweight (those that there are)."""
    some = dr if dr is not None else dz
    N, C = some.shape[1], some.shape[2]
    w, wp = (np.ones(C) if v is None else np.asarray(v, np.float64) for v in (weight, post_weight))
    s, g = per_token(scale, N, group, 0.0), per_token(gate, N, group, 1.0)
    out = {}
    D = np.zeros_like(some) if dr is None else dr
    if pre != NONE:
        n, inverse = norm(r, pre, eps)
        D = D + _through_norm(dz * w * (1.0 + s), n, inverse, pre)
        along = _over_groups(dz * n, group)
        out["dscale"], out["dshift"] = along * w, _over_groups(dz, group)
        out["dweight"] = (dz * n * (1.0 + s)).sum((0, 1))
    out["dx"] = residual_scale * D
    if y is not None:
        m, inverse = norm(y, post, eps)
        out["dgate"] = _over_groups(D * m * wp, group)
        out["dpost_weight"] = (D * m * g).sum((0, 1))
        out["dy"] = _through_norm(D * g * wp, m, inverse, post)
    return out


# ---- rotary positions ---------------------------------------------------------------------------

def frequencies(dims, theta=1e4, scaling="none", factor=1.0, original=0, fast=32.0, slow=1.0):
    out = []
    if scaling == "base" and dims > 2:
        theta = theta * factor ** (dims / (dims - 2))
    for j in range(dims // 2):
        f = theta ** (-2.0 * j / dims)
        if scaling == "linear":
            f /= factor
        elif scaling == "parts":
            keep = min(1.0, max(0.0, (original * f / (2 * math.pi) - slow) / (fast - slow)))
            f = f * keep + f * (1.0 - keep) / factor
        out.append(f)
    return np.array(out)


def rope_table(sizes, freqs, magnitude=1.0):
    """[turns, 2]: cos and sin of every position of every axis, axis after axis."""
    angles = np.concatenate([(np.arange(n, dtype=np.float64)[:, None] * f[None]).ravel() for n, f in zip(sizes, freqs)])
    return magnitude * np.stack([np.cos(angles), np.sin(angles)], -1)


def rope(x, index, sizes, freqs, layout, magnitude=1.0, gradient=False):
    """x [B, H, N, D] turned to grid index `index` [B, N] (outside of the grid: as it is)."""
    total = math.prod(sizes)
    on = (index >= 0) & (index < total)
    at, angles = np.where(on, index, 0), []
    for size, f in zip(reversed(sizes), reversed(freqs)):
        angles.insert(0, (at % size).astype(np.float64)[..., None] * f)
        at = at // size
    angle = np.concatenate(angles, -1)
    c = np.where(on[..., None], magnitude * np.cos(angle), 1.0)[:, None]
    s = np.where(on[..., None], magnitude * np.sin(angle), 0.0)[:, None] * (-1.0 if gradient else 1.0)
    pairs = angle.shape[-1]
    one = np.arange(pairs) * 2 if layout == "interleaved" else np.arange(pairs)
    two = one + 1 if layout == "interleaved" else one + pairs
    out = np.array(x, np.float64)
    u, v = out[..., one].copy(), out[..., two].copy()
    out[..., one], out[..., two] = u * c - v * s, u * s + v * c
    return out


# ---- 8-bit codes --------------------------------------------------------------------------------

def e4m3_values():
    """Value of each of the 256 codes (NaN for 0x7f and 0xff)."""
    code = np.arange(256)
    e, m = code >> 3 & 15, code & 7
    v = np.where(e > 0, np.ldexp(1.0 + m / 8.0, e - 7), np.ldexp(m / 8.0, -6)) * np.where(code & 128, -1.0, 1.0)
    v[[0x7f, 0xff]] = np.nan
    return v


def e4m3_codes(q):
    """Codes of float32 values of at most 448 and a little, ties to the even code."""
    q = np.asarray(q, np.float64)
    positive = e4m3_values()[:127]
    a = np.abs(q)
    hi = np.clip(np.searchsorted(positive, a), 1, 126)
    lo = hi - 1
    below, above = a - positive[lo], positive[hi] - a
    code = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    code = np.where(a == 0, 0, code) | np.where(np.signbit(q), 128, 0)
    return np.where(np.isnan(q), 0x7f, code).astype(np.uint8)


def quantize(x, blocks=False):
    """(codes [rows, P], scales [P/128, rows or row blocks]) of a float32 matrix."""
    rows, cols = x.shape
    P, R = -(-cols // 128) * 128, -(-rows // 128) * 128
    full = np.zeros((R, P), np.float32)
    full[:rows, :cols] = x
    a = np.abs(np.where(np.isnan(full), 0, full))
    if blocks:
        amax = a.reshape(R // 128, 128, P // 128, 128).max((1, 3))
    else:
        amax = a.reshape(R, P // 128, 128).max(2)[:rows]
    scale = np.maximum(amax / np.float32(448.0), np.float32(2.0 ** -126))
    assert scale.dtype == np.float32
    each = np.repeat(np.repeat(scale, 128, 0)[:rows] if blocks else scale, 128, 1)
    return e4m3_codes(full[:rows] / each), np.ascontiguousarray(scale.T)


def values(codes, scales, blocks=False):
    """What codes and scales stand for, in float64."""
    s = scales.T.astype(np.float64)
    return e4m3_values()[codes] * np.repeat(np.repeat(s, 128, 0)[:codes.shape[0]] if blocks else s, 128, 1)
