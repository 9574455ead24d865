"""Rotary positions against the float64 oracle (run with -m gpu).

Bounds.  cos and sin are float32 (half a step of u = 2^-24 each), a turn is two products and a sum in float32: at most 4 u magnitude (|u| + |v|), then
one rounding to the type."""
import numpy as np
import pytest
import torch

from layer_util import DEV, HALF_STEP, U32, assert_within, inside, rounded, surroundings_kept, to64
from oracle import layer as ol
from paper_2506_19852_amd import layer as rl

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32

# sizes, dims, head dimension, layout, B, q heads, k heads, N, first
CASES = [
    ([1], [2], 8, "interleaved", 1, 1, 0, 1, 0),
    ([50], [64], 64, "half", 2, 3, 1, 37, 5),
    ([5, 6, 7], [16, 56, 56], 128, "interleaved", 1, 5, 5, 5 * 6 * 7, 0),
    ([5, 6, 7], [16, 56, 56], 128, "half", 2, 9, 2, 5 * 6 * 7 + 11, 0),      # text behind the video
    ([4, 5], [6, 10], 24, "interleaved", 3, 2, 2, 13, 4),                     # axes that end inside a piece
    ([100], [20], 64, "half", 2, 7, 1, 90, 0),                                # a half that is not 16-byte aligned
    ([100], [34], 40, "interleaved", 1, 2, 1, 90, 30),
    ([3, 3], [32, 32], 128, "half", 1, 2, 0, 9, 0),                           # part of a head
    ([70000], [128], 128, "interleaved", 4, 40, 8, 1, 69999),
    ([9], [1024], 1024, "half", 1, 1, 1, 9, 0),
]


def _table(sizes, dims, **kw):
    p = rl.rope_params(sizes, dims, **kw)
    table = torch.full((rl.radial_rope_table_bytes(p) // 4 + 2,), 9.0, device=DEV)
    rl.radial_rope_table(p, table)
    assert (table[-2:] == 9.0).all()
    return p, table


@pytest.mark.parametrize("scaling", ["none", "linear", "base", "parts"])
def test_table(scaling):
    sizes, dims = [2000, 7, 1], [32, 2, 6]
    p, table = _table(sizes, dims, theta=5e4, scaling=scaling, factor=3.7, original=500, fast=20.0, slow=2.0, magnitude=1.25)
    freqs = [ol.frequencies(d, 5e4, scaling, 3.7, 500, 20.0, 2.0) for d in dims]
    want = ol.rope_table(sizes, freqs, 1.25)
    # the angle in 64 bits: its error is position * 2^-50, far below a float32 step of the result
    assert_within(table[:-2].view(-1, 2), want, 1.25 * (U32 + 1e-9), "table")


def test_table_at_far_positions():
    p, table = _table([1 << 24], [2])
    n = np.array([0, 1, 12345678, (1 << 24) - 1])
    got = to64(table[:-2].view(-1, 2))[n]
    assert_within(got, np.stack([np.cos(n.astype(np.float64)), np.sin(n.astype(np.float64))], -1), U32 + 1e-9, "far table")


@pytest.mark.parametrize("gradient", [False, True], ids=["fwd", "bwd"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_turns(case, dtype, gradient):
    sizes, dims, D, layout, B, H, Hk, N, first = case
    g = np.random.default_rng(21)
    kw = dict(scaling="linear", factor=2.0, magnitude=1.1)
    p, table = _table(sizes, dims, layout=layout, **kw)
    freqs = [ol.frequencies(d, scaling="linear", factor=2.0) for d in dims]
    total = int(np.prod(sizes))
    call = rl.radial_rope_bwd if gradient else rl.radial_rope_fwd
    for given in (False, True):
        index = g.integers(-3, total + 3, (B, N)) if given else np.broadcast_to(np.arange(first, first + N), (B, N))
        args = []
        for heads in (H, Hk):
            if heads:
                a = rounded(g.normal(size=(B, N, heads, D)), dtype)      # token-major in, head-major out
                x = inside(a.reshape(B, N, heads * D), dtype)[0].unflatten(2, (heads, D)).transpose(1, 2)
                out, whole = inside(np.zeros((B, heads, N, D)), dtype)
                args.append((a.transpose(0, 2, 1, 3), x, out, whole))
        kw = {"positions": torch.tensor(index, dtype=torch.int32, device=DEV)} if given else {"first": first}
        call(p, table, *(t for _, x, out, _ in args for t in (x, out)), **kw)
        for a, x, out, whole in args:
            want = ol.rope(a, index, sizes, freqs, layout, 1.1, gradient)
            other = np.abs(ol.rope(a, index * 0 + total, sizes, freqs, layout)) + _partner(np.abs(a), sum(dims), layout)
            assert_within(out, want, HALF_STEP[dtype] * np.abs(want) + 4 * U32 * 1.1 * other, "turned")
            assert surroundings_kept(out, whole)
            stays = (index < 0) | (index >= total)
            for b in range(B):
                assert np.array_equal(to64(out)[b][:, stays[b]], a[b][:, stays[b]])
            assert np.array_equal(to64(out)[..., sum(dims):], a[..., sum(dims):])


def _partner(a, R, layout):
    """The other dimension of each dimension's pair (0 where it has none)."""
    out = np.zeros_like(a)
    if layout == "interleaved":
        out[..., 0:R:2], out[..., 1:R:2] = a[..., 1:R:2], a[..., 0:R:2]
    else:
        out[..., :R // 2], out[..., R // 2:R] = a[..., R // 2:R], a[..., :R // 2]
    return out


@pytest.mark.parametrize("case", CASES, ids=str)
def test_in_place_is_the_same(case):
    sizes, dims, D, layout, B, H, Hk, N, first = case
    p, table = _table(sizes, dims, layout=layout)
    g = torch.Generator(device=DEV).manual_seed(3)
    q = torch.randn(B, H, N, D, device=DEV, generator=g).to(BF16)
    out = torch.empty_like(q)
    rl.radial_rope_fwd(p, table, q, out, first=first)
    rl.radial_rope_fwd(p, table, q, q, first=first)
    assert torch.equal(q, out)


def test_masked_values_that_are_not_finite_stay_in_their_pair():
    p, table = _table([10], [16], layout="half")
    q = torch.ones(1, 1, 10, 24, device=DEV, dtype=BF16)
    q[0, 0, 4, 3], q[0, 0, 5, 20] = float("nan"), float("inf")
    out = torch.empty_like(q)
    rl.radial_rope_fwd(p, table, q, out)
    bad = ~out.isfinite()
    assert sorted(map(tuple, bad[0, 0].nonzero().tolist())) == [(4, 3), (4, 11), (5, 20)]


def test_more_than_2_to_the_31_elements():
    D, N = 128, (1 << 24) + 5
    p, table = _table([N], [2])
    q = torch.zeros(1, 1, N, D, dtype=BF16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(4)
    some = torch.randn(1, 1, 7, D, device=DEV, generator=g).to(BF16)
    q[:, :, -7:] = some
    out = torch.empty_like(q)
    rl.radial_rope_fwd(p, table, q, out)
    want = torch.empty_like(some)
    rl.radial_rope_fwd(p, table, some, want, first=N - 7)
    assert torch.equal(out[:, :, -7:], want) and not torch.equal(want, some)


@pytest.mark.parametrize("gradient", [False, True], ids=["fwd", "bwd"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("dims,D,layout", [([16, 14], 48, "interleaved"), ([16, 16], 48, "half"), ([10, 10], 48, "half")], ids=str)
def test_what_is_not_turned_is_copied(dims, D, layout, dtype, gradient):
    """Text, padding and the dimensions behind the turned ones keep their values beside infinities, and the sign of a zero."""
    p, table = _table([4, 5], dims, layout=layout)
    R, N = sum(dims), 20
    x = rounded(np.random.default_rng(8).normal(size=(1, 3, N, D)), dtype).astype(np.float32)
    for at, value in ((1, np.inf), (2, -np.inf), (5, np.nan), (8, -0.0), (9, -1.0), (24, -np.inf)):
        x[..., 3, at] = value            # the token off the grid
        if R + at < D:
            x[..., R + at] = value       # behind the turned dimensions, of every token
    positions = torch.arange(N, dtype=torch.int32, device=DEV).view(1, N).clone()
    positions[0, 3] = -1
    q = torch.tensor(x, dtype=dtype, device=DEV)
    out = torch.empty_like(q)
    (rl.radial_rope_bwd if gradient else rl.radial_rope_fwd)(p, table, q, out, positions=positions)
    got, want = out.float().cpu(), torch.tensor(x)
    for a, b in ((got[..., 3, :], want[..., 3, :]), (got[..., R:], want[..., R:])):
        assert torch.equal(a.isnan(), b.isnan())
        assert torch.equal(a.nan_to_num(7.0, 8.0, 9.0), b.nan_to_num(7.0, 8.0, 9.0)) and torch.equal(a.signbit() & ~b.isnan(), b.signbit() & ~b.isnan())


@pytest.mark.parametrize("gradient", [False, True], ids=["fwd", "bwd"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("dims,D", [([2], 8), ([6], 8), ([6], 16), ([12], 24), ([18], 24), ([22], 24), ([14, 8], 32), ([26], 40), ([30], 32), ([10, 20, 12], 48),
                                    ([46], 64), ([78], 80), ([90], 96), ([122], 128)], ids=str)
def test_halves_that_end_anywhere(dims, D, dtype, gradient):
    """One to seven pairs, and dimensions that stay, in the last piece of each."""
    case = ([3, 4, 5][:len(dims)], dims, D, "half", 2, 3, 1, 11, 1)
    test_turns(case, dtype, gradient)
    test_in_place_is_the_same(case)


@pytest.mark.parametrize("gradient", [False, True], ids=["fwd", "bwd"])
@pytest.mark.parametrize("dims,layout", [([24], "interleaved"), ([6, 14], "interleaved"), ([16], "half"), ([20], "half"), ([64], "half")], ids=str)
def test_copies_keep_every_bit(dims, layout, gradient):
    """Of every bf16 pattern, NaNs that signal and carry a payload among them, and of float32 ones."""
    p, table = _table([4] * len(dims), dims, layout=layout)
    R, D = sum(dims), 64
    patterns = np.arange(1 << 16, dtype=np.uint16).view(np.int16)
    words = np.random.default_rng(9).integers(0, 1 << 32, 1 << 16, dtype=np.uint32)
    words[1::2] |= 0x7f800000                       # infinities and NaNs
    call = rl.radial_rope_bwd if gradient else rl.radial_rope_fwd
    for whole, dtype in ((patterns, BF16), (words.view(np.int32), F32)):
        bits = torch.tensor(whole.reshape(1, 1, -1, D), device=DEV)
        x = bits.view(dtype)
        N = x.shape[2]
        for on in (0, 1):
            positions = torch.full((1, N), 1 if on else -1, dtype=torch.int32, device=DEV)
            for in_place in (False, True):
                out = x.clone() if in_place else torch.empty_like(x)
                call(p, table, out if in_place else x, out, positions=positions)
                from_ = R if on else 0
                assert torch.equal(out.view(bits.dtype)[..., from_:], bits[..., from_:]), (dtype, on, in_place)
