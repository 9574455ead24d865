"""8-bit codes with a scale for each 128 values, and their products, against the float64 oracle (run with -m gpu).

Bounds.  Codes and scales are equal: the scheme is float32 arithmetic with one rounding each.  Of a product's 128 terms per group the matrix pipe
adds eight neighbours at a time and drops what is below 2^-13 of the largest, from each of the seven others; all other additions are float32's, with
a step 2^-23 relative to the sum of the magnitudes.  The result is rounded once, to bf16."""
import numpy as np
import pytest
import torch

from layer_util import DEV, HALF_STEP, assert_within, inside, rounded, surroundings_kept, to64
from oracle import layer as ol
from paper_2506_19852_amd import layer as rl

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def _buffers(rows, cols, scale_rows):
    groups = -(-cols // 128)
    return (torch.full((rows, groups * 128), 0xA5, dtype=torch.uint8, device=DEV), torch.full((groups, scale_rows), np.nan, device=DEV))


def _bound(a, b, want):
    """Of a product of values a [M, K] and b [N, K]."""
    K = a.shape[1]
    size = np.abs(a) @ np.abs(b).T
    largest = lambda m: np.abs(m).reshape(len(m), -1, 8).max(2)  # noqa: E731
    dropped = largest(a) @ largest(b).T
    return HALF_STEP[BF16] * np.abs(want) + 7 * 2.0 ** -13 * np.minimum(dropped, size) + (20 + K // 128) * 2.0 ** -23 * size


def _spread_values(rows, cols, seed):
    g = np.random.default_rng(seed)
    x = g.normal(size=(rows, cols)) * np.exp(g.normal(size=(rows, 1)) * 4)
    x[g.random((rows, cols)) < 0.1] = 0
    return x


@pytest.mark.parametrize("blocks", [False, True], ids=["groups", "blocks"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", [(1, 1), (3, 200), (128, 128), (129, 127), (257, 384), (40, 1000), (1000, 40), (2, 5120)], ids=str)
def test_codes_and_scales(shape, dtype, blocks):
    rows, cols = shape
    a = rounded(_spread_values(rows, cols, 31), dtype).astype(np.float32)
    a[0, :min(cols, 128)] = 0   # a group of zeros
    if rows > 2:
        a[1, 0], a[2, 0] = np.float32(1e-38), np.float32(3e38)
    a = rounded(a, dtype).astype(np.float32)
    scale_rows = lambda n: -(-n // 128) if blocks else n  # noqa: E731
    for lead, both in ((8, (True, True)), (1, (True, False)), (0, (False, True))):
        x, _ = inside(a, dtype, lead)
        straight, turned = _buffers(rows, cols, scale_rows(rows)), _buffers(cols, rows, scale_rows(cols))
        rl.radial_quantize_groups_fp8(x, *(straight if both[0] else (None, None)), *(turned if both[1] else (None, None)),
                                      grouping=rl.RADIAL_BLOCKS if blocks else rl.RADIAL_GROUPS)
        for there, (codes, scales), m in zip(both, (straight, turned), (a, a.T)):
            if there:
                want_codes, want_scales = ol.quantize(m, blocks)
                assert np.array_equal(scales.cpu().numpy(), want_scales)
                assert np.array_equal(codes.cpu().numpy(), want_codes)
        if blocks and all(both):
            assert torch.equal(turned[0][:, :rows], straight[0][:, :cols].T)


def test_what_is_not_finite_stays_in_its_group():
    a = np.random.default_rng(32).normal(size=(4, 384)).astype(np.float32)
    a[1, 130], a[2, 5] = np.nan, np.inf
    codes, scales = _buffers(4, 384, 4)
    rl.radial_quantize_groups_fp8(torch.tensor(a, device=DEV), codes, scales)
    clean = np.where(np.isfinite(a), a, 0)
    want, want_scales = ol.quantize(clean)
    got = codes.cpu().numpy()
    nan = (got & 0x7f) == 0x7f
    assert nan[1, 130] and nan[2, :128].all() and nan.sum() == 129
    assert np.array_equal(got[~nan], want[~nan])
    s = scales.cpu().numpy()
    assert np.isinf(s[0, 2]) and np.array_equal(np.delete(s.ravel(), 2), np.delete(want_scales.ravel(), 2))


# M, N, K
SIZES = [(1, 1, 1), (1, 5120, 5120), (2, 300, 1000), (16, 128, 128), (17, 129, 256), (33, 64, 384), (64, 512, 1536), (65, 96, 128), (100, 1961, 1000),
         (128, 128, 128), (256, 256, 512), (257, 255, 130), (700, 900, 640), (1024, 1024, 1024), (1237, 520, 2048), (2048, 1792, 384),
         (517, 3604, 740), (517, 3608, 600), (385, 2519, 1400), (3601, 1032, 600), (2050, 3999, 640), (3604, 3601, 600), (3604, 3608, 384),
         (4109, 3999, 1560)]


@pytest.mark.parametrize("blocks", [False, True], ids=["groups", "blocks"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_product(size, blocks):
    M, N, K = size
    g = np.random.default_rng(33)
    a, b = _spread_values(M, K, 34).astype(np.float32), g.normal(size=(N, K)).astype(np.float32)
    ac, asc = ol.quantize(a)
    bc, bs = ol.quantize(b, blocks)
    lead = 8 if N % 8 == 0 else 3
    out, whole = inside(np.zeros((M, N)), BF16, lead, lead)
    rl.radial_product_fp8(*(torch.tensor(t, device=DEV) for t in (ac, asc, bc, bs)), out)
    av, bv = ol.values(ac, asc), ol.values(bc, bs, blocks)
    want = av @ bv.T
    assert_within(out, want, _bound(av, bv, want), "product")
    # and as a whole: the errors are of either sign, so that their mean is far below the bound of a single one
    assert np.linalg.norm(to64(out) - want) <= 2.0 ** -8 * np.linalg.norm(want)
    assert surroundings_kept(out, whole)


def test_every_code_and_every_place_of_a_group():
    """Each product of two codes, at a k of its own: one value per row, one per column."""
    v = ol.e4m3_values()
    codes = np.array([c for c in range(256) if c & 0x7f != 0x7f], np.uint8)
    a = np.zeros((len(codes) * 2, 256), np.uint8)
    k = np.arange(len(a)) % 256
    a[np.arange(len(a)), k] = np.tile(codes, 2)
    b = np.tile(codes[:, None], (1, 256))
    one = lambda rows: torch.ones((2, rows), device=DEV)  # noqa: E731
    out = torch.empty((len(a), len(b)), dtype=BF16, device=DEV)
    rl.radial_product_fp8(torch.tensor(a, device=DEV), one(len(a)), torch.tensor(b, device=DEV), one(len(b)), out)
    # a product of two codes has eight significant bits: bf16 holds it
    assert np.array_equal(to64(out), v[np.tile(codes, 2)][:, None] * v[codes][None])


@pytest.mark.parametrize("size", [(2, 384, 256), (300, 384, 256)], ids=str)
def test_codes_of_nan_reach_their_row_and_column_alone(size):
    M, N, K = size
    g = np.random.default_rng(35)
    ac, asc = ol.quantize(g.normal(size=(M, K)).astype(np.float32))
    bc, bs = ol.quantize(g.normal(size=(N, K)).astype(np.float32))
    ac[1, 200], bc[7, 3] = 0x7f, 0xff
    out = torch.empty((M, N), dtype=BF16, device=DEV)
    rl.radial_product_fp8(*(torch.tensor(t, device=DEV) for t in (ac, asc, bc, bs)), out)
    bad = np.zeros((M, N), bool)
    bad[1], bad[:, 7] = True, True
    assert np.array_equal(np.isnan(to64(out)), bad)


@pytest.mark.parametrize("size", [(300, 260, 500), (5, 260, 500)], ids=str)
def test_both_gradients(size):
    """dX = dY W and dW = dY^T X from codes, against the products of the values they stand for, and of the values before quantisation: each operand is
    off by at most 2^-4 of its value or 2^-10 of its scale."""
    M, N, K = size
    g = np.random.default_rng(36)
    x, w, dy = (rounded(g.normal(size=s), BF16).astype(np.float32) for s in ((M, K), (N, K), (M, N)))
    t = {n: torch.tensor(v).to(BF16).to(DEV) for n, v in (("x", x), ("w", w), ("dy", dy))}
    wt = _buffers(K, N, -(-K // 128))
    rl.radial_quantize_groups_fp8(t["w"], None, None, *wt, grouping=rl.RADIAL_BLOCKS)
    dyq, dyt, xt = _buffers(M, N, M), _buffers(N, M, N), _buffers(K, M, K)
    rl.radial_quantize_groups_fp8(t["dy"], *dyq, *dyt)
    rl.radial_quantize_groups_fp8(t["x"], None, None, *xt)
    dx, dw = torch.empty((M, K), dtype=BF16, device=DEV), torch.empty((N, K), dtype=BF16, device=DEV)
    rl.radial_product_fp8(*dyq, *wt, dx)
    rl.radial_product_fp8(*dyt, *xt, dw)

    def of(m, blocks=False):
        return ol.values(*ol.quantize(np.ascontiguousarray(m), blocks), blocks)

    for got, (p, q), (p0, q0), what in ((dx, (of(dy), of(w.T, True)), (dy, w.T), "dX"), (dw, (of(dy.T), of(x.T)), (dy.T, x.T), "dW")):
        want = p @ q.T
        bound = _bound(p, q, want)
        assert_within(got, want, bound, what)
        e, f = np.abs(p[:, :p0.shape[1]] - p0), np.abs(q[:, :q0.shape[1]] - q0)
        assert (e <= 2.0 ** -4 * np.abs(p0) + np.abs(p0).max() / 448 * 2.0 ** -10).all() and (f <= 2.0 ** -4 * np.abs(q0) + np.abs(q0).max() / 448 * 2.0 ** -10).all()
        assert_within(got, p0 @ q0.T, e @ np.abs(q0).T + np.abs(p0) @ f.T + e @ f.T + bound, what + " against the values")


def test_more_than_2_to_the_31_elements():
    M, N = (1 << 16) + 70, (1 << 15) + 128
    g = torch.Generator(device=DEV).manual_seed(5)
    x, w = (torch.randn(n, 128, device=DEV, generator=g).to(BF16) for n in (M, N))
    a, b = _buffers(M, 128, M), _buffers(N, 128, N // 128)
    rl.radial_quantize_groups_fp8(x, *a)
    rl.radial_quantize_groups_fp8(w, *b, grouping=rl.RADIAL_BLOCKS)
    out = torch.empty((M, N), dtype=BF16, device=DEV)
    rl.radial_product_fp8(*a, *b, out)
    last = torch.empty((70, N), dtype=BF16, device=DEV)
    rl.radial_product_fp8(a[0][-70:], a[1][:, -70:].contiguous(), *b, last)
    assert torch.equal(out[-70:], last)
    codes, scales = _buffers(M, N, M)     # and an input of that size
    rl.radial_quantize_groups_fp8(out, codes, scales)
    few = _buffers(70, N, 70)
    rl.radial_quantize_groups_fp8(last, *few)
    assert torch.equal(codes[-70:], few[0]) and torch.equal(scales[:, -70:], few[1])


# few results of many groups, in pieces of 16 x 16; tiles of every form that are too many for that
MORE_SIZES = [(17, 2048, 384), (256, 128, 20519), (128, 127, 2048), (250, 250, 130), (31, 33, 8000), (65, 1111, 128), (600, 120, 4100), (333, 333, 2000)]


@pytest.mark.parametrize("blocks", [False, True], ids=["groups", "blocks"])
@pytest.mark.parametrize("size", MORE_SIZES, ids=str)
def test_product_of_few_results(size, blocks):
    test_product(size, blocks)


@pytest.mark.parametrize("blocks", [False, True], ids=["groups", "blocks"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", [(4, 130), (130, 130), (129, 257), (300, 7), (7, 300)], ids=str)
def test_codes_behind_the_matrix_are_zero_beside_an_infinity(shape, dtype, blocks):
    """An infinite scale makes NaN of its whole group, but of the group's columns alone."""
    rows, cols = shape
    a = rounded(np.random.default_rng(37).normal(size=shape), dtype).astype(np.float32)
    a[-1, -1], a[1, 2], a[2, -1] = np.inf, -np.inf, np.nan
    x = torch.tensor(a, dtype=dtype, device=DEV)
    scale_rows = lambda n: -(-n // 128) if blocks else n  # noqa: E731
    for both in ((True, True), (True, False), (False, True)):
        straight, turned = _buffers(rows, cols, scale_rows(rows)), _buffers(cols, rows, scale_rows(cols))
        rl.radial_quantize_groups_fp8(x, *(straight if both[0] else (None, None)), *(turned if both[1] else (None, None)),
                                      grouping=rl.RADIAL_BLOCKS if blocks else rl.RADIAL_GROUPS)
        for there, (codes, scales), m in zip(both, (straight, turned), (a, a.T)):
            if not there:
                continue
            R, P = -(-m.shape[0] // 128) * 128, codes.shape[1]
            full = np.zeros((R, P), np.float32)
            full[:m.shape[0], :m.shape[1]] = m
            tiles = np.isinf(full).reshape(R // 128, 128, P // 128, 128).any((1, 3) if blocks else 3)
            infinite = np.repeat(np.repeat(tiles, 128, 0) if blocks else tiles.reshape(R, -1), 128, 1)[:m.shape[0]]
            got = codes.cpu().numpy()
            assert not got[:, m.shape[1]:].any()
            assert (((got & 0x7f) == 0x7f) == ((infinite | np.isnan(full[:m.shape[0]])) & (np.arange(P) < m.shape[1]))).all()
            clean, _ = ol.quantize(np.where(infinite[:, :m.shape[1]], 0, m).astype(np.float32), blocks)
            ok = ~infinite & ~np.isnan(full[:m.shape[0]])
            assert np.array_equal(got[ok], clean[ok])


# rows that two launches share: whole rounds in one of the two largest forms, the rest in a large one or a small one
TWO_LAUNCHES = [(12919, 1822, 6000), (10838, 2091, 3400), (13249, 2624, 1000), (10862, 1305, 2750), (12580, 2832, 2400)]


@pytest.mark.parametrize("blocks", [False, True], ids=["groups", "blocks"])
@pytest.mark.parametrize("size", [(3, 1961, 1000), (16, 2000, 520), (250, 250, 1000), (257, 255, 130), (1024, 1024, 1024), *TWO_LAUNCHES], ids=str)
def test_results_are_off_by_little_more_than_their_rounding(size, blocks):
    """Random codes and scales, against the products of their values in float64.  One by one as in test_product; and as a whole, where what is dropped, of
    either sign as the codes are, adds up as squares: from each eight products at most 7 parts of 2^-13 of the largest, whose square is at most that of all
    eight together, sqrt(7) 2^-13 of the result in all.  1 % is for what the two errors have in common."""
    M, N, K = size
    g = torch.Generator(device=DEV).manual_seed(38)
    v = torch.tensor(ol.e4m3_values(), device=DEV)
    P = -(-K // 128) * 128

    def operand(rows, scale_rows):
        codes = torch.randint(0, 254, (rows, P), generator=g, device=DEV, dtype=torch.int32)
        codes = codes + (codes >= 127)                 # all but 0x7f and 0xff
        codes[:, K:] = 0
        scales = torch.randn((P // 128, scale_rows), generator=g, device=DEV).exp()
        full = scales.t().double().repeat_interleave(128, 0)[:rows] if scale_rows != rows else scales.t().double()
        values = v[codes.long()].view(rows, -1, 128) * full[..., None]
        return codes.to(torch.uint8), scales, values.view(rows, P)

    (ac, asc, av), (bc, bs, bv) = operand(M, M), operand(N, -(-N // 128) if blocks else N)
    lead = 8 if N % 8 == 0 else 3
    whole = torch.full((M + 1, N + 2 * lead), 7.5, dtype=BF16, device=DEV)
    out = whole[:M, lead:lead + N]
    rl.radial_product_fp8(ac, asc, bc, bs, out)
    want = av @ bv.t()
    size_ = av.abs() @ bv.abs().t()
    largest = lambda m: m.abs().view(len(m), -1, 8).amax(2)  # noqa: E731
    bound = HALF_STEP[BF16] * want.abs() + 7 * 2.0 ** -13 * torch.minimum(largest(av) @ largest(bv).t(), size_) + (20 + P // 128) * 2.0 ** -23 * size_
    off = out.double() - want
    assert off.isfinite().all() and (off.abs() <= bound).all(), float((off.abs() / bound).max())
    rounding = (want.to(BF16).double() - want).norm()
    assert off.norm() <= 1.01 * (rounding ** 2 + 7 * 2.0 ** -26 * want.norm() ** 2) ** 0.5, (float(off.norm() / rounding))
    out.fill_(7.5)
    assert (whole == 7.5).all()


@pytest.mark.parametrize("M", [1, 16, 300], ids=["one row", "few rows", "tiles"])
def test_what_is_left_where_large_products_cancel(M):
    """256 - 256 + p: beside neither of the two (another eight of the 128) p is exact, in float32's reach; beside one of them it is exact down to 2^-13 of it,
    and what is smaller is off by at most itself."""
    v = ol.e4m3_values()
    values = {v[c]: c for c in range(127)}
    N, cases = 300, []
    for first, second in ((0, 127), (64, 65), (13, 40)):
        for spot in (1, 5, 7, 8, 12, 33, 66, 71, 72, 120, 126):
            for e in range(0, 18):
                x = 2.0 ** max(-6, 4 - e // 2)
                if spot not in (first, second):
                    cases.append((first, second, spot, x, 2.0 ** (8 - e) / x))
    a, b = np.zeros((len(cases), 128), np.uint8), np.zeros((len(cases), 128), np.uint8)
    for i, (first, second, spot, x, y) in enumerate(cases):
        a[i, [first, second, spot]] = values[16.0], values[16.0], values[x]
        b[i, [first, second, spot]] = values[16.0], values[16.0] | 128, values[y]
    one = lambda n: torch.ones((1, n), device=DEV)  # noqa: E731
    for at in range(0, len(cases), M):
        # row m of A against all columns: its own is the case, wherever it lies in the tile
        rows, some = a[at:at + M], b[at:at + M]
        columns = np.resize(some, (N, 128)) if M < N else some
        out = torch.empty((len(rows), len(columns)), dtype=BF16, device=DEV)
        rl.radial_product_fp8(torch.tensor(rows, device=DEV), one(len(rows)), torch.tensor(columns, device=DEV), one(len(columns)), out)
        for i, (first, second, spot, x, y) in enumerate(cases[at:at + M]):
            p, beside = x * y, spot // 8 in (first // 8, second // 8)
            got = to64(out[i, i::len(rows)])
            assert len(got) and (got == got[0]).all()
            if not beside or p >= 256 * 2.0 ** -13:
                assert got[0] == p, (first, second, spot, p, got[0])
            else:
                assert abs(got[0] - p) <= p, (first, second, spot, p, got[0])
