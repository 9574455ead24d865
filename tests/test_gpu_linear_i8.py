"""8-bit integer products: codes, products, the projection and its gradients against the oracle (run with -m gpu).

Bounds.  Codes and scales are equal: float32 arithmetic with one rounding each.  A product's sum is a whole number and exact; its conversion to float32, the
product of the scales, the scaled sum with the bias and what is added to take one rounding each, 2^-24 relative, and the result is rounded once to its type."""
import numpy as np
import pytest
import torch

from layer_util import DEV, HALF_STEP, U32, assert_within, inside, rounded, surroundings_kept, to64
from oracle import step as os_
from paper_2506_19852_amd import layer as rl

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def bound(want, size, dtype, additions=1):
    """Of a product: conversion, scales and their product with the sum; then each addition; then the type."""
    exact = 3 * U32 * size + additions * U32 * np.abs(want) * (1 + U32)
    return exact + (HALF_STEP[dtype] * (np.abs(want) + exact) if dtype is BF16 else 0) + 1e-44


def put_codes(codes, scales):
    return torch.tensor(codes, device=DEV), torch.tensor(scales, device=DEV)


def buffers(rows, cols):
    return torch.full((rows, -(-cols // 128) * 128), 77, dtype=torch.int8, device=DEV), torch.full((rows,), float("nan"), device=DEV)


def workspace(size):
    return torch.full((size,), 255, dtype=torch.uint8, device=DEV)


def random_codes(rows, cols, seed, extreme=False):
    g = np.random.default_rng(seed)
    codes = np.zeros((rows, -(-cols // 128) * 128), np.int8)
    codes[:, :cols] = g.integers(-128, 128, (rows, cols)) if not extreme else g.choice([-128, 127], (rows, cols))
    return codes, np.exp(g.normal(size=rows) * 2).astype(np.float32)


def spread_values(rows, cols, seed):
    g = np.random.default_rng(seed)
    x = g.normal(size=(rows, cols)) * np.exp(g.normal(size=(rows, 1)) * 4)
    x[g.random((rows, cols)) < 0.1] = 0
    return x


# ---- codes --------------------------------------------------------------------------------------

# a width of each number of pieces that a wave keeps, and beyond
SHAPES = [(1, 1), (3, 200), (128, 128), (129, 127), (5, 1000), (257, 384), (40, 2048), (1000, 40), (2, 5120), (7, 2999), (3, 8192), (2, 8200), (4, 20001), (300, 513), (5, 2049), (6, 6144), (7, 6145), (2049, 900), (2050, 1500), (2051, 2050), (2052, 3000), (2053, 5000), (2054, 8000), (2055, 8193)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_codes_and_scales(shape, dtype):
    rows, cols = shape
    a = rounded(spread_values(rows, cols, 41), dtype).astype(np.float32)
    if rows > 2:
        a[0] = 0
        a[1, 0], a[2, 0] = np.float32(1e-38), np.float32(3e38)
        a = rounded(a, dtype).astype(np.float32)
    with np.errstate(over="ignore"):
        sums, size = a.astype(np.float64).sum(0), np.abs(a.astype(np.float64)).sum(0)
    for lead, both in ((8, (True, True)), (1, (True, False)), (0, (False, True)), (3, (False, False))):
        x, whole = inside(a, dtype, lead)
        straight, turned = buffers(rows, cols), buffers(cols, rows)
        total = torch.full((cols,), float("nan"), device=DEV)
        rl.radial_quantize_rows_i8(x, *(straight if both[0] else (None, None)), *(turned if both[1] else (None, None)),
                                   workspace(rl.radial_quantize_rows_i8_workspace(rows, cols)), sums_t=total)
        for there, (codes, scales), m in zip(both, (straight, turned), (a, np.ascontiguousarray(a.T))):
            if there:
                want_codes, want_scales = os_.quantize_rows(m)
                assert np.array_equal(scales.cpu().numpy(), want_scales)
                assert np.array_equal(codes.cpu().numpy(), want_codes)
        assert_within(total, sums, rows * U32 * size, "sums")
        assert surroundings_kept(x, whole)


def test_half_of_the_largest_is_a_tie_of_float32():
    """amax/2 over amax/127 is 63.5 or its neighbour, as the quotient's rounding to float32 has it."""
    largest = np.arange(128, 256, dtype=np.float32)
    a = np.stack([largest, largest / 2, -largest / 2, largest / 254 * 3], 1)
    a = rounded(a, BF16).astype(np.float32)
    codes, scales = buffers(len(a), 4)
    rl.radial_quantize_rows_i8(torch.tensor(a, device=DEV).to(BF16), codes, scales)
    want, _ = os_.quantize_rows(a)
    assert np.array_equal(codes.cpu().numpy(), want) and {63, 64} <= set(np.unique(np.abs(want)))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_rows_and_columns_that_are_not_finite_say_so_and_no_others(dtype):
    a = np.random.default_rng(42).normal(size=(300, 700)).astype(np.float32)
    a[5, 600], a[7, 3], a[299, 699] = np.nan, np.inf, -np.inf
    x = torch.tensor(a, device=DEV).to(dtype)
    a = x.float().cpu().numpy()
    straight, turned = buffers(300, 700), buffers(700, 300)
    rl.radial_quantize_rows_i8(x, *straight, *turned, workspace(rl.radial_quantize_rows_i8_workspace(300, 700)))
    for (codes, scales), m in ((straight, a), (turned, a.T)):
        want_codes, want_scales = os_.quantize_rows(np.ascontiguousarray(m))
        assert np.isnan(want_scales).sum() == 3
        assert np.array_equal(scales.cpu().numpy(), want_scales, equal_nan=True) and np.array_equal(codes.cpu().numpy(), want_codes)


def test_sums_are_added_to_what_is_there():
    a = np.random.default_rng(43).normal(size=(130, 70))
    x = torch.tensor(a, device=DEV).to(BF16)
    a = to64(x)
    total = torch.full((70,), 3.0, device=DEV)
    rl.radial_quantize_rows_i8(x, workspace=workspace(rl.radial_quantize_rows_i8_workspace(130, 70)), sums_t=total, accumulate=True)
    assert_within(total, a.sum(0) + 3, 130 * U32 * np.abs(a).sum(0) + U32 * 30, "sums")


# ---- products -------------------------------------------------------------------------------------

# M, N, K
SIZES = [(1, 1, 1), (1, 5120, 5120), (2, 300, 1000), (16, 128, 128), (17, 129, 256), (33, 64, 384), (64, 512, 1536), (65, 96, 128), (100, 1961, 1000),
         (128, 128, 128), (129, 4100, 300), (200, 333, 2049), (256, 2048, 640), (257, 257, 257), (512, 5120, 4096), (600, 1536, 1000), (1237, 1961, 1001),
         (2000, 5120, 384), (3333, 2500, 130), (8200, 5000, 256), (4, 700, 900), (5, 700, 900), (64, 5120, 2048), (64, 2048, 4096), (20, 5120, 640), (300, 2048, 4096),
         (700, 5120, 256), (450, 5120, 900), (1560, 5120, 384), (5000, 2000, 300), (14040, 333, 130), (1560, 2000, 2048), (6000, 3000, 4096)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_product(size, dtype):
    M, N, K = size
    a, sa = random_codes(M, K, 44)
    b, sb = random_codes(N, K, 45)
    g = np.random.default_rng(46)
    bias = (g.normal(size=N) * 100).astype(np.float32)
    want, scaled = os_.product(a, sa, b, sb, bias)
    lead = 8 if (M + N) % 2 else 3
    out, whole = inside(np.full((M, N), np.nan), dtype, lead)
    rl.radial_product_i8(*put_codes(a, sa), *put_codes(b, sb), out, bias=torch.tensor(bias, device=DEV))
    assert_within(out, want, bound(want, scaled, dtype), "with bias")
    assert surroundings_kept(out, whole)
    rl.radial_product_i8(*put_codes(a, sa), *put_codes(b, sb), out)
    assert_within(out, want - bias, bound(want - bias, scaled, dtype), "without")
    if dtype is F32:
        before = to64(out)
        rl.radial_product_i8(*put_codes(a, sa), *put_codes(b, sb), out, bias=torch.tensor(bias, device=DEV), accumulate=True)
        assert_within(out, before + want, bound(want, scaled, dtype) + 2 * U32 * np.abs(before + want), "added")
        assert surroundings_kept(out, whole)


@pytest.mark.parametrize("size", [(16, 16, 131071), (300, 257, 131071), (40, 40, 131071)], ids=str)
def test_the_longest_sum_is_exact(size):
    """Codes of the largest magnitude: the sum is 2^31 - 2^14."""
    M, N, K = size
    a = np.full((M, 131072), -128, np.int8)
    a[:, K:] = 0
    b = a[:1].repeat(N, 0)
    b[1::2] = np.where(b[1::2] == 0, 0, 127)
    ones = lambda n: np.ones(n, np.float32)  # noqa: E731
    out = torch.empty((M, N), device=DEV)
    rl.radial_product_i8(*put_codes(a, ones(M)), *put_codes(b, ones(N)), out)
    want = np.where(np.arange(N) % 2, -128 * 127 * K, 128 * 128 * K).astype(np.float64)
    assert np.array_equal(to64(out), np.broadcast_to(want.astype(np.float32).astype(np.float64), (M, N)))


@pytest.mark.parametrize("size", [(5, 40, 131072), (70, 130, 270000)], ids=str)
def test_longer_sums_are_added_in_parts(size):
    M, N, K = size
    a, sa = random_codes(M, K, 47)
    b, sb = random_codes(N, K, 48)
    want, _ = os_.product(a, sa, b, sb)
    out = torch.full((M, N), float("nan"), device=DEV)
    rl.radial_product_i8(*put_codes(a, sa), *put_codes(b, sb), out)
    most = 0.0   # what is rounded: the sums of the parts, and each partial total
    for at in range(0, K, 130944):
        most = most + os_.product(a[:, at:at + 130944], sa, b[:, at:at + 130944], sb)[1]
    assert_within(out, want, 6 * U32 * most, "parts")
    # added to, with a bias, which counts once
    before, bias = to64(out), np.linspace(-1e3, 1e3, N).astype(np.float32)
    rl.radial_product_i8(*put_codes(a, sa), *put_codes(b, sb), out, bias=torch.tensor(bias, device=DEV), accumulate=True)
    assert_within(out, before + want + bias, 10 * U32 * (most + np.abs(before) + np.abs(bias)), "parts added")


def test_more_than_2_to_the_31_codes_and_results():
    """Rows of codes and of results that lie beyond 2^31 bytes from the first."""
    M, N, K = 300_000, 3600, 8192
    a = torch.zeros((M, K), dtype=torch.int8, device=DEV)
    a[-1] = 1
    a[-260, 5] = 3
    b = torch.zeros((N, K), dtype=torch.int8, device=DEV)
    b[-1], b[7] = 2, 1
    out = torch.full((M, N), float("nan"), dtype=BF16, device=DEV)
    rl.radial_product_i8(a, torch.ones(M, device=DEV), b, torch.ones(N, device=DEV), out)
    assert out[-1, -1] == 2 * K and out[-1, 7] == K and out[-260, 7] == 3 and out[-260, -1] == 6
    assert out[:-260].abs().max() == 0 and out.float().sum(dtype=torch.float64) == 3 * K + 9
    codes, scales = torch.empty((M, N + 112), dtype=torch.int8, device=DEV), torch.empty(M, device=DEV)
    rl.radial_quantize_rows_i8(out, codes, scales)
    assert codes[-1, N - 1] == 127 and codes[-1, 7] == 64 and codes[-260, 7] == 64 and int(codes[:-260].abs().max()) == 0


@pytest.mark.parametrize("M", [2, 300], ids=str)
def test_a_scale_of_nan_reaches_its_row_and_column_alone(M):
    a, sa = random_codes(M, 200, 49)
    b, sb = random_codes(90, 200, 50)
    a[1], sa[1], b[5], sb[5] = 0, np.nan, 0, np.nan
    out = torch.empty((M, 90), device=DEV)
    rl.radial_product_i8(*put_codes(a, sa), *put_codes(b, sb), out)
    nan = out.isnan().cpu().numpy()
    assert nan[1].all() and nan[:, 5].all() and nan.sum() == 90 + M - 1


# ---- projection -----------------------------------------------------------------------------------

LINEAR = [(1, 64, 64), (2, 5120, 5120), (1, 333, 8192), (3, 77, 1000), (4, 130, 8191), (4, 40, 8193), (2, 16, 1), (5, 100, 3000), (16, 40, 20000), (77, 640, 1000), (130, 257, 300), (1001, 333, 2049)]


def _linear(M, N, K, dtype, seed):
    g = np.random.default_rng(seed)
    x, xw = inside(g.normal(size=(M, K)) * np.exp(g.normal(size=K)), dtype, 8 if seed % 2 else 1)
    w = (g.normal(size=(N, K)) * K ** -0.5).astype(np.float32)
    dy, _ = inside(g.normal(size=(M, N)) * 0.02, dtype, 5)
    return x, w, (g.normal(size=N) * 0.1).astype(np.float32), dy


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("size", LINEAR, ids=str)
def test_projection(size, dtype):
    M, N, K = size
    x, w, bias, _ = _linear(M, N, K, dtype, 51)
    wc, ws = os_.quantize_rows(w)
    xc, xs = os_.quantize_rows(x.float().cpu().numpy())
    for out_type in (BF16, F32):
        want, scaled = os_.product(xc, xs, wc, ws, bias)
        y, whole = inside(np.full((M, N), np.nan), out_type, 4)
        rl.radial_linear_i8_fwd(x, *put_codes(wc, ws), y, workspace(rl.radial_linear_i8_fwd_workspace(M, N, K)), bias=torch.tensor(bias, device=DEV))
        assert_within(y, want, bound(want, scaled, out_type), "y")
        assert surroundings_kept(y, whole)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("size", LINEAR, ids=str)
def test_gradients_of_a_projection(size, dtype):
    M, N, K = size
    x, w, _, dy = _linear(M, N, K, dtype, 52)
    x64, dy64 = to64(x), to64(dy)
    f32 = lambda a: np.ascontiguousarray(a, dtype=np.float32)  # noqa: E731
    wt = os_.quantize_rows(f32(w.T))
    want_dx, size_dx = os_.product(*os_.quantize_rows(f32(dy64)), *wt)
    want_dw, size_dw = os_.product(*os_.quantize_rows(f32(dy64.T)), *os_.quantize_rows(f32(x64.T)))
    ws = workspace(rl.radial_linear_i8_bwd_workspace(M, N, K))
    for out_type in (BF16, F32):
        dx, dx_whole = inside(np.full((M, K), np.nan), out_type, 3)
        dw, dw_whole = inside(np.full((N, K), np.nan), out_type, 8)
        dbias = torch.full((N,), float("nan"), device=DEV)
        rl.radial_linear_i8_bwd(dy, ws, x=x, wt_codes=put_codes(*wt)[0], wt_scales=put_codes(*wt)[1], dx=dx, dw=dw, dbias=dbias)
        assert_within(dx, want_dx, bound(want_dx, size_dx, out_type), "dx")
        assert_within(dw, want_dw, bound(want_dw, size_dw, out_type), "dw")
        assert_within(dbias, dy64.sum(0), M * U32 * np.abs(dy64).sum(0), "dbias")
        assert surroundings_kept(dx, dx_whole) and surroundings_kept(dw, dw_whole)
    before, bias_before = to64(dw), to64(dbias)
    rl.radial_linear_i8_bwd(dy, ws, x=x, dw=dw, dbias=dbias, accumulate=True)
    assert_within(dw, before + want_dw, bound(want_dw, size_dw, F32) + 2 * U32 * np.abs(before + want_dw), "dw added")
    assert_within(dbias, bias_before + dy64.sum(0), (M + 2) * U32 * np.abs(dy64).sum(0), "dbias added")
    # each alone
    alone = torch.full_like(dw, float("nan")), torch.full((M, K), float("nan"), device=DEV), torch.full_like(dbias, float("nan"))
    rl.radial_linear_i8_bwd(dy, ws, x=x, dw=alone[0])
    rl.radial_linear_i8_bwd(dy, ws, wt_codes=put_codes(*wt)[0], wt_scales=put_codes(*wt)[1], dx=alone[1])
    rl.radial_linear_i8_bwd(dy, ws, dbias=alone[2])
    for got, want, scaled in ((alone[0], want_dw, size_dw), (alone[1], want_dx, size_dx)):
        assert_within(got, want, bound(want, scaled, F32), "alone")
    assert_within(alone[2], dy64.sum(0), M * U32 * np.abs(dy64).sum(0), "dbias alone")


def test_gradients_against_differences():
    """y is linear in x, W and bias but for the codes' rounding: differences of the loss sum(dy y) over steps of one are the gradients.  A code is off by
    at most half a scale on either side, which bounds the gradients' distance from those of the product without codes."""
    M, N, K = 40, 70, 90
    x, w, bias, dy = _linear(M, N, K, F32, 53)
    x64, dy64, w64 = to64(x), to64(dy), w.astype(np.float64)

    def loss(x, w, b):
        return (dy64 * (x @ w.T + b)).sum()

    base = loss(x64, w64, bias)
    g = np.random.default_rng(54)
    wt = os_.quantize_rows(np.ascontiguousarray(w.T))
    dx, dw, dbias = torch.empty((M, K), device=DEV), torch.empty((N, K), device=DEV), torch.empty(N, device=DEV)
    rl.radial_linear_i8_bwd(dy, workspace(rl.radial_linear_i8_bwd_workspace(M, N, K)), x=x, wt_codes=put_codes(*wt)[0], wt_scales=put_codes(*wt)[1], dx=dx, dw=dw, dbias=dbias)
    half = lambda m, axis: np.abs(m).max(axis, keepdims=True) / 127 / 2 * 1.001  # noqa: E731
    off_dx = half(dy64, 1) * np.abs(w64).sum(0) + (np.abs(dy64) + half(dy64, 1)).sum(1, keepdims=True) * half(w64, 0)
    off_dw = (half(dy64, 0).T * np.abs(x64).sum(0)) + (np.abs(dy64) + half(dy64, 0)).sum(0)[:, None] * half(x64, 0)
    for _ in range(20):
        m, n, k = g.integers(M), g.integers(N), g.integers(K)
        step = np.zeros_like(x64); step[m, k] = 1  # noqa: E702
        assert abs(loss(x64 + step, w64, bias) - base - float(dx[m, k])) <= off_dx[m, k] + 1e-9
        step = np.zeros_like(w64); step[n, k] = 1  # noqa: E702
        assert abs(loss(x64, w64 + step, bias) - base - float(dw[n, k])) <= off_dw[n, k] + 1e-9
        step = np.zeros(N); step[n] = 1  # noqa: E702
        assert abs(loss(x64, w64, bias + step) - base - float(dbias[n])) <= 1e-6


def _pass(s, stream=None):
    rl.radial_linear_i8_fwd(s["x"], s["wc"], s["ws"], s["y"], s["work"], bias=s["bias"], stream=stream)
    rl.radial_linear_i8_bwd(s["dy"], s["work_bwd"], x=s["x"], wt_codes=s["wtc"], wt_scales=s["wts"], dx=s["dx"], dw=s["dw"], dbias=s["db"], stream=stream)


def _state(M, N, K, seed):
    x, w, bias, dy = _linear(M, N, K, BF16, seed)
    (wc, ws), (wtc, wts) = put_codes(*os_.quantize_rows(w)), put_codes(*os_.quantize_rows(np.ascontiguousarray(w.T)))
    return dict(x=x, dy=dy, wc=wc, ws=ws, wtc=wtc, wts=wts, bias=torch.tensor(bias, device=DEV), y=torch.empty((M, N), dtype=BF16, device=DEV),
                dx=torch.empty((M, K), dtype=BF16, device=DEV), dw=torch.empty((N, K), device=DEV), db=torch.empty(N, device=DEV),
                work=workspace(rl.radial_linear_i8_fwd_workspace(M, N, K)), work_bwd=workspace(rl.radial_linear_i8_bwd_workspace(M, N, K)))


RESULTS, WRITTEN = ("y", "dx", "dw", "db"), ("y", "dx", "dw", "db", "work", "work_bwd")


def _clear(s):
    for k in WRITTEN:
        s[k].fill_(255 if s[k].dtype == torch.uint8 else float("nan"))


@pytest.mark.parametrize("by_argument", [True, False], ids=["argument", "current"])
def test_on_a_busy_stream_of_its_own(by_argument):
    s = _state(700, 384, 1000, 55)
    _pass(s)
    want = [s[k].clone() for k in RESULTS]
    busy = torch.zeros(1 << 28, device=DEV)
    _clear(s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(30):
            busy.add_(1.0)
        _clear(s)
        if not by_argument:
            _pass(s)
    if by_argument:
        _pass(s, stream=side)
    side.synchronize()
    assert all(torch.equal(s[k], w) for k, w in zip(RESULTS, want))


def test_captured_and_replayed():
    """Two graphs that share their workspaces, replayed in turn with eager work between, on inputs that change in place."""
    states = [_state(2, 640, 1000, 56), _state(300, 640, 1000, 57)]
    for k in ("work", "work_bwd"):
        states[0][k] = states[1][k]
    graphs = []
    for s in states:
        _pass(s)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            _pass(s)
        graphs.append(graph)
    for turn in range(4):
        for s, graph in zip(states, graphs):
            s["x"].mul_(1.1).add_(0.01 * turn)
            _pass(s)
            want = [s[k].clone() for k in RESULTS]
            _clear(s)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(s[k], w) for k, w in zip(RESULTS, want)), turn
