"""8-bit integer products at the sizes of training: gradients of matrices that go through their passes one after the other, columns of many slabs, matrices of more than 2^31 values (run
with -m gpu)."""
import numpy as np
import pytest
import torch

from layer_util import DEV, U32, assert_within, inside, surroundings_kept, to64
from oracle import step as os_
from paper_2506_19852_amd import layer as rl
from test_gpu_linear_i8 import BF16, F32, bound, buffers, put_codes, workspace

pytestmark = pytest.mark.gpu

# M, N, K: dy and x of more than 128 MiB together, so that each is read in launches of its own; dx of the first and dw of the second leave rows over that take a launch more
LONG = [(6100, 4096, 3000), (4096, 6000, 3000)]


@pytest.mark.parametrize("size", LONG, ids=str)
def test_gradients_of_long_inputs(size):
    M, N, K = size
    g = np.random.default_rng(61)
    x, _ = inside((g.normal(size=(M, K)) * np.exp(g.normal(size=K))).astype(np.float32), F32, 4)
    dy, _ = inside((g.normal(size=(M, N)) * 0.02).astype(np.float32), F32, 4)
    assert (x.numel() + dy.numel()) * 4 > 128 << 20
    x32, dy32 = x.cpu().numpy(), dy.cpu().numpy()
    wt = os_.quantize_rows((g.normal(size=(K, N)) * K ** -0.5).astype(np.float32))
    dx, dx_whole = inside(np.full((M, K), np.nan, np.float32), F32, 3)
    dw, dw_whole = inside(np.full((N, K), np.nan, np.float32), F32, 8)
    dbias = torch.full((N,), float("nan"), device=DEV)
    wt_codes, wt_scales = put_codes(*wt)
    rl.radial_linear_i8_bwd(dy, workspace(rl.radial_linear_i8_bwd_workspace(M, N, K)), x=x, wt_codes=wt_codes, wt_scales=wt_scales, dx=dx, dw=dw, dbias=dbias)
    want, scaled = os_.product(*os_.quantize_rows(dy32), *wt)
    assert_within(dx, want, bound(want, scaled, F32), "dx")
    want, scaled = os_.product(*os_.quantize_rows(np.ascontiguousarray(dy32.T)), *os_.quantize_rows(np.ascontiguousarray(x32.T)))
    assert_within(dw, want, bound(want, scaled, F32), "dw")
    dy64 = dy32.astype(np.float64)
    assert_within(dbias, dy64.sum(0), 61 * U32 * np.abs(dy64).sum(0), "dbias")   # M/(4 slabs) + 4 + slabs/2 + 1 additions one after the other, 42 to 64 slabs: at most 61
    assert surroundings_kept(dx, dx_whole) and surroundings_kept(dw, dw_whole)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", [(32760, 16), (32760, 64), (16400, 333), (9001, 600), (5000, 1500)], ids=str)
def test_columns_of_many_slabs(shape, dtype):
    """Up to 512 slabs of the rows."""
    rows, cols = shape
    g = np.random.default_rng(62)
    x, whole = inside(g.normal(size=shape) * np.exp(g.normal(size=(rows, 1)) * 2), dtype, 5)
    a = x.float().cpu().numpy()
    for both in (True, False):
        straight, turned, total = buffers(rows, cols), buffers(cols, rows), torch.full((cols,), float("nan"), device=DEV)
        rl.radial_quantize_rows_i8(x, *(straight if both else (None, None)), *turned, workspace(rl.radial_quantize_rows_i8_workspace(rows, cols)), sums_t=total)
        for (codes, scales), m in ((straight, a), (turned, np.ascontiguousarray(a.T)))[not both:]:
            want_codes, want_scales = os_.quantize_rows(m)
            assert np.array_equal(scales.cpu().numpy(), want_scales) and np.array_equal(codes.cpu().numpy(), want_codes)
        a64 = a.astype(np.float64)
        assert_within(total, a64.sum(0), 300 * U32 * np.abs(a64).sum(0), "sums")   # 16 + 4 + 256 + 1 additions one after the other with 512 slabs
    assert surroundings_kept(x, whole)


def test_columns_of_more_than_2_to_the_31_values():
    """Values on both sides of 2^31 elements and at the ends, both ways; 10 GB."""
    rows, cols = 70_001, 32_768
    x = torch.zeros((rows, cols), dtype=BF16, device=DEV)
    edge = (1 << 31) // cols   # the first row behind 2^31 values
    put = {(0, 0): 1.0, (edge - 1, cols - 1): 2.0, (edge, 0): 4.0, (edge, 777): -3.0, (rows - 1, 777): 1.5, (rows - 1, cols - 1): -8.0, (40_000, 5): 0.5}
    for (r, c), v in put.items():
        x[r, c] = v
    codes, scales = torch.full((rows, cols), 77, dtype=torch.int8, device=DEV), torch.full((rows,), float("nan"), device=DEV)
    padded = -(-rows // 128) * 128
    codes_t, scales_t = torch.full((cols, padded), 77, dtype=torch.int8, device=DEV), torch.full((cols,), float("nan"), device=DEV)
    total = torch.full((cols,), float("nan"), device=DEV)
    rl.radial_quantize_rows_i8(x, codes, scales, codes_t, scales_t, workspace(rl.radial_quantize_rows_i8_workspace(rows, cols)), sums_t=total)
    for got, found, turned in ((codes, scales, False), (codes_t, scales_t, True)):
        lines = {}
        for (r, c), v in put.items():
            lines.setdefault(c if turned else r, {})[r if turned else c] = v
        assert int(got.count_nonzero()) == len(put)
        assert int((found != 2.0 ** -126).sum()) == len(lines)
        for line, values in lines.items():
            want = np.float32(max(abs(v) for v in values.values())) / np.float32(127)
            assert float(found[line]) == want
            for at, v in values.items():
                assert int(got[line, at]) == int(np.rint(np.float32(v) / want)), (line, at)
    sums = np.zeros(cols)
    for (_, c), v in put.items():
        sums[c] += v
    assert np.array_equal(to64(total), sums)
