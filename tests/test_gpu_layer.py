"""The operators together, as a layer calls them: norm, projection of q, k, v, rotary positions, block-sparse attention, output projection, gated
residual and norm, and back; on another stream and in a HIP graph (run with -m gpu)."""
import numpy as np
import pytest
import torch

from layer_util import DEV, HALF_STEP, U32, assert_within, to64
from oracle import layer as ol
from paper_2506_19852_amd import binding as rb
from paper_2506_19852_amd import layer as rl
from test_gpu_product import _bound

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
EPS = 1e-6


class Layer:
    """Attention half of a layer of a video model: buffers and weights are allocated once; `forward` and `backward` only call the library."""

    def __init__(self, seed, frames=4, grid_h=8, grid_w=10, H=3, D=64, text=7):
        g = torch.Generator(device=DEV).manual_seed(seed)
        s = grid_h * grid_w
        self.N, self.H, self.D, self.C = frames * s + text, H, D, H * D
        N, C = self.N, self.C
        new = lambda *shape, dtype=BF16: torch.full(shape, float("nan"), dtype=dtype, device=DEV)  # noqa: E731
        rand = lambda *shape, size=1.0, dtype=BF16: (torch.randn(shape, device=DEV, generator=g) * size).to(dtype)  # noqa: E731
        self.x, self.dr, self.dz = rand(1, N, C), rand(1, N, C), rand(1, N, C)
        self.mod = rand(1, 1, 6, C, size=0.3, dtype=F32)
        self.w = {"qkv": rand(3 * C, C, size=C ** -0.5), "out": rand(C, C, size=C ** -0.5)}
        self.q8 = {}
        for k, w in self.w.items():
            self.q8[k], self.q8[k + "_t"] = self.codes(*w.shape, True), self.codes(*w.shape[::-1], True)
            rl.radial_quantize_groups_fp8(w, *self.q8[k], *self.q8[k + "_t"], grouping=rl.RADIAL_BLOCKS)
        self.params = rl.rope_params([frames, grid_h, grid_w], [16, 24, 24], scaling=["linear", "none", "none"], factor=[2.0, 1.0, 1.0])
        self.table = torch.empty(rl.radial_rope_table_bytes(self.params) // 4, device=DEV)
        rl.radial_rope_table(self.params, self.table)
        self.mask = rb.radial_mask_build(frames, s, 64, 1, rb.RADIAL_MASK_TRANSPOSE, extra_tokens=text)
        for k in ("h", "o", "z", "r", "attn", "dh", "do", "dx", "dattn", "da"):
            setattr(self, k, new(1, N, C))
        self.qkv, self.dqkv = new(N, 3, H, D), new(N, 3, H, D)
        self.q, self.k, self.dq, self.dk = (new(1, H, N, D) for _ in range(4))
        self.lse = new(1, H, N, dtype=F32)
        self.dmod = new(1, 1, 6, C, dtype=F32)
        self.dw = {k: new(*w.shape) for k, w in self.w.items()}
        self.act = {k: self.codes(N, c) for k, c in (("h", C), ("attn", C), ("do", C), ("dqkv", 3 * C))}
        self.act_t = {k: self.codes(c, N) for k, c in (("h", C), ("attn", C), ("do", C), ("dqkv", 3 * C))}
        self.ws = torch.empty(rl.radial_norm_bwd_workspace(1, N, C), dtype=torch.uint8, device=DEV)
        self.ws_attn = torch.empty(rb.radial_attn_bwd_workspace(1, H, N, D, self.mask), dtype=torch.uint8, device=DEV)

    @staticmethod
    def codes(rows, cols, blocks=False):
        groups = -(-cols // 128)
        return torch.empty((rows, groups * 128), dtype=torch.uint8, device=DEV), torch.empty((groups, -(-rows // 128) if blocks else rows), device=DEV)

    def heads(self, t, i):
        """q, k or v of a projection's output [N, 3, H, D], as [1, H, N, D]."""
        return t[:, i].transpose(0, 1)[None]

    def tokens(self, t):
        """[1, N, C] as the attention's [1, H, N, D]."""
        return t.view(1, self.N, self.H, self.D).transpose(1, 2)

    def forward(self, stream=None):
        m, C, N = self.mod, self.C, self.N
        rl.radial_norm_fwd(self.x, None, self.h, scale=m[:, :, 0], shift=m[:, :, 1], eps=EPS, stream=stream)
        rl.radial_quantize_groups_fp8(self.h[0], *self.act["h"], *self.act_t["h"], stream=stream)
        rl.radial_product_fp8(*self.act["h"], *self.q8["qkv"], self.qkv.view(N, 3 * C), stream=stream)
        rl.radial_rope_fwd(self.params, self.table, self.heads(self.qkv, 0), self.q, self.heads(self.qkv, 1), self.k, stream=stream)
        rb.radial_attn_fwd(self.q, self.k, self.heads(self.qkv, 2), self.tokens(self.attn), self.lse, self.mask, self.D ** -0.5, stream=stream)
        rl.radial_quantize_groups_fp8(self.attn[0], *self.act["attn"], *self.act_t["attn"], stream=stream)
        rl.radial_product_fp8(*self.act["attn"], *self.q8["out"], self.o[0], stream=stream)
        rl.radial_norm_fwd(self.x, self.r, self.z, y=self.o, gate=m[:, :, 2], scale=m[:, :, 3], shift=m[:, :, 4], eps=EPS, stream=stream)

    def backward(self, stream=None):
        m, d, C, N = self.mod, self.dmod, self.C, self.N
        rl.radial_norm_bwd(self.r, self.dz, self.dx, self.ws, dr=self.dr, y=self.o, dy=self.do, gate=m[:, :, 2], scale=m[:, :, 3], dgate=d[:, :, 2],
                           dscale=d[:, :, 3], dshift=d[:, :, 4], eps=EPS, stream=stream)
        rl.radial_quantize_groups_fp8(self.do[0], *self.act["do"], *self.act_t["do"], stream=stream)
        rl.radial_product_fp8(*self.act["do"], *self.q8["out_t"], self.dattn[0], stream=stream)
        rl.radial_product_fp8(*self.act_t["do"], *self.act_t["attn"], self.dw["out"], stream=stream)
        rb.radial_attn_bwd(self.q, self.k, self.heads(self.qkv, 2), self.tokens(self.attn), self.tokens(self.dattn), self.lse, self.dq, self.dk,
                           self.heads(self.dqkv, 2), self.mask, self.D ** -0.5, self.ws_attn, stream=stream)
        rl.radial_rope_bwd(self.params, self.table, self.dq, self.heads(self.dqkv, 0), self.dk, self.heads(self.dqkv, 1), stream=stream)
        rl.radial_quantize_groups_fp8(self.dqkv.view(N, 3 * C), *self.act["dqkv"], *self.act_t["dqkv"], stream=stream)
        rl.radial_product_fp8(*self.act["dqkv"], *self.q8["qkv_t"], self.dh[0], stream=stream)
        rl.radial_product_fp8(*self.act_t["dqkv"], *self.act_t["h"], self.dw["qkv"], stream=stream)
        # the residual's gradient joins that of the norm at the layer's entrance
        rl.radial_norm_bwd(self.x, self.dh, self.da, self.ws, dr=self.dx, scale=m[:, :, 0], dscale=d[:, :, 0], dshift=d[:, :, 1], eps=EPS, stream=stream)

    def results(self):
        kept = [self.h, self.qkv, self.q, self.k, self.attn, self.lse, self.o, self.r, self.z, self.dx, self.do, self.dattn, self.dq, self.dk, self.dqkv, self.dh, self.da,
                self.dw["qkv"], self.dw["out"], *(self.dmod[:, :, i] for i in range(5))]
        return [t.clone() for t in kept]


def _values(m, blocks=False):
    return ol.values(*ol.quantize(np.ascontiguousarray(m, dtype=np.float32), blocks), blocks)


def test_forward_and_backward_of_a_layer():
    """Every step against the oracle on the step's own inputs."""
    L = Layer(1)
    L.forward()
    L.backward()
    torch.cuda.synchronize()
    N, C = L.N, L.C
    index = np.arange(N)[None]
    sizes, freqs = [4, 8, 10], [ol.frequencies(16, scaling="linear", factor=2.0), ol.frequencies(24), ol.frequencies(24)]
    mod = to64(L.mod)

    def near(got, want, size, what, dtype=BF16, units=128):
        assert_within(got, want, HALF_STEP[dtype] * np.abs(want) + units * U32 * size, what)

    _, h = ol.norm_fwd(to64(L.x), scale=mod[:, :, 0], shift=mod[:, :, 1], group=N, eps=EPS)
    near(L.h, h, 4 + 4 * np.abs(h), "h")
    for got, act, w, what in ((L.qkv.view(N, 3 * C), L.h, "qkv", "qkv"), (L.o[0], L.attn, "out", "o")):
        a, b = _values(to64(act)[0]), _values(to64(L.w[w]), True)
        want = a @ b.T
        assert_within(got, want, _bound(a, b, want), what)
    for i, (out, din, dout) in enumerate(((L.q, L.dq, L.dqkv), (L.k, L.dk, L.dqkv))):
        x = to64(L.heads(L.qkv, i))
        near(out, ol.rope(x, index, sizes, freqs, "interleaved"), 4 * np.abs(x).max(), "turned")
        x = to64(din)
        near(L.heads(dout, i), ol.rope(x, index, sizes, freqs, "interleaved", gradient=True), 4 * np.abs(x).max(), "turned back")
    r, z = ol.norm_fwd(to64(L.x), to64(L.o), mod[:, :, 2], scale=mod[:, :, 3], shift=mod[:, :, 4], group=N, eps=EPS)
    near(L.r, r, 4 + np.abs(r), "r")
    near(L.z, z, 4 + 4 * np.abs(z), "z")
    for x, dz, dr, y, got_dx, got_dy, at in ((L.r, L.dz, L.dr, L.o, L.dx, L.do, 2), (L.x, L.dh, L.dx, None, L.da, None, -1)):
        kw = dict(y=to64(y), gate=mod[:, :, 2]) if y is not None else {}
        want = ol.norm_bwd(to64(x), to64(dz), to64(dr), scale=mod[:, :, at + 1], group=N, eps=EPS, **kw)
        large = np.abs(to64(dr)).max() + 4 * np.abs(to64(dz)).max()
        near(got_dx, want["dx"], large, "dx")
        for k, i in (("dscale", at + 1), ("dshift", at + 2)) + ((("dgate", 2),) if y is not None else ()):
            near(L.dmod[:, :, i], want[k], N * large * 4, k, F32, 4)   # N terms, each below 4 * large, added N / 100 at a time
        if y is not None:
            near(got_dy, want["dy"], large, "dy")
    for got, (a, ta), (b, tb, blocks), what in (
            (L.dattn[0], (L.do[0], False), (L.w["out"], True, True), "dattn"), (L.dw["out"], (L.do[0], True), (L.attn[0], True, False), "dW out"),
            (L.dh[0], (L.dqkv.view(N, 3 * C), False), (L.w["qkv"], True, True), "dh"), (L.dw["qkv"], (L.dqkv.view(N, 3 * C), True), (L.h[0], True, False), "dW qkv")):
        a, b = to64(a), to64(b)
        p, q = _values(a.T if ta else a), _values(b.T if tb else b, blocks)
        want = p @ q.T
        assert_within(got, want, _bound(p, q, want), what)


def test_on_a_stream_of_its_own():
    L = Layer(2)
    L.forward(); L.backward()  # noqa: E702
    want = L.results()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for t in (L.h, L.q, L.o, L.z, L.da):
        t.fill_(float("nan"))
    torch.cuda.synchronize()
    L.forward(stream=side)
    with torch.cuda.stream(side):
        L.backward()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(L.results(), want))


def test_captured_and_replayed():
    """Two graphs of layers of their own, replayed in turn with eager work between, on inputs that change in place."""
    layers = [Layer(3), Layer(4, frames=3)]
    graphs = []
    for L in layers:
        L.forward(); L.backward()  # noqa: E702
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            L.forward(); L.backward()  # noqa: E702
        graphs.append(graph)
    other = Layer(5)
    for turn in range(4):
        for L, graph in zip(layers, graphs):
            L.x.mul_(1.1).add_(0.01 * turn)
            L.forward(); L.backward()  # noqa: E702
            want = L.results()
            for t in (L.h, L.q, L.o, L.z, L.da, L.dmod):
                t.fill_(float("nan"))
            other.forward()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(L.results(), want)), turn


def test_the_benchmark_times_a_layer(capsys):
    import json
    import os
    import sys
    import types
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    import bench
    from paper_2506_19852_amd import workloads as wl
    bench.layer_times(wl.WORKLOADS["cfg1_tiny"], types.SimpleNamespace(warmup=1, steps=2))
    line = json.loads(capsys.readouterr().out.strip().split("\n")[-1])
    assert line["unit"] == "ms" and line["steps"] == 2 and len(line["ms"]) == 8 and all(t > 0 for t in line["ms"].values())
    assert line["value"] == pytest.approx(sum(line["ms"].values()), rel=1e-2)


INPUTS = {"x", "dr", "dz", "mod", "w", "q8", "params", "table", "mask"}


def _clear(L):
    """NaN, or bytes of ones, into everything that a pass writes: results, codes, scales and workspaces."""
    def each(v):
        if isinstance(v, torch.Tensor):
            yield v
        elif isinstance(v, (tuple, dict)):
            for part in v.values() if isinstance(v, dict) else v:
                yield from each(part)
    cleared = [t for name, v in vars(L).items() if name not in INPUTS for t in each(v)]
    for t in cleared:
        t.fill_(255 if t.dtype == torch.uint8 else float("nan"))
    return cleared


def test_every_result_is_cleared():
    L = Layer(6)
    L.forward(); L.backward()  # noqa: E702
    assert len(_clear(L)) == 10 + 2 + 4 + 2 + 2 + 16 + 2 and all(r.isnan().all() for r in L.results())


@pytest.mark.parametrize("by_argument", [True, False], ids=["argument", "current"])
def test_every_result_on_a_stream_of_its_own(by_argument):
    """The stream is busy when the calls are made, and everything is cleared behind that work: a launch on another stream comes before its inputs, and its
    results are lost."""
    L = Layer(7)
    L.forward(); L.backward()  # noqa: E702
    want = L.results()
    busy = torch.zeros(1 << 28, device=DEV)
    _clear(L)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(30):
            busy.add_(1.0)
        _clear(L)
        if not by_argument:
            L.forward(); L.backward()  # noqa: E702
    if by_argument:
        L.forward(stream=side)
        L.backward(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(L.results(), want))


def test_every_result_of_a_replay():
    """Each replay alone leaves every result: nothing is left over from the eager pass."""
    layers = [Layer(8), Layer(9, frames=3)]
    graphs = []
    for L in layers:
        L.forward(); L.backward()  # noqa: E702
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            L.forward(); L.backward()  # noqa: E702
        graphs.append(graph)
    other = Layer(10)
    for turn in range(4):
        for L, graph in zip(layers, graphs):
            L.x.mul_(1.1).add_(0.01 * turn)
            L.dz.neg_()
            L.forward(); L.backward()  # noqa: E702
            want = L.results()
            _clear(L)
            other.forward(); other.backward()  # noqa: E702
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(L.results(), want)), turn
