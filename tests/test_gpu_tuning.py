"""A tuning step of the attention half of a layer, as a program runs it: projections in 8-bit integers, gradients, their norm, AdamW with states in 8 bits, the weights' new codes;
every new operator against the oracle on the step's own inputs, and the whole step captured (run with -m gpu)."""
import json
import os
import sys
import types

import numpy as np
import pytest
import torch

from layer_util import DEV, U32, assert_within, to64
from oracle import step as os_
from paper_2506_19852_amd import binding as rb
from paper_2506_19852_amd import layer as rl
from test_gpu_layer import EPS, Layer
from test_gpu_linear_i8 import bound

pytestmark = pytest.mark.gpu
BF16, F32, U8 = torch.bfloat16, torch.float32, torch.uint8
LR, DECAY, MAX_NORM, SEED = 1e-3, 0.1, 0.05, 77


class Tuned(Layer):
    """The layer with float32 weights and biases that a step changes, projections in 8-bit integers."""

    def __init__(self, seed, **kw):
        super().__init__(seed, **kw)
        N, nan = self.N, float("nan")
        full = lambda *shape, dtype=F32: torch.full(shape, 85 if dtype in (torch.int8, U8) else nan, dtype=dtype, device=DEV)  # noqa: E731
        self.w = {k: w.float() for k, w in self.w.items()}
        self.b = {k: torch.linspace(-0.1, 0.1, len(w), device=DEV) for k, w in self.w.items()}
        self.dw, self.db = {k: full(*w.shape) for k, w in self.w.items()}, {k: full(len(w)) for k, w in self.w.items()}
        self.i8, self.ws_fwd, self.ws_bwd, self.ws_q = {}, {}, {}, {}
        for k, (rows, cols) in ((k, w.shape) for k, w in self.w.items()):
            self.i8[k] = (full(rows, -(-cols // 128) * 128, dtype=torch.int8), full(rows), full(cols, -(-rows // 128) * 128, dtype=torch.int8), full(cols))
            self.ws_fwd[k], self.ws_bwd[k] = full(rl.radial_linear_i8_fwd_workspace(N, rows, cols), dtype=U8), full(rl.radial_linear_i8_bwd_workspace(N, rows, cols), dtype=U8)
            self.ws_q[k] = full(rl.radial_quantize_rows_i8_workspace(rows, cols), dtype=U8)
        weights = [t for k in self.w for t in (self.w[k], self.b[k])]
        zeros = lambda block, dtype: [torch.zeros(-(-t.numel() // block), dtype=dtype, device=DEV) for t in weights]  # noqa: E731
        self.states = dict(firsts=zeros(1, U8), seconds=zeros(1, U8), first_scales=zeros(128, F32), second_scales=zeros(128, F32))
        self.weights, self.grads = weights, [t for k in self.w for t in (self.dw[k], self.db[k])]
        self.decays = [DECAY, 0.0] * len(self.w)
        tensors = rl.adamw_tensors(weights, self.grads, **self.states, decay=self.decays)
        self.plan = rl.radial_adamw_plan(tensors)
        self.adamw = torch.empty(self.plan.table_bytes, dtype=U8, device=DEV)
        rl.radial_adamw_table(tensors, self.plan, self.adamw)
        self.norm, self.ws_norm = full(2), full(rl.radial_grad_norm_workspace(self.plan), dtype=U8)
        self.count = torch.zeros(1, dtype=torch.int64, device=DEV)
        self.encode()

    def encode(self):
        for k, w in self.w.items():
            rl.radial_quantize_rows_i8(w, *self.i8[k], self.ws_q[k])

    def project(self, k, x, y):
        rl.radial_linear_i8_fwd(x, *self.i8[k][:2], y, self.ws_fwd[k], bias=self.b[k])

    def gradients(self, k, dy, x, dx):
        rl.radial_linear_i8_bwd(dy, self.ws_bwd[k], x=x, wt_codes=self.i8[k][2], wt_scales=self.i8[k][3], dx=dx, dw=self.dw[k], dbias=self.db[k])

    def forward(self):
        m, C, N = self.mod, self.C, self.N
        rl.radial_norm_fwd(self.x, None, self.h, scale=m[:, :, 0], shift=m[:, :, 1], eps=EPS)
        self.project("qkv", self.h[0], self.qkv.view(N, 3 * C))
        rl.radial_rope_fwd(self.params, self.table, self.heads(self.qkv, 0), self.q, self.heads(self.qkv, 1), self.k)
        rb.radial_attn_fwd(self.q, self.k, self.heads(self.qkv, 2), self.tokens(self.attn), self.lse, self.mask, self.D ** -0.5)
        self.project("out", self.attn[0], self.o[0])
        rl.radial_norm_fwd(self.x, self.r, self.z, y=self.o, gate=m[:, :, 2], scale=m[:, :, 3], shift=m[:, :, 4], eps=EPS)

    def backward(self):
        m, d, C, N = self.mod, self.dmod, self.C, self.N
        rl.radial_norm_bwd(self.r, self.dz, self.dx, self.ws, dr=self.dr, y=self.o, dy=self.do, gate=m[:, :, 2], scale=m[:, :, 3], dgate=d[:, :, 2], dscale=d[:, :, 3],
                           dshift=d[:, :, 4], eps=EPS)
        self.gradients("out", self.do[0], self.attn[0], self.dattn[0])
        rb.radial_attn_bwd(self.q, self.k, self.heads(self.qkv, 2), self.tokens(self.attn), self.tokens(self.dattn), self.lse, self.dq, self.dk, self.heads(self.dqkv, 2), self.mask,
                           self.D ** -0.5, self.ws_attn)
        rl.radial_rope_bwd(self.params, self.table, self.dq, self.heads(self.dqkv, 0), self.dk, self.heads(self.dqkv, 1))
        self.gradients("qkv", self.dqkv.view(N, 3 * C), self.h[0], self.dh[0])
        rl.radial_norm_bwd(self.x, self.dh, self.da, self.ws, dr=self.dx, scale=m[:, :, 0], dscale=d[:, :, 0], dshift=d[:, :, 1], eps=EPS)

    def update(self):
        self.count.add_(1)
        rl.radial_grad_norm(self.plan, self.adamw, self.norm, self.ws_norm, max_norm=MAX_NORM)
        rl.radial_adamw_step(self.plan, self.adamw, lr=LR, step_at=self.count, factor=self.norm, rounding="random", seed=SEED)
        self.encode()

    def step(self):
        self.forward()
        self.backward()
        self.update()

    def kept(self):
        lists = [self.weights, self.grads, *self.states.values(), *self.i8.values(), (self.z, self.da, self.norm, self.dmod[:, :, :5])]
        return [t.clone() for ts in lists for t in ts]


def _f32(t):
    return np.ascontiguousarray(t.float().cpu().numpy())


def test_two_steps_of_a_layer():
    """Every new operator against the oracle on the step's own inputs."""
    L = Tuned(1)
    N, C = L.N, L.C
    for t in (1, 2):
        before = {k: v.clone() for k, v in L.w.items()}
        i8 = {k: [x.cpu().numpy() for x in v] for k, v in L.i8.items()}
        bias = {k: to64(v) for k, v in L.b.items()}
        for k, w in before.items():
            for (codes, scales), m in ((i8[k][:2], _f32(w)), (i8[k][2:], _f32(w.t()))):
                want = os_.quantize_rows(m)
                assert np.array_equal(codes, want[0]) and np.array_equal(scales, want[1])
        L.forward()
        L.backward()
        torch.cuda.synchronize()
        for k, x, y in (("qkv", L.h[0], L.qkv.view(N, 3 * C)), ("out", L.attn[0], L.o[0])):
            want, size = os_.product(*os_.quantize_rows(_f32(x)), *i8[k][:2], bias[k])
            assert_within(y, want, bound(want, size, BF16), k)
        for k, dy, x, dx in (("out", L.do[0], L.attn[0], L.dattn[0]), ("qkv", L.dqkv.view(N, 3 * C), L.h[0], L.dh[0])):
            want, size = os_.product(*os_.quantize_rows(_f32(dy)), *i8[k][2:])
            assert_within(dx, want, bound(want, size, BF16), "dx of " + k)
            want, size = os_.product(*os_.quantize_rows(_f32(dy.t())), *os_.quantize_rows(_f32(x.t())))
            assert_within(L.dw[k], want, bound(want, size, F32), "dw of " + k)
            assert_within(L.db[k], to64(dy).sum(0), N * U32 * np.abs(to64(dy)).sum(0), "db of " + k)
        old = [[x.cpu().numpy().copy() for x in v] for v in L.states.values()]
        weights = [to64(x) for x in L.weights]
        L.update()
        torch.cuda.synchronize()
        length = np.sqrt(sum(float((g.double() ** 2).sum()) for g in L.grads))
        norm, factor = L.norm.cpu().numpy()
        assert length > MAX_NORM and abs(norm - length) <= 2 * U32 * length and abs(factor * length / MAX_NORM - 1) <= 3 * U32
        for i, (w, g) in enumerate(zip(weights, L.grads)):
            x = _f32(g).ravel() * factor
            m0, r0 = os_.decode(old[0][i], old[2][i], np.float32), os_.decode(old[1][i], old[3][i], np.float32)
            m1, v1 = os_.moments(x, m0, r0 * r0, 0.9, 0.999)
            bits = os_.random_bits(SEED, t, i, len(x))
            for k, value, b, positive in (("first", m1, bits[0], False), ("second", np.sqrt(v1), bits[1], True)):
                codes, scales = os_.encode(value, b, positive)
                assert np.array_equal(L.states[k + "s"][i].cpu().numpy(), codes) and np.array_equal(L.states[k + "_scales"][i].cpu().numpy(), scales), (k, i)
            m, v = os_.moments(x.astype(np.float64), m0.astype(np.float64), np.square(r0.astype(np.float64)), 0.9, 0.999)
            want = os_.update(w.ravel(), m, v, LR, t, 0.9, 0.999, 1e-8, L.decays[i])
            # the bounds of test_gpu_adamw.py, with the step's number from the device
            c, d = LR / (1 - 0.9 ** t), np.sqrt(v / (1 - 0.999 ** t)) + 1e-8
            em = 6 * U32 * (np.abs(0.9 * m0) + np.abs(0.1 * x))
            assert_within(to64(L.weights[i]).ravel(), want, c / d * (em + 24 * U32 * np.abs(m)) + 3 * U32 * np.abs(w.ravel()) + U32 * np.abs(want), f"weight {i}")


def test_whole_steps_captured_and_replayed():
    """Every replay is the eager step of its number, also with another layer's work between."""
    graphed, eager, other = Tuned(2), Tuned(2), Tuned(3, frames=3)
    other.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.step()
    for turn in range(4):
        for L in (graphed, eager):
            L.x.mul_(1.05)
        graph.replay()
        other.step()
        eager.step()
        torch.cuda.synchronize()
        assert int(graphed.count) == int(eager.count) == turn + 1
        assert all(torch.equal(a, b) for a, b in zip(graphed.kept(), eager.kept())), turn
        assert all(torch.isfinite(t).all() for t in graphed.weights)


def test_the_benchmark_times_a_tuning_step(capsys):
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    import bench
    from paper_2506_19852_amd import workloads as wl
    bench.layer_step_times(wl.WORKLOADS["cfg1_tiny"], types.SimpleNamespace(warmup=1, steps=2))
    line = json.loads(capsys.readouterr().out.strip().split("\n")[-1])
    assert line["unit"] == "ms" and line["steps"] == 2 and len(line["ms"]) == 15 and all(t > 0 for t in line["ms"].values())
    assert line["value"] == pytest.approx(sum(line["ms"].values()), rel=1e-2)
