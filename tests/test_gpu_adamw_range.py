"""AdamW where float32 is left or nearly so: gradients whose squares overflow or lie below the normal numbers, states of one block that are far apart, decays far below a weight's last
bit, numbers of steps below 1 (run with -m gpu).

Bounds.  u = 2^-24.  m and v are float32 operations one by one, whose bits numpy gives; from them on, in 64 bits: the root u, its product with a constant 2u, the sum with eps u; the inverse one unit,
2u; the products with m and with c, and c's own rounding, 3u: c m/d is off by 9u of itself (12u are allowed).  The decay's share of the weight is off by 2u of itself, the sum and the difference by u each."""
import numpy as np
import pytest
import torch

from layer_util import DEV, U32, assert_within
from oracle import layer as ol
from oracle import step as os_
from test_gpu_adamw import BETA1, BETA2, BF16, EPS, F32, LR, Group, check

pytestmark = pytest.mark.gpu


def zero_states(group):
    for k in ("m", "v", "ms", "vs"):
        for t in group.views.get(k, ()):
            t.zero_()


def check_from_moments(group, before, after, step, eps, rounding="nearest", seed=0):
    """One tensor: codes and scales equal, weights from the float32 moments."""
    g = before["g"][0].float().numpy()
    if group.coded:
        m0, r0 = (os_.decode(before[k][0].numpy(), before[k + "s"][0].numpy(), np.float32) for k in ("m", "v"))
        v0 = r0 * r0
    else:
        m0, v0 = before["m"][0].numpy(), before["v"][0].numpy()
    m, v = os_.moments(g, m0, v0, BETA1, BETA2)
    assert m.dtype == v.dtype == np.float32 and np.isfinite(v).all()
    if group.coded:
        bits = os_.random_bits(seed, step, 0, len(g)) if rounding == "random" else (None, None)
        for name, value, b, positive in (("m", m, bits[0], False), ("v", np.sqrt(v), bits[1], True)):
            codes, scales = os_.encode(value, b, positive)
            assert np.array_equal(after[name + "s"][0].numpy(), scales), name
            assert np.array_equal(after[name][0].numpy(), codes), (name, (after[name][0].numpy() != codes).sum())
    else:
        assert np.array_equal(after["m"][0].numpy(), m) and np.array_equal(after["v"][0].numpy(), v)
    w, m, v = before["w"][0].double().numpy(), m.astype(np.float64), v.astype(np.float64)
    c, d = LR / (1 - BETA1 ** step), np.sqrt(v / (1 - BETA2 ** step)) + eps
    want = w * (1 - LR * group.decay) - c * m / d
    assert_within(after["w"][0].double().numpy(), want, 12 * U32 * c * np.abs(m) / d + 2 * U32 * (np.abs(w) + np.abs(want)), "w")


@pytest.mark.parametrize("states", ["f32", "8bit", "random"])
@pytest.mark.parametrize("grad", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", [2e19, 1e20, 3e38], ids=str)
def test_a_gradient_whose_square_overflows_leaves_its_weight_but_for_the_decay(size, grad, states):
    """v is infinite, and m over its root 0: the weight is not lost, nor in the next step.  A code of the root says NaN, in its value alone."""
    group = Group([300, 5000], grad=grad, coded=states != "f32", copy=True)
    large = [torch.arange(300) % 7 == 3, torch.arange(5000) > 4990]
    for g, at in zip(group.views["g"], large):
        g[at.to(DEV)] = size
        g[at.to(DEV).nonzero()[0]] = -size
    before = group.read()
    group.step(rounding="random" if states == "random" else "nearest", seed=4)
    after = group.read()
    for i, at in enumerate(large):
        w, got = before["w"][i].double().numpy(), after["w"][i].double().numpy()
        want = w * (1 - LR * group.decay)
        assert_within(got[at], want[at], 2 * U32 * (np.abs(w) + np.abs(want))[at], "w")
        assert np.isfinite(got).all() and (got != want)[~at].any()
        assert torch.equal(after["c"][i], after["w"][i].to(BF16))
        if group.coded:
            v = ol.e4m3_values()[after["v"][i].numpy()]
            assert np.array_equal(np.isnan(v), at.numpy()) and torch.isfinite(after["vs"][i]).all() and torch.isfinite(after["ms"][i]).all()
            assert not np.isnan(ol.e4m3_values()[after["m"][i].numpy()]).any()
        else:
            assert np.array_equal(np.isinf(after["v"][i].numpy()), at.numpy())
    # and stays where it is
    for g, at in zip(group.views["g"], large):
        g[at.to(DEV)] = 1e-3
    group.step(step=8)
    again = group.read()
    for i, at in enumerate(large):
        w = after["w"][i].double().numpy()
        want = w * (1 - LR * group.decay)
        got = again["w"][i].double().numpy()
        assert_within(got[at], want[at], 2 * U32 * (np.abs(w) + np.abs(want))[at], "w of the next step")
        assert np.isfinite(got).all()
    assert group.guards_kept()


@pytest.mark.parametrize("states", ["f32", "8bit", "random"])
@pytest.mark.parametrize("eps", [1e-8, 1e-20, 1e-30, 2e-38], ids=str)
@pytest.mark.parametrize("size", [1e-14, 1e-16, 1e-17, 1e-18, 1e-19, 1e-20, 1e-21], ids=str)
def test_gradients_whose_squares_are_hardly_there(size, eps, states):
    """v below the normal numbers of float32, down to its smallest and to nothing: its root is that of the v there is.  Two steps, the second from the states of the first."""
    group, rounding = Group([300], coded=states != "f32"), "random" if states == "random" else "nearest"
    zero_states(group)
    group.views["g"][0].copy_(torch.linspace(-size, size, 300))
    for step in (1, 2):
        before = group.read()
        group.step(step=step, eps=eps, rounding=rounding, seed=11)
        check_from_moments(group, before, group.read(), step, eps, rounding, 11)
    assert group.guards_kept()


@pytest.mark.parametrize("rounding", ["nearest", "random"])
@pytest.mark.parametrize("largest", [1e4, 1e12, 1e18, 1.5e19], ids=str)
def test_the_smallest_root_of_a_block_keeps_the_smallest_code(largest, rounding):
    """Beside a root up to 2^138 times as large, too: only what is nothing becomes 0."""
    group = Group([256], coded=True)
    zero_states(group)
    group.views["g"][0].copy_(torch.tensor(np.geomspace(1e-21, 1e-10, 256)))
    group.views["g"][0][5] = group.views["g"][0][200] = largest
    group.views["g"][0][9] = 0
    before = group.read()
    group.step(step=1, rounding=rounding, seed=12)
    after = group.read()
    codes = after["v"][0].numpy()
    assert codes[9] == 0 and (np.delete(codes, 9) >= 1).all()
    check_from_moments(group, before, after, 1, EPS, rounding, 12)


@pytest.mark.parametrize("from_device", [False, True], ids=["host", "device"])
@pytest.mark.parametrize("states", ["f32", "8bit"])
@pytest.mark.parametrize("by", [1e-6, 1e-7, 1e-8, 2e-9], ids=str)
def test_a_small_decay_is_right_on_average(by, states, from_device):
    """Weights of [1/2, 1) whose last bit is 2^-24, updates many times that: a decay of lr decay = `by` is lost in each but not in their mean.  The difference's rounding is spread evenly over 2^-24, a variance of
    2^-48/12, and what is rounded before it 4u of the update and of the decay; five standard deviations."""
    n, lr = 1 << 20, 1e-4
    group = Group([n], coded=states == "8bit", decay=by / lr)
    group.views["w"][0].copy_(torch.linspace(0.5, 1.0, n + 1)[:-1])
    before = group.read()
    if from_device:
        group.step(lr=0.0, lr_at=torch.tensor([lr], device=DEV), step=1000)
        lr = float(np.float32(lr))
    else:
        group.step(lr=lr, step=1000)
    after = group.read()
    g = before["g"][0].numpy()
    if group.coded:
        m0, r0 = (os_.decode(before[k][0].numpy(), before[k + "s"][0].numpy(), np.float32) for k in ("m", "v"))
        m, v = os_.moments(g, m0, r0 * r0, BETA1, BETA2)
    else:
        m, v = os_.moments(g, before["m"][0].numpy(), before["v"][0].numpy(), BETA1, BETA2)
    w = before["w"][0].double().numpy()
    want = os_.update(w, m.astype(np.float64), v.astype(np.float64), lr, 1000, BETA1, BETA2, EPS, by / lr if not from_device else float(np.float32(by / 1e-4)))
    moved, update = after["w"][0].double().numpy() - w, want - w + by * w
    share = (moved - update).mean() / -(by * w).mean()   # of the decay
    off = 5 * 2.0 ** -24 / np.sqrt(12 * n) + (4 + 12 * from_device) * U32 * (np.abs(update).mean() + by)
    assert np.abs(update).mean() > 2.0 ** -17 and off < 0.1 * by
    assert abs((after["w"][0].double().numpy() - want).mean()) <= off, share


@pytest.mark.parametrize("decay", [0.0, 0.1])
def test_weights_that_are_not_finite_stay_what_they_are(decay):
    group = Group([300], decay=decay)
    inf = float("inf")
    group.views["w"][0][:3] = torch.tensor([inf, -inf, float("nan")])
    group.step()
    w = group.read()["w"][0]
    assert w[0] == inf and w[1] == -inf and w[2].isnan() and torch.isfinite(w[3:]).all()


@pytest.mark.parametrize("number", [1, 0, -5, -(1 << 40)], ids=str)
def test_a_number_below_1_draws_the_bits_of_the_first_step(number):
    t = torch.tensor([number], device=DEV)
    group = Group([300, 4100], coded=True)
    before = group.read()
    group.step(step=0, step_at=t, rounding="random", seed=21)
    check(group, before, group.read(), step=1, rounding="random", seed=21, more=6 * U32)
