"""The float64 definitions of the layer operators against differences, a library and facts that hold for any implementation (CPU)."""
import numpy as np
import pytest
import torch

from oracle import layer as ol

RNG = np.random.default_rng


def _case(seed, B=2, N=7, C=6, group=3):
    g = RNG(seed)
    G = -(-N // group)
    r = lambda *s: g.normal(size=s)  # noqa: E731
    return dict(x=r(B, N, C), y=r(B, N, C), gate=r(B, G, C), post_weight=r(C), weight=r(C), scale=r(B, G, C), shift=r(B, G, C)), r(B, N, C), r(B, N, C)


@pytest.mark.parametrize("post", [ol.NONE, ol.LAYER, ol.RMS])
@pytest.mark.parametrize("pre", [ol.NONE, ol.LAYER, ol.RMS])
def test_gradients_of_the_norms_are_their_differences(post, pre):
    t, dr, dz = _case(3)
    if post == ol.NONE:
        t["post_weight"] = None
    if pre == ol.NONE:
        dz = None
        for k in ("weight", "scale", "shift"):
            t[k] = None
    kw = dict(group=3, post=post, pre=pre, residual_scale=0.7, eps=1e-3)

    def loss(**change):
        r, z = ol.norm_fwd(**{**t, **change}, **kw)
        return (r * dr).sum() + (0.0 if z is None else (z * dz).sum())

    r, _ = ol.norm_fwd(**t, **kw)
    shift = t.pop("shift")
    got = ol.norm_bwd(r, dz, dr, **{k: v for k, v in t.items() if k != "x"}, **kw)
    t["shift"] = shift
    h = 1e-5
    for name, v in t.items():
        if v is None:
            continue
        for at in list(np.ndindex(v.shape))[::5]:
            up, down = v.copy(), v.copy()
            up[at] += h
            down[at] -= h
            want = (loss(**{name: up}) - loss(**{name: down})) / (2 * h)
            # a central difference is off by h^2 times the third derivative and by 2^-52 loss / h
            assert abs(got["d" + name][at] - want) < 1e-5 * (1 + abs(want)), (name, at)


def test_layer_norm_is_the_library_s():
    t, _, _ = _case(4)
    _, z = ol.norm_fwd(t["x"], weight=t["weight"], group=7, eps=1e-5)
    want = torch.nn.functional.layer_norm(torch.tensor(t["x"]), (6,), torch.tensor(t["weight"]), None, 1e-5)
    assert np.abs(z - want.numpy()).max() < 1e-12


@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_turns_depend_on_distances_alone_and_keep_lengths(layout):
    g = RNG(5)
    f = [ol.frequencies(6), ol.frequencies(4, scaling="linear", factor=2.0)]
    q, k = g.normal(size=(1, 1, 1, 12)), g.normal(size=(1, 1, 1, 12))
    at = lambda x, i, j: ol.rope(x, np.array([[i * 30 + j]]), [20, 30], f, layout)  # noqa: E731
    a = (at(q, 3, 5) * at(k, 7, 11)).sum()
    b = (at(q, 13, 12) * at(k, 17, 18)).sum()
    assert abs(a - b) < 1e-12
    assert abs(np.linalg.norm(at(q, 19, 29)) - np.linalg.norm(q)) < 1e-12
    assert np.array_equal(at(q, 9, 9)[..., 10:], q[..., 10:])
    # the gradient is the transpose: <rope(q), k> = <q, gradient(k)>
    i = np.array([[77]])
    left = (ol.rope(q, i, [20, 30], f, layout, 1.3) * k).sum()
    assert abs(left - (q * ol.rope(k, i, [20, 30], f, layout, 1.3, gradient=True)).sum()) < 1e-12


def test_scalings():
    plain, base = ol.frequencies(64), ol.frequencies(64, scaling="base", factor=8.0)
    assert base[0] == plain[0] == 1.0 and abs(base[-1] * 8.0 / plain[-1] - 1) < 1e-12
    parts = ol.frequencies(64, scaling="parts", factor=8.0, original=4096)
    turns = 4096 * plain / (2 * np.pi)
    assert np.array_equal(parts[turns > 32], plain[turns > 32]) and np.allclose(parts[turns < 1] * 8, plain[turns < 1])
    assert (np.diff(parts) < 0).all()


def test_codes_are_nearest_and_ties_go_to_even():
    v = ol.e4m3_values()
    assert v[0x7e] == 448.0 and v[1] == 2.0 ** -9
    pos = v[:127]
    assert np.array_equal(ol.e4m3_codes(pos), np.arange(127)) and np.array_equal(ol.e4m3_codes(-pos[1:]), np.arange(129, 255))
    middle = (pos[1:] + pos[:-1]) / 2
    assert (ol.e4m3_codes(middle) % 2 == 0).all()
    x = RNG(6).normal(size=5000) * np.exp(RNG(7).normal(size=5000) * 3)
    x = x[np.abs(x) <= 448]
    want = torch.tensor(x, dtype=torch.float32).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ol.e4m3_codes(x.astype(np.float32)), want)


@pytest.mark.parametrize("blocks", [False, True])
def test_quantised_values_are_within_half_a_step(blocks):
    x = RNG(8).normal(size=(200, 300)).astype(np.float32)
    codes, scales = ol.quantize(x, blocks)
    assert codes.shape == (200, 384) and scales.shape == (3, 2 if blocks else 200) and not codes[:, 300:].any()
    got = ol.values(codes, scales, blocks)[:, :300]
    each = np.repeat(np.repeat(scales.T, 128, 0)[:200] if blocks else scales.T, 128, 1)[:, :300]
    assert (np.abs(got - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * each) * (1 + 1e-6)).all()
