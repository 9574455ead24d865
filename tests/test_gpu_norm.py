"""Gated residual and norms against the float64 oracle (run with -m gpu).

Bounds.  A result is rounded once to its type (half a step).  Before that it is float32 arithmetic on exact inputs, u = 2^-24 per operation
relative to the magnitudes that are added: a row's sums are at most 16 additions in a lane, 6 over lanes and 16 over waves (< 40), a few products
and a square root follow; 64 u times the magnitudes covers a norm's result, 128 u that of two norms in turn.  A sum over the tokens of a group
is at most one operation per token more."""
import numpy as np
import pytest
import torch

from layer_util import DEV, HALF_STEP, U32, assert_within, inside, rounded, surroundings_kept, to64
from oracle import layer as ol
from paper_2506_19852_amd import layer as rl

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
EPS = 1e-5

# B, N, C, group, post, pre, residual type, branch type, first channel's place in a larger row (8: aligned)
CASES = [
    (1, 1, 1, 1, ol.NONE, ol.RMS, BF16, BF16, 8),
    (2, 3, 7, 2, ol.LAYER, ol.LAYER, F32, BF16, 8),
    (1, 5, 8, 5, ol.RMS, ol.LAYER, BF16, BF16, 8),
    (3, 50, 64, 7, ol.NONE, ol.LAYER, BF16, BF16, 8),
    (2, 33, 128, 33, ol.RMS, ol.RMS, F32, F32, 8),
    (1, 40, 200, 1, ol.LAYER, ol.RMS, BF16, F32, 8),
    (2, 9, 256, 4, ol.RMS, ol.LAYER, BF16, BF16, 8),
    (1, 300, 512, 100, ol.NONE, ol.RMS, BF16, BF16, 8),
    (1, 12, 520, 12, ol.LAYER, ol.LAYER, F32, BF16, 8),
    (2, 5, 1000, 3, ol.RMS, ol.RMS, BF16, BF16, 1),
    (1, 70, 1536, 35, ol.NONE, ol.LAYER, BF16, BF16, 8),
    (1, 6, 5120, 6, ol.RMS, ol.LAYER, BF16, BF16, 8),
    (2, 3, 5121, 2, ol.NONE, ol.LAYER, F32, F32, 3),
    (1, 3, 8192, 3, ol.LAYER, ol.RMS, BF16, BF16, 8),
    (1, 3, 8200, 2, ol.RMS, ol.LAYER, F32, BF16, 8),
    (1, 2, 16384, 1, ol.RMS, ol.LAYER, BF16, F32, 8),
    (1, 2, 16383, 2, ol.LAYER, ol.LAYER, BF16, BF16, 8),
]


def _norm_magnitude(v, size, kind):
    """(magnitude of N(v)'s terms, 1 / size): what its float32 error is relative to."""
    if kind == ol.NONE:
        return size, np.ones_like(v[..., :1])
    _, inverse = ol.norm(v, kind, EPS)
    mean = np.abs(v).mean(-1, keepdims=True) if kind == ol.LAYER else 0.0
    n, _ = ol.norm(v, kind, EPS)
    # errors of mean and size move the whole row: |n| (1 + error), (|v| + |mean|) / size from the difference
    return (size + mean) * inverse + np.abs(n), inverse


def _inputs(case, seed, mean=0.0):
    B, N, C, group, post, pre, xt, yt, lead = case
    g = np.random.default_rng(seed)
    G = -(-N // group)
    a = {"x": rounded(g.normal(mean, 1.5, (B, N, C)), xt), "y": rounded(g.normal(mean, 0.8, (B, N, C)), yt)}
    for k in ("gate", "scale", "shift"):
        a[k] = rounded(g.normal(0, 0.4, (B, G, C)), F32)
    a["weight"] = rounded(g.normal(1, 0.2, C), F32)
    if post != ol.NONE:
        a["post_weight"] = rounded(g.normal(1, 0.2, C), F32)
    return a, g


def _mods(a, names, lead):
    """The conditioning as chunks of one tensor [B, G, k, C (+ lead)]."""
    B, G, C = a["gate"].shape
    whole = torch.zeros((B, G, len(names), C + lead), dtype=F32, device=DEV)
    out = {}
    for i, k in enumerate(names):
        out[k] = whole[:, :, i, lead:]
        if k in a:
            out[k].copy_(torch.tensor(a[k]))
    return out


@pytest.mark.parametrize("mean", [0.0, 300.0])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward(case, mean):
    B, N, C, group, post, pre, xt, yt, lead = case
    a, _ = _inputs(case, 11, mean)
    x, _ = inside(a["x"], xt, lead)
    y, _ = inside(a["y"], yt, lead)
    r, r_whole = inside(np.zeros((B, N, C)), xt, lead)
    z, z_whole = inside(np.zeros((B, N, C)), yt, lead)
    t = {k: torch.tensor(a[k], dtype=F32, device=DEV) for k in ("weight", "post_weight") if k in a}
    mods = _mods(a, ("gate", "scale", "shift"), lead % 8)
    rl.radial_norm_fwd(x, r, z, y=y, **t, **mods, group=group, post=post, pre=pre, residual_scale=0.7, eps=EPS)
    want_r, want_z = ol.norm_fwd(**a, group=group, post=post, pre=pre, residual_scale=np.float32(0.7).astype(np.float64), eps=EPS)
    gate = np.abs(ol.per_token(a["gate"], N, group, 1.0)) * np.abs(a.get("post_weight", 1.0))
    y_size, _ = _norm_magnitude(a["y"], np.abs(a["y"]), post)
    r_size = np.abs(a["x"]) + gate * y_size
    assert_within(r, want_r, HALF_STEP[xt] * np.abs(want_r) + 64 * U32 * r_size, "r")
    z_size, _ = _norm_magnitude(want_r, r_size, pre)
    factor = np.abs(a["weight"] * (1 + ol.per_token(a["scale"], N, group, 0.0)))
    # an error of a whole row of r moves its norm by as much again
    row = np.sqrt((r_size ** 2).mean(-1, keepdims=True)) * ol.norm(want_r, pre, EPS)[1] * (1 + np.abs(ol.norm(want_r, pre, EPS)[0]))
    assert_within(z, want_z, HALF_STEP[yt] * np.abs(want_z) + 128 * U32 * ((z_size + row) * factor + np.abs(ol.per_token(a["shift"], N, group, 0.0))), "z")
    assert surroundings_kept(r, r_whole) and surroundings_kept(z, z_whole)


def _backward(case, seed=12, in_place=False, drop=()):
    B, N, C, group, post, pre, xt, yt, lead = case
    a, g = _inputs(case, seed)
    a["dz"] = rounded(g.normal(0, 1, (B, N, C)), yt)
    a["dr"] = rounded(g.normal(0, 1, (B, N, C)), xt)
    a = {k: v for k, v in a.items() if k not in drop}
    named = {"r": xt, "dr": xt, "y": yt, "dz": yt}
    t = {}
    for k, dtype in named.items():
        if k not in drop:
            t[k], _ = inside(a["x" if k == "r" else k], dtype, lead)
    wholes = {}
    for k, dtype, of in (("dx", xt, "dr"), ("dy", yt, "dz")):
        if k == "dy" and "y" in drop:
            continue
        if in_place and of in t:
            t[k] = t[of]
        else:
            t[k], wholes[k] = inside(np.zeros((B, N, C)), dtype, lead)
    for k in ("weight", "post_weight"):
        if k in a:
            t[k] = torch.tensor(a[k], dtype=F32, device=DEV)
            t["d" + k] = torch.full((C,), np.nan, device=DEV)
    mods = _mods({"gate": np.zeros((B, -(-N // group), C)), **a}, [k for k in ("gate", "scale") if k in a], lead % 8)
    grads = _mods({"gate": np.zeros((B, -(-N // group), C))}, [k for k in ("dgate", "dscale", "dshift") if k != "dgate" or "y" not in drop], lead % 8)
    for v in grads.values():
        v.fill_(np.nan)
    ws = torch.empty(rl.radial_norm_bwd_workspace(B, N, C, group=group, post=post, pre=pre), dtype=torch.uint8, device=DEV).fill_(255)
    args = {k: v for k, v in t.items() if k not in ("r", "dz", "dx")}
    alpha = 1.0 if "y" in drop else 0.7
    rl.radial_norm_bwd(t["r"], t["dz"], t["dx"], ws, **args, **mods, **grads, group=group, post=post, pre=pre, residual_scale=alpha, eps=EPS)
    kw = dict(group=group, post=post, pre=pre, residual_scale=np.float64(np.float32(alpha)), eps=EPS)
    want = ol.norm_bwd(a["x"], a["dz"], a.get("dr"), **{k: a[k] for k in ("y", "gate", "post_weight", "weight", "scale") if k in a}, **kw)
    return a, {**t, **grads}, want, wholes, alpha


def _check_backward(case, a, got, want, alpha):
    B, N, C, group, post, pre, xt, yt, lead = case
    w, wp = np.abs(a.get("weight", 1.0)), np.abs(a.get("post_weight", 1.0))
    s, gt = 1 + ol.per_token(a.get("scale"), N, group, 0.0), np.abs(ol.per_token(a.get("gate"), N, group, 1.0))

    def through(d_size, v, kind):
        size, inverse = _norm_magnitude(v, np.abs(v), kind)
        if kind == ol.NONE:
            return d_size, size
        return inverse * (d_size + (d_size.mean(-1, keepdims=True) if kind == ol.LAYER else 0.0) + size * (d_size * size).mean(-1, keepdims=True)), size

    d_size, n_size = through(np.abs(a["dz"] * w * s), a["x"], pre)
    D_size = np.abs(a["dr"] if "dr" in a else 0.0) + d_size
    assert_within(got["dx"], want["dx"], HALF_STEP[xt] * np.abs(want["dx"]) + 64 * U32 * alpha * D_size, "dx")
    tokens = min(group, N)

    def summed(v):
        return ol._over_groups(v, group)

    sums = {"dscale": summed(np.abs(a["dz"]) * n_size) * w, "dshift": summed(np.abs(a["dz"])), "dweight": (np.abs(a["dz"]) * n_size * np.abs(s)).sum((0, 1))}
    if "y" in a:
        e_size, m_size = through(D_size * gt * wp, a["y"], post)
        assert_within(got["dy"], want["dy"], HALF_STEP[yt] * np.abs(want["dy"]) + 128 * U32 * e_size, "dy")
        sums["dgate"] = summed(D_size * m_size) * wp
        sums["dpost_weight"] = (D_size * m_size * gt).sum((0, 1))
    for k, size in sums.items():
        if k in got:
            assert_within(got[k], want[k], (128 + (tokens if k in ("dscale", "dshift", "dgate") else B * N)) * U32 * size, k)


@pytest.mark.parametrize("case", CASES, ids=str)
def test_gradients(case):
    a, got, want, wholes, alpha = _backward(case)
    _check_backward(case, a, got, want, alpha)
    for k, whole in wholes.items():
        assert surroundings_kept(got[k], whole), k


@pytest.mark.parametrize("case", [CASES[3], CASES[6], CASES[11]], ids=str)
@pytest.mark.parametrize("drop", [("y", "gate", "post_weight"), ("dr",), ("weight", "scale"), ("gate", "post_weight"), ("dr", "y", "gate", "post_weight", "weight", "scale")], ids=str)
def test_gradients_of_parts(case, drop):
    if "y" in drop:
        case = case[:4] + (ol.NONE,) + case[5:]
    a, got, want, _, alpha = _backward(case, drop=drop)
    _check_backward(case, a, got, want, alpha)


@pytest.mark.parametrize("case", [CASES[3], CASES[9], CASES[11]], ids=str)
def test_in_place(case):
    a, got, want, _, alpha = _backward(case, in_place=True)
    _check_backward(case, a, got, want, alpha)
    B, N, C, group, post, pre, xt, yt, lead = case
    x, y = inside(a["x"], xt, lead)[0], inside(a["y"], yt, lead)[0]
    r, z = torch.empty((B, N, C), dtype=xt, device=DEV), torch.empty((B, N, C), dtype=yt, device=DEV)
    rl.radial_norm_fwd(x, r, z, y=y, group=group, post=post, pre=pre, eps=EPS)
    rl.radial_norm_fwd(x, x, y, y=y, group=group, post=post, pre=pre, eps=EPS)
    assert torch.equal(x, r) and torch.equal(y, z)


def test_only_the_residual_and_only_its_gradients():
    B, N, C, group = 2, 30, 640, 7
    case = (B, N, C, group, ol.RMS, ol.NONE, BF16, BF16, 8)
    a, g = _inputs(case, 13)
    x, y = (torch.tensor(a[k]).to(BF16).to(DEV) for k in "xy")
    gate = torch.tensor(a["gate"], dtype=F32, device=DEV)
    r = torch.empty_like(x)
    rl.radial_norm_fwd(x, r, None, y=y, gate=gate, group=group, post=ol.RMS, pre=ol.NONE, eps=EPS)
    want, _ = ol.norm_fwd(a["x"], a["y"], a["gate"], group=group, post=ol.RMS, pre=ol.NONE, eps=EPS)
    size = np.abs(a["x"]) + np.abs(ol.per_token(a["gate"], N, group, 1)) * _norm_magnitude(a["y"], np.abs(a["y"]), ol.RMS)[0]
    assert_within(r, want, HALF_STEP[BF16] * np.abs(want) + 64 * U32 * size, "r")
    dr = torch.tensor(rounded(g.normal(size=(B, N, C)), BF16)).to(BF16).to(DEV)
    dx, dy, dgate = torch.empty_like(x), torch.empty_like(x), torch.empty_like(gate)
    ws = torch.empty(rl.radial_norm_bwd_workspace(B, N, C, group=group, post=ol.RMS, pre=ol.NONE), dtype=torch.uint8, device=DEV)
    rl.radial_norm_bwd(None, None, dx, ws, dr=dr, y=y, dy=dy, gate=gate, dgate=dgate, group=group, post=ol.RMS, pre=ol.NONE, eps=EPS)
    want = ol.norm_bwd(None, None, to64(dr), a["y"], a["gate"], group=group, post=ol.RMS, pre=ol.NONE, eps=EPS)
    assert torch.equal(dx, dr)
    m, inverse = ol.norm(a["y"], ol.RMS, EPS)
    e = np.abs(to64(dr) * ol.per_token(a["gate"], N, group, 1))
    assert_within(dy, want["dy"], HALF_STEP[BF16] * np.abs(want["dy"]) + 64 * U32 * inverse * (e + np.abs(m) * (e * np.abs(m)).mean(-1, keepdims=True)), "dy")
    assert_within(dgate, want["dgate"], 128 * U32 * ol._over_groups(np.abs(to64(dr) * m), group), "dgate")


@pytest.mark.parametrize("C", [64, 5120])
def test_a_row_that_is_not_finite_is_alone(C):
    N = 20
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(1, N, C, device=DEV, generator=g).to(BF16)
    z, clean = torch.empty_like(x), torch.empty_like(x)
    rl.radial_norm_fwd(x, None, clean)
    x[0, 3, 5], x[0, 11, 0] = float("inf"), float("nan")
    rl.radial_norm_fwd(x, None, z)
    bad = torch.zeros(N, dtype=torch.bool, device=DEV)
    bad[[3, 11]] = True
    assert torch.equal(z[0, ~bad], clean[0, ~bad]) and z[0, 11].isnan().all() and z[0, 3].isnan().all()
    # rows of zeros and of one value
    x[:] = 0
    rl.radial_norm_fwd(x, None, z, pre=ol.RMS)
    assert not z.any()
    x[:] = 3.0
    rl.radial_norm_fwd(x, None, z)
    assert not z.any()


def test_more_than_2_to_the_31_elements():
    C, N = 8192, (1 << 18) + 3
    x = torch.empty(1, N, C, dtype=BF16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(2)
    some = torch.randn(5, C, device=DEV, generator=g).to(BF16)
    x.zero_()
    x[0, -5:] = some
    z = torch.empty_like(x)
    rl.radial_norm_fwd(x, None, z)
    want = torch.empty(1, 5, C, dtype=BF16, device=DEV)
    rl.radial_norm_fwd(some[None], None, want)
    assert torch.equal(z[0, -5:], want[0])


@pytest.mark.parametrize("C", [2, 6, 9, 12, 15, 100, 121, 131, 250, 254, 259, 383, 511, 513, 518, 1023, 1029, 2051, 4095, 4101, 8187])
@pytest.mark.parametrize("types", [(BF16, BF16), (F32, F32), (F32, BF16)], ids=["bf16", "f32", "f32-bf16"])
def test_rows_that_end_anywhere(C, types):
    """The last eight channels are 1 to 8, rows start at any element's address."""
    for lead in (8, 1 + C % 5):
        case = (2, 7, C, 3, ol.LAYER if C % 2 else ol.RMS, ol.RMS if C % 3 else ol.LAYER, *types, lead)
        test_forward(case, 0.0)
        test_gradients(case)
    test_in_place(case)


@pytest.mark.parametrize("groups", [1, 2, 3, 4, 5, 8, 9, 16, 17, 40, 700])
@pytest.mark.parametrize("C", [24, 1000])
def test_gradients_of_weights_over_many_groups(C, groups):
    """However the groups are added up: in shares of one launch, one after the other, or in a launch of their own."""
    test_gradients((1, 3 * groups - (groups > 1), C, 3, ol.RMS, ol.LAYER, F32, BF16, 8))
    test_gradients((2, 5 * groups, C, 5, ol.RMS, ol.LAYER, BF16, BF16, 8))
