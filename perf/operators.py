"""The operators of a transformer layer around the attention, as timed cases.

A case is one pass through one operator of `paper_2506_19852_amd.layer`:

  norm    gated residual and norms: r = residual_scale x + gate N_post(y) post_weight and
          z = N_pre(r) weight (1 + scale) + shift, forward, or its gradients;
  rope    rotary positions of q and k, forward, or its gradient;
  linear  product in E4M3 with a scale for each 128 columns of an activation and each 128 x 128 of a weight:
          activations are quantised and multiplied, forward, or both gradients.

The plain forms are the formulas in elementary torch operations, in 32 bits.  A program keeps the table of a
rotary embedding, the codes of its weights and its buffers, so these are prepared.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
GROUP = 128          # values that share a scale
LARGEST = 448.0      # of E4M3
SMALLEST_SCALE = 2.0 ** -126
NONE, LAYER, RMS = 0, 1, 2
EPS = 1e-6


def _norm(direction, B, N, C, **kw):
    c = {"op": "norm", "direction": direction, "B": B, "N": N, "C": C, "group": N, "post": NONE, "pre": LAYER, "branch": True,
         "weights": False, "modulated": True, "residual_scale": 1.0, "stream_type": "bf16"}
    c.update(kw)
    return c


def _rope(direction, B, N, H, D, **kw):
    c = {"op": "rope", "direction": direction, "B": B, "N": N, "H": H, "Hk": H, "D": D, "size_t": 0, "size_h": 1, "size_w": 1,
         "dims_t": D, "dims_h": 0, "dims_w": 0, "layout": "interleaved", "scaling": "none", "factor": 1.0, "original": 0,
         "magnitude": 1.0, "given_positions": False, "first": 0, "type": "bf16"}
    c.update(kw)
    c["size_t"] = c["size_t"] or N
    return c


def _linear(direction, M, N, K, **kw):
    return {"op": "linear", "direction": direction, "M": M, "N": N, "K": K, **kw}


def listed():
    return [
        # What a layer does with the one conditioning token of each of two batch entries: latency alone.
        _norm("fwd", 2, 1, 5120, name="modulate_one_token", branch=False),
        # Between attention and feed-forward of a 480p layer, 21 frames of 1560 tokens, modulated frame by frame.
        _norm("fwd", 1, 32760, 5120, name="residual_norm_480p", group=1560),
        # Norms on both sides of a branch, residual stream in 32 bits, a padded batch of ragged size and width.
        _norm("bwd", 2, 1237, 1000, name="two_norms_train_ragged", post=RMS, pre=RMS, weights=True, stream_type="f32", residual_scale=0.5),
        # Tuning step: the same place of the 480p layer, one modulation for the whole clip.
        _norm("bwd", 1, 32760, 5120, name="residual_norm_train_480p"),
        # One new token of four sequences at far positions of a length scaled by parts.
        _rope("fwd", 4, 1, 40, 128, name="rope_one_token", size_t=131072, layout="half", scaling="parts", factor=8.0, original=16384,
              magnitude=1.2, given_positions=True),
        # q and k of a 480p layer, as the projection lays them out.
        _rope("fwd", 1, 32760, 40, 128, name="rope_480p", size_t=21, size_h=30, size_w=52, dims_t=16, dims_h=56, dims_w=56),
        # Gradient of the same step at 720p, frames interpolated to four times the length.
        _rope("bwd", 1, 118800, 24, 128, name="rope_720p_train", size_t=33, size_h=45, size_w=80, dims_t=16, dims_h=56, dims_w=56,
              scaling="linear", factor=4.0),
        # Part of a head, keys shared by the heads, a padded batch with its own positions, 32 bits.
        _rope("fwd", 3, 1023, 7, 64, name="rope_part_ragged", Hk=1, size_t=1200, dims_t=20, layout="half", given_positions=True, type="f32"),
        # A projection of one conditioning vector for each of two batch entries: the weight is all there is to read.
        _linear("fwd", 2, 5120, 5120, name="linear_two_rows"),
        # The output projection of a 480p layer.
        _linear("fwd", 32760, 5120, 5120, name="linear_480p"),
        # Both gradients of a projection over a clip of 9 frames of 1560 tokens.
        _linear("bwd", 14040, 5120, 5120, name="linear_train_clip"),
        # Sizes that fit no tile.
        _linear("fwd", 1237, 1961, 1000, name="linear_ragged"),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["norm", "rope", "linear"])
    direction = rng.choice(["fwd", "bwd"])
    if op == "norm":
        C = _spread(rng, 64, 8192)
        if rng.random() < 0.6:
            C = max(64, C // 64 * 64)
        B = rng.randint(1, 4)
        N = _spread(rng, 1, max(2, min(40000, 32760 * 5120 // (C * B))))
        branch = rng.random() < 0.7
        return _norm(direction, B, N, C, group=rng.choice([N, max(1, N // rng.randint(2, 21))]), branch=branch,
                     post=rng.choice([NONE, RMS, LAYER]) if branch else NONE, pre=rng.choice([LAYER, RMS]), weights=rng.random() < 0.5,
                     modulated=rng.random() < 0.8, residual_scale=rng.choice([1.0, 0.7]) if branch else 1.0,
                     stream_type=rng.choice(["bf16", "f32"]))
    if op == "rope":
        D = rng.choice([64, 128, 128, 80])
        H = rng.randint(1, 40)
        B = rng.randint(1, 3)
        kind = rng.choice(["grid", "line", "part"])
        if kind == "grid":
            t, h, w = _spread(rng, 1, 33), rng.randint(4, 45), rng.randint(4, 60)
            extra = rng.choice([0, 0, 77])
            N = min(t * h * w + extra, 80000)
            kw = dict(size_t=t, size_h=h, size_w=w, dims_t=D - 2 * (D // 16 * 6), dims_h=D // 16 * 6, dims_w=D // 16 * 6)
        else:
            N = _spread(rng, 1, 40000)
            kw = dict(size_t=N + _spread(rng, 1, 100000), dims_t=D if kind == "line" else rng.choice([D // 2, D // 4, 2 * rng.randint(1, D // 2)]))
        B = max(1, min(B, 118800 * 24 * 128 // (N * H * D)))
        scaling = rng.choice(["none", "linear", "base", "parts"])
        if scaling != "none":
            kw.update(scaling=scaling, factor=rng.choice([2.0, 4.0, 8.0]), original=max(1, kw["size_t"] // 4), magnitude=rng.choice([1.0, 1.15]))
        return _rope(direction, B, N, H, D, Hk=rng.choice([H, 1]), layout=rng.choice(["interleaved", "half"]),
                     given_positions=rng.random() < 0.4, first=0 if kind == "grid" else rng.randint(0, 9), type=rng.choice(["bf16", "bf16", "f32"]), **kw)
    M = _spread(rng, 1, 32760)
    N, K = _spread(rng, 64, 8192), _spread(rng, 64, 8192)
    if rng.random() < 0.6:
        N, K = max(128, N // 128 * 128), max(128, K // 128 * 128)
    while M * N * K * (2 if direction == "bwd" else 1) > 32760 * 5120 * 5120:
        M = max(1, M * 2 // 3)
    return _linear(direction, M, N, K)


# ---- inputs ---------------------------------------------------------------------------------

def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


class _Source:
    """Normal values from a seed, on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEVICE).manual_seed(seed)

    def __call__(self, *shape, size=1.0, mean=0.0, dtype=torch.float32):
        x = torch.randn(shape, generator=self.g, device=DEVICE)
        return x.mul_(size).add_(mean).to(dtype)


def prepare(case, seed):
    rand = _Source(seed)
    return {"case": case, **{"norm": _prepare_norm, "rope": _prepare_rope, "linear": _prepare_linear}[case["op"]](case, rand)}


def _prepare_norm(case, rand):
    B, N, C = case["B"], case["N"], case["C"]
    stream, bf16 = _type(case["stream_type"]), torch.bfloat16
    G = -(-N // case["group"])
    s = {}
    # a residual stream has a few channels that are far larger than the rest, and an offset
    channel = 1.0 + 8.0 * (rand(C) > 2.3)
    full = (rand(B, N, C, size=1.5, mean=0.1) * channel).to(stream)
    if case["branch"]:
        s["y"] = rand(B, N, C, size=0.8, dtype=bf16)
    # shift, scale and gate are chunks of one row of conditioning, as a layer has them
    mod = rand(B, G, 3, C, size=0.3)
    if case["modulated"]:
        s["shift"], s["scale"] = mod[:, :, 0], mod[:, :, 1]
        if case["branch"]:
            s["gate"] = mod[:, :, 2]
    if case["weights"]:
        s["weight"] = rand(C, size=0.1, mean=1.0)
        if case["post"] != NONE:
            s["post_weight"] = rand(C, size=0.1, mean=1.0)
    if case["direction"] == "fwd":
        s["x"] = full
        s["z"] = torch.empty(B, N, C, dtype=bf16, device=DEVICE)
        if case["branch"]:
            s["r"] = torch.empty_like(full)
        return s
    s["r"] = full
    s["dz"] = rand(B, N, C, size=0.02, dtype=bf16)
    s["dr"] = rand(B, N, C, size=0.02).to(stream)
    s["dx"] = torch.empty_like(full)
    grads = ["shift", "scale", "weight"]
    if case["branch"]:
        s["dy"] = torch.empty(B, N, C, dtype=bf16, device=DEVICE)
        grads += ["gate", "post_weight"]
    for name in grads:
        if name in s:
            s["d" + name] = torch.empty(s[name].shape, dtype=torch.float32, device=DEVICE)
    s["workspace"] = torch.empty(0, dtype=torch.uint8, device=DEVICE)
    if own:
        from paper_2506_19852_amd import layer
        s["workspace"] = torch.empty(layer.radial_norm_bwd_workspace(B, N, C, group=case["group"], post=case["post"], pre=case["pre"]),
                                     dtype=torch.uint8, device=DEVICE)
    return s


def _axes(case):
    """(positions, head dimensions) of each axis that has any."""
    return [(case["size_" + a], case["dims_" + a]) for a in "thw" if case["dims_" + a]]


def _frequencies(case, dims):
    """Angle per position of each pair of an axis, in 64 bits."""
    m = torch.arange(dims // 2, dtype=torch.float64, device=DEVICE)
    factor, theta = case["factor"], 10000.0
    if case["scaling"] == "base" and dims > 2:
        theta = theta * factor ** (dims / (dims - 2))
    f = theta ** (-2.0 * m / dims)
    if case["scaling"] == "linear":
        f = f / factor
    elif case["scaling"] == "parts":
        turns = case["original"] * f / (2 * math.pi)
        keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / factor)
    return f


def _prepare_rope(case, rand):
    B, N, D = case["B"], case["N"], case["D"]
    dtype = _type(case["type"])
    s = {}
    for name, H in (("q", case["H"]), ("k", case["Hk"])):
        # the projection's output [B, N, H, D]; the attention's input [B, H, N, D].  Gradients come and go the other way.
        token_major = rand(B, N, H, D, dtype=dtype).transpose(1, 2)
        head_major = torch.empty(B, H, N, D, dtype=dtype, device=DEVICE)
        if case["direction"] == "bwd":
            head_major.copy_(token_major)
            token_major, head_major = head_major, torch.empty_like(token_major)
        s[name], s[name + "_out"] = token_major, head_major
    total = math.prod(size for size, _ in _axes(case))
    s["positions"] = None
    if case["given_positions"]:
        at = torch.randint(0, total, (B, N), generator=rand.g, device=DEVICE)
        keep = torch.rand((B, N), generator=rand.g, device=DEVICE) > 0.05   # the others are padding, or text: not rotated
        s["positions"] = torch.where(keep, at, -1).to(torch.int32)
    if own:
        from paper_2506_19852_amd import layer
        s["params"] = layer.rope_params([size for size, _ in _axes(case)], [dims for _, dims in _axes(case)], layout=case["layout"],
                                        scaling=case["scaling"], factor=case["factor"], original=case["original"], magnitude=case["magnitude"])
        s["table"] = torch.empty(layer.radial_rope_table_bytes(s["params"]) // 4, dtype=torch.float32, device=DEVICE)
        layer.radial_rope_table(s["params"], s["table"])
    else:
        s["tables"] = []
        for size, dims in _axes(case):
            angle = torch.arange(size, dtype=torch.float64, device=DEVICE)[:, None] * _frequencies(case, dims)[None, :]
            s["tables"].append(((angle.cos() * case["magnitude"]).float(), (angle.sin() * case["magnitude"]).float()))
    return s


def _prepare_linear(case, rand):
    M, N, K = case["M"], case["N"], case["K"]
    channel = torch.exp(rand(K, size=0.7))
    s = {"x": (rand(M, K) * channel).to(torch.bfloat16)}
    # codes [rows, columns rounded up to 128] and scales [128-column groups, 128-row blocks] of the weight, and of its transpose
    w = rand(N, K, size=K ** -0.5)
    padded = torch.zeros(-(-N // GROUP) * GROUP, -(-K // GROUP) * GROUP, device=DEVICE)
    padded[:N, :K] = w
    blocks = padded.view(padded.shape[0] // GROUP, GROUP, padded.shape[1] // GROUP, GROUP)
    scale = (blocks.abs().amax((1, 3)) / LARGEST).clamp_min(SMALLEST_SCALE)
    codes = (blocks / scale[:, None, :, None]).view(padded.shape).to(torch.float8_e4m3fn).view(torch.uint8)
    if case["direction"] == "fwd":
        s["w_codes"], s["w_scales"] = codes[:N].contiguous(), scale.t().contiguous()
        s["out"] = torch.empty(M, N, dtype=torch.bfloat16, device=DEVICE)
        kept = [("x", M, K)]
    else:
        s["wt_codes"], s["wt_scales"] = codes.t()[:K].contiguous(), scale.contiguous()
        s["dout"] = rand(M, N, size=0.02, dtype=torch.bfloat16)
        s["dx"] = torch.empty(M, K, dtype=torch.bfloat16, device=DEVICE)
        s["dw"] = torch.empty(N, K, dtype=torch.bfloat16, device=DEVICE)
        kept = [("dout", M, N), ("dout_t", N, M), ("x_t", K, M)]
    for name, rows, columns in kept:   # buffers of the quantised activations
        groups = -(-columns // GROUP)
        s[name + "_codes"] = torch.empty(rows, groups * GROUP, dtype=torch.uint8, device=DEVICE)
        s[name + "_scales"] = torch.empty(groups, rows, dtype=torch.float32, device=DEVICE)
    return s


# ---- one pass -------------------------------------------------------------------------------

def run(state):
    op, direction = state["case"]["op"], state["case"]["direction"]
    if own:
        return {"norm": {"fwd": _own_norm_fwd, "bwd": _own_norm_bwd}, "rope": {"fwd": _own_rope, "bwd": _own_rope},
                "linear": {"fwd": _own_linear_fwd, "bwd": _own_linear_bwd}}[op][direction](state)
    return {"norm": {"fwd": _plain_norm_fwd, "bwd": _plain_norm_bwd}, "rope": {"fwd": _plain_rope, "bwd": _plain_rope},
            "linear": {"fwd": _plain_linear_fwd, "bwd": _plain_linear_bwd}}[op][direction](state)


def _own_norm_fwd(s):
    from paper_2506_19852_amd import layer
    c = s["case"]
    layer.radial_norm_fwd(s["x"], s.get("r"), s["z"], y=s.get("y"), gate=s.get("gate"), post_weight=s.get("post_weight"), weight=s.get("weight"),
                          scale=s.get("scale"), shift=s.get("shift"), group=c["group"], post=c["post"], pre=c["pre"],
                          residual_scale=c["residual_scale"], eps=EPS)
    return {k: s[k] for k in ("r", "z") if k in s}


def _own_norm_bwd(s):
    from paper_2506_19852_amd import layer
    c = s["case"]
    grads = {k: s[k] for k in ("dgate", "dscale", "dshift", "dweight", "dpost_weight") if k in s}
    layer.radial_norm_bwd(s["r"], s["dz"], s["dx"], s["workspace"], dr=s["dr"], y=s.get("y"), dy=s.get("dy"), gate=s.get("gate"),
                          post_weight=s.get("post_weight"), weight=s.get("weight"), scale=s.get("scale"), group=c["group"], post=c["post"],
                          pre=c["pre"], residual_scale=c["residual_scale"], eps=EPS, **grads)
    return {"dx": s["dx"], **({"dy": s["dy"]} if "dy" in s else {}), **grads}


def _own_rope(s):
    from paper_2506_19852_amd import layer
    call = layer.radial_rope_fwd if s["case"]["direction"] == "fwd" else layer.radial_rope_bwd
    call(s["params"], s["table"], s["q"], s["q_out"], s["k"], s["k_out"], positions=s["positions"], first=s["case"]["first"])
    return [s["q_out"], s["k_out"]]


def _own_linear_fwd(s):
    from paper_2506_19852_amd import layer
    layer.radial_quantize_groups_fp8(s["x"], s["x_codes"], s["x_scales"])
    layer.radial_product_fp8(s["x_codes"], s["x_scales"], s["w_codes"], s["w_scales"], s["out"])
    return s["out"]


def _own_linear_bwd(s):
    from paper_2506_19852_amd import layer
    layer.radial_quantize_groups_fp8(s["dout"], s["dout_codes"], s["dout_scales"], s["dout_t_codes"], s["dout_t_scales"])
    layer.radial_quantize_groups_fp8(s["x"], None, None, s["x_t_codes"], s["x_t_scales"])
    layer.radial_product_fp8(s["dout_codes"], s["dout_scales"], s["wt_codes"], s["wt_scales"], s["dx"])
    layer.radial_product_fp8(s["dout_t_codes"], s["dout_t_scales"], s["x_t_codes"], s["x_t_scales"], s["dw"])
    return {"dx": s["dx"], "dw": s["dw"]}


def _per_token(m, N, group):
    """A row of conditioning for each group of tokens, as one for each token (one for all, where there is one group)."""
    return m if m.shape[1] == 1 else m.repeat_interleave(group, dim=1)[:, :N]


def _normalised(v, kind):
    """(normalised rows, 1 / their size)"""
    if kind == LAYER:
        v = v - v.mean(-1, keepdim=True)
    inverse = torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS)
    return v * inverse, inverse


def _plain_norm_fwd(s):
    c = s["case"]
    N, group = c["N"], c["group"]
    r = s["x"].float()
    out = {}
    if c["branch"]:
        u = s["y"].float()
        if c["post"] != NONE:
            u, _ = _normalised(u, c["post"])
            if "post_weight" in s:
                u = u * s["post_weight"]
        if "gate" in s:
            u = u * _per_token(s["gate"], N, group)
        r = c["residual_scale"] * r + u
        out["r"] = s["r"].copy_(r)
    z, _ = _normalised(r, c["pre"])
    if "weight" in s:
        z = z * s["weight"]
    if "scale" in s:
        z = z * (1.0 + _per_token(s["scale"], N, group)) + _per_token(s["shift"], N, group)
    out["z"] = s["z"].copy_(z)
    return out


def _back_through_norm(d, n, inverse, kind):
    d_mean = d.mean(-1, keepdim=True) if kind == LAYER else 0.0
    return inverse * (d - d_mean - n * (d * n).mean(-1, keepdim=True))


def _over_groups(v, N, group):
    """Sums over the tokens of each group."""
    B, C = v.shape[0], v.shape[2]
    G = -(-N // group)
    if G * group != N:
        v = torch.nn.functional.pad(v, (0, 0, 0, G * group - N))
    return v.view(B, G, group, C).sum(2)


def _plain_norm_bwd(s):
    c = s["case"]
    N, group = c["N"], c["group"]
    out = {}
    n, inverse = _normalised(s["r"].float(), c["pre"])
    dz = s["dz"].float()
    along = _over_groups(dz * n, N, group)
    d = dz
    if "scale" in s:
        d = d * (1.0 + _per_token(s["scale"], N, group))
        out["dscale"] = s["dscale"].copy_(along * s["weight"] if "weight" in s else along)
        out["dshift"] = s["dshift"].copy_(_over_groups(dz, N, group))
    if "weight" in s:
        d = d * s["weight"]
        out["dweight"] = s["dweight"].copy_((along * (1.0 + s["scale"]) if "scale" in s else along).sum((0, 1)))
    total = s["dr"].float() + _back_through_norm(d, n, inverse, c["pre"])
    out["dx"] = s["dx"].copy_(c["residual_scale"] * total)
    if c["branch"]:
        u, inverse = _normalised(s["y"].float(), c["post"]) if c["post"] != NONE else (s["y"].float(), None)
        along = _over_groups(total * u, N, group) if "gate" in s or "post_weight" in s else None
        d = total
        if "gate" in s:
            out["dgate"] = s["dgate"].copy_(along * s["post_weight"] if "post_weight" in s else along)
            d = d * _per_token(s["gate"], N, group)
        if "post_weight" in s:
            out["dpost_weight"] = s["dpost_weight"].copy_((along * s["gate"] if "gate" in s else along).sum((0, 1)))
            d = d * s["post_weight"]
        out["dy"] = s["dy"].copy_(_back_through_norm(d, u, inverse, c["post"]) if c["post"] != NONE else d)
    return out


def _token_positions(s):
    """Index of each token on the grid, and whether it is on it."""
    c = s["case"]
    total = math.prod(size for size, _ in _axes(c))
    at = s["positions"] if s["positions"] is not None else (torch.arange(c["N"], device=DEVICE) + c["first"]).view(1, -1)
    on = (at >= 0) & (at < total)
    return torch.where(on, at, 0).long(), on


def _pairs(x, layout, pairs):
    """The two halves of the pairs of the first 2 * pairs dimensions."""
    return (x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2]) if layout == "interleaved" else (x[..., :pairs], x[..., pairs:2 * pairs])


def _plain_rope(s):
    c = s["case"]
    at, on = _token_positions(s)
    axes = _axes(c)
    cos, sin, rest = [], [], at
    for (size, _), (ct, st) in zip(reversed(axes), reversed(s["tables"])):
        cos.insert(0, ct[rest % size])
        sin.insert(0, st[rest % size])
        rest = rest // size
    cos, sin = torch.cat(cos, -1), torch.cat(sin, -1)
    cos, sin = torch.where(on[..., None], cos, 1.0)[:, None], torch.where(on[..., None], sin, 0.0)[:, None]
    if c["direction"] == "bwd":
        sin = -sin
    pairs = cos.shape[-1]
    for name in ("q", "k"):
        x, out = s[name].float(), s[name + "_out"]
        a, b = _pairs(x, c["layout"], pairs)
        to_a, to_b = _pairs(out, c["layout"], pairs)
        to_a.copy_(a * cos - b * sin)
        to_b.copy_(a * sin + b * cos)
        out[..., 2 * pairs:] = s[name][..., 2 * pairs:]
    return [s["q_out"], s["k_out"]]


def _quantised(x):
    """Values that the E4M3 codes of x, with a scale for each 128 columns, stand for: [rows, columns rounded up to 128]."""
    rows, columns = x.shape
    x = x.float()
    if columns % GROUP:
        x = torch.nn.functional.pad(x, (0, -columns % GROUP))
    x = x.view(rows, -1, GROUP)
    largest = x.abs().amax(-1, keepdim=True)
    # a quotient of tensors: one by a number is a product with its rounded inverse, which moves the many ties
    scale = (largest / torch.full_like(largest, LARGEST)).clamp_min(SMALLEST_SCALE)
    return ((x / scale).to(torch.float8_e4m3fn).float() * scale).view(rows, -1)


def _of_blocks(codes, scales):
    """Values of a weight's codes [rows, columns] with scales [128-column groups, 128-row blocks]."""
    full = scales.t().repeat_interleave(GROUP, 0)[:codes.shape[0]].repeat_interleave(GROUP, 1)
    return codes.view(torch.float8_e4m3fn).float() * full


def _plain_linear_fwd(s):
    return s["out"].copy_(_quantised(s["x"]) @ _of_blocks(s["w_codes"], s["w_scales"]).t())


def _plain_linear_bwd(s):
    s["dx"].copy_(_quantised(s["dout"]) @ _of_blocks(s["wt_codes"], s["wt_scales"]).t())
    s["dw"].copy_(_quantised(s["dout"].t()) @ _quantised(s["x"].t()).t())
    return {"dx": s["dx"], "dw": s["dw"]}


# ---- what a pass cannot do without ------------------------------------------------------------

def work(case):
    if case["op"] == "norm":
        B, N, C = case["B"], case["N"], case["C"]
        stream = 4 if case["stream_type"] == "f32" else 2
        G, rows = -(-N // case["group"]), B * N * C
        moved = 2 * stream + 2 + (2 if case["branch"] else 0) if case["direction"] == "fwd" else 3 * stream + 2 + (4 if case["branch"] else 0)
        if case["direction"] == "fwd" and not case["branch"]:
            moved -= stream   # r is x
        rows_of_mod = (3 if case["branch"] else 2) * (2 if case["direction"] == "bwd" else 1) if case["modulated"] else 0
        return {"bytes": rows * moved + 4 * C * B * G * rows_of_mod + (8 * C if case["weights"] else 0), "flops": rows * (12 if case["direction"] == "fwd" else 30)}
    if case["op"] == "rope":
        n = case["B"] * case["N"] * (case["H"] + case["Hk"]) * case["D"]
        table = sum(size * dims for size, dims in _axes(case)) * 4
        return {"bytes": 2 * n * (4 if case["type"] == "f32" else 2) + min(table, case["B"] * case["N"] * case["D"] * 4), "flops": 3 * n}
    M, N, K = case["M"], case["N"], case["K"]
    if case["direction"] == "fwd":
        return {"bytes": 2 * M * K + N * K + 2 * M * N, "flops": 2 * M * N * K}
    return {"bytes": 2 * M * K + 2 * M * N + N * K + 2 * M * K + 2 * N * K, "flops": 4 * M * N * K}


# ---- 64 bits ----------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "rope": _exact_rope, "linear": _exact_linear}[case["op"]](case, s)


def _statistics64(v, kind):
    mean = v.mean(-1) if kind == LAYER else torch.zeros_like(v[..., 0])
    size = ((v - mean[..., None]) ** 2).sum(-1) / v.shape[-1]
    return mean[..., None], 1.0 / torch.sqrt(size + EPS)[..., None]


def _exact_norm(c, s):
    B, N, C, group = c["B"], c["N"], c["C"], c["group"]
    which = torch.arange(N, device=DEVICE) // group
    of = lambda name, default: s[name].double()[:, which] if name in s else default  # noqa: E731
    wide = lambda name: s[name].double() if name in s else torch.ones(C, dtype=torch.float64, device=DEVICE)  # noqa: E731
    factor = wide("weight") * (1.0 + of("scale", 0.0))
    if c["branch"]:
        y = s["y"].double()
        y_mean, y_inverse = _statistics64(y, c["post"]) if c["post"] != NONE else (0.0, 1.0)
        y_n = (y - y_mean) * y_inverse
        y_factor = wide("post_weight") * of("gate", 1.0)
    if c["direction"] == "fwd":
        r = s["x"].double() * c["residual_scale"] + (y_n * y_factor if c["branch"] else 0.0)
        mean, inverse = _statistics64(r, c["pre"])
        z = (r - mean) * inverse * factor + of("shift", 0.0)
        return {"r": r, "z": z} if c["branch"] else {"z": z}

    def add_up(v):
        return torch.stack([v[:, which == g].sum(1) for g in range(int(which[-1]) + 1)], 1)

    def before_norm(d, n, inverse, kind):
        # the part of d along n, and for a layer norm along the constant, does not reach the input
        flat = d - n * ((d * n).sum(-1, keepdim=True) / C)
        return inverse * (flat - d.sum(-1, keepdim=True) / C if kind == LAYER else flat)

    out = {}
    r, dz = s["r"].double(), s["dz"].double()
    mean, inverse = _statistics64(r, c["pre"])
    n = (r - mean) * inverse
    of_n = add_up(dz * n)
    total = s["dr"].double() + before_norm(dz * factor, n, inverse, c["pre"])
    out["dx"] = total * c["residual_scale"]
    if c["branch"]:
        d = total * y_factor
        out["dy"] = before_norm(d, y_n, y_inverse, c["post"]) if c["post"] != NONE else d
    if "scale" in s:
        out["dscale"], out["dshift"] = of_n * wide("weight"), add_up(dz)
    if "weight" in s:
        out["dweight"] = (of_n * (1.0 + (s["scale"].double() if "scale" in s else 0.0))).sum((0, 1))
    if c["branch"] and ("gate" in s or "post_weight" in s):
        of_y = add_up(total * y_n)
        if "gate" in s:
            out["dgate"] = of_y * wide("post_weight")
        if "post_weight" in s:
            out["dpost_weight"] = (of_y * (s["gate"].double() if "gate" in s else 1.0)).sum((0, 1))
    return out


def _exact_rope(c, s):
    B, N = c["B"], c["N"]
    axes = _axes(c)
    total = math.prod(size for size, _ in axes)
    at = s["positions"].long() if s["positions"] is not None else torch.arange(c["first"], c["first"] + N, device=DEVICE).expand(B, N)
    angles, below = [], total
    for size, dims in axes:
        below //= size
        along = torch.div(at, below, rounding_mode="floor") % size
        angles.append(along.double()[..., None] * _frequencies64(c, dims))
    angle = torch.cat(angles, -1)
    on = ((at >= 0) & (at < total))[:, None, :, None]
    turn = torch.polar(torch.full_like(angle, c["magnitude"]), angle if c["direction"] == "fwd" else -angle)[:, None]
    pairs = angle.shape[-1]
    out = []
    for name in ("q", "k"):
        x = s[name].double()
        first = list(range(0, 2 * pairs, 2)) if c["layout"] == "interleaved" else list(range(pairs))
        second = [i + 1 for i in first] if c["layout"] == "interleaved" else [i + pairs for i in first]
        z = torch.complex(x[..., first], x[..., second])
        z = torch.where(on, z * turn, z)
        y = x.clone()
        y[..., first], y[..., second] = z.real, z.imag
        out.append(y)
    return out


def _frequencies64(c, dims):
    base, found = 10000.0, []
    if c["scaling"] == "base" and dims > 2:
        base *= c["factor"] ** (dims / (dims - 2.0))
    for m in range(dims // 2):
        f = math.exp(-2.0 * m / dims * math.log(base))
        if c["scaling"] == "linear":
            f /= c["factor"]
        if c["scaling"] == "parts":
            turns = c["original"] * f / (2.0 * math.pi)
            keep = min(1.0, max(0.0, (turns - 1.0) / 31.0))
            f = keep * f + (1.0 - keep) * f / c["factor"]
        found.append(f)
    return torch.tensor(found, dtype=torch.float64, device=DEVICE)


def _nearest_e4m3(v):
    """The nearest E4M3 values, ties to the even one, by arithmetic in 64 bits."""
    e = torch.frexp(v.abs().clamp_min(2.0 ** -6)).exponent - 1      # at least that of the smallest normal value
    step = torch.ldexp(torch.ones_like(v), e - 3)
    return (torch.round(v / step) * step).clamp(-LARGEST, LARGEST)


def _quantised64(x):
    rows, columns = x.shape
    v = torch.zeros(rows, -(-columns // GROUP) * GROUP, dtype=torch.float64, device=DEVICE)
    v[:, :columns] = x.double()
    v = v.view(rows, -1, GROUP)
    scale = torch.maximum(v.abs().amax(-1) / LARGEST, torch.full_like(v[..., 0], SMALLEST_SCALE)).float().double()[..., None]
    # the scheme's scales and quotients are float32 values (ties are common: both are quotients of short numbers)
    return (_nearest_e4m3((v / scale).float().double()) * scale).view(rows, -1)


def _weight64(codes, scales):
    rows, columns = codes.shape
    sign = torch.where(codes >= 128, -1.0, 1.0).double()
    e, m = ((codes >> 3) & 15).double(), (codes & 7).double()
    value = sign * torch.where(e > 0, torch.ldexp(1.0 + m / 8.0, e - 7.0), torch.ldexp(m / 8.0, torch.full_like(m, -6.0)))
    i, j = torch.arange(rows, device=DEVICE) // GROUP, torch.arange(columns, device=DEVICE) // GROUP
    return value * scales.double()[j[None, :], i[:, None]]


def _exact_linear(c, s):
    if c["direction"] == "fwd":
        return _quantised64(s["x"]) @ _weight64(s["w_codes"], s["w_scales"]).t()
    dx = _quantised64(s["dout"]) @ _weight64(s["wt_codes"], s["wt_scales"]).t()
    dw = _quantised64(s["dout"].t().contiguous()) @ _quantised64(s["x"].t().contiguous()).t()
    return {"dx": dx, "dw": dw}
