"""The operators of a tuning step on 8-bit integer products, as timed cases.

A case is one pass through one operator of `paper_2506_19852_amd.layer`:

  linear  a projection in 8-bit integers: activations get a scale for each token, weights one for each channel, their codes are
          multiplied and summed as whole numbers; forward, or its gradients with respect to activations, weights and bias;
  adamw   one step over many tensors at once, with states in 32 bits or in 8 (a scale for each 128 values), gradients
          clipped by their common norm or not.

The plain forms are the formulas in elementary torch operations, in 32 bits.  A program keeps the codes of its weights, its buffers and the
table of its tensors, so these are prepared.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
LARGEST_I8 = 127.0
LARGEST_E4M3 = 448.0
SMALLEST_SCALE = 2.0 ** -126
BLOCK = 128          # values of a state that share a scale
BETA1, BETA2, EPS, LR, MAX_NORM = 0.9, 0.999, 1e-8, 1e-4, 1.0


def _linear(direction, M, N, K, **kw):
    c = {"op": "linear", "direction": direction, "M": M, "N": N, "K": K, "bias": True, "type": "bf16", "out_type": "bf16"}
    c.update(kw)
    return c


def _adamw(matrices, rows, cols, vectors, length, **kw):
    c = {"op": "adamw", "matrices": matrices, "rows": rows, "cols": cols, "vectors": vectors, "length": length, "more": 0, "states": "f32",
         "weight_type": "f32", "grad_type": "bf16", "copy": False, "clip": False, "rounding": "nearest", "decay": 0.01}
    c.update(kw)
    return c


def listed():
    return [
        # A projection of one conditioning vector for each of two batch entries: the weight is all there is to read.
        _linear("fwd", 2, 5120, 5120, name="linear_i8_two_rows"),
        # The text tokens of a prompt, from the width of their encoder.
        _linear("fwd", 512, 5120, 4096, name="linear_i8_text"),
        # A projection of a 480p layer, 21 frames of 1560 tokens.
        _linear("fwd", 32760, 5120, 5120, name="linear_i8_480p"),
        # Sizes that fit no tile, activations and results in 32 bits.
        _linear("fwd", 1237, 1961, 1001, name="linear_i8_ragged", bias=False, type="f32", out_type="f32"),
        # All gradients of a projection over a clip of 9 frames of 1560 tokens, those of the weights in 32 bits.
        _linear("bwd", 14040, 5120, 5120, name="linear_i8_train_clip", out_type="f32"),
        # The same of a small projection whose sizes fit no tile.
        _linear("bwd", 1001, 333, 2049, name="linear_i8_train_ragged"),
        # The weight of one norm: latency alone.
        _adamw(0, 0, 0, 1, 5120, name="adamw_one_vector", grad_type="f32"),
        # The weights of an attention layer (q, k, v, output) with a bf16 copy for the products, clipped.
        _adamw(4, 5120, 5120, 8, 5120, name="adamw_layer", copy=True, clip=True),
        # The same with states in 8 bits.
        _adamw(4, 5120, 5120, 8, 5120, name="adamw_layer_8bit", copy=True, clip=True, states="8bit"),
        # Low-rank adapters on the four projections of 40 layers: many small tensors.
        _adamw(320, 16, 5120, 0, 0, name="adamw_adapters", grad_type="f32"),
        # Weights in bf16 alone, tensors of odd sizes one behind the other, states in 8 bits rounded at random.
        _adamw(24, 777, 1001, 24, 1001, name="adamw_8bit_ragged", more=13, states="8bit", weight_type="bf16", rounding="random"),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    if rng.random() < 0.5:
        direction = rng.choice(["fwd", "bwd"])
        M = _spread(rng, 1, 32760)
        N, K = _spread(rng, 64, 8192), _spread(rng, 64, 8192)
        if rng.random() < 0.6:
            N, K = max(128, N // 128 * 128), max(128, K // 128 * 128)
        while M * N * K * (2 if direction == "bwd" else 1) > 32760 * 5120 * 5120:
            M = max(1, M * 2 // 3)
        return _linear(direction, M, N, K, bias=rng.random() < 0.6, type=rng.choice(["bf16", "bf16", "f32"]), out_type=rng.choice(["bf16", "f32"]))
    most = 40_000_000
    matrices = _spread(rng, 1, 400)
    rows, cols = _spread(rng, 1, 5120), _spread(rng, 8, 5120)
    while matrices * rows * cols > most:
        rows = max(1, rows // 2)
        matrices = max(1, matrices * 3 // 4)
    return _adamw(matrices, rows, cols, rng.choice([0, 1, 40]), _spread(rng, 1, 8192), more=rng.choice([0, 0, 1, 13]), states=rng.choice(["f32", "8bit"]),
                  weight_type=rng.choice(["f32", "f32", "bf16"]), grad_type=rng.choice(["f32", "bf16"]), copy=rng.random() < 0.4, clip=rng.random() < 0.5,
                  rounding=rng.choice(["nearest", "random"]), decay=rng.choice([0.0, 0.01, 0.1]))


# ---- inputs ---------------------------------------------------------------------------------

def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


class _Source:
    """Normal values from a seed, on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEVICE).manual_seed(seed)

    def __call__(self, *shape, size=1.0, dtype=torch.float32):
        return torch.randn(shape, generator=self.g, device=DEVICE).mul_(size).to(dtype)


def prepare(case, seed):
    rand = _Source(seed)
    return {"case": case, **{"linear": _prepare_linear, "adamw": _prepare_adamw}[case["op"]](case, rand)}


def _prepare_linear(case, rand):
    M, N, K = case["M"], case["N"], case["K"]
    channel = torch.exp(rand(K, size=0.7))   # a few channels of the activations are far larger than the rest
    s = {"x": (rand(M, K) * channel).to(_type(case["type"]))}
    w = rand(N, K, size=K ** -0.5)
    out_type = _type(case["out_type"])
    if case["direction"] == "fwd":
        s["w_codes"], s["w_scales"] = _padded_codes(w)
        s["out"] = torch.empty(M, N, dtype=out_type, device=DEVICE)
        if case["bias"]:
            s["bias"] = rand(N, size=0.1)
    else:
        s["wt_codes"], s["wt_scales"] = _padded_codes(w.t().contiguous())
        s["dout"] = rand(M, N, size=0.02, dtype=_type(case["type"]))
        s["dx"] = torch.empty(M, K, dtype=_type(case["type"]), device=DEVICE)
        s["dw"] = torch.empty(N, K, dtype=out_type, device=DEVICE)
        if case["bias"]:
            s["dbias"] = torch.empty(N, device=DEVICE)
    if own:
        from paper_2506_19852_amd import layer
        size = layer.radial_linear_i8_fwd_workspace if case["direction"] == "fwd" else layer.radial_linear_i8_bwd_workspace
        s["workspace"] = torch.empty(size(M, N, K), dtype=torch.uint8, device=DEVICE)
    return s


def _row_codes(x):
    """(whole numbers of at most 127 as float32, scale of each row)"""
    x = x.float()
    largest = x.abs().amax(1, keepdim=True)
    # a quotient of tensors: one by a number is a product with its rounded inverse
    scale = (largest / torch.full_like(largest, LARGEST_I8)).clamp_min(SMALLEST_SCALE)
    return torch.round(x / scale), scale[:, 0]


def _padded_codes(w):
    """A weight's codes as they are kept: int8, columns rounded up to 128."""
    codes, scales = _row_codes(w)
    kept = torch.zeros(w.shape[0], -(-w.shape[1] // 128) * 128, dtype=torch.int8, device=DEVICE)
    kept[:, :w.shape[1]] = codes.to(torch.int8)
    return kept, scales.contiguous()


def _sizes(case):
    return [case["rows"] * case["cols"] + i * case["more"] for i in range(case["matrices"])] + \
           [case["length"] + i * case["more"] for i in range(case["vectors"])]


def _prepare_adamw(case, rand):
    # The tensors of a kind lie one behind the other in a buffer, matrices first; a state's blocks begin with each tensor.
    sizes = _sizes(case)
    blocks = [-(-n // BLOCK) for n in sizes]
    total, decayed = sum(sizes), sum(sizes[:case["matrices"]])
    whole = all(n % BLOCK == 0 for n in sizes)
    count = torch.tensor(sizes, device=DEVICE)
    tensor = torch.repeat_interleave(torch.arange(len(sizes), device=DEVICE), count)
    first_of = torch.cumsum(count, 0) - count
    index = torch.arange(total, device=DEVICE) - first_of[tensor]
    s = {"weight": rand(total, size=0.02, dtype=_type(case["weight_type"])), "decayed": decayed, "step": 100, "seed": 0x5241444941}
    # gradients differ in size from one row of 1001 to the next
    size = torch.exp(rand(total // 1001 + 1, size=1.5)).mul_(1e-4).repeat_interleave(1001)[:total]
    s["grad"] = (rand(total) * size).to(_type(case["grad_type"]))
    first, root = rand(total, size=0.3) * size, rand(total).abs_().add_(0.1) * size
    if case["states"] == "f32":
        s["first"], s["second"] = first, root.square_()
    else:
        if not whole:
            block_of = torch.cumsum(torch.tensor(blocks, device=DEVICE), 0)
            s["block"] = (block_of - torch.tensor(blocks, device=DEVICE))[tensor] + index // BLOCK
        s["blocks"] = sum(blocks)
        s["first"], s["first_scales"] = _state_codes(s, first, None, False)
        s["second"], s["second_scales"] = _state_codes(s, root, None, True)
    if case["rounding"] == "random" and case["states"] == "8bit":
        s["tensor"], s["index"] = tensor, index
    if case["copy"]:
        s["copy"] = torch.empty(total, dtype=torch.bfloat16, device=DEVICE)
    s["norm"] = torch.empty(2, device=DEVICE)
    if own:
        from paper_2506_19852_amd import layer
        cut = lambda name: list(s[name].split(sizes)) if name in s else None  # noqa: E731
        scales = lambda name: list(s[name].split(blocks)) if name in s else None  # noqa: E731
        tensors = layer.adamw_tensors(cut("weight"), cut("grad"), cut("first"), cut("second"), first_scales=scales("first_scales"),
                                      second_scales=scales("second_scales"), copies=cut("copy"),
                                      decay=[case["decay"]] * case["matrices"] + [0.0] * case["vectors"])
        s["plan"] = layer.radial_adamw_plan(tensors)
        s["table"] = torch.empty(s["plan"].table_bytes, dtype=torch.uint8, device=DEVICE)
        layer.radial_adamw_table(tensors, s["plan"], s["table"])
        s["workspace"] = torch.empty(layer.radial_grad_norm_workspace(s["plan"]), dtype=torch.uint8, device=DEVICE)
    return s


# ---- one pass -------------------------------------------------------------------------------

def run(state):
    op, direction = state["case"]["op"], state["case"].get("direction")
    if own:
        return {"adamw": _own_adamw, "linear": _own_linear_fwd if direction == "fwd" else _own_linear_bwd}[op](state)
    return {"adamw": _plain_adamw, "linear": _plain_linear_fwd if direction == "fwd" else _plain_linear_bwd}[op](state)


def _own_linear_fwd(s):
    from paper_2506_19852_amd import layer
    layer.radial_linear_i8_fwd(s["x"], s["w_codes"], s["w_scales"], s["out"], s["workspace"], bias=s.get("bias"))
    return s["out"]


def _own_linear_bwd(s):
    from paper_2506_19852_amd import layer
    layer.radial_linear_i8_bwd(s["dout"], s["workspace"], x=s["x"], wt_codes=s["wt_codes"], wt_scales=s["wt_scales"], dx=s["dx"], dw=s["dw"], dbias=s.get("dbias"))
    return {k: s[k] for k in ("dx", "dw", "dbias") if k in s}


def _own_adamw(s):
    from paper_2506_19852_amd import layer
    c = s["case"]
    factor = None
    if c["clip"]:
        layer.radial_grad_norm(s["plan"], s["table"], s["norm"], s["workspace"], max_norm=MAX_NORM)
        factor = s["norm"]
    layer.radial_adamw_step(s["plan"], s["table"], lr=LR, step=s["step"], beta1=BETA1, beta2=BETA2, eps=EPS, factor=factor, rounding=c["rounding"], seed=s["seed"])
    s["step"] += 1
    return _updated(s)


def _updated(s):
    """What a step changes; the codes of a state as the E4M3 values that they are."""
    out = {k: s[k] for k in ("weight", "copy", "first_scales", "second_scales") if k in s}
    for k in ("first", "second"):
        out[k] = s[k].view(torch.float8_e4m3fn) if s[k].dtype is torch.uint8 else s[k]
    if s["case"]["clip"]:
        out["norm"] = s["norm"]
    return out


def _plain_linear_fwd(s):
    codes, scales = _row_codes(s["x"])
    y = (codes @ s["w_codes"][:, :codes.shape[1]].float().t()) * (scales[:, None] * s["w_scales"][None, :])
    if "bias" in s:
        y = y + s["bias"]
    return s["out"].copy_(y)


def _plain_linear_bwd(s):
    codes, scales = _row_codes(s["dout"])
    s["dx"].copy_((codes @ s["wt_codes"][:, :codes.shape[1]].float().t()) * (scales[:, None] * s["wt_scales"][None, :]))
    of_dout, dout_scales = _row_codes(s["dout"].t())
    of_x, x_scales = _row_codes(s["x"].t())
    s["dw"].copy_((of_dout @ of_x.t()) * (dout_scales[:, None] * x_scales[None, :]))
    out = {"dx": s["dx"], "dw": s["dw"]}
    if "dbias" in s:
        out["dbias"] = s["dbias"].copy_(s["dout"].double().sum(0))
    return out


def _mixed(x):
    """32 bits of a number, mixed (whole numbers of 64 bits that hold 32)."""
    x = x ^ (x >> 16)
    x = (x * 0x9E3779B1) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0x6A09E667) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random_bits(s):
    """32 random bits for each value of a step: the low 16 for its first moment, the others for its second."""
    key = torch.tensor(0, dtype=torch.int64, device=DEVICE)
    for word in (s["seed"] & 0xFFFFFFFF, s["seed"] >> 32, s["step"] & 0xFFFFFFFF):
        key = _mixed(key ^ word)
    return _mixed(_mixed(key ^ s["tensor"]) ^ s["index"])


def _per_block(s, v):
    """The largest of each block of 128 values of a tensor."""
    if "block" not in s:
        return v.view(-1, BLOCK).amax(1)
    return torch.zeros(s["blocks"], device=DEVICE).scatter_reduce_(0, s["block"], v, "amax")


def _per_value(s, v):
    return v[s["block"]] if "block" in s else v.repeat_interleave(BLOCK)


def _state_codes(s, v, bits, positive):
    """E4M3 codes of v with a scale for each block: to nearest, or up with the probability of what is left; positive values stay positive."""
    largest = _per_block(s, v.abs())
    scales = largest / torch.full_like(largest, LARGEST_E4M3)
    inverse = torch.where(largest > 0, torch.full_like(largest, LARGEST_E4M3) / largest, 0.0)
    y = v * _per_value(s, inverse)
    if bits is None:
        y = y.to(torch.float8_e4m3fn)
    else:
        y64 = y.double()
        exponent = (torch.frexp(y64.abs())[1] - 1).clamp_min(-6)
        step = torch.ldexp(torch.ones_like(y64), exponent - 3)
        y = (torch.floor(y64.abs() / step + bits.double() / 65536.0) * step).clamp_max(LARGEST_E4M3).copysign(y64).float().to(torch.float8_e4m3fn)
    codes = y.view(torch.uint8)
    if positive:
        codes = torch.where((v > 0) & (codes == 0), 1, codes).to(torch.uint8)
    return codes, scales


def _plain_adamw(s):
    c = s["case"]
    g = s["grad"].float()
    if c["clip"]:
        norm = g.double().square().sum().sqrt()
        factor = (MAX_NORM / norm).clamp_max(1.0)
        s["norm"].copy_(torch.stack([norm, factor]))
        g = g * s["norm"][1]
    packed = c["states"] == "8bit"
    m, v = s["first"], s["second"]
    if packed:
        m = m.view(torch.float8_e4m3fn).float() * _per_value(s, s["first_scales"])
        root = v.view(torch.float8_e4m3fn).float() * _per_value(s, s["second_scales"])
        v = root * root
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + (g * g) * (1.0 - BETA2)
    root = v.sqrt()
    by_first = LR / (1.0 - BETA1 ** s["step"])
    by_second = 1.0 / math.sqrt(1.0 - BETA2 ** s["step"])
    w = s["weight"].float()
    w[:s["decayed"]].mul_(1.0 - LR * c["decay"])
    w = w - by_first * (m / (root * by_second + EPS))
    s["weight"].copy_(w)
    if "copy" in s:
        s["copy"].copy_(w)
    if packed:
        bits = _random_bits(s) if c["rounding"] == "random" else None
        codes, scales = _state_codes(s, m, bits & 0xFFFF if bits is not None else None, False)
        s["first"].copy_(codes), s["first_scales"].copy_(scales)
        codes, scales = _state_codes(s, root, bits >> 16 if bits is not None else None, True)
        s["second"].copy_(codes), s["second_scales"].copy_(scales)
    else:
        s["first"].copy_(m), s["second"].copy_(v)
    s["step"] += 1
    return _updated(s)


# ---- what a pass cannot do without ------------------------------------------------------------

def work(case):
    size = lambda name: 4 if name == "f32" else 2  # noqa: E731
    if case["op"] == "adamw":
        n = sum(_sizes(case))
        each = 2 * size(case["weight_type"]) + size(case["grad_type"]) + (16 if case["states"] == "f32" else 4) + (2 if case["copy"] else 0)
        scales = 16 * sum(-(-m // BLOCK) for m in _sizes(case)) if case["states"] == "8bit" else 0
        return {"bytes": n * each + scales, "flops": n * 16}
    M, N, K = case["M"], case["N"], case["K"]
    x, out = size(case["type"]), size(case["out_type"])
    if case["direction"] == "fwd":
        return {"bytes": x * M * K + N * K + out * M * N, "flops": 2 * M * N * K}
    return {"bytes": 2 * x * M * K + x * M * N + N * K + out * N * K, "flops": 4 * M * N * K}


# ---- 64 bits ----------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "adamw": _exact_adamw}[case["op"]](case, s)


def _whole64(x):
    """Whole numbers and the scales (values of 32 bits) of the rows of x."""
    x = x.double()
    scale = (x.abs().max(1).values.float() / torch.tensor(127.0, device=DEVICE)).double().clamp_min(2.0 ** -126)
    # a code is the whole number next to the quotient as a value of 32 bits: half of a row's largest is 63.5 there, and near it in 64
    return torch.round((x / scale[:, None]).float()).double(), scale


def _exact_linear(c, s):
    if c["direction"] == "fwd":
        a, sa = _whole64(s["x"])
        b = s["w_codes"][:, :c["K"]].double()
        y = sa[:, None] * (a @ b.t().contiguous()) * s["w_scales"].double()
        return y + s["bias"].double() if c["bias"] else y
    a, sa = _whole64(s["dout"])
    b = s["wt_codes"][:, :c["N"]].double()
    out = {"dx": sa[:, None] * (a @ b.t().contiguous()) * s["wt_scales"].double()}
    a, sa = _whole64(s["dout"].t().contiguous())
    b, sb = _whole64(s["x"].t().contiguous())
    out["dw"] = sa[:, None] * (a @ b.t().contiguous()) * sb
    if c["bias"]:
        out["dbias"] = s["dout"].double().sum(0)
    return out


def _exact_adamw(c, s):
    sizes, at, block = _sizes(c), 0, 0
    t = s["step"]
    factor = 1.0
    if c["clip"]:
        norm = float(torch.linalg.vector_norm(s["grad"].double()))
        factor = min(1.0, MAX_NORM / norm)
    names = ["weight", "first", "second"] + (["copy"] if c["copy"] else []) + (["first_scales", "second_scales"] if c["states"] == "8bit" else [])
    parts = {k: [] for k in names}
    for i, n in enumerate(sizes):
        of = slice(at, at + n)
        g = s["grad"][of].double() * factor
        if c["states"] == "8bit":
            blocks = -(-n // BLOCK)
            which = torch.arange(n, device=DEVICE) // BLOCK
            read = lambda k: s[k][of].view(torch.float8_e4m3fn).double() * s[k + "_scales"][block:block + blocks].double()[which]  # noqa: B023, E731
            m, r = read("first"), read("second")
            v = r ** 2
        else:
            m, v = s["first"][of].double(), s["second"][of].double()
        m = BETA1 * m + (1 - BETA1) * g
        v = BETA2 * v + (1 - BETA2) * g ** 2
        w = s["weight"][of].double() * (1 - LR * (c["decay"] if i < c["matrices"] else 0.0))
        w = w - LR * (m / (1 - BETA1 ** t)) / (torch.sqrt(v / (1 - BETA2 ** t)) + EPS)
        parts["weight"].append(w)
        if c["copy"]:
            parts["copy"].append(w)
        if c["states"] == "8bit":
            # the values that are rounded to codes, in units of their scales
            for k, x in (("first", m), ("second", v.sqrt())):
                largest = torch.nn.functional.pad(x.abs(), (0, blocks * BLOCK - n)).view(blocks, BLOCK).max(1).values
                parts[k].append(x / (largest / LARGEST_E4M3).clamp_min(1e-300)[which])
                parts[k + "_scales"].append(largest / LARGEST_E4M3)
            block += blocks
        else:
            parts["first"].append(m), parts["second"].append(v)
        at += n
    out = {k: torch.cat(v) for k, v in parts.items()}
    if c["clip"]:
        out["norm"] = torch.tensor([norm, factor], dtype=torch.float64, device=DEVICE)
    return out
