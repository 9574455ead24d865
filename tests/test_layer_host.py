"""The layer operators' interface without a GPU: the header's symbols, every refusal of the library before it launches anything, marshalling."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

from paper_2506_19852_amd import binding as rb
from paper_2506_19852_amd import layer as rl
from test_binding_host import FakeTensor

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, EUNSUPPORTED, ESHAPE = -1, -4, -5
BF16, F32 = rl.RADIAL_BF16, rl.RADIAL_F32
AT = 1 << 20  # an address that is never read


def test_header_symbols_are_exported():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "radial_layer.h")).read(), flags=re.S)
    names = set(re.findall(r"RADIAL_API\s+[\w\s\*]+?\b(radial_\w+)\s*\(", text))
    assert names == set(rl.EXPORTS) and not names & set(rb.EXPORTS)
    lib = ctypes.CDLL(rb.lib_path())
    for n in names:
        assert hasattr(lib, n), n


def test_structures_are_laid_out_as_the_header_says(tmp_path):
    import shutil
    import subprocess
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    src = tmp_path / "sizes.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "radial_layer.h"\nint main(void) {\n'
                   'printf("%zu %zu %zu %zu %zu %zu\\n", sizeof(radial_rows), sizeof(radial_norm_params), offsetof(radial_norm_params, mod_stride), '
                   'sizeof(radial_rope_params), offsetof(radial_rope_params, factor), offsetof(radial_rope_params, magnitude)); return 0; }\n')
    exe = tmp_path / "sizes"
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    got = [int(v) for v in subprocess.check_output([str(exe)], text=True).split()]
    assert got == [ctypes.sizeof(rl.radial_rows), ctypes.sizeof(rl.radial_norm_params), rl.radial_norm_params.mod_stride.offset,
                   ctypes.sizeof(rl.radial_rope_params), rl.radial_rope_params.factor.offset, rl.radial_rope_params.magnitude.offset]


def _refused(rc, code, text):
    assert rc == code and text in rb.radial_last_error(), (rc, rb.radial_last_error())


# ---- norms ------------------------------------------------------------------------------------

def _norm(direction="fwd", params=None, **change):
    lib = rl.load()
    p = dict(B=2, N=8, C=64, group=4, post=rl.RADIAL_NORM_RMS, pre=rl.RADIAL_NORM_LAYER, eps=1e-6, residual_scale=0.5, mod_stride=64, dmod_stride=64)
    p.update(params or {})
    p = rl.radial_norm_params(**p)
    rows = lambda t=BF16: rl.radial_rows(AT, 8 * 64, 64, t)  # noqa: E731
    a = dict(x=rows(), y=rows(), r=rows(), z=rows(), dz=rows(), dr=rows(), dx=rows(), dy=rows(), gate=AT, post_weight=AT, weight=AT, scale=AT, shift=AT,
             dgate=AT, dscale=AT, dshift=AT, dpost_weight=AT, dweight=AT, workspace=AT, bytes=1 << 30)
    a.update(change)
    for k in ("x", "y", "r", "z", "dz", "dr", "dx", "dy"):
        if a[k] is None:
            a[k] = rl.radial_rows(None, 0, 0, BF16)
    ref = ctypes.byref(p) if params != "null" else None
    if direction == "fwd":
        return lib.radial_norm_fwd(ref, a["x"], a["y"], a["gate"], a["post_weight"], a["weight"], a["scale"], a["shift"], a["r"], a["z"], None)
    return lib.radial_norm_bwd(ref, a["r"], a["y"], a["dz"], a["dr"], a["gate"], a["post_weight"], a["weight"], a["scale"], a["dx"], a["dy"], a["dgate"],
                               a["dscale"], a["dshift"], a["dpost_weight"], a["dweight"], a["workspace"], a["bytes"], None)


@pytest.mark.parametrize("params, code, text", [
    (dict(B=0), EINVAL, ">= 1"), (dict(N=0), EINVAL, ">= 1"), (dict(C=0), EINVAL, ">= 1"), (dict(group=0), EINVAL, ">= 1"), (dict(group=-3), EINVAL, ">= 1"),
    (dict(B=1 << 16, N=1 << 15), EINVAL, "2^31"), (dict(C=16385), EUNSUPPORTED, "16384"), (dict(post=3), EINVAL, "post"), (dict(pre=-1), EINVAL, "pre"),
    (dict(B=1, N=(1 << 31) - 1), EINVAL, "2^31"), (dict(B=1, N=(1 << 31) - 1024), EINVAL, "2^31"),  # rows behind the last would pass 32 bits
    (dict(eps=0.0), EINVAL, "eps"), (dict(eps=float("nan")), EINVAL, "eps"), (dict(eps=float("inf")), EINVAL, "eps"),
    (dict(residual_scale=float("inf")), EINVAL, "residual_scale"),
], ids=str)
def test_norm_parameters(params, code, text):
    for direction in ("fwd", "bwd"):
        _refused(_norm(direction, params), code, text)
    p = dict(B=2, N=8, C=64, group=4, post=2, pre=1, eps=1e-6, residual_scale=0.5, mod_stride=64, dmod_stride=64)
    p.update(params)
    assert rl.load().radial_norm_bwd_workspace(ctypes.byref(rl.radial_norm_params(**p))) == 0


def _at(ptr=AT, sb=512, sn=64, kind=BF16):
    return rl.radial_rows(ptr, sb, sn, kind)


@pytest.mark.parametrize("change, code, text", [
    (dict(x=None), EINVAL, "x.ptr"), (dict(r=None), EINVAL, "r.ptr"), (dict(z=None), EINVAL, "z.ptr"), (dict(x=_at(kind=2)), EINVAL, "x.type"),
    (dict(x=_at(AT + 1)), ESHAPE, "x.ptr"), (dict(z=_at(sn=63)), ESHAPE, "z strides"), (dict(y=_at(sb=-8)), ESHAPE, "y strides"),
    (dict(r=_at(kind=F32)), EINVAL, "x and r"), (dict(z=_at(kind=F32)), EINVAL, "y and z"), (dict(y=None), EINVAL, "without y"),
    (dict(gate=AT + 2), ESHAPE, "gate"), (dict(weight=AT + 1), ESHAPE, "weight"),
], ids=lambda v: str(list(v)) if isinstance(v, dict) else str(v))
def test_norm_tensors(change, code, text):
    _refused(_norm("fwd", **change), code, text)


def test_norm_parts_that_do_not_go_together():
    none = dict(pre=rl.RADIAL_NORM_NONE)
    _refused(_norm("fwd", none), EINVAL, "need a norm")
    _refused(_norm("fwd", none, z=None, weight=None, shift=None), EINVAL, "need a norm")
    _refused(_norm("fwd", dict(post=0)), EINVAL, "post_weight")
    _refused(_norm("fwd", dict(mod_stride=63)), ESHAPE, "stride of gate")
    _refused(_norm("bwd", dict(dmod_stride=63)), ESHAPE, "stride of dgate")
    alone = dict(y=None, r=None, gate=None, post_weight=None)
    _refused(_norm("fwd", dict(post=0), **alone), EINVAL, "without y")                        # residual_scale
    _refused(_norm("fwd", dict(post=0, pre=0, residual_scale=1.0), **alone, z=None, weight=None, scale=None, shift=None), EINVAL, "neither")
    _refused(_norm("bwd", none), EINVAL, "need a norm")
    parts = dict(dz=None, weight=None, scale=None, dscale=None, dshift=None, dweight=None)
    _refused(_norm("bwd", none, **{**parts, "dshift": AT}), EINVAL, "need a norm")
    _refused(_norm("bwd", none, **parts, dr=None), EINVAL, "dr.ptr")
    _refused(_norm("bwd", dy=None), EINVAL, "dy.ptr")
    _refused(_norm("bwd", dict(post=0), dpost_weight=None), EINVAL, "post_weight")
    _refused(_norm("bwd", dict(post=0), post_weight=None), EINVAL, "post_weight")
    _refused(_norm("bwd", y=None), EINVAL, "without y")
    for k, other in (("dr", "dx"), ("r", "dx"), ("dy", "y"), ("dz", "y")):
        _refused(_norm("bwd", **{k: _at(kind=F32)}), EINVAL, "one type")
    _refused(_norm("bwd", workspace=None), ESHAPE, "workspace")
    _refused(_norm("bwd", workspace=AT + 64), ESHAPE, "256-byte")
    need = rl.radial_norm_bwd_workspace(2, 8, 64, group=4, post=2, pre=1)
    _refused(_norm("bwd", bytes=need - 1), ESHAPE, "needed")
    many = dict(B=1 << 10, N=1 << 20, C=4096, group=1, mod_stride=4096, dmod_stride=4096)   # a workgroup of 512 threads for each token: beyond a launch
    wide = {k: rl.radial_rows(AT, 4096 << 20, 4096, BF16) for k in ("x", "y", "r", "z", "dz", "dr", "dx", "dy")}
    _refused(_norm("fwd", many, **wide), ESHAPE, "too many groups")
    _refused(_norm("bwd", many, **wide), ESHAPE, "too many groups")
    assert rl.radial_norm_bwd_workspace(2, 8, 64, group=1 << 31) == rl.radial_norm_bwd_workspace(2, 8, 64)


# ---- rotary positions ---------------------------------------------------------------------------

def _params(**change):
    p = rl.rope_params([4, 5, 6], [16, 24, 24], scaling="parts", factor=2.0, original=100)
    for k, v in change.items():
        if k[-1].isdigit():
            getattr(p, k[:-1])[int(k[-1])] = v
        else:
            setattr(p, k, v)
    return p


BAD_PARAMS = [
    (dict(axes=0), "axes"), (dict(axes=4), "axes"), (dict(layout=2), "layout"), (dict(size1=0), "size[1]"), (dict(size0=1 << 20, size1=1 << 20), "grid"),
    (dict(dims0=3), "dims[0]"), (dict(dims2=0), "dims[2]"), (dict(dims0=1026), "dims[0]"), (dict(dims0=1000), "dimensions"), (dict(scaling0=4), "scaling[0]"),
    (dict(scaling0=-1), "scaling[0]"), (dict(factor1=0.0), "factor[1]"), (dict(factor1=float("nan")), "factor[1]"), (dict(factor1=float("inf")), "factor[1]"),
    (dict(original2=0), "original[2]"), (dict(fast=1.0), "fast"), (dict(slow=-1.0), "fast"), (dict(fast=float("nan")), "fast"), (dict(theta=0.0), "theta"),
    (dict(theta=float("inf")), "theta"), (dict(magnitude=float("nan")), "magnitude"),
]


@pytest.mark.parametrize("change, text", BAD_PARAMS, ids=str)
def test_rope_parameters(change, text):
    p = _params(**change)
    assert rl.radial_rope_table_bytes(p) == 0
    _refused(rl.load().radial_rope_table(ctypes.byref(p), AT, 1 << 30, None), EINVAL, text)
    for direction in ("fwd", "bwd"):
        _refused(_rope(direction, p), EINVAL, text)


def _rope(direction="fwd", p=None, **change):
    t = rb.radial_tensor(AT, 4096, 128, 512)
    a = dict(table=AT, bytes=1 << 30, B=1, N=10, D=64, q_heads=4, q=t, q_out=t, k_heads=2, k=t, k_out=t, type=BF16, positions=None, first=0)
    a.update(change)
    fn = getattr(rl.load(), "radial_rope_" + direction)
    return fn(ctypes.byref(p or _params()), *a.values(), None)


def _heads(ptr=AT, sb=4096, sh=128, sn=512):
    return rb.radial_tensor(ptr, sb, sh, sn)


@pytest.mark.parametrize("change, code, text", [
    (dict(table=None), EINVAL, "table"), (dict(table=AT + 4), ESHAPE, "table"), (dict(bytes=(4 * 8 + 5 * 12 + 6 * 12) * 8 - 1), ESHAPE, "needed"), (dict(B=0), EINVAL, ">= 1"), (dict(N=-1), EINVAL, ">= 1"), (dict(q_heads=0), EINVAL, ">= 1"),
    (dict(D=4), EUNSUPPORTED, "head dimension"), (dict(D=68), EUNSUPPORTED, "head dimension"), (dict(D=1032), EUNSUPPORTED, "head dimension"), (dict(type=2), EINVAL, "type"),
    (dict(D=56), ESHAPE, "turn 64"), (dict(q=_heads(None)), EINVAL, "ptr is NULL"), (dict(q_out=_heads(AT + 8)), ESHAPE, "16-byte"), (dict(q=_heads(sn=56)), ESHAPE, "strides"),
    (dict(q=_heads(sn=516)), ESHAPE, "strides"), (dict(k=_heads(sh=-8)), ESHAPE, "strides"), (dict(k=_heads(None)), EINVAL, "ptr is NULL"),
    (dict(k_out=_heads(None)), EINVAL, "ptr is NULL"), (dict(k_heads=0), EINVAL, "k_heads"), (dict(k_heads=-1), EINVAL, "k_heads"), (dict(first=-1), EINVAL, "first"),
    (dict(positions=AT + 2), ESHAPE, "positions"), (dict(B=1 << 20, N=1 << 20), ESHAPE, "too large"),
], ids=lambda v: str(list(v.items())[0][0]) if isinstance(v, dict) else str(v))
def test_rope_arguments(change, code, text):
    for direction in ("fwd", "bwd"):
        _refused(_rope(direction, **change), code, text)


def test_rope_table_arguments():
    lib, p = rl.load(), _params()
    _refused(lib.radial_rope_table(None, AT, 1 << 30, None), EINVAL, "params")
    _refused(lib.radial_rope_table(ctypes.byref(p), None, 1 << 30, None), EINVAL, "table")
    _refused(lib.radial_rope_table(ctypes.byref(p), AT, 8, None), ESHAPE, "needed")
    _refused(lib.radial_rope_table(ctypes.byref(p), AT + 8, 1 << 30, None), ESHAPE, "table")
    assert rl.radial_rope_table_bytes(p) == (4 * 8 + 5 * 12 + 6 * 12) * 8
    assert lib.radial_rope_table_bytes(None) == 0
    for bad in (dict(sizes=[], dims=[]), dict(sizes=[1, 2], dims=[4]), dict(sizes=[1], dims=[4], layout="other"), dict(sizes=[1], dims=[4], scaling="other"),
                dict(sizes=[1, 2], dims=[4, 4], factor=[1.0])):
        with pytest.raises(ValueError):
            rl.rope_params(**bad)


# ---- products -----------------------------------------------------------------------------------

@pytest.mark.parametrize("change, code, text", [
    (dict(rows=0), EINVAL, ">= 1"), (dict(cols=-1), EINVAL, ">= 1"), (dict(x=None), EINVAL, "x is NULL"), (dict(type=7), EINVAL, "type"), (dict(grouping=2), EINVAL, "grouping"),
    (dict(codes=None), EINVAL, "together"), (dict(scales_t=None), EINVAL, "together"), (dict(codes=None, scales=None, codes_t=None, scales_t=None), EINVAL, "neither"),
    (dict(x=AT + 1), ESHAPE, "x is not"), (dict(stride=99), ESHAPE, "stride"), (dict(codes=AT + 8), ESHAPE, "codes"), (dict(codes_t=AT + 1), ESHAPE, "codes"),
    (dict(scales=AT + 2), ESHAPE, "scales"), (dict(rows=0x7fffffff, stride=1 << 40), ESHAPE, "too large"), (dict(rows=1 << 29, cols=1 << 19, stride=1 << 40), ESHAPE, "too large"),
], ids=str)
def test_quantise_arguments(change, code, text):
    a = dict(rows=10, cols=100, x=AT, type=BF16, stride=100, grouping=0, codes=AT, scales=AT, codes_t=AT, scales_t=AT)
    a.update(change)
    _refused(rl.load().radial_quantize_groups_fp8(*a.values(), None), code, text)


@pytest.mark.parametrize("change, code, text", [
    (dict(M=0), EINVAL, ">= 1"), (dict(N=0), EINVAL, ">= 1"), (dict(K=-5), EINVAL, ">= 1"), (dict(a=None), EINVAL, "NULL"), (dict(sa=None), EINVAL, "NULL"),
    (dict(b=None), EINVAL, "NULL"), (dict(sb=None), EINVAL, "NULL"), (dict(out=None), EINVAL, "NULL"), (dict(grouping=3), EINVAL, "b_grouping"), (dict(a=AT + 8), ESHAPE, "codes"),
    (dict(b=AT + 4), ESHAPE, "codes"), (dict(sb=AT + 2), ESHAPE, "scales"), (dict(out=AT + 1), ESHAPE, "out"), (dict(stride=9), ESHAPE, "out_stride"),
    (dict(K=0x7fffffff), ESHAPE, "too large"), (dict(M=(1 << 29) + 1), ESHAPE, "too large"), (dict(N=1 << 28, stride=1 << 28), ESHAPE, "too large"), (dict(M=1 << 29, N=1 << 29, stride=1 << 29), ESHAPE, "too large"),
], ids=str)
def test_product_arguments(change, code, text):
    a = dict(M=10, N=10, K=100, a=AT, sa=AT, b=AT, sb=AT, grouping=0, out=AT, stride=10)
    a.update(change)
    _refused(rl.load().radial_product_fp8(*a.values(), None), code, text)


# ---- marshalling --------------------------------------------------------------------------------

@pytest.fixture
def one_device(monkeypatch):
    rl.load()
    monkeypatch.setattr(rl, "_device", lambda: 0)


def _fake(dtype, *shape, device=0):
    t = FakeTensor(dtype, *shape)
    t.get_device = lambda: device
    full = t.stride()
    t.stride = lambda i=None: full if i is None else full[i]
    return t


def test_shapes_and_types_are_checked_before_the_library_is_entered(one_device):
    bf16, f32, u8, i32 = torch.bfloat16, torch.float32, torch.uint8, torch.int32
    x = _fake(bf16, 2, 8, 64)
    for bad in (dict(x=_fake(torch.float16, 2, 8, 64), r=None, z=x), dict(x=x, r=None, z=_fake(bf16, 2, 8, 32)), dict(x=x, r=None, z=x, weight=_fake(bf16, 64)),
                dict(x=x, r=None, z=x, scale=_fake(f32, 2, 64)), dict(x=x, r=None, z=x, scale=_fake(f32, 2, 1, 64), shift=_fake(f32, 2, 1, 64), group=4),
                dict(x=x, r=x, z=x, y=x, gate=_fake(f32, 2, 1, 32))):
        with pytest.raises(ValueError):
            rl.radial_norm_fwd(**bad, stream=1)
    wide = _fake(f32, 2, 1, 64)
    wide.stride = lambda i=None: (192, 192, 1) if i is None else (192, 192, 1)[i]
    with pytest.raises(ValueError, match="same strides"):
        rl.radial_norm_fwd(x, None, x, scale=wide, shift=_fake(f32, 2, 1, 64), stream=1)
    p, q = rl.rope_params([8], [64]), _fake(bf16, 1, 2, 8, 64)
    table = _fake(f32, 8 * 64)
    for bad in (dict(q=_fake(torch.float16, 1, 2, 8, 64), q_out=q), dict(q=q, q_out=_fake(bf16, 1, 2, 8, 128)), dict(q=q, q_out=q, k=q), dict(q=q, q_out=q, k=q, k_out=_fake(f32, 1, 2, 8, 64)),
                dict(q=q, q_out=q, positions=_fake(torch.int64, 1, 8)), dict(q=q, q_out=q, positions=_fake(i32, 8)), dict(q=q, q_out=q, first=1 << 31)):
        with pytest.raises(ValueError):
            rl.radial_rope_fwd(p, table, **bad, stream=1)
    with pytest.raises(rb.RadialError, match="needed"):
        rl.radial_rope_fwd(p, _fake(f32, 8 * 64 - 1), q, q, stream=1)
    m = _fake(bf16, 100, 200)
    codes, scales = _fake(u8, 100, 256), _fake(f32, 2, 100)
    for bad in ((_fake(torch.float16, 100, 200), codes, scales), (m, _fake(u8, 100, 200), scales), (m, codes, _fake(f32, 100, 2)), (m, codes, None), (m, None, scales),
                (m, None, None, codes, scales)):
        with pytest.raises(ValueError):
            rl.radial_quantize_groups_fp8(*bad, stream=1)
    out = _fake(bf16, 100, 300)
    b, sb = _fake(u8, 300, 256), _fake(f32, 2, 3)
    for bad in ((codes, scales, b, sb, _fake(f32, 100, 300)), (codes, scales, b, sb, _fake(bf16, 99, 300)), (codes, scales, _fake(u8, 300, 128), sb, out), (codes, scales, b, _fake(f32, 2, 4), out)):
        with pytest.raises(ValueError):
            rl.radial_product_fp8(*bad, stream=1)


def test_tensors_of_another_device_or_of_none_are_refused(one_device):
    bf16, f32, u8, i32 = torch.bfloat16, torch.float32, torch.uint8, torch.int32
    for other in (1, -1):
        x, there = _fake(bf16, 2, 8, 64), _fake(bf16, 2, 8, 64, device=other)
        mod = _fake(f32, 2, 1, 64, device=other)
        for bad in (dict(x=there, r=None, z=x), dict(x=x, r=None, z=there), dict(x=x, r=None, z=x, scale=mod), dict(x=x, r=None, z=x, weight=_fake(f32, 64, device=other)),
                    dict(x=x, r=there, z=x, y=x)):
            with pytest.raises(ValueError):
                rl.radial_norm_fwd(**bad, stream=1)
        for bad in (dict(dz=there), dict(dx=there), dict(workspace=_fake(u8, 1 << 20, device=other)), dict(dscale=mod)):
            with pytest.raises(ValueError):
                rl.radial_norm_bwd(**{**dict(r=x, dz=x, dx=x, workspace=_fake(u8, 1 << 20)), **bad}, stream=1)
        p, q, table = rl.rope_params([8], [64]), _fake(bf16, 1, 2, 8, 64), _fake(f32, 512)
        q_there = _fake(bf16, 1, 2, 8, 64, device=other)
        for bad in (dict(q=q_there), dict(q_out=q_there), dict(k=q, k_out=q_there), dict(table=_fake(f32, 512, device=other)), dict(positions=_fake(i32, 1, 8, device=other))):
            with pytest.raises(ValueError):
                rl.radial_rope_bwd(p, **{"dq_out" if k == "q" else "dq" if k == "q_out" else "dk_out" if k == "k" else "dk" if k == "k_out" else k: v
                                         for k, v in {**dict(q=q, q_out=q, table=table), **bad}.items()}, stream=1)
        m, codes, scales = _fake(bf16, 100, 200), _fake(u8, 100, 256), _fake(f32, 2, 100)
        for bad in ((_fake(bf16, 100, 200, device=other), codes, scales), (m, _fake(u8, 100, 256, device=other), scales), (m, codes, _fake(f32, 2, 100, device=other))):
            with pytest.raises(ValueError):
                rl.radial_quantize_groups_fp8(*bad, stream=1)
        for i in range(5):
            args = [codes, scales, _fake(u8, 300, 256), _fake(f32, 2, 300), _fake(bf16, 100, 300)]
            args[i] = _fake(args[i].dtype, *args[i].shape, device=other)
            with pytest.raises(ValueError):
                rl.radial_product_fp8(*args, stream=1)


def test_numpy_numbers_and_defaults():
    p = rl.rope_params(np.array([3, 4]), [8, np.int64(8)], scaling=["linear", "none"], factor=[4.0, 1.0])
    assert list(p.size)[:2] == [3, 4] and list(p.scaling)[:2] == [1, 0] and p.theta == 1e4


def test_sizes_beyond_32_bits_are_refused_not_cut(one_device):
    bf16, f32, u8 = torch.bfloat16, torch.float32, torch.uint8
    more = (1 << 32) + 8
    for shape in ((2, more, 64), (1 << 16, 1 << 15, 64), (more, 8, 64), (2, 8, more)):
        x = _fake(bf16, *shape)
        with pytest.raises(ValueError, match="2\\^31"):
            rl.radial_norm_fwd(x, None, x, stream=1)
        with pytest.raises(ValueError, match="2\\^31"):
            rl.radial_norm_bwd(x, x, x, _fake(u8, 1 << 20), stream=1)
    for shape in ((more, 8, 64), (2, more, 64), (2, 8, more)):
        with pytest.raises(ValueError, match="2\\^31"):
            rl.radial_norm_bwd_workspace(*shape)
    x = _fake(bf16, 2, 8, 64)
    with pytest.raises(rb.RadialError, match=">= 1"):
        rl.radial_norm_fwd(x, None, x, group=4 - (1 << 32), stream=1)
    p, table, q = rl.rope_params([8], [64]), _fake(f32, 512), _fake(bf16, 1, 2, 8, 64)
    for shape in ((more, 2, 8, 64), (1, more, 8, 64), (1, 2, more, 64), (1, 2, 8, more)):
        big = _fake(bf16, *shape)
        with pytest.raises(ValueError, match="2\\^31"):
            rl.radial_rope_fwd(p, table, big, big, stream=1)
    keys = _fake(bf16, 1, more, 8, 64)
    with pytest.raises(ValueError, match="2\\^31"):
        rl.radial_rope_fwd(p, table, q, q, keys, keys, stream=1)
    for first in (1 << 31, more, 8 - (1 << 32)):
        with pytest.raises(ValueError, match="2\\^31"):
            rl.radial_rope_fwd(p, table, q, q, first=first, stream=1)
    for bad in (dict(sizes=[more]), dict(dims=[more]), dict(original=more)):
        with pytest.raises(ValueError, match="2\\^31"):
            rl.rope_params(**{**dict(sizes=[8], dims=[64]), **bad})
    for rows, cols in ((more, 128), (128, more)):
        with pytest.raises(ValueError, match="2\\^31"):
            rl.radial_quantize_groups_fp8(_fake(bf16, rows, cols), _fake(u8, rows, cols), _fake(f32, -(-cols // 128), rows), stream=1)
    for M, N, K in ((more, 128, 128), (128, more, 128), (128, 128, (1 << 32) + 128)):
        with pytest.raises(ValueError, match="2\\^31"):
            rl.radial_product_fp8(_fake(u8, M, K), _fake(f32, K // 128, M), _fake(u8, N, K), _fake(f32, K // 128, N), _fake(bf16, M, N), stream=1)


@pytest.mark.parametrize("change", [dict(original=np.int64(100)), dict(factor=np.float32(2.0)), dict(factor=np.int32(2)), dict(scaling=np.str_("linear"), factor=2)], ids=str)
def test_one_number_of_numpy_is_for_all_axes(change):
    p = rl.rope_params([3, 4], [8, 8], **change)
    q = rl.rope_params([3, 4], [8, 8], **{k: [v, v] for k, v in change.items()})
    assert bytes(p) == bytes(q)
