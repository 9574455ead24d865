"""The 8-bit integer products and AdamW without a GPU: every refusal of the library before it launches anything, layouts, marshalling."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import step as os_
from paper_2506_19852_amd import binding as rb
from paper_2506_19852_amd import layer as rl
from test_layer_host import AT, BF16, EINVAL, ESHAPE, EUNSUPPORTED, F32, ROOT, _fake, _refused, one_device  # noqa: F401

I8, U8, T32, T16 = torch.int8, torch.uint8, torch.float32, torch.bfloat16


def test_structures_are_laid_out_as_the_header_says(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    fields = [(s, f) for s in (rl.radial_adamw_tensor, rl.radial_adamw_plan_info, rl.radial_adamw_params) for f, _ in s._fields_]
    src = tmp_path / "sizes.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "radial_layer.h"\nint main(void) {\n' + "".join(
        f'printf("%zu %zu\\n", offsetof({s.__name__}, {f}), sizeof({s.__name__}));\n' for s, f in fields) + "return 0; }\n")
    exe = tmp_path / "sizes"
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    got = [tuple(int(v) for v in line.split()) for line in subprocess.check_output([str(exe)], text=True).strip().split("\n")]
    assert got == [(getattr(s, f).offset, ctypes.sizeof(s)) for s, f in fields]


# ---- integer products -----------------------------------------------------------------------------

@pytest.mark.parametrize("change, code, text", [
    (dict(rows=0), EINVAL, ">= 1"), (dict(cols=-1), EINVAL, ">= 1"), (dict(x=None), EINVAL, "x is NULL"), (dict(type=7), EINVAL, "type"),
    (dict(codes=None), EINVAL, "together"), (dict(scales_t=None), EINVAL, "together"),
    (dict(codes=None, scales=None, codes_t=None, scales_t=None, sums_t=None), EINVAL, "none of"), (dict(x=AT + 1), ESHAPE, "x is not"), (dict(stride=99), ESHAPE, "stride"),
    (dict(codes=AT + 8), ESHAPE, "codes"), (dict(codes_t=AT + 1), ESHAPE, "codes"), (dict(scales=AT + 2), ESHAPE, "scales"), (dict(sums_t=AT + 1), ESHAPE, "sums_t"),
    (dict(workspace=None), EINVAL, "workspace"), (dict(bytes=10), EINVAL, "needed"), (dict(workspace=AT + 128), ESHAPE, "256-byte"),
    (dict(rows=0x7fffffff), ESHAPE, "too large"), (dict(cols=0x7fffffff, stride=1 << 40), ESHAPE, "too large"),
    (dict(rows=1 << 28, codes_t=None, scales_t=None, sums_t=None), ESHAPE, "too large"), (dict(cols=1 << 29, rows=1 << 20, stride=1 << 29, codes=None, scales=None, codes_t=None, scales_t=None, bytes=1), EINVAL, "needed"),
], ids=str)
def test_quantise_arguments(change, code, text):
    a = dict(rows=10, cols=100, x=AT, type=BF16, stride=100, codes=AT, scales=AT, codes_t=AT, scales_t=AT, sums_t=AT, accumulate=0, workspace=AT, bytes=1 << 30)
    a.update(change)
    _refused(rl.load().radial_quantize_rows_i8(*a.values(), None), code, text)


@pytest.mark.parametrize("change, code, text", [
    (dict(M=0), EINVAL, ">= 1"), (dict(N=0), EINVAL, ">= 1"), (dict(K=-5), EINVAL, ">= 1"), (dict(a=None), EINVAL, "NULL"), (dict(sa=None), EINVAL, "NULL"),
    (dict(b=None), EINVAL, "NULL"), (dict(sb=None), EINVAL, "NULL"), (dict(out=None), EINVAL, "NULL"), (dict(type=3), EINVAL, "type"), (dict(accumulate=1), EINVAL, "float32"),
    (dict(K=131072), EUNSUPPORTED, "float32"), (dict(a=AT + 8), ESHAPE, "codes"), (dict(b=AT + 4), ESHAPE, "codes"), (dict(sb=AT + 2), ESHAPE, "scales"),
    (dict(bias=AT + 2), ESHAPE, "bias"), (dict(out=AT + 1), ESHAPE, "out"), (dict(out=AT + 2, type=F32), ESHAPE, "out"), (dict(stride=9), ESHAPE, "stride"),
    (dict(K=(1 << 23) + 1), ESHAPE, "too large"), (dict(M=(1 << 29) + 1), ESHAPE, "too large"), (dict(M=2, N=1 << 28, stride=1 << 28), ESHAPE, "too large"),
    (dict(M=1 << 29, N=1 << 29, stride=1 << 29), ESHAPE, "too large"),
], ids=str)
def test_product_arguments(change, code, text):
    a = dict(M=10, N=10, K=100, a=AT, sa=AT, b=AT, sb=AT, bias=AT, out=AT, type=BF16, stride=10, accumulate=0)
    a.update(change)
    _refused(rl.load().radial_product_i8(*a.values(), None), code, text)


@pytest.mark.parametrize("change, code, text", [
    (dict(M=0), EINVAL, ">= 1"), (dict(K=(1 << 23) + 1, x_stride=1 << 24), ESHAPE, "too large"), (dict(x=None), EINVAL, "x is NULL"), (dict(type=-1), EINVAL, "type"),
    (dict(x=AT + 1), ESHAPE, "x is not"), (dict(x_stride=99), ESHAPE, "stride of x"), (dict(w=None), EINVAL, "w codes"), (dict(w=AT + 1), ESHAPE, "w codes"), (dict(ws=AT + 1), ESHAPE, "w scales"),
    (dict(bias=AT + 1), ESHAPE, "bias"), (dict(y=None), EINVAL, "y is NULL"), (dict(y_type=9), EINVAL, "type of y"), (dict(y_stride=9), ESHAPE, "stride"),
    (dict(workspace=None), EINVAL, "workspace"), (dict(bytes=1), EINVAL, "needed"), (dict(workspace=AT + 16), ESHAPE, "256-byte"),
], ids=str)
def test_projection_arguments(change, code, text):
    a = dict(M=10, N=10, K=100, x=AT, type=BF16, x_stride=100, w=AT, ws=AT, bias=None, y=AT, y_type=BF16, y_stride=10, workspace=AT, bytes=1 << 30)
    a.update(change)
    _refused(rl.load().radial_linear_i8_fwd(*a.values(), None), code, text)


@pytest.mark.parametrize("change, code, text", [
    (dict(M=0), EINVAL, ">= 1"), (dict(N=(1 << 23) + 1), ESHAPE, "too large"), (dict(dy=None), EINVAL, "dy is NULL"), (dict(type=2), EINVAL, "type"), (dict(dy=AT + 1), ESHAPE, "dy is not"),
    (dict(dy_stride=9), ESHAPE, "stride of dy"), (dict(dx=None, dw=None, dbias=None), EINVAL, "none of"), (dict(wt=None), EINVAL, "wt codes"), (dict(wts=AT + 1), ESHAPE, "wt scales"),
    (dict(dx_type=5), EINVAL, "type of dx"), (dict(dx_stride=99), ESHAPE, "dx"), (dict(x=None), EINVAL, "x is NULL"), (dict(x=AT + 1), ESHAPE, "x is not"), (dict(x_stride=3), ESHAPE, "stride of x"),
    (dict(dw=AT + 2), ESHAPE, "dw"), (dict(dw_type=BF16, accumulate=1), EINVAL, "float32"), (dict(M=131072, dw_type=BF16), EUNSUPPORTED, "dw has to be float32"),
    (dict(dbias=AT + 1), ESHAPE, "dbias"), (dict(workspace=None), EINVAL, "workspace"), (dict(bytes=1), EINVAL, "needed"), (dict(workspace=AT + 16), ESHAPE, "256-byte"),
], ids=str)
def test_gradient_arguments(change, code, text):
    a = dict(M=10, N=10, K=100, dy=AT, type=BF16, dy_stride=10, x=AT, x_stride=100, wt=AT, wts=AT, dx=AT, dx_type=BF16, dx_stride=100, dw=AT, dw_type=F32, dw_stride=100,
             dbias=AT, accumulate=0, workspace=AT, bytes=1 << 40)
    a.update(change)
    _refused(rl.load().radial_linear_i8_bwd(*a.values(), None), code, text)


def test_workspaces():
    lib = rl.load()
    for call, sizes in ((lib.radial_quantize_rows_i8_workspace, (0, 5)), (lib.radial_linear_i8_fwd_workspace, (1, 0, 1)), (lib.radial_linear_i8_bwd_workspace, (1, 1, -1)),
                        (lib.radial_linear_i8_fwd_workspace, (1, 1, (1 << 23) + 1)), (lib.radial_linear_i8_bwd_workspace, ((1 << 23) + 1, 1, 1))):
        assert call(*sizes) == 0
    assert rl.radial_quantize_rows_i8_workspace(1, 1) >= 8
    assert rl.radial_linear_i8_fwd_workspace(10, 7, 100) >= 10 * 128 + 40
    assert rl.radial_linear_i8_bwd_workspace(10, 7, 100) >= 10 * 128 + 7 * 128 + 100 * 128
    with pytest.raises(ValueError, match="2\\^31"):
        rl.radial_linear_i8_fwd_workspace(1 << 32, 1, 1)


def test_shapes_types_and_devices_are_checked_before_the_library_is_entered(one_device):  # noqa: F811
    x, codes, scales, work = _fake(T16, 10, 100), _fake(I8, 10, 128), _fake(T32, 10), _fake(U8, 1 << 20)
    there = lambda t: _fake(t.dtype, *t.shape, device=1)  # noqa: E731
    for bad in ((_fake(torch.float16, 10, 100), codes, scales), (there(x), codes, scales), (x, _fake(I8, 10, 100), scales), (x, _fake(U8, 10, 128), scales), (x, codes, _fake(T32, 11)),
                (x, codes, None), (x, None, scales), (x, codes, there(scales)), (x, None, None, codes, scales, work), (x, codes, scales, None, None, there(work))):
        with pytest.raises(ValueError):
            rl.radial_quantize_rows_i8(*bad, stream=1)
    with pytest.raises(ValueError):
        rl.radial_quantize_rows_i8(x, workspace=work, sums_t=_fake(T32, 10), stream=1)
    w, ws, out = _fake(I8, 30, 128), _fake(T32, 30), _fake(T16, 10, 30)
    for bad in ((codes, scales, w, ws, _fake(torch.float16, 10, 30)), (codes, scales, w, ws, _fake(T16, 11, 30)), (codes, scales, _fake(I8, 30, 256), ws, out), (codes, scales, w, there(ws), out),
                (codes, scales, w, ws, there(out))):
        with pytest.raises(ValueError):
            rl.radial_product_i8(*bad, stream=1)
    with pytest.raises(ValueError):
        rl.radial_product_i8(codes, scales, w, ws, out, bias=_fake(T16, 30), stream=1)
    with pytest.raises(ValueError, match="2\\^31"):
        rl.radial_product_i8(_fake(I8, 1 << 32, 128), _fake(T32, 1 << 32), w, ws, _fake(T16, 1 << 32, 30), stream=1)
    for bad in (dict(x=there(x)), dict(w=_fake(I8, 30, 100)), dict(y=_fake(T16, 9, 30)), dict(bias=_fake(T32, 31)), dict(work=there(work)), dict(y=there(out))):
        a = {**dict(x=x, w=w, ws=ws, y=out, work=work, bias=None), **bad}
        with pytest.raises(ValueError):
            rl.radial_linear_i8_fwd(a["x"], a["w"], a["ws"], a["y"], a["work"], bias=a["bias"], stream=1)
    wt, wts, dx, dw = _fake(I8, 100, 128), _fake(T32, 100), _fake(T16, 10, 100), _fake(T32, 30, 100)
    for bad in (dict(x=None), dict(x=_fake(T32, 10, 100)), dict(x=there(x)), dict(wt_codes=_fake(I8, 100, 256)), dict(dx=_fake(T16, 10, 101)), dict(dw=_fake(T32, 30, 99)), dict(dbias=_fake(T32, 29))):
        with pytest.raises(ValueError):
            rl.radial_linear_i8_bwd(out, work, **{**dict(x=x, wt_codes=wt, wt_scales=wts, dx=dx, dw=dw), **bad}, stream=1)


# ---- AdamW ----------------------------------------------------------------------------------------

def _tensor(**change):
    return rl.radial_adamw_tensor(**{**dict(weight=AT, copy=None, grad=AT, first=AT, second=AT, first_scales=None, second_scales=None, n=5000, weight_type=F32, grad_type=BF16, decay=0.1), **change})


def _plan(*tensors):
    plan, array = rl.radial_adamw_plan_info(), (rl.radial_adamw_tensor * len(tensors))(*tensors)
    return rl.load().radial_adamw_plan(array, len(tensors), ctypes.byref(plan)), plan, array


@pytest.mark.parametrize("change, code, text", [
    (dict(n=-1), EINVAL, "n must"), (dict(n=1 << 40), EINVAL, "n must"), (dict(weight_type=2), EINVAL, "types"), (dict(grad_type=-1), EINVAL, "types"), (dict(decay=-0.1), EINVAL, "decay"),
    (dict(decay=float("nan")), EINVAL, "decay"), (dict(decay=float("inf")), EINVAL, "decay"), (dict(first_scales=AT), EINVAL, "together"), (dict(weight=None), EINVAL, "NULL"),
    (dict(grad=None), EINVAL, "NULL"), (dict(second=None), EINVAL, "NULL"), (dict(weight=AT + 2), ESHAPE, "aligned"), (dict(grad=AT + 1), ESHAPE, "aligned"), (dict(copy=AT + 1), ESHAPE, "aligned"),
    (dict(first=AT + 2), ESHAPE, "aligned"), (dict(first_scales=AT, second_scales=AT + 2), ESHAPE, "aligned"), (dict(n=(1 << 35) + 1), ESHAPE, "2^23"),
], ids=str)
def test_tensors(change, code, text):
    rc, _, _ = _plan(_tensor(), _tensor(**change))
    _refused(rc, code, "tensor 1" if text != "2^23" else text)
    assert text in rb.radial_last_error()


def test_plan_and_table():
    lib = rl.load()
    rc, plan, array = _plan(_tensor(), _tensor(n=0, weight=None, grad=None, first=None, second=None), _tensor(n=4096), _tensor(first=AT + 1, second=AT + 3, first_scales=AT, second_scales=AT))
    assert rc == 0 and (plan.count, plan.pieces) == (4, 5) and plan.table_bytes == 4 * 72 + 5 * 8
    _refused(lib.radial_adamw_plan(None, 1, ctypes.byref(plan)), EINVAL, "NULL")
    _refused(lib.radial_adamw_plan(array, 0, ctypes.byref(plan)), EINVAL, "count")
    table = lambda p=plan, at=AT, size=1 << 20: lib.radial_adamw_table(array, ctypes.byref(p) if p else None, at, size, None)  # noqa: E731
    _refused(table(p=None), EINVAL, "plan is NULL")
    _refused(table(at=None), EINVAL, "table")
    _refused(table(size=plan.table_bytes - 1), EINVAL, "needed")
    _refused(table(at=AT + 8), ESHAPE, "16-byte")
    _refused(table(p=rl.radial_adamw_plan_info(4, 6, 4 * 72 + 6 * 8)), EINVAL, "not that of")
    _refused(table(p=rl.radial_adamw_plan_info(4, 6, 1)), EINVAL, "not one of")
    assert lib.radial_grad_norm_workspace(None) == 0 and lib.radial_grad_norm_workspace(ctypes.byref(plan)) == 40


@pytest.mark.parametrize("change, code, text", [
    (dict(lr=-1.0), EINVAL, "lr"), (dict(lr=float("nan")), EINVAL, "lr"), (dict(beta1=1.0), EINVAL, "beta"), (dict(beta2=-0.1), EINVAL, "beta"), (dict(eps=0.0), EINVAL, "eps"),
    (dict(eps=1e-60), EINVAL, "eps"), (dict(eps=float("inf")), EINVAL, "eps"), (dict(step=0), EINVAL, "step"), (dict(rounding=2), EINVAL, "rounding"), (dict(factor=AT + 1), ESHAPE, "factor"),
    (dict(lr_at=AT + 2), ESHAPE, "lr_at"), (dict(step_at=AT + 4), ESHAPE, "step_at"),
], ids=str)
def test_step_arguments(change, code, text):
    _, plan, _ = _plan(_tensor())
    p = rl.radial_adamw_params(**{**dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, seed=0, rounding=0), **change})
    _refused(rl.load().radial_adamw_step(ctypes.byref(p), ctypes.byref(plan), AT, 1 << 20, None), code, text)
    good = rl.radial_adamw_params(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
    _refused(rl.load().radial_adamw_step(None, ctypes.byref(plan), AT, 1 << 20, None), EINVAL, "params")
    _refused(rl.load().radial_adamw_step(ctypes.byref(good), ctypes.byref(plan), None, 1 << 20, None), EINVAL, "table")


@pytest.mark.parametrize("change, code, text", [
    (dict(scale=0.0), EINVAL, "scale"), (dict(scale=float("inf")), EINVAL, "scale"), (dict(max_norm=0.0), EINVAL, "max_norm"), (dict(max_norm=float("nan")), EINVAL, "max_norm"),
    (dict(norm=None), EINVAL, "norm"), (dict(norm=AT + 2), ESHAPE, "norm"), (dict(workspace=None), EINVAL, "workspace"), (dict(bytes=0), EINVAL, "needed"), (dict(workspace=AT + 4), ESHAPE, "8-byte"),
], ids=str)
def test_norm_arguments(change, code, text):
    _, plan, _ = _plan(_tensor())
    a = {**dict(scale=1.0, max_norm=1.0, norm=AT, workspace=AT, bytes=1 << 20), **change}
    _refused(rl.load().radial_grad_norm(ctypes.byref(plan), AT, 1 << 20, *a.values(), None), code, text)


def _at(t, address):
    t.data_ptr = lambda: address
    t.element_size = lambda: torch.empty((), dtype=t.dtype).element_size()
    return t


def _lists(n=(300, 200), coded=False, at=1 << 16):
    """Fake tensors one behind the other."""
    out = {"weights": T32, "grads": T16, "firsts": U8 if coded else T32, "seconds": U8 if coded else T32, "copies": T16}
    if coded:
        out.update(first_scales=T32, second_scales=T32)
    for name, dtype in out.items():
        out[name] = []
        for k in n:
            size = -(-k // 128) if name.endswith("scales") else k
            out[name].append(_at(_fake(dtype, size), at))
            at += 4 * size
    return out


def test_lists_of_tensors(one_device):  # noqa: F811
    for coded in (False, True):
        array = rl.adamw_tensors(**_lists(coded=coded), decay=[0.0, 0.5])
        assert [e.n for e in array] == [300, 200] and [e.decay for e in array] == [0.0, 0.5] and bool(array[0].first_scales) == coded
        assert array[1].weight - array[0].weight == 1200 and array[0].weight_type == F32 and array[0].grad_type == BF16
        for name in _lists(coded=coded):
            for wrong in (_fake(torch.float16, 300), _fake(T32, 299), None, _fake(T32, 300, device=1)):
                if name == "copies" and wrong is None:
                    continue
                lists = _lists(coded=coded)
                lists[name][0] = wrong if wrong is None else _at(wrong, 1 << 30)
                with pytest.raises(ValueError):
                    rl.adamw_tensors(**lists)
            lists = _lists(coded=coded)
            lists[name] = lists[name][:1]
            if name == "weights":
                continue
            with pytest.raises(ValueError, match="one entry"):
                rl.adamw_tensors(**lists)
    with pytest.raises(ValueError, match="one entry"):
        rl.adamw_tensors(**_lists(), decay=[0.1])


def test_tensors_that_overlap_are_refused(one_device):  # noqa: F811
    for name, other in (("weights", "weights"), ("firsts", "weights"), ("grads", "weights"), ("weights", "grads"), ("copies", "seconds")):
        lists = _lists()
        _at(lists[name][1], lists[other][0].data_ptr() + 4)
        with pytest.raises(ValueError, match="overlaps"):
            rl.adamw_tensors(**lists)
    lists = _lists()
    _at(lists["grads"][1], lists["grads"][0].data_ptr())   # only read
    rl.adamw_tensors(**lists)


def test_step_marshalling(one_device):  # noqa: F811
    _, plan, _ = _plan(_tensor())
    table, norm = _fake(U8, plan.table_bytes), _fake(T32, 2)
    for bad in (dict(rounding="up"), dict(seed=-1), dict(seed=1 << 64), dict(step=1 << 63), dict(factor=_fake(T32, 1)), dict(lr_at=_fake(T16, 1)), dict(step_at=_fake(torch.int32, 1)),
                dict(step_at=_fake(torch.int64, 2)), dict(factor=_fake(T32, 2, device=1))):
        with pytest.raises(ValueError):
            rl.radial_adamw_step(plan, table, **{**dict(lr=1e-3, step=1, factor=norm), **bad}, stream=1)
    with pytest.raises(rb.RadialError, match="step"):
        rl.radial_adamw_step(plan, table, lr=1e-3, stream=1)
    with pytest.raises(rb.RadialError, match="needed"):
        rl.radial_adamw_step(plan, _fake(U8, plan.table_bytes - 1), lr=1e-3, step=1, stream=1)
    for bad in (dict(norm=_fake(T32, 3)), dict(workspace=_fake(U8, 64, device=1)), dict(table=_fake(U8, plan.table_bytes, device=-1))):
        a = {**dict(table=table, norm=norm, workspace=_fake(U8, 64)), **bad}
        with pytest.raises(ValueError):
            rl.radial_grad_norm(plan, a["table"], a["norm"], a["workspace"], stream=1)


def test_numbers_of_numpy(one_device):  # noqa: F811
    array = rl.adamw_tensors(**_lists(), decay=np.float32(0.5))
    assert [e.decay for e in array] == [0.5, 0.5]
    _, plan, _ = _plan(_tensor())
    with pytest.raises(rb.RadialError, match="needed"):   # the last check before the launch
        rl.radial_adamw_step(plan, _fake(U8, plan.table_bytes - 1), lr=np.float32(1e-3), step=np.int64(3), seed=np.int32(5), eps=np.float64(1e-8), stream=1)
    with pytest.raises(TypeError):
        rl.radial_adamw_step(plan, _fake(U8, plan.table_bytes), lr=1e-3, step=1.5, stream=1)


def test_a_step_without_a_rate_is_refused(one_device):  # noqa: F811
    """It would move the states and leave the weights, and report success."""
    _, plan, _ = _plan(_tensor())
    small = _fake(U8, plan.table_bytes - 1)   # the last check before the launch
    with pytest.raises(ValueError, match="lr or lr_at"):
        rl.radial_adamw_step(plan, small, step=1, stream=1)
    for how in (dict(lr=0.0), dict(lr=1e-3), dict(lr_at=_fake(T32, 1)), dict(lr=1e-3, lr_at=_fake(T32, 1))):
        with pytest.raises(rb.RadialError, match="needed"):
            rl.radial_adamw_step(plan, small, step=1, stream=1, **how)


# ---- the oracle itself --------------------------------------------------------------------------

def test_codes_of_the_oracle():
    x = np.array([[1.0, -0.5, 0.25, 0.0], [np.nan, 1, 2, 3], [0, 0, 0, 0], [1e-45, 0, 0, 0]], np.float32)
    codes, scales = os_.quantize_rows(x)
    assert codes.shape == (4, 128) and codes[0, 0] == 127 and abs(int(codes[0, 1])) in (63, 64) and codes[0, 2] == 32 and not codes[1:].any()
    assert np.isnan(scales[1]) and scales[2] == scales[3] == np.float32(2.0 ** -126)


def test_rounding_of_the_oracle():
    v = np.linspace(-3, 3, 500).astype(np.float32)
    for bits in (None, np.full(500, 0), np.full(500, 65535)):
        codes, scales = os_.encode(v, bits)
        got = os_.decode(codes, scales)
        step = np.maximum(np.abs(v) * 2.0 ** -3, np.repeat(scales, 128)[:500] * 2.0 ** -9)
        assert (np.abs(got - v) <= (0.51 if bits is None else 1.0) * step).all()
    codes, scales = os_.encode(np.array([1.0, 1e-12, 0.0], np.float32), positive=True)
    assert codes.tolist() == [0x7e, 1, 0]


def test_update_of_the_oracle_is_the_textbooks():
    g = np.array([0.3, -0.2])
    m, v = os_.moments(g, np.zeros(2), np.zeros(2), 0.9, 0.999)
    w = os_.update(np.array([1.0, 2.0]), m, v, 0.01, 1, 0.9, 0.999, 0.0, 0.1)
    assert np.allclose(w, np.array([1.0, 2.0]) * 0.999 - 0.01 * np.sign(g), rtol=0, atol=1e-12)   # the first step is the rate along each sign
