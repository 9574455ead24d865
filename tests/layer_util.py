"""What the tests of the layer operators share: tensors inside larger ones whose surroundings are watched, and error bounds."""
import numpy as np
import torch

DEV = "cuda:0"
U32 = 2.0 ** -24                                              # half a step of float32
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: U32}   # relative; torch.finfo(t).eps / 2
GUARD = 7.5


def to64(t):
    return t.detach().double().cpu().numpy()


def inside(values, dtype, lead=8, trail=8, rows=1):
    """A copy of `values` (array) as a view into a larger tensor: `rows` rows more along the last but one axis, `lead` and `trail` elements more
    along the last.  Returns (view, whole)."""
    shape = list(values.shape)
    shape[-1] += lead + trail
    if len(shape) > 1:
        shape[-2] += rows
    whole = torch.full(shape, GUARD, dtype=dtype, device=DEV)
    view = whole[..., lead:lead + values.shape[-1]]
    if len(shape) > 1:
        view = view[..., :values.shape[-2], :]
    view.copy_(torch.as_tensor(values).to(dtype))
    return view, whole


def surroundings_kept(view, whole):
    """Whether everything of `whole` outside of `view` still holds the guard."""
    rest = whole.clone()
    lead = (view.data_ptr() - whole.data_ptr()) // whole.element_size()
    part = rest.as_strided(view.shape, view.stride(), lead)
    part.fill_(GUARD)
    return bool((rest == GUARD).all())


def rounded(a, dtype):
    """The array after one rounding to dtype, in float64."""
    return torch.as_tensor(np.ascontiguousarray(a)).to(dtype).double().numpy()


def assert_within(got, want, bound, what):
    got = to64(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert np.isfinite(got).all(), f"{what}: values that are not finite"
    bad = np.abs(got - want) > bound
    worst = (np.abs(got - want) / np.maximum(bound, 1e-300)).max()
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} beyond the bound, at most {worst:.3g} times it"
