"""Helpers of the step operators' tests: tensors with guard bands, spread rows, and bounds."""
import torch

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
#: largest relative error of one rounding to the type (8 and 24 significant bits)
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def spread(t, pad):
    """The same values in rows `pad` elements further apart (NaN between them)."""
    full = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device=t.device)
    full[:, :t.shape[1]] = t
    return full[:, :t.shape[1]]


def within(got, ref, bound):
    """Every element of `got` within `bound` (same shape, or a number) of fp64 `ref`."""
    err = (got.double() - ref).abs()
    bad = ~(err <= bound)
    assert not bool(bad.any()), "%d of %d elements off, worst excess %.3g at error %.3g" % (
        int(bad.sum()), err.numel(), float((err - bound)[bad].max()), float(err[bad].max()))
