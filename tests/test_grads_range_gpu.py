"""Clipping by factors below fp32's normal numbers: a finite gradient of any size comes out right.

Bar: the factor to 2^-24, its product with an element to 2^-24 and the type's rounding."""
import pytest
import torch

from step_util import DT, UNIT, gen, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("src", DT)
@pytest.mark.parametrize("dst", DT)
@pytest.mark.parametrize("size,max_norm", [(2.0 ** 126, 1.0), (2.0 ** 126, 1e-6), (2.0 ** 100, 1e-8), (2.0 ** 120, 1e-30),
                                           (1.0, 1e-36), (1.0, 0.5), (2.0 ** -60, 1e-30)])
def test_clip_of_any_size(sn, src, dst, size, max_norm):
    g = gen(1)
    grads = [(size * (2 * torch.rand(n, generator=g, device="cuda") - 1)).to(DT[src]) for n in (5000, 3, 70001)]
    grads.append(grads[1][1:])                               # off the 16-byte boundary
    out = [torch.empty(t.shape, dtype=DT[dst], device="cuda") for t in grads]
    L = sn.GradList(grads, out=out)
    norm = sn.sn_grads_clip(L, sn.sn_grads_sumsq(L), max_norm)
    norm64 = sum(t.double().square().sum() for t in grads).sqrt()
    c = float(torch.tensor(max_norm, dtype=torch.float32)) / max(float(norm64), max_norm)
    if float(norm64) < 2.0 ** 128:
        assert abs(float(norm) - float(norm64)) <= 2.0 ** -22 * float(norm64)
    smallest = 2.0 ** (-133 if dst == "bf16" else -149)
    for t, o in zip(grads, out):
        ref = t.double() * c
        within(o, ref, ref.abs() * (2.0 ** -22 + 1.01 * UNIT[DT[dst]]) + smallest)
