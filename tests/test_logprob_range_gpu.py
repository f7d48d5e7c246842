"""Log probabilities and their gradient at scales and gradients of every size, masks among the logits.

Bars as in test_logprob_gpu.py: S to 2^-15, z to 2^-22 of itself where p matters (|z| < 40)."""
import math

import pytest
import torch

from step_util import DT, UNIT, gen, within
from test_logprob_gpu import S_REL, best

pytestmark = pytest.mark.gpu


def near_zero(T, V, dt, scale, g):
    """Logits whose products with the scale are ordinary, with masks of three kinds."""
    x = (3 * torch.randn(T, V, generator=g, device="cuda") / scale).to(DT[dt])
    x[0, V // 2:] = -math.inf
    x[1, V // 3:] = torch.finfo(DT[dt]).min
    x[2, V // 4:] = -1.0
    x[2, 0] = 0.0
    x[3:, ::7] = -math.inf
    x[3] = x[3].clamp(max=0.0)                               # the largest is 0
    x[3, 1] = 0.0
    return x


def reference(x, scale):
    q = torch.log_softmax(x.double() * float(torch.tensor(scale, dtype=torch.float32)), 1)
    p = q.exp()
    qf = torch.where(p > 0, q, 0.0)
    return q, p, qf, -(p * qf).sum(1)


# a warp's row, a block's of 128 and 256 threads, a cluster's
@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("T,V", [(5, 300), (5, 5000), (400, 9000), (5, 40000)])
@pytest.mark.parametrize("scale", [1e9, 1e17, 1e18, 1e20, 1e30, 2e38])
def test_large_scales(sn, dt, T, V, scale):
    g = gen(V)
    x = near_zero(T, V, dt, scale, g)
    target = x.argmax(1).int()
    logp, lse, H, ids, alt = sn.sn_logprob_fwd(x, target, scale=scale, top=4)
    q, p, qf, ent = reference(x, scale)
    assert torch.equal(ids.long(), best(x, 4))
    within(logp, q.gather(1, target.long()[:, None])[:, 0], S_REL + 40 * 2.0 ** -22)
    at = q.gather(1, ids.long())
    near = at > -40
    within(alt[near], at[near], S_REL + 40 * 2.0 ** -22)
    within(H, ent, 2 * S_REL * (math.log(V) + 1) + 2.0 ** -19)
    if scale > 1e30:                                         # the gradient's terms pass fp32's range
        return
    a, b = (torch.randn(T, generator=g, device="cuda") for _ in range(2))
    hot = torch.zeros_like(p).scatter_(1, target.long()[:, None], 1.0)
    s64 = float(torch.tensor(scale, dtype=torch.float32))
    a64, b64 = a.double()[:, None], b.double()[:, None]
    size = p * (a64.abs() + b64.abs() * (qf.abs() + ent[:, None] + 2 + math.log(V)))
    for ga, gb in ((a, b), (a, None), (None, b)):
        dx = sn.sn_logprob_bwd(x, lse, target if ga is not None else None, ga, scale=scale,
                               entropy=H if gb is not None else None, dentropy=gb)
        ref = s64 * ((a64 * (hot - p) if ga is not None else 0) - (b64 * p * (qf + ent[:, None]) if gb is not None else 0))
        within(dx, ref, s64 * (size * 2.0 ** -12 + a64.abs() * hot * 2.0 ** -22) + ref.abs() * UNIT[DT[dt]] * 1.02)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("scale,size", [(1.0, 1e19), (1.0, 1e30), (1e10, 1.0), (1e12, 1e10)])
def test_large_gradients_of_the_entropy(sn, dt, scale, size):
    """A masked column's gradient is 0 however large the entropy's is."""
    T, V = 6, 700
    g = gen(3)
    x = near_zero(T, V, dt, scale, g)
    _, lse, H, _, _ = sn.sn_logprob_fwd(x, scale=scale)
    b = size * (1 + torch.rand(T, generator=g, device="cuda"))
    dx = sn.sn_logprob_bwd(x, lse, scale=scale, entropy=H, dentropy=b)
    q, p, qf, ent = reference(x, scale)
    s64, b64 = float(torch.tensor(scale, dtype=torch.float32)), b.double()[:, None]
    assert bool((dx[p == 0] == 0).all())
    ref = -s64 * b64 * p * (qf + ent[:, None])
    within(dx, ref, s64 * b64 * p * (qf.abs() + ent[:, None] + 2 + math.log(V)) * 2.0 ** -12
           + ref.abs() * UNIT[DT[dt]] * 1.02)


def test_scales_that_have_no_exponent(sn):
    """The scale in base 2 has to be a number: past 2.35e38 it is refused, in both directions."""
    x, f = torch.zeros(2, 8, device="cuda"), torch.zeros(2, device="cuda")
    t = torch.zeros(2, dtype=torch.int32, device="cuda")
    _, lse, _, _, _ = sn.sn_logprob_fwd(x, t, scale=2.3e38)
    for call in (lambda: sn.sn_logprob_fwd(x, t, scale=2.4e38), lambda: sn.sn_logprob_bwd(x, lse, t, f, scale=2.4e38)):
        with pytest.raises(sn.SNError) as e:
            call()
        assert e.value.status == sn.SN_ERR_INVALID_ARG
