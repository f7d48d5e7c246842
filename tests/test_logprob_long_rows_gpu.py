"""Log probabilities and their gradient for a vocabulary close to the largest that the calls take, 2^31
- 513: places within a row close to 2^31.  All logits are alike, so every log probability is -ln V,
to the sum's 2^-15 and a rounding, and every gradient -1 / V but the target's."""
import math

import pytest
import torch

from step_util import DT, UNIT

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", DT)
def test_a_row_of_two_billion(sn, dt):
    V = 2 ** 31 - 600
    x = torch.zeros(1, V, dtype=DT[dt], device="cuda")
    target = torch.tensor([V - 3], dtype=torch.int32, device="cuda")
    logp, lse, H, ids, alt = sn.sn_logprob_fwd(x, target, top=3)
    want = math.log(V)
    for got, ref in ((logp, -want), (lse[:, 1], want), (H, want), (alt[0], -want)):
        assert bool(((got.double() - ref).abs() <= 2.0 ** -14).all())
    assert ids[0].tolist() == [0, 1, 2]
    one = torch.ones(1, device="cuda")
    dx = sn.sn_logprob_bwd(x, lse, target, one, out=x)
    assert abs(float(dx[0, V - 3]) - 1) <= 2.0 ** -7
    dx[0, V - 3] = dx[0, 0]
    bound = (2.0 ** -13 + UNIT[DT[dt]]) / V
    for part in dx[0].split(1 << 28):
        low, high = part.aminmax()
        assert abs(float(low) + 1 / V) <= bound and abs(float(high) + 1 / V) <= bound
