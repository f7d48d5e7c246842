"""Alternatives of rows with fewer tokens left than asked for, the rest at the type's lowest value: as
fast as with -infinity, whose ties take the same steps (one more look at the row's elements).  A
look for each alternative would take several times as long; the bar is twice."""
import math

import pytest
import torch

from step_util import DT, gen
from test_logprob_gpu import best

pytestmark = pytest.mark.gpu


def timed(call):
    """The shortest of five times in ms, after two calls."""
    times = []
    for _ in range(7):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        for _ in range(10):
            call()
        b.record()
        b.synchronize()
        times.append(a.elapsed_time(b) / 10)
    return min(times[2:])


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("T,V", [(65536, 1000), (8192, 8000), (2048, 128256)])
def test_masks_of_the_lowest_value(sn, dt, T, V):
    g = gen(V)
    left = torch.rand(T, V, generator=g, device="cuda") < 5.0 / V
    left[:, 3] = True
    x = torch.randn(T, V, generator=g, device="cuda").to(DT[dt])
    lowest = torch.where(left, x, torch.finfo(DT[dt]).min)
    none = torch.where(left, x, -math.inf)
    del x, left
    for t in (lowest, none):
        ids = sn.sn_logprob_fwd(t[:300].contiguous(), top=20)[3]
        assert torch.equal(ids.long(), best(t[:300], 20))
    assert timed(lambda: sn.sn_logprob_fwd(lowest, top=20)) <= 2 * timed(lambda: sn.sn_logprob_fwd(none, top=20))


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("T,V", [(9, 1000), (9, 6000), (400, 20000), (3, 60000)])
@pytest.mark.parametrize("value", [-1e-40, -0.5, -1.0, -3e4, -1e30])
def test_ties_at_negative_values(sn, dt, T, V, value):
    """Many equals at a negative value, a few above and below: every number of alternatives."""
    g = gen(V)
    x = torch.full((T, V), value, device="cuda").to(DT[dt])
    pick = torch.rand(T, V, generator=g, device="cuda")
    x[pick < 4.0 / V] = 1.0
    x[(pick > 0.5) & (pick < 0.5 + 4.0 / V)] = value / 2
    x[pick > 0.9] = value * 2
    for top in (1, 5, 9, 32):
        assert torch.equal(sn.sn_logprob_fwd(x, top=top)[3].long(), best(x, top))
