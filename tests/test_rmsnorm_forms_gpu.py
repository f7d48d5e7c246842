"""RMS norm's 8-bit output with and without a residual at the widths of every kernel, and the outputs
that may take an input's place.  Bars of test_rmsnorm_gpu.py."""
import pytest
import torch

from step_util import DT, gen, within
from test_rmsnorm_gpu import EPS, QMAX, RS, batch, ref_norm

pytestmark = pytest.mark.gpu

# a warp's row of one, two and four pieces, full and not; blocks of 64 to 1024 lanes, full and
# not; single elements
WIDTHS = [24, 128, 256, 264, 512, 520, 1024, 2048, 2056, 3000, 4096, 4104, 8192, 8200, 16384, 20000, 1003]


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("fmt", QMAX)
@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("d", WIDTHS)
def test_codes_with_and_without_a_residual(sn, dt, fmt, group, residual, d):
    T = 19
    g = gen(d + group)
    x, r = batch(T, d, dt, g), batch(T, d, dt, g) if residual else None
    w = batch(1, d, "f32", g)[0]
    w[:group] = 0.0                                          # a group of zeros
    codes, scale, H = sn.sn_rmsnorm_fwd_quant(x, w, EPS, fmt, R=r, group=group)
    assert H is x if not residual else torch.equal(H, (x.float() + r.float()).to(x.dtype))
    y, _ = ref_norm(x.double() + (r.double() if residual else 0.0), w)
    n = group or d
    groups = -(-d // n)
    a = torch.nn.functional.pad(y, (0, groups * n - d)).view(T, groups, n).abs().amax(2)
    within(scale.view(T, groups), a / QMAX[fmt], a / QMAX[fmt] * (2 * RS))
    per = scale.view(T, groups).double().repeat_interleave(n, 1)[:, :d]
    value = codes.view(torch.int8 if fmt == "int8" else torch.float8_e4m3fn).double() * per
    step = per * 0.5 if fmt == "int8" else torch.maximum(y.abs() * 2.0 ** -4, per * 2.0 ** -10)
    within(value, y, step * 1.001 + y.abs() * 4 * RS)
    assert bool((value[per == 0] == 0).all())


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("d", WIDTHS)
def test_outputs_in_an_inputs_place(sn, dt, d):
    T = 37
    g = gen(d)
    x, r, dy, dh = (batch(T, d, dt, g) for _ in range(4))
    w = batch(1, d, "f32", g)[0]
    Y, H = sn.sn_rmsnorm_fwd(x, w, EPS, R=r)
    for y_at, h_at in ((0, None), (1, None), (None, 0), (None, 1), (0, 1), (1, 0)):
        t = [x.clone(), r.clone()]
        h = torch.empty_like(x) if h_at is None else t[h_at]
        Y2, H2 = sn.sn_rmsnorm_fwd(t[0], w, EPS, R=t[1], H=h, out=None if y_at is None else t[y_at])
        assert torch.equal(Y2, Y) and torch.equal(H2, H), (y_at, h_at)
        assert H2 is h and (y_at is None or Y2 is t[y_at])
    for fmt in QMAX:
        want = sn.sn_rmsnorm_fwd_quant(x, w, EPS, fmt, R=r, group=32)
        for h_at in range(2):
            t = [x.clone(), r.clone()]
            got = sn.sn_rmsnorm_fwd_quant(t[0], w, EPS, fmt, R=t[1], H=t[h_at], group=32)
            assert all(torch.equal(a, b) for a, b in zip(got, want))
    alone = sn.sn_rmsnorm_fwd(x, w, EPS)[0]
    t = x.clone()
    assert torch.equal(sn.sn_rmsnorm_fwd(t, w, EPS, out=t)[0], alone)
    dX, dw = sn.sn_rmsnorm_bwd(dy, H, w, EPS, dH=dh)
    for i in range(3):
        t = [dy.clone(), H.clone(), dh.clone()]
        dX2, dw2 = sn.sn_rmsnorm_bwd(t[0], t[1], w, EPS, dH=t[2], out=t[i])
        assert dX2 is t[i] and torch.equal(dX2, dX) and torch.equal(dw2, dw), i
