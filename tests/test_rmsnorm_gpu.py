"""RMS norm with residual, its 8-bit output and its gradient against fp64.

Bars.  The mean of squares is a sum of d non-negative fp32 terms in chains of at most 32 and a
tree: relative error at most 64 * 2^-24, half of it in the root, plus the reciprocal root's 2
units: rs is right to 2^-18.  y is two more products and one rounding to its type.  A code is at
most half a step (plus y's error) from y; e4m3 steps are 2^-3 of the value, at least 2^-9 of the
scale.  The gradient's mean of g h is a signed sum: 64 * 2^-24 of the mean of magnitudes.  dw is a
sum of T fp32 terms, each right to 2^-18."""
import pytest
import torch

from gpu_util import guarded, guards_intact
from step_util import DT, UNIT, gen, spread, within

pytestmark = pytest.mark.gpu
EPS = 1e-5
RS = 2.0 ** -18
QMAX = {"int8": 127.0, "e4m3": 448.0}

# one lane, ragged lanes, 32 to 1024 lanes with 1 to 4 pieces, single elements, rows past the registers
WIDTHS = [1, 7, 8, 64, 136, 200, 1001, 1024, 2056, 4096, 8200, 16392, 40000]


def batch(T, d, dt, g, scale=1.0):
    return (scale * torch.randn(T, d, generator=g, device="cuda")).to(DT[dt])


def ref_norm(h, w):
    rs = (h.square().mean(1, keepdim=True) + EPS).rsqrt()
    return h * rs * w.double(), rs


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("T,wdt,residual,pad", [(1, "f32", True, 0), (37, "bf16", True, 0), (130, "f32", False, 8),
                                                (5, "f32", True, 3)])
def test_forward(sn, dt, d, T, wdt, residual, pad):
    g = gen(d + T)
    x, r = spread(batch(T, d, dt, g), pad), batch(T, d, dt, g, 3.0)
    w = batch(1, d, wdt, g)[0]
    full, out = guarded((T, d), DT[dt])
    Y, H = sn.sn_rmsnorm_fwd(x, w, EPS, R=r if residual else None, out=out)
    h = x.double() + (r.double() if residual else 0.0)
    y, _ = ref_norm(h, w)
    within(Y, y, y.abs() * (RS + UNIT[DT[dt]] * 1.01))
    assert guards_intact(full)
    if residual:
        within(H, h, h.abs() * UNIT[DT[dt]] * 1.01 + (x.double().abs() + r.double().abs()) * 2.0 ** -24)
        inplace = r.clone()                                  # the residual stream updated in place
        Y2, H2 = sn.sn_rmsnorm_fwd(x, w, EPS, R=inplace, H=inplace)
        assert H2 is inplace and torch.equal(H2, H) and torch.equal(Y2, Y)
    else:
        assert H is x


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("fmt", QMAX)
@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("T,d", [(3, 7), (9, 136), (40, 200), (5, 1001), (33, 4096), (2, 8200), (3, 40000)])
def test_codes(sn, dt, fmt, group, T, d):
    g = gen(d + T + group)
    x, r = batch(T, d, dt, g), batch(T, d, dt, g)
    w = batch(1, d, "f32", g)[0]
    n = group or d
    w[: n] = 0.0                                             # a group of zeros (a row of them, for one scale)
    if not group:
        w[d // 2:] = 1.5
    codes, scale, H = sn.sn_rmsnorm_fwd_quant(x, w, EPS, fmt, R=r, group=group)
    assert torch.equal(H, sn.sn_rmsnorm_fwd(x, w, EPS, R=r)[1])
    y, _ = ref_norm(x.double() + r.double(), w)
    groups = -(-d // n)
    yp = torch.nn.functional.pad(y, (0, groups * n - d)).view(T, groups, n)
    a = yp.abs().amax(2)
    within(scale.view(T, groups), a / QMAX[fmt], a / QMAX[fmt] * (2 * RS))
    per = scale.view(T, groups).double().repeat_interleave(n, 1)[:, :d]
    value = codes.view(torch.int8 if fmt == "int8" else torch.float8_e4m3fn).double() * per
    step = per * 0.5 if fmt == "int8" else torch.maximum(y.abs() * 2.0 ** -4, per * 2.0 ** -10)
    within(value, y, step * 1.001 + y.abs() * 4 * RS)
    assert bool((value[per == 0] == 0).all())


def test_codes_and_scales_of_special_rows(sn):
    """A row of zeros, tiny rows, and rows with infinities or NaN, which stay in their rows."""
    for d in (256, 251):
        x = torch.ones(6, d, device="cuda")
        x[0] = 0.0
        x[1] = 1e-36
        x[2, 3] = float("nan")
        x[3, 5] = float("inf")
        w = torch.ones(d, device="cuda")
        Y, _ = sn.sn_rmsnorm_fwd(x, w, EPS)
        assert bool((Y[0] == 0).all()) and bool(Y[2].isnan().all()) and bool(Y[3, 5].isnan())
        within(Y[4:], torch.full((2, d), (1 + EPS) ** -0.5, dtype=torch.float64, device="cuda"), RS + 2.0 ** -24)
        for fmt in QMAX:
            codes, scale, _ = sn.sn_rmsnorm_fwd_quant(x, w, EPS, fmt)
            assert float(scale[0]) == 0 and bool((codes[0] == 0).all())
            assert 0 < float(scale[1]) and not bool(scale[2:4].isfinite().any())
            assert bool((codes[4] == codes[5]).all()) and bool(scale[4:].isfinite().all())


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("T,wdt,along,pad", [(1, "f32", False, 0), (37, "bf16", True, 8), (700, "f32", True, 0),
                                             (6, "f32", True, 5)])
def test_gradient(sn, dt, d, T, wdt, along, pad):
    if d >= 16000 and T > 100:
        T = 200
    g = gen(3 * d + T)
    dy, h = spread(batch(T, d, dt, g), pad), batch(T, d, dt, g, 2.0)
    dh = batch(T, d, dt, g) if along else None
    w = batch(1, d, wdt, g)[0]
    full, out = guarded((T, d), DT[dt])
    wfull, dw = guarded((d,), torch.float32)
    sn.sn_rmsnorm_bwd(dy, h, w, EPS, dH=dh, out=out, dw=dw)
    h64, dy64, w64 = h.double(), dy.double(), w.double()
    rs = (h64.square().mean(1, keepdim=True) + EPS).rsqrt()
    n, q = h64 * rs, dy64 * w64
    first, second = rs * q, rs * n * (q * n).mean(1, keepdim=True)
    dx = first - second + (dh.double() if along else 0.0)
    worst = rs * n.abs() * (q * n).abs().mean(1, keepdim=True)
    bound = (first.abs() + 4 * second.abs()) * RS + worst * 2.0 ** -17
    within(out, dx, bound + (dx.abs() + (dh.double().abs() if along else 0.0)) * UNIT[DT[dt]] * 1.02)
    terms = (dy64 * n).abs().sum(0)
    within(dw, (dy64 * n).sum(0), terms * (RS + min(T, 64) * 2.0 ** -23))
    assert guards_intact(full) and guards_intact(wfull)
    # the same bits again, in place, and added to what is there
    more = dw.clone()
    where = dh.clone() if along else h.clone()
    o2, _ = sn.sn_rmsnorm_bwd(dy, h if along else where, w, EPS, dH=where if along else None, out=where, dw=more,
                              accumulate=True)
    assert torch.equal(o2, out) and torch.equal(more, dw + dw)


def test_no_rows(sn):
    w = torch.ones(64, device="cuda")
    x = torch.empty(0, 64, device="cuda")
    assert sn.sn_rmsnorm_fwd(x, w, EPS)[0].shape == (0, 64)
    assert sn.sn_rmsnorm_fwd_quant(x, w, EPS, "int8", group=32)[1].shape == (0, 2)
    dw = torch.full((64,), 2.0, device="cuda")
    sn.sn_rmsnorm_bwd(x, x, w, EPS, dw=dw, accumulate=True)
    assert bool((dw == 2).all())
    sn.sn_rmsnorm_bwd(x, x, w, EPS, dw=dw)
    assert bool((dw == 0).all())


@pytest.mark.parametrize("d", [96, 99])
def test_gradient_against_differences(sn, d):
    """Central differences of the kernel's own forward in fp32: f = <G, y(h)> + <G2, h>.  Step 1/64:
    the third derivative's term is below 1e-3 of the derivative, the fp32 forward's error (2^-18 of
    the sum of magnitudes over the step) below 1e-3 of the sum's root."""
    g = gen(d)
    T = 16
    h, D, G, G2 = (torch.randn(T, d, generator=g, device="cuda") for _ in range(4))
    w = torch.randn(d, generator=g, device="cuda")
    dw_dir = torch.randn(d, generator=g, device="cuda")
    dx, dw = sn.sn_rmsnorm_bwd(G, h, w, EPS, dH=G2)

    def f(s, v):
        hs = h + s * D
        return (G.double() * sn.sn_rmsnorm_fwd(hs, w + v * dw_dir, EPS)[0].double()).sum() + \
            (G2.double() * hs.double()).sum()

    e = 1.0 / 64
    size = float(G.double().abs().sum()) * 1e-3
    assert abs(float((f(e, 0) - f(-e, 0)) / (2 * e) - (dx.double() * D.double()).sum())) <= size
    assert abs(float((f(0, e) - f(0, -e)) / (2 * e) - (dw.double() * dw_dir.double()).sum())) <= size


def test_refusals(sn):
    x, w = torch.zeros(4, 64, device="cuda"), torch.ones(64, device="cuda")
    for call in (lambda: sn.sn_rmsnorm_fwd(x.half(), w, EPS), lambda: sn.sn_rmsnorm_fwd(x, w, EPS, R=x.bfloat16()),
                 lambda: sn.sn_rmsnorm_bwd(x, x.bfloat16(), w, EPS)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: sn.sn_rmsnorm_fwd(x, w[:32], EPS), lambda: sn.sn_rmsnorm_fwd(x.t(), w, EPS),
                 lambda: sn.sn_rmsnorm_fwd(x, w, EPS, R=x[:2]), lambda: sn.sn_rmsnorm_bwd(x, x, w, EPS, accumulate=True),
                 lambda: sn.sn_rmsnorm_fwd(x.cpu(), w, EPS)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(KeyError):
        sn.sn_rmsnorm_fwd_quant(x, w, EPS, "int4")
    big = torch.zeros(8, 64, device="cuda")
    for call, status in (
            (lambda: sn.sn_rmsnorm_fwd(x, w, -1.0), sn.SN_ERR_INVALID_ARG),
            (lambda: sn.sn_rmsnorm_fwd(x, w, float("nan")), sn.SN_ERR_INVALID_ARG),
            (lambda: sn.sn_rmsnorm_fwd_quant(x, w, EPS, "int8", group=48), sn.SN_ERR_INVALID_ARG),
            (lambda: sn.sn_rmsnorm_fwd(big[:4], w, EPS, out=big[2:6]), sn.SN_ERR_INVALID_ARG),
            (lambda: sn.sn_rmsnorm_fwd(x, w, EPS, R=big[:4], H=big[:4], out=big[:4]), sn.SN_ERR_INVALID_ARG),
            (lambda: sn.sn_rmsnorm_fwd(torch.zeros(300, device="cuda")[1:257].view(4, 64), w, EPS), sn.SN_ERR_ALIGNMENT),
            (lambda: sn.sn_rmsnorm_bwd(x, big[:4], w, EPS, out=big[1:5]), sn.SN_ERR_INVALID_ARG),
            (lambda: sn.sn_rmsnorm_bwd(x, x, w, EPS, workspace=torch.zeros(4, device="cuda")), sn.SN_ERR_INVALID_ARG)):
        with pytest.raises(sn.SNError) as e:
            call()
        assert e.value.status == status
