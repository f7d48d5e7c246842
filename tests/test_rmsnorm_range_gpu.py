"""RMS norm of rows whose squares leave fp32's range, and of rows with an infinity or a NaN.

Bars as in test_rmsnorm_gpu.py: the reciprocal root to 2^-18, which holds for scaled rows too (the
scale is a power of two).  The gradient's results near the type's smallest numbers: a unit of those."""
import math

import pytest
import torch

from step_util import DT, UNIT, gen, within
from test_rmsnorm_gpu import QMAX, RS

pytestmark = pytest.mark.gpu
SMALLEST = {torch.bfloat16: 2.0 ** -133, torch.float32: 2.0 ** -149}

# a warp's rows (one, two and four pieces, full and not), blocks of 64 to 1024 lanes, single elements
WIDTHS = [7, 128, 136, 256, 512, 1000, 1001, 1024, 2048, 2056, 4096, 8192, 8200, 16392, 40000]
SIZES = [1.0, 2e18, 3e25, 4e31, 6e36, 1e-22, 1e-28, 1e-37, 6e-39]


def rows(d, dt, g, T=2):
    """Rows of every size, `T` of each, between ordinary ones."""
    x = torch.randn(T * len(SIZES), d, generator=g, device="cuda", dtype=torch.float64)
    size = torch.tensor(SIZES, dtype=torch.float64, device="cuda").repeat_interleave(T)[:, None]
    return (x.clamp(-5, 5) * size).to(DT[dt]), size


def ref_norm(h, w, eps):
    rs = (h.square().mean(1, keepdim=True) + eps).rsqrt()
    return h * rs * w.double(), rs


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("eps", [0.0, 1e-35, 1e-5])
def test_rows_of_every_size(sn, dt, d, residual, eps):
    g = gen(d)
    x, size = rows(d, dt, g)
    r = (size * torch.randn(x.shape, generator=g, device="cuda")).to(x.dtype) if residual else None
    w = torch.randn(d, generator=g, device="cuda")
    Y, H = sn.sn_rmsnorm_fwd(x, w, eps, R=r)
    h = (x.float() + r.float() if residual else x).double()
    y, _ = ref_norm(h, w, eps)
    # y below the type's normal numbers, and an element far below its row's size
    small = SMALLEST[x.dtype] + (RS + UNIT[x.dtype]) * 2.0 ** -100
    within(Y, y, y.abs() * (RS + 1.01 * UNIT[x.dtype]) + small)
    if residual:
        assert torch.equal(H, (x.float() + r.float()).to(x.dtype))
    for fmt in QMAX:
        for group in (0, 32, 128):
            codes, scale, _ = sn.sn_rmsnorm_fwd_quant(x, w, eps, fmt, R=r, group=group)
            n = group or d
            groups = -(-d // n)
            a = torch.nn.functional.pad(y, (0, groups * n - d)).view(len(x), groups, n).abs().amax(2)
            fine = a > 2.0 ** -90                            # below 2^-100 it counts as that
            per = scale.view(len(x), groups).double()
            within(per[fine], a[fine] / QMAX[fmt], a[fine] / QMAX[fmt] * (2 * RS))
            per = per.repeat_interleave(n, 1)[:, :d]
            value = codes.view(torch.int8 if fmt == "int8" else torch.float8_e4m3fn).double() * per
            step = per * 0.5 if fmt == "int8" else torch.maximum(y.abs() * 2.0 ** -4, per * 2.0 ** -10)
            within(value, y, step * 1.001 + y.abs() * 4 * RS + 2.0 ** -100)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("along", [False, True])
def test_gradient_of_rows_of_every_size(sn, dt, d, along):
    g = gen(2 * d)
    h, size = rows(d, dt, g, T=40 if d < 3000 else 3)
    # dx is dy / size: ordinary numbers where fp32 has them
    dy = (torch.randn(h.shape, generator=g, device="cuda") * size.clamp(1e-12, 1e12)).to(h.dtype)
    dh = (dy.double() / size.clamp(1e-24, 1e24)).to(h.dtype) if along else None
    w = torch.randn(d, generator=g, device="cuda")
    dx, dw = sn.sn_rmsnorm_bwd(dy, h, w, 0.0, dH=dh)
    h64, dy64, w64 = h.double(), dy.double(), w.double()
    rs = h64.square().mean(1, keepdim=True).rsqrt()
    n, q = h64 * rs, dy64 * w64
    first, second = rs * q, rs * n * (q * n).mean(1, keepdim=True)
    ref = first - second + (dh.double() if along else 0.0)
    worst = rs * n.abs() * (q * n).abs().mean(1, keepdim=True)
    bound = (first.abs() + 4 * second.abs()) * RS + worst * 2.0 ** -17 + 2 * SMALLEST[h.dtype]
    fine = ref.abs() < 1e38
    bound = bound + (ref.abs() + (dh.double().abs() if along else 0.0)) * UNIT[h.dtype] * 1.02
    assert bool(fine.all())
    within(dx, ref, bound)
    terms = (dy64 * n).abs().sum(0)
    within(dw, (dy64 * n).sum(0), terms * (RS + 64 * 2.0 ** -23))


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("d", WIDTHS)
def test_rows_of_any_size_leave_the_others(sn, dt, d):
    """Ordinary rows have the same bits beside rows of other sizes, infinities and NaN as alone; a
    row with an infinity or a NaN is NaN whole: its norm, every scale and its gradient."""
    g = gen(d + 5)
    x = torch.randn(20, d, generator=g, device="cuda").to(DT[dt])
    dy = torch.randn(20, d, generator=g, device="cuda").to(DT[dt])
    w = torch.randn(d, generator=g, device="cuda")
    mixed = x.clone()
    mixed[1] *= 1e25
    mixed[4, d // 2] = math.inf
    mixed[9, 0] = -math.inf
    mixed[10, d - 1] = math.nan
    mixed[12] = 0.0
    mixed[15, :] = math.inf
    none = [4, 9, 10, 15]
    same = [t for t in range(20) if t not in none + [1, 12]]
    Y, want = sn.sn_rmsnorm_fwd(mixed, w, 1e-5)[0], sn.sn_rmsnorm_fwd(x, w, 1e-5)[0]
    assert torch.equal(Y[same], want[same])
    assert bool(Y[none].isnan().all()) and bool((Y[12] == 0).all()) and bool(Y[1].isfinite().all())
    for group in (0, 32, 64, 128):
        for fmt in QMAX:
            codes, scale, _ = sn.sn_rmsnorm_fwd_quant(mixed, w, 1e-5, fmt, group=group)
            codes0, scale0, _ = sn.sn_rmsnorm_fwd_quant(x, w, 1e-5, fmt, group=group)
            assert torch.equal(codes[same], codes0[same]) and torch.equal(scale[same], scale0[same])
            assert bool(scale[none].isnan().all()) and bool((scale[12] == 0).all())
    dx, dw = sn.sn_rmsnorm_bwd(dy, mixed, w, 1e-5)
    dx0, _ = sn.sn_rmsnorm_bwd(dy, x, w, 1e-5)
    assert torch.equal(dx[same], dx0[same]) and bool(dx[none].isnan().all()) and bool(dw.isnan().all())
    assert bool(dx[[1, 12]].isfinite().all())


def test_no_gradient_at_tiny_rows(sn):
    """dy = 0 gives dx = 0 at rows of the smallest numbers, whose reciprocal root is past fp32."""
    for dt in DT.values():
        h = torch.full((3, 256), 1e-40, device="cuda").to(dt)
        dx, dw = sn.sn_rmsnorm_bwd(torch.zeros_like(h), h, torch.ones(256, device="cuda"), 0.0)
        assert bool((dx == 0).all()) and bool((dw == 0).all())


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("d", WIDTHS)
def test_gradient_where_the_weight_is_zero(sn, dt, d):
    """Columns whose weight is 0 have the second term of dx alone, far smaller than the others' dx
    at rows that eps outweighs (n is small there); it keeps its bits as long as fp32 holds it."""
    g = gen(3 * d)
    h, size = rows(d, dt, g, T=3)
    dy = (torch.randn(h.shape, generator=g, device="cuda") * size.clamp(1e-6, 1e6)).to(h.dtype)
    w = torch.randn(d, generator=g, device="cuda")
    w[::2] = 0.0
    h64, dy64, w64 = h.double(), dy.double(), w.double()
    for eps in (0.0, 1e-33):
        dx, _ = sn.sn_rmsnorm_bwd(dy, h, w, eps)
        rs = (h64.square().mean(1, keepdim=True) + eps).rsqrt()
        n, q = h64 * rs, dy64 * w64
        first, second = rs * q, rs * n * (q * n).mean(1, keepdim=True)
        worst = rs * n.abs() * (q * n).abs().mean(1, keepdim=True)
        ref = first - second
        # (n mean(g n) itself below fp32's normal numbers: a unit of those, times the reciprocal root)
        bound = (first.abs() + 4 * second.abs()) * RS + worst * 2.0 ** -17 + 2 * SMALLEST[h.dtype] + rs * 2.0 ** -148
        within(dx, ref, bound + ref.abs() * UNIT[h.dtype] * 1.02)
