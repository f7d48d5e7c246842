"""Norms after and before a block, with its gate and residual scale, against fp64 torch.

Bars.  A mean of d fp32 squares is within 2^-20 for d up to 16384 (sums of at most 64 elements a
thread, then a tree: far fewer than 16 roundings of 2^-24 each way, plus those of the squares), its
reciprocal root within 2^-21 + 2^-22, and a product of six such numbers within 2^-18 of itself; the
terms of h and of the gradients are such products, so their sums are within 2^-18 of the sum of
the terms' magnitudes.  A column's sum over T tokens adds at most T 2^-24 of the magnitudes.  Each
output is rounded once, 2^-8 of itself in bf16."""
import pytest
import torch

from step_util import DT, UNIT, gen, spread, within

pytestmark = pytest.mark.gpu

EPS, Q = 1e-5, 2.0 ** -18
BF16, F32 = torch.bfloat16, torch.float32
# T, d, gates: warps' rows, blocks' rows of every number of lanes, single elements, gates of one
# token, of odd runs, of many, of every token
SIZES = [(1, 1, 0), (1, 256, 1), (5, 7, 0), (33, 64, 11), (100, 128, 100), (64, 256, 0), (37, 512, 37),
         (1200, 520, 3), (75, 1000, 25), (64, 1001, 4), (300, 2056, 2), (129, 4096, 1), (40, 4104, 5),
         (700, 2048, 0), (33, 8192, 33), (17, 8200, 1), (9, 16384, 3), (6, 32768, 2), (3, 40000, 0),
         (5000, 264, 8), (4099, 48, 4099), (2600, 1024, 26)]


def inputs(T, d, gates, dt, seed, wdt=F32):
    g = gen(seed)

    def normal(*shape, mean=0.0, std=1.0, dtype=dt):
        return (mean + std * torch.randn(*shape, generator=g, device="cuda")).to(dtype)

    wide = 1 + 7 * (torch.rand(d, generator=g, device="cuda") < 0.05).to(dt)
    s = {"Y": normal(T, d, std=3.0) * wide, "R": normal(T, d) * wide,
         "w_post": normal(d, mean=1.0, std=0.2, dtype=wdt), "w_pre": normal(d, mean=1.0, std=0.2, dtype=wdt),
         "gate": normal(gates, d, mean=1.0, std=0.5) if gates else None,
         "dZ": normal(T, d), "dH": normal(T, d)}
    s["H"] = s["R"] + normal(T, d)
    return s


def parts(s, scale, eps):
    """fp64: n1, the branch's multiplier of every element, and the roots of the mean squares."""
    y = s["Y"].double()
    T, d = y.shape
    q1 = (y.square().mean(1, keepdim=True) + eps).sqrt()
    m = torch.full((T, d), float(scale), device="cuda", dtype=torch.float64)
    if s["gate"] is not None:
        m = m * s["gate"].double().repeat_interleave(T // s["gate"].shape[0], 0)
    return y / q1, m, q1


def check_fwd(s, scale, Z, H, eps=EPS, rows=slice(None)):
    n1, m, _ = parts(s, scale, eps)
    b, r = n1 * m * s["w_post"].double(), s["R"].double()
    h = b + r
    e = Q * (b.abs() + r.abs())
    unit = UNIT[H.dtype]
    within(H[rows], h[rows], (e + unit * (h.abs() + e))[rows])
    q2 = (h.square().mean(1, keepdim=True) + eps).sqrt()
    w = s["w_pre"].double()
    z = h / q2 * w
    # h off by e moves the mean square by at most 2 |h| e
    ez = (e / q2 + h.abs() * (h.abs() * e).mean(1, keepdim=True) / q2 ** 3) * w.abs() + Q * z.abs()
    within(Z[rows], z[rows], (ez + unit * (z.abs() + ez))[rows])


def check_bwd(s, scale, got, dH=True, eps=EPS, add=None):
    dY, dR, dw_post, dw_pre, dgate = got
    T, d = dY.shape
    n1, m, q1 = parts(s, scale, eps)
    h, dz, w1, w2 = (s[k].double() for k in ("H", "dZ", "w_post", "w_pre"))
    q2 = (h.square().mean(1, keepdim=True) + eps).sqrt()
    n2, g = h / q2, dz * w2
    r = s["dH"].double() if dH else torch.zeros_like(h)
    mean = lambda x: x.mean(1, keepdim=True)
    unit = UNIT[dY.dtype]
    dh = (g - n2 * mean(g * n2)) / q2 + r
    sh = (g.abs() + n2.abs() * mean((g * n2).abs())) / q2 + r.abs()      # the terms' magnitudes
    within(dR, dh, Q * sh + unit * (dh.abs() + Q * sh))
    e, se = dh * m * w1, sh * (m * w1).abs()
    dy = (e - n1 * mean(e * n1)) / q1
    sy = (se + n1.abs() * mean(se * n1.abs())) / q1
    within(dY, dy, Q * sy + unit * (dy.abs() + Q * sy))
    sums = [(dw_pre, dz * n2, (dz * n2).abs(), 1), (dw_post, dh * m * n1, sh * (m * n1).abs(), 1)]
    if dgate is not None:
        sums.append((dgate, scale * dh * w1 * n1, sh * abs(scale) * (w1 * n1).abs(), dgate.shape[0]))
    else:
        assert s["gate"] is None
    for i, (out, x, size, n) in enumerate(sums):
        ref, size = x.view(n, -1, d).sum(1).view(out.shape), size.view(n, -1, d).sum(1).view(out.shape)
        was = add[i].double() if add else torch.zeros_like(ref)
        within(out, ref + was, (Q + (T // n) * 2.0 ** -24) * size + 2.0 ** -23 * (ref.abs() + was.abs()))


def guarded(rows, cols, dt):
    full = torch.full((rows + 2, cols), 7.25, dtype=dt, device="cuda")
    return full, full[1:-1]


def aligned(cols, dt):
    return cols * torch.empty(0, dtype=dt).element_size() % 16 == 0


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,gates", SIZES)
def test_forward(sn, dt, T, d, gates):
    s = inputs(T, d, gates, DT[dt], T + d, BF16 if d % 3 == 0 else F32)
    scale = (1.0, 0.25, -1.5)[T % 3]
    if not aligned(d, DT[dt]):
        Z, H = sn.sn_blocknorm_fwd(s["Y"], s["R"], s["w_post"], s["w_pre"], EPS, scale, s["gate"])
    else:
        (fz, Z), (fh, H) = guarded(T, d, DT[dt]), guarded(T, d, DT[dt])
        sn.sn_blocknorm_fwd(s["Y"], s["R"], s["w_post"], s["w_pre"], EPS, scale, s["gate"], H=H, out=Z)
        assert all(bool((f[[0, -1]] == 7.25).all()) for f in (fz, fh))
    check_fwd(s, scale, Z, H)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,gates", SIZES)
def test_gradient(sn, dt, T, d, gates):
    s = inputs(T, d, gates, DT[dt], T + d + 1, BF16 if d % 3 == 1 else F32)
    scale, dH = (1.0, 0.25, -1.5)[T % 3], T % 2 == 1
    kw = {}
    if aligned(d, DT[dt]):
        (fy, dY), (fr, dR) = guarded(T, d, DT[dt]), guarded(T, d, DT[dt])
        kw = dict(dY=dY, dR=dR)
    got = sn.sn_blocknorm_bwd(s["dZ"], s["H"], s["Y"], s["w_post"], s["w_pre"], EPS, scale, s["gate"],
                              dH=s["dH"] if dH else None, **kw)
    check_bwd(s, scale, got, dH)
    if kw:
        assert all(bool((f[[0, -1]] == 7.25).all()) for f in (fy, fr))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [264, 1000, 4096])
@pytest.mark.parametrize("pad", [1, 8])
def test_row_strides(sn, dt, d, pad):
    s = inputs(50, d, 5, DT[dt], d)
    Z, H = sn.sn_blocknorm_fwd(spread(s["Y"], pad), s["R"], s["w_post"], s["w_pre"], EPS, 0.5, s["gate"])
    check_fwd(s, 0.5, Z, H)
    got = sn.sn_blocknorm_bwd(spread(s["dZ"], pad), s["H"], spread(s["Y"], 2 * pad), s["w_post"], s["w_pre"],
                              EPS, 0.5, s["gate"], dH=s["dH"])
    check_bwd(s, 0.5, got)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [100, 512, 2056])
def test_in_place(sn, dt, d):
    s = inputs(90, d, 3, DT[dt], d)
    w = (s["w_post"], s["w_pre"], EPS, 0.5, s["gate"])
    Z, H = sn.sn_blocknorm_fwd(s["Y"], s["R"], *w)
    for h, z in (("R", "Y"), ("Y", "R"), ("R", None), (None, "Y")):
        c = {k: s[k].clone() for k in ("Y", "R")}
        z2, h2 = sn.sn_blocknorm_fwd(c["Y"], c["R"], *w, H=c.get(h), out=c.get(z))
        assert torch.equal(z2, Z) and torch.equal(h2, H)
    want = sn.sn_blocknorm_bwd(s["dZ"], s["H"], s["Y"], *w, dH=s["dH"])
    names = ("dZ", "H", "Y", "dH")
    for y, r in ((a, b) for a in names for b in names if a != b):
        c = {k: s[k].clone() for k in names}
        got = sn.sn_blocknorm_bwd(c["dZ"], c["H"], c["Y"], *w, dH=c["dH"], dY=c[y], dR=c[r])
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("T,d,gates", [(200, 512, 0), (200, 264, 2), (60, 100, 60), (60, 264, 60), (3000, 2056, 3)])
def test_accumulated(sn, T, d, gates):
    s = inputs(T, d, gates, BF16, 3)
    g = gen(4)
    was = [torch.randn(*shape, generator=g, device="cuda") for shape in ((d,), (d,), (gates, d))][:3 if gates else 2]
    out = [w.clone() for w in was]
    got = sn.sn_blocknorm_bwd(s["dZ"], s["H"], s["Y"], s["w_post"], s["w_pre"], EPS, 0.5, s["gate"], dH=s["dH"],
                              dw_pre=out[0], dw_post=out[1], dgate=out[2] if gates else None, accumulate=True)
    check_bwd(s, 0.5, got, add=was)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [100, 256, 2056, 4096])
@pytest.mark.parametrize("y,h", [(1e-25, 1.0), (1.0, 1e-25), (1e25, 1.0), (1.0, 1e25), (1e25, 1e-25), (1e-25, 1e-25)])
def test_rows_whose_squares_leave_fp32(sn, dt, d, y, h):
    """Every second row far from 1: the others are as they are without them, and those are right."""
    T = 24
    s = inputs(T, d, 0, DT[dt], 5)
    s["w_post"].mul_(0.5)
    plain = {k: s[k].clone() for k in ("Y", "R", "H")}
    s["Y"][::2] *= y
    s["R"][::2] *= h
    s["H"][::2] *= h
    s["dH"][::2] *= 1 / h
    scale = 1.0
    # eps = 0: a tiny row's norm is a number
    Z, H = sn.sn_blocknorm_fwd(s["Y"], s["R"], s["w_post"], s["w_pre"], 0.0, scale)
    check_fwd(s, scale, Z, H, eps=0.0)
    Zp, Hp = sn.sn_blocknorm_fwd(plain["Y"], plain["R"], s["w_post"], s["w_pre"], 0.0, scale)
    assert torch.equal(Z[1::2], Zp[1::2]) and torch.equal(H[1::2], Hp[1::2])
    got = sn.sn_blocknorm_bwd(s["dZ"], s["H"], s["Y"], s["w_post"], s["w_pre"], 0.0, scale, dH=s["dH"])
    if y * h > 1e-30:            # elsewhere dy passes fp32's range
        check_bwd(s, scale, got, eps=0.0)
    else:
        assert not torch.isnan(got[1]).any()


def test_rows_of_zeros_infinities_and_nans(sn):
    for d in (100, 256, 4096):
        s = inputs(12, d, 0, BF16, 6)
        s["Y"][0] = 0.0
        s["Y"][1] = 0.0
        s["R"][1] = 0.0
        s["Y"][2, d // 2], s["R"][3, 0], s["Y"][4, d - 1], s["R"][5, 1] = (float(x) for x in ("inf", "-inf", "nan", "nan"))
        Z, H = sn.sn_blocknorm_fwd(s["Y"], s["R"], s["w_post"], s["w_pre"], EPS)
        assert torch.equal(H[0], s["R"][0]) and not Z[1].any() and not H[1].any()
        for t in (2, 3, 4, 5):
            assert torch.isnan(Z[t]).all()
        rest = [0, 1] + list(range(6, 12))
        ok = {k: (v[rest] if v is not None and v.dim() == 2 else v) for k, v in s.items()}
        check_fwd(ok, 1.0, Z[rest], H[rest])


def test_gradient_against_differences(sn):
    """fp32 gradients against central differences of the formula in fp64."""
    T, d, gates, scale = 6, 20, 3, 0.7
    s = inputs(T, d, gates, F32, 7)
    x = {k: s[k].double() for k in ("Y", "R", "w_post", "w_pre", "gate")}

    def run(v):
        n1 = v["Y"] / (v["Y"].square().mean(1, keepdim=True) + EPS).sqrt()
        h = v["R"] + scale * v["gate"].repeat_interleave(T // gates, 0) * n1 * v["w_post"]
        return h, h / (h.square().mean(1, keepdim=True) + EPS).sqrt() * v["w_pre"]

    def value(v):
        h, z = run(v)
        return float((z * s["dZ"].double()).sum() + (h * s["dH"].double()).sum())

    H = run(x)[0].float()
    dY, dR, dw_post, dw_pre, dgate = sn.sn_blocknorm_bwd(s["dZ"], H, s["Y"], s["w_post"], s["w_pre"], EPS, scale,
                                                         s["gate"], dH=s["dH"])
    for name, grad in (("Y", dY), ("R", dR), ("w_post", dw_post), ("w_pre", dw_pre), ("gate", dgate)):
        for i in (0, grad.numel() // 2 + 1, grad.numel() - 1):
            ends = []
            for step in (1e-5, -1e-5):
                v = {k: t.clone() for k, t in x.items()}
                v[name].view(-1)[i] += step
                ends.append(value(v))
            want = (ends[0] - ends[1]) / 2e-5
            # differences: 1e-10 of third derivatives, 1e-16 / 1e-5 of the value; fp32: 2^-18 of the terms
            assert abs(float(grad.view(-1)[i]) - want) <= 2e-4 * float(grad.abs().max())


def test_no_tokens_and_same_bits(sn):
    s = inputs(800, 1032, 8, BF16, 8)
    w = (s["w_post"], s["w_pre"], EPS, 0.5)
    Z, H = sn.sn_blocknorm_fwd(s["Y"][:0], s["R"][:0], *w)
    assert Z.shape == H.shape == (0, 1032)
    got = sn.sn_blocknorm_bwd(s["dZ"][:0], s["H"][:0], s["Y"][:0], *w, s["gate"])
    assert not any(g.any() for g in got) and got[4].shape == (8, 1032)
    runs = [sn.sn_blocknorm_fwd(s["Y"], s["R"], *w, s["gate"]) +
            sn.sn_blocknorm_bwd(s["dZ"], s["H"], s["Y"], *w, s["gate"], dH=s["dH"]) for _ in range(3)]
    assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(runs[0], r))


def test_refusals(sn):
    s = inputs(24, 64, 4, BF16, 9)
    bad = sn.SNError

    def fwd(**kw):
        a = dict(Y=s["Y"], R=s["R"], w_post=s["w_post"], w_pre=s["w_pre"], eps=EPS, gate=s["gate"])
        a.update(kw)
        return lambda: sn.sn_blocknorm_fwd(**a)

    def bwd(**kw):
        a = dict(dZ=s["dZ"], H=s["H"], Y=s["Y"], w_post=s["w_post"], w_pre=s["w_pre"], eps=EPS, gate=s["gate"])
        a.update(kw)
        return lambda: sn.sn_blocknorm_bwd(**a)

    same, flat = torch.empty_like(s["Y"]), torch.zeros(24 * 64 + 8, device="cuda", dtype=BF16)
    f32 = torch.zeros(64, device="cuda")
    for call, error in (
            (fwd(eps=-1.0), bad), (fwd(eps=float("nan")), bad), (fwd(scale=float("inf")), bad),
            (fwd(H=same, out=same), bad), (fwd(H=flat[8:].view(24, 64), out=flat[:-8].view(24, 64)), bad),
            (fwd(R=s["R"][:3]), ValueError), (fwd(gate=s["gate"][:, :32]), ValueError),
            (fwd(gate=torch.ones(5, 64, device="cuda", dtype=BF16)), ValueError),
            (fwd(gate=torch.ones(48, 64, device="cuda", dtype=BF16)), ValueError),
            (fwd(gate=s["gate"].float()), TypeError), (fwd(w_pre=s["w_pre"].to(BF16)), TypeError),
            (fwd(Y=s["Y"].half()), TypeError), (fwd(out=flat[1:1537].view(24, 64)), bad),
            (fwd(H=s["gate"].repeat(6, 1)[:, :32]), ValueError), (fwd(Y=s["Y"].cpu()), ValueError),
            (bwd(dY=same, dR=same), bad), (bwd(dw_post=f32, dw_pre=f32), bad), (bwd(accumulate=True), ValueError),
            (bwd(gate=None, dgate=torch.zeros(4, 64, device="cuda")), ValueError),
            (bwd(dw_pre=f32.to(BF16)), TypeError), (bwd(dH=s["dH"][:3]), ValueError),
            (bwd(workspace=torch.empty(16, device="cuda")), bad), (bwd(dw_pre=s["w_pre"]), bad)):
        with pytest.raises(error):
            call()
    torch.cuda.synchronize()
