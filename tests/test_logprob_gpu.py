"""Log probabilities, entropy, alternatives and their gradient against fp64.

Bars.  S is a sum of at most V positive fp32 terms, each with ex2's error (2^-22) and that of its
argument (one fma: 2^-24 of |z - m| in base 2, which only counts where e^(z-m) does: below 2^-20),
in chains of at most V / 512 + 64 (one block) or V / 128 + 64: with V below 2^17 relative error
below 2^-15.  ln S is right to 2^-15 absolute, lse to that and one rounding, the entropy's quotient
to 2^-14 of ln V + 1.  Alternatives are exact.  The gradient's p is right to 2^-22 (|z| + |lse|) +
2^-14 relative (lse's own error)."""
import math

import pytest
import torch

from gpu_util import guarded, guards_intact
from step_util import DT, UNIT, gen, spread, within

pytestmark = pytest.mark.gpu
S_REL = 2.0 ** -15


def logits(T, V, dt, g, pad=0, ties=False):
    x = 3 * torch.randn(T, V, generator=g, device="cuda")
    if ties:
        x = x.round()
    return spread(x.to(DT[dt]), pad)


def best(x, top):
    """Columns of the `top` largest of each row, the lower column first among equals."""
    return torch.sort(x.double() + 0.0, dim=1, descending=True, stable=True).indices[:, :top]


def check_forward(sn, x, target, scale, top):
    V = x.shape[1]
    logp, lse, H, ids, alt = sn.sn_logprob_fwd(x, target, scale=scale, top=top)
    z = x.double() * float(torch.tensor(scale, dtype=torch.float32))
    q = torch.log_softmax(z, 1)
    assert torch.equal(lse[:, 0], x.amax(1).float())
    within(lse[:, 1], torch.logsumexp(z - z.amax(1, keepdim=True), 1), S_REL)
    p = q.exp()
    ent = -torch.where(p > 0, p * q, 0.0).sum(1)
    within(H, ent, 2 * S_REL * (math.log(V) + 1) + 2.0 ** -22 * math.log(V + 1))
    t = target.long()
    good = (t >= 0) & (t < V)
    lp = torch.where(good, q.gather(1, t.clamp(0, V - 1)[:, None])[:, 0], 0.0)
    fine = lp.isfinite()
    within(logp[fine], lp[fine], S_REL + lp[fine].abs() * 2.0 ** -22)
    assert torch.equal(logp[~fine], lp[~fine].float())       # a masked target: -infinity
    if top:
        at = best(x, top)
        assert torch.equal(ids.long(), at)
        ref = q.gather(1, at)
        fine = ref.isfinite()
        within(alt[fine], ref[fine], S_REL + ref[fine].abs() * 2.0 ** -22)
        assert torch.equal(alt[~fine], ref[~fine].float())
    return logp, lse, H


# one block of 128 or 512 threads, clusters of 2 to 8, rows of fewer elements than a 16-byte piece,
# rows off the alignment
@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("T,V,top,pad,scale", [
    (1, 1, 1, 0, 1.0), (3, 3, 2, 0, 1.0), (5, 7, 7, 1, 1.0), (40, 9, 5, 0, 0.5), (2, 33, 32, 3, 1.25),
    (400, 1000, 20, 0, 1.0), (7, 1024, 32, 47, 1.0), (1, 4101, 5, 0, 2.0), (1, 8197, 32, 0, 1.0),
    (9, 20000, 20, 5, 1.0), (1, 50257, 20, 0, 0.7), (30, 50257, 1, 0, 1.0), (70, 50257, 8, 1, 1.0),
    (160, 33000, 0, 0, 1.0), (3, 128256, 32, 0, 1.0)])
@pytest.mark.parametrize("ties", [False, True])
def test_forward(sn, dt, T, V, top, pad, scale, ties):
    g = gen(T + V)
    x = logits(T, V, dt, g, pad, ties)
    target = torch.randint(V, (T,), generator=g, device="cuda", dtype=torch.int32)
    target[::5] = -100
    check_forward(sn, x, target, scale, top)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("T,V", [(4, 300), (3, 40000), (200, 40000)])
def test_masks(sn, dt, T, V):
    """Most of the vocabulary at -infinity, fewer tokens left than alternatives asked for, one left,
    masks of the type's lowest value, and a row of each kind among ordinary ones."""
    g = gen(V)
    x = logits(T, V, dt, g).clone()
    x[0, 5:] = -math.inf
    x[1] = -math.inf
    x[1, V // 2] = 0.25
    x[2, torch.rand(V, generator=g, device="cuda") < 0.999] = torch.finfo(DT[dt]).min
    target = torch.zeros(T, dtype=torch.int32, device="cuda")
    target[1] = V // 2
    check_forward(sn, x, target, 1.0, 20)
    x[-1] = torch.finfo(DT[dt]).min                          # nothing but masks: all tokens alike
    logp, lse, H = check_forward(sn, x, target, 1.0, 20)
    one = torch.ones(T, device="cuda")
    dx = sn.sn_logprob_bwd(x, lse, target, one, entropy=H, dentropy=one)
    within(dx[-1, 1:], torch.full((V - 1,), -1.0 / V, dtype=torch.float64, device="cuda"),
           (2.0 ** -13 + UNIT[DT[dt]]) / V)
    target[:] = V - 1                                        # a masked target
    logp, _, _ = check_forward(sn, x, target, 1.0, 20)
    assert float(logp[0]) == -math.inf


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("size", [1e-30, 1e6, 2e7, 1e19, 1e25, 3e37])
@pytest.mark.parametrize("scale", [1.0, 1e-18, 30.0])
def test_logits_of_any_size(sn, dt, size, scale):
    """Differences of logits that the type still tells apart, however large or small they are.  The
    exponent's rounding counts here: z is right to 2^-22 of itself where p matters (|z| < 40)."""
    g = gen(11)
    T, V = 6, 3000
    x = (size * torch.randn(T, V, generator=g, device="cuda")).to(DT[dt])
    x[1] = -x[1].abs() - size
    x[2, 5:] = x[2, 4]                                       # many at the maximum
    x[2, :5] = -x[2, 4].abs()
    target = x.argmax(1).int()
    logp, lse, H, ids, alt = sn.sn_logprob_fwd(x, target, scale=scale, top=4)
    s64 = float(torch.tensor(scale, dtype=torch.float32))
    q = torch.log_softmax(x.double() * s64, 1)
    p = q.exp()
    assert torch.equal(ids.long(), best(x, 4))
    within(logp, q.gather(1, target.long()[:, None])[:, 0], S_REL)
    at = q.gather(1, ids.long())
    near = at > -40
    within(alt[near], at[near], S_REL + 40 * 2.0 ** -22)
    within(H, -torch.where(p > 0, p * q, 0.0).sum(1), 2 * S_REL * (math.log(V) + 1) + 2.0 ** -19)
    one = torch.ones(T, device="cuda")
    dx = sn.sn_logprob_bwd(x, lse, target, one, scale=scale, entropy=H, dentropy=one)
    hot = torch.zeros_like(p).scatter_(1, target.long()[:, None], 1.0)
    qf = torch.where(p > 0, q, 0.0)
    ent = -(p * qf).sum(1, keepdim=True)
    ref = s64 * (hot - p - p * (qf + ent))
    within(dx, ref, s64 * (p * (2 + 2 * qf.abs() + ent + math.log(V)) * 2.0 ** -13 + hot * 2.0 ** -23 + 2.0 ** -60)
           + ref.abs() * UNIT[DT[dt]] * 1.02)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("T,V", [(3, 9), (2, 5000), (2, 40000), (200, 9001)])
def test_rows_without_a_token(sn, dt, T, V):
    g = gen(V + 1)
    x = logits(T, V, dt, g).clone()
    x[1] = -math.inf
    target = torch.zeros(T, dtype=torch.int32, device="cuda")
    logp, lse, H, ids, alt = sn.sn_logprob_fwd(x, target, top=5)
    assert float(logp[1]) == float(lse[1, 0]) == float(lse[1, 1]) == -math.inf and float(H[1]) == 0
    assert ids[1].tolist() == [0, 1, 2, 3, 4] and bool((alt[1] == -math.inf).all())
    one = torch.ones(T, device="cuda")
    dx = sn.sn_logprob_bwd(x, lse, target, one, entropy=H, dentropy=one)
    assert bool((dx[1] == 0).all()) and bool(dx.isfinite().all())
    keep = [t for t in range(T) if t != 1]
    check_forward(sn, x[keep].contiguous(), target[keep], 1.0, 5)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("V", [77, 5000, 40000])
def test_rows_that_are_no_numbers(sn, dt, bad, V):
    """A NaN or an infinity makes its own row NaN and no other; it is the first alternative."""
    g = gen(V + 2)
    x = logits(4, V, dt, g).clone()
    x[2, V - 3] = bad
    target = torch.ones(4, dtype=torch.int32, device="cuda")
    logp, lse, H, ids, alt = sn.sn_logprob_fwd(x, target, top=3)
    for v in (logp, lse[:, 1], H, alt[:, 0]):
        assert v.isnan().tolist() == [False, False, True, False]
    assert int(ids[2, 0]) == V - 3
    dx = sn.sn_logprob_bwd(x, lse, target, torch.ones(4, device="cuda"))
    assert bool(dx[2].isnan().all()) and bool(dx[[0, 1, 3]].isfinite().all())


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("T", [1, 200])
@pytest.mark.parametrize("kind", ["constant", "few values", "one thread's columns", "rising", "zeros of both signs"])
def test_selection_of_many_equal_or_clustered(sn, dt, T, kind):
    """Rows whose largest logits are many equals, or lie in few threads' columns (more than the list
    of candidates holds)."""
    V, top = 128256, 32
    g = gen(T)
    x = logits(T, V, dt, g).clone()
    if kind == "constant":
        x[:] = 1.5
    elif kind == "few values":
        x[:] = torch.randint(3, (T, V), generator=g, device="cuda").to(x.dtype)
    elif kind == "one thread's columns":
        per = 8 if dt == "bf16" else 4                       # columns of a 16-byte piece
        hot = (torch.arange(V, device="cuda") // per) % 512 < 20
        x[:, hot] = 50 + torch.rand(T, int(hot.sum()), generator=g, device="cuda").to(x.dtype)
    elif kind == "rising":
        x[:] = torch.linspace(-5, 5, V, device="cuda").to(x.dtype)
    else:
        x[:] = torch.where(torch.rand(T, V, generator=g, device="cuda") < 0.5, -0.0, 0.0).to(x.dtype)
    _, _, _, ids, _ = sn.sn_logprob_fwd(x, top=top)
    assert torch.equal(ids.long(), best(x, top))


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("T,V", [(320, 9001), (320, 40000), (320, 1000), (20, 60000)])
@pytest.mark.parametrize("top", [1, 8, 32])
def test_alternatives_that_few_threads_hold(sn, dt, T, V, top):
    """The best elements at the same place of one, two or five steps of a row, of any number of
    threads a row, with a few equal ones, -infinities and a row's ends among them."""
    g = gen(V + top)
    x = logits(T, V, dt, g).clone()
    per = 16 // x.element_size()
    for t in range(T):
        piece = 37 * t % (V // per)
        step = (512, 1024, 2048, 4096, 2048 + 256)[t % 5]
        cols = (piece * per + t % per + torch.arange(1 + t % 40, device="cuda") * step * per) % V
        x[t, cols] = 40 + torch.randint(6, cols.shape, generator=g, device="cuda").to(x.dtype)
        if t % 7 == 0:
            x[t, :9] = 41
            x[t, -9:] = 43
        if t % 11 == 0:
            x[t, 50:] = -math.inf
    _, _, _, ids, _ = sn.sn_logprob_fwd(x, top=top)
    assert torch.equal(ids.long(), best(x, top))


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("V,pad", [(5, 0), (12, 3), (40, 1), (259, 0), (1000, 5), (1024, 0), (1024, 3), (1025, 0)])
@pytest.mark.parametrize("kind", ["constant", "few values", "some above a tie", "masked", "rising", "NaN", "one lane's"])
def test_alternatives_of_narrow_rows(sn, dt, V, pad, kind):
    """Rows that a warp holds, from below one 16-byte piece to the widest, on and off the
    alignment: ties, masks and values that are no numbers, at each number of alternatives."""
    g = gen(V + pad)
    T = 37
    x = logits(T, V, dt, g, pad)
    new = x.clone()
    if kind == "constant":
        new[:] = torch.randn(T, 1, generator=g, device="cuda").to(x.dtype)
    elif kind == "few values":
        new[:] = torch.randint(3, (T, V), generator=g, device="cuda").to(x.dtype)
    elif kind == "some above a tie":
        new[:] = torch.where(torch.rand(T, V, generator=g, device="cuda") < 9 / V, 1.0, -2.0).to(x.dtype)
    elif kind == "masked":
        new[torch.rand(T, V, generator=g, device="cuda") < torch.linspace(0.5, 1, T, device="cuda")[:, None]] = -math.inf
        new[::3] = new[::3].clamp(min=torch.finfo(x.dtype).min)
    elif kind == "rising":
        new[:] = torch.linspace(-5, 5, V, device="cuda").to(x.dtype)
    elif kind == "NaN":
        new[torch.rand(T, V, generator=g, device="cuda") < torch.linspace(0, 1, T, device="cuda")[:, None]] = math.nan
        new[::4, 0] = math.nan
    else:
        per = 16 // x.element_size()
        new[:, (torch.arange(V, device="cuda") // per) % 32 < 2] += 40
    x.copy_(new)
    for top in {1, min(V, 7), min(V, 32)}:
        _, _, _, ids, _ = sn.sn_logprob_fwd(x, top=top)
        # NaN first, then by value
        key = torch.where(x.isnan(), math.inf, x.double() + 0.0)
        assert torch.equal(ids.long(), torch.sort(key, dim=1, descending=True, stable=True).indices[:, :top])


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("T,V,pad,opad,scale", [
    (1, 1, 0, 0, 1.0), (3, 7, 0, 0, 1.0), (9, 33, 2, 2, 0.5), (40, 1000, 0, 3, 1.0), (6, 50257, 0, 0, 1.25),
    (5, 50257, 7, 7, 1.0), (4, 8200, 8, 0, 2.0), (300, 257, 0, 0, 1.0)])
@pytest.mark.parametrize("terms", ["both", "logp", "entropy"])
def test_gradient(sn, dt, T, V, pad, opad, scale, terms):
    g = gen(V + T)
    x = logits(T, V, dt, g, pad).clone()
    x = spread(x.contiguous(), pad)
    if V > 5:
        x[0, 3:] = -math.inf
    target = torch.randint(min(V, 3), (T,), generator=g, device="cuda", dtype=torch.int32)
    target[1::4] = -1
    a, b = (torch.randn(T, generator=g, device="cuda") for _ in range(2))
    _, lse, H, _, _ = sn.sn_logprob_fwd(x, target, scale=scale)
    lp = dict(target=target, dlogp=a) if terms != "entropy" else {}
    en = dict(entropy=H, dentropy=b) if terms != "logp" else {}
    full, flat = guarded((T * (V + opad),), DT[dt])
    out = flat.view(T, V + opad)[:, :V]
    before = flat.view(T, V + opad)[:, V:].clone()
    sn.sn_logprob_bwd(x, lse, scale=scale, out=out, **lp, **en)
    s64 = float(torch.tensor(scale, dtype=torch.float32))
    z = x.double() * s64
    q = torch.log_softmax(z, 1)
    p = q.exp()
    qf = torch.where(p > 0, q, 0.0)
    ent = -(p * qf).sum(1, keepdim=True)
    one = torch.zeros_like(p)
    some = target >= 0
    one[some, target[some].long()] = 1.0
    ga = torch.where(some, a.double(), 0.0)[:, None] if lp else torch.zeros(T, 1, dtype=torch.float64, device="cuda")
    gb = b.double()[:, None] if en else torch.zeros(T, 1, dtype=torch.float64, device="cuda")
    ref = s64 * (ga * (one - p) - gb * p * (qf + ent))
    zf = torch.where(p > 0, z, 0.0)
    rel = 2.0 ** -22 * (zf.abs() + lse.double().abs().sum(1, keepdim=True)) + 2.0 ** -14
    size = p * (ga.abs() + gb.abs() * (qf.abs() + ent + 2 + math.log(V)))
    within(out, ref, s64 * size * rel + (s64 * ga.abs() * one) * 2.0 ** -23 + ref.abs() * UNIT[DT[dt]] * 1.02)
    assert guards_intact(full)
    after = flat.view(T, V + opad)[:, V:]
    bits = torch.int16 if dt == "bf16" else torch.int32
    assert torch.equal(after.contiguous().view(bits), before.contiguous().view(bits))
    place = x.clone(memory_format=torch.preserve_format) if not pad else spread(x.contiguous(), pad)
    assert torch.equal(sn.sn_logprob_bwd(place, lse, scale=scale, out=place, **lp, **en), out)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("T,V,pad,opad", [(9, 5, 0, 1), (17, 40, 3, 0), (17, 300, 1, 8), (18, 1000, 5, 2), (9, 1030, 47, 0),
                                          (10, 4099, 0, 3), (9, 50257, 47, 0)])
def test_gradient_of_rows_that_lie_differently(sn, dt, T, V, pad, opad):
    """Logits and gradient at every distance from their 16-byte boundaries, steps of 32 to 256 threads."""
    test_gradient(sn, dt, T, V, pad, opad, 1.25, "both")


def test_gradient_against_differences(sn):
    """Central differences of the forward in fp32, step 1/32 along a direction of unit elements: the
    third derivative's term (step^2 / 6) is below 1e-3 of the weights' sum, the forward's error
    (2^-14 a row over the step) below 4e-3 of it."""
    g = gen(3)
    T, V = 12, 1000
    x, D = (torch.randn(T, V, generator=g, device="cuda") for _ in range(2))
    target = torch.randint(V, (T,), generator=g, device="cuda", dtype=torch.int32)
    a, b = (torch.randn(T, generator=g, device="cuda") for _ in range(2))

    def f(y):
        logp, _, H, _, _ = sn.sn_logprob_fwd(y, target, scale=1.25)
        return (a.double() * logp.double()).sum() + (b.double() * H.double()).sum()

    _, lse, H, _, _ = sn.sn_logprob_fwd(x, target, scale=1.25)
    dx = sn.sn_logprob_bwd(x, lse, target, a, scale=1.25, entropy=H, dentropy=b)
    e = 1.0 / 32
    got = (f(x + e * D) - f(x - e * D)) / (2 * e)
    assert abs(float(got - (dx.double() * D.double()).sum())) <= 5e-3 * float(a.abs().sum() + b.abs().sum())


def test_invalid_targets(sn):
    basis = sn.Basis(torch.eye(16, 2, device="cuda").contiguous())
    x = torch.zeros(3, 10, device="cuda")
    target = torch.tensor([10, 2, -1], dtype=torch.int32, device="cuda")
    logp, lse, _, _, _ = sn.sn_logprob_fwd(x, target, basis=basis)
    with pytest.raises(sn.SNError) as e:
        sn.sn_check_errors(basis)
    assert e.value.status == sn.SN_ERR_BAD_ID
    assert float(logp[0]) == float(logp[2]) == 0 and abs(float(logp[1]) + math.log(10)) < 1e-5
    dx = sn.sn_logprob_bwd(x, lse, target, torch.ones(3, device="cuda"))
    assert bool((dx[[0, 2]] == 0).all())
    basis.destroy()


def test_refusals(sn):
    x = torch.zeros(4, 64, device="cuda")
    t = torch.zeros(4, dtype=torch.int32, device="cuda")
    f, l = torch.zeros(4, device="cuda"), torch.zeros(4, 2, device="cuda")
    for call in (lambda: sn.sn_logprob_fwd(x.half(), t), lambda: sn.sn_logprob_fwd(x, t.long()),
                 lambda: sn.sn_logprob_bwd(x, l.double(), t, f), lambda: sn.sn_logprob_bwd(x, l, t, f, out=x.bfloat16())):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: sn.sn_logprob_fwd(x.t(), t), lambda: sn.sn_logprob_fwd(x, t[:3]),
                 lambda: sn.sn_logprob_fwd(x.cpu(), t), lambda: sn.sn_logprob_bwd(x, f, t, f)):
        with pytest.raises(ValueError):
            call()
    big = torch.zeros(8, 64, device="cuda")
    for call, status in (
            (lambda: sn.sn_logprob_fwd(x, t, scale=0.0), sn.SN_ERR_INVALID_ARG),
            (lambda: sn.sn_logprob_fwd(x, t, scale=math.inf), sn.SN_ERR_INVALID_ARG),
            (lambda: sn.sn_logprob_fwd(x, t, top=33), sn.SN_ERR_INVALID_ARG),
            (lambda: sn.sn_logprob_fwd(x[:, :4], t, top=5), sn.SN_ERR_INVALID_ARG),
            (lambda: sn.sn_logprob_fwd(big.view(-1)[1:257].view(4, 64), t), sn.SN_ERR_ALIGNMENT),
            (lambda: sn.sn_logprob_bwd(x, l), sn.SN_ERR_INVALID_ARG),
            (lambda: sn.sn_logprob_bwd(x, l, t), sn.SN_ERR_INVALID_ARG),
            (lambda: sn.sn_logprob_bwd(x, l, dentropy=f), sn.SN_ERR_INVALID_ARG),
            (lambda: sn.sn_logprob_bwd(big[:4], l, t, f, out=big[2:6]), sn.SN_ERR_INVALID_ARG)):
        with pytest.raises(sn.SNError) as e:
            call()
        assert e.value.status == status
