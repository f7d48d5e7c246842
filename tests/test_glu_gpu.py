"""Gated projections H = act(X Wg^T) * (X Wu^T) and their gradients against fp64 torch.

Bars.  Products of bf16 values are exact in fp32; 16 of them are added at a time to the sum so far,
each step off by at most 2^-22 of what has been summed (a truncated, not a rounded, addition of the
16 and of the sum), so an inner dimension n costs (n / 16 + 2) 2^-22 of the sum of magnitudes.  The
activation and its slope are within 2^-17 of 1 + |g| (exponentials of |g| < 32 within 2^-19,
a division and a few products beside them).  Every output is rounded once: 2^-8 in bf16."""
import math

import pytest
import torch

from step_util import gen, spread, within

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
ACTS = ["silu", "gelu", "gelu_tanh", "relu"]
# one token to several tiles, widths that fill no tile, more tiles than CTAs
SIZES = [(1, 8, 8), (1, 64, 64), (3, 72, 40), (15, 256, 512), (16, 96, 1224), (17, 520, 128),
         (75, 136, 2056), (128, 200, 264), (129, 136, 264), (200, 512, 384), (256, 256, 256),
         (257, 264, 1032), (300, 64, 2056), (515, 1032, 136), (1000, 8, 16), (3000, 256, 5000)]
#: every way of the outer products: long and short sums, one tile and many
GRADS = SIZES + [(4100, 72, 40), (9000, 264, 136), (5, 2048, 264), (700, 2056, 24), (130, 24, 8200)]


def acc(n):
    return (n / 16 + 2) * 2.0 ** -22


def act64(g, act):
    """The activation and its slope."""
    if act == "relu":
        return g.clamp(min=0), (g > 0).double()
    if act == "silu":
        p = torch.sigmoid(g)
        return g * p, p + g * p * (1 - p)
    if act == "gelu":
        p = 0.5 * torch.erfc(-g / math.sqrt(2))
        return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    t = torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 0.134145 * g * g)


def inputs(T, d, f, seed):
    g = gen(seed)

    def normal(*shape, std=1.0):
        return (std * torch.randn(*shape, generator=g, device="cuda")).to(BF16)

    return normal(T, d, std=2.0), normal(f, d, std=d ** -0.5), normal(f, d, std=d ** -0.5), normal(T, f)


def guarded(rows, cols, dtype=BF16):
    """A tensor with rows in front and behind, all of one pattern."""
    full = torch.full((rows + 4, cols), 7.25, dtype=dtype, device="cuda")
    return full, full[2:-2]


def untouched(full):
    return bool((full[:2] == 7.25).all() and (full[-2:] == 7.25).all())


def check_fwd(X, Wg, Wu, act, H, G=None, U=None):
    x, wg, wu = X.double(), Wg.double(), Wu.double()
    g, u = x @ wg.T, x @ wu.T
    eg, eu = (acc(x.shape[1]) * (x.abs() @ w.abs().T) for w in (wg, wu))
    if G is not None:
        within(G, g, eg + 2.0 ** -8 * (g.abs() + eg))
        within(U, u, eu + 2.0 ** -8 * (u.abs() + eu))
    a = act64(g, act)[0]
    e = (1.2 * eg + 2.0 ** -17 * (1 + g.abs()) * g.abs()) * (u.abs() + eu) + a.abs() * eu
    within(H, a * u, e + 2.0 ** -8 * ((a * u).abs() + e))


@pytest.mark.parametrize("T,d,f", SIZES)
@pytest.mark.parametrize("keep", [False, True])
def test_forward(sn, T, d, f, keep):
    act = ACTS[(T + d) % 4]
    X, Wg, Wu, _ = inputs(T, d, f, T + d + f)
    (fh, H), (fg, G), (fu, U) = (guarded(T, f) for _ in range(3))
    if keep:
        sn.sn_glu_fwd(X, Wg, Wu, act, out=H, G=G, U=U)
        check_fwd(X, Wg, Wu, act, H, G, U)
    else:
        assert sn.sn_glu_fwd(X, Wg, Wu, act, out=H)[1:] == (None, None)
        check_fwd(X, Wg, Wu, act, H)
    assert untouched(fh) and untouched(fg) and untouched(fu)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T", [40, 300])
def test_activations_and_row_strides(sn, act, T):
    X, Wg, Wu, _ = inputs(T, 264, 136, 3)
    H, G, U = sn.sn_glu_fwd(spread(X, 24), Wg, Wu, act, keep=True)
    check_fwd(X, Wg, Wu, act, H, G, U)
    plain = sn.sn_glu_fwd(X, Wg, Wu, act)[0]
    assert torch.equal(plain, H)


def check_bwd(dH, X, Wg, Wu, G, U, act, got, add=None):
    dX, dWg, dWu, dG, dU = got
    h, g, u = dH.double(), G.double(), U.double()
    a, s = act64(g, act)
    within(dG, h * u * s, (h * u).abs() * 2.0 ** -17 * (1 + g.abs()) + 2.0 ** -8 * (h * u * s).abs())
    within(dU, h * a, h.abs() * 2.0 ** -17 * (1 + g.abs()) * g.abs() + 2.0 ** -8 * (h * a).abs())
    T, f = dH.shape
    q, r, x, wg, wu = dG.double(), dU.double(), X.double(), Wg.double(), Wu.double()
    if dX is not None:
        ref = q @ wg + r @ wu
        e = acc(2 * f) * (q.abs() @ wg.abs() + r.abs() @ wu.abs())
        within(dX, ref, e + 2.0 ** -8 * (ref.abs() + e))
    for out, p, was in ((dWg, q, add and add[0]), (dWu, r, add and add[1])):
        if out is None:
            continue
        ref, e = p.T @ x, acc(T) * (p.abs().T @ x.abs())
        if was is not None:
            ref = ref + was.double()
        e = e + 2.0 ** -23 * (ref.abs() + (0 if was is None else was.double().abs()))
        within(out, ref, e + (2.0 ** -8 if out.dtype == BF16 else 2.0 ** -24) * (ref.abs() + e))


@pytest.mark.parametrize("T,d,f", GRADS)
def test_gradients(sn, T, d, f):
    act = ACTS[(T + f) % 4]
    X, Wg, Wu, dH = inputs(T, d, f, T + d + f)
    _, G, U = sn.sn_glu_fwd(X, Wg, Wu, act, keep=True)
    outs = [guarded(T, d), guarded(f, d), guarded(f, d), guarded(T, f), guarded(T, f)]
    dX, dWg, dWu, dG, dU = (o[1] for o in outs)
    got = sn.sn_glu_bwd(dH, X, Wg, Wu, G, U, act, dG=dG, dU=dU, dX=dX, dW_gate=dWg, dW_up=dWu)
    check_bwd(dH, X, Wg, Wu, G, U, act, got)
    assert all(untouched(o[0]) for o in outs)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("T,d,f", [(300, 136, 264), (5000, 72, 40)])
def test_accumulated_gradients_strides_and_in_place(sn, dt, T, d, f):
    X, Wg, Wu, dH = inputs(T, d, f, 5)
    _, G, U = sn.sn_glu_fwd(X, Wg, Wu, "silu", keep=True)
    was = [torch.randn(f, d, generator=gen(6), device="cuda").to(dt) for _ in range(2)]
    out = [w.clone() for w in was]
    g, u = G.clone(), U.clone()
    got = sn.sn_glu_bwd(spread(dH, 8), spread(X, 16), Wg, Wu, g, u, dG=g, dU=u, dW_gate=out[0],
                        dW_up=out[1], accumulate=True)
    assert got[1] is out[0] and got[3] is g
    check_bwd(dH, X, Wg, Wu, G, U, "silu", got, add=was)


def test_parts_left_out(sn):
    X, Wg, Wu, dH = inputs(200, 136, 264, 7)
    _, G, U = sn.sn_glu_fwd(X, Wg, Wu, "gelu", keep=True)
    whole = sn.sn_glu_bwd(dH, X, Wg, Wu, G, U, "gelu", grad_dtype=F32)
    assert whole[1].dtype == F32
    only_x = sn.sn_glu_bwd(dH, X, Wg, Wu, G, U, "gelu", need_dW=False)
    only_w = sn.sn_glu_bwd(dH, X, Wg, Wu, G, U, "gelu", need_dX=False, grad_dtype=F32)
    neither = sn.sn_glu_bwd(dH, X, Wg, Wu, G, U, "gelu", need_dX=False, need_dW=False)
    assert only_x[1] is None and only_w[0] is None and neither[:3] == (None, None, None)
    assert torch.equal(only_x[0], whole[0]) and torch.equal(only_w[1], whole[1])
    assert torch.equal(only_w[2], whole[2]) and torch.equal(neither[3], whole[3])


def test_gradient_against_differences(sn):
    """dX and the weights' gradients against central differences of the fp64 formula."""
    T, d, f = 6, 24, 16
    X, Wg, Wu, dH = inputs(T, d, f, 9)
    _, G, U = sn.sn_glu_fwd(X, Wg, Wu, "silu", keep=True)
    dX, dWg, dWu, _, _ = sn.sn_glu_bwd(dH, X, Wg, Wu, G, U, "silu")
    at = [t.double() for t in (X, Wg, Wu)]

    def value(x, wg, wu):
        return (act64(x @ wg.T, "silu")[0] * (x @ wu.T) * dH.double()).sum()

    for which, grad in enumerate((dX, dWg, dWu)):
        scale = float(grad.double().abs().max())
        for i, j in ((0, 0), (3, 5), (grad.shape[0] - 1, d - 1)):
            ends = []
            for step in (1e-4, -1e-4):
                moved = [t.clone() for t in at]
                moved[which][i, j] += step
                ends.append(float(value(*moved)))
            # G, U, dG, dU rounded to bf16 in between: 4 2^-8 of the terms of a sum of at most 24
            assert abs(float(grad[i, j]) - (ends[0] - ends[1]) / 2e-4) <= 0.04 * scale


def test_extreme_projections(sn):
    """Saturated activations: large magnitudes of either sign give no NaN and the right side."""
    d = 16
    X = torch.ones(1, d, device="cuda", dtype=BF16)
    sizes = torch.tensor([-1e30, -1e10, -200.0, -30.0, 0.0, 30.0, 200.0, 1e10], device="cuda")
    Wg = (sizes[:, None] / d).expand(8, d).to(BF16).contiguous()
    Wu = torch.full((8, d), 1 / 16, device="cuda", dtype=BF16)
    for act in ACTS:
        H, G, U = sn.sn_glu_fwd(X, Wg, Wu, act, keep=True)
        dH = torch.ones_like(H)
        _, _, _, dG, dU = sn.sn_glu_bwd(dH, X, Wg, Wu, G, U, act)
        g = G.double()
        on = g > 0
        for got in (H, dU):
            assert torch.isfinite(got).all()
            assert (got[~on].abs() <= 1e-10).all() and torch.equal(got[on], G[on])
        # at |g| = 30 the slope is within |g| exp(-|g|) < 3e-12 of its limit
        far = g.abs() > 20
        assert ((dG[far].double() - on[far].double()).abs() <= 1e-10).all()


@pytest.mark.parametrize("T", [20, 300])
@pytest.mark.parametrize("act", ACTS)
def test_nans_and_infinities_stay_in_their_rows(sn, act, T):
    """A NaN in a token's row, an infinity in a weight's: that row and that feature, nothing else."""
    X, Wg, Wu, dH = inputs(T, 72, 136, 21)
    H, G, U = sn.sn_glu_fwd(X, Wg, Wu, act, keep=True)
    x, wu = X.clone(), Wu.clone()
    x[7, 3] = float("nan")
    wu[130, 0] = float("inf")
    h, g, u = sn.sn_glu_fwd(x, Wg, wu, act, keep=True)
    assert bool(torch.isnan(h[7]).all()) and bool(torch.isnan(g[7]).all()) and bool(torch.isnan(u[7]).all())
    rows = [t for t in range(T) if t != 7]
    cols = [j for j in range(136) if j != 130]
    assert torch.equal(h[rows][:, cols], H[rows][:, cols]) and torch.equal(g[rows], G[rows])
    assert not bool(torch.isfinite(u[rows, 130]).any())
    dh = dH.clone()
    dh[11, 5] = float("nan")
    was = sn.sn_glu_bwd(dH, X, Wg, Wu, G, U, act)
    got = sn.sn_glu_bwd(dh, X, Wg, Wu, G, U, act)
    assert bool(torch.isnan(got[0][11]).all()) and bool(torch.isnan(got[1][5]).all()) and bool(torch.isnan(got[2][5]).all())
    for i, bad in ((0, 11), (1, 5), (2, 5)):
        keep = [r for r in range(got[i].shape[0]) if r != bad]
        assert torch.equal(got[i][keep], was[i][keep])


def test_no_tokens(sn):
    X, Wg, Wu, dH = inputs(1, 64, 32, 1)
    H, G, U = sn.sn_glu_fwd(X[:0], Wg, Wu, keep=True)
    assert H.shape == G.shape == (0, 32)
    dX, dWg, dWu, _, _ = sn.sn_glu_bwd(dH[:0], X[:0], Wg, Wu, G, U)
    assert dX.shape == (0, 64) and not dWg.any() and not dWu.any()
    keep = dWg.fill_(3.0)
    sn.sn_glu_bwd(dH[:0], X[:0], Wg, Wu, G, U, dW_gate=keep, dW_up=dWu, accumulate=True)
    assert (keep == 3.0).all()


def test_same_bits_every_time(sn):
    X, Wg, Wu, dH = inputs(700, 520, 1032, 11)
    first = None
    for _ in range(3):
        H, G, U = sn.sn_glu_fwd(X, Wg, Wu, "silu", keep=True)
        all_ = (H, G, U) + tuple(sn.sn_glu_bwd(dH, X, Wg, Wu, G, U, grad_dtype=F32))
        first = first or all_
        assert all(torch.equal(a, b) for a, b in zip(first, all_))


def test_refusals(sn):
    X, Wg, Wu, dH = inputs(40, 64, 32, 13)
    H, G, U = sn.sn_glu_fwd(X, Wg, Wu, keep=True)
    bad = sn.SNError

    def fwd(**kw):
        a = dict(X=X, W_gate=Wg, W_up=Wu)
        a.update(kw)
        return lambda: sn.sn_glu_fwd(**a)

    def bwd(**kw):
        a = dict(dH=dH, X=X, W_gate=Wg, W_up=Wu, G=G, U=U)
        a.update(kw)
        return lambda: sn.sn_glu_bwd(**a)

    flat = torch.zeros(40 * 64 + 8, device="cuda", dtype=BF16)
    for call, error in (
            (fwd(act="tanh"), KeyError), (fwd(W_up=Wu[:16]), ValueError), (fwd(W_gate=Wg.float()), TypeError),
            (fwd(X=X.cpu()), ValueError), (fwd(X=X.T.contiguous().T), ValueError), (fwd(out=H[:3]), ValueError),
            (fwd(X=X.float(), W_gate=Wg.float(), W_up=Wu.float()), bad),
            (fwd(X=X[:, :60].contiguous(), W_gate=Wg[:, :60].contiguous(), W_up=Wu[:, :60].contiguous()), bad),
            (fwd(W_gate=Wg[:20], W_up=Wu[:20]), bad),
            (fwd(X=flat[1:2561].view(40, 64)), bad), (fwd(X=spread(X, 3)), bad),
            (fwd(out=G, G=G, U=U), bad), (fwd(G=G, U=G), bad),
            (bwd(dX=X), bad), (bwd(dG=U), bad), (bwd(dG=dH), bad), (bwd(dG=G, dU=G), bad),
            (bwd(dW_gate=Wg), bad), (bwd(accumulate=True), ValueError), (bwd(G=G[:, :16]), ValueError),
            (bwd(dH=spread(dH, 4)), bad), (bwd(X=X[:20]), ValueError)):
        with pytest.raises(error):
            call()
    torch.cuda.synchronize()
