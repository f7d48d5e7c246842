"""Activations and slopes of the gated projections where they vanish, relative to themselves.

Bars, relative: an exponential of x is within (1.173 |x| + 3) 2^-23 of itself, and what its argument is
off by counts |x| times: up to six roundings of 2^-24 of gelu_tanh's, two of gelu's slope's.  gelu's share is
half of erfc(-g / sqrt 2): within 4 2^-23, and its argument's two roundings count g^2 + 1 times.  A handful
of products and a division are within 2^-20 together.  Every output is rounded once, 2^-8 of itself or 2^-134
below bf16's normal numbers, where the shares are fp32 numbers off by up to 4 2^-149 and have been multiplied
by |g| < 128."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def tails(act):
    """All bf16 numbers from -128 to -4 (silu) or -16 to -4."""
    bits = torch.arange(0xC080, 0xC300 if act == "silu" else 0xC180, dtype=torch.int32)
    return (bits << 16).view(torch.float32).to(BF16).cuda()


def shares(g, act):
    """g Phi and the slope's two terms in fp64, and how far the share and the slope's term may be off."""
    if act == "silu":
        p = torch.sigmoid(g)
        e = (1.173 * g.abs() + 3 + g.abs()) * 2.0 ** -23
        return p, p, g * p * (1 - p), e, e
    if act == "gelu":
        p = 0.5 * torch.erfc(-g / math.sqrt(2))
        x = g * g / 2
        return (p, p, g * torch.exp(-x) / math.sqrt(2 * math.pi), (g * g + 5) * 2.0 ** -23,
                (1.173 * x + 3 + x) * 2.0 ** -23)
    k = 2 * math.sqrt(2 / math.pi)
    y = k * g * (1 + 0.044715 * g * g)
    p = torch.sigmoid(y)
    e = (1.173 * y.abs() + 3 + 3 * y.abs()) * 2.0 ** -23
    return p, p, g * p * (1 - p) * k * (1 + 3 * 0.044715 * g * g), e, e


def close(got, ref, e, size):
    """Within e + 2^-20 of `size` and a rounding."""
    bound = (e + 2.0 ** -20) * size
    err = (got.double() - ref).abs()
    ok = err <= bound + 2.0 ** -8 * (ref.abs() + bound) + 2.0 ** -134 + 2.0 ** -140
    assert bool(ok.all()), (int((~ok).sum()), got[~ok][:4], ref[~ok][:4])


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_gradients_where_the_activation_vanishes(sn, act):
    g = tails(act)
    G = g[:, None].expand(-1, 8).contiguous()
    one, W, X = torch.ones_like(G), torch.zeros(8, 8, device="cuda", dtype=BF16), torch.zeros_like(G)
    _, _, _, dG, dU = sn.sn_glu_bwd(one, X, W, W, G, one, act, need_dX=False, need_dW=False)
    x = G.double()
    p, a, b, ep, eb = shares(x, act)
    close(dU, x * p, ep, (x * p).abs())
    close(dG, a + b, torch.maximum(ep, eb), a.abs() + b.abs())


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("few", [False, True])
def test_forward_where_the_activation_vanishes(sn, act, few):
    """G is a bf16 number exactly and U is 1."""
    g = tails(act)
    X = torch.zeros(len(g), 8, device="cuda", dtype=BF16)
    X[:, 0], X[:, 1] = g, 1
    Wg, Wu = (torch.zeros(8, 8, device="cuda", dtype=BF16) for _ in range(2))
    Wg[:, 0], Wu[:, 1] = 1, 1
    step = 100 if few else len(g)
    if not few and len(g) <= 224:                  # (as many tokens as take the tiles)
        X, g = X.repeat(2, 1), g.repeat(2)
        step = len(g)
    H = torch.cat([sn.sn_glu_fwd(X[i:i + step], Wg, Wu, act)[0] for i in range(0, len(g), step)])
    x = g.double()[:, None].expand(-1, 8)
    p, _, _, ep, _ = shares(x, act)
    close(H, x * p, ep, (x * p).abs())
