"""The step operators where offsets pass 32 bits: more than 2^31 elements in a buffer, the last rows
against fp64 (the bars of the operators' own tests)."""
import pytest
import torch

from step_util import UNIT, gen, within

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def test_norm_of_many_rows(sn):
    T, d = 270000, 8192
    assert T * d > 2 ** 31
    g = gen(1)
    x = torch.randn(T, d, generator=g, device="cuda", dtype=BF16)
    w = torch.randn(d, generator=g, device="cuda")
    Y, H = sn.sn_rmsnorm_fwd(x, w, 1e-5, R=x)
    codes, scale, _ = sn.sn_rmsnorm_fwd_quant(x, w, 1e-5, "int8", group=128)
    dX, dw = sn.sn_rmsnorm_bwd(x, H, w, 1e-5, dH=Y)
    for r in (slice(0, 2), slice(T - 2, T)):
        h = 2 * x[r].double()
        rs = (h.square().mean(1, keepdim=True) + 1e-5).rsqrt()
        y = h * rs * w.double()
        within(Y[r], y, y.abs() * (2.0 ** -18 + 1.01 * UNIT[BF16]))
        n, q = h * rs, x[r].double() * w.double()
        dx = rs * (q - n * (q * n).mean(1, keepdim=True)) + Y[r].double()
        within(dX[r], dx, (dx.abs() + Y[r].double().abs()) * 1.02 * UNIT[BF16] + 2.0 ** -14)
        y = y / 2 * (h.square().mean(1, keepdim=True) + 1e-5).sqrt() * ((h / 2).square().mean(1, keepdim=True) + 1e-5).rsqrt()
        per = scale[r].double().repeat_interleave(128, 1)
        within(codes[r].view(torch.int8).double() * per, y, per * 0.501 + y.abs() * 2.0 ** -16)
    assert bool(dw.isfinite().all())


def test_table_of_many_rows(sn):
    V, d, T = 300000, 8192, 3000
    assert V * d > 2 ** 31
    g = gen(2)
    table = torch.randn(V, d, generator=g, device="cuda", dtype=BF16)
    ids = torch.randint(V - 500, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    X = sn.sn_embed_fwd(table, ids)
    assert torch.equal(X, table[ids.long()])
    dE = sn.sn_embed_bwd(X, ids, V, out=table)
    ref = torch.zeros(500, d, dtype=torch.float64, device="cuda").index_add_(0, ids.long() - (V - 500), X.double())
    mag = torch.zeros_like(ref).index_add_(0, ids.long() - (V - 500), X.double().abs())
    within(dE[-500:], ref, mag * 2.0 ** -17 + ref.abs() * 1.01 * UNIT[BF16])
    assert not bool(dE[:-500].any())


def test_many_logits(sn):
    T, V = 17000, 128257
    assert T * V > 2 ** 31
    g = gen(3)
    x = torch.randn(T, V, generator=g, device="cuda", dtype=BF16)
    target = torch.randint(V, (T,), generator=g, device="cuda", dtype=torch.int32)
    logp, lse, H, ids, alt = sn.sn_logprob_fwd(x, target, top=4)
    last = x[-3:].clone()
    dx = sn.sn_logprob_bwd(x, lse, target, torch.ones(T, device="cuda"), out=x)
    q = torch.log_softmax(last.double(), 1)
    within(logp[-3:], q.gather(1, target[-3:].long()[:, None])[:, 0], 2.0 ** -14)
    assert torch.equal(ids[-3:].long(), torch.sort(last.double(), dim=1, descending=True, stable=True).indices[:, :4])
    ref = -q.exp()
    ref[torch.arange(3), target[-3:].long()] += 1
    within(dx[-3:], ref, ref.abs() * (1.02 * UNIT[BF16] + 2.0 ** -13))


def test_a_gradient_of_many_elements(sn):
    n = 2 ** 31 + 70001
    t = torch.full((n,), 2.0 ** -8, device="cuda", dtype=BF16)
    L = sn.GradList([t])
    norm = sn.sn_grads_clip(L, sn.sn_grads_sumsq(L), 1.0)
    want = 2.0 ** -8 * n ** 0.5
    assert abs(float(norm) - want) <= 2.0 ** -18 * want
    assert bool((t == torch.tensor(2.0 ** -8 / want).bfloat16().cuda()).all())
