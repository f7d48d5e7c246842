"""The step operators run together around a boundary: the example's gradients against autograd of
the same model in fp64, its training, its scores, and the calls in a CUDA graph.

Bars.  The example's products and activations are bf16 (2^-8 a rounding); a gradient has passed six
to ten of them, so 10 * 2^-8 = 4e-2 of its norm, where each rounding's part is random, with the
boundary's projection of the gradient (Sec. 4.4) in the reference too."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lm(sn):
    from paper_2506_01260_gb300 import lm_step
    return lm_step


class Project(torch.autograd.Function):
    """The boundary: the stream as it is (it lies in S apart from the fixed embeddings), its
    gradient projected onto S."""

    @staticmethod
    def forward(ctx, x, P):
        ctx.P = P
        return x

    @staticmethod
    def backward(ctx, g):
        return g @ ctx.P, None


def reference(m, ids, target, U):
    """Loss and gradients of the same model in fp64."""
    p = {n: getattr(m, n).double().requires_grad_() for n in m.grads}

    def norm(x, w):
        return x * (x.square().mean(1, keepdim=True) + 1e-5).rsqrt() * w

    i = ids.long()
    h0 = m.T_fixed.double()[i] + p["T_S"][i]
    x0 = h0 + torch.relu(norm(h0, p["w0"]) @ p["W_up"].T) @ p["W_down"].T
    x1 = Project.apply(x0, U @ U.T)
    q = torch.log_softmax(norm(x1, p["w1"]) @ p["W_head"].T, 1)
    some = target >= 0
    loss = -q[some, target[some].long()].mean()
    loss.backward()
    return loss.detach(), {n: t.grad for n, t in p.items()}


def test_gradients_match_autograd(sn, lm):
    m = lm.TwoStage(vocab=300, d=128, d_ff=192, k=12, seed=3)
    U = torch.zeros(m.d, 12, device="cuda", dtype=torch.float64)
    # the basis' columns, from the library: rows of the identity times U
    U[:] = sn.sn_compress_bwd(m.basis, torch.eye(m.d, device="cuda")).double()
    ids, target = lm.chain(700, m.vocab, seed=1)
    target[::9] = -1
    loss = m.backward(ids, target)
    sn.sn_check_errors(m.basis)
    ref_loss, ref = reference(m, ids, target, U)
    assert abs(float(loss) - float(ref_loss)) <= 4e-2 * float(ref_loss)
    for n, g in m.grads.items():
        assert float((g.double() - ref[n]).norm() / ref[n].norm()) <= 4e-2, n


def test_training_learns_the_chain(sn, lm):
    m = lm.TwoStage(seed=1)
    losses = [float(m.step(*lm.chain(2048, m.vocab, seed=i))[0]) for i in range(60)]
    sn.sn_check_errors(m.basis)
    assert all(math.isfinite(x) for x in losses)
    assert abs(losses[0] - math.log(m.vocab)) < 1.0 and sum(losses[-5:]) / 5 < 0.8 * losses[0]
    ids, _ = lm.chain(500, m.vocab, seed=99)
    logp, H, alt, alt_logp = m.score(ids)
    assert float(logp[-1]) == 0 and bool((alt_logp[:, :-1] >= alt_logp[:, 1:]).all())
    assert bool((H > 0).all()) and bool((H <= math.log(m.vocab) + 1e-3).all())
    hit = alt[:-1] == ids[1:, None]                          # an alternative's score is its token's
    assert torch.equal(alt_logp[:-1][hit], logp[:-1][hit.any(1)])


def test_the_calls_in_a_cuda_graph(sn):
    """Every step operator, captured and replayed on new inputs: the eager calls' bits."""
    g = torch.Generator(device="cuda").manual_seed(2)
    T, d, V = 1500, 264, 1001
    x, r, dy = (torch.randn(T, d, generator=g, device="cuda").bfloat16() for _ in range(3))
    w = torch.randn(d, generator=g, device="cuda")
    ids = torch.randint(V, (T,), generator=g, device="cuda", dtype=torch.int32)
    table = torch.randn(V, d, generator=g, device="cuda").bfloat16()
    head = torch.randn(V, d, generator=g, device="cuda").bfloat16() / 16
    logits = torch.empty(T, V, device="cuda", dtype=torch.bfloat16)
    da, db = torch.randn(T, generator=g, device="cuda"), torch.randn(T, generator=g, device="cuda")
    grads = [torch.randn(n, generator=g, device="cuda") for n in (1000, 70000)]
    clipped = [torch.empty_like(t) for t in grads]
    glist = sn.GradList(grads, out=clipped)

    def calls():
        X = sn.sn_embed_fwd(table, ids, scale=2.0)
        Y, H = sn.sn_rmsnorm_fwd(x, w, 1e-5, R=r)
        codes, scale, _ = sn.sn_rmsnorm_fwd_quant(x, w, 1e-5, "int8", R=r, group=64)
        dX, dw = sn.sn_rmsnorm_bwd(dy, H, w, 1e-5, dH=x)
        dE = sn.sn_embed_bwd(dX, ids, V, out_dtype=torch.float32)
        few = sn.sn_embed_bwd(dX[:300], ids[:300], V)
        logp, lse, ent, alt, alt_logp = sn.sn_logprob_fwd(logits, ids, top=6)
        dl = sn.sn_logprob_bwd(logits, lse, ids, da, entropy=ent, dentropy=db)
        one = sn.sn_logprob_fwd(logits[:1], ids[:1], top=3)
        norm = sn.sn_grads_clip(glist, sn.sn_grads_sumsq(glist), 1.0)
        return [X, Y, H, codes, scale, dX, dw, dE, few, logp, lse, ent, alt, alt_logp, dl, *one, norm,
                *[c.clone() for c in clipped]]

    def fill(seed):
        k = torch.Generator(device="cuda").manual_seed(seed)
        for t in (x, r, dy, *grads):
            t.copy_(torch.randn(t.shape, generator=k, device="cuda"))
        ids.copy_(torch.randint(V, (T,), generator=k, device="cuda"))
        torch.matmul(x, head.T, out=logits)

    fill(1)
    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = calls()
    for seed in (5, 6):
        fill(seed)
        want = [t.clone() for t in calls()]
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(got, want)):
            assert torch.equal(a, b), i


def test_calls_do_not_allocate(sn):
    """With outputs and workspaces given, no call touches the caching allocator or the device's
    free memory."""
    T, d, V = 2000, 512, 3000
    x, r, h, y = (torch.randn(T, d, device="cuda").bfloat16() for _ in range(4))
    w, dw = torch.ones(d, device="cuda"), torch.empty(d, device="cuda")
    ids = torch.randint(V, (T,), device="cuda", dtype=torch.int32)
    dE = torch.empty(V, d, device="cuda")
    we = torch.empty(sn.sn_embed_bwd_workspace(T, V, d), dtype=torch.uint8, device="cuda")
    wn = torch.empty(sn.sn_rmsnorm_bwd_workspace(T, d), dtype=torch.uint8, device="cuda")
    codes, scale = torch.empty(T, d, dtype=torch.uint8, device="cuda"), torch.empty(T, device="cuda")
    L = sn.GradList([dE])
    sq, nrm = torch.empty(1, dtype=torch.float64, device="cuda"), torch.empty(1, device="cuda")

    def calls():
        sn.sn_embed_fwd(dE, ids, out=y)
        sn.sn_rmsnorm_fwd(x, w, 1e-5, R=r, H=h, out=y)
        sn.sn_rmsnorm_fwd_quant(x, w, 1e-5, "e4m3", R=r, H=h, codes=codes, scale=scale)
        sn.sn_rmsnorm_bwd(x, h, w, 1e-5, dH=r, out=y, dw=dw, workspace=wn)
        sn.sn_embed_bwd(y, ids, V, out=dE, workspace=we)
        sn.sn_grads_clip(L, sn.sn_grads_sumsq(L, out=sq), 1.0, norm=nrm)

    calls()
    torch.cuda.synchronize()
    before = (torch.cuda.memory_stats()["allocation.all.allocated"], torch.cuda.mem_get_info()[0])
    for _ in range(3):
        calls()
    torch.cuda.synchronize()
    assert (torch.cuda.memory_stats()["allocation.all.allocated"], torch.cuda.mem_get_info()[0]) == before
