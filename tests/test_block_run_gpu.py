"""The gated projections and the norms around a block as they are used: together in the example's
block (against autograd of the same model in fp64), in CUDA graphs, on other streams, on a part of
the SMs, past 32-bit offsets, two calls at once.

Bars of the example: as for the two-stage model's (ten roundings of 2^-8 at most on a gradient's way)."""
import pytest
import torch

from step_util import gen, spread
from test_glu_gpu import act64, check_bwd, check_fwd, inputs
from test_blocknorm_gpu import check_bwd as check_norm_bwd, check_fwd as check_norm_fwd, inputs as norm_inputs
from test_green_context_gpu import GreenContext, IGNORE_COSCHEDULING
from test_lm_step_gpu import Project, lm  # noqa: F401
from test_stream_memory import BUSY, overwrite

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
EPS = 1e-5


def reference(m, ids, target, U):
    """Loss and gradients of the gated model in fp64."""
    p = {n: getattr(m, n).double().requires_grad_() for n in m.grads}

    def norm(x, w):
        return x * (x.square().mean(1, keepdim=True) + EPS).rsqrt() * w

    i = ids.long()
    h0 = m.T_fixed.double()[i] + p["T_S"][i]
    x0 = h0 + torch.relu(norm(h0, p["w0"]) @ p["W_up"].T) @ p["W_down"].T
    x1 = Project.apply(x0, U @ U.T)
    y1 = norm(x1, p["w1"])
    H = act64(y1 @ p["V_gate"].T, m.act)[0] * (y1 @ p["V_up"].T)
    h = x1 + m.scale * p["gate"] * norm(H @ p["V_down"].T, p["w_post"])
    q = torch.log_softmax(norm(h, p["w_pre"]) @ p["W_head"].T, 1)
    some = target >= 0
    loss = -q[some, target[some].long()].mean()
    loss.backward()
    return loss.detach(), {n: t.grad for n, t in p.items()}


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated_example_matches_autograd(sn, lm, act):  # noqa: F811
    m = lm.GatedTwoStage(vocab=300, d=128, d_ff=192, k=12, seed=3)
    m.act = act
    U = sn.sn_compress_bwd(m.basis, torch.eye(m.d, device="cuda")).double()
    ids, target = lm.chain(700, m.vocab, seed=1)
    target[::9] = -1
    loss = m.backward(ids, target)
    sn.sn_check_errors(m.basis)
    ref_loss, ref = reference(m, ids, target, U)
    assert abs(float(loss) - float(ref_loss)) <= 4e-2 * float(ref_loss)
    assert set(ref) == set(m.grads) and len(ref) == 12
    for n, g in m.grads.items():
        assert float((g.double() - ref[n]).norm() / ref[n].norm()) <= 4e-2, n


def test_gated_example_runs(sn, lm):  # noqa: F811
    m = lm.GatedTwoStage(seed=1)
    for i in range(3):
        loss, norm = m.step(*lm.chain(500, m.vocab, seed=i))
        assert bool(torch.isfinite(loss)) and bool(torch.isfinite(norm))
    logp, H, alt, alt_logp = m.score(lm.chain(9, m.vocab, seed=5)[0])
    sn.sn_check_errors(m.basis)
    assert bool(torch.isfinite(H).all()) and alt.shape == (9, 5) and float(logp[-1]) == 0


def block(sn, x, Wg, Wu, down, dz, w, gate, stream=None):
    """A block forward and back, and what it gives."""
    H, G, U = sn.sn_glu_fwd(x, Wg, Wu, "silu", keep=True, stream=stream)
    few = sn.sn_glu_fwd(x[:37], Wg, Wu, "gelu_tanh", stream=stream)[0]
    z, h = sn.sn_blocknorm_fwd(down, x, w, w, EPS, scale=0.5, gate=gate, stream=stream)
    dY, dR, a, b, c = sn.sn_blocknorm_bwd(dz, h, down, w, w, EPS, scale=0.5, gate=gate, dH=z, stream=stream)
    back = sn.sn_glu_bwd(H, x, Wg, Wu, G, U, grad_dtype=F32, stream=stream)
    one = sn.sn_glu_bwd(H[:40], x[:40], Wg, Wu, G[:40], U[:40], stream=stream)
    return [H, G, U, few, z, h, dY, dR, a, b, c, *back, *one]


def block_inputs(T=1200, d=264, f=1032, gates=8, seed=1):
    g = gen(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda").to(BF16)

    return [normal(T, d), normal(f, d) / 16, normal(f, d) / 16, normal(T, d), normal(T, d),
            torch.rand(d, generator=g, device="cuda") + 0.5, normal(gates, d)]


def test_in_a_cuda_graph(sn):
    """Captured with the workspaces that the calls make, replayed on new inputs: the eager bits."""
    args = block_inputs()
    block(sn, *args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = block(sn, *args)
    for seed in (5, 6):
        for t, new in zip(args, block_inputs(seed=seed)):
            t.copy_(new)
        want = [t.clone() for t in block(sn, *args)]
        for t in got:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(got, want)):
            assert torch.equal(a, b), i


@pytest.mark.parametrize("raw", [False, True])
def test_on_a_busy_stream(sn, raw):
    args = block_inputs(T=3000)
    want = block(sn, *args)
    overwrite()
    for turn in range(2):
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            torch.cuda._sleep(BUSY)
        got = block(sn, *args, stream=side.cuda_stream if raw else side)
        kept = overwrite()
        assert not side.query()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(got, want)):
            assert torch.equal(a, b), (turn, i)
        del kept, got


def test_two_at_once(sn):
    """Blocks on two streams at the same time, each with its own workspaces."""
    sets = [block_inputs(T=2400, seed=s) for s in (1, 2)]
    want = [block(sn, *s) for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for s, args in zip(streams, sets):
            with torch.cuda.stream(s):
                got.append(block(sn, *args))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_no_allocation_with_everything_given(sn):
    T, d, f = 700, 264, 1032
    x, Wg, Wu, down, dz, w, gate = block_inputs(T, d, f, 7)
    H, G, U, dG, dU = (torch.empty(T, f, device="cuda", dtype=BF16) for _ in range(5))
    z, h, dX, dY, dR = (torch.empty(T, d, device="cuda", dtype=BF16) for _ in range(5))
    a, b = torch.empty(f, d, device="cuda"), torch.empty(f, d, device="cuda")
    dw = [torch.empty(d, device="cuda") for _ in range(2)] + [torch.empty(7, d, device="cuda")]
    w1 = torch.empty(max(16, sn.sn_glu_bwd_workspace(T, d, f)), dtype=torch.uint8, device="cuda")
    w2 = torch.empty(sn.sn_blocknorm_bwd_workspace(T, d, 7), dtype=torch.uint8, device="cuda")

    def calls():
        sn.sn_glu_fwd(x, Wg, Wu, out=H, G=G, U=U)
        sn.sn_blocknorm_fwd(down, x, w, w, EPS, gate=gate, H=h, out=z)
        sn.sn_blocknorm_bwd(dz, h, down, w, w, EPS, gate=gate, dY=dY, dR=dR, dw_post=dw[0], dw_pre=dw[1],
                            dgate=dw[2], workspace=w2)
        sn.sn_glu_bwd(H, x, Wg, Wu, G, U, dG=dG, dU=dU, dX=dX, dW_gate=a, dW_up=b, workspace=w1)

    calls()
    torch.cuda.synchronize()
    before = (torch.cuda.memory_stats()["allocation.all.allocated"], torch.cuda.mem_get_info()[0])
    for _ in range(3):
        calls()
    torch.cuda.synchronize()
    assert (torch.cuda.memory_stats()["allocation.all.allocated"], torch.cuda.mem_get_info()[0]) == before


@pytest.mark.parametrize("T,d,f", [(40, 264, 136), (75, 136, 20008), (300, 264, 1032), (2000, 72, 40)])
@pytest.mark.parametrize("sms,flags", [(16, 0), (2, IGNORE_COSCHEDULING)])
def test_on_part_of_the_sms(sn, T, d, f, sms, flags):
    """No pairs of CTAs there, and no cut tiles: the same bars."""
    green = GreenContext(sms, flags)
    X, Wg, Wu, dH = inputs(T, d, f, 3)
    s = norm_inputs(T, d, 0, BF16, 4)
    torch.cuda.synchronize()
    on = green.stream.value
    H, G, U = sn.sn_glu_fwd(X, Wg, Wu, "silu", keep=True, stream=on)
    got = sn.sn_glu_bwd(dH, X, Wg, Wu, G, U, "silu", stream=on)
    Z, h = sn.sn_blocknorm_fwd(s["Y"], s["R"], s["w_post"], s["w_pre"], EPS, stream=on)
    back = sn.sn_blocknorm_bwd(s["dZ"], s["H"], s["Y"], s["w_post"], s["w_pre"], EPS, dH=s["dH"], stream=on)
    green.synchronize()
    torch.cuda.synchronize()
    check_fwd(X, Wg, Wu, "silu", H, G, U)
    check_bwd(dH, X, Wg, Wu, G, U, "silu", got)
    check_norm_fwd(s, 1.0, Z, h)
    check_norm_bwd(s, 1.0, back)
    green.destroy()


def test_offsets_past_32_bits(sn):
    """More than 2^31 elements in H, in its gradient and in a stream of rows: the last rows."""
    T, d, f = 300000, 16, 8192
    assert T * f > 2 ** 31
    X, Wg, Wu, _ = inputs(T, d, f, 5)
    H, G, U = sn.sn_glu_fwd(X, Wg, Wu, "silu", keep=True)
    check_fwd(X[-3:], Wg, Wu, "silu", H[-3:], G[-3:], U[-3:])
    check_fwd(X[:3], Wg, Wu, "silu", H[:3], G[:3], U[:3])
    last = [t[-2:].clone() for t in (H, X, G, U)]
    dX, _, _, dG, dU = sn.sn_glu_bwd(H, X, Wg, Wu, G, U, "silu", dG=G, dU=U, need_dW=False)
    check_bwd(last[0], last[1], Wg, Wu, last[2], last[3], "silu", (dX[-2:], None, None, dG[-2:], dU[-2:]))
    del H, G, U, dG, dU
    T, d = 270000, 8192
    g = gen(6)
    y = torch.randn(T, d, generator=g, device="cuda", dtype=BF16)
    w = torch.ones(d, device="cuda")
    gate = torch.randn(T // 27, d, generator=g, device="cuda", dtype=BF16)
    Z, h = sn.sn_blocknorm_fwd(y, y, w, w, EPS, 0.5, gate)
    got = sn.sn_blocknorm_bwd(y, h, y, w, w, EPS, 0.5, gate, dH=Z)
    r = slice(T - 27, T)
    s = {"Y": y[r], "R": y[r], "w_post": w, "w_pre": w, "gate": gate[-1:], "H": h[r], "dZ": y[r], "dH": Z[r]}
    check_norm_fwd(s, 0.5, Z[r], h[r])
    one = sn.sn_blocknorm_bwd(s["dZ"], s["H"], s["Y"], w, w, EPS, 0.5, s["gate"], dH=s["dH"])
    assert torch.equal(got[0][r], one[0]) and torch.equal(got[1][r], one[1])
    check_norm_bwd(s, 0.5, (got[0][r], got[1][r], one[2], one[3], got[4][-1:]))


def test_more_tiles_than_a_grid_and_row_strides(sn):
    """Tiles of several rounds with a cut last one, from rows that lie further apart."""
    T, d, f = 2500, 1544, 1032
    X, Wg, Wu, dH = inputs(T, d, f, 8)
    H, G, U = sn.sn_glu_fwd(spread(X, 8), Wg, Wu, "silu", keep=True)
    check_fwd(X, Wg, Wu, "silu", H, G, U)
    check_bwd(dH, X, Wg, Wu, G, U, "silu", sn.sn_glu_bwd(spread(dH, 40), spread(X, 24), Wg, Wu, G, U, "silu"))


@pytest.mark.parametrize("T,d,f,pad", [(9000, 264, 4104, 0), (8200, 1032, 1032, 0), (8200, 264, 4104, 40)])
def test_operands_laid_out_anew(sn, T, d, f, pad):
    """Rows of neither operand on 128 bytes, and enough of them: X and the weights are copied for the
    products; the results lie in the same bars, and nothing of the operands changes."""
    X, Wg, Wu, dH = inputs(T, d, f, 12)
    _, G, U = sn.sn_glu_fwd(X, Wg, Wu, "silu", keep=True)
    was = [t.clone() for t in (X, Wg, Wu)]
    got = sn.sn_glu_bwd(dH, spread(X, pad) if pad else X, Wg, Wu, G, U, "silu", grad_dtype=F32)
    check_bwd(dH, X, Wg, Wu, G, U, "silu", got)
    assert all(torch.equal(a, b) for a, b in zip(was, (X, Wg, Wu)))
    aligned = sn.sn_glu_bwd(dH, spread(X, -d % 64), Wg, Wu, G, U, "silu", grad_dtype=F32)
    assert all(torch.equal(a, b) for a, b in zip(got, aligned))
