"""The step operators on a stream whose context has only a part of the GPU's SMs: a decode step's
scores take clusters on the whole GPU and none here; the other calls size their grids by the
whole GPU and must still end.  The same bits as on the whole GPU but for the scores' sums, whose
order differs with the clusters: 2^-15 (the bar of the log probabilities' tests)."""
import pytest
import torch

from test_green_context_gpu import GreenContext, IGNORE_COSCHEDULING

pytestmark = pytest.mark.gpu


@pytest.fixture(params=[(16, 0), (2, IGNORE_COSCHEDULING)], ids=["16 SMs", "any 2 SMs"])
def green(sn, request):
    g = GreenContext(*request.param)
    yield g
    g.destroy()


def test_on_part_of_the_sms(sn, green):
    T, d, V = 3000, 256, 40000
    g = torch.Generator(device="cuda").manual_seed(1)
    x, r = (torch.randn(T, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    w = torch.ones(d, device="cuda")
    ids = torch.randint(700, (T,), generator=g, device="cuda", dtype=torch.int32)
    logits = torch.randn(3, V, generator=g, device="cuda")
    L = sn.GradList([torch.randn(3000000, generator=g, device="cuda")])
    L2 = sn.GradList(L.grads, out=[torch.empty_like(t) for t in L.grads])

    def calls(stream):
        Y, H = sn.sn_rmsnorm_fwd(x, w, 1e-5, R=r, stream=stream)
        dX, dw = sn.sn_rmsnorm_bwd(x, H, w, 1e-5, dH=r, stream=stream)
        dE = sn.sn_embed_bwd(dX, ids, 700, stream=stream)
        E = sn.sn_embed_fwd(dE, ids, stream=stream)
        scores = sn.sn_logprob_fwd(logits, ids[:3], top=9, stream=stream)
        norm = sn.sn_grads_clip(L2, sn.sn_grads_sumsq(L2, stream=stream), 1.0, stream=stream)
        return [Y, H, dX, dw, dE, E, norm, L2.out[0].clone()], scores

    side = torch.cuda.current_stream().cuda_stream
    want, scores = calls(side)
    torch.cuda.synchronize()
    got, parts = calls(green.stream.value)
    green.synchronize()
    torch.cuda.synchronize()
    # the gradient of w is summed over the rows of the blocks that there are: the same grid
    for i, (a, b) in enumerate(zip(got[:-1], want[:-1])):
        assert torch.equal(a, b), i
    assert torch.equal(parts[3], scores[3])
    for a, b in zip((parts[0], parts[2], parts[4]), (scores[0], scores[2], scores[4])):
        assert float((a - b).abs().max()) <= 2.0 ** -15
