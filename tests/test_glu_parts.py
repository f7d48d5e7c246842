"""Gradients of the gated projections with operands left out that no asked product reads, as the C entry
point has them."""
import pytest
import torch

from test_stream_memory import BF16, F32, device, stand_in  # noqa: F401


@pytest.fixture
def binding(stand_in):  # noqa: F811
    sn = stand_in[0]
    sn.sn_glu_bwd_workspace.cache_clear()
    yield sn
    sn.sn_glu_bwd_workspace.cache_clear()


def test_operands_that_no_product_reads(binding, monkeypatch):
    sn = binding
    given = []
    monkeypatch.setattr(sn._lib, "sn_glu_bwd", lambda *a: given.append(a) or 0, raising=False)
    X, H, W = device(4, 64), device(4, 32), device(32, 64)
    dX, dWg, dWu, dG, dU = sn.sn_glu_bwd(H, X, None, None, H, H, need_dX=False)
    assert dX is None and dWg.shape == dWu.shape == (32, 64) and dWg.dtype == BF16 and dG.shape == dU.shape == (4, 32)
    assert given[-1][6] is None and given[-1][7] is None and given[-1][11] == 64
    assert sn.sn_glu_bwd(H, None, W, W, H, H, need_dW=False)[0].shape == (4, 64)
    assert given[-1][4] is None and given[-1][11] == 64
    assert sn.sn_glu_bwd(H, X, None, None, H, H, need_dX=False, grad_dtype=F32)[1].dtype == F32
    assert sn.sn_glu_bwd(H, None, None, None, H, H, need_dX=False, need_dW=False)[:3] == (None, None, None)


def test_operands_that_a_product_reads_are_asked_for(binding):
    sn = binding
    X, H, W = device(4, 64), device(4, 32), device(32, 64)
    for call in (lambda: sn.sn_glu_bwd(H, None, W, W, H, H), lambda: sn.sn_glu_bwd(H, X, None, W, H, H),
                 lambda: sn.sn_glu_bwd(H, X, W, None, H, H), lambda: sn.sn_glu_bwd(H, None, W, W, H, H, need_dX=False),
                 lambda: sn.sn_glu_bwd(H, X, W, None, H, H, need_dW=False),
                 lambda: sn.sn_glu_bwd(H, X, device(32, 56), None, H, H, need_dX=False),
                 lambda: sn.sn_glu_bwd(H, device(4, 56), W, W, H, H, need_dW=False)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,f", [(40, 264, 136), (9000, 264, 4104)])
def test_same_bits_as_with_every_operand(sn, T, d, f):
    from test_glu_gpu import inputs
    X, Wg, Wu, dH = inputs(T, d, f, 3)
    _, G, U = sn.sn_glu_fwd(X, Wg, Wu, "silu", keep=True)
    whole = sn.sn_glu_bwd(dH, X, Wg, Wu, G, U)
    for got in (sn.sn_glu_bwd(dH, X, None, None, G, U, need_dX=False),
                sn.sn_glu_bwd(dH, None, Wg, Wu, G, U, need_dW=False),
                sn.sn_glu_bwd(dH, None, None, None, G, U, need_dX=False, need_dW=False)):
        assert all(a is None or torch.equal(a, b) for a, b in zip(got, whole))
        assert got[3] is not None and got[4] is not None


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,f", [(40, 264, 136), (2000, 520, 2088), (1000, 8, 16), (3000, 1024, 520)])
def test_without_products_any_workspace_will_do(sn, T, d, f):
    """One of the size for this width, a small one, and none: dG and dU alone have no use for it."""
    from test_glu_gpu import inputs
    X, Wg, Wu, dH = inputs(T, d, f, 3)
    _, G, U = sn.sn_glu_fwd(X, Wg, Wu, "silu", keep=True)
    whole = sn.sn_glu_bwd(dH, X, Wg, Wu, G, U)
    for operands in ((X, Wg, Wu), (None, None, None)):
        for n in (sn.sn_glu_bwd_workspace(T, d, f), 16, None):
            ws = None if n is None else torch.empty(max(16, n), dtype=torch.uint8, device="cuda")
            got = sn.sn_glu_bwd(dH, *operands, G, U, need_dX=False, need_dW=False, workspace=ws)
            assert torch.equal(got[3], whole[3]) and torch.equal(got[4], whole[4])
