"""Expired waits of calls that were given no basis: the next sn_check_errors on the device reports them
once, with a basis or without."""
import types

import pytest
import torch

LIMIT_S = 2.0       # the library's wait limit


def test_the_binding_checks_without_a_basis(monkeypatch):
    from paper_2506_01260_gb300 import sn
    got = []
    monkeypatch.setattr(sn, "_lib", types.SimpleNamespace(sn_check_errors=lambda *a: got.append(a) or 0))
    monkeypatch.setattr(sn, "_stream", lambda s: s or 5)
    sn.sn_check_errors()
    sn.sn_check_errors(None, 7)
    sn.sn_check_errors(types.SimpleNamespace(handle=3))
    assert got == [(None, 5), (None, 7), (3, 5)]


def test_a_check_without_a_basis_is_no_argument_error():
    from paper_2506_01260_gb300 import sn
    assert sn._lib.sn_check_errors(None, None) != sn.SN_ERR_INVALID_ARG     # (on a CPU, SN_ERR_CUDA)


@pytest.mark.gpu
@pytest.mark.parametrize("claimed", [False, True])
def test_an_expired_wait_without_a_basis_is_reported_once(sn, claimed):
    from test_glu_gpu import check_fwd, inputs
    U = torch.linalg.qr(torch.randn(64, 8, generator=torch.Generator().manual_seed(1)))[0]
    basis = sn.Basis(U.contiguous().cuda()) if claimed else None
    sn.sn_check_errors(basis)
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    torch.cuda.synchronize()
    a.record()
    sn.sn_selftest_unclaimed_timeout()
    b.record()
    with pytest.raises(sn.SNError) as e:
        sn.sn_check_errors(basis)
    assert e.value.status == sn.SN_ERR_TIMEOUT
    elapsed = a.elapsed_time(b) / 1e3
    assert LIMIT_S * 0.95 <= elapsed <= LIMIT_S * 1.5, elapsed
    sn.sn_check_errors(basis)
    sn.sn_check_errors()
    for T in (20, 600):                               # the calls run as before
        X, Wg, Wu, _ = inputs(T, 72, 136, 2)
        H, _, _ = sn.sn_glu_fwd(X, Wg, Wu, "silu", basis=basis)
        sn.sn_check_errors(basis)
        check_fwd(X, Wg, Wu, "silu", H)
    if claimed:
        basis.destroy()


@pytest.mark.gpu
def test_what_a_basis_records_stays_its_own(sn):
    """A bad id that a basis recorded is not reported to a check of another, or of none."""
    g = torch.Generator().manual_seed(2)
    one, two = (sn.Basis(torch.linalg.qr(torch.randn(64, 8, generator=g))[0].contiguous().cuda()) for _ in range(2))
    table = torch.ones(5, 64, device="cuda")
    sn.sn_embed_fwd(table, torch.tensor([1, 9], dtype=torch.int32, device="cuda"), basis=one)
    sn.sn_check_errors()
    sn.sn_check_errors(two)
    with pytest.raises(sn.SNError) as e:
        sn.sn_check_errors(one)
    assert e.value.status == sn.SN_ERR_BAD_ID
    sn.sn_check_errors(one)
    one.destroy()
    two.destroy()
