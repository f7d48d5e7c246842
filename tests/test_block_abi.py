"""Entry points of the gated projections and of the norms around a block, on the CPU: argument errors
that return before any CUDA call, and the stream that a call's memory belongs to."""
import ctypes
import types

import pytest
import torch

from test_stream_memory import BF16, CURRENT, F32, GIVEN, device, stand_in  # noqa: F401

P = ctypes.c_void_p
INVALID, ALIGNMENT, UNSUPPORTED = 1, 2, 3


@pytest.fixture(scope="module")
def lib():
    from paper_2506_01260_gb300 import sn
    return sn._lib


def glu_fwd(lib, basis=None, dt=0, X=256, ldx=64, Wg=512, Wu=768, T=4, d=64, f=32, act=0, G=None, U=None, H=1024):
    return lib.sn_glu_fwd(basis, dt, X, ldx, Wg, Wu, T, d, f, act, G, U, H, None)


def glu_bwd(lib, dt=0, dH=4096, lddh=32, X=8192, ldx=64, Wg=16384, Wu=32768, G=65536, U=69632, T=4, d=64, f=32,
            act=0, dG=73728, dU=77824, dX=81920, gdt=0, dWg=98304, dWu=114688, add=0, ws=131072, nbytes=1 << 30):
    return lib.sn_glu_bwd(None, dt, dH, lddh, X, ldx, Wg, Wu, G, U, T, d, f, act, dG, dU, dX, gdt, dWg, dWu, add, ws,
                          nbytes, None)


def norm_fwd(lib, dt=0, Y=4096, ldy=64, R=8192, gate=None, gates=0, wdt=1, w1=12288, w2=16384, T=4, d=64, eps=1e-5,
             scale=1.0, H=20480, Z=24576):
    return lib.sn_blocknorm_fwd(dt, Y, ldy, R, gate, gates, wdt, w1, w2, T, d, eps, scale, H, Z, None)


def norm_bwd(lib, dt=0, dZ=4096, lddz=64, H=8192, Y=12288, ldy=64, dH=None, gate=None, gates=0, wdt=1, w1=16384,
             w2=20480, T=4, d=64, eps=1e-5, scale=1.0, dY=24576, dR=28672, a=32768, b=36864, c=None, add=0, ws=40960,
             nbytes=1 << 30):
    return lib.sn_blocknorm_bwd(dt, dZ, lddz, H, Y, ldy, dH, gate, gates, wdt, w1, w2, T, d, eps, scale, dY, dR, a, b,
                                c, add, ws, nbytes, None)


@pytest.mark.parametrize("call,status", [
    (dict(dt=7), INVALID), (dict(dt=1), UNSUPPORTED), (dict(T=-1), INVALID), (dict(d=0), INVALID),
    (dict(f=-8), INVALID), (dict(d=1 << 21, ldx=1 << 21), INVALID), (dict(ldx=56), INVALID), (dict(act=4), INVALID),
    (dict(act=-1), INVALID), (dict(d=60), ALIGNMENT), (dict(f=36), ALIGNMENT), (dict(ldx=68), ALIGNMENT),
    (dict(X=None), INVALID), (dict(Wg=None), INVALID), (dict(H=None), INVALID), (dict(G=2048), INVALID),
    (dict(X=264), ALIGNMENT), (dict(H=1032), ALIGNMENT), (dict(T=1 << 31), INVALID), (dict(ldx=1 << 31), INVALID),
    (dict(H=256), INVALID), (dict(T=0, X=None, H=None), 0)])
def test_glu_fwd(lib, call, status):
    assert glu_fwd(lib, **call) == status


@pytest.mark.parametrize("call,status", [
    (dict(dt=1), UNSUPPORTED), (dict(gdt=5), INVALID), (dict(lddh=24), INVALID), (dict(lddh=36), ALIGNMENT),
    (dict(ldx=48), INVALID), (dict(dWu=None), INVALID), (dict(act=9), INVALID), (dict(d=20, ldx=20), ALIGNMENT),
    (dict(dH=None), INVALID), (dict(X=None), INVALID), (dict(dG=None), INVALID), (dict(dX=81928), ALIGNMENT),
    (dict(dG=69632), INVALID), (dict(dX=8192), INVALID), (dict(dWg=16384), INVALID), (dict(dG=65536 + 16), INVALID),
    (dict(T=0, dX=None, dWg=None, dWu=None), 0), (dict(T=0, add=1), 0)])
def test_glu_bwd(lib, call, status):
    if call.get("T") == 0:
        call = dict(call, dH=None, G=None, U=None, dG=None, dU=None, X=None, Wg=None, Wu=None, dX=None, ws=None)
        if call.get("add"):
            call.update(dWg=None, dWu=None)
    assert glu_bwd(lib, **call) == status


@pytest.mark.parametrize("call,status", [
    (dict(dt=3), INVALID), (dict(wdt=3), INVALID), (dict(d=0), INVALID), (dict(ldy=63), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=float("inf")), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(gates=1), INVALID), (dict(gate=28672), INVALID), (dict(gate=28672, gates=3), INVALID),
    (dict(gate=28672, gates=8), INVALID), (dict(R=None), INVALID), (dict(Z=None), INVALID), (dict(H=20488), ALIGNMENT),
    (dict(H=24576), INVALID), (dict(H=8208), INVALID), (dict(Z=12288), INVALID), (dict(T=0, Y=None), 0)])
def test_blocknorm_fwd(lib, call, status):
    assert norm_fwd(lib, **call) == status


@pytest.mark.parametrize("call,status", [
    (dict(lddz=32), INVALID), (dict(ldy=32), INVALID), (dict(eps=-0.1), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(c=45056), INVALID), (dict(gate=45056, gates=2), INVALID), (dict(a=None), INVALID), (dict(dZ=None), INVALID),
    (dict(dY=28672), INVALID), (dict(a=36864), INVALID), (dict(dR=4112), INVALID), (dict(T=1 << 32), INVALID)])
def test_blocknorm_bwd(lib, call, status):
    # (with tokens, the size of the workspace asks for the device's SMs, which a CPU answers with one)
    assert norm_bwd(lib, **call) == status


def test_workspaces(lib):
    n = ctypes.c_size_t()
    for T, d, f, status in ((10, 60, 32, ALIGNMENT), (-1, 64, 32, INVALID), (10, 64, 0, INVALID), (10, 64, 32, 0)):
        assert lib.sn_glu_bwd_workspace(T, d, f, ctypes.byref(n)) == status
    assert lib.sn_glu_bwd_workspace(10, 64, 32, None) == INVALID
    for T, d, gates, status in ((10, 64, 3, INVALID), (10, 64, -1, INVALID), (10, 0, 0, INVALID), (10, 64, 5, 0)):
        assert lib.sn_blocknorm_bwd_workspace(T, d, gates, ctypes.byref(n)) == status


@pytest.fixture
def no_sizes():
    """Sizes that the stand-in library gives are not kept."""
    from paper_2506_01260_gb300 import sn
    kept = (sn.sn_glu_bwd_workspace, sn.sn_blocknorm_bwd_workspace)
    for f in kept:
        f.cache_clear()
    yield
    for f in kept:
        f.cache_clear()


@pytest.mark.parametrize("name", ["glu_fwd", "glu_fwd_keep", "glu_bwd", "blocknorm_fwd", "blocknorm_bwd"])
def test_memory_is_the_given_streams(stand_in, no_sizes, name):  # noqa: F811
    sn, streams, made = stand_in
    X, H, W = device(4, 64), device(4, 32), device(32, 64)
    w, gate = device(64, dtype=F32), device(2, 64)
    call = {
        "glu_fwd": lambda s: sn.sn_glu_fwd(X, W, W, stream=s),
        "glu_fwd_keep": lambda s: sn.sn_glu_fwd(X, W, W, keep=True, stream=s),
        "glu_bwd": lambda s: sn.sn_glu_bwd(H, X, W, W, H, H, stream=s),
        "blocknorm_fwd": lambda s: sn.sn_blocknorm_fwd(X, X, w, w, 1e-5, gate=gate, stream=s),
        "blocknorm_bwd": lambda s: sn.sn_blocknorm_bwd(X, X, X, w, w, 1e-5, gate=gate, dH=X, stream=s),
    }[name]
    many = {"glu_fwd": 1, "glu_fwd_keep": 3, "glu_bwd": 5, "blocknorm_fwd": 2, "blocknorm_bwd": 6}[name]
    for given in (GIVEN, types.SimpleNamespace(cuda_stream=GIVEN)):
        del streams[:], made[:]
        call(given)
        assert set(streams) == {GIVEN} and len(made) == many and all(m == (GIVEN, [CURRENT]) for m in made)
    for given in (None, CURRENT):
        del streams[:], made[:]
        call(given)
        assert set(streams) == {CURRENT} and len(made) == many and all(m == (CURRENT, []) for m in made)


def test_shapes_are_refused(stand_in, no_sizes):  # noqa: F811
    sn = stand_in[0]
    X, H, W, w = device(4, 64), device(4, 32), device(32, 64), device(64, dtype=F32)
    for call, error in (
            (lambda: sn.sn_glu_fwd(X, W, device(32, 56)), ValueError),
            (lambda: sn.sn_glu_fwd(X, device(32, 56), W), ValueError),
            (lambda: sn.sn_glu_fwd(X, W, W, out=device(4, 31)), ValueError),
            (lambda: sn.sn_glu_fwd(X, W, W, G=device(4, 32, dtype=F32)), TypeError),
            (lambda: sn.sn_glu_fwd(X.t(), W, W), ValueError),
            (lambda: sn.sn_glu_bwd(H, device(3, 64), W, W, H, H), ValueError),
            (lambda: sn.sn_glu_bwd(H, X, W, W, H, X), ValueError),
            (lambda: sn.sn_glu_bwd(H, X, W, W, H, H, accumulate=True), ValueError),
            (lambda: sn.sn_glu_bwd(H, X, W, W, H, H, grad_dtype=torch.float64), TypeError),
            (lambda: sn.sn_glu_bwd(H, X, W, W, H, H, dW_gate=device(32, 64), grad_dtype=F32), TypeError),
            (lambda: sn.sn_blocknorm_fwd(X, device(4, 63), w, w, 1e-5), ValueError),
            (lambda: sn.sn_blocknorm_fwd(X, X, w, device(63, dtype=F32), 1e-5), ValueError),
            (lambda: sn.sn_blocknorm_fwd(X, X, w, w, 1e-5, gate=device(3, 64)), ValueError),
            (lambda: sn.sn_blocknorm_fwd(X, X, w, w, 1e-5, gate=device(0, 64)), ValueError),
            (lambda: sn.sn_blocknorm_fwd(X, X, w, w, 1e-5, gate=device(64)), ValueError),
            (lambda: sn.sn_blocknorm_bwd(X, X, device(3, 64), w, w, 1e-5), ValueError),
            (lambda: sn.sn_blocknorm_bwd(X, X, X, w, w, 1e-5, gate=device(2, 64), dgate=device(3, 64, dtype=F32)),
             ValueError)):
        with pytest.raises(error):
            call()
