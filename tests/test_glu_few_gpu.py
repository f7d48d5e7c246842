"""Gated projections of a few tokens in every form of their kernel: more and fewer than 64 rows of each
weight a CTA, one round and two, one accumulator and two of up to 224 columns, stages of one chunk and of
two, odd numbers of chunks; and the numbers of tokens from which on the tiles are taken.  Bars as in
test_glu_gpu.py."""
import pytest
import torch

from test_block_run_gpu import IGNORE_COSCHEDULING, GreenContext
from test_glu_gpu import ACTS, check_fwd, guarded, inputs, untouched

pytestmark = pytest.mark.gpu

# on about 150 SMs: more than 64 rows a CTA from f = 9728 on, a second round from 19456 on
WHOLE = [(1, 264, 14336), (75, 264, 14336), (33, 72, 9736), (128, 200, 9720), (96, 136, 14336), (129, 136, 10000),
         (160, 200, 14336), (161, 40, 12000), (200, 264, 14336), (224, 72, 14336), (224, 520, 19456), (225, 72, 14336),
         (128, 72, 28672), (40, 264, 28680), (129, 72, 28672), (17, 1032, 20000)]


def check(sn, T, d, f, keep, stream=None, synchronize=lambda: None):
    act = ACTS[(T + d + keep) % 4]
    X, Wg, Wu, _ = inputs(T, d, f, T + d + f)
    (fh, H), (fg, G), (fu, U) = (guarded(T, f) for _ in range(3))
    torch.cuda.synchronize()
    if keep:
        sn.sn_glu_fwd(X, Wg, Wu, act, out=H, G=G, U=U, stream=stream)
    else:
        sn.sn_glu_fwd(X, Wg, Wu, act, out=H, stream=stream)
    synchronize()
    sn.sn_check_errors()
    check_fwd(X, Wg, Wu, act, H, *((G, U) if keep else ()))
    assert untouched(fh) and untouched(fg) and untouched(fu)
    if not keep:
        assert bool((fg == 7.25).all()) and bool((fu == 7.25).all())


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("T,d,f", WHOLE)
def test_on_the_whole_gpu(sn, T, d, f, keep):
    check(sn, T, d, f, keep)


@pytest.mark.parametrize("T,d,f", [(130, 72, 136), (200, 136, 256), (224, 264, 136), (224, 8, 256), (225, 72, 256),
                                   (128, 200, 520), (1, 72, 1032)])
def test_on_two_sms(sn, T, d, f):
    green = GreenContext(2, IGNORE_COSCHEDULING)
    check(sn, T, d, f, True, green.stream.value, green.synchronize)
    green.destroy()
