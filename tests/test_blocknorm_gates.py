"""Gradients of the norms around a block with a gate for every few tokens: the gates whose tokens several
workers have, and the workspace that their parts lie in."""
import ctypes

import pytest
import torch

from step_util import gen

BF16, F32, EPS = torch.bfloat16, torch.float32, 1e-5


@pytest.mark.parametrize("T,d", [(65536, 8192), (16384, 4096), (4096, 1001), (65536, 40)])
def test_workspace_does_not_grow_with_the_gates(T, d):
    """A worker shares two gates at most: their parts take no more than the weights' two, and none where
    every token has a gate of its own."""
    from paper_2506_01260_gb300 import sn

    def size(gates):
        n = ctypes.c_size_t()
        assert sn._lib.sn_blocknorm_bwd_workspace(T, d, gates, ctypes.byref(n)) == 0
        return n.value

    alone = size(0)
    assert size(1) == size(T) == alone
    for gates in (2, 16, T // 16, T // 4, T // 2):
        assert alone <= size(gates) <= 2 * alone


# T, d, gates: runs of tokens that workers' bounds cut, with fewer gates than workers and with more; rows
# of a warp, of a block, and of single elements
CASES = [(9000, 264, 3000), (9000, 264, 90), (5000, 48, 1000), (2600, 1024, 1300), (2600, 2056, 520),
         (1500, 4096, 500), (1500, 1001, 500), (1400, 1001, 100), (900, 8200, 300), (1208, 2056, 302), (7, 520, 7)]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,gates", CASES)
def test_shared_gates(sn, dt, T, d, gates):
    from step_util import DT
    from test_blocknorm_gpu import check_bwd, inputs
    s = inputs(T, d, gates, DT[dt], T + d)
    g = gen(4)
    was = [torch.randn(*shape, generator=g, device="cuda") for shape in ((d,), (d,), (gates, d))]
    out = [w.clone() for w in was]
    n = sn.sn_blocknorm_bwd_workspace(T, d, gates)
    ws = torch.full((n + 1024,), 0xFF, dtype=torch.uint8, device="cuda")        # NaN wherever it is read unwritten
    call = (s["dZ"], s["H"], s["Y"], s["w_post"], s["w_pre"], EPS, 0.5, s["gate"])
    got = sn.sn_blocknorm_bwd(*call, dH=s["dH"], workspace=ws[:n])
    check_bwd(s, 0.5, got)
    assert bool((ws[n:] == 0xFF).all())
    added = sn.sn_blocknorm_bwd(*call, dH=s["dH"], dw_pre=out[0], dw_post=out[1], dgate=out[2], accumulate=True)
    check_bwd(s, 0.5, added, add=was)
    assert torch.equal(added[0], got[0]) and torch.equal(added[1], got[1])
