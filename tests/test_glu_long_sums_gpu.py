"""The weights' gradients of so many tokens that one CTA's products of a tile outlast the limit of a wait
(2 s): on a part of the SMs a tile's inner dimension, the tokens, is not divided, and its epilogue waits
for all of it.  The wait is bounded by what stands still, not by what takes long."""
import pytest
import torch

from test_block_run_gpu import IGNORE_COSCHEDULING, GreenContext

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
T, D, F = 640_000_001, 8, 8         # 10 million chunks of 64 tokens, 3.3 s on a GB300


def test_a_tile_that_takes_longer_than_a_wait_may(sn):
    def zeros():
        return torch.zeros(T, D, device="cuda", dtype=BF16)

    # whole numbers in a few rows, the first and the last among them: every sum is exact
    rows = torch.tensor([0, 1, 63, 64, 4097, T // 2, T - 70, T - 1], device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    X, dH, G, U = (zeros() for _ in range(4))
    for t in (X, dH, G, U):
        t[rows] = torch.randint(-3, 4, (len(rows), D), generator=g, device="cuda").to(BF16)
    x, h, gate, up = (t[rows].double() for t in (X, dH, G, U))
    want = ((h * up * (gate > 0)).T @ x, (h * gate.clamp(min=0)).T @ x)
    W = torch.zeros(F, D, device="cuda", dtype=BF16)
    dWg, dWu = (torch.full((F, D), float("nan"), device="cuda") for _ in range(2))
    green = GreenContext(2, IGNORE_COSCHEDULING)
    torch.cuda.synchronize()
    sn.sn_glu_bwd(dH, X, W, W, G, U, "relu", dG=G, dU=U, dW_gate=dWg, dW_up=dWu, need_dX=False,
                  stream=green.stream.value)
    green.synchronize()
    sn.sn_check_errors()
    assert torch.equal(dWg.double(), want[0]) and torch.equal(dWu.double(), want[1])
    green.destroy()
