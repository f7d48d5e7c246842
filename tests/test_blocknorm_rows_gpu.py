"""Gradients of the norms around a block: rows whose squares leave fp32's range under a gate, and infinities
and NaNs, which stay where the formulas put them.  Bars as in test_blocknorm_gpu.py."""
import pytest
import torch

from step_util import DT
from test_blocknorm_gpu import check_bwd, check_fwd, inputs

pytestmark = pytest.mark.gpu

BF16, F32, EPS = torch.bfloat16, torch.float32, 1e-5


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,gates", [(24, 100, 3), (24, 256, 24), (24, 4096, 1), (2002, 256, 7), (1500, 2056, 500)])
@pytest.mark.parametrize("y,h", [(1e-25, 1.0), (1.0, 1e-25), (1e25, 1.0), (1.0, 1e25), (1e25, 1e-25)])
def test_scaled_rows_under_a_gate(sn, dt, T, d, gates, y, h):
    """Every second row far from 1."""
    s = inputs(T, d, gates, DT[dt], 5)
    s["Y"][::2] *= y
    s["R"][::2] *= h
    s["H"][::2] *= h
    s["dH"][::2] *= 1 / h
    w = (s["w_post"], s["w_pre"], 0.0, 0.5, s["gate"])
    check_fwd(s, 0.5, *sn.sn_blocknorm_fwd(s["Y"], s["R"], *w), eps=0.0)
    check_bwd(s, 0.5, sn.sn_blocknorm_bwd(s["dZ"], s["H"], s["Y"], *w, dH=s["dH"]), eps=0.0)


def nan(x):
    return bool(torch.isnan(x).all())


@pytest.mark.parametrize("gates", [0, 1, 4, 20])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [100, 256, 2056, 4096, 8192, 16384])
def test_infinities_and_nans(sn, dt, d, gates):
    T, t, j = 20, 7, d // 2
    s = inputs(T, d, gates, DT[dt], 6)
    w = (s["w_post"], s["w_pre"], EPS, 0.5, s["gate"])

    def run(**other):
        v = dict(s, **other)
        return sn.sn_blocknorm_bwd(v["dZ"], v["H"], v["Y"], *w, dH=v["dH"])

    clean = run()
    rows, cols = [i for i in range(T) if i != t], [i for i in range(d) if i != j]
    mine = t * gates // T                                   # the gate of row t
    others = [i for i in range(gates) if i != mine]
    for name in ("Y", "H", "dZ", "dH"):
        for x in ("nan", "inf"):
            if x == "inf" and name in ("dZ", "dH"):         # (where infinities meet goes by the sums' order)
                continue
            bad = s[name].clone()
            bad[t, j] = float(x)
            dY, dR, dw_post, dw_pre, dgate = run(**{name: bad})
            assert torch.equal(dY[rows], clean[0][rows]) and torch.equal(dR[rows], clean[1][rows])
            assert nan(dY[t])
            if name == "Y":
                assert torch.equal(dR, clean[1]) and torch.equal(dw_pre, clean[3]) and nan(dw_post)
            elif name == "H":
                assert nan(dR[t]) and nan(dw_pre) and nan(dw_post)
            elif name == "dZ":
                assert nan(dR[t]) and nan(dw_post)
                assert nan(dw_pre[j]) and torch.equal(dw_pre[cols], clean[3][cols])
            else:
                assert nan(dR[t, j]) and torch.equal(dR[t, cols], clean[1][t, cols])
                assert torch.equal(dw_pre, clean[3])
                assert nan(dw_post[j]) and torch.equal(dw_post[cols], clean[2][cols])
            if gates:
                assert torch.equal(dgate[others], clean[4][others])
                if name == "dH":
                    assert nan(dgate[mine, j]) and torch.equal(dgate[mine, cols], clean[4][mine, cols])
                else:
                    assert nan(dgate[mine])
