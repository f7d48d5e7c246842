"""The global gradient norm and clipping against fp64.

Bars.  A thread's squares are summed in fp32 in chains of at most 64, everything else in fp64: the
norm is right to 32 * 2^-24, plus its own rounding.  A clipped value is the quotient (one rounding
to fp32), the norm's error and one product, then one rounding to its type."""
import math

import pytest
import torch

from gpu_util import guarded, guards_intact
from step_util import DT, UNIT, gen, within

pytestmark = pytest.mark.gpu
NORM = 33 * 2.0 ** -24


def tensors(g, sizes, std=1.0):
    """Of both types in turn, and views at every offset into one buffer."""
    out = []
    for i, n in enumerate(sizes):
        t = (std * torch.randn(n + 16, generator=g, device="cuda")).to(DT["bf16" if i % 2 else "f32"])
        out.append(t[i % 9:i % 9 + n])
    return out


def norm64(ts):
    return math.sqrt(sum(float(t.double().square().sum()) for t in ts))


# around a chunk (16384 elements), around a piece, empty ones, many small ones
SIZES = [[1], [16384, 16383, 16385, 32768], [0, 7, 0, 8, 9, 100001], [3] * 400 + [2000000], [5000000, 17]]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "%d tensors" % len(s))
@pytest.mark.parametrize("other", ["same types", "other types", "in place"])
def test_norm_and_clip(sn, sizes, other):
    g = gen(len(sizes))
    ts = tensors(g, sizes)
    ref = [t.double().clone() for t in ts]
    norm = norm64(ts)
    outs = None
    if other != "in place":
        flip = {torch.bfloat16: torch.float32, torch.float32: torch.bfloat16}
        outs = [torch.empty_like(t) if other == "same types" else torch.empty_like(t, dtype=flip[t.dtype]) for t in ts]
    L = sn.GradList(ts, out=outs)
    for most in (0.5 * norm, 2 * norm):
        if other == "in place":
            for t, r in zip(ts, ref):
                t.copy_(r.to(t.dtype))
        got = sn.sn_grads_clip(L, sn.sn_grads_sumsq(L), most)
        assert abs(float(got) - norm) <= NORM * norm
        c = most / max(norm, float(torch.tensor(most, dtype=torch.float32)))
        for t, r in zip(outs or ts, ref):
            if c < 1:
                within(t, r * c, (r * c).abs() * (NORM + 2.0 ** -22 + UNIT[t.dtype] * 1.01))
            else:
                assert torch.equal(t, r.to(t.dtype))         # untouched, or copied
    L.destroy()
    with pytest.raises(RuntimeError):
        sn.sn_grads_sumsq(L)


def test_nothing_outside_is_touched(sn):
    fulls, views = zip(*[guarded((n,), DT[dt]) for n in (1, 1000, 16385) for dt in DT])
    for v in views:
        v.fill_(3.0)
    L = sn.GradList(views)
    sn.sn_grads_clip(L, sn.sn_grads_sumsq(L), 1.0)
    assert all(guards_intact(f) for f in fulls) and all(bool((v < 3).all()) for v in views)


@pytest.mark.parametrize("size", [1e30, 1e-25, 1e-38, 3e37])
@pytest.mark.parametrize("n", [100003, 40])
def test_norms_past_the_range_of_squares(sn, size, n):
    g = gen(n)
    ts = [t for t in tensors(g, [n, n], std=1.0)]
    ts = [(t.double() * size).to(t.dtype) for t in ts] + [torch.zeros(50000, device="cuda")]
    L = sn.GradList(ts)
    norm = norm64(ts)
    sumsq = sn.sn_grads_sumsq(L)
    assert abs(math.sqrt(float(sumsq)) - norm) <= NORM * norm
    if norm < 3e38:
        assert abs(float(sn.sn_grads_clip(L, sumsq, 1.0)) - norm) <= NORM * norm + 2.0 ** -149


def test_sums_of_several_lists(sn):
    """Stages that hold parts of a model add their sums."""
    g = gen(4)
    ts = tensors(g, [1000, 70000, 12345])
    parts = [sn.GradList([t]) for t in ts]
    total = sn.sn_grads_sumsq(parts[0])
    for p in parts[1:]:
        sn.sn_grads_sumsq(p, out=total, accumulate=True)
    norm = norm64(ts)
    for p in parts:
        assert abs(float(sn.sn_grads_clip(p, total, 1.0)) - norm) <= NORM * norm
    assert abs(norm64(ts) - 1.0) <= 2.0 ** -9
    empty = sn.GradList([])
    assert float(sn.sn_grads_sumsq(empty)) == 0 and float(sn.sn_grads_clip(empty, total, 1.0)) > 0


def test_infinities_and_nan(sn):
    for bad, norm_is in ((math.inf, math.isinf), (-math.inf, math.isinf), (math.nan, math.isnan)):
        ts = [torch.ones(100, device="cuda"), torch.ones(40000, device="cuda", dtype=torch.bfloat16)]
        ts[1][33333] = bad
        L = sn.GradList(ts)
        norm = sn.sn_grads_clip(L, sn.sn_grads_sumsq(L), 1.0)
        assert norm_is(float(norm))
        if math.isnan(bad):
            assert all(bool(t.isnan().all()) for t in ts)
        else:
            assert bool((ts[0] == 0).all()) and int(ts[1].isnan().sum()) == 1


def test_the_same_bits_every_time_and_on_another_stream(sn):
    ts = tensors(gen(6), [3000000, 12345, 999999])
    L = sn.GradList(ts, out=[torch.empty_like(t) for t in ts])
    first = sn.sn_grads_sumsq(L)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = [sn.sn_grads_sumsq(L) for _ in range(5)]
        sn.sn_grads_clip(L, again[0], 1.0)
    side.synchronize()
    assert all(float(a) == float(first) for a in again)
    assert abs(norm64(L.out) - 1.0) <= 2.0 ** -9


def test_refusals(sn):
    a, b = torch.zeros(100, device="cuda"), torch.zeros(100, device="cuda")
    with pytest.raises(TypeError):
        sn.GradList([a.half()])
    for call in (lambda: sn.GradList([a], out=[]), lambda: sn.GradList([a], out=[b[:50]]),
                 lambda: sn.GradList([a[::2]]), lambda: sn.GradList([a.cpu()])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: sn.GradList([a, a]), lambda: sn.GradList([a[:60], a[40:]]),
                 lambda: sn.GradList([a[:50]], out=[a[10:60]]), lambda: sn.GradList([a, b], out=[b, a]),
                 lambda: sn.GradList([a[:10]], out=[a.view(torch.bfloat16)[:10]])):
        with pytest.raises(sn.SNError) as e:
            call()
        assert e.value.status == sn.SN_ERR_INVALID_ARG
    sn.GradList([a, a], out=[b, torch.zeros(100, device="cuda")]).destroy()    # a source may come twice
    L = sn.GradList([a])
    sumsq = sn.sn_grads_sumsq(L)
    for most in (0.0, -1.0, math.inf, math.nan):
        with pytest.raises(sn.SNError) as e:
            sn.sn_grads_clip(L, sumsq, most)
        assert e.value.status == sn.SN_ERR_INVALID_ARG
    with pytest.raises(TypeError):
        sn.sn_grads_clip(L, sumsq.float(), 1.0)
