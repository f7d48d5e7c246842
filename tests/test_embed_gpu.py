"""Embedding lookup and its gradient against plain fp64 sums.

Bars: a lookup is one fp32 product and one rounding to the output's type, 2^-24 + its unit
relative.  A gradient row is a sum of n fp32 terms, at most n roundings of 2^-24 of the sum of
magnitudes, the scale's product and one rounding to the output's type."""
import pytest
import torch

from gpu_util import guarded, guards_intact
from step_util import DT, UNIT, gen, spread, within

pytestmark = pytest.mark.gpu


def ids_of(T, V, how, g):
    if how == "one":
        return torch.full((T,), V // 2, dtype=torch.int32, device="cuda")
    if how == "distinct":
        return torch.randperm(V, generator=g, device="cuda")[:T].int()
    if how == "skewed":                       # half the tokens share three ids
        ids = torch.randint(V, (T,), generator=g, device="cuda")
        few = torch.randint(3, (T,), generator=g, device="cuda") * (V // 4)
        return torch.where(torch.rand(T, generator=g, device="cuda") < 0.5, few, ids).int()
    return torch.randint(V, (T,), generator=g, device="cuda", dtype=torch.int32)


@pytest.mark.parametrize("tdt", DT)
@pytest.mark.parametrize("xdt", DT)
@pytest.mark.parametrize("T,d,V", [(1, 8, 3), (5, 7, 11), (333, 200, 97), (64, 4104, 50), (3, 16392, 9),
                                   (1000, 1, 5), (17, 2048, 1)])
def test_lookup(sn, tdt, xdt, T, d, V):
    g = gen(T + d)
    table = torch.randn(V, d, generator=g, device="cuda").to(DT[tdt])
    ids = ids_of(T, V, "uniform", g)
    scale = 1.7320508
    full, out = guarded((T, d), DT[xdt])
    sn.sn_embed_fwd(table, ids, scale=scale, out=out)
    ref = table.double()[ids.long()] * float(torch.tensor(scale, dtype=torch.float32))
    within(out, ref, ref.abs() * (2.0 ** -24 + UNIT[DT[xdt]] * 1.01))
    assert guards_intact(full)


def test_lookup_of_invalid_ids(sn):
    basis = sn.Basis(torch.eye(16, 2, device="cuda").contiguous())
    table = torch.ones(4, 24, device="cuda")
    ids = torch.tensor([0, -1, 4, 3, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    X = sn.sn_embed_fwd(table, ids, basis=basis)
    with pytest.raises(sn.SNError) as e:
        sn.sn_check_errors(basis)
    assert e.value.status == sn.SN_ERR_BAD_ID
    assert X.sum(1).tolist() == [24, 0, 0, 24, 0, 0]
    assert torch.equal(X, sn.sn_embed_fwd(table, ids))      # without a basis: the same, unreported
    sn.sn_check_errors(basis)
    dE = sn.sn_embed_bwd(torch.ones(6, 24, device="cuda"), ids, 4, basis=basis)
    with pytest.raises(sn.SNError):
        sn.sn_check_errors(basis)
    assert dE.sum(1).tolist() == [24, 0, 0, 24]
    basis.destroy()


def grad_ref(G, ids, V, scale):
    """(sum, sum of magnitudes, terms) of every row, fp64."""
    good = (ids >= 0) & (ids < V)
    i, g = ids[good].long(), G[good].double() * scale
    zero = torch.zeros(V, G.shape[1], dtype=torch.float64, device="cuda")
    n = torch.bincount(i, minlength=V).double()[:, None]
    return zero.index_add(0, i, g), zero.index_add(0, i, g.abs()), n


# windows of 8 to 128 places, ids within one and across many, ranges of one and several blocks,
# widths with and without whole 16-byte pieces
@pytest.mark.parametrize("gdt", DT)
@pytest.mark.parametrize("edt", DT)
@pytest.mark.parametrize("T,d,V,how", [
    (1, 8, 1, "uniform"), (1, 4096, 300, "uniform"), (7, 9, 40, "uniform"), (8, 16, 8, "distinct"),
    (65, 200, 31, "skewed"), (1000, 72, 5000, "skewed"), (4097, 264, 1000, "uniform"),
    (3001, 2056, 33, "skewed"), (5000, 136, 4000, "one"), (20000, 8, 700, "one"),
    (300, 8, 1500000, "uniform"), (40000, 4096, 777, "skewed"), (129, 1, 64, "skewed"),
    (2000, 33, 100, "one")])
def test_gradient(sn, gdt, edt, T, d, V, how):
    g = gen(T * 7 + d)
    G = torch.randn(T, d, generator=g, device="cuda").to(DT[gdt])
    ids = ids_of(T, V, how, g)
    scale = 0.75
    full, out = guarded((V, d), DT[edt])
    sn.sn_embed_bwd(G, ids, V, scale=scale, out=out)
    ref, mag, n = grad_ref(G, ids, V, scale)
    within(out, ref, mag * (n + 1) * 2.0 ** -24 + ref.abs() * UNIT[DT[edt]] * 1.01)
    assert guards_intact(full)
    again = sn.sn_embed_bwd(G, ids, V, scale=scale, out_dtype=DT[edt])
    assert torch.equal(again, out)            # the same bits


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("T,d,V,pad", [(700, 136, 50, 0), (700, 136, 50, 8), (700, 136, 50, 3),
                                       (513, 45, 400, 5), (0, 64, 20, 0)])
def test_accumulation_and_strides(sn, dt, T, d, V, pad):
    g = gen(d + pad)
    G = spread(torch.randn(T, d, generator=g, device="cuda").to(DT[dt]), pad)
    ids = ids_of(T, V, "skewed", g)
    ids[::7] = -1                             # tokens without a row
    start = torch.randn(V, d, generator=g, device="cuda").to(DT[dt])
    full, out = guarded((V, d), DT[dt])
    out.copy_(start)
    sn.sn_embed_bwd(G, ids, V, scale=2.0, out=out, accumulate=True)
    ref, mag, n = grad_ref(G, ids, V, 2.0)
    bound = (mag + start.double().abs()) * (n + 2) * 2.0 ** -24
    within(out, start.double() + ref, bound + (start.double() + ref).abs() * UNIT[DT[dt]] * 1.01)
    none = (n == 0)[:, 0]
    assert torch.equal(out[none], start[none]) and guards_intact(full)
    out.fill_(float("nan"))                   # not accumulating, every row is written
    sn.sn_embed_bwd(G, ids, V, scale=2.0, out=out)
    within(out, ref, mag * (n + 1) * 2.0 ** -24 + ref.abs() * UNIT[DT[dt]] * 1.01)


def test_gradient_against_differences(sn):
    """The lookup is linear in the table: <G, X(E + D) - X(E)> = <dE, D>.  The sums' bars: one fp32
    rounding of each of the T d products' factors, 2^-22 of the sum of magnitudes."""
    g = gen(5)
    T, d, V, scale = 300, 96, 40, 0.5
    ids = ids_of(T, V, "skewed", g)
    E, D, G = (torch.randn(*s, generator=g, device="cuda") for s in ((V, d), (V, d), (T, d)))
    diff = (sn.sn_embed_fwd(E + D, ids, scale=scale).double() - sn.sn_embed_fwd(E, ids, scale=scale).double())
    left = (G.double() * diff).sum()
    dE = sn.sn_embed_bwd(G, ids, V, scale=scale)
    terms = (G.double().abs() * (diff.abs() + 2 * E[ids.long()].double().abs())).sum()
    assert abs(float(left - (dE.double() * D.double()).sum())) <= 2.0 ** -22 * float(terms)


def test_on_another_stream(sn):
    g = gen(9)
    G = torch.randn(999, 520, generator=g, device="cuda").bfloat16()
    ids = ids_of(999, 77, "skewed", g)
    ref = sn.sn_embed_bwd(G, ids, 77)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = sn.sn_embed_bwd(G, ids, 77)
        back = sn.sn_embed_fwd(got, ids)
    side.synchronize()
    assert torch.equal(got, ref) and torch.equal(back, ref[ids.long()])


def test_refusals(sn):
    t = torch.zeros(4, 8, device="cuda")
    ids = torch.zeros(3, dtype=torch.int32, device="cuda")
    G = torch.zeros(3, 8, device="cuda")
    for call in (lambda: sn.sn_embed_fwd(t, ids.long()), lambda: sn.sn_embed_fwd(t.half(), ids),
                 lambda: sn.sn_embed_bwd(G, ids, 4, out=torch.zeros(4, 8, device="cuda").half())):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: sn.sn_embed_fwd(t.cpu(), ids), lambda: sn.sn_embed_fwd(t.t(), ids),
                 lambda: sn.sn_embed_fwd(t, ids, out=torch.zeros(2, 8, device="cuda")),
                 lambda: sn.sn_embed_bwd(G, ids[:2], 4), lambda: sn.sn_embed_bwd(G.t(), ids, 4),
                 lambda: sn.sn_embed_bwd(G, ids, 4, accumulate=True)):
        with pytest.raises(ValueError):
            call()
    buf = torch.zeros(64, device="cuda")
    for call, status in (
            (lambda: sn.sn_embed_bwd(G, ids, 0), sn.SN_ERR_INVALID_ARG),
            (lambda: sn.sn_embed_fwd(buf[:32].view(4, 8), ids, out=buf[8:32].view(3, 8)), sn.SN_ERR_INVALID_ARG),
            (lambda: sn.sn_embed_fwd(buf[1:33].view(4, 8), ids), sn.SN_ERR_ALIGNMENT),
            (lambda: sn.sn_embed_bwd(G, ids, 4, workspace=torch.zeros(16, device="cuda")), sn.SN_ERR_INVALID_ARG),
            (lambda: sn.sn_embed_bwd(buf[:24].view(3, 8), ids, 4, out=buf[16:48].view(4, 8)), sn.SN_ERR_INVALID_ARG)):
        with pytest.raises(sn.SNError) as e:
            call()
        assert e.value.status == status
