"""The feed-forward half of a transformer block as a stage runs it between its boundary calls, in
cases that can be timed one by one: the gated pair of projections (H = act(X Wgᵀ) ⊙ (X Wuᵀ)) with
its gradients, and the norms before and after a block, fused with the block's gate and residual
scale, and their gradients.

`prepare` makes the inputs, `run` takes one pass: in elementary torch operations in fp32, rounded
once at the end, or, where `own` is true, through `paper_2506_01260_gb300.sn`.  `work` counts the
bytes and operations that a pass cannot do without, `exact` gives its results in 64 bits and `draw`
makes further cases of the same ranges.
"""
import functools
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ES = {"bf16": 2, "f32": 4}
EPS = 1e-5


@functools.lru_cache(None)
def _sn():
    from paper_2506_01260_gb300 import sn
    return sn


def listed():
    return [
        # The smallest block of the repository's own example, a few tokens of a decode step: latency.
        _glu("glu_decode_tiny", "fwd", 8, 256, 512, act="relu"),
        # One token of one request through an 8B-class block: the weights are read once.
        _glu("glu_decode_1_8b", "fwd", 1, 4096, 14336),
        # A decode step of a batch of requests, odd in number.
        _glu("glu_decode_75_8b", "fwd", 75, 4096, 14336),
        # A prompt of 2048 tokens at the large stream's width: forward alone, nothing kept.
        _glu("glu_prompt_stream", "fwd", 2048, 8192, 28672),
        # A micro-batch of an 8B-class model: forward that keeps the projections, and the gradients.
        _glu("glu_train_8b", "train", 8192, 4096, 14336),
        # Gradients over packed documents, sizes that fill no tile.
        _glu("glu_bwd_packed_gelu", "bwd", 4173, 2056, 5512, act="gelu_tanh"),
        # The norms after and before a block in a decode step: latency.
        _norms("norms_decode_bf16", "fwd", 64, 4096, gates=0),
        # The large stream's norms, each of 16 sequences with a gate of its own.
        _norms("norms_stream_gated_bf16", "fwd", 65536, 8192, gates=16, scale=0.5),
        # The gradients for a micro-batch of an 8B-class model, one gate a channel for all tokens.
        _norms("norms_bwd_8b_bf16", "bwd", 16384, 4096, gates=1),
        # Gradients in fp32 over packed documents: sizes that fill no tile, no gate.
        _norms("norms_bwd_packed_f32", "bwd", 4173, 2056, dtype="f32", gates=0, scale=0.25),
    ]


def _glu(name, path, T, d, f, act="silu"):
    return {"name": name, "kind": "glu", "path": path, "T": T, "d": d, "f": f, "act": act}


def _norms(name, path, T, d, dtype="bf16", gates=0, scale=1.0):
    """`gates`: rows of the gate, each for T / gates tokens in a run (0: none)."""
    return {"name": name, "kind": "norms", "path": path, "T": T, "d": d, "dtype": dtype,
            "gates": gates, "scale": scale}


# ---- more cases of the same ranges ---------------------------------------------------

MOST_FLOPS = 12 * 8192 * 4096 * 14336        # the largest listed case


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A model width: mostly a power of two, sometimes a multiple of 8 alone."""
    d = _log(rng, lo, hi)
    if rng.random() < 0.6:
        return max(lo, min(hi, 1 << round(math.log2(d))))
    return max(lo, d // 16 * 16 - 8)


def _tokens(rng, hi):
    """A number of tokens: a power of two as in training, or an odd one."""
    T = _log(rng, 1, hi)
    return min(hi, 1 << round(math.log2(T))) if rng.random() < 0.4 else min(hi, T | 1)


def draw(rng):
    if rng.random() < 0.55:
        d = _width(rng, 256, 8192)
        f = int(d * rng.choice([1.0, 2.0, 2.6875, 3.5, 4.0])) // 8 * 8
        path = rng.choice(["fwd", "fwd", "bwd", "train"])
        T = _tokens(rng, max(1, min(16384, MOST_FLOPS // (12 * d * f))))
        c = _glu("", path, T, d, f, act=rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu"]))
    else:
        d = _width(rng, 256, 8192)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        T = _tokens(rng, min(65536, (1 << 29) // (d * ES[dtype])))
        per = rng.choice([1, 3, 16, 128])            # tokens that share a gate
        how = rng.choice(["none", "one", "many"])
        if how == "many" and T >= per:
            T = T // per * per
        gates = 0 if how == "none" else 1 if how == "one" or T < per else T // per
        c = _norms("", rng.choice(["fwd", "bwd"]), T, d, dtype=dtype, gates=gates,
                   scale=rng.choice([1.0, 0.5, 0.1]))
    return {k: v for k, v in c.items() if k != "name"}


# ---- inputs --------------------------------------------------------------------------------

def _glu_inputs(c, g):
    """Normed activations, weights of a network at work, a gradient of a mean loss."""
    T, d, f = c["T"], c["d"], c["f"]

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.bfloat16).mul_(std)

    s = {"X": normal(T, d), "Wg": normal(f, d, std=1 / math.sqrt(d)),
         "Wu": normal(f, d, std=1 / math.sqrt(d)), "act": c["act"]}
    if c["path"] != "fwd":
        s["dH"] = normal(T, f, std=1e-3)
    if c["path"] == "bwd":
        s["G"], s["U"] = normal(T, f), normal(T, f)
    return s


def _norms_inputs(c, g):
    """A residual stream with a few channels much larger, and a block's output beside it."""
    T, d, dt, n = c["T"], c["d"], DTYPES[c["dtype"]], c["gates"]
    big = 1 + 7 * (torch.rand(d, generator=g, device="cuda") < 0.01).float()

    def batch(spread=True):
        x = torch.randn(T, d, generator=g, device="cuda", dtype=dt)
        return x.mul_(big.to(dt)) if spread else x

    s = {"Y": batch(), "scale": c["scale"], "gate": None,
         "w_post": 1 + 0.1 * torch.randn(d, generator=g, device="cuda"),
         "w_pre": 1 + 0.1 * torch.randn(d, generator=g, device="cuda")}
    if n:
        s["gate"] = torch.randn(n, d, generator=g, device="cuda").mul_(0.5).add_(1.0).to(dt)
    if c["path"] == "bwd":
        s["H"] = batch()
    else:
        s["R"] = batch()
    if c["path"] != "fwd":
        s["dZ"], s["dH"] = batch(False), batch(False)
    return s


_INPUTS = {"glu": _glu_inputs, "norms": _norms_inputs}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = _INPUTS[case["kind"]](case, g)
    s["kind"], s["path"] = case["kind"], case["path"]
    return s


# ---- one pass --------------------------------------------------------------------------------

def run(s):
    return (_OWN if own else _PLAIN)[s["kind"]](s)


def _own_glu(s):
    sn, out, G, U = _sn(), {}, s.get("G"), s.get("U")
    if s["path"] != "bwd":
        out["H"], G, U = sn.sn_glu_fwd(s["X"], s["Wg"], s["Wu"], s["act"], keep=s["path"] == "train")
        if s["path"] == "fwd":
            return out
        out["G"], out["U"] = G, U
    dX, dWg, dWu, dG, dU = sn.sn_glu_bwd(s["dH"], s["X"], s["Wg"], s["Wu"], G, U, s["act"])
    out.update(dX=dX, dWg=dWg, dWu=dWu, dG=dG, dU=dU)
    return out


def _act(g, act):
    """The activation and its derivative."""
    if act == "relu":
        on = (g > 0).float()
        return g * on, on
    if act == "silu":
        p = 1 / (1 + torch.exp(-g))
        return g * p, p * (1 + g * (1 - p))
    if act == "gelu":
        p = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * p, p + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    k = math.sqrt(2 / math.pi)
    t = torch.tanh(k * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * k * (1 + 0.134145 * g * g)


def _plain_glu(s):
    out, bf16 = {}, torch.bfloat16
    X, Wg, Wu = s["X"].float(), s["Wg"].float(), s["Wu"].float()
    if s["path"] != "bwd":
        g, u = X @ Wg.T, X @ Wu.T
        out["H"] = (_act(g, s["act"])[0] * u).to(bf16)
        if s["path"] == "fwd":
            return out
        out["G"], out["U"] = g.to(bf16), u.to(bf16)
    # the gradient reads the projections as the forward stored them, and the products read dG and
    # dU as they are stored
    G, U, dH = out.get("G", s.get("G")).float(), out.get("U", s.get("U")).float(), s["dH"].float()
    a, da = _act(G, s["act"])
    out["dG"], out["dU"] = (dH * U * da).to(bf16), (dH * a).to(bf16)
    dG, dU = out["dG"].float(), out["dU"].float()
    out["dX"] = (dG @ Wg + dU @ Wu).to(bf16)
    out["dWg"], out["dWu"] = (dG.T @ X).to(bf16), (dU.T @ X).to(bf16)
    return out


def _own_norms(s):
    sn = _sn()
    if s["path"] == "fwd":
        Z, H = sn.sn_blocknorm_fwd(s["Y"], s["R"], s["w_post"], s["w_pre"], EPS, scale=s["scale"],
                                   gate=s["gate"])
        return {"Z": Z, "H": H}
    dY, dR, dw_post, dw_pre, dgate = sn.sn_blocknorm_bwd(s["dZ"], s["H"], s["Y"], s["w_post"],
                                                         s["w_pre"], EPS, scale=s["scale"],
                                                         gate=s["gate"], dH=s["dH"])
    out = {"dY": dY, "dR": dR, "dw_post": dw_post, "dw_pre": dw_pre}
    if dgate is not None:
        out["dgate"] = dgate
    return out


def _plain_norms(s):
    Y, gate, d, dt = s["Y"].float(), s["gate"], s["Y"].shape[1], s["Y"].dtype
    if gate is None:
        a = torch.full((1, 1, d), s["scale"], device="cuda")
    else:
        a = gate.float()[:, None, :] * s["scale"]
    rows = (a.shape[0], -1, d)                       # the tokens of each gate
    r1 = torch.rsqrt(Y.square().mean(1, keepdim=True) + EPS)
    b = Y * r1 * s["w_post"]
    if s["path"] == "fwd":
        h = s["R"].float() + (a * b.view(rows)).view(Y.shape)
        z = h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * s["w_pre"]
        return {"Z": z.to(dt), "H": h.to(dt)}
    h, dz = s["H"].float(), s["dZ"].float()
    r2 = torch.rsqrt(h.square().mean(1, keepdim=True) + EPS)
    g = dz * s["w_pre"]
    dh = r2 * (g - h * (r2 * r2 * (g * h).mean(1, keepdim=True))) + s["dH"].float()
    db = (a * dh.view(rows)).view(Y.shape)
    g = db * s["w_post"]
    dy = r1 * (g - Y * (r1 * r1 * (g * Y).mean(1, keepdim=True)))
    out = {"dY": dy.to(dt), "dR": dh.to(dt), "dw_post": (db * Y * r1).sum(0),
           "dw_pre": (dz * h * r2).sum(0)}
    if gate is not None:
        out["dgate"] = (dh * b).view(rows).sum(1) * s["scale"]
    return out


_OWN = {"glu": _own_glu, "norms": _own_norms}
_PLAIN = {"glu": _plain_glu, "norms": _plain_norms}


# ---- what a pass cannot do without -----------------------------------------------------------

def work(case):
    return _WORK[case["kind"]](case)


def _work_glu(c):
    T, d, f, path = c["T"], c["d"], c["f"], c["path"]
    n, flops = T * d + 2 * f * d, 0                  # X and the weights
    if path != "bwd":
        n, flops = n + T * f, 4 * T * d * f          # H
    if path != "fwd":
        # dH; G and U, written by the forward or read; dG, dU, dX and the weights' gradients
        n, flops = n + T * f + 2 * T * f + 2 * T * f + T * d + 2 * f * d, flops + 8 * T * d * f
    return {"bytes": 2 * n, "flops": flops}


def _work_norms(c):
    T, d, es, path, gates = c["T"], c["d"], ES[c["dtype"]], c["path"], c["gates"]
    n, one = 8 * d + es * gates * d, es * T * d
    if path == "fwd":
        return {"bytes": n + 4 * one, "flops": 11 * T * d}       # Y, R, H, Z
    # dZ, dH, Y, H, dY, dR, the gradients of the weights and the gate
    return {"bytes": n + 6 * one + 8 * d + 4 * gates * d, "flops": 28 * T * d}


_WORK = {"glu": _work_glu, "norms": _work_norms}


# ---- the results in 64 bits --------------------------------------------------------------------

def exact(case, seed):
    if work(case)["flops"] > 1e13:                   # over a few seconds in 64 bits
        return None
    return _EXACT[case["kind"]](case, prepare(case, seed))


def _exact_act(g, act):
    if act == "relu":
        return torch.clamp(g, min=0), torch.where(g > 0, 1.0, 0.0).double()
    if act == "silu":
        p = torch.sigmoid(g)
        return p * g, p + p * g * torch.sigmoid(-g)
    if act == "gelu":
        p = 0.5 * torch.erfc(-g / math.sqrt(2.0))
        return p * g, p + g * torch.exp(-g.pow(2) / 2) / math.sqrt(2 * math.pi)
    # tanh form: (1 + tanh(x)) / 2 = sigmoid(2 x)
    k = 2 * math.sqrt(2 / math.pi)
    p = torch.sigmoid(k * g * (1 + 0.044715 * g.pow(2)))
    return p * g, p + g * p * (1 - p) * k * (1 + 3 * 0.044715 * g.pow(2))


def _exact_glu(c, s):
    out, bf16 = {}, torch.bfloat16
    X, Wg, Wu = s["X"].double(), s["Wg"].double(), s["Wu"].double()
    if c["path"] != "bwd":
        out["G"], out["U"] = torch.mm(X, Wg.t()), torch.mm(X, Wu.t())
        out["H"] = _exact_act(out["G"], c["act"])[0].mul_(out["U"])
        if c["path"] == "fwd":
            return {"H": out["H"]}
        G, U = out["G"].to(bf16).double(), out["U"].to(bf16).double()
    else:
        G, U = s["G"].double(), s["U"].double()
    a, da = _exact_act(G, c["act"])
    dH = s["dH"].double()
    out["dU"], out["dG"] = a.mul_(dH), da.mul_(dH).mul_(U)
    dG, dU = out["dG"].to(bf16).double(), out["dU"].to(bf16).double()
    out["dX"] = torch.addmm(torch.mm(dG, Wg), dU, Wu)
    out["dWg"], out["dWu"] = torch.mm(dG.t(), X), torch.mm(dU.t(), X)
    return {k: out[k] for k in ("H", "G", "U", "dG", "dU", "dX", "dWg", "dWu") if k in out}


def _exact_norms(c, s):
    T, d, n = c["T"], c["d"], c["gates"]
    w1, w2 = s["w_post"].double(), s["w_pre"].double()
    token = torch.arange(T, device="cuda") // (T // n if n else 1)
    names = ("Z", "H") if c["path"] == "fwd" else ("dY", "dR")
    out = {name: torch.empty(T, d, device="cuda", dtype=torch.float64) for name in names}
    if c["path"] == "bwd":
        out["dw_post"], out["dw_pre"] = (torch.zeros(d, device="cuda", dtype=torch.float64) for _ in "12")
        if n:
            out["dgate"] = torch.zeros(n, d, device="cuda", dtype=torch.float64)
    for t0 in range(0, T, 4096):
        r = slice(t0, min(T, t0 + 4096))
        y = s["Y"][r].double()
        q1 = (y.pow(2).sum(1, keepdim=True) / d + EPS).sqrt()
        n1 = y / q1
        m = s["gate"].double()[token[r]] * c["scale"] if n else torch.full_like(y, c["scale"])
        if c["path"] == "fwd":
            h = s["R"][r].double() + m * n1 * w1
            out["H"][r] = h
            out["Z"][r] = h / (h.pow(2).sum(1, keepdim=True) / d + EPS).sqrt() * w2
            continue
        h = s["H"][r].double()
        q2 = (h.pow(2).sum(1, keepdim=True) / d + EPS).sqrt()
        n2, dz = h / q2, s["dZ"][r].double()
        dh = (dz * w2 - n2 * ((dz * w2 * n2).sum(1, keepdim=True) / d)) / q2 + s["dH"][r].double()
        e = dh * m * w1
        out["dR"][r] = dh
        out["dY"][r] = (e - n1 * ((e * n1).sum(1, keepdim=True) / d)) / q1
        out["dw_pre"] += (dz * n2).sum(0)
        out["dw_post"] += (dh * m * n1).sum(0)
        if n:
            out["dgate"].index_add_(0, token[r], c["scale"] * dh * n1 * w1)
    return out


_EXACT = {"glu": _exact_glu, "norms": _exact_norms}
