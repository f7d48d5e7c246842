"""The operators of a training or serving step around a pipeline boundary, as cases that can be
timed one by one: embedding lookup and its gradient, RMS norm with the residual's addition (and an
8-bit output) and its gradient, log probabilities with entropy and alternatives and their gradient,
the global gradient norm with clipping.

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
E4M3_MAX = 448.0


@functools.lru_cache(None)
def _sn():
    from paper_2506_01260_gb300 import sn
    return sn


def listed():
    return [
        # Embedding rows of the tokens that a server decodes in one step: latency.
        _embed("embed_decode_bf16", "fwd", 64, 4096, 128256),
        # Both directions for a micro-batch of an 8B-class model: uniform ids, so that most rows are
        # gathered once, and a bf16 gradient of the whole table.
        _embed("embed_train_8b_bf16", "train", 16384, 4096, 128256),
        # The gradient for the large stream: Zipf ids as in text (a few tokens take thousands of
        # rows), summed into an fp32 gradient.
        _embed("embed_bwd_stream_f32grad", "bwd", 65536, 8192, 32000, grad="f32", ids="zipf"),
        # The norm before a decode step's 8-bit products: a few rows, one scale each.
        _norm("rmsnorm_decode_e4m3", "quant", 64, 4096),
        # Norm and gradient for a micro-batch of an 8B-class model.
        _norm("rmsnorm_train_8b_bf16", "train", 16384, 4096),
        # The large stream's norm with e4m3 codes, a scale for every 128 columns.
        _norm("rmsnorm_stream_e4m3", "quant", 65536, 8192, group=128),
        # The gradient in fp32 over packed documents: sizes that fill no tile.
        _norm("rmsnorm_bwd_packed_f32", "bwd", 4173, 2056, dtype="f32"),
        # A decode step's scores: fp32 logits of a few rows, a part of the vocabulary masked out,
        # and the 20 best alternatives.
        _logp("logprob_decode_f32", "score", 8, 128256, dtype="f32", top=20, masked=0.05),
        # Scoring a prompt: one log probability per token, entropy and 8 alternatives.
        _logp("logprob_score_8b_bf16", "score", 4096, 128256, top=8),
        # The last stage's loss and its gradient with an entropy term; rows of an odd vocabulary
        # that start off every alignment, some tokens without a target.
        _logp("logprob_train_odd_bf16", "train", 8191, 50257, ignored=0.1),
        # All gradients of the smallest model: latency.
        _grads("grads_tiny_f32", 2, 256, 256, 1024, 1024, dtype="f32"),
        # A pipeline stage's gradients: eight layers of an 8B-class model.
        _grads("grads_stage_8b_bf16", 8, 4096, 1024, 14336, 0),
    ]


def _embed(name, path, T, d, vocab, dtype="bf16", grad="bf16", ids="uniform", scale=None):
    return {"name": name, "kind": "embed", "path": path, "T": T, "d": d, "vocab": vocab,
            "dtype": dtype, "grad": grad, "ids": ids, "scale": math.sqrt(d) if scale is None else scale}


def _norm(name, path, T, d, dtype="bf16", group=0, residual=True):
    """`group`: columns that share a scale (0: the whole row)."""
    return {"name": name, "kind": "norm", "path": path, "T": T, "d": d, "dtype": dtype,
            "group": group, "residual": residual}


def _logp(name, path, T, vocab, dtype="bf16", top=0, masked=0.0, ignored=0.0, scale=1.0, pad=0):
    """`masked`: share of the vocabulary at -inf; `ignored`: share of the tokens without a target;
    `pad`: unused columns at the end of the logits' rows."""
    return {"name": name, "kind": "logp", "path": path, "T": T, "vocab": vocab, "dtype": dtype,
            "top": top, "masked": masked, "ignored": ignored, "scale": scale, "pad": pad}


def _grads(name, layers, d, kv, ff, vocab, dtype="bf16", std=0.01):
    return {"name": name, "kind": "grads", "path": "clip", "layers": layers, "d": d, "kv": kv,
            "ff": ff, "vocab": vocab, "dtype": dtype, "std": std}


# ---- more cases of the same ranges ---------------------------------------------------

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
    kind = rng.choice(["embed", "norm", "logp", "grads"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    es = ES[dtype]
    if kind == "embed":
        d = _width(rng, 256, 8192)
        vocab = rng.choice([1024, 32000, 50257, 128256])
        path = rng.choice(["fwd", "bwd", "train"])
        T = _tokens(rng, min(65536, (1 << 29) // d))
        return {k: v for k, v in _embed("", path, T, d, vocab if vocab * d <= 1 << 28 else 32000,
                                        dtype=dtype, grad=rng.choice([dtype, "f32"]),
                                        ids=rng.choice(["uniform", "zipf"]),
                                        scale=rng.choice([1.0, None])).items() if k != "name"}
    if kind == "norm":
        d = _width(rng, 256, 8192)
        path = rng.choice(["fwd", "quant", "bwd", "train"])
        T = _tokens(rng, min(65536, (1 << 29) // (d * es)))
        return {k: v for k, v in _norm("", path, T, d, dtype=dtype, group=rng.choice([0, 128]),
                                       residual=rng.random() < 0.7).items() if k != "name"}
    if kind == "logp":
        vocab = rng.choice([1024, 32000, 50257, 128256])
        path = rng.choice(["score", "train"])
        T = _tokens(rng, min(16384, (1 << 29) // (vocab * es)))
        return {k: v for k, v in _logp("", path, T, vocab, dtype=dtype,
                                       top=rng.choice([0, 1, 5, 20, 32]) if path == "score" else 0,
                                       masked=rng.choice([0.0, 0.05, 0.9]),
                                       ignored=rng.choice([0.0, 0.3]),
                                       scale=rng.choice([1.0, 1.25, 0.5]),
                                       pad=rng.choice([0, 0, 47])).items() if k != "name"}
    d = _width(rng, 128, 4096)
    layers = rng.randrange(1, 7) if d > 2048 else rng.randrange(1, 25)
    ff = int(d * rng.choice([2.0, 2.6875, 3.5, 4.0])) + rng.choice([0, 0, 1])
    vocab = rng.choice([0, 1024, 32000])
    if es == 4:
        layers = max(1, layers // 2)
    return {k: v for k, v in _grads("", layers, d, max(8, d // rng.choice([1, 4])), ff, vocab,
                                    dtype=dtype, std=rng.choice([1e-7, 0.01, 0.01])).items()
            if k != "name"}


# ---- inputs --------------------------------------------------------------------------------

def _ids(T, vocab, how, g):
    if how == "uniform":
        return torch.randint(vocab, (T,), generator=g, device="cuda", dtype=torch.int32)
    p = torch.arange(1, vocab + 1, device="cuda", dtype=torch.float64) ** -1.1
    ranks = torch.multinomial(p, T, replacement=True, generator=g)
    return torch.randperm(vocab, generator=g, device="cuda")[ranks].int()


def _embed_inputs(c, g):
    T, d, vocab, dt = c["T"], c["d"], c["vocab"], DTYPES[c["dtype"]]
    s = {"ids": _ids(T, vocab, c["ids"], g), "vocab": vocab, "scale": c["scale"],
         "gdt": DTYPES[c["grad"]]}
    if c["path"] != "bwd":
        s["table"] = torch.randn(vocab, d, generator=g, device="cuda", dtype=dt).mul_(0.02)
    if c["path"] != "fwd":
        s["G"] = torch.randn(T, d, generator=g, device="cuda", dtype=dt)
    return s


def _norm_inputs(c, g):
    """A residual stream as the norm sees it: unit variance, a few channels much larger."""
    T, d, dt = c["T"], c["d"], DTYPES[c["dtype"]]
    big = 1 + 7 * (torch.rand(d, generator=g, device="cuda") < 0.01).float()

    def batch():
        return torch.randn(T, d, generator=g, device="cuda", dtype=dt).mul_(big.to(dt))

    s = {"w": 1 + 0.1 * torch.randn(d, generator=g, device="cuda"), "group": c["group"]}
    if c["path"] == "bwd":
        s["H"] = batch()
    else:
        s["X"] = batch()
    if c["residual"]:
        s["R" if c["path"] != "bwd" else "dH"] = batch()
        if c["path"] == "train":
            s["dH"] = torch.randn(T, d, generator=g, device="cuda", dtype=dt)
    if c["path"] in ("bwd", "train"):
        s["dY"] = torch.randn(T, d, generator=g, device="cuda", dtype=dt)
    return s


def _logp_inputs(c, g):
    """Logits with a few likely tokens a row, the target among them more often than not."""
    T, V, dt = c["T"], c["vocab"], DTYPES[c["dtype"]]
    full = torch.randn(T, V + c["pad"], generator=g, device="cuda", dtype=dt).mul_(2.5)
    x = full[:, :V]
    target = torch.randint(V, (T,), generator=g, device="cuda", dtype=torch.int32)
    rows = torch.arange(T, device="cuda")
    x[rows, target.long()] += torch.rand(T, generator=g, device="cuda").mul_(14).to(dt)
    if c["masked"]:
        x.masked_fill_(torch.rand(V, generator=g, device="cuda") < c["masked"], -math.inf)
        x[:, V // 2] = 1.0                                   # no row is left without a token
    if c["ignored"]:
        none = torch.rand(T, generator=g, device="cuda") < c["ignored"]
        target = torch.where(none, torch.full_like(target, -100), target)
    s = {"x": x, "target": target, "scale": c["scale"], "top": c["top"], "train": c["path"] == "train"}
    if s["train"]:
        s["dlogp"] = torch.randn(T, generator=g, device="cuda").mul_(1.0 / T)
        s["dentropy"] = torch.full((T,), 0.01 / T, device="cuda")
    return s


def _shapes(c):
    d, kv, ff = c["d"], c["kv"], c["ff"]
    layer = [(d, d), (kv, d), (kv, d), (d, d), (ff, d), (ff, d), (d, ff), (d,), (d,)]
    return ([(c["vocab"], d)] if c["vocab"] else []) + layer * c["layers"]


def _grads_inputs(c, g):
    """Gradients as views of one buffer, one behind the other."""
    shapes = _shapes(c)
    sizes = [math.prod(x) for x in shapes]
    flat = torch.randn(sum(sizes), generator=g, device="cuda", dtype=DTYPES[c["dtype"]]).mul_(c["std"])
    return {"flat": flat, "grads": [v.view(x) for v, x in zip(flat.split(sizes), shapes)],
            "sizes": sizes, "max_norm": 1.0}


_INPUTS = {"embed": _embed_inputs, "norm": _norm_inputs, "logp": _logp_inputs,
           "grads": _grads_inputs}


def _make(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = _INPUTS[case["kind"]](case, g)
    s["kind"], s["path"] = case["kind"], case["path"]
    return s


def prepare(case, seed):
    s = _make(case, seed)
    if case["kind"] == "grads":
        s["flat_out"] = torch.empty_like(s["flat"])
        s["out"] = [v.view(x.shape) for v, x in zip(s["flat_out"].split(s["sizes"]), s["grads"])]
        if own:                                              # the list's handle, made once
            s["list"] = _sn().GradList(s["grads"], out=s["out"])
    return s


# ---- one pass --------------------------------------------------------------------------------

def run(s):
    return (_OWN if own else _PLAIN)[s["kind"]](s)


def _own_embed(s):
    sn, out = _sn(), {}
    if "table" in s:
        out["X"] = sn.sn_embed_fwd(s["table"], s["ids"], scale=s["scale"])
    if "G" in s:
        out["dE"] = sn.sn_embed_bwd(s["G"], s["ids"], s["vocab"], scale=s["scale"], out_dtype=s["gdt"])
    return out


def _plain_embed(s):
    out, ids = {}, s["ids"].long()
    if "table" in s:
        out["X"] = (s["table"][ids].float() * s["scale"]).to(s["table"].dtype)
    if "G" in s:
        dE = torch.zeros(s["vocab"], s["G"].shape[1], device="cuda")
        out["dE"] = dE.index_add_(0, ids, s["G"].float() * s["scale"]).to(s["gdt"])
    return out


def _own_norm(s):
    sn, out = _sn(), {}
    if s["path"] == "quant":
        codes, scale, H = sn.sn_rmsnorm_fwd_quant(s["X"], s["w"], EPS, "e4m3", R=s.get("R"),
                                                  group=s["group"])
        return {"codes": codes.view(torch.float8_e4m3fn), "scale": scale, "H": H}
    H = s.get("H")
    if "X" in s:
        out["Y"], H = sn.sn_rmsnorm_fwd(s["X"], s["w"], EPS, R=s.get("R"))
        out["H"] = H
    if "dY" in s:
        out["dX"], out["dw"] = sn.sn_rmsnorm_bwd(s["dY"], H, s["w"], EPS, dH=s.get("dH"))
    return out


def _plain_norm(s):
    out, w, H = {}, s["w"], s.get("H")
    if "X" in s:
        h = s["X"].float() + s["R"].float() if "R" in s else s["X"].float()
        y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * w
        H = h.to(s["X"].dtype) if "R" in s else s["X"]
        out["H"] = H
        if s["path"] == "quant":
            T, d = y.shape
            n = s["group"] or d
            y = torch.nn.functional.pad(y, (0, -d % n)).view(T, -1, n)
            a = y.abs().amax(2, keepdim=True)
            codes = (y * torch.where(a > 0, E4M3_MAX / a, 0.0)).clamp(-E4M3_MAX, E4M3_MAX)
            out["codes"] = codes.view(T, -1)[:, :d].to(torch.float8_e4m3fn)
            out["scale"] = (a / E4M3_MAX).view(T, -1) if s["group"] else (a / E4M3_MAX).view(T)
            return out
        out["Y"] = y.to(s["X"].dtype)
    if "dY" in s:
        h, dy = H.float(), s["dY"].float()
        rs = torch.rsqrt(h.square().mean(1, keepdim=True) + EPS)
        g = dy * w
        dx = rs * (g - h * (rs * rs * (g * h).mean(1, keepdim=True)))
        out["dX"] = (dx + s["dH"].float() if "dH" in s else dx).to(H.dtype)
        out["dw"] = (dy * h * rs).sum(0)
    return out


def _own_logp(s):
    sn = _sn()
    logp, lse, H, ids, alt = sn.sn_logprob_fwd(s["x"], s["target"], scale=s["scale"], top=s["top"])
    out = {"logp": logp, "entropy": H}
    if s["top"]:
        out["top_ids"], out["top_logp"] = ids, alt
    if s["train"]:
        out["dx"] = sn.sn_logprob_bwd(s["x"], lse, s["target"], s["dlogp"], scale=s["scale"],
                                      entropy=H, dentropy=s["dentropy"])
    return out


def _plain_logp(s):
    z = s["x"].float() * s["scale"]
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    total = e.sum(1, keepdim=True)
    lse = m + torch.log(total)
    t = s["target"].long()[:, None]
    some = t >= 0
    at = t.clamp(min=0)
    logp = torch.where(some, z.gather(1, at) - lse, 0.0)
    H = lse - torch.where(e > 0, e * z, 0.0).sum(1, keepdim=True) / total
    out = {"logp": logp[:, 0], "entropy": H[:, 0]}
    if s["top"]:
        # unique whole keys: the value's order in the upper half, the lower id first in the lower
        bits = (s["x"].float() + 0.0).view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        ids = torch.arange(z.shape[1], device=z.device)
        keys = order * (1 << 32) + ((1 << 32) - 1 - ids)
        best = torch.topk(keys, s["top"], dim=1).indices
        out["top_ids"], out["top_logp"] = best.int(), z.gather(1, best) - lse
    if s["train"]:
        a, b = s["dlogp"][:, None], s["dentropy"][:, None]
        p, q = e / total, z - lse
        a = torch.where(some, a, 0.0)
        dx = -p * a - torch.where(e > 0, p * (q + H), 0.0) * b
        dx.scatter_add_(1, at, a)
        out["dx"] = (dx * s["scale"]).to(s["x"].dtype)
    return out


def _own_grads(s):
    sn = _sn()
    sumsq = sn.sn_grads_sumsq(s["list"])
    return {"norm": sn.sn_grads_clip(s["list"], sumsq, s["max_norm"]), "grads": s["flat_out"]}


def _plain_grads(s):
    norm = torch.stack([g.float().square().sum() for g in s["grads"]]).sum().sqrt()
    c = s["max_norm"] / norm.clamp(min=s["max_norm"])
    return {"norm": norm.reshape(1), "grads": (s["flat"].float() * c).to(s["flat"].dtype)}


_OWN = {"embed": _own_embed, "norm": _own_norm, "logp": _own_logp, "grads": _own_grads}
_PLAIN = {"embed": _plain_embed, "norm": _plain_norm, "logp": _plain_logp, "grads": _plain_grads}


# ---- what a pass cannot do without -----------------------------------------------------------

def work(case):
    return _WORK[case["kind"]](case)


def _work_embed(c):
    T, d, V, es = c["T"], c["d"], c["vocab"], ES[c["dtype"]]
    n, flops = 4 * T, 0
    if c["path"] != "bwd":
        n += es * d * (_expected_unique(c) + T)
        flops += T * d
    if c["path"] != "fwd":
        n += es * T * d + ES[c["grad"]] * V * d
        flops += 2 * T * d
    return {"bytes": n, "flops": flops}


def _expected_unique(c):
    T, V = c["T"], c["vocab"]
    if c["ids"] == "uniform":
        return int(V * (1 - (1 - 1 / V) ** T))
    w = [(r + 1) ** -1.1 for r in range(V)]
    z = sum(w)
    return int(sum(1 - (1 - x / z) ** T for x in w))


def _work_norm(c):
    T, d, es = c["T"], c["d"], ES[c["dtype"]]
    more = 1 if c["residual"] else 0
    one = es * T * d
    n, flops = 4 * d, 0
    if c["path"] in ("fwd", "train"):
        n, flops = n + (2 + 2 * more) * one, flops + 5 * T * d
    if c["path"] == "quant":
        n += (1 + 2 * more) * one + T * d + 4 * T * (-(-d // c["group"]) if c["group"] else 1)
        flops += 8 * T * d
    if c["path"] in ("bwd", "train"):
        # in a training pass the gradient's h is the forward's output
        n += (2 + more + (1 if c["path"] == "bwd" else 0)) * one + 4 * d
        flops += 11 * T * d
    return {"bytes": n, "flops": flops}


def _work_logp(c):
    T, V, es = c["T"], c["vocab"], ES[c["dtype"]]
    n = es * T * V + 4 * T * (3 + 2 * c["top"])
    if c["path"] == "train":
        n += es * T * V + 8 * T
    return {"bytes": n, "flops": T * V * (6 + (8 if c["path"] == "train" else 0))}


def _work_grads(c):
    n = sum(math.prod(x) for x in _shapes(c))
    return {"bytes": 2 * ES[c["dtype"]] * n, "flops": 3 * n}


_WORK = {"embed": _work_embed, "norm": _work_norm, "logp": _work_logp, "grads": _work_grads}


# ---- the results in 64 bits --------------------------------------------------------------------

def exact(case, seed):
    return _EXACT[case["kind"]](case, _make(case, seed))


def _exact_embed(c, s):
    out, ids = {}, s["ids"].long()
    if "table" in s:
        out["X"] = c["scale"] * s["table"].double()[ids]
    if "G" in s:
        # running sums over the tokens in order of their ids, taken where an id's tokens end
        G, T = s["G"], c["T"]
        order = torch.argsort(ids, stable=True)
        ended = torch.cumsum(torch.bincount(ids, minlength=c["vocab"]), 0)
        dE = torch.empty(c["vocab"], G.shape[1], device="cuda", dtype=torch.float64)
        for c0 in range(0, G.shape[1], 512):
            part = G[:, c0:c0 + 512].double()[order]
            run_ = torch.zeros(T + 1, part.shape[1], device="cuda", dtype=torch.float64)
            run_[1:] = torch.cumsum(part, 0)
            at = run_[ended]
            at[1:] -= run_[ended[:-1]]
            dE[:, c0:c0 + 512] = c["scale"] * at
        out["dE"] = dE
    return out


def _exact_norm(c, s):
    out, w, d = {}, s["w"].double(), c["d"]
    h = None
    if "X" in s:
        h = s["X"].double()
        if "R" in s:
            h = h + s["R"].double()
        y = h / (h.pow(2).sum(1, keepdim=True) / d + EPS).sqrt() * w
        out["H"] = h
        if c["path"] == "quant":
            n = c["group"] or d
            parts = [y[:, j:j + n] for j in range(0, d, n)]
            scale = torch.stack([p.abs().amax(1) for p in parts], 1) / E4M3_MAX
            out["codes"] = torch.cat([p / scale[:, j:j + 1] for j, p in enumerate(parts)], 1)
            out["scale"] = scale if c["group"] else scale[:, 0]
            return out
        out["Y"] = y
        # the gradient reads h as the forward stored it
        h = h.to(DTYPES[c["dtype"]]).double()
    if "dY" in s:
        if h is None:
            h = s["H"].double()
        dy = s["dY"].double()
        r = (h.pow(2).sum(1) / d + EPS).sqrt()
        n = h / r[:, None]
        g = dy * w
        dx = (g - n * (g * n).sum(1, keepdim=True) / d) / r[:, None]
        out["dX"] = dx + s["dH"].double() if "dH" in s else dx
        out["dw"] = (dy * n).sum(0)
    return out


def _exact_logp(c, s):
    T, V = s["x"].shape
    target = s["target"].long()
    out = {"logp": torch.zeros(T, device="cuda", dtype=torch.float64),
           "entropy": torch.empty(T, device="cuda", dtype=torch.float64)}
    if c["top"]:
        out["top_ids"] = None
        out["top_logp"] = torch.empty(T, c["top"], device="cuda", dtype=torch.float64)
    if s["train"]:
        out["dx"] = torch.empty(T, V, device="cuda", dtype=torch.float64)
    for t0 in range(0, T, 1024):
        r = slice(t0, min(T, t0 + 1024))
        q = torch.log_softmax(c["scale"] * s["x"][r].double(), 1)
        p = q.exp()
        H = -torch.where(p > 0, p * q, 0.0).sum(1)
        out["entropy"][r] = H
        i = torch.nonzero(target[r] >= 0)[:, 0]
        j = target[r][i]
        out["logp"][r][i] = q[i, j]
        if c["top"]:
            out["top_logp"][r] = torch.topk(q, c["top"], dim=1).values
        if s["train"]:
            one = torch.zeros_like(q)
            one[i, j] = 1.0
            a = torch.zeros(q.shape[0], device="cuda", dtype=torch.float64)
            a[i] = s["dlogp"][r].double()[i]
            dq = a[:, None] * (one - p)
            dH = -torch.where(p > 0, p * (q + H[:, None]), 0.0)
            out["dx"][r] = c["scale"] * (dq + s["dentropy"][r].double()[:, None] * dH)
    return out


def _exact_grads(c, s):
    norm = s["flat"].double().pow(2).sum().sqrt()
    clipped = s["flat"].double()
    if float(norm) > s["max_norm"]:
        clipped = clipped * (s["max_norm"] / norm)
    return {"norm": norm.reshape(1), "grads": clipped}


_EXACT = {"embed": _exact_embed, "norm": _exact_norm, "logp": _exact_logp, "grads": _exact_grads}
