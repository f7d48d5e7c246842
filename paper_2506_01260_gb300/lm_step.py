"""A two-stage language model's training step and scoring around one pipeline boundary, on one GPU.

Stage 0 looks tokens up, adds one block's output and compresses the residual stream onto the
subspace; stage 1 reconstructs it, norms it and scores it against the next tokens; the gradients
take the same way back.  The library's calls do everything but the matrix products, which are
torch's.  Weights are random and the text is a synthetic chain of tokens, so the model only shows
how the calls fit together:

    python -m paper_2506_01260_gb300.lm_step [gated]

`gated`: stage 1 has a gated feed-forward block of its own, with norms before and after it.  (Behind
a boundary: a norm's weights take a block's output out of S, which the streams that cross one stay in.)

The embedding is T_fixed[ids] + T_S[ids] with T_S's rows in S = Col(U), and the block writes to the
residual stream through a weight whose columns lie in S, so the stream minus T_fixed[ids] stays in
S (Sec. 4.3) and the boundary loses nothing but roundings.
"""
import math
import sys

import torch

from . import sn

EPS = 1e-5
BF16 = torch.bfloat16


class TwoStage:
    """Parameters (bf16 where the products read them), their fp32 gradients and the optimizer."""

    def __init__(self, vocab=512, d=256, d_ff=512, k=16, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)

        def normal(*shape, std=0.02):
            return std * torch.randn(*shape, generator=g, device=device)

        self.vocab, self.d = vocab, d
        U = torch.linalg.qr(normal(d, k, std=1.0).double().cpu())[0].float().contiguous().to(device)
        self.basis = sn.Basis(U)
        self.T_fixed = normal(vocab, d).to(BF16)
        self.T_S = sn.sn_build_ts(self.basis, normal(vocab, d, std=0.2).to(BF16))
        self.W_up = normal(d_ff, d, std=1 / math.sqrt(d)).to(BF16)
        self.W_down = sn.sn_project_weight(self.basis, normal(d, d_ff, std=1 / math.sqrt(d_ff)).to(BF16))
        self.W_head = normal(vocab, d, std=1 / math.sqrt(d)).to(BF16)
        self.w0, self.w1 = torch.ones(d, device=device), torch.ones(d, device=device)
        # fp32 master weight and moments of the row-constant AdamW step on W_down
        self.master = self.W_down.float()
        self.M, self.V = torch.zeros_like(self.master), torch.zeros_like(self.master)
        self.t = 0
        # gradients in fixed buffers, listed once for the norm and the clipping
        names = {"T_S": (vocab, d), "W_up": (d_ff, d), "W_down": (d, d_ff), "W_head": (vocab, d),
                 "w0": (d,), "w1": (d,)}
        names.update(self._more(d, d_ff, normal))
        self.grads = {n: torch.zeros(s, device=device) for n, s in names.items()}
        self.list = sn.GradList(self.grads.values())

    def _more(self, d, d_ff, normal):
        """Makes stage 1's further parameters; their shapes."""
        return {}

    # ---- forward -----------------------------------------------------------------------------

    def _stage0(self, ids):
        b = self.basis
        fixed = sn.sn_embed_fwd(self.T_fixed, ids, basis=b)
        low = sn.sn_embed_fwd(self.T_S, ids, basis=b)
        y0, h0 = sn.sn_rmsnorm_fwd(low, self.w0, EPS, R=fixed)       # h0 = fixed + low
        up = torch.relu(y0 @ self.W_up.T)
        return y0, h0, up, h0 + up @ self.W_down.T

    def _boundary(self, x, ids):
        """The residual stream as it arrives: only its k coefficients are sent."""
        n = ids.shape[0]
        C = sn.sn_compress_fwd(self.basis, x, ids, self.T_fixed, n)
        return sn.sn_decompress_fwd(self.basis, C, ids, self.T_fixed, n)

    def _stage1(self, x1):
        """What the head reads, and what the gradient needs."""
        y1, _ = sn.sn_rmsnorm_fwd(x1, self.w1, EPS)
        return y1, (x1,)

    def _stage1_back(self, dy1, x1):
        """The gradient of x1; the parameters' in self.grads."""
        return sn.sn_rmsnorm_bwd(dy1, x1, self.w1, EPS, dw=self.grads["w1"])[0]

    # ---- one step -------------------------------------------------------------------------------

    def backward(self, ids, target):
        """The loss (mean negative log probability of the targets that there are) as a tensor, and
        every gradient in self.grads.  ids, target: int32 [T]; a negative target is none, and so is
        one past the vocabulary, which sn_check_errors reports."""
        g = self.grads
        y0, h0, up, x0 = self._stage0(ids)
        x1 = self._boundary(x0, ids)
        y1, kept = self._stage1(x1)
        logits = y1 @ self.W_head.T
        logp, lse, _, _, _ = sn.sn_logprob_fwd(logits, target, entropy=False, basis=self.basis)
        n = ((target >= 0) & (target < self.vocab)).sum().clamp(min=1).float()
        # back through stage 1; the logits' gradient takes the logits' place
        dlogp = (-1.0 / n).expand(ids.shape[0]).contiguous()
        dlogits = sn.sn_logprob_bwd(logits, lse, target, dlogp, out=logits)
        g["W_head"].copy_(dlogits.T @ y1)
        dx1 = self._stage1_back(dlogits @ self.W_head, *kept)
        # the gradient crosses the boundary the same way
        dx0 = sn.sn_decompress_bwd(self.basis, sn.sn_compress_bwd(self.basis, dx1))
        g["W_down"].copy_(dx0.T @ up)
        dup = (dx0 @ self.W_down) * (up > 0)
        g["W_up"].copy_(dup.T @ y0)
        dh0, _ = sn.sn_rmsnorm_bwd(dup @ self.W_up, h0, self.w0, EPS, dH=dx0, dw=g["w0"])
        sn.sn_embed_bwd(dh0, ids, self.vocab, out=g["T_S"], basis=self.basis)
        return -logp.sum() / n

    def step(self, ids, target, lr=0.5, max_norm=1.0):
        """One training step; returns (loss, gradient norm before clipping) as tensors."""
        loss = self.backward(ids, target)
        norm = sn.sn_grads_clip(self.list, sn.sn_grads_sumsq(self.list), max_norm)
        g, b = self.grads, self.basis
        self.t += 1
        # W_down and T_S stay in S: a rate per column, and a projected update
        sn.sn_adamw_rowconst(self.master, g["W_down"], self.M, self.V, self.t, lr=lr * 1e-2)
        sn.sn_project_weight(b, self.master.to(BF16), out=self.W_down)
        dT = g["T_S"].to(BF16)
        in_S = sn.sn_decompress_bwd(b, sn.sn_compress_bwd(b, dT))
        self.T_S.add_(in_S, alpha=-lr)
        for n in g:
            if n not in ("T_S", "W_down"):
                p = getattr(self, n)
                p.add_(g[n].to(p.dtype), alpha=-lr)
        return loss, norm

    def score(self, ids, top=5):
        """For every position: the log probability of the token that follows (none for the last),
        the entropy and the `top` alternatives."""
        _, _, _, x0 = self._stage0(ids)
        y1 = self._scored(self._boundary(x0, ids))
        target = torch.cat([ids[1:], ids.new_full((1,), -1)])
        logp, _, H, alt, alt_logp = sn.sn_logprob_fwd(y1 @ self.W_head.T, target, top=top)
        return logp, H, alt, alt_logp

    def _scored(self, x1):
        """What the head reads for scores.  It passes through 8 bits (e4m3, a scale a row), to show what
        that does to them; the products themselves are bf16."""
        codes, scale, _ = sn.sn_rmsnorm_fwd_quant(x1, self.w1, EPS, "e4m3")
        return sn.sn_quant_restore(codes, scale, "e4m3")


class GatedTwoStage(TwoStage):
    """Stage 1 with a gated block between two norms: h = x1 + scale gate norm(down(act(gate y1) up y1)),
    y1 = norm(x1), and the head reads norm(h)."""

    act, scale = "silu", 0.5

    def _more(self, d, d_ff, normal):
        self.V_gate, self.V_up = (normal(d_ff, d, std=1 / math.sqrt(d)).to(BF16) for _ in range(2))
        self.V_down = normal(d, d_ff, std=1 / math.sqrt(d_ff)).to(BF16)
        self.w_post, self.w_pre = (torch.ones_like(self.w1) for _ in range(2))
        self.gate = torch.ones(1, d, device=self.w1.device, dtype=BF16)
        return {"V_gate": (d_ff, d), "V_up": (d_ff, d), "V_down": (d, d_ff), "w_post": (d,),
                "w_pre": (d,), "gate": (1, d)}

    def _stage1(self, x1, keep=True):
        y1, _ = sn.sn_rmsnorm_fwd(x1, self.w1, EPS)
        H, G, U = sn.sn_glu_fwd(y1, self.V_gate, self.V_up, self.act, keep=keep, basis=self.basis)
        y = H @ self.V_down.T
        z, h = sn.sn_blocknorm_fwd(y, x1, self.w_post, self.w_pre, EPS, scale=self.scale, gate=self.gate)
        return z, (x1, y1, H, G, U, y, h)

    def _stage1_back(self, dz, x1, y1, H, G, U, y, h):
        g = self.grads
        dy, dx1, _, _, _ = sn.sn_blocknorm_bwd(dz, h, y, self.w_post, self.w_pre, EPS, scale=self.scale,
                                               gate=self.gate, dw_post=g["w_post"], dw_pre=g["w_pre"],
                                               dgate=g["gate"])
        g["V_down"].copy_(dy.T @ H)
        dy1 = sn.sn_glu_bwd(dy @ self.V_down, y1, self.V_gate, self.V_up, G, U, self.act, dG=G, dU=U,
                            dW_gate=g["V_gate"], dW_up=g["V_up"], basis=self.basis)[0]
        return sn.sn_rmsnorm_bwd(dy1, x1, self.w1, EPS, dH=dx1, dw=g["w1"])[0]

    def _scored(self, x1):
        """In 16 bits, as for training; nothing is kept for a gradient."""
        return self._stage1(x1, keep=False)[0]


def chain(T, vocab, seed=0, device="cuda"):
    """Tokens that mostly follow one another by a fixed rule: ids int32 [T] and the next ones."""
    g = torch.Generator().manual_seed(seed)
    step = torch.where(torch.rand(T + 1, generator=g) < 0.9, 1, torch.randint(vocab, (T + 1,), generator=g))
    ids = torch.cumsum(step, 0) % vocab
    return ids[:-1].int().to(device), ids[1:].int().to(device)


def main(steps=60, T=2048, gated=False):
    model = GatedTwoStage() if gated else TwoStage()
    for i in range(steps):
        loss, norm = model.step(*chain(T, model.vocab, seed=i))
        if i % 10 == 0 or i == steps - 1:
            print("step %d: loss %.3f, gradient norm %.3f" % (i, float(loss), float(norm)))
    sn.sn_check_errors(model.basis)
    ids, _ = chain(8, model.vocab, seed=steps)
    logp, H, alt, alt_logp = model.score(ids)
    for t in range(7):
        print("after %4d: next %4d at %6.2f, best %4d at %6.2f, entropy %.2f" % (
            ids[t], ids[t + 1], logp[t], alt[t, 0], alt_logp[t, 0], H[t]))


if __name__ == "__main__":
    main(gated="gated" in sys.argv[1:])
