"""The end of a tensor-parallel transformer, R ranks whose buffers lie in this GPU's memory: the last norm, the vocabulary projection and its loss, and their
backward pass.

Rank r holds M / R tokens of the stream and V columns of the vocabulary; model width D:

    forward     S = X + R, a chunk of Y = norm(S)                          flux_norm (X: what flux_gemm_rs left of the last MLP)
                lse, logit over the rank's columns of Y W^T, all tokens    flux_loss (on the gathered chunks)
                the whole vocabulary's lse, every token's loss             flux_loss_join
    backward    the rank's part of dY, dW of its columns                   flux_loss_backward
                a chunk of dY, out of the ranks' parts of it               flux_rs_reduce_slice
                dS, dw of the norm                                         flux_norm_backward

Serving in 4 bits needs no launch between norm and MLP: `Block4Bit`, whose norm writes the blocks that flux_mx4_glu reads.
Run `python examples/loss_head.py` on a GPU for the width of a Llama-2-70B-like model and 32000 columns over 8 ranks.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2406_06858_amd import binding as fb  # noqa: E402
from paper_2406_06858_amd import ffn, loss, norm  # noqa: E402


class LossHead:
    """Plans, workspace and buffers of the ranks, made once and used by every step."""

    def __init__(self, M, D, V, R, eps=1e-5, device="cuda:0"):
        if M < R or M % R:
            raise ValueError(f"{M} tokens cannot be shared out over {R} ranks")
        self.M, self.D, self.V, self.R, self.chunk = M, D, V, R, M // R
        self.norm = norm.norm_problem(self.chunk, D, eps=eps, dw_accumulate=1)
        self.shards = [loss.loss_problem(M, V, D, v0=r * V, vocab=R * V) for r in range(R)]
        self.reduce = [fb.problem(M, D, 8, R, r) for r in range(R)]
        ops = (loss.FLUX_LOSS_FORWARD, loss.FLUX_LOSS_BACKWARD)
        need = max([loss.flux_loss_workspace_bytes(op, p) for op in ops for p in self.shards] + [norm.flux_norm_workspace_bytes(self.norm)])
        self.ws = torch.empty(need, dtype=torch.uint8, device=device)
        ffn.flux_ffn_init(self.ws)
        new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=device)      # noqa: E731
        self.S, self.Y, self.dY, self.dS = (new(M, D, dtype=torch.bfloat16) for _ in range(4))
        self.rstd, self.lse, self.loss, self.dw = new(M), new(M), new(M), new(D)
        self.lses, self.logits = [new(M) for _ in range(R)], [new(M) for _ in range(R)]
        self.parts = [new(M, D, dtype=torch.bfloat16) for _ in range(R)]
        self.dW = [new(V, D, dtype=torch.bfloat16) for _ in range(R)]

    def rows(self, t, r):
        return t[r * self.chunk:(r + 1) * self.chunk]

    def forward(self, X, stream, w, W, target):
        """Every token's loss.  W: the ranks' columns [V,D]."""
        for r in range(self.R):
            norm.flux_norm(self.norm, *(self.rows(t, r) for t in (X, stream)), w, self.rows(self.S, r), self.rows(self.Y, r), None, self.rows(self.rstd, r))
        for r, p in enumerate(self.shards):
            loss.flux_loss(p, self.Y, W[r], target, self.lses[r], self.logits[r], None, self.ws)
        loss.flux_loss_join(self.shards[0], self.lses, self.logits, target, self.lse, None, self.loss)
        return self.loss

    def backward(self, w, W, target, dloss):
        """(dS, dw, the ranks' dW); dloss: the gradient of every token's loss."""
        for r, p in enumerate(self.shards):
            loss.flux_loss_backward(p, self.Y, W[r], target, self.lse, dloss, self.parts[r], self.dW[r], self.ws)
        self.dw.zero_()
        for r, p in enumerate(self.reduce):
            fb.flux_rs_reduce_slice(p, [self.rows(part, r) for part in self.parts], self.rows(self.dY, r))
            norm.flux_norm_backward(self.norm, *(self.rows(t, r) for t in (self.dY, self.S)), w, self.rows(self.rstd, r), None, self.rows(self.dS, r), None,
                                    self.dw, self.ws)
        return self.dS, self.dw, self.dW


class Block4Bit:
    """Residual, norm and the gated up projections for serving, weights in 4-bit blocks (q, scales)."""

    def __init__(self, M, D, N, act="silu", eps=1e-5, device="cuda:0"):
        self.norm, self.glu = norm.norm_problem(M, D, out="mx4", eps=eps), ffn.mx4_problem(M, N, D, act=act)
        self.q = torch.empty(M, ffn.flux_mx4_row_bytes(D), dtype=torch.uint8, device=device)
        self.scales = torch.empty(M, ffn.flux_mx4_scale_row_bytes(D), dtype=torch.uint8, device=device)
        self.H = torch.empty(M, N, dtype=torch.bfloat16, device=device)
        self.ws = torch.empty(max(ffn.flux_mx4_workspace_bytes(ffn.FLUX_MX4_GLU, self.glu), 16), dtype=torch.uint8, device=device)
        ffn.flux_ffn_init(self.ws)

    def __call__(self, X, stream, w, Wg, Wu):
        """H; the stream takes X's addition in place."""
        norm.flux_norm(self.norm, X, stream, w, stream, self.q, self.scales)
        ffn.flux_mx4_glu(self.glu, self.q, self.scales, *Wg, *Wu, self.H, self.ws)
        return self.H


def _timed(f, reps=10):
    for _ in range(3):
        f()
    a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    a.record()
    for _ in range(reps):
        f()
    b.record()
    torch.cuda.synchronize()
    return a.elapsed_time(b) / reps


def main():
    M, D, V, R = 8192, 8192, 4000, 8
    gen = torch.Generator(device="cuda:0").manual_seed(1)
    draw = lambda *shape, std=1.0: (torch.randn(shape, generator=gen, device="cuda:0") * std).to(torch.bfloat16)      # noqa: E731
    X, stream, w, W = draw(M, D), draw(M, D), draw(D), [draw(V, D, std=0.02) for _ in range(R)]
    target = torch.randint(0, R * V, (M,), generator=gen, device="cuda:0")
    dloss = torch.full((M,), 1.0 / M, device="cuda:0")
    head = LossHead(M, D, V, R)
    print(f"{M} tokens, {R} ranks of {V} columns in turn: forward {_timed(lambda: head.forward(X, stream, w, W, target)):.2f} ms, "
          f"backward {_timed(lambda: head.backward(w, W, target, dloss)):.2f} ms")


if __name__ == "__main__":
    main()
