"""One tensor-parallel rank's gated MLP, trained and served.

Training (bf16), tokens M, model width D, hidden columns N of this rank, R ranks whose buffers lie in this GPU's memory:

    forward     H = act(X Wg) * (X Wu)                        flux_glu, which keeps G and U
                Y[r] = rows of (H Wd + the peers' partials)    flux_gemm_rs
    backward    dH = (the ranks' dY, gathered) Wd^T           flux_ag_gemm
                dX, dWg, dWu                                   flux_glu_backward (dX: this rank's partial)

Serving (4 bits, weights quantised once):

    X -> flux_mx4_quantize -> flux_mx4_glu -> flux_mx4_quantize -> flux_mx4_gemm -> this rank's partial of Y in fp32

Weights are laid out as linear layers store them: Wg, Wu [N,D] and the down projection as Wd [N,D] (in features by out features).
Run `python examples/gated_mlp.py` on a GPU for the shapes of a Llama-2-70B-like layer at TP=8.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2406_06858_amd import binding as fb  # noqa: E402
from paper_2406_06858_amd import ffn  # noqa: E402


def _bytes(n, device):
    return torch.zeros(max(n, 16), dtype=torch.uint8, device=device)


class GatedMlp:
    """Plans, workspaces and buffers of one rank, made once and used by every step."""

    def __init__(self, M, D, N, R, rank, act="silu", device="cuda:0"):
        self.M, self.D, self.N, self.R, self.rank = M, D, N, R, rank
        self.glu = ffn.glu_problem(M, N, D, act=act, w_is_nk=1)
        self.down = fb.problem(M, D, N, R, rank)                                # Y = H Wd
        self.up_t = fb.problem(M, N, D, R, rank, b_is_nk=1)                     # dH = dY Wd^T
        self.ws = _bytes(max(ffn.flux_glu_workspace_bytes(op, self.glu) for op in (ffn.FLUX_GLU_FORWARD, ffn.FLUX_GLU_BACKWARD)), device)
        ffn.flux_ffn_init(self.ws)
        self.ws_rs = _bytes(fb.flux_workspace_bytes(fb.FLUX_OP_RS, self.down), device)
        self.ws_ag = _bytes(fb.flux_workspace_bytes(fb.FLUX_OP_AG, self.up_t), device)
        self.signals = torch.zeros(R, dtype=torch.int32, device=device)
        if fb.flux_workspace_bytes(fb.FLUX_OP_RS, self.down):
            fb.flux_init_buffers(fb.FLUX_OP_RS, self.down, self.ws_rs)
        fb.flux_init_buffers(fb.FLUX_OP_AG, self.up_t, self.ws_ag, self.signals)
        self.copy_stream = torch.cuda.Stream()
        new = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device=device)      # noqa: E731
        self.H, self.G, self.U, self.dH = (new(M, N) for _ in range(4))
        self.dY, self.dX = new(M, D), new(M, D)
        self.dWg, self.dWu = new(N, D), new(N, D)
        self.Y = [new(M // R, D) for _ in range(R)]

    def forward(self, X, Wg, Wu, Wd, peers):
        """The R row slices of Y.  `peers`: the other ranks' partials [M,D], None in this rank's place."""
        ffn.flux_glu(self.glu, X, Wg, Wu, self.H, self.G, self.U, self.ws)
        fb.flux_gemm_rs(self.down, self.H, Wd, peers, self.Y, self.ws_rs)
        return self.Y

    def backward(self, X, Wg, Wu, Wd, dY_chunks):
        """(dX, dWg, dWu) from the ranks' row slices of dY."""
        fb.flux_ag_gemm(self.up_t, dY_chunks, self.dY, Wd, self.dH, self.signals, None, self.ws_ag, torch.cuda.current_stream(), self.copy_stream)
        ffn.flux_glu_backward(self.glu, X, Wg, Wu, self.G, self.U, self.dH, self.dX, self.dWg, self.dWu, self.ws)
        return self.dX, self.dWg, self.dWu


class Mx4:
    """A matrix in 4-bit blocks along its rows."""

    def __init__(self, rows, K, device="cuda:0"):
        self.q = torch.empty(rows, ffn.flux_mx4_row_bytes(K), dtype=torch.uint8, device=device)
        self.scales = torch.empty(rows, ffn.flux_mx4_scale_row_bytes(K), dtype=torch.uint8, device=device)

    def fill(self, x):
        ffn.flux_mx4_quantize(x, self.q, self.scales)
        return self

    def read(self, K, dtype=torch.float32):
        out = torch.empty(self.q.shape[0], K, dtype=dtype, device=self.q.device)
        ffn.flux_mx4_dequantize(self.q, self.scales, out)
        return out


class GatedMlp4Bit:
    """The same block for serving: weights quantised once, activations on the way."""

    def __init__(self, M, Wg, Wu, Wd, act="silu"):
        (N, D), device = Wg.shape, Wg.device
        self.up, self.down = ffn.mx4_problem(M, N, D, act=act), ffn.mx4_problem(M, D, N, out_dtype="f32")
        self.Wg, self.Wu = (Mx4(N, D, device).fill(w) for w in (Wg, Wu))
        self.Wd = Mx4(D, N, device).fill(Wd.t().contiguous())                   # (blocks lie along the contraction)
        self.ws = _bytes(max(ffn.flux_mx4_workspace_bytes(ffn.FLUX_MX4_GLU, self.up), ffn.flux_mx4_workspace_bytes(ffn.FLUX_MX4_GEMM, self.down)), device)
        ffn.flux_ffn_init(self.ws)
        self.X, self.H4 = Mx4(M, D, device), Mx4(M, N, device)
        self.H = torch.empty(M, N, dtype=torch.bfloat16, device=device)
        self.Y = torch.empty(M, D, dtype=torch.float32, device=device)

    def __call__(self, X):
        self.X.fill(X)
        ffn.flux_mx4_glu(self.up, self.X.q, self.X.scales, self.Wg.q, self.Wg.scales, self.Wu.q, self.Wu.scales, self.H, self.ws)
        self.H4.fill(self.H)
        ffn.flux_mx4_gemm(self.down, self.H4.q, self.H4.scales, self.Wd.q, self.Wd.scales, self.Y, self.ws)
        return self.Y


def _timed(f, reps=20):
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
    M, D, N, R, rank = 4096, 8192, 3584, 8, 3
    gen = torch.Generator(device="cuda:0").manual_seed(1)
    draw = lambda *shape, std=1.0: (torch.randn(shape, generator=gen, device="cuda:0") * std).to(torch.bfloat16)      # noqa: E731
    X, Wg, Wu, Wd = draw(M, D), draw(N, D, std=0.02), draw(N, D, std=0.02), draw(N, D, std=0.02)
    peers = [None if r == rank else draw(M, D) for r in range(R)]
    chunks = [draw(M // R, D) for _ in range(R)]
    mlp = GatedMlp(M, D, N, R, rank)
    print(f"training, {M} tokens: forward {_timed(lambda: mlp.forward(X, Wg, Wu, Wd, peers)):.3f} ms, "
          f"backward {_timed(lambda: mlp.backward(X, Wg, Wu, Wd, chunks)):.3f} ms")
    for m in (1, 64, 4096):
        serve = GatedMlp4Bit(m, Wg, Wu, Wd)
        x = X[:m]
        print(f"serving in 4 bits, {m} tokens: {1e3 * _timed(lambda: serve(x)):.1f} us")


if __name__ == "__main__":
    main()
