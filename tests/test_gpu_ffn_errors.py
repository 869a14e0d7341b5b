"""A runtime error that the caller has not fetched yet, from a call of its own before, is neither reported by these operators as theirs nor
taken from the caller.  (The error: an attribute that no device has, asked for from the host.)"""
import ctypes

import pytest
import torch

from paper_2406_06858_amd import ffn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _runtime():
    """The HIP runtime that this process has loaded."""
    torch.cuda.synchronize()
    paths = [line.split()[-1] for line in open("/proc/self/maps") if "libamdhip64" in line]
    return ctypes.CDLL(paths[0])


def _bf16(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).to(DEV)


def _calls():
    """(name, call, outputs) of every entry point that launches, the products on either kernel."""
    out = []
    M, N, K = 40, 64, 96
    x, w = _bf16(1, M, K), [_bf16(i, N, K) for i in (2, 3)]
    g, u, dh = (_bf16(i, M, N) for i in (4, 5, 6))
    new = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=DEV)      # noqa: E731
    blocks = lambda r: [torch.zeros(r, n, dtype=torch.uint8, device=DEV) for n in (ffn.flux_mx4_row_bytes(K), ffn.flux_mx4_scale_row_bytes(K))]      # noqa: E731
    ws = torch.zeros(1 << 22, dtype=torch.uint8, device=DEV)
    out.append(("flux_ffn_init", lambda: ffn.flux_ffn_init(ws), []))
    a, b = blocks(M), [blocks(N) for _ in range(2)]
    out.append(("flux_mx4_quantize", lambda: ffn.flux_mx4_quantize(x, *a), a))
    for q, t in zip(b, w):
        ffn.flux_mx4_quantize(t, *q)
    back = new(M, K)
    out.append(("flux_mx4_dequantize", lambda: ffn.flux_mx4_dequantize(*a, back), [back]))
    for cfg in (0, 1, ffn.flux_ffn_tile_config_count()):
        p, pm, h = ffn.glu_problem(M, N, K, w_is_nk=1, tile_config=cfg), ffn.mx4_problem(M, N, K, tile_config=cfg), [new(M, N) for _ in range(3)]
        out.append((f"flux_glu {cfg}", lambda p=p, h=h: ffn.flux_glu(p, x, *w, h[0], None, None, ws), h[:1]))
        out.append((f"flux_mx4_gemm {cfg}", lambda p=pm, h=h: ffn.flux_mx4_gemm(p, *a, *b[0], h[1], ws), h[1:2]))
        out.append((f"flux_mx4_glu {cfg}", lambda p=pm, h=h: ffn.flux_mx4_glu(p, *a, *b[0], *b[1], h[2], ws), h[2:]))
    grads = [new(M, K), new(N, K), new(N, K)]
    pb = ffn.glu_problem(M, N, K, w_is_nk=1)
    out.append(("flux_glu_backward", lambda: ffn.flux_glu_backward(pb, x, *w, g, u, dh, *grads, ws), grads))
    return out


def test_an_earlier_error_of_the_caller_stays_its_own():
    calls = _calls()
    for _, call, _ in calls:
        call()
    torch.cuda.synchronize()
    want = [[t.clone() for t in outs] for _, _, outs in calls]
    hip, value = _runtime(), ctypes.c_int()
    for (name, call, outs), ref in zip(calls, want):
        for t in outs:
            t.fill_(77)
        error = hip.hipDeviceGetAttribute(ctypes.byref(value), 999999, 0)
        try:
            assert error != 0 and hip.hipPeekAtLastError() == error
            call()
            assert hip.hipPeekAtLastError() == error, name
        finally:
            hip.hipGetLastError()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, ref)), name
