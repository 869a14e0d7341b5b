"""Long contractions on the kernel for few rows in 4 bits, whose scales come for 8192 numbers at a time into two places in turn; and gradients
that are added to what the buffers hold where the tiles are cut along the tokens.  Bounds as in test_gpu_mx4 and test_gpu_glu."""
import pytest
from test_gpu_glu import _backward, _check_backward
from test_gpu_mx4 import _check_gemm, _check_glu, _gemm, _packed

from paper_2406_06858_amd import ffn

pytestmark = pytest.mark.gpu
FEW = ffn.flux_ffn_tile_config_count()


@pytest.mark.parametrize("M,N,K", [
    (1, 40, 8193), (16, 72, 16384), (7, 24, 33000), (17, 40, 8224), (32, 72, 24640), (33, 40, 16385), (64, 264, 24608), (64, 16, 41000),
    (1, 4104, 8224), (20, 4104, 16416), (64, 4104, 8256),
])
def test_chunks_of_scales(M, N, K):
    (a, va), (b, vb) = _packed(M, K, 21), _packed(N, K, 22, 0.1)
    _check_gemm(_gemm(a, b, M, N, K, "f32", tile_config=FEW), va, vb, "f32")


@pytest.mark.parametrize("M,N,K", [(1, 40, 8193), (16, 72, 16416), (24, 40, 24640), (64, 72, 8224), (50, 24, 33000)])
def test_chunks_of_scales_of_a_gated_product(M, N, K):
    _check_glu(M, N, K, "silu", "f32", 0, tile_config=FEW)


@pytest.mark.parametrize("nk", [0, 1])
@pytest.mark.parametrize("M,N,K,split", [(4096, 256, 256, 0), (2048, 264, 136, 8), (1032, 712, 264, 3), (520, 72, 72, 16)])
def test_accumulated_gradients_of_cut_tiles(M, N, K, split, nk):
    whole, cut = (ffn.flux_glu_workspace_bytes(ffn.FLUX_GLU_BACKWARD, ffn.glu_problem(M, N, K, w_is_nk=nk, split_k=s)) for s in (1, split))
    assert cut > whole, "sums of parts in the workspace"
    for dw in ("bf16", "f32"):
        _check_backward(*_backward(M, N, K, "silu", nk, dw=dw, accumulate=1, seed=61, want_x=False, split_k=split), "silu", dw=dw, start=7.0)
