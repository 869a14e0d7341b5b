"""CPU-only: which products of few rows the library gives to cut tiles.  The kernel for few rows wants no workspace and cut tiles do, so
the workspace tells them apart.  The products are ones where either is far ahead (1.35 times and more, measured)."""
import pytest

from paper_2406_06858_amd import ffn


def _bytes(kind, M, N, K, **choice):
    if kind == "glu":
        return ffn.flux_glu_workspace_bytes(ffn.FLUX_GLU_FORWARD, ffn.glu_problem(M, N, K, w_is_nk=1, **choice))
    return ffn.flux_mx4_workspace_bytes(ffn.FLUX_MX4_GLU if kind == "mx4_glu" else ffn.FLUX_MX4_GEMM, ffn.mx4_problem(M, N, K, **choice))


@pytest.mark.parametrize("kind,M,N,K", [
    ("glu", 16, 256, 8192), ("glu", 64, 256, 8192), ("glu", 1, 256, 12288), ("glu", 32, 256, 12288), ("glu", 64, 1024, 8192), ("glu", 16, 1024, 12288),
    ("glu", 64, 1024, 12288), ("glu", 48, 64, 28672), ("mx4_glu", 64, 256, 12288),
])
def test_few_columns_over_a_long_contraction_are_cut(kind, M, N, K):
    assert _bytes(kind, M, N, K) > 0
    # named, or without a cut, it is the kernel for few rows or whole tiles: no workspace
    assert _bytes(kind, M, N, K, tile_config=ffn.flux_ffn_tile_config_count()) == 0 and _bytes(kind, M, N, K, split_k=1) == 0


@pytest.mark.parametrize("kind,M,N,K", [
    ("glu", 1, 3584, 8192), ("glu", 8, 3584, 2048), ("glu", 1, 256, 2048), ("glu", 16, 1024, 512), ("mx4_gemm", 8, 8192, 3584), ("mx4_gemm", 1, 256, 8192),
    ("mx4_gemm", 64, 3584, 8192), ("mx4_gemm", 16, 1024, 12288), ("mx4_glu", 1, 3584, 8192), ("mx4_glu", 16, 1024, 8192),
])
def test_other_products_of_few_rows_are_not(kind, M, N, K):
    assert _bytes(kind, M, N, K) == 0
