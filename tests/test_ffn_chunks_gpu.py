"""Products with an epilogue on pairs of CTAs whose sums are made in several pieces (k beyond 2048 in fp32, 4096 with an 8-bit result), in every form; tolerances from test_ffn_gpu.py."""
import pytest
import torch

from test_ffn_gpu import run_product

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("m,n,k,pad", [(1536, 1600, 2176, 0), (1536, 1600, 8320, 8), (1600, 1504, 4224, 0), (1601, 1500, 4224, 3), (1608, 1600, 6272, 8)])
@pytest.mark.parametrize("out", [BF, F32])
@pytest.mark.parametrize("gradient", [False, True])
@pytest.mark.parametrize("parts", [{}, {"c": False, "res": False}, {"q": False}])
def test_pieces(b2, m, n, k, pad, out, gradient, parts):
    run_product(b2, m, n, k, "gelu" if gradient else "silu", gradient=gradient, ta="N" if gradient else "T", out=out, pad=pad, seed=13, **parts)


@pytest.mark.parametrize("m,n,pad", [(1536, 1600, 0), (1601, 1500, 3), (300, 200, 0), (512, 40, 0), (1003, 8, 1)])
@pytest.mark.parametrize("k", [2048, 2049, 4096, 4100, 10000])
def test_integers_are_exact(b2, m, n, k, pad):
    run_product(b2, m, n, k, "none", out=F32, integers=True, q=False, pad=pad, seed=14)
    run_product(b2, m, n, k, "none", out=F32, integers=True, q=True, pad=pad, seed=15)
