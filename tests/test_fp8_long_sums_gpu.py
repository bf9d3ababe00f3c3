"""Long contractions of the FP8 products are summed in parts: none is left out or counted twice, and the sums stay as close as those of the
longest part.

The tensor core truncates when it adds to its accumulator, so that an error grows with the number of additions: 7.2e-7 of the norm at 86
blocks of 128 normal values, hence 8.1e-7 at 96, the longest part.  Parts are added in fp32 with rounding, at most half a step (6e-8) for
each of a few: 1e-6 in all.  A sum without parts has 1.2e-6 at 128 blocks and more beyond (2.5e-6 at 224, 7.7e-6 at 512)."""
import pytest
import torch

import fp8_reference as ref
from paper_2505_19115_b200 import binding as nb

pytestmark = pytest.mark.gpu
BOUND = 1e-6


def _normal(shape, seed):
    return torch.randn(shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda", dtype=torch.bfloat16)


def _small(shape, seed, most=2):
    """Whole numbers that the format holds; sums of their products stay below 2^24, where every sum is exact."""
    return torch.randint(-most, most + 1, shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda", dtype=torch.int8).to(torch.bfloat16)


def _close(D, want):
    error = float((D.double() - want).norm() / want.norm())
    assert error < BOUND, error
    assert nb.nvfp4_device_error_word() == 0


# Few rows: a block alone with all of the contraction (tiles for every multiprocessor), shared by 2, 4 and 8; one accumulator or two in
# turn; and the tiles of CTA pairs, in each width.
SHAPES = [(1, 9600, 28672), (64, 9600, 28672), (65, 9600, 16384), (128, 9600, 28672), (17, 8192, 28672), (128, 8192, 28672), (3, 4104, 60000),
          (100, 264, 131072), (1, 130, 131072), (300, 600, 16384), (300, 600, 65536), (1100, 3008, 28672), (3000, 3008, 16384)]


@pytest.mark.parametrize("shape", SHAPES)
def test_long_sums_of_normal_values(shape):
    M, N, K = shape
    A, B = _normal((M, K), 1), _normal((N, K), 2)
    a, b = nb.nvfp4_quantize_fp8(A)[:2], nb.nvfp4_quantize_fp8(B)[:2]
    D = nb.nvfp4_gemm_fp8(*a, *b)
    rows = torch.cat([torch.arange(0, min(N, 256)), torch.arange(max(N - 256, 0), N)])        # of B: the whole in 64 bits would take long
    _close(D[:, rows], ref.values(A) @ ref.values(B[rows]).T)


@pytest.mark.parametrize("shape", SHAPES + [(2, 9600, 12288), (2, 9600, 12289), (70, 9600, 12300), (2, 9600, 24577), (90, 9600, 24704)])
def test_long_sums_of_whole_numbers_are_exact(shape):
    M, N, K = shape
    A, B = _small((M, -(-K // 8) * 8), 3)[:, :K], _small((N, -(-K // 8) * 8), 4)[:, :K]
    a, b = nb.nvfp4_quantize_fp8(A)[:2], nb.nvfp4_quantize_fp8(B)[:2]
    D = nb.nvfp4_gemm_fp8(*a, *b)
    want = A.double() @ B.double().T
    assert float(want.abs().max()) < 2 ** 24 and torch.equal(D.double(), want)
    assert nb.nvfp4_device_error_word() == 0


@pytest.mark.parametrize("N", [128, 40])
def test_weight_gradient_of_few_output_features_over_many_tokens(N):
    T, K = 32768, 9600
    X, dY, W = _normal((T, K), 5), _normal((T, N), 6), _normal((N, K), 7)
    _, dW = nb.nvfp4_linear_fp8_bwd(dY, W, X)
    cols = torch.cat([torch.arange(0, 256), torch.arange(K - 256, K)])
    _close(dW[:, cols], ref.values(dY.T) @ ref.values(X[:, cols].T).T)


@pytest.mark.parametrize("counts", [[0, 1, 130, 0, 17], [3, 100, 64, 64, 20]])
@pytest.mark.parametrize("K", [12296, 28672])
def test_long_sums_of_few_rows_of_experts(K, counts):
    E, N = len(counts), 264
    expert_of = torch.repeat_interleave(torch.arange(E), torch.tensor(counts)).int().cuda()[:, None].contiguous()
    plan = nb.nvfp4_expert_sort(expert_of, E)
    for make, check in ((_small, lambda D, want: torch.equal(D.double(), want)), (_normal, lambda D, want: _close(D, want) is None)):
        x, W = make((sum(counts), K), 8), make((E, N, K), 9)
        w = nb.nvfp4_quantize_fp8(W, 128)[:2]
        Y = nb.nvfp4_gemm_fp8_experts(*nb.nvfp4_quantize_fp8_experts(x, plan)[:2], *w, plan)
        for e, n in enumerate(counts):
            begin, first = int(plan.offsets[e]), sum(counts[:e])
            if n:
                assert check(Y[begin:begin + n], ref.values(x[first:first + n]) @ ref.values(W[e], True).T)
    assert nb.nvfp4_device_error_word() == 0
