"""The experts' products with contractions that are summed in parts: weight gradients over more than 12288 rows, and forward products
and input gradients of more than 12288 features, in tiles of every width.  Whole numbers, whose sums are exact, and the norm of the error
on normal values (test_fp8_long_sums_gpu.py has the bound's reason)."""
import pytest
import torch

import fp8_reference as ref
from paper_2505_19115_b200 import binding as nb
from test_fp8_long_sums_gpu import _close, _normal, _small

pytestmark = pytest.mark.gpu


def _plan(counts, seed):
    """A plan with so many rows for each expert, their tokens in any order."""
    order = torch.randperm(sum(counts), generator=torch.Generator().manual_seed(seed))
    expert_of = torch.repeat_interleave(torch.arange(len(counts)), torch.tensor(counts))[order].int().cuda()[:, None].contiguous()
    plan = nb.nvfp4_expert_sort(expert_of, len(counts))
    assert plan.counts.tolist() == counts
    return plan


def _segments(plan):
    return [(e, int(plan.offsets[e]), c) for e, c in enumerate(plan.counts.tolist())]


# all short; one beyond 12288 that begins at block 1, 2, 3 and 0 of a scale tile; at its ends; with empty ones between; several parts
COUNTS = [[300] * 45, [100, 13000, 0, 200], [130, 14000, 5], [300, 0, 25000, 1, 0], [12288, 12289, 1], [0, 0, 40000], [12416, 0, 300, 24577]]


@pytest.mark.parametrize("N,K", [(264, 136), (200, 2056), (256, 2816)])       # with five experts: tiles of 128, 192 and 256 columns
@pytest.mark.parametrize("counts", COUNTS)
def test_weight_gradient_over_long_and_short_segments(counts, N, K):
    plan, T = _plan(counts, 1), sum(counts)
    assert plan.rows > 12288
    row_slot = plan.slot_of.long()
    for make, whole in ((_small, True), (_normal, False)):
        x, dy = make((T, K), 2), make((T, N), 3)
        xt, dyt = (nb.nvfp4_quantize_fp8_experts(t, plan, row=False, transposed=True)[2:] for t in (x, dy))
        dW = torch.full((len(counts), N, K), 5.0, device="cuda")
        nb.nvfp4_gemm_fp8_experts_dw(*dyt, *xt, plan, out=dW)
        for e, begin, n in _segments(plan):
            tokens = row_slot[begin:begin + n]
            if n == 0:
                assert not bool(dW[e].any())
            elif whole:
                assert torch.equal(dW[e].double(), dy[tokens].double().T @ x[tokens].double())
            else:
                _close(dW[e], ref.values(dy[tokens].T) @ ref.values(x[tokens].T).T)
    assert nb.nvfp4_device_error_word() == 0


@pytest.mark.parametrize("out_features", [136, 2056, 2816])
@pytest.mark.parametrize("contraction", [12296, 16384, 28672])
@pytest.mark.parametrize("counts", [[300, 0, 129, 700], [1000, 150]])
def test_layer_of_experts_with_a_long_contraction(counts, contraction, out_features):
    plan, T, E = _plan(counts, 4), sum(counts), len(counts)
    row_slot = plan.slot_of.long()
    for make, whole in ((_small, True), (_normal, False)):
        x, W = make((T, contraction), 5), make((E, out_features, contraction), 6)
        Y = nb.nvfp4_experts_fp8_fwd(x, W, plan, out_dtype=torch.float32)
        for e, begin, n in _segments(plan):
            if n:
                tokens, rows = row_slot[begin:begin + n], torch.arange(0, out_features, max(out_features // 256, 1), device="cuda")
                if whole:
                    assert torch.equal(Y[begin:begin + n].double(), x[tokens].double() @ W[e].double().T)
                else:
                    _close(Y[begin:begin + n][:, rows], ref.values(x[tokens]) @ ref.values(W[e], True)[rows].T)
    assert nb.nvfp4_device_error_word() == 0


def test_input_gradient_with_a_long_contraction():
    counts, N, K = [300, 0, 700], 16384, 264
    plan, T = _plan(counts, 7), sum(counts)
    x, dy, W = _small((T, K), 8), _small((T, N), 9), _small((3, N, K), 10)
    dX, dW = nb.nvfp4_experts_fp8_bwd(dy, W, x, plan, dx_dtype=torch.float32)
    for e, begin, n in _segments(plan):
        tokens = plan.slot_of.long()[begin:begin + n]
        assert torch.equal(dX[begin:begin + n].double(), dy[tokens].double() @ W[e].double())
        assert torch.equal(dW[e].double(), dy[tokens].double().T @ x[tokens].double())
    assert nb.nvfp4_device_error_word() == 0
