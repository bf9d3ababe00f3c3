"""Tensors that an FP8 or expert call cannot take are refused with an error that names the call, also where Python runs without
assertions: a kernel would read or write behind a buffer that is too small (no GPU)."""
import subprocess
import sys

import pytest
import torch

from paper_2505_19115_b200 import binding as nb

T, TOPK, E, N, K = 5, 2, 3, 24, 40
R = nb.nvfp4_expert_rows(T, TOPK, E)


def _z(*size, dtype=torch.float32):
    return torch.zeros(size, dtype=dtype)


def _codes(*size):
    return torch.zeros(*size[:-1], -(-size[-1] // 16) * 16, dtype=torch.uint8)[..., :size[-1]]


def _sf(rows, cols, matrices=1):
    return torch.zeros(matrices * nb.nvfp4_sf_bytes_fp8(rows, cols), dtype=torch.uint8)


PLAN = nb.ExpertPlan(T, TOPK, E, torch.zeros(1))
OTHER = nb.ExpertPlan(T + 1, TOPK, E, torch.zeros(1))
A, B = (_codes(8, K), _sf(8, K)), (_codes(N, K), _sf(N, K))
ROWS, WE = (_codes(R, K), _sf(R, K)), (_codes(E, N, K), _sf(N, K, E))
DT, XT = (_codes(N, R), _sf(N, R)), (_codes(K, R), _sf(K, R))
X, W, DY, WX = _z(8, K), _z(N, K), _z(8, N), _z(E, N, K)

BAD = [
    ("nvfp4_gemm_fp8", lambda: nb.nvfp4_gemm_fp8(*A, _codes(N, K + 16), _sf(N, K + 16))),
    ("nvfp4_gemm_fp8", lambda: nb.nvfp4_gemm_fp8(*A, *WE)),
    ("nvfp4_gemm_fp8", lambda: nb.nvfp4_gemm_fp8(*A, *B, out=_z(7, N))),
    ("nvfp4_gemm_fp8", lambda: nb.nvfp4_gemm_fp8(*A, *B, out=_z(8, N + 1))),
    ("nvfp4_gemm_fp8", lambda: nb.nvfp4_gemm_fp8(*A, *B, out=_z(N, 8).T)),
    ("nvfp4_linear_fp8_fwd", lambda: nb.nvfp4_linear_fp8_fwd(X, _z(N, K + 8))),
    ("nvfp4_linear_fp8_fwd", lambda: nb.nvfp4_linear_fp8_fwd(X, W.to(torch.bfloat16))),
    ("nvfp4_linear_fp8_fwd", lambda: nb.nvfp4_linear_fp8_fwd(X, W, out=_z(7, N))),
    ("nvfp4_linear_fp8_fwd", lambda: nb.nvfp4_linear_fp8_fwd(_z(8, 2 * K)[:, :K], W)),
    ("nvfp4_linear_fp8_bwd", lambda: nb.nvfp4_linear_fp8_bwd(DY, W, _z(7, K))),
    ("nvfp4_linear_fp8_bwd", lambda: nb.nvfp4_linear_fp8_bwd(DY, _z(N + 8, K), X)),
    ("nvfp4_linear_fp8_bwd", lambda: nb.nvfp4_linear_fp8_bwd(DY, W, X, dX=_z(8, K - 8))),
    ("nvfp4_linear_fp8_bwd", lambda: nb.nvfp4_linear_fp8_bwd(DY, W, X, dW=_z(K, N))),
    ("nvfp4_expert_sort", lambda: nb.nvfp4_expert_sort(_z(TOPK, T, dtype=torch.int32).T, E)),
    ("nvfp4_expert_sort", lambda: nb.nvfp4_expert_sort(_z(T, TOPK, dtype=torch.int32), E, OTHER)),
    ("nvfp4_expert_sort", lambda: nb.nvfp4_expert_sort(_z(T, TOPK, dtype=torch.int32), E + 1, PLAN)),
    ("nvfp4_expert_gather", lambda: nb.nvfp4_expert_gather(_z(T, K), PLAN, out=_z(R - 1, K))),
    ("nvfp4_expert_gather", lambda: nb.nvfp4_expert_gather(_z(T, K), PLAN, out=_z(R, K, dtype=torch.bfloat16))),
    ("nvfp4_expert_gather", lambda: nb.nvfp4_expert_gather(_z(T, K), PLAN, _z(T, TOPK - 1))),
    ("nvfp4_expert_combine", lambda: nb.nvfp4_expert_combine(_z(R, 2 * K)[:, :K], PLAN)),
    ("nvfp4_expert_combine", lambda: nb.nvfp4_expert_combine(_z(R, K), PLAN, out=_z(T - 1, K))),
    ("nvfp4_expert_combine", lambda: nb.nvfp4_expert_combine(_z(R, K), PLAN, _z(T * TOPK))),
    ("nvfp4_expert_combine_bwd", lambda: nb.nvfp4_expert_combine_bwd(_z(T, K), _z(R - 128, K), PLAN, _z(T, TOPK))),
    ("nvfp4_expert_combine_bwd", lambda: nb.nvfp4_expert_combine_bwd(_z(T, K), _z(R, K), PLAN, _z(T - 1, TOPK))),
    ("nvfp4_expert_combine_bwd", lambda: nb.nvfp4_expert_combine_bwd(_z(T, K), _z(R, K), PLAN, _z(T, TOPK), drows=_z(R, K - 8))),
    ("nvfp4_expert_combine_bwd", lambda: nb.nvfp4_expert_combine_bwd(_z(T, K), _z(R, K), PLAN, _z(T, TOPK), dweights=_z(T, TOPK, dtype=torch.bfloat16))),
    ("nvfp4_quantize_fp8_experts", lambda: nb.nvfp4_quantize_fp8_experts(_z(T, K), PLAN, _z(T, TOPK + 1))),
    ("nvfp4_gemm_fp8_experts", lambda: nb.nvfp4_gemm_fp8_experts(*ROWS, *WE, OTHER) if OTHER.rows != R else nb.nvfp4_gemm_fp8_experts(*A, *WE, PLAN)),
    ("nvfp4_gemm_fp8_experts", lambda: nb.nvfp4_gemm_fp8_experts(*ROWS, _codes(E - 1, N, K), _sf(N, K, E), PLAN)),
    ("nvfp4_gemm_fp8_experts", lambda: nb.nvfp4_gemm_fp8_experts(*ROWS, *WE, PLAN, out=_z(R - 1, N))),
    ("nvfp4_gemm_fp8_experts_dw", lambda: nb.nvfp4_gemm_fp8_experts_dw(*DT, _codes(K, R - 128), _sf(K, R), PLAN)),
    ("nvfp4_gemm_fp8_experts_dw", lambda: nb.nvfp4_gemm_fp8_experts_dw(*DT, *XT, PLAN, out=_z(E, N, K - 8))),
    ("nvfp4_gemm_fp8_experts_dw", lambda: nb.nvfp4_gemm_fp8_experts_dw(*DT, *XT, PLAN, out=_z(E, K, N).transpose(1, 2))),
    ("nvfp4_experts_fp8_fwd", lambda: nb.nvfp4_experts_fp8_fwd(_z(T + 1, K), WX, PLAN)),
    ("nvfp4_experts_fp8_fwd", lambda: nb.nvfp4_experts_fp8_fwd(_z(T, K), _z(E + 1, N, K), PLAN)),
    ("nvfp4_experts_fp8_fwd", lambda: nb.nvfp4_experts_fp8_fwd(_z(T, K), WX, PLAN, sorted_rows=True)),
    ("nvfp4_experts_fp8_fwd", lambda: nb.nvfp4_experts_fp8_fwd(_z(T, K), WX, PLAN, out=_z(R - 1, N))),
    ("nvfp4_experts_fp8_bwd", lambda: nb.nvfp4_experts_fp8_bwd(_z(T - 1, N), WX, _z(T, K), PLAN)),
    ("nvfp4_experts_fp8_bwd", lambda: nb.nvfp4_experts_fp8_bwd(_z(T, N), WX, _z(T, K + 8), PLAN)),
    ("nvfp4_experts_fp8_bwd", lambda: nb.nvfp4_experts_fp8_bwd(_z(T, N), WX, _z(T, K), PLAN, weights=_z(T - 1, TOPK))),
    ("nvfp4_experts_fp8_bwd", lambda: nb.nvfp4_experts_fp8_bwd(_z(T, N), WX, _z(T, K), PLAN, dX=_z(R - 128, K))),
    ("nvfp4_experts_fp8_bwd", lambda: nb.nvfp4_experts_fp8_bwd(_z(T, N), WX, _z(T, K), PLAN, dW=_z(E - 1, N, K))),
]


@pytest.mark.parametrize("i", range(len(BAD)))
def test_refused_with_the_name_of_the_call(i):
    name, call = BAD[i]
    with pytest.raises(ValueError, match=f"^{name}: "):
        call()


def test_refused_without_assertions_too():
    # this file's cases once more, in an interpreter that drops assert statements
    done = subprocess.run([sys.executable, "-O", "-c", "import test_fp8_refusals as t; t.run_all()"], cwd=__file__.rsplit("/", 1)[0], capture_output=True, text=True,
                          env={**__import__("os").environ, "PYTHONPATH": __file__.rsplit("/", 2)[0]})
    assert done.returncode == 0 and done.stdout.split() == [str(len(BAD)), "refused"], done.stdout + done.stderr


def run_all():
    refused = 0
    for name, call in BAD:
        try:
            call()
        except ValueError as e:
            refused += str(e).startswith(name + ": ")
        except Exception:                            # the next check, in the extension module: not the one that is meant
            pass
    print(refused, "refused")
