"""Operands of the FP8 products, as the binding takes them: what would be read wrongly, or behind its end, is refused (no GPU)."""
import pytest
import torch

from paper_2505_19115_b200 import binding as nb


def _bytes(*size):
    return torch.zeros(size, dtype=torch.uint8)


@pytest.mark.parametrize("lead,R,K", [((), 128, 512), ((), 256, 1024), ((), 4096, 4096), ((), 256, 500), ((3,), 128, 512), ((2,), 384, 2048), ((), 128, 65536)])
def test_linear_scales_are_refused_where_they_take_as_many_bytes(lead, R, K):
    # whole tiles of 128 rows and 4 blocks: only the shape tells linear scales from swizzled ones
    n, codes, b = nb._native(), _bytes(*lead, R, -(-K // 16) * 16)[..., :K], lead[0] if lead else 1
    linear, flat = _bytes(*lead, R, -(-K // 128)), _bytes(b * nb.nvfp4_sf_bytes_fp8(R, K))
    assert linear.numel() == flat.numel()
    assert n.fp8_operand(codes, flat) == (b, R, K)
    larger = _bytes(*lead, 2 * R, -(-K // 128))
    for bad in (linear, larger, linear.view(-1, linear.shape[-1])):
        with pytest.raises(ValueError, match="swizzled"):
            n.fp8_operand(codes, bad)


def test_swizzled_scales_in_whole_tiles_are_taken_whatever_their_shape():
    n, codes = nb._native(), _bytes(3, 200, 528)
    each = nb.nvfp4_sf_bytes_fp8(200, 528)
    for good in (_bytes(3 * each), _bytes(3 * each + 4096), _bytes(3, each), _bytes(3 * each // 512, 512), _bytes(3, each // 512, 512)):
        assert n.fp8_operand(codes, good) == (3, 200, 528)
    for bad in (_bytes(3 * each - 1), _bytes(2, each), torch.tensor(0, dtype=torch.uint8), torch.zeros(3 * each, dtype=torch.int16), _bytes(3, 2 * each)[:, :each]):
        with pytest.raises(ValueError, match="swizzled"):
            n.fp8_operand(codes, bad)


@pytest.mark.parametrize("which", [0, 1])
def test_the_products_refuse_them(which):
    good, linear = (_bytes(256, 512), _bytes(1 * 2 * 512)), (_bytes(256, 512), _bytes(256, 4))
    operands = (good, linear) if which else (linear, good)
    with pytest.raises(ValueError, match="swizzled"):
        nb.nvfp4_gemm_fp8(*operands[0], *operands[1], out=torch.zeros((256, 256)))
