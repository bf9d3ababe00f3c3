"""FP8 with a power-of-two scale for each block of 128: the quantizer bit for bit, products within the rounding of fp32 sums, the
linear layer, kept weights, special values, strides, streams and captured graphs."""
import pytest
import torch

import fp8_reference as ref
from paper_2505_19115_b200 import binding as nb
from paper_2505_19115_b200 import synth
from util import canaries_intact, guarded_u8

pytestmark = pytest.mark.gpu


def _x(shape, seed, dtype=torch.bfloat16, spread=12):
    """Normal values, rows and columns of very different size."""
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn(shape, generator=g, device="cuda")
    for d in (-1, -2):
        e = torch.randint(-spread, spread + 1, [n if i == len(shape) + d else 1 for i, n in enumerate(shape)], generator=g, device="cuda")
        x = x * torch.exp2(e.float())
    return x.to(dtype)


def _check_quantized(x, block_rows, sf_layout, codes, scales, codes_t, scales_t):
    square = block_rows == 128
    for src, c, s in ((x, codes, scales), (x.T, codes_t, scales_t)):
        if c is None:
            continue
        y, e = ref.codes_and_exponents(src, square)
        assert torch.equal(c, ref.code_bytes(y))
        want = ref.scale_bytes(e).cpu()
        if sf_layout == nb.SF_SWIZZLED:
            assert torch.equal(s.cpu(), torch.from_numpy(ref.swizzled(want)))
        else:
            assert torch.equal(s.cpu(), want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("sf_layout", [nb.SF_LINEAR, nb.SF_SWIZZLED])
@pytest.mark.parametrize("shape", [(1, 1), (1, 8), (200, 3), (7, 130), (128, 128), (129, 136), (300, 1031), (513, 640), (16, 2056)])
def test_quantizer_matches_the_definition(shape, sf_layout, block_rows, dtype):
    rows, cols = shape
    x = _x((rows, -(-cols // 8) * 8), rows + cols, dtype)[:, :cols]
    for row, transposed in ((True, True), (True, False), (False, True)):
        out = nb.nvfp4_quantize_fp8(x, block_rows, row, transposed, sf_layout)
        _check_quantized(x, block_rows, sf_layout, *out)


def test_quantizer_of_a_batch_and_of_a_strided_matrix():
    x = _x((3, 200, 328), 1)
    codes, scales, codes_t, scales_t = nb.nvfp4_quantize_fp8(x, 128, True, True)
    each = scales.numel() // 3, scales_t.numel() // 3
    for b in range(3):
        _check_quantized(x[b], 128, nb.SF_SWIZZLED, codes[b], scales[b * each[0]:(b + 1) * each[0]], codes_t[b], scales_t[b * each[1]:(b + 1) * each[1]])
    wide = _x((260, 512), 2)
    part = wide[:, 128:128 + 200]
    _check_quantized(part, 1, nb.SF_LINEAR, *nb.nvfp4_quantize_fp8(part, 1, True, True, nb.SF_LINEAR))


def test_quantizer_writes_nothing_else():
    x = _x((131, 264), 3)
    rows, cols = x.shape
    bufs = [guarded_u8(n) for n in (nb.nvfp4_codes_bytes_fp8(rows, cols), nb.nvfp4_sf_bytes_fp8(rows, cols),
                                    nb.nvfp4_codes_bytes_fp8(cols, rows), nb.nvfp4_sf_bytes_fp8(cols, rows))]
    st = nb._native().nvfp4_quantize_fp8(x, x, 1, rows, cols, cols, 1, *[v for _, v in bufs], nb.SF_SWIZZLED, None)
    assert st == 0
    torch.cuda.synchronize()
    assert all(canaries_intact(w) for w, _ in bufs)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantizer_of_special_values(dtype):
    x = torch.zeros((256, 256), dtype=torch.float32, device="cuda")
    x[0, :6] = torch.tensor([448.0, 432.0, 440.0, -424.0, 0.001953125, 0.0009765625])    # scale 1, ties, the smallest code and half of it
    x[1, 0] = 449.0 if dtype == torch.float32 else 450.0                                    # just above: scale 2
    x[2, 0] = 3.3e38
    x[3, :2] = torch.tensor([1e-38, -1e-40])                                                # near and below the smallest normal number
    x[4, 7] = -0.0
    x[5, 200] = 1.75
    x[6, 0] = 2.0 ** -126
    x = x.to(dtype)
    _check_quantized(x, 1, nb.SF_LINEAR, *nb.nvfp4_quantize_fp8(x, 1, True, True, nb.SF_LINEAR))
    _check_quantized(x, 128, nb.SF_LINEAR, *nb.nvfp4_quantize_fp8(x, 128, True, True, nb.SF_LINEAR))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_non_finite_blocks_are_nan_and_reach_the_product(bad, dtype):
    x = torch.ones((130, 264), dtype=dtype, device="cuda")
    x[3, 140] = bad
    codes, scales, codes_t, scales_t = nb.nvfp4_quantize_fp8(x, 1, True, True, nb.SF_LINEAR)
    assert scales[3, 1] == 255 and scales_t[140, 0] == 255
    assert int((scales == 255).sum()) == 1 and int((scales_t == 255).sum()) == 1
    assert bool((codes[3, 128:256] & 127 == 127).all()) and not bool((codes[3, :128] & 127 == 127).any())
    w = torch.ones((16, 264), dtype=dtype, device="cuda")
    c, s, _, _ = nb.nvfp4_quantize_fp8(x)
    wc, ws, _, _ = nb.nvfp4_quantize_fp8(w, 128)
    D = nb.nvfp4_gemm_fp8(c, s, wc, ws)
    assert bool(D[3].isnan().all()) and int(D.isnan().any(1).sum()) == 1
    assert nb.nvfp4_device_error_word() == 0


def _operands(M, N, K, seed, square=True):
    # the last dimension of a source row is padded to 8 elements where the size is odd
    a = _x((M, -(-K // 8) * 8), seed, spread=4)[:, :K]
    b = _x((N, -(-K // 8) * 8), seed + 1, spread=4)[:, :K]
    ac, asf, _, _ = nb.nvfp4_quantize_fp8(a)
    bc, bsf, _, _ = nb.nvfp4_quantize_fp8(b, 128 if square else 1)
    return (ac, asf, bc, bsf), ref.values(a), ref.values(b, square)


def test_product_of_one_hot_rows_reads_back_the_other_operand():
    # a row of A with a single value selects a column of dequantized B: any mistake in the scales' places shows exactly
    M, N, K = 300, 520, 1160
    a = torch.zeros((M, K), device="cuda")
    at = (torch.arange(M, device="cuda") * 37) % K
    a[torch.arange(M), at] = torch.exp2((torch.arange(M, device="cuda") % 5).float())
    b = _x((N, K), 5)
    for square in (1, 128):
        ac, asf, _, _ = nb.nvfp4_quantize_fp8(a)
        bc, bsf, _, _ = nb.nvfp4_quantize_fp8(b, square)
        D = nb.nvfp4_gemm_fp8(ac, asf, bc, bsf)
        want = (ref.values(b, square == 128)[:, at] * a[torch.arange(M), at].double()).T
        assert torch.equal(D.double(), want)
    assert nb.nvfp4_device_error_word() == 0


SHAPES = [(1, 8, 8), (1, 16, 128), (2, 264, 1000), (16, 512, 4096), (128, 128, 32), (130, 136, 320), (257, 392, 1056), (384, 520, 2081),
          (1000, 1000, 17), (512, 1024, 512), (2500, 2600, 256), (33, 4096, 640), (128, 256, 16384), (5000, 4104, 130)]


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", SHAPES)
def test_product_is_within_the_rounding_of_its_sums(shape, out_dtype):
    M, N, K = shape
    ops, a, b = _operands(M, N, K, M + N)
    D = nb.nvfp4_gemm_fp8(*ops, out_dtype=out_dtype)
    torch.cuda.synchronize()
    assert nb.nvfp4_device_error_word() == 0
    ref.assert_product(D, *ref.product(a, b), K)


@pytest.mark.parametrize("shape", [(1, 8, 64), (64, 72, 200), (300, 1000, 700), (4000, 2048, 384), (9500, 264, 1056)])
def test_product_of_small_integers_is_exact(shape):
    M, N, K = shape
    g = torch.Generator("cuda").manual_seed(M)
    a, b = (torch.randint(-2, 3, (r, -(-K // 8) * 8), generator=g, device="cuda").to(torch.bfloat16)[:, :K] for r in (M, N))
    ac, asf, _, _ = nb.nvfp4_quantize_fp8(a)
    bc, bsf, _, _ = nb.nvfp4_quantize_fp8(b, 128)
    assert torch.equal(nb.nvfp4_gemm_fp8(ac, asf, bc, bsf).double(), a.double() @ b.double().T)


def test_product_leaves_what_lies_beside_its_output():
    M, N, K = 131, 200, 264
    ops, a, b = _operands(M, N, K, 9)
    for dtype, ld in ((torch.float32, 208), (torch.bfloat16, 216)):
        whole = torch.full((M + 2, ld), 7.0, dtype=dtype, device="cuda")
        nb.nvfp4_gemm_fp8(*ops, out=whole[1:M + 1, :N])
        assert bool((whole[0] == 7).all()) and bool((whole[-1] == 7).all()) and bool((whole[:, N:] == 7).all())
        ref.assert_product(whole[1:M + 1, :N], *ref.product(a, b), K)


@pytest.mark.parametrize("dtype,out", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32)])
@pytest.mark.parametrize("shape", [(1, 64, 128), (5, 136, 72), (256, 512, 512), (777, 264, 1160), (1040, 1416, 328)])
def test_layer_and_its_gradients(shape, dtype, out):
    M, N, K = shape
    X, W, dY = _x((M, K), 1, dtype, 3), _x((N, K), 2, dtype, 3), _x((M, N), 3, dtype, 3)
    Y = nb.nvfp4_linear_fp8_fwd(X, W, out_dtype=out)
    dX, dW = nb.nvfp4_linear_fp8_bwd(dY, W, X, dx_dtype=out)
    torch.cuda.synchronize()
    assert nb.nvfp4_device_error_word() == 0
    Wq = ref.values(W, True)
    ref.assert_product(Y, *ref.product(ref.values(X), Wq), K)
    ref.assert_product(dX, *ref.product(ref.values(dY), Wq.T), N)
    ref.assert_product(dW, *ref.product(ref.values(dY.T), ref.values(X.T)), M)


def test_layer_gradients_against_differences():
    # entries that are exact in the format, so that quantization is the identity and the loss sum(Y * dY) is bilinear: a difference
    # of the forward product along one weight, or one input, is the gradient
    M, N, K = 48, 40, 136
    g = torch.Generator("cuda").manual_seed(0)
    X, W, dY = (torch.randint(-4, 5, s, generator=g, device="cuda").to(torch.bfloat16) for s in ((M, K), (N, K), (M, N)))
    dX, dW = nb.nvfp4_linear_fp8_bwd(dY, W, X)

    def loss(X, W):
        return float((nb.nvfp4_linear_fp8_fwd(X, W).double() * dY.double()).sum())
    for n, k in ((0, 0), (39, 135), (17, 64), (20, 127), (21, 128)):
        up, down = W.clone(), W.clone()
        up[n, k] += 1
        down[n, k] -= 1
        assert (loss(X, up) - loss(X, down)) / 2 == float(dW[n, k])
    for m, k in ((0, 0), (47, 135), (31, 128), (32, 127)):
        up, down = X.clone(), X.clone()
        up[m, k] += 1
        down[m, k] -= 1
        assert (loss(up, W) - loss(down, W)) / 2 == float(dX[m, k])


def test_layer_products_are_those_of_the_parts():
    M, N, K = 320, 456, 648
    X, W, dY = _x((M, K), 1), _x((N, K), 2), _x((M, N), 3)
    xc, xs, xtc, xts = nb.nvfp4_quantize_fp8(X, 1, True, True)
    wc, ws, wtc, wts = nb.nvfp4_quantize_fp8(W, 128, True, True)
    yc, ys, ytc, yts = nb.nvfp4_quantize_fp8(dY, 1, True, True)
    dX, dW = nb.nvfp4_linear_fp8_bwd(dY, W, X)
    assert torch.equal(nb.nvfp4_linear_fp8_fwd(X, W), nb.nvfp4_gemm_fp8(xc, xs, wc, ws))
    assert torch.equal(dX, nb.nvfp4_gemm_fp8(yc, ys, wtc, wts)) and torch.equal(dW, nb.nvfp4_gemm_fp8(ytc, yts, xtc, xts))


def test_steps_share_a_workspace_on_any_stream_and_in_a_graph():
    # every call reads what the one before wrote; inputs change from step to step
    M, N, K = 200, 264, 328
    steps = [(_x((M, K), 10 + i, spread=2), _x((N, K), 20 + i, spread=2), _x((M, N), 30 + i, spread=2)) for i in range(3)]
    ws = torch.empty(max(nb.nvfp4_linear_fp8_workspace_bytes(M, N, K, w) for w in (nb.FP8_FWD, nb.FP8_BWD)), dtype=torch.uint8, device="cuda")

    def run(stream=None, pause=False):
        out = []
        for X, W, dY in steps:
            Y = nb.nvfp4_linear_fp8_fwd(X, W, out_dtype=torch.bfloat16, workspace=ws, stream=stream)
            if pause:
                torch.cuda.synchronize()
            out += [Y, *nb.nvfp4_linear_fp8_bwd(dY, W, X, workspace=ws, stream=stream)]
            if pause:
                torch.cuda.synchronize()
        return out
    want = run(pause=True)
    assert all(torch.equal(a, b) for a, b in zip(run(), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for _ in range(2):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_repeated_products_agree_bit_for_bit():
    for M, N, K in ((2048, 4096, 1024), (3001, 1416, 2056)):
        ops, _, _ = _operands(M, N, K, M)
        first = nb.nvfp4_gemm_fp8(*ops)
        for _ in range(12):
            assert torch.equal(nb.nvfp4_gemm_fp8(*ops), first)
    assert nb.nvfp4_device_error_word() == 0


def test_layer_of_the_350m_block_at_full_size():
    K, N, M = 1024, 2816, 16384
    X, W, dY = synth.linear_inputs(M, K, N, seed=5, device="cuda")
    Y = nb.nvfp4_linear_fp8_fwd(X, W, out_dtype=torch.bfloat16)
    dX, dW = nb.nvfp4_linear_fp8_bwd(dY, W, X, dx_dtype=torch.bfloat16)
    Wq = ref.values(W, True)
    ref.assert_product(Y, *ref.product(ref.values(X), Wq), K)
    ref.assert_product(dX, *ref.product(ref.values(dY), Wq.T), N)
    ref.assert_product(dW, *ref.product(ref.values(dY.T), ref.values(X.T)), M)


@pytest.mark.parametrize("K", [12288, 12289, 12416, 12680, 16384, 24600, 40000])
@pytest.mark.parametrize("M,N", [(300, 600), (200, 5000), (3000, 3008)])
def test_long_contractions_are_summed_in_parts(M, N, K):
    ops, a, b = _operands(M, N, K, K)
    D = nb.nvfp4_gemm_fp8(*ops)
    torch.cuda.synchronize()
    assert nb.nvfp4_device_error_word() == 0
    # additions in the tensor core: those of the longest part, at most 96 blocks; then one for each part
    ref.assert_product(D, *ref.product(a, b), 96 * 128 + 32 * (K // 12288 + 1))


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M", [1, 2, 7, 8, 15, 16, 17, 31, 33, 63, 64, 65, 100, 127, 128, 129])
def test_products_of_few_rows(M, out_dtype):
    # tiles of B alone, shared by 2, 4 and 8 blocks along K, and more of them than multiprocessors
    for N, K in ((20000, 264), (9000, 1000), (4104, 1000), (1000, 2056), (136, 4100), (5, 130)):
        ops, a, b = _operands(M, N, K, M + N)
        D = torch.full((M, -(-N // 8) * 8), 7.0, dtype=out_dtype, device="cuda")
        nb.nvfp4_gemm_fp8(*ops, out=D[:, :N])
        torch.cuda.synchronize()
        assert nb.nvfp4_device_error_word() == 0
        ref.assert_product(D[:, :N], *ref.product(a, b), K)
        assert bool((D[:, N:] == 7).all())


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (3, 5, 9), (129, 131, 257), (300, 1, 40), (700, 1003, 129)])
def test_products_of_any_size_without_an_output_given(M, N, K, out_dtype):
    ops, a, b = _operands(M, N, K, M + N)
    D = nb.nvfp4_gemm_fp8(*ops, out_dtype=out_dtype)
    assert D.shape == (M, N)
    ref.assert_product(D, *ref.product(a, b), K)
    assert nb.nvfp4_device_error_word() == 0


def test_quantizer_of_single_rows_wherever_they_lie():
    whole = _x((6, 44), 3)
    for x in (whole[2:3, 8:20], whole[1:2, :44], whole[4:5, 16:24]):             # strides that say nothing, and are no multiple of 8
        if x.data_ptr() % 16 == 0:
            _check_quantized(x, 1, nb.SF_LINEAR, *nb.nvfp4_quantize_fp8(x, transposed=True, sf_layout=nb.SF_LINEAR))
    batch = _x((3, 1, 24), 4)
    codes, scales, _, _ = nb.nvfp4_quantize_fp8(batch, sf_layout=nb.SF_LINEAR)
    for i in range(3):
        one = nb.nvfp4_quantize_fp8(batch[i], sf_layout=nb.SF_LINEAR)
        assert torch.equal(codes[i], one[0]) and torch.equal(scales[i], one[1])
    with pytest.raises(nb.NvFp4Error):                                            # the next matrix would begin inside a vector
        nb.nvfp4_quantize_fp8(_x((3, 1, 12), 5))
    nb.nvfp4_quantize_fp8(_x((1, 1, 12), 5))


@pytest.mark.parametrize("dx_dtype,dw_dtype", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("shape", [(129, 136, 136), (256, 512, 512), (777, 1000, 1160), (700, 704, 2048), (1024, 1024, 2048), (1000, 1400, 1536),
                                   (1024, 1600, 2048), (129, 9472, 8), (200, 136, 12296)])
def test_gradients_of_one_launch_are_those_of_two(shape, dx_dtype, dw_dtype):
    # every tile with a pair of its own, in each width; more tiles than pairs; a contraction too long for it; few rows
    M, N, K = shape
    X, W, dY = _x((M, K), 1), _x((N, K), 2), _x((M, N), 3)
    want_dx, want_dw = (torch.empty(s, dtype=t, device="cuda") for s, t in (((M, K), dx_dtype), ((N, K), dw_dtype)))
    _, _, wt, wts = nb.nvfp4_quantize_fp8(W, 128, False, True)
    _, _, xt, xts = nb.nvfp4_quantize_fp8(X, 1, False, True)
    dy, dys, dyt, dyts = nb.nvfp4_quantize_fp8(dY, 1, True, True)
    nb.nvfp4_gemm_fp8(dy, dys, wt, wts, out=want_dx)
    nb.nvfp4_gemm_fp8(dyt, dyts, xt, xts, out=want_dw)
    for _ in range(3):
        dX, dW = nb.nvfp4_linear_fp8_bwd(dY, W, X, dx_dtype=dx_dtype, dw_dtype=dw_dtype)
        assert torch.equal(dX, want_dx) and torch.equal(dW, want_dw)
    assert nb.nvfp4_device_error_word() == 0
