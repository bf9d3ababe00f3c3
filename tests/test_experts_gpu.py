"""Layers whose weights are split among experts: routing bit for bit, rows moved and summed, their gradients, the experts' products in
FP8, and all of it one after the other, against plain 64-bit forms."""
import pytest
import torch

import fp8_reference as ref
from paper_2505_19115_b200 import binding as nb

pytestmark = pytest.mark.gpu


def _choices(T, topk, E, seed, drop=0.1, distinct=True, skew=1.0, dtype=torch.int32):
    g = torch.Generator("cuda").manual_seed(seed)
    if distinct:
        scores = torch.randn((T, E), generator=g, device="cuda") + skew * torch.randn((1, E), generator=g, device="cuda")
        chosen = scores.topk(topk, 1).indices
    else:
        chosen = torch.randint(0, E, (T, topk), generator=g, device="cuda")
    return torch.where(torch.rand((T, topk), generator=g, device="cuda") < drop, -1, chosen).to(dtype)


def _normal(shape, seed, dtype=torch.bfloat16, std=1.0):
    g = torch.Generator("cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _check_plan(expert_of, E, plan):
    counts, offsets, row_of, slot_of = ref.route(expert_of.cpu(), E, plan.rows)
    assert plan.counts.tolist() == counts and plan.offsets.tolist() == offsets
    assert plan.row_of.reshape(-1).tolist() == row_of and plan.slot_of.tolist() == slot_of


@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
@pytest.mark.parametrize("size", [(1, 1, 1), (1, 8, 64), (3, 2, 5), (31, 1, 7), (130, 4, 8), (1000, 2, 3), (777, 6, 61), (2049, 8, 256),
                                  (4096, 2, 1024), (20000, 1, 2), (9001, 4, 33)])
def test_sort_matches_the_definition(size, dtype):
    T, topk, E = size
    for drop in (0.0, 0.3, 1.0):
        expert_of = _choices(T, topk, E, T + topk, drop, dtype=dtype)
        _check_plan(expert_of, E, nb.nvfp4_expert_sort(expert_of, E))


def test_sort_of_one_sided_repeated_and_foreign_choices():
    T, topk, E = 700, 4, 16
    for fill in (0, 15):
        expert_of = torch.full((T, topk), fill, dtype=torch.int32, device="cuda")           # one expert, the same for every choice
        _check_plan(expert_of, E, nb.nvfp4_expert_sort(expert_of, E))
    _check_plan(_choices(T, topk, E, 1, 0.0, False), E, nb.nvfp4_expert_sort(_choices(T, topk, E, 1, 0.0, False), E))
    for dtype, low, high in ((torch.int32, -2 ** 31, 2 ** 31 - 1), (torch.int64, -2 ** 62, 2 ** 62)):
        expert_of = _choices(T, topk, E, 2, 0.0, dtype=dtype)
        expert_of[5], expert_of[6], expert_of[7] = E, low, high
        if dtype == torch.int64:
            expert_of[8] = (1 << 32) + 3                                                     # its low half names an expert
        plan = nb.nvfp4_expert_sort(expert_of, E)
        _check_plan(torch.where((expert_of >= 0) & (expert_of < E), expert_of, -1), E, plan)


def test_sort_writes_nothing_behind_its_outputs():
    T, topk, E = 333, 3, 17
    expert_of = _choices(T, topk, E, 3)
    R = nb.nvfp4_expert_rows(T, topk, E)
    bufs = [torch.full((n + 64,), -77, dtype=torch.int32, device="cuda") for n in (E, E + 1, T * topk, R)]
    views = [b[32:-32] for b in bufs]
    assert nb._native().nvfp4_expert_sort(expert_of, 0, T, topk, E, *views, None) == 0
    assert all(bool((b[:32] == -77).all()) and bool((b[-32:] == -77).all()) for b in bufs)


def _reference(plan):
    row_of, slot_of = plan.row_of.long(), plan.slot_of.long()
    return row_of, slot_of, int(plan.offsets[-1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("w_dtype", [None, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("size", [(1, 8, 16, 64), (5, 1, 3, 8), (300, 2, 8, 520), (129, 6, 40, 1032), (1000, 5, 7, 2048), (40, 40, 64, 72),
                                  (3000, 3, 6, 264), (2500, 1, 4, 1032), (2400, 34, 40, 136)])
def test_rows_moved_and_summed_with_gradients(size, w_dtype, dtype):
    T, topk, E, H = size
    plan = nb.nvfp4_expert_sort(_choices(T, topk, E, T, 0.2), E)
    row_of, slot_of, used = _reference(plan)
    wide = _normal((T, H + 24), 1, dtype)
    x, dy = wide[:, 8:8 + H], _normal((T, H), 2, dtype)
    w = None if w_dtype is None else _normal((T, topk), 3, w_dtype)
    wd = torch.ones((T, topk), dtype=torch.float64, device="cuda") if w is None else w.double()
    eps = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24

    # gather: one rounding of the product in fp32 and one to the type
    rows = torch.full((plan.rows, H), 5.0, dtype=dtype, device="cuda")
    nb.nvfp4_expert_gather(x, plan, w, out=rows)
    assert bool((rows[used:] == 5).all())
    source = slot_of[:used].clamp(min=0)
    want = torch.where((slot_of[:used] >= 0)[:, None], wd.reshape(-1)[source][:, None] * x.double()[source // topk], 0)
    assert bool(((rows[:used].double() - want).abs() <= want.abs() * (eps + 2.0 ** -24) * 1.01).all())
    if w is None:
        assert torch.equal(rows[:used].double(), want)

    # combine: topk terms, each sum and product rounded once in fp32, then to the type
    rows = _normal((plan.rows, H), 4, dtype)
    rows[:used][slot_of[:used] < 0] = float("nan")                                          # padding and unused rows are not read
    rows[used:] = float("nan")
    picked = torch.where((row_of >= 0)[..., None], rows.double()[row_of.clamp(min=0)], 0) * wd[..., None]
    y = nb.nvfp4_expert_combine(rows, plan, w)
    want, size_ = picked.sum(1), picked.abs().sum(1)
    assert bool(((y.double() - want).abs() <= want.abs() * eps + size_ * (topk + 1) * 2.0 ** -24 * (1 + eps) + 1e-40).all())
    if w is None:
        return

    # its gradients
    drows = torch.full((plan.rows, H), 5.0, dtype=dtype, device="cuda")
    got, dw = nb.nvfp4_expert_combine_bwd(dy, rows, plan, w, drows=drows)
    assert got is drows and bool((drows[used:] == 5).all())
    want = torch.where((slot_of[:used] >= 0)[:, None], wd.reshape(-1)[source][:, None] * dy.double()[source // topk], 0)
    assert bool(((drows[:used].double() - want).abs() <= want.abs() * (eps + 2.0 ** -24) * 1.01).all())
    terms = torch.where((row_of >= 0)[..., None], rows.double()[row_of.clamp(min=0)] * dy.double()[:, None], 0)
    want = terms.sum(-1)
    # a lane sums H / 32 terms, five more sums join the lanes
    tol = terms.abs().sum(-1) * (H // 32 + 14) * 2.0 ** -24 + want.abs() * (2.0 ** -8 if w_dtype == torch.bfloat16 else 2.0 ** -24)
    assert bool(((dw.double() - want).abs() <= tol * (1 + 2.0 ** -8)).all())
    assert bool((dw[row_of < 0] == 0).all())
    none, again = nb.nvfp4_expert_combine_bwd(dy, rows, plan, w, rows_gradient=False)
    assert none is None and torch.equal(again, dw)


def test_combine_and_gather_are_each_other_s_transposes():
    # <gather(x), r> = <x, combine(r)> exactly for small integers, weights included
    T, topk, E, H = 257, 3, 9, 136
    plan = nb.nvfp4_expert_sort(_choices(T, topk, E, 8, 0.1, False), E)
    g = torch.Generator("cuda").manual_seed(4)
    x = torch.randint(-3, 4, (T, H), generator=g, device="cuda").float()
    r = torch.randint(-3, 4, (plan.rows, H), generator=g, device="cuda").float()
    w = torch.randint(-2, 3, (T, topk), generator=g, device="cuda").float()
    rows = torch.zeros_like(r)
    nb.nvfp4_expert_gather(x, plan, w, out=rows)
    left, right = (rows.double() * r).sum(), (x.double() * nb.nvfp4_expert_combine(r, plan, w)).sum()
    assert float(left) == float(right)
    _, dw = nb.nvfp4_expert_combine_bwd(x, r, plan, w)
    assert float((dw.double() * w).sum()) == float(right)


# ---- the experts' products ----
CASES = [(1, 2, 4, 64, 128), (5, 1, 3, 136, 72), (64, 8, 64, 96, 256), (300, 2, 8, 264, 520), (513, 4, 5, 1032, 136), (1000, 1, 2, 200, 1160),
         (2000, 2, 3, 712, 328)]


def _segments(plan):
    o = plan.offsets.tolist()
    return [(e, o[e], o[e] + c) for e, c in enumerate(plan.counts.tolist())]


@pytest.mark.parametrize("sorted_rows", [False, True])
@pytest.mark.parametrize("weighted", [None, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("size", [(1, 2, 4, 128), (200, 3, 7, 136), (700, 2, 5, 1030)])
def test_quantizer_of_sorted_rows(size, dtype, weighted, sorted_rows):
    T, topk, E, C = size
    plan = nb.nvfp4_expert_sort(_choices(T, topk, E, T), E)
    _, slot_of, used = _reference(plan)
    w = None if weighted is None else _normal((T, topk), 3, weighted)
    source = slot_of[:used].clamp(min=0)
    pad = (slot_of[:used] < 0)[:, None]
    x = _normal((plan.rows if sorted_rows else T, -(-C // 8) * 8), 5, dtype)[:, :C]
    rows = x[:used] if sorted_rows else x[source // topk]
    if sorted_rows:
        x[:used][pad[:, 0]] = float("nan")                                                  # what padding rows hold does not count
        x[used:] = float("nan")
    rows = torch.where(pad, 0, rows.float() * (1.0 if w is None else w.reshape(-1)[source].float()[:, None]))    # one rounding in fp32
    codes, scales, codes_t, scales_t = nb.nvfp4_quantize_fp8_experts(x, plan, w, sorted_rows, True, True)
    y, e = ref.codes_and_exponents(rows)
    assert torch.equal(codes[:used], ref.code_bytes(y))
    tile = -(-C // 512) * 512
    assert torch.equal(scales.cpu()[:used // 128 * tile], torch.from_numpy(ref.swizzled(ref.scale_bytes(e))))
    y, e = ref.codes_and_exponents(rows.T)
    assert torch.equal(codes_t[:, :used], ref.code_bytes(y))
    full = torch.from_numpy(ref.swizzled(ref.scale_bytes(torch.nn.functional.pad(e, (0, plan.rows - used)))))
    got = scales_t.cpu().view(-1, 512)                                                      # tiles: [C / 128][rows / 512]
    for kb in range(used // 128):
        for c0 in range(-(-C // 128)):
            t = c0 * (-(-plan.rows // 512)) + kb // 4
            assert torch.equal(got[t][kb % 4::4], full.view(-1, 512)[t][kb % 4::4])


@pytest.mark.parametrize("dtype,out", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32)])
@pytest.mark.parametrize("size", CASES)
def test_layer_of_experts_and_its_gradients(size, dtype, out):
    T, topk, E, N, K = size
    plan = nb.nvfp4_expert_sort(_choices(T, topk, E, T + N, 0.1, skew=2.0), E)
    _, slot_of, used = _reference(plan)
    source, pad = slot_of[:used].clamp(min=0), (slot_of[:used] < 0)[:, None]
    x, dy, W = _normal((T, K), 1, dtype), _normal((T, N), 2, dtype), _normal((E, N, K), 3, dtype, 0.05)
    w = _normal((T, topk), 4, torch.float32)
    Y = torch.full((plan.rows, N), 5.0, dtype=out, device="cuda")
    dX = torch.full((plan.rows, K), 5.0, dtype=out, device="cuda")
    nb.nvfp4_experts_fp8_fwd(x, W, plan, out=Y)
    _, dW = nb.nvfp4_experts_fp8_bwd(dy, W, x, plan, weights=w, dX=dX)
    torch.cuda.synchronize()
    assert nb.nvfp4_device_error_word() == 0
    assert bool((Y[used:] == 5).all()) and bool((dX[used:] == 5).all())
    rows = torch.where(pad, 0, x[source // topk].float())
    drows = torch.where(pad, 0, dy[source // topk].float() * w.reshape(-1)[source][:, None])
    for e, begin, end in _segments(plan):
        if begin == end:
            assert not bool(dW[e].any())
            continue
        Wq, X, D = ref.values(W[e], True), rows[begin:end], drows[begin:end]
        ref.assert_product(Y[begin:end], *ref.product(ref.values(X), Wq), K)
        ref.assert_product(dX[begin:end], *ref.product(ref.values(D), Wq.T), N)
        ref.assert_product(dW[e], *ref.product(ref.values(D.T), ref.values(X.T)), end - begin)
    assert not bool(Y[:used][pad[:, 0]].any()) and not bool(dX[:used][pad[:, 0]].any())     # padding rows come out as zeros
    # rows that are sorted already give the same
    rows, drows = nb.nvfp4_expert_gather(x, plan), nb.nvfp4_expert_gather(dy, plan)
    again = nb.nvfp4_experts_fp8_fwd(rows, W, plan, sorted_rows=True, out_dtype=out)
    dX2, dW2 = nb.nvfp4_experts_fp8_bwd(drows, W, rows, plan, weights=w, dy_sorted_rows=True, sorted_rows=True, dx_dtype=out)
    assert torch.equal(again[:used], Y[:used]) and torch.equal(dX2[:used], dX[:used]) and torch.equal(dW2, dW)


def test_layer_is_that_of_the_parts_and_of_single_layers():
    T, topk, E, N, K = 600, 2, 6, 264, 392
    plan = nb.nvfp4_expert_sort(_choices(T, topk, E, 11), E)
    x, dy, W = _normal((T, K), 1), _normal((T, N), 2), _normal((E, N, K), 3, std=0.05)
    used = int(plan.offsets[-1])
    wc, ws, wtc, wts = nb.nvfp4_quantize_fp8(W, 128, True, True)
    xc, xs, xtc, xts = nb.nvfp4_quantize_fp8_experts(x, plan, transposed=True)
    dc, ds, dtc, dts = nb.nvfp4_quantize_fp8_experts(dy, plan, transposed=True)
    Y = nb.nvfp4_experts_fp8_fwd(x, W, plan)
    dX, dW = nb.nvfp4_experts_fp8_bwd(dy, W, x, plan)
    assert torch.equal(nb.nvfp4_gemm_fp8_experts(xc, xs, wc, ws, plan, out_dtype=Y.dtype)[:used], Y[:used])
    assert torch.equal(nb.nvfp4_gemm_fp8_experts(dc, ds, wtc, wts, plan, out_dtype=dX.dtype)[:used], dX[:used])
    assert torch.equal(nb.nvfp4_gemm_fp8_experts_dw(dtc, dts, xtc, xts, plan), dW)
    rows, drows = nb.nvfp4_expert_gather(x, plan), nb.nvfp4_expert_gather(dy, plan)
    for e, begin, end in _segments(plan):
        X, D = rows[begin:end].contiguous(), drows[begin:end].contiguous()
        assert torch.equal(nb.nvfp4_linear_fp8_fwd(X, W[e], out_dtype=Y.dtype), Y[begin:end])
        dx, dw = nb.nvfp4_linear_fp8_bwd(D, W[e], X, dx_dtype=dX.dtype)
        assert torch.equal(dx, dX[begin:end]) and torch.equal(dw, dW[e])


def test_empty_experts_all_dropped_and_one_expert_for_all():
    T, topk, E, N, K = 300, 2, 5, 72, 136
    x, dy, W = _normal((T, K), 1), _normal((T, N), 2), _normal((E, N, K), 3)
    none = torch.full((T, topk), -1, dtype=torch.int32, device="cuda")
    plan = nb.nvfp4_expert_sort(none, E)
    Y = torch.full((plan.rows, N), 5.0, dtype=x.dtype, device="cuda")
    nb.nvfp4_experts_fp8_fwd(x, W, plan, out=Y)
    dX = torch.full((plan.rows, K), 5.0, dtype=x.dtype, device="cuda")
    _, dW = nb.nvfp4_experts_fp8_bwd(dy, W, x, plan, dX=dX, dW=torch.full_like(W, 3.0, dtype=torch.float32))
    assert bool((Y == 5).all()) and bool((dX == 5).all()) and not bool(dW.any())
    assert not bool(nb.nvfp4_expert_combine(Y, plan, torch.ones((T, topk), device="cuda")).any())
    plan = nb.nvfp4_expert_sort(torch.full((T, topk), 3, dtype=torch.int32, device="cuda"), E)
    Y = nb.nvfp4_experts_fp8_fwd(x, W, plan)
    one = nb.nvfp4_linear_fp8_fwd(x.repeat_interleave(topk, 0), W[3], out_dtype=x.dtype)
    assert torch.equal(Y[:T * topk], one)
    assert nb.nvfp4_device_error_word() == 0


def test_offsets_that_are_none_stay_inside_the_tensors():
    # what a plan can never hold: the products cut it to multiples of 128 within the rows, so that no access leaves a buffer
    T, topk, E, N, K = 200, 2, 4, 136, 264
    expert_of = _choices(T, topk, E, 5, 0.0)
    plan = nb.nvfp4_expert_sort(expert_of, E)
    x, W = _normal((T, K), 1), _normal((E, N, K), 3)
    wc, ws, _, _ = nb.nvfp4_quantize_fp8(W, 128)
    xc, xs, xtc, xts = nb.nvfp4_quantize_fp8_experts(x, plan, transposed=True)
    whole = torch.full((plan.rows + 256, N), 5.0, device="cuda")
    for bad in ([0, -4096, 2 ** 31 - 1, 128, 2 ** 31 - 1], [-5, 77, 300, 10 ** 6, -1]):
        plan.offsets.copy_(torch.tensor(bad, dtype=torch.int32))
        nb.nvfp4_gemm_fp8_experts(xc, xs, wc, ws, plan, out=whole[128:-128])
        nb.nvfp4_gemm_fp8_experts_dw(xtc, xts, xtc, xts, plan)
        torch.cuda.synchronize()
        assert bool((whole[:128] == 5).all()) and bool((whole[-128:] == 5).all())
    assert nb.nvfp4_device_error_word() == 0


def _step(x, dy, W, w, expert_of, E, ws):
    """One training step of a layer of experts, as a program runs it."""
    plan = nb.nvfp4_expert_sort(expert_of, E)
    Y = nb.nvfp4_experts_fp8_fwd(x, W, plan, workspace=ws)
    y = nb.nvfp4_expert_combine(Y, plan, w)
    _, dw = nb.nvfp4_expert_combine_bwd(dy, Y, plan, w, rows_gradient=False)
    dX, dW = nb.nvfp4_experts_fp8_bwd(dy, W, x, plan, weights=w, workspace=ws)
    return y, nb.nvfp4_expert_combine(dX, plan), dW, dw


def _workspace(T, topk, E, N, K):
    return torch.empty(max(nb.nvfp4_experts_fp8_workspace_bytes(T, topk, E, N, K, k) for k in (nb.FP8_FWD, nb.FP8_BWD)), dtype=torch.uint8, device="cuda")


def test_a_step_of_the_layer_against_64_bits():
    T, topk, E, N, K = 500, 2, 6, 200, 264
    x, dy, W, w = _normal((T, K), 1), _normal((T, N), 2), _normal((E, N, K), 3, std=0.05), _normal((T, topk), 4, torch.float32)
    expert_of = _choices(T, topk, E, 6)
    y, dx, dW, dw = _step(x, dy, W, w, expert_of, E, _workspace(T, topk, E, N, K))
    want = [torch.zeros(t.shape, dtype=torch.float64, device="cuda") for t in (y, dx, dw)]
    size = [torch.zeros_like(t) for t in want]
    bf = 2.0 ** -8
    for e in range(E):
        t, j = (expert_of == e).nonzero(as_tuple=True)
        X, D, we = x[t], dy[t].float() * w[t, j][:, None], w[t, j].double()[:, None]
        Wq = ref.values(W[e], True)
        (Y, TY), (G, TG) = ref.product(ref.values(X), Wq), ref.product(ref.values(D), Wq.T)
        want[0].index_add_(0, t, we * Y)
        want[1].index_add_(0, t, G)
        want[2][t, j] = (Y * dy[t].double()).sum(1)
        # a row is rounded to bf16 behind its sum
        size[0].index_add_(0, t, we.abs() * (Y.abs() * bf + TY * ref.accumulation(K)))
        size[1].index_add_(0, t, G.abs() * bf + TG * ref.accumulation(N))
        size[2][t, j] = ((Y.abs() * bf + TY * ref.accumulation(K)) * dy[t].double().abs()).sum(1)
        ref.assert_product(dW[e], *ref.product(ref.values(D.T), ref.values(X.T)), len(t))
    for got, exact, tol in zip((y, dx, dw), want, size):
        assert bool(((got.double() - exact).abs() <= exact.abs() * bf + tol * 1.02 + 1e-30).all())


def test_steps_share_a_workspace_on_any_stream_and_in_a_graph():
    T, topk, E, N, K = 300, 2, 6, 200, 264
    ws = _workspace(T, topk, E, N, K)
    inputs = [(_normal((T, K), 10 + i), _normal((T, N), 20 + i), _normal((E, N, K), 30 + i, std=0.05), _normal((T, topk), 40 + i, torch.float32),
               _choices(T, topk, E, 50 + i), E, ws) for i in range(3)]

    def run():
        return [t for i in inputs for t in _step(*i)]
    want = []
    for i in inputs:
        want += _step(*i)
        torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(run(), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run()
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
    # other routing through the same captured graph: the rows' places are read on the device
    inputs[1][4].copy_(_choices(T, topk, E, 99, 0.5, skew=3.0))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got[4:8], _step(*inputs[1])))
    assert nb.nvfp4_device_error_word() == 0


def test_single_token_through_kept_weights():
    E, N, K, topk = 16, 264, 520, 4
    W = _normal((E, N, K), 1, std=0.05)
    wc, ws, _, _ = nb.nvfp4_quantize_fp8(W, 128)
    for T in (1, 2, 7):
        x, w, expert_of = _normal((T, K), 2 + T), _normal((T, topk), 3, torch.float32), _choices(T, topk, E, T, 0.0, dtype=torch.int64)
        plan = nb.nvfp4_expert_sort(expert_of, E)
        xc, xs, _, _ = nb.nvfp4_quantize_fp8_experts(x, plan)
        Y = nb.nvfp4_gemm_fp8_experts(xc, xs, wc, ws, plan)
        y = nb.nvfp4_expert_combine(Y, plan, w)
        for t in range(T):
            terms = torch.stack([w[t, j].double() * ref.product(ref.values(x[t:t + 1]), ref.values(W[expert_of[t, j]], True))[0][0] for j in range(topk)])
            sizes = torch.stack([w[t, j].double().abs() * ref.product(ref.values(x[t:t + 1]), ref.values(W[expert_of[t, j]], True))[1][0] for j in range(topk)])
            tol = sizes.sum(0) * (ref.accumulation(K) + (topk + 2) * 2.0 ** -24)
            assert bool(((y[t].double() - terms.sum(0)).abs() <= tol).all())
    assert nb.nvfp4_device_error_word() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_weights_and_values_next_to_the_smallest_and_the_largest_numbers(dtype):
    # a row's weight and its scale are one factor where that is exact; these are not, or are nearly not
    T, topk, E, C = 40, 2, 3, 264
    plan = nb.nvfp4_expert_sort(_choices(T, topk, E, 1, 0.0), E)
    _, slot_of, used = _reference(plan)
    source, pad = slot_of[:used].clamp(min=0), (slot_of[:used] < 0)[:, None]
    x = _normal((T, C), 5, torch.float32)
    x = (x * torch.exp2(torch.linspace(-126, 100, T, device="cuda"))[:, None]).to(dtype)
    x[3], x[4, 5] = 0, float("nan")
    for weights in (torch.exp2(torch.linspace(-20, 26, T * topk, device="cuda")) * 1.1, torch.full((T * topk,), 1e-38, device="cuda"),
                    torch.full((T * topk,), -3e37, device="cuda"), torch.zeros(T * topk, device="cuda"), torch.full((T * topk,), float("inf"), device="cuda")):
        w = weights.view(T, topk)
        rows = torch.where(pad, 0, x[source // topk].float() * w.reshape(-1)[source][:, None])
        codes, scales, codes_t, scales_t = nb.nvfp4_quantize_fp8_experts(x, plan, w, transposed=True)
        for src, c, sf in ((rows, codes[:used], scales), (rows.T, codes_t[:, :used], scales_t)):
            R, Cq = src.shape
            bad = torch.nn.functional.pad(~src.isfinite(), (0, -Cq % 128)).view(R, -1, 128).any(2)
            tiles = -(-(C if src is rows else plan.rows) // 512)
            r, kb = torch.meshgrid(torch.arange(R, device="cuda"), torch.arange(bad.shape[1], device="cuda"), indexing="ij")
            got = sf[((r // 128) * tiles + kb // 4) * 512 + (r % 32) * 16 + ((r % 128) // 32) * 4 + kb % 4]
            assert torch.equal(got == 255, bad)
            # a NaN or an infinity of a block hides its other values: those blocks are NaN, the others as defined
            keep = ~bad.repeat_interleave(128, 1)[:, :Cq]
            clean = torch.where(bad.repeat_interleave(128, 1)[:, :Cq], 0, src.nan_to_num(0, 0, 0))
            y, e = ref.codes_and_exponents(clean)
            assert torch.equal(c[keep], ref.code_bytes(y)[keep])
            assert torch.equal(got[~bad], ref.scale_bytes(e)[~bad])
            assert bool((c[~keep] & 127 == 127).all())


def test_two_streams_at_once_with_workspaces_of_their_own():
    T, topk, E, N, K = 700, 2, 6, 328, 392
    work = [(_normal((T, K), 10 + i), _normal((T, N), 20 + i), _normal((E, N, K), 30 + i, std=0.05), _normal((T, topk), 40 + i, torch.float32),
             _choices(T, topk, E, 50 + i), E, _workspace(T, topk, E, N, K)) for i in range(2)]
    want = []
    for w in work:
        want.append(_step(*w))
        torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    got = [None, None]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(6):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = _step(*work[i])
    torch.cuda.synchronize()
    assert nb.nvfp4_device_error_word() == 0
    for g, w in zip(got, want):
        assert all(torch.equal(a, b) for a, b in zip(g, w))


def test_few_rows_of_experts_in_every_number():
    # the product of few rows for each expert: none, one, those of a tile and more than a tile, and experts that share nothing
    E, N, K = 7, 392, 648
    W = _normal((E, N, K), 1, std=0.05)
    wc, ws, _, _ = nb.nvfp4_quantize_fp8(W, 128)
    for counts in ([0, 1, 2, 15, 16, 17, 0], [128, 0, 0, 129, 31, 33, 1], [300, 0, 0, 0, 0, 0, 0], [0, 0, 0, 0, 0, 0, 1]):
        expert_of = torch.repeat_interleave(torch.arange(E), torch.tensor(counts))[torch.randperm(sum(counts), generator=torch.Generator().manual_seed(1))]
        expert_of = expert_of.int().cuda()[:, None].contiguous()
        plan = nb.nvfp4_expert_sort(expert_of, E)
        assert plan.counts.tolist() == counts
        x = _normal((len(expert_of), K), 2)
        xc, xs, _, _ = nb.nvfp4_quantize_fp8_experts(x, plan)
        rows = nb.nvfp4_expert_gather(x, plan)
        for dtype in (torch.float32, torch.bfloat16):
            Y = torch.full((plan.rows, N), 5.0, dtype=dtype, device="cuda")
            nb.nvfp4_gemm_fp8_experts(xc, xs, wc, ws, plan, out=Y)
            torch.cuda.synchronize()
            assert nb.nvfp4_device_error_word() == 0
            assert bool((Y[int(plan.offsets[-1]):] == 5).all())
            for e, begin, end in _segments(plan):
                if begin < end:
                    ref.assert_product(Y[begin:end], *ref.product(ref.values(rows[begin:end]), ref.values(W[e], True)), K)
