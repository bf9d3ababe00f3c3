"""Calls that are given a stream and make their own outputs and scratch.  That memory belongs to the given stream: work queued on the
current stream before the call does not write to it, and it is handed out again only when the call's kernels are done with it, and
when work queued on the current stream on an output is."""
import pytest
import torch

from paper_2505_19115_b200 import binding as nb
from paper_2505_19115_b200 import synth

pytestmark = pytest.mark.gpu

M, N, K = 256, 512, 768
T, TOPK, E = 300, 2, 6
PAUSE = 300_000_000                                  # cycles: about 150 ms, longer than everything that is queued behind it


def _x(shape, seed, std=1.0, dtype=torch.bfloat16):
    return synth.normal(shape, std, seed, device="cuda", dtype=dtype)


class Inputs:
    def __init__(self):
        self.X, self.W, self.dY = _x((M, K), 1), _x((N, K), 2, 0.05), _x((M, N), 3)
        self.g = torch.ones(1, device="cuda")
        self.xq, self.wq = (nb.nvfp4_quantize(t, sf_layout=nb.SF_SWIZZLED) for t in (self.X, self.W))
        self.mx = [nb.nvfp4_quantize_mx(t, sf_layout=nb.SF_SWIZZLED) for t in (self.X, self.W)]
        self.saved = nb.nvfp4_linear_fwd_save(self.X, self.W)[1]
        self.x8, self.w8 = nb.nvfp4_quantize_fp8(self.X)[:2], nb.nvfp4_quantize_fp8(self.W, 128)[:2]
        g = torch.Generator("cuda").manual_seed(5)
        self.expert_of = torch.randint(0, E, (T, TOPK), generator=g, device="cuda").int()
        self.plan = nb.nvfp4_expert_sort(self.expert_of, E)
        self.x, self.dy, self.We = _x((T, K), 6), _x((T, N), 7), _x((E, N, K), 8, 0.05)
        self.w = _x((T, TOPK), 9, dtype=torch.float32)
        R = self.plan.rows
        # every row of an output that is looked at is written: rows behind the last segment are cut off below
        self.rows = torch.zeros((R, N), dtype=torch.bfloat16, device="cuda")
        self.we8 = nb.nvfp4_quantize_fp8(self.We, 128)[:2]
        self.rows8 = nb.nvfp4_quantize_fp8_experts(self.x, self.plan, transposed=True)
        self.drows8 = nb.nvfp4_quantize_fp8_experts(self.dy, self.plan, transposed=True)
        torch.cuda.synchronize()
        self.used = int(self.plan.offsets[-1])


# name -> (the call, bytes of what it makes besides the outputs that are looked at)
CALLS = {
    "quantize": (lambda i, s: nb.nvfp4_quantize(i.X, stream=s), None),
    "quantize_swizzled": (lambda i, s: nb.nvfp4_quantize(i.X, True, sf_layout=nb.SF_SWIZZLED, stream=s), None),
    "quantize_dual": (lambda i, s: nb.nvfp4_quantize_dual(i.X, stream=s), None),
    "quantization_noise": (lambda i, s: nb.nvfp4_quantization_noise(i.X, *i.xq, sf_layout=nb.SF_SWIZZLED, stream=s), None),
    "amax_scale": (lambda i, s: nb.nvfp4_tensor_amax_scale(i.X, stream=s), None),
    "gemm": (lambda i, s: nb.nvfp4_gemm(*i.xq, None, *i.wq, None, stream=s), None),
    "gemm_quantized": (lambda i, s: nb.nvfp4_gemm_quantized(*i.xq, None, *i.wq, None, stream=s), None),
    "quantize_mx": (lambda i, s: nb.nvfp4_quantize_mx(i.X, stream=s), None),
    "quantize_mx_transposed": (lambda i, s: nb.nvfp4_quantize_mx(i.X, True, sf_layout=nb.SF_SWIZZLED, stream=s), None),
    "gemm_mx": (lambda i, s: nb.nvfp4_gemm_mx(*i.mx[0], None, *i.mx[1], None, stream=s), None),
    "gemm_bf16": (lambda i, s: nb.nvfp4_gemm_bf16(i.X, i.W, stream=s), None),
    "gemm_bf16_ex": (lambda i, s: nb.nvfp4_gemm_bf16_ex(i.X, False, i.W, False, stream=s), None),
    "transpose_bf16": (lambda i, s: nb.nvfp4_transpose_bf16(i.X, stream=s), None),
    "linear_fwd": (lambda i, s: nb.nvfp4_linear_fwd(i.X, i.W, stream=s), lambda: [nb.nvfp4_linear_workspace_bytes(M, N, K, nb.LINEAR_FWD)]),
    "linear_bwd_dx": (lambda i, s: nb.nvfp4_linear_bwd_dx(i.dY, i.W, stream=s), lambda: [nb.nvfp4_linear_workspace_bytes(M, N, K, nb.LINEAR_BWD_DX)]),
    "linear_bwd_dw": (lambda i, s: nb.nvfp4_linear_bwd_dw(i.dY, i.X, stream=s), lambda: [nb.nvfp4_linear_workspace_bytes(M, N, K, nb.LINEAR_BWD_DW)]),
    "linear_fwd_qout": (lambda i, s: nb.nvfp4_linear_fwd_qout(i.X, i.W, i.g, stream=s), lambda: [nb.nvfp4_linear_workspace_bytes(M, N, K, nb.LINEAR_FWD)]),
    "linear_fwd_qin": (lambda i, s: nb.nvfp4_linear_fwd_qin(*i.xq, None, i.W, stream=s), lambda: [nb.nvfp4_linear_workspace_bytes(M, N, K, nb.LINEAR_FWD)]),
    "linear_fwd_save": (lambda i, s: nb.nvfp4_linear_fwd_save(i.X, i.W, stream=s)[:1],
                        lambda: [nb.nvfp4_linear_fused_workspace_bytes(M, N, K, nb.FUSED_FWD_SAVE), nb.nvfp4_linear_saved_bytes(M, N, K)]),
    "linear_bwd_saved": (lambda i, s: nb.nvfp4_linear_bwd_saved(i.dY, i.saved, K, stream=s),
                         lambda: [nb.nvfp4_linear_fused_workspace_bytes(M, N, K, nb.FUSED_BWD_SAVED)]),
    "linear_bwd": (lambda i, s: nb.nvfp4_linear_bwd(i.dY, i.W, i.X, stream=s), lambda: [nb.nvfp4_linear_fused_workspace_bytes(M, N, K, nb.FUSED_BWD)]),
    "linear_bwd_bf16": (lambda i, s: nb.nvfp4_linear_bwd_bf16(i.dY, i.W, i.X, stream=s),
                        lambda: [nb.lib().nvfp4_linear_bwd_bf16_workspace_bytes(M, N, K)]),
    "linear_fwd_static": (lambda i, s: nb.nvfp4_linear_fwd_static(i.X, i.W, stream=s), None),
    "quantize_fp8": (lambda i, s: nb.nvfp4_quantize_fp8(i.X, transposed=True, stream=s), None),
    "gemm_fp8": (lambda i, s: nb.nvfp4_gemm_fp8(*i.x8, *i.w8, stream=s), None),
    "linear_fp8_fwd": (lambda i, s: nb.nvfp4_linear_fp8_fwd(i.X, i.W, stream=s), lambda: [nb.nvfp4_linear_fp8_workspace_bytes(M, N, K, nb.FP8_FWD)]),
    "linear_fp8_bwd": (lambda i, s: nb.nvfp4_linear_fp8_bwd(i.dY, i.W, i.X, stream=s), lambda: [nb.nvfp4_linear_fp8_workspace_bytes(M, N, K, nb.FP8_BWD)]),
    "expert_sort": (lambda i, s: _parts(nb.nvfp4_expert_sort(i.expert_of, E, stream=s)), None),
    "expert_gather": (lambda i, s: nb.nvfp4_expert_gather(i.x, i.plan, i.w, stream=s), None),
    "expert_combine": (lambda i, s: nb.nvfp4_expert_combine(i.rows, i.plan, i.w, stream=s), None),
    "expert_combine_bwd": (lambda i, s: nb.nvfp4_expert_combine_bwd(i.dy, i.rows, i.plan, i.w, stream=s), None),
    "quantize_fp8_experts": (lambda i, s: nb.nvfp4_quantize_fp8_experts(i.x, i.plan, i.w, stream=s)[:1], None),
    "gemm_fp8_experts": (lambda i, s: nb.nvfp4_gemm_fp8_experts(*i.rows8[:2], *i.we8, i.plan, stream=s), None),
    "gemm_fp8_experts_dw": (lambda i, s: nb.nvfp4_gemm_fp8_experts_dw(*i.drows8[2:], *i.rows8[2:], i.plan, stream=s), None),
    "experts_fp8_fwd": (lambda i, s: nb.nvfp4_experts_fp8_fwd(i.x, i.We, i.plan, stream=s),
                        lambda: [nb.nvfp4_experts_fp8_workspace_bytes(T, TOPK, E, N, K, nb.FP8_FWD)]),
    "experts_fp8_bwd": (lambda i, s: nb.nvfp4_experts_fp8_bwd(i.dy, i.We, i.x, i.plan, i.w, stream=s),
                        lambda: [nb.nvfp4_experts_fp8_workspace_bytes(T, TOPK, E, N, K, nb.FP8_BWD)]),
}


def _parts(plan):
    return plan.counts, plan.offsets, plan.row_of, plan.slot_of


def _tensors(out):
    return [t for t in (out if isinstance(out, tuple) else (out,)) if t is not None]


def _written(name, i, t):
    """What of an output the call writes: rows behind the last segment are left, few rows' products leave padding too, and codes' rows
    may have a pitch."""
    if "expert" in name and t.dim() == 2 and t.shape[0] == i.plan.rows:
        t = t[:i.used]
        if name == "gemm_fp8_experts":
            t = t[i.plan.slot_of[:i.used] >= 0]
    return t


@pytest.fixture(scope="module")
def inputs():
    # a kernel's first launch loads it, which waits for the device
    torch.cuda._sleep(1)
    torch.full((8,), 0x5A, dtype=torch.uint8, device="cuda").fill_(0x5A)
    for t in (torch.uint8, torch.int32, torch.bfloat16, torch.float32, torch.float64):
        torch.zeros(8, dtype=t, device="cuda").clone()
    return Inputs()


@pytest.mark.parametrize("name", CALLS)
def test_memory_of_a_call_is_not_given_away_while_it_runs(name, inputs):
    call, scratch = CALLS[name]
    sizes = [t.untyped_storage().nbytes() for t in _tensors(call(inputs, None))] + (scratch() if scratch else [])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    with torch.cuda.stream(side):
        torch.cuda._sleep(PAUSE)
    call(inputs, side)                                # its outputs are dropped at once
    # the current stream takes what blocks of these sizes there are
    later = [torch.full((n,), 0x5A, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(2)]
    torch.cuda.current_stream().synchronize()
    assert not side.query()                           # the call has not begun
    torch.cuda.synchronize()
    assert all(bool((t == 0x5A).all()) for t in later)


@pytest.mark.parametrize("name", CALLS)
def test_memory_of_a_call_is_not_written_by_work_queued_before_it(name, inputs):
    call, _ = CALLS[name]
    first = _tensors(call(inputs, None))
    want = [_written(name, inputs, t).clone() for t in first]
    sizes = [t.untyped_storage().nbytes() for t in first]
    del first
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    earlier = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(2)]
    torch.cuda._sleep(PAUSE)
    for t in earlier:
        t.fill_(0x5A)
    del earlier, t                                    # free on the current stream, written there in 150 ms
    got = _tensors(call(inputs, side))
    side.synchronize()
    assert not torch.cuda.current_stream().query()
    torch.cuda.synchronize()
    assert all(torch.equal(_written(name, inputs, g), w) for g, w in zip(got, want))


@pytest.mark.parametrize("name", CALLS)
def test_an_output_read_on_the_current_stream_and_dropped_is_not_written_by_the_next_call(name, inputs):
    call, _ = CALLS[name]
    want = [_written(name, inputs, t).clone() for t in _tensors(call(inputs, None))]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    got = _tensors(call(inputs, side))
    places = [t.data_ptr() for t in got]
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(PAUSE)
    read = [t.clone() for t in got]                   # in 150 ms
    del got
    again = _tensors(call(inputs, side))              # the same bits, so that places are what tells
    assert not set(places) & {t.data_ptr() for t in again}
    torch.cuda.synchronize()
    assert all(torch.equal(_written(name, inputs, g), w) for out in (read, again) for g, w in zip(out, want))


def test_a_chain_on_a_given_stream_that_drops_its_intermediate_results():
    i = Inputs()

    def chain(s, pause=lambda: None):
        plan = nb.nvfp4_expert_sort(i.expert_of, E, stream=s)
        codes, sf, _, _ = nb.nvfp4_quantize_fp8_experts(i.x, plan, stream=s)
        Y = nb.nvfp4_gemm_fp8_experts(codes, sf, *i.we8, plan, out_dtype=torch.bfloat16, stream=s)
        y = nb.nvfp4_expert_combine(Y, plan, i.w, stream=s)
        w = nb.nvfp4_quantize_fp8(i.W, 128, stream=s)[:2]
        h = nb.nvfp4_linear_fp8_fwd(i.X, i.W, out_dtype=torch.bfloat16, stream=s)
        return y, h, nb.nvfp4_gemm_fp8(*nb.nvfp4_quantize_fp8(i.X, stream=s)[:2], *w, stream=s)
    want = chain(None)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(PAUSE)
    got = chain(side)
    noise = [torch.full((n,), 0x5A, dtype=torch.uint8, device="cuda") for n in (1 << 10, 1 << 16, 1 << 18, 1 << 20, 1 << 22) for _ in range(8)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(bool((t == 0x5A).all()) for t in noise)


def test_two_layers_on_two_streams_that_are_only_named():
    layers = [(_x((1500, 1024), 10 + i), _x((2048, 1024), 20 + i, 0.05), _x((1500, 2048), 30 + i)) for i in range(2)]

    def step(layer, s):
        X, W, dY = layer
        return nb.nvfp4_linear_fp8_fwd(X, W, stream=s), *nb.nvfp4_linear_fp8_bwd(dY, W, X, stream=s), nb.nvfp4_linear_fwd(X, W, stream=s)
    want = []
    for layer in layers:
        want.append(step(layer, None))
        torch.cuda.synchronize()
    sides = [torch.cuda.Stream() for _ in layers]
    for _ in range(8):
        got = [step(layer, s) for layer, s in zip(layers, sides)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))
    assert nb.nvfp4_device_error_word() == 0


def test_a_given_stream_that_is_captured():
    i = Inputs()
    want = nb.nvfp4_linear_fp8_fwd(i.X, i.W)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        here = torch.cuda.current_stream()
        side.wait_stream(here)
        got = nb.nvfp4_linear_fp8_fwd(i.X, i.W, stream=side)
        same = nb.nvfp4_linear_fp8_fwd(i.X, i.W, stream=here)
        here.wait_stream(side)
    for _ in range(2):
        got.zero_(), same.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(same, want)


def test_the_default_stream_and_other_handles_are_streams_too():
    i = Inputs()
    want = nb.nvfp4_linear_fp8_fwd(i.X, i.W)
    side = torch.cuda.Stream()

    class Handle:                                     # what another library has in hand
        cuda_stream = side.cuda_stream

    class Default:
        cuda_stream = 0
    for s in (torch.cuda.default_stream(), Handle, Default, torch.cuda.ExternalStream(side.cuda_stream), torch.cuda.current_stream()):
        torch.cuda.synchronize()
        got = nb.nvfp4_linear_fp8_fwd(i.X, i.W, stream=s)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
    with torch.cuda.stream(side):
        got = nb.nvfp4_linear_fp8_fwd(i.X, i.W, stream=torch.cuda.default_stream())
        torch.cuda.synchronize()
        assert torch.equal(got, want)
