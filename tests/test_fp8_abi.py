"""FP8 and expert entry points: sizes, and arguments refused on the host before any launch (no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2505_19115_b200 import binding as nb

P, ODD = 0x1000, 0x1004           # never dereferenced: every call below fails validation first
BIG = 1 << 40


def test_sizes():
    assert nb.nvfp4_codes_bytes_fp8(3, 17) == 96 and nb.nvfp4_codes_bytes_fp8(0, 17) == 0
    assert nb.nvfp4_sf_bytes_fp8(3, 129, nb.SF_LINEAR) == 6
    assert nb.nvfp4_sf_bytes_fp8(129, 513, nb.SF_SWIZZLED) == 2 * 2 * 512
    assert nb.nvfp4_sf_bytes_fp8(129, 513, 2) == 0 and nb.nvfp4_sf_bytes_fp8(-1, 5, 0) == 0
    for which in (nb.FP8_FWD, nb.FP8_BWD):
        assert nb.nvfp4_linear_fp8_workspace_bytes(1, 512, 512, which) % 256 == 0 < nb.nvfp4_linear_fp8_workspace_bytes(1, 512, 512, which)
        assert nb.nvfp4_linear_fp8_workspace_bytes(16, 500, 512, which) == 0 == nb.nvfp4_linear_fp8_workspace_bytes(0, 512, 512, which)
        assert nb.nvfp4_experts_fp8_workspace_bytes(16, 2, 8, 64, 64, which) > 0 == nb.nvfp4_experts_fp8_workspace_bytes(16, 2, 1025, 64, 64, which)
    assert nb.nvfp4_linear_fp8_workspace_bytes(16, 512, 512, 2) == 0


@pytest.mark.parametrize("size,rows", [((1, 1, 1), 128), ((1, 8, 64), 1024), ((1, 8, 4), 512), ((100, 2, 3), 512), ((128, 1, 1), 128), ((129, 1, 1), 256)])
def test_expert_rows_hold_any_distribution(size, rows):
    T, k, E = size
    assert nb.nvfp4_expert_rows(T, k, E) == rows
    n = T * k
    spread = [n // min(n, E) + (i < n % min(n, E)) for i in range(min(n, E))]
    worst = [1] * (min(n, E) - 1) + [n - min(n, E) + 1]
    for counts in (spread, worst, [n]):
        assert sum(-(-c // 128) * 128 for c in counts) <= rows


def test_expert_rows_refuse():
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1, 1, 1025), (1 << 31, 1, 1), (1 << 30, 1 << 30, 8), (-1, 2, 2)):
        assert nb.nvfp4_expert_rows(*bad) == 0


def _call(name, defaults, status, **changes):
    args = [changes.get(k, v) for k, v in defaults.items()]
    assert set(changes) <= set(defaults)
    got = getattr(nb.lib(), name)(*[C.c_void_p(a) if isinstance(a, int) and k in POINTERS else a for (k, _), a in zip(defaults.items(), args)])
    assert got == status, (name, changes, got)


POINTERS = {"x", "cr", "sr", "ct", "st", "a", "asf", "b", "bsf", "d", "X", "W", "Y", "dY", "dX", "dW", "ws", "offsets", "slot", "row", "w", "rows", "y", "dy",
            "drows", "dw", "e", "counts", "stream"}


def test_quantizer_refusals():
    q = dict(x=P, dtype=0, batch=1, rows_=16, cols=32, ld=32, block=1, cr=P, sr=P, ct=P, st=P, layout=1, stream=None)
    for status, changes in ((1, dict(x=None)), (1, dict(cr=None)), (1, dict(st=None)), (1, dict(cr=None, sr=None, ct=None, st=None)), (4, dict(dtype=2)),
                            (4, dict(layout=2)), (4, dict(block=64)), (2, dict(batch=0)), (2, dict(rows_=0)), (2, dict(cols=-1)), (2, dict(ld=24)),
                            (2, dict(rows_=1 << 33)), (2, dict(batch=1 << 20, rows_=1 << 20, cols=1 << 20, ld=1 << 20)), (3, dict(x=ODD)), (3, dict(ld=36)),
                            (3, dict(cr=ODD)), (3, dict(st=ODD))):
        _call("nvfp4_quantize_fp8", q, status, **changes)


def test_product_refusals():
    g = dict(a=P, asf=P, b=P, bsf=P, M=1, N=8, K=100, d=P, dtype=1, ldd=8, stream=None)
    for status, changes in ((1, dict(a=None)), (1, dict(bsf=None)), (1, dict(d=None)), (4, dict(dtype=7)), (2, dict(M=0)), (2, dict(K=0)), (2, dict(ldd=4)),
                            (2, dict(M=BIG)), (2, dict(M=1 << 30, N=1 << 30, ldd=1 << 30)), (3, dict(a=ODD)), (3, dict(d=ODD)), (3, dict(ldd=10)), (3, dict(dtype=0, ldd=12))):
        _call("nvfp4_gemm_fp8", g, status, **changes)
    g = dict(a=P, asf=P, b=P, bsf=P, T=99, k=2, E=4, counts=P, offsets=P, N=8, K=100, d=P, dtype=1, ldd=8, stream=None)
    for status, changes in ((1, dict(a=None)), (1, dict(offsets=None)), (4, dict(dtype=7)), (2, dict(E=0)), (2, dict(E=1025)), (2, dict(T=0)), (2, dict(k=-1)),
                            (2, dict(E=1024, N=1 << 22, ldd=1 << 22)), (3, dict(offsets=0x1002)), (3, dict(counts=0x1002)), (3, dict(ldd=9))):
        _call("nvfp4_gemm_fp8_experts", g, status, **changes)
    g = dict(a=P, asf=P, b=P, bsf=P, T=99, k=2, E=4, offsets=P, N=8, K=104, d=P, dtype=1, stream=None)
    for status, changes in ((1, dict(b=None)), (1, dict(offsets=None)), (4, dict(dtype=7)), (2, dict(E=1025)), (2, dict(T=0)), (2, dict(N=0)), (3, dict(K=102)), (3, dict(d=ODD))):
        _call("nvfp4_gemm_fp8_experts_dw", g, status, **changes)


def test_layer_refusals():
    f = dict(X=P, W=P, dtype=0, M=7, N=64, K=64, Y=P, ydtype=1, ws=P, wsb=1 << 30, stream=None)
    for status, changes in ((1, dict(X=None)), (1, dict(Y=None)), (4, dict(dtype=5)), (4, dict(ydtype=5)), (2, dict(M=0)), (2, dict(N=60)), (2, dict(K=4)), (2, dict(M=BIG)),
                            (3, dict(W=ODD)), (3, dict(Y=ODD)), (5, dict(ws=None)), (5, dict(wsb=100)), (5, dict(ws=0x1010))):
        _call("nvfp4_linear_fp8_fwd", f, status, **changes)
    b = dict(dY=P, W=P, X=P, dtype=0, M=7, N=64, K=64, dX=P, dxdtype=1, dW=P, dwdtype=1, ws=P, wsb=1 << 30, stream=None)
    for status, changes in ((1, dict(dY=None)), (1, dict(dW=None)), (4, dict(dxdtype=5)), (4, dict(dwdtype=-1)), (2, dict(N=63)), (3, dict(dX=ODD)), (5, dict(ws=None)), (5, dict(wsb=0))):
        _call("nvfp4_linear_fp8_bwd", b, status, **changes)


def test_routing_refusals():
    s = dict(e=P, wide=0, T=4, k=2, E=8, counts=P, offsets=P, row=P, slot=P, stream=None)
    for status, changes in ((1, dict(e=None)), (1, dict(slot=None)), (4, dict(wide=2)), (2, dict(T=0)), (2, dict(E=1025)), (2, dict(k=0)), (3, dict(e=0x1002)), (3, dict(e=ODD, wide=1)),
                            (3, dict(row=0x1001))):
        _call("nvfp4_expert_sort", s, status, **changes)
    g = dict(x=P, dtype=0, T=4, k=2, E=8, cols=64, ld=64, offsets=P, slot=P, row=P, w=P, wdtype=1, rows=P, stream=None)
    for status, changes in ((1, dict(x=None)), (1, dict(offsets=None)), (4, dict(dtype=3)), (4, dict(wdtype=3)), (2, dict(cols=60)), (2, dict(ld=56)), (2, dict(T=0)), (3, dict(x=ODD)),
                            (3, dict(ld=68)), (3, dict(w=0x1002)), (3, dict(rows=ODD))):
        _call("nvfp4_expert_gather", g, status, **changes)
    c = dict(rows=P, dtype=0, T=4, k=2, E=8, cols=64, row=P, w=P, wdtype=0, y=P, stream=None)
    for status, changes in ((1, dict(rows=None)), (1, dict(row=None)), (4, dict(dtype=3)), (2, dict(cols=0)), (2, dict(E=0)), (3, dict(y=ODD)), (3, dict(w=0x1001))):
        _call("nvfp4_expert_combine", c, status, **changes)
    b = dict(dy=P, dtype=0, T=4, k=2, E=8, cols=64, ld=64, offsets=P, slot=P, row=P, rows=P, w=P, wdtype=1, drows=None, dw=P, stream=None)
    for status, changes in ((1, dict(dy=None)), (1, dict(w=None)), (1, dict(dw=None)), (4, dict(wdtype=9)), (2, dict(cols=12)), (2, dict(k=-1)), (3, dict(drows=ODD)), (3, dict(dw=0x1002))):
        _call("nvfp4_expert_combine_bwd", b, status, **changes)


def test_experts_refusals():
    q = dict(x=P, dtype=0, by=1, T=4, k=2, E=8, cols=60, ld=64, offsets=P, slot=P, w=None, wdtype=0, cr=P, sr=P, ct=None, st=None, stream=None)
    for status, changes in ((1, dict(x=None)), (1, dict(cr=None)), (1, dict(slot=None)), (4, dict(by=2)), (4, dict(wdtype=4)), (2, dict(ld=56)), (2, dict(T=0)), (3, dict(x=ODD)), (3, dict(ld=60)),
                            (3, dict(w=0x1001)), (3, dict(sr=ODD))):
        _call("nvfp4_quantize_fp8_experts", q, status, **changes)
    f = dict(X=P, by=1, W=P, dtype=0, T=4, k=2, E=8, N=64, K=64, offsets=P, slot=P, Y=P, ydtype=0, ws=P, wsb=1 << 30, stream=None)
    for status, changes in ((1, dict(W=None)), (1, dict(offsets=None)), (4, dict(by=-1)), (4, dict(ydtype=2)), (2, dict(N=60)), (2, dict(E=1025)), (2, dict(T=0)), (3, dict(Y=ODD)), (3, dict(slot=0x1001)),
                            (5, dict(ws=None)), (5, dict(wsb=1))):
        _call("nvfp4_experts_fp8_fwd", f, status, **changes)
    b = dict(dY=P, by=1, w=None, wdtype=0, W=P, X=P, xby=1, dtype=0, T=4, k=2, E=8, N=64, K=64, offsets=P, slot=P, dX=P, dxdtype=0, dW=P, dwdtype=1, ws=P, wsb=1 << 30, stream=None)
    for status, changes in ((1, dict(dY=None)), (1, dict(dX=None)), (4, dict(xby=2)), (4, dict(wdtype=2)), (2, dict(K=60)), (3, dict(dW=ODD)), (3, dict(w=0x1001)), (5, dict(ws=0x1001))):
        _call("nvfp4_experts_fp8_bwd", b, status, **changes)


def test_codes_that_are_not_laid_out_as_the_quantizer_leaves_them_are_refused():
    good = torch.zeros((4, 32), dtype=torch.uint8)
    sf = torch.zeros(512, dtype=torch.uint8)
    for bad in (torch.zeros((4, 24), dtype=torch.uint8), torch.zeros((4, 64), dtype=torch.uint8)[:, :32], good.T, torch.zeros((4, 32), dtype=torch.int16)):
        with pytest.raises(ValueError):
            nb.nvfp4_gemm_fp8(bad, sf, good, sf, out=torch.zeros((4, 4)))


def test_scales_of_another_layout_are_refused():
    # the products would read behind them
    good, sf = torch.zeros((200, 528), dtype=torch.uint8), torch.zeros(2 * 2 * 512, dtype=torch.uint8)
    n = nb._native()
    assert n.fp8_operand(good, sf) == (1, 200, 528)
    assert n.fp8_operand(good[:, :520], sf) == (1, 200, 520)
    assert n.fp8_operand(good.view(4, 50, 528), torch.zeros(4 * 2 * 512, dtype=torch.uint8)) == (4, 50, 528)
    for bad in (torch.zeros((200, 5), dtype=torch.uint8), sf[:-1], torch.zeros(512, dtype=torch.int32), torch.zeros(4096, dtype=torch.uint8)[::2]):
        for operands in ((good, bad, good, sf), (good, sf, good, bad)):
            with pytest.raises(ValueError):
                nb.nvfp4_gemm_fp8(*operands, out=torch.zeros((200, 200)))
    for bad in ((good,), (good, None), (1, sf)):
        with pytest.raises(TypeError):
            n.fp8_operand(*bad)


def test_expert_choices_are_whole_numbers():
    class OnDevice(torch.Tensor):
        is_cuda = True
    with pytest.raises(TypeError):
        nb.nvfp4_expert_sort(torch.zeros((2, 2)).as_subclass(OnDevice), 4)


HERE = ("nvfp4_quantize_fp8", "nvfp4_gemm_fp8", "nvfp4_linear_fp8_fwd", "nvfp4_linear_fp8_bwd", "nvfp4_expert_sort", "nvfp4_expert_gather", "nvfp4_expert_combine",
        "nvfp4_expert_combine_bwd", "nvfp4_quantize_fp8_experts", "nvfp4_gemm_fp8_experts", "nvfp4_gemm_fp8_experts_dw", "nvfp4_experts_fp8_fwd", "nvfp4_experts_fp8_bwd")


@pytest.mark.parametrize("name", HERE)
def test_tensors_elsewhere_are_refused(name):
    # a kernel would read a host tensor's address, or another device's memory, on the current device
    argtypes = getattr(nb.lib(), name).argtypes
    class Stream:
        cuda_stream = 0
    args = [None if t is C.c_void_p else 0 for t in argtypes[:-1]] + [Stream]
    for i, t in enumerate(argtypes[:-1]):
        if t is C.c_void_p:
            with pytest.raises((ValueError, RuntimeError)):       # RuntimeError: no CUDA device to be current
                getattr(nb._native(), name)(*args[:i], torch.zeros(64), *args[i + 1:])


def test_outputs_are_laid_out_as_the_calls_take_them():
    n, like = nb._native(), torch.zeros(1)
    codes, sf, codes_t, sf_t = n.empty_fp8(like, 0, 130, 24, 1, 1, nb.SF_SWIZZLED)
    assert codes.shape == (130, 24) and codes.stride() == (32, 1) and codes_t.shape == (24, 130) and codes_t.stride() == (144, 1)
    assert codes.untyped_storage().nbytes() == nb.nvfp4_codes_bytes_fp8(130, 24) and sf.numel() == nb.nvfp4_sf_bytes_fp8(130, 24)
    assert codes_t.untyped_storage().nbytes() == nb.nvfp4_codes_bytes_fp8(24, 130) and sf_t.numel() == nb.nvfp4_sf_bytes_fp8(24, 130)
    codes, sf, none, none_t = n.empty_fp8(like, 3, 130, 264, 1, 0, nb.SF_LINEAR)
    assert codes.shape == (3, 130, 264) and codes.stride() == (130 * 272, 272, 1) and sf.shape == (3, 130, 3) and none is none_t is None
    assert [t.shape for t in n.expert_buffers(like, 5, 2, 3, 256)] == [(3,), (4,), (5, 2), (256,)]
    assert n.empty_rows(like.to(torch.bfloat16), 4, 8).dtype == torch.bfloat16
    for bad in (lambda: n.empty_fp8(like, 0, 1, 1, 1, 0), lambda: n.empty_fp8(5, 0, 1, 1, 1, 0, 1), lambda: n.empty_rows(like, 1.5, 8), lambda: n.expert_buffers(like, 1, 1, 1, None)):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(RuntimeError):
        n.empty_rows(like, -1, 8)


def test_shapes_are_read_as_the_calls_take_them():
    n, t = nb._native(), torch.zeros((6, 40))
    assert n.matrix(t, 6) == (40, 40) and n.matrix(t[:, :24], 6) == (24, 40) and n.matrix(t[1:2, :12], 1) == (12, 16)
    for bad in (lambda: n.matrix(t, 5), lambda: n.matrix(t.T, 40), lambda: n.matrix(t[0], 40)):
        with pytest.raises(ValueError):
            bad()
    assert n.dense(t, None, 6, 40) and n.dense(t, t, 6, 40) and n.dense(t.view(2, 3, 40), t, 2, 3, 40)
    for bad in ((t, None, 6, 41), (t, None, 240), (t, t.half(), 6, 40), (t[:, :8], None, 6, 8), (t.T, None, 40, 6)):
        assert not n.dense(*bad)
    for bad in (lambda: n.matrix(t), lambda: n.matrix(5, 6), lambda: n.dense(t), lambda: n.dense(None, None, 1), lambda: n.dense(t, 5, 6, 40)):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises((ValueError, RuntimeError)):                   # a host tensor; RuntimeError: no CUDA device to be current
        nb.nvfp4_quantize_fp8(torch.zeros((8, 8)))
