"""Performance cases of the 8-bit floating point operators and of the layers whose weights are split among experts.

A case is a dict of plain values; its "op" names the sequence of calls.  Sizes are those of the Llama blocks in synth.py
(hidden 1024 or 4096, inner 2816 or 11008) and generic ones around them.

  linear    one training step of one linear layer in FP8, blocks of 128: nvfp4_linear_fp8_fwd + nvfp4_linear_fp8_bwd
  kept      evaluation with weights quantized once: activations quantized, one product
  quantize  the quantizer alone, row and transposed output
  route     tokens sorted by expert, gathered, combined with weights, and the gradients of both
  experts   one training step of a layer of experts: sort, product on gathered rows, combine, and all gradients
  decode    a layer of experts with weights quantized once, for few tokens: sort, quantize, product, combine
"""
import math

import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "fp32": torch.float32}
_BYTES = {"bf16": 2, "fp32": 4}
BLOCK = 128


def listed():
    return [
        # the single small layer: launches and host time are what it costs
        dict(name="linear_small_256", op="linear", M=256, K=512, N=512, x="bf16", y="fp32"),
        # 7B-class gate projection, bf16 activations, fp32 weight gradient: the bulk of a training step
        dict(name="linear_7b_gate", op="linear", M=16384, K=4096, N=11008, x="bf16", y="bf16"),
        # a short, odd micro-batch with fp32 tensors: no size a multiple of a block
        dict(name="linear_odd_2077", op="linear", M=2077, K=1064, N=2840, x="fp32", y="fp32"),
        # evaluation of a single token on kept weights
        dict(name="kept_7b_1_token", op="kept", M=1, K=4096, N=11008, y="bf16"),
        # evaluation of a ragged handful of tokens, down projection
        dict(name="kept_7b_67_tokens", op="kept", M=67, K=11008, N=4096, y="fp32"),
        # activations quantized for the forward product and for the weight gradient
        dict(name="quantize_8192", op="quantize", rows=8192, cols=8192, x="bf16", block_rows=1),
        # fp32 weights in square blocks, sizes that fill no block
        dict(name="quantize_weights_odd", op="quantize", rows=2840, cols=1064, x="fp32", block_rows=128),
        # routing of one token: launches are what it costs
        dict(name="route_1_token", op="route", T=1, topk=8, E=64, H=1024, x="bf16", w="fp32", drop=0.0),
        # routing of a training batch, some tokens beyond their experts' capacity
        dict(name="route_16384", op="route", T=16384, topk=2, E=8, H=4096, x="bf16", w="fp32", drop=0.02),
        # a few tokens through kept experts: many small matrices, most of them read for one or two rows
        dict(name="decode_16_tokens", op="decode", T=16, topk=8, E=64, K=1024, N=2816, w="fp32"),
        # training step of the 350M-class gate projection split among eight experts
        dict(name="experts_350m", op="experts", T=16384, topk=2, E=8, K=1024, N=2816, x="bf16", w="bf16", drop=0.0),
        # many uneven experts, odd sizes, dropped assignments
        dict(name="experts_ragged", op="experts", T=3001, topk=6, E=61, K=1064, N=712, x="bf16", w="bf16", drop=0.02),
    ]


def _log(rng, lo, hi, step):
    """A multiple of `step` in [lo, hi], spread evenly over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(-(-lo // step) * step, min(hi // step * step, int(round(v / step)) * step))


def draw(rng):
    op = rng.choice(["linear", "linear", "kept", "quantize", "route", "experts", "experts", "decode"])
    if op == "linear":
        return dict(op=op, M=_log(rng, 256, 16384, 1), K=_log(rng, 512, 4096, 8), N=_log(rng, 512, 11008, 8),
                    x=rng.choice(["bf16", "bf16", "fp32"]), y=rng.choice(["bf16", "fp32"]))
    if op == "kept":
        return dict(op=op, M=_log(rng, 1, 512, 1), K=_log(rng, 512, 11008, 8), N=_log(rng, 512, 11008, 8), y=rng.choice(["bf16", "fp32"]))
    if op == "quantize":
        return dict(op=op, rows=_log(rng, 512, 8192, 1), cols=_log(rng, 512, 8192, 8), x=rng.choice(["bf16", "bf16", "fp32"]),
                    block_rows=rng.choice([1, 1, 128]))
    E = rng.choice([4, 8, 16, 33, 61, 64])
    topk = rng.choice([1, 2, 2, 4])
    drop = rng.choice([0.0, 0.0, 0.02])
    if op == "route":
        return dict(op=op, T=_log(rng, 1, 16384, 1), topk=topk, E=E, H=_log(rng, 512, 4096, 8), x=rng.choice(["bf16", "bf16", "fp32"]),
                    w="fp32", drop=drop)
    if op == "decode":
        return dict(op=op, T=_log(rng, 1, 48, 1), topk=topk, E=E, K=_log(rng, 512, 1024, 8), N=_log(rng, 512, 2816, 8), w="fp32")
    return dict(op=op, T=_log(rng, 256, 8192, 1), topk=topk, E=E, K=_log(rng, 512, 1064, 8), N=_log(rng, 512, 2816, 8), x="bf16",
                w="bf16", drop=drop)


# ---------------------------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------------------------
def _normal(shape, std, g, dtype):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(_TORCH[dtype])


def _rows(tokens, topk, experts):
    """Rows that the segments of all experts, each a multiple of 128 rows long, take at most."""
    n = tokens * topk
    return (n + (BLOCK - 1) * min(n, experts)) // BLOCK * BLOCK


def _routing(T, topk, E, drop, g, w):
    """Distinct experts for every token, some more wanted than others; -1: beyond the expert's capacity.  Weights sum to one."""
    scores = torch.randn((T, E), generator=g, device="cuda") + 0.5 * torch.randn((1, E), generator=g, device="cuda")
    value, expert = scores.topk(topk, dim=1)
    lost = torch.rand((T, topk), generator=g, device="cuda") < drop
    return torch.where(lost, -1, expert).to(torch.int32), torch.softmax(value, 1).to(_TORCH[w])


def prepare(case, seed):
    s = dict(case)
    op = case["op"]
    g = torch.Generator("cuda")
    g.manual_seed(int(seed))
    if op == "quantize":
        x = _normal((case["rows"], case["cols"]), 1.0, g, case["x"])
        # activations and weights have rows and channels of very different size
        s["x"] = x * torch.exp2(torch.randint(-6, 7, (case["rows"], 1), generator=g, device="cuda")).to(x.dtype)
        return s
    if op in ("route", "experts", "decode"):
        T, topk, E = case["T"], case["topk"], case["E"]
        s["expert_of"], s["weights"] = _routing(T, topk, E, case.get("drop", 0.0), g, case["w"])
        R = s["R"] = _rows(T, topk, E)
        if op == "route":
            s["x"], s["dy"] = _normal((T, case["H"]), 1.0, g, case["x"]), _normal((T, case["H"]), 1e-2, g, case["x"])
            # rows behind the last segment stay as they are
            s["rows"], s["drows"] = (torch.zeros((R, case["H"]), dtype=_TORCH[case["x"]], device="cuda") for _ in range(2))
            return s
        K, N = case["K"], case["N"]
        s["x"] = _normal((T, K), 1.0, g, case.get("x", "bf16"))
        W = _normal((E, N, K), 0.02, g, "bf16")
        s["Y"] = torch.zeros((R, N), dtype=torch.bfloat16, device="cuda")
        if op == "experts":
            s["W"], s["dy"] = W, _normal((T, N), 1e-3, g, case["x"])
            s["dX"] = torch.zeros((R, K), dtype=torch.bfloat16, device="cuda")
            s["dW"] = torch.empty((E, N, K), dtype=torch.float32, device="cuda")
        else:
            s["w_codes"], s["w_scales"] = _kept(W.float())
        return s
    M, K, N = case["M"], case["K"], case["N"]
    x = case.get("x", "bf16")
    s["X"] = _normal((M, K), 1.0, g, x)
    W = _normal((N, K), 0.02, g, x)
    s["Y"] = torch.empty((M, N), dtype=_TORCH[case["y"]], device="cuda")
    if op == "kept":
        s["w_codes"], s["w_scales"] = _kept(W.float())
        return s
    s["W"], s["dY"] = W, _normal((M, N), 1e-3, g, x)
    s["dX"] = torch.empty((M, K), dtype=_TORCH[case["y"]], device="cuda")
    s["dW"] = torch.empty((N, K), dtype=torch.float32, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------------------------------
# The format in elementary operations: E4M3 values, a power-of-two scale for a block of 128 (or 128 x 128)
# ---------------------------------------------------------------------------------------------------------------------
def _up(n, m):
    return -(-n // m) * m


def _quantized(x, block_rows=1):
    """fp32 x [..., R, C] -> codes (float8, [..., R, C]) and E8M0 scale codes (int32, [..., R, ceil(C / 128)])."""
    R, C = x.shape[-2:]
    p = torch.nn.functional.pad(x, (0, _up(C, BLOCK) - C, 0, _up(R, block_rows) - R))
    blocks = p.unflatten(-1, (-1, BLOCK)).unflatten(-3, (-1, block_rows))                 # [..., R/b, b, C/128, 128]
    amax = blocks.abs().amax((-3, -1), keepdim=True)
    # the smallest power of two that brings amax to 448 = 1.75 * 2^8 or less: one more where the mantissa is above 1.75
    code = (((amax.view(torch.int32) + 0x1FFFFF) >> 23) - 8).clamp_(min=0)
    codes = (blocks * ((254 - code) << 23).view(torch.float32)).to(torch.float8_e4m3fn)
    code = code.expand(*blocks.shape[:-1], 1).flatten(-4, -3).squeeze(-1)[..., :R, :]
    return codes.flatten(-4, -3).flatten(-2)[..., :R, :C], code


def _scale(code):
    return torch.where(code > 0, code << 23, 0x400000).view(torch.float32)               # 2^(code - 127); code 0: 2^-127


def _values(x, block_rows=1):
    """What x is after quantization, fp32."""
    codes, code = _quantized(x, block_rows)
    return codes.float() * _scale(code).repeat_interleave(BLOCK, -1)[..., : x.shape[-1]]


def _tiled(code):
    """Scale codes [..., R, nb] -> tiles of 128 rows x 4 blocks, 512 bytes each (the layout that the product reads)."""
    R, nb = code.shape[-2:]
    p = torch.nn.functional.pad(code, (0, _up(nb, 4) - nb, 0, _up(R, 128) - R)).to(torch.uint8)
    t = p.unflatten(-1, (-1, 4)).unflatten(-3, (-1, 4, 32))                                # [..., R/128, 4, 32, nb/4, 4]
    return t.movedim(-2, -4).movedim(-2, -3).reshape(-1)                                    # [..., R/128, nb/4, 32, 4, 4]


def _untiled(tiles, lead, R, nb):
    t = tiles.view(*lead, _up(R, 128) // 128, _up(nb, 4) // 4, 32, 4, 4)
    return t.movedim(-2, -3).movedim(-4, -2).flatten(-2).flatten(-4, -2)[..., :R, :nb].int()


def _pitched(codes):
    """Codes with rows of a multiple of 16 bytes, as a view of the given width."""
    C = codes.shape[-1]
    padded = torch.zeros((*codes.shape[:-1], _up(C, 16)), dtype=torch.uint8, device=codes.device)
    padded[..., :C] = codes.view(torch.uint8)
    return padded[..., :C]


def _kept(W):
    """Weights [..., N, K] quantized once in blocks of 128 x 128: codes and tiled scales."""
    codes, code = _quantized(W, 128)
    return _pitched(codes), _tiled(code)


def _kept_values(s, N, K):
    codes = s["w_codes"].view(torch.float8_e4m3fn).float()
    code = _untiled(s["w_scales"], codes.shape[:-2], N, -(-K // BLOCK))
    return codes * _scale(code).repeat_interleave(BLOCK, -1)[..., :K]


# ---------------------------------------------------------------------------------------------------------------------
# Routing in elementary operations
# ---------------------------------------------------------------------------------------------------------------------
def _sorted(expert_of, E, R):
    """counts [E], offsets [E + 1], row_of [T, k] (-1: dropped), slot_of [R] (-1: padding)."""
    flat = expert_of.reshape(-1).long()
    valid = (flat >= 0) & (flat < E)
    one = (flat[:, None] == torch.arange(E, device=flat.device)).int()
    counts = one.sum(0)
    offsets = torch.nn.functional.pad(((counts + BLOCK - 1) // BLOCK * BLOCK).cumsum(0), (1, 0))
    rank = (one.cumsum(0) * one).sum(1) - 1
    row_of = torch.where(valid, offsets[flat.clamp(0, E - 1)] + rank, -1)
    slot_of = torch.full((R + 1,), -1, dtype=torch.int64, device=flat.device)
    slot_of[torch.where(valid, row_of, R)] = torch.arange(flat.numel(), device=flat.device)
    return counts.int(), offsets.int(), row_of.view_as(expert_of).int(), slot_of[:R].int()


def _gathered(x, slot_of, topk, weights=None, to=torch.float32):
    slot = slot_of.long().clamp(min=0)
    rows = x[slot // topk].to(to)
    if weights is not None:
        rows = rows * weights.reshape(-1)[slot].to(to)[:, None]
    return torch.where(slot_of[:, None] >= 0, rows, 0)


def _combined(rows, row_of, weights=None, to=torch.float32):
    picked = torch.where(row_of[..., None] >= 0, rows[row_of.long().clamp(min=0)].to(to), 0)
    if weights is not None:
        picked = picked * weights.to(to)[..., None]
    return picked.sum(1)


def _weight_gradient(dy, rows, row_of, to=torch.float32):
    dots = (rows[row_of.long().clamp(min=0)].to(to) * dy.to(to)[:, None, :]).sum(-1)
    return torch.where(row_of >= 0, dots, 0)


def _expert_of_block(offsets, R, E):
    at = torch.arange(0, R, BLOCK, device=offsets.device)
    return torch.searchsorted(offsets[1:].long().contiguous(), at, right=True).clamp(max=E - 1)


# ---------------------------------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_plain(s):
    op = s["op"]
    if op == "linear":
        X, W, dY = s["X"].float(), s["W"].float(), s["dY"].float()
        Wq = _values(W, 128)
        return {"Y": (_values(X) @ Wq.T).to(s["Y"].dtype), "dX": (_values(dY) @ Wq).to(s["dX"].dtype),
                "dW": _values(dY.T) @ _values(X.T).T}
    if op == "kept":
        return {"Y": (_values(s["X"].float()) @ _kept_values(s, s["N"], s["K"]).T).to(s["Y"].dtype)}
    if op == "quantize":
        x = s["x"].float()
        codes, code = _quantized(x, s["block_rows"])
        if s["block_rows"] == 1:
            codes_t, code_t = _quantized(x.T)
        else:
            codes_t, code_t = codes.T, code[::128].repeat_interleave(128, 1)[:, : s["cols"]].T
        return {"codes": codes, "scales": _tiled(code), "codes_t": codes_t, "scales_t": _tiled(code_t)}
    topk, E, R = s["topk"], s["E"], s["R"]
    counts, offsets, row_of, slot_of = _sorted(s["expert_of"], E, R)
    plan = {"counts": counts, "offsets": offsets, "row_of": row_of, "slot_of": slot_of}
    if op == "route":
        rows = _gathered(s["x"], slot_of, topk).to(s["x"].dtype)
        drows = _gathered(s["dy"], slot_of, topk, s["weights"]).to(s["x"].dtype)
        return {**plan, "rows": rows, "y": _combined(rows, row_of, s["weights"]).to(s["x"].dtype), "drows": drows,
                "dw": _weight_gradient(s["dy"], rows, row_of), "dx": _combined(drows, row_of).to(s["x"].dtype)}
    N, K = s["N"], s["K"]
    of = _expert_of_block(offsets, R, E)
    Wq = _values(s["W"].float(), 128) if op == "experts" else _kept_values(s, N, K)
    rows = _gathered(s["x"], slot_of, topk)
    Y = torch.bmm(_values(rows).view(-1, BLOCK, K), Wq[of].transpose(1, 2)).view(R, N).to(s["Y"].dtype)
    y = _combined(Y, row_of, s["weights"]).to(s["x"].dtype)
    if op == "decode":
        return {**plan, "y": y}
    drows = _gathered(s["dy"], slot_of, topk, s["weights"])
    dX = torch.bmm(_values(drows).view(-1, BLOCK, N), Wq[of]).view(R, K).to(s["dX"].dtype)
    part = torch.bmm(_values(drows.T).view(N, -1, BLOCK).transpose(0, 1), _values(rows.T).view(K, -1, BLOCK).permute(1, 2, 0))
    dW = torch.zeros_like(s["dW"]).index_add_(0, of, part)
    return {**plan, "y": y, "dx": _combined(dX, row_of).to(s["x"].dtype), "dW": dW,
            "dw": _weight_gradient(s["dy"], Y, row_of).to(s["weights"].dtype)}


def _scratch(s, name, nbytes):
    """The program's workspace: allocated at the first pass and kept."""
    if name not in s:
        s[name] = torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device="cuda")
    return s[name]


def _run_own(s):
    from paper_2505_19115_b200 import binding as nb
    op = s["op"]
    if op == "linear":
        M, N, K = s["M"], s["N"], s["K"]
        if "ws" not in s:
            _scratch(s, "ws", max(nb.nvfp4_linear_fp8_workspace_bytes(M, N, K, w) for w in (nb.FP8_FWD, nb.FP8_BWD)))
        Y = nb.nvfp4_linear_fp8_fwd(s["X"], s["W"], out=s["Y"], workspace=s["ws"])
        dX, dW = nb.nvfp4_linear_fp8_bwd(s["dY"], s["W"], s["X"], dX=s["dX"], dW=s["dW"], workspace=s["ws"])
        return {"Y": Y, "dX": dX, "dW": dW}
    if op == "kept":
        codes, scales, _, _ = nb.nvfp4_quantize_fp8(s["X"])
        return {"Y": nb.nvfp4_gemm_fp8(codes, scales, s["w_codes"], s["w_scales"], out=s["Y"])}
    if op == "quantize":
        codes, scales, codes_t, scales_t = nb.nvfp4_quantize_fp8(s["x"], block_rows=s["block_rows"], transposed=True)
        return {"codes": codes.view(torch.float8_e4m3fn), "scales": scales, "codes_t": codes_t.view(torch.float8_e4m3fn), "scales_t": scales_t}
    plan = nb.nvfp4_expert_sort(s["expert_of"], s["E"])
    said = {"counts": plan.counts, "offsets": plan.offsets, "row_of": plan.row_of, "slot_of": plan.slot_of}
    if op == "route":
        rows = nb.nvfp4_expert_gather(s["x"], plan, out=s["rows"])
        y = nb.nvfp4_expert_combine(rows, plan, s["weights"])
        drows, dw = nb.nvfp4_expert_combine_bwd(s["dy"], rows, plan, s["weights"], drows=s["drows"])
        return {**said, "rows": rows, "y": y, "drows": drows, "dw": dw, "dx": nb.nvfp4_expert_combine(drows, plan)}
    if op == "decode":
        codes, scales, _, _ = nb.nvfp4_quantize_fp8_experts(s["x"], plan)
        Y = nb.nvfp4_gemm_fp8_experts(codes, scales, s["w_codes"], s["w_scales"], plan, out=s["Y"])
        return {**said, "y": nb.nvfp4_expert_combine(Y, plan, s["weights"])}
    if "ws" not in s:
        _scratch(s, "ws", max(nb.nvfp4_experts_fp8_workspace_bytes(s["T"], s["topk"], s["E"], s["N"], s["K"], w) for w in (nb.FP8_FWD, nb.FP8_BWD)))
    Y = nb.nvfp4_experts_fp8_fwd(s["x"], s["W"], plan, out=s["Y"], workspace=s["ws"])
    y = nb.nvfp4_expert_combine(Y, plan, s["weights"])
    _, dw = nb.nvfp4_expert_combine_bwd(s["dy"], Y, plan, s["weights"], rows_gradient=False)
    dX, dW = nb.nvfp4_experts_fp8_bwd(s["dy"], s["W"], s["x"], plan, weights=s["weights"], dX=s["dX"], dW=s["dW"], workspace=s["ws"])
    return {**said, "y": y, "dx": nb.nvfp4_expert_combine(dX, plan), "dW": dW, "dw": dw}


# ---------------------------------------------------------------------------------------------------------------------
# The definition in 64 bits, written apart from the above
# ---------------------------------------------------------------------------------------------------------------------
def _two_to(e):
    return ((e.long() + 1023) << 52).view(torch.float64)                                   # no rounding, unlike a power function's


def _exact_codes(x, along_rows=1):
    """Double x [R, C] -> (code values, exponents) of blocks of along_rows x 128; the grid is spelt out."""
    R, C = x.shape
    up = torch.zeros((_up(R, along_rows), _up(C, 128)), dtype=torch.float64, device=x.device)
    up[:R, :C] = x
    b = up.view(up.shape[0] // along_rows, along_rows, up.shape[1] // 128, 128)
    m, e = torch.frexp(b.abs().amax(dim=(1, 3)))                                          # amax = m 2^e, m in [1/2, 1)
    e = torch.where(m > 0, e - 9 + (m > 0.875).int(), -127).clamp(min=-127)                # 448 = 0.875 * 2^9
    y = b * _two_to(-e)[:, None, :, None]
    _, ey = torch.frexp(y)
    step = _two_to((ey - 4).clamp(min=-9))                                                  # three bits behind the leading one
    y = torch.round(y / step) * step                                                        # ties to even
    e = e[:, None, :].expand(-1, along_rows, -1).reshape(up.shape[0], -1)
    return y.view_as(up)[:R, :C], e[:R]


def _exact_values(x, along_rows=1):
    y, e = _exact_codes(x, along_rows)
    return y * _two_to(e)[:, :, None].expand(-1, -1, 128).reshape(e.shape[0], -1)[:, : x.shape[1]]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "linear":
        X, W, dY = s["X"].double(), s["W"].double(), s["dY"].double()
        Wq = _exact_values(W, 128)
        return {"Y": _exact_values(X) @ Wq.T, "dX": _exact_values(dY) @ Wq, "dW": _exact_values(dY.T) @ _exact_values(X.T).T}
    if op == "kept":
        Wq = _kept_values(s, case["N"], case["K"]).double()      # kept weights are an input: powers of two times 8-bit values, exact in fp32
        return {"Y": _exact_values(s["X"].double()) @ Wq.T}
    if op == "quantize":
        y, _ = _exact_codes(s["x"].double(), case["block_rows"])
        yt = y.T if case["block_rows"] == 128 else _exact_codes(s["x"].double().T)[0]
        return {"codes": y, "scales": None, "codes_t": yt, "scales_t": None}
    T, topk, E, R = case["T"], case["topk"], case["E"], s["R"]
    expert_of, w = s["expert_of"].cpu().tolist(), s["weights"].double()
    segments = [[] for _ in range(E)]
    for t in range(T):
        for j in range(topk):
            if 0 <= expert_of[t][j] < E:
                segments[expert_of[t][j]].append(t * topk + j)
    begin, at = [], 0
    for members in segments:
        begin.append(at)
        at += -(-len(members) // 128) * 128
    pad = {"counts": None, "offsets": None, "row_of": None, "slot_of": None}
    if op == "route":
        H = case["H"]
        x, dy = s["x"].double(), s["dy"].double()
        rows, drows = torch.zeros((2, R, H), dtype=torch.float64, device="cuda")
        y, dx = torch.zeros((2, T, H), dtype=torch.float64, device="cuda")
        dw = torch.zeros(T * topk, dtype=torch.float64, device="cuda")
        for e, members in enumerate(segments):
            if not members:
                continue
            slot = torch.tensor(members, device="cuda")
            t, ws = slot // topk, w.reshape(-1)[slot][:, None]
            rows[begin[e] : begin[e] + len(members)] = x[t]
            drows[begin[e] : begin[e] + len(members)] = ws * dy[t]
            y.index_add_(0, t, ws * x[t])
            dx.index_add_(0, t, ws * dy[t])
            dw[slot] = (x[t] * dy[t]).sum(1)
        return {**pad, "rows": rows, "y": y, "drows": drows, "dw": dw.view(T, topk), "dx": dx}
    N, K = case["N"], case["K"]
    kept = _kept_values(s, N, K).double() if op == "decode" else None
    x, y = s["x"].double(), torch.zeros((T, N), dtype=torch.float64, device="cuda")
    if op == "experts":
        dy, dx = s["dy"].double(), torch.zeros((T, K), dtype=torch.float64, device="cuda")
        dW, dw = torch.zeros((E, N, K), dtype=torch.float64, device="cuda"), torch.zeros(T * topk, dtype=torch.float64, device="cuda")
    for e, members in enumerate(segments):
        if not members:
            continue
        slot = torch.tensor(members, device="cuda")
        t, ws = slot // topk, w.reshape(-1)[slot][:, None]
        We = kept[e] if op == "decode" else _exact_values(s["W"][e].double(), 128)
        Ye = _exact_values(x[t]) @ We.T
        y.index_add_(0, t, ws * Ye)
        if op == "experts":
            d = ws * dy[t]
            dx.index_add_(0, t, _exact_values(d) @ We)
            dW[e] = _exact_values(d.T) @ _exact_values(x[t].T).T
            dw[slot] = (Ye * dy[t]).sum(1)
    if op == "decode":
        return {**pad, "y": y}
    return {**pad, "y": y, "dx": dx, "dW": dW, "dw": dw.view(T, topk)}


def work(case):
    """What a pass cannot do without: every input read once, every output written once, the products' operations."""
    op = case["op"]
    x = _BYTES[case.get("x", "bf16")]
    if op == "quantize":
        n = case["rows"] * case["cols"]
        return dict(bytes=n * (x + 2), flops=0)
    if op in ("linear", "kept"):
        M, K, N, y = case["M"], case["K"], case["N"], _BYTES[case["y"]]
        if op == "kept":
            return dict(bytes=2 * M * K + N * K + y * M * N, flops=2 * M * N * K)
        return dict(bytes=x * (M * K + N * K + M * N) + y * (M * N + M * K) + 4 * N * K, flops=6 * M * N * K)
    T, topk, E = case["T"], case["topk"], case["E"]
    n = T * topk
    if op == "route":
        # x, dy read; rows, drows written; y, dx written (the rows in between need not leave the chip's caches)
        return dict(bytes=case["H"] * x * (2 * T + 2 * n + 2 * T) + 20 * n, flops=6 * n * case["H"])
    K, N = case["K"], case["N"]
    if op == "decode":
        return dict(bytes=2 * T * K + min(n, E) * N * K + 2 * T * N, flops=2 * n * N * K)
    return dict(bytes=x * (T * K + T * N) + 2 * E * N * K + 2 * (T * N + T * K) + 4 * E * N * K, flops=6 * n * N * K)
