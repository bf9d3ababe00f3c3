"""Plain 64-bit forms of the FP8 operators and of the routing, for the tests: the formats are spelt out, nothing is blocked."""
import numpy as np
import torch

BLOCK = 128


def codes_and_exponents(x, square=False):
    """x [R, C] (any float type) -> (code values in double, exponents int64 per element)."""
    x = x.double()
    R, C = x.shape
    rows = -(-R // BLOCK) if square else R
    amax = torch.zeros((rows, -(-C // BLOCK)), dtype=torch.float64, device=x.device)
    for i in range(amax.shape[1]):
        m = x[:, i * BLOCK:(i + 1) * BLOCK].abs().amax(1)
        if square:
            m = torch.nn.functional.pad(m, (0, rows * BLOCK - R)).view(rows, BLOCK).amax(1)
        amax[:, i] = m
    e = torch.full(amax.shape, -127, dtype=torch.int64, device=x.device)
    for k in range(-126, 128):                                      # the smallest e with 448 * 2^e >= amax, by trying them
        e += (amax > 448.0 * 2.0 ** (k - 1)).long()
    if square:
        e = e.repeat_interleave(BLOCK, 0)[:R]
    wide = e.repeat_interleave(BLOCK, 1)[:, :C]
    y = (x * two_to(-wide)).float().to(torch.float8_e4m3fn).double()   # exact product; the library's cast rounds to nearest, ties to even
    return y, wide


def two_to(e):
    return ((e + 1023) << 52).view(torch.float64)


def values(x, square=False):
    y, e = codes_and_exponents(x, square)
    return y * two_to(e)


def code_bytes(y):
    return y.float().to(torch.float8_e4m3fn).view(torch.uint8)


def scale_bytes(e):
    """One byte per row and block from exponents per element."""
    return (e[:, ::BLOCK] + 127).to(torch.uint8)


def swizzled(sf):
    """[R, nb] -> the bytes of the tiles of 128 rows x 4 blocks."""
    sf = sf.cpu().numpy()
    R, nb = sf.shape
    tiles = -(-nb // 4)
    out = np.zeros(-(-R // 128) * tiles * 512, dtype=np.uint8)
    r, kb = np.meshgrid(np.arange(R), np.arange(nb), indexing="ij")
    out[((r // 128) * tiles + kb // 4) * 512 + (r % 32) * 16 + ((r % 128) // 32) * 4 + kb % 4] = sf
    return out


def product(a, b):
    """(a . b^T, sum |a_i b_i|) in double."""
    return a @ b.T, a.abs() @ b.abs().T


def accumulation(K):
    """What fp32 accumulation over K may be off, relative to sum |a_i b_i|: an instruction adds 32 products to the running sum; the sum of
    their roundings (alignment, the sum itself) is taken as two units in the last place, 2^-23 of the largest magnitude, for each."""
    return 2 * (-(-K // 32) + 1) * 2.0 ** -23


def assert_product(D, ref, T, K):
    tol = accumulation(K) * T + (ref.abs() * 2.0 ** -8 if D.dtype == torch.bfloat16 else ref.abs() * 2.0 ** -24)
    over = (D.double() - ref).abs() - tol
    assert not bool((over > 0).any()) and not bool(D.isnan().any()), f"{int((over > 0).sum())} of {D.numel()} off, worst by {float(over.max()):.3e}"


def route(expert_of, experts, rows):
    """counts, offsets, row_of, slot_of, slot by slot."""
    e = expert_of.reshape(-1).tolist()
    members = [[s for s, x in enumerate(e) if x == k] for k in range(experts)]
    offsets = [0]
    for m in members:
        offsets.append(offsets[-1] + -(-len(m) // BLOCK) * BLOCK)
    row_of, slot_of = [-1] * len(e), [-1] * rows
    for k, m in enumerate(members):
        for i, s in enumerate(m):
            row_of[s], slot_of[offsets[k] + i] = offsets[k] + i, s
    return [len(m) for m in members], offsets, row_of, slot_of
