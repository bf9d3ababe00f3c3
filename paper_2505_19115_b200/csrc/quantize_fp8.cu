// Quantizer to 8-bit floating point with one power-of-two scale for each block of 128 (fp8.cuh has the format):
//   code = E4M3(x * 2^-e),  2^e the smallest power of two with 448 * 2^e >= max|x| of the block,
// along the rows' contiguous axis, along the rows (stored transposed), or both from one read.
//
// Bound by memory: 2 or 4 bytes read and 1 written per element and output.  A block of 256 threads takes a tile of 128 x 128,
// which is one block of 128 for every row and every column, so no scale needs a second read.  A thread holds 8 rows x 8
// columns in registers (eight 16-byte loads in flight): a row's maximum is a reduction over 16 lanes, a column's one over the
// thread's own rows and then, through shared memory, over the warps.  Row codes leave from registers, 128 bytes of a row per
// half warp; transposed ones are packed along the thread's 8 rows and turned round in shared memory.  Nothing behind the last row or
// column is written.
// 8192 x 8192 bf16 (buffers in turn, nothing in the caches): row output 30 us = 6.7 TB/s, transposed 31 = 6.5, both 44 = 6.1; 16384 x
// 11008 80 / 82 / 114 us = 6.7 / 6.6 / 6.3; fp32 8192 x 8192 50 / 54 / 65.  Blocks of 128 x 128 take no more: 8192 x 8192 30 (row) and
// 43.5 (both), fp32 50 and 63, 11008 x 4096 20.6 and 30.0.  (A copy: 6.3-6.5 TB/s.)  Instructions come next: between products that hold the clock down they decide (dY both ways, X^T and W^T of a 16384 x 11008 x 4096 layer 171 us alone, 206 there).  Hence
// the absence of branches around loads and, in tiles that are full, around stores, 32-bit tile indices without a division, and maxima that
// stay packed until the last (12.3 a value for both outputs; 16.5 before the last three: 48, 182 and 242 us).  Transposed codes
// moved 16 bytes at a time take fewer still, 11.4, and no less time.
// 33000 rows of 2816 gathered from 16384, both outputs: 62 us, with weights 76 (with a fifth, or four fifths, of the tokens zero 75-76).
#include <cuda_bf16.h>

#include <type_traits>

#include "fp8.cuh"
#include "quantize_core.cuh"

namespace nvfp4 {
namespace {

struct Fp8Op {
  Fp8Operand o;
  int64_t pitch_r, pitch_t;
  int64_t sf_r, sf_t;            // bytes of one matrix's scales
  int rows, cols;
  int col_tiles, row_tiles;      // = blocks per quantized row of codes_r, codes_t
  uint32_t per_col_tile, per_slot;   // (2^32 - 1) / col_tiles, / slots of a token
  int first;                     // first tile of the launch that belongs to it
};
struct Fp8Ops {
  Fp8Op op[kMaxFp8Operands];
  int n, swizzled;
};

__device__ __forceinline__ uint32_t absmax_nan_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;                                            // the sign bits mean nothing
}
__device__ __forceinline__ uint32_t absmax3_nan(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}
// Bits of the largest |value| of 8, NaN above all.
__device__ __forceinline__ uint32_t absmax8(uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t e, uint32_t f, uint32_t g, uint32_t h) {
  return absmax3_nan(absmax3_nan(a, b, c), absmax3_nan(d, e, f), absmax3_nan(g, g, h));
}

// n / d of non-negative numbers, given (2^32 - 1) / d: the product with that is one too small at most.
__device__ __forceinline__ int quotient(int n, int d, uint32_t reciprocal) {
  const int q = (int)__umulhi((uint32_t)n, reciprocal);
  return q + (n - q * d >= d);
}

__device__ __forceinline__ float load_weight(const void* w, int dtype, int64_t i) {
  if (dtype == NVFP4_BF16) return __uint_as_float((uint32_t)reinterpret_cast<const volatile uint16_t*>(w)[i] << 16);
  return reinterpret_cast<const volatile float*>(w)[i];
}

// Two products, each rounded by itself.
__device__ __forceinline__ void mul2_each(float a0, float a1, float b0, float b1, float& y0, float& y1) {
  asm("{\n\t.reg .b64 a, b, y;\n\t"
      "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
      "mul.rn.f32x2 y, a, b;\n\t"
      "mov.b64 {%0, %1}, y;\n\t}"
      : "=f"(y0), "=f"(y1) : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}
// Four values scaled, as codes.
__device__ __forceinline__ uint32_t scaled_codes(float v0, float v1, float v2, float v3, float inv) {
  float y0, y1, y2, y3;
  mul2(v0, v1, inv, y0, y1);
  mul2(v2, v3, inv, y2, y3);
  return e4m3x4(y0, y1, y2, y3);
}

// A thread's 8 x 8 values, and the weights of its rows, which are multiplied in where the values are used (all values widened and
// multiplied first: 12 % more time).
template <typename T, bool WEIGHTED>
struct Values {
  static constexpr bool kBf16 = std::is_same_v<T, __nv_bfloat16>;
  static constexpr int kWords = kBf16 ? 4 : 8;
  uint32_t raw[8][kWords];
  float weight[WEIGHTED ? 8 : 1];
  float weight_mine;                                     // of row (lane % 16) / 2

  __device__ __forceinline__ float get(int i, int j) const {
    if constexpr (kBf16) return __uint_as_float((j & 1) ? raw[i][j >> 1] & 0xFFFF0000u : raw[i][j >> 1] << 16);
    else return __uint_as_float(raw[i][j]);
  }
  // Row i, all 8 values of it.
  __device__ __forceinline__ void load(int i, const T* src) {
    const uint4 a = load_vec16(src);
    raw[i][0] = a.x; raw[i][1] = a.y; raw[i][2] = a.z; raw[i][3] = a.w;
    if constexpr (!kBf16) {
      const uint4 b = load_vec16(src + 4);
      raw[i][4] = b.x; raw[i][5] = b.y; raw[i][6] = b.z; raw[i][7] = b.w;
    }
  }
  __device__ __forceinline__ void clear(int i) {
#pragma unroll
    for (int q = 0; q < kWords; ++q) raw[i][q] = 0u;
  }
  // The first `left` values of row i.
  __device__ __forceinline__ void load_some(int i, const T* src, int left) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (j >= left) break;
      if constexpr (kBf16) raw[i][j >> 1] |= (uint32_t)reinterpret_cast<const volatile uint16_t*>(src)[j] << (16 * (j & 1));
      else raw[i][j] = reinterpret_cast<const volatile uint32_t*>(src)[j];
    }
  }
  // Maxima of |value|, NaN above all, in the form that joins with the least work: bf16 two to a word, whose signs mean nothing.
  __device__ __forceinline__ uint32_t row_max(int i) const {
    if constexpr (kBf16) return absmax_nan_bf16x2(absmax_nan_bf16x2(raw[i][0], raw[i][1]), absmax_nan_bf16x2(raw[i][2], raw[i][3]));
    else return absmax8(raw[i][0], raw[i][1], raw[i][2], raw[i][3], raw[i][4], raw[i][5], raw[i][6], raw[i][7]);
  }
  static __device__ __forceinline__ uint32_t join(uint32_t a, uint32_t b) {
    if constexpr (kBf16) return absmax_nan_bf16x2(a, b);
    else return max(a, b);
  }
  // fp32 bits of the largest.
  static __device__ __forceinline__ uint32_t bits(uint32_t m) {
    if constexpr (kBf16) return max(m << 16 & 0x7FFF0000u, m & 0x7FFF0000u);
    else return m;
  }
  // Maxima of the columns: a word for two where they are bf16 as they stand, one for each where there are weights.
  static constexpr int kColWords = kBf16 && !WEIGHTED ? 4 : 8;
  __device__ __forceinline__ void col_max(uint32_t (&m)[kColWords]) const {
    if constexpr (WEIGHTED) {
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        float y[2][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) mul2(get(i, j), get(i, j + 1), weight[i], y[0][i], y[1][i]);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t u[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) u[i] = __float_as_uint(y[q][i]);
          m[j + q] = absmax8(u[0], u[1], u[2], u[3], u[4], u[5], u[6], u[7]);
        }
      }
    } else if constexpr (kBf16) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        m[j] = raw[0][j];
#pragma unroll
        for (int i = 1; i < 8; ++i) m[j] = absmax_nan_bf16x2(m[j], raw[i][j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) m[j] = absmax8(raw[0][j], raw[1][j], raw[2][j], raw[3][j], raw[4][j], raw[5][j], raw[6][j], raw[7][j]);
    }
  }
  static __device__ __forceinline__ uint32_t join_cols(uint32_t a, uint32_t b) {
    if constexpr (kColWords == 4) return absmax_nan_bf16x2(a, b);
    else return max(a, b);
  }
  // Codes of the values from (i, j) on: four of row i, or of column j.
  __device__ __forceinline__ uint32_t row_codes(int i, int j, float factor) const {
    return scaled_codes(get(i, j), get(i, j + 1), get(i, j + 2), get(i, j + 3), factor);
  }
  __device__ __forceinline__ uint32_t col_codes(int i, int j, float inv) const {
    if constexpr (WEIGHTED) {
      float y0, y1, y2, y3;
      mul2_each(get(i, j), get(i + 1, j), weight[i], weight[i + 1], y0, y1);
      mul2_each(get(i + 2, j), get(i + 3, j), weight[i + 2], weight[i + 3], y2, y3);
      return scaled_codes(y0, y1, y2, y3, inv);
    } else {
      return scaled_codes(get(i, j), get(i + 1, j), get(i + 2, j), get(i + 3, j), inv);
    }
  }
};

// The scale of row r (of `rows`) in block kb (of nb), written by the thread that has it; tiles hold zero where there is no row or block.
__device__ __forceinline__ void store_scale(uint8_t* sf, int r, int rows, int kb, int nb, int swizzled, uint32_t code) {
  if (!swizzled) {
    if (r < rows) sf[(int64_t)r * nb + kb] = (uint8_t)code;
    return;
  }
  uint8_t* const at = sf + sf_swizzled_offset(r, kb, (nb + 3) >> 2);
  *at = r < rows ? (uint8_t)code : (uint8_t)0;
  if (kb == nb - 1)
    for (int q = 1; (kb + q) & 3; ++q) at[q] = 0;
}

// Of the `n` bytes at dst that are to be written, up to 8.
__device__ __forceinline__ void store_codes(uint8_t* dst, int n, uint32_t lo, uint32_t hi) {
  if (n >= 8) {
    *reinterpret_cast<uint2*>(dst) = make_uint2(lo, hi);
  } else {
    for (int q = 0; q < n; ++q) dst[q] = (uint8_t)((q < 4 ? lo : hi) >> (8 * (q & 3)));
  }
}

// The maxima of a thread's 8 rows -> the one of row l16 / 2 over all 16 lanes.  Each step hands half of the rows to the other lane
// of a pair, so that 8 exchanges do what 32 would, and a row's scale is computed by one lane pair, not by all.
template <typename V>
__device__ __forceinline__ uint32_t own_row_max(const uint32_t (&m)[8], int l16) {
  uint32_t a[4], b[2], c;
#pragma unroll
  for (int q = 0; q < 4; ++q) {                          // lanes 8-15 keep rows 4-7
    const bool up = l16 & 8;
    const uint32_t keep = up ? m[q + 4] : m[q], give = up ? m[q] : m[q + 4];
    a[q] = V::join(keep, __shfl_xor_sync(0xFFFFFFFFu, give, 8));
  }
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const bool up = l16 & 4;
    const uint32_t keep = up ? a[q + 2] : a[q], give = up ? a[q] : a[q + 2];
    b[q] = V::join(keep, __shfl_xor_sync(0xFFFFFFFFu, give, 4));
  }
  const bool up = l16 & 2;
  c = V::join(up ? b[1] : b[0], __shfl_xor_sync(0xFFFFFFFFu, up ? b[0] : b[1], 2));
  return V::bits(V::join(c, __shfl_xor_sync(0xFFFFFFFFu, c, 1)));
}

struct Shared {
  __align__(16) uint8_t turned[128 * 128];
  __align__(16) uint32_t col_bits[8][128];
  __align__(16) float col_inverse[128];
};

// Scales, codes and stores of a tile.  FULL: nothing of it lies behind the last row or column.
template <bool FULL, typename T, bool WEIGHTED>
__device__ __forceinline__ void finish_tile(const Fp8Op& op, int swizzled, const Values<T, WEIGHTED>& v, int b, int rt, int ct, int warp, int lane,
                                            Shared& sm) {
  using V = Values<T, WEIGHTED>;
  const Fp8Operand& o = op.o;
  const int half = lane >> 4, l16 = lane & 15;
  const int r0 = rt * 128, c0 = ct * 128, row = r0 + warp * 16 + half * 8, col = c0 + l16 * 8;
  const int left = FULL ? 8 : min(8, op.cols - col);
  auto& turned = sm.turned;
  auto& col_bits = sm.col_bits;
  auto& col_inverse = sm.col_inverse;
  // codes of the thread's 8 rows x 8 columns go into shared memory as 8 columns x 8 rows; piece (8 rows) XOR column / 8, so that
  // the 16 lanes of a row, 8 columns apart, meet all banks
  const int piece = (warp * 2 + half) ^ l16;
  uint32_t square_code = 0u;
  if (o.square) {
    uint32_t m = v.row_max(0);
#pragma unroll
    for (int i = 1; i < 8; ++i) m = V::join(m, v.row_max(i));
    m = __reduce_max_sync(0xFFFFFFFFu, V::bits(m));
    if (lane == 0) col_bits[0][warp] = m;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 8; ++q) m = max(m, col_bits[0][q]);
    square_code = fp8_scale_code(m);
  }
  if (o.codes_r) {
    uint32_t code = square_code;                         // of row l16 / 2 (bits 3, 2, 1 of the lane)
    if (!o.square) {
      uint32_t m[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) m[i] = v.row_max(i);
      uint32_t amax = own_row_max<V>(m, l16);            // rounding is monotone: the largest product is that of the largest value
      if constexpr (WEIGHTED) amax = __float_as_uint(__fmul_rn(__uint_as_float(amax), v.weight_mine)) & 0x7FFFFFFFu;
      code = fp8_scale_code(amax);
    }
    if (!(lane & 1)) store_scale(o.scales_r + b * op.sf_r, row + (l16 >> 1), op.rows, ct, op.col_tiles, swizzled, code);
    float own = fp8_scale_inverse(code);
    // A weight times a power of two is exact, so that one multiplication by both rounds as one by the weight; where it is not (numbers
    // next to the smallest or the largest; padding and other rows of zeros count as such), the warp multiplies its values twice, which
    // takes at most 1 % more time.
    [[maybe_unused]] bool twice = false;
    if constexpr (WEIGHTED) {
      const float both = __fmul_rn(v.weight_mine, own);
      const uint32_t exponent = (__float_as_uint(both) >> 23) & 255u;
      twice = __any_sync(0xFFFFFFFFu, v.weight_mine != 0.0f && (code < 32u || exponent == 0u || exponent == 255u));
      if (!twice) own = both;
    }
    uint8_t* dst = o.codes_r + ((int64_t)b * op.rows + row) * op.pitch_r + col;
    const int rows = FULL ? 8 : min(8, op.rows - row);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float inv = __shfl_sync(0xFFFFFFFFu, own, 2 * i, 16);
      uint32_t lo, hi;
      if (WEIGHTED && twice) {
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; j += 2) mul2(v.get(i, j), v.get(i, j + 1), v.weight[i], y[j], y[j + 1]);
        lo = scaled_codes(y[0], y[1], y[2], y[3], inv);
        hi = scaled_codes(y[4], y[5], y[6], y[7], inv);
      } else {
        lo = v.row_codes(i, 0, inv);
        hi = v.row_codes(i, 4, inv);
      }
      if (i < rows) store_codes(dst, left, lo, hi);
      dst += op.pitch_r;
    }
  }
  if (o.codes_t) {
    if (!o.square) {
      uint32_t m[V::kColWords];
      v.col_max(m);
#pragma unroll
      for (int j = 0; j < V::kColWords; ++j) m[j] = V::join_cols(m[j], __shfl_xor_sync(0xFFFFFFFFu, m[j], 16));
      if (half == 0) {
#pragma unroll
        for (int j = 0; j < V::kColWords; j += 4)
          *reinterpret_cast<uint4*>(&col_bits[warp][l16 * V::kColWords + j]) = make_uint4(m[j], m[j + 1], m[j + 2], m[j + 3]);
      }
      __syncthreads();
    }
    if (threadIdx.x < 128) {
      const int c = threadIdx.x;
      uint32_t code = square_code;
      if (!o.square) {
        uint32_t m = 0u;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          if constexpr (V::kColWords == 4) m = absmax_nan_bf16x2(m, reinterpret_cast<const uint16_t*>(col_bits[q])[c]);
          else m = max(m, col_bits[q][c]);
        }
        code = fp8_scale_code(V::kColWords == 4 ? m << 16 & 0x7FFF0000u : m);
      }
      col_inverse[c] = fp8_scale_inverse(code);
      store_scale(o.scales_t + b * op.sf_t, c0 + c, op.cols, rt, op.row_tiles, swizzled, code);
    }
    __syncthreads();
    float inv[8];
#pragma unroll
    for (int j = 0; j < 8; j += 4) *reinterpret_cast<float4*>(inv + j) = *reinterpret_cast<const float4*>(col_inverse + l16 * 8 + j);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t lo = v.col_codes(0, j, inv[j]), hi = v.col_codes(4, j, inv[j]);
      *reinterpret_cast<uint2*>(turned + (l16 * 8 + j) * 128 + piece * 8) = make_uint2(lo, hi);
    }
    __syncthreads();
    // a half warp takes columns warp * 2 + half + 16 i
    const int c = warp * 2 + half;
    const int rows = FULL ? 8 : min(8, op.rows - r0 - l16 * 8);
    uint8_t* dst = o.codes_t + ((int64_t)b * op.cols + c0 + c) * op.pitch_t + r0 + l16 * 8;
    const int cols = FULL ? 128 : min(128, op.cols - c0);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int at = i * 16 + c;
      const uint2 q = *reinterpret_cast<const uint2*>(turned + at * 128 + ((l16 ^ (at >> 3)) * 8));
      if (at < cols) store_codes(dst, rows, q.x, q.y);
      dst += 16 * op.pitch_t;
    }
  }
}

template <typename T, bool WEIGHTED>
__global__ void __launch_bounds__(256, std::is_same_v<T, __nv_bfloat16> ? WEIGHTED ? 3 : 4 : 2) quantize_fp8_kernel(const __grid_constant__ Fp8Ops ops) {
  __shared__ Shared sm;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, half = lane >> 4, l16 = lane & 15;
  int w = 0;
  while (w + 1 < ops.n && (int)blockIdx.x >= ops.op[w + 1].first) ++w;
  const Fp8Op& op = ops.op[w];
  const Fp8Operand& o = op.o;
  const int t = (int)blockIdx.x - op.first;
  int rt = quotient(t, op.col_tiles, op.per_col_tile);
  const int ct = t - rt * op.col_tiles;
  const int b = o.batch == 1 ? 0 : rt / op.row_tiles;
  rt -= b * op.row_tiles;
  const int r0 = rt * 128, c0 = ct * 128, row = r0 + warp * 16 + half * 8, col = c0 + l16 * 8;      // of this thread's first value

  grid_dependency_wait();
  grid_dependency_trigger();
  Values<T, WEIGHTED> v;
  const T* const x = static_cast<const T*>(o.x) + (int64_t)b * op.rows * o.ld + col;
  const int left = min(8, op.cols - col);
  // Loads wait for no branch: rows that do not exist are loaded from one that does (columns likewise) and cleared afterwards.  Only
  // a row's last few values, where their number is no multiple of 8, are fetched one by one, and rows of fewer than 8 as a whole.
  const bool some = left > 0 && left < 8, eight = op.cols >= 8;
  const T* const from = left < 8 ? x - col : x;
  if (o.from.slot_of) {                                  // rows: a multiple of 128
    // lane i of a half warp finds row i's source (asked for with the end of the rows in use: one behind the other they cost two latencies)
    int slot = reinterpret_cast<const volatile int32_t*>(o.from.slot_of)[row + (l16 & 7)];
    if (r0 >= *reinterpret_cast<const volatile int32_t*>(o.from.used)) return;
    if (slot >= o.from.slots) slot = -1;
    const int source = slot < 0 ? -1 : o.from.per_row ? quotient(slot, o.from.per_row, op.per_slot) : row + (l16 & 7);
    float weight = 1.0f;
    if constexpr (WEIGHTED)
      if (o.from.weights && slot >= 0) weight = load_weight(o.from.weights, o.from.weights_dtype, slot);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = max(__shfl_sync(0xFFFFFFFFu, source, i, 16), 0);
      if (eight) v.load(i, from + (int64_t)r * o.ld);
    }
    if (c0 + 128 > op.cols || __any_sync(0xFFFFFFFFu, source < 0)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = __shfl_sync(0xFFFFFFFFu, source, i, 16);
        if (r < 0 || left < 8) v.clear(i);
        if (r >= 0 && some) v.load_some(i, x + (int64_t)r * o.ld, left);
      }
    }
    if constexpr (WEIGHTED) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v.weight[i] = __shfl_sync(0xFFFFFFFFu, weight, i, 16);
      v.weight_mine = __shfl_sync(0xFFFFFFFFu, weight, l16 >> 1, 16);
    }
  } else if (r0 + 128 <= op.rows && c0 + 128 <= op.cols) {
    const T* src = x + (int64_t)row * o.ld;
#pragma unroll
    for (int i = 0; i < 8; ++i) v.load(i, src + i * o.ld);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (eight) v.load(i, from + (int64_t)min(row + i, op.rows - 1) * o.ld);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (row + i >= op.rows || left < 8) v.clear(i);
      if (row + i < op.rows && some) v.load_some(i, x + (int64_t)(row + i) * o.ld, left);
    }
  }

  if (r0 + 128 <= op.rows && c0 + 128 <= op.cols) finish_tile<true, T, WEIGHTED>(op, ops.swizzled, v, b, rt, ct, warp, lane, sm);
  else finish_tile<false, T, WEIGHTED>(op, ops.swizzled, v, b, rt, ct, warp, lane, sm);
}

template <typename T, bool WEIGHTED>
int launch(const Fp8Ops& ops, int64_t tiles, cudaStream_t s) {
  return launch_overlapped(quantize_fp8_kernel<T, WEIGHTED>, dim3((unsigned)tiles), 256, 0, s, ops) == cudaSuccess ? NVFP4_OK : NVFP4_ERR_CUDA;
}

}  // namespace

int quantize_fp8(const Fp8Operand* list, int n, int dtype, int sf_layout, cudaStream_t s) {
  // operands with weights in a launch of their own: the multiplications take a fifth more time
  for (const bool weighted : {false, true}) {
    Fp8Ops ops;
    ops.n = 0;
    ops.swizzled = sf_layout == NVFP4_SF_SWIZZLED_128x4;
    int64_t tiles = 0;
    for (int i = 0; i < n; ++i) {
      if ((list[i].from.weights != nullptr) != weighted) continue;
      Fp8Op& op = ops.op[ops.n++];
      const Fp8Operand& o = op.o = list[i];
      op.pitch_r = fp8_pitch(o.cols); op.pitch_t = fp8_pitch(o.rows);
      op.sf_r = (int64_t)nvfp4_sf_bytes_fp8(o.rows, o.cols, sf_layout); op.sf_t = (int64_t)nvfp4_sf_bytes_fp8(o.cols, o.rows, sf_layout);
      op.rows = (int)o.rows; op.cols = (int)o.cols;
      op.col_tiles = (int)fp8_blocks(o.cols); op.row_tiles = (int)fp8_blocks(o.rows);
      op.per_col_tile = 0xFFFFFFFFu / (uint32_t)op.col_tiles;
      op.per_slot = o.from.per_row ? 0xFFFFFFFFu / (uint32_t)o.from.per_row : 0u;
      op.first = (int)tiles;
      tiles += o.batch * op.col_tiles * op.row_tiles;
      if (tiles > 0x7FFFFFFFll) return NVFP4_ERR_SHAPE;
    }
    if (ops.n == 0) continue;
    const bool bf16 = dtype == NVFP4_BF16;
    if (int st = weighted ? bf16 ? launch<__nv_bfloat16, true>(ops, tiles, s) : launch<float, true>(ops, tiles, s)
                          : bf16 ? launch<__nv_bfloat16, false>(ops, tiles, s) : launch<float, false>(ops, tiles, s))
      return st;
  }
  return NVFP4_OK;
}

}  // namespace nvfp4

using namespace nvfp4;

extern "C" size_t nvfp4_codes_bytes_fp8(int64_t Rq, int64_t Kq) {
  return Rq > 0 && Kq > 0 ? (size_t)(Rq * fp8_pitch(Kq)) : 0;
}

extern "C" size_t nvfp4_sf_bytes_fp8(int64_t Rq, int64_t Kq, int sf_layout) {
  if (Rq <= 0 || Kq <= 0) return 0;
  if (sf_layout == NVFP4_SF_LINEAR) return (size_t)(Rq * fp8_blocks(Kq));
  if (sf_layout == NVFP4_SF_SWIZZLED_128x4) return (size_t)(fp8_sf_tiles(Rq, Kq) * 512);
  return 0;
}

extern "C" int nvfp4_quantize_fp8(const void* x, int dtype, int64_t batch, int64_t rows, int64_t cols, int64_t ld, int block_rows,
                                  uint8_t* codes_row, uint8_t* scales_row, uint8_t* codes_t, uint8_t* scales_t, int sf_layout,
                                  void* cuda_stream) {
  if (!x || (!codes_row && !codes_t) || (!codes_row != !scales_row) || (!codes_t != !scales_t)) return NVFP4_ERR_NULL;
  if (dtype != NVFP4_BF16 && dtype != NVFP4_FP32) return NVFP4_ERR_ENUM;
  if (sf_layout != NVFP4_SF_LINEAR && sf_layout != NVFP4_SF_SWIZZLED_128x4) return NVFP4_ERR_ENUM;
  if (block_rows != 1 && block_rows != kFp8Block) return NVFP4_ERR_ENUM;
  if (batch <= 0 || rows <= 0 || cols <= 0 || ld < cols) return NVFP4_ERR_SHAPE;
  if (batch >= (1ll << 31) || rows >= (1ll << 31) - 256 || cols >= (1ll << 31) - 256) return NVFP4_ERR_SHAPE;
  if (fp8_blocks(rows) * fp8_blocks(cols) > 0x7FFFFFFFll / batch) return NVFP4_ERR_SHAPE;
  if (!aligned16(x) || (ld % 8) != 0 || !aligned16(codes_row) || !aligned16(codes_t) || !aligned16(scales_row) || !aligned16(scales_t))
    return NVFP4_ERR_ALIGN;
  if (int st = check_arch()) return st;
  const Fp8Operand op = {x, batch, rows, cols, ld, block_rows == kFp8Block, codes_row, scales_row, codes_t, scales_t, {}};
  return quantize_fp8(&op, 1, dtype, sf_layout, static_cast<cudaStream_t>(cuda_stream));
}
