// Quantizer to 8-bit floating point with one power-of-two scale for each block of 128 (fp8.cuh has the format):
//   code = E4M3(x * 2^-e),  2^e the smallest power of two with 448 * 2^e >= max|x| of the block,
// along the rows' contiguous axis, along the rows (stored transposed), or both from one read.
//
// Bound by memory: 2 or 4 bytes read and 1 written per element and output.  A block of 256 threads takes a tile of 128 x 128,
// which is one block of 128 for every row and every column, so no scale needs a second read.  A thread holds 8 rows x 8
// columns in registers (eight 16-byte loads in flight): a row's maximum is a reduction over 16 lanes, a column's one over the
// thread's own rows and then, through shared memory, over the warps.  Row codes leave from registers, 128 bytes of a row per
// half warp; transposed ones are packed along the thread's 8 rows and turned round in shared memory.
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
  int64_t nb_r, nb_t;            // blocks per quantized row
  int64_t col_tiles, row_tiles;
  int64_t first;                 // first tile of the launch that belongs to it
};
struct Fp8Ops {
  Fp8Op op[kMaxFp8Operands];
  int n, swizzled;
};

__device__ __forceinline__ uint32_t absmax_nan_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r & 0x7FFF7FFFu;
}

__device__ __forceinline__ float load_weight(const void* w, int dtype, int64_t i) {
  if (dtype == NVFP4_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(w)[i]);
  return static_cast<const float*>(w)[i];
}

// A thread's 8 x 8 values.  bf16 stays packed, unless it is multiplied by a weight.
template <typename T, bool WEIGHTED>
struct Values {
  static constexpr bool kPacked = std::is_same_v<T, __nv_bfloat16> && !WEIGHTED;
  static constexpr int kWords = kPacked ? 4 : 8;
  uint32_t raw[8][kWords];

  __device__ __forceinline__ float get(int i, int j) const {
    if constexpr (kPacked) return __uint_as_float((j & 1) ? raw[i][j >> 1] & 0xFFFF0000u : raw[i][j >> 1] << 16);
    else return __uint_as_float(raw[i][j]);
  }
  // The row's 8 values from `src` (null: zeros), of which `left` exist.
  __device__ __forceinline__ void load(int i, const T* src, int left, [[maybe_unused]] float weight) {
    uint32_t w[8];
    constexpr int kSource = std::is_same_v<T, __nv_bfloat16> ? 4 : 8;
#pragma unroll
    for (int q = 0; q < 8; ++q) w[q] = 0u;
    if (src && left >= 8) {
      const uint4 a = load_vec16(src);
      w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
      if constexpr (kSource == 8) {
        const uint4 b = load_vec16(src + 4);
        w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
      }
    } else if (src) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (j >= left) break;
        if constexpr (kSource == 8) w[j] = reinterpret_cast<const volatile uint32_t*>(src)[j];
        else w[j >> 1] |= (uint32_t)reinterpret_cast<const volatile uint16_t*>(src)[j] << (16 * (j & 1));
      }
    }
#pragma unroll
    for (int q = 0; q < kWords; ++q) {
      if constexpr (kPacked || !WEIGHTED) raw[i][q] = w[q];
      else if constexpr (kSource == 8) raw[i][q] = __float_as_uint(__fmul_rn(__uint_as_float(w[q]), weight));
      else raw[i][q] = __float_as_uint(__fmul_rn(__uint_as_float((q & 1) ? w[q >> 1] & 0xFFFF0000u : w[q >> 1] << 16), weight));
    }
  }
  // Bits of the largest |value| of row i, and of every column.
  __device__ __forceinline__ uint32_t row_max(int i) const {
    if constexpr (kPacked) {
      const uint32_t m = absmax_nan_bf16x2(absmax_nan_bf16x2(raw[i][0], raw[i][1]), absmax_nan_bf16x2(raw[i][2], raw[i][3]));
      return max(m & 0xFFFFu, m >> 16) << 16;
    } else {
      uint32_t m = 0u;
#pragma unroll
      for (int j = 0; j < 8; ++j) m = max(m, raw[i][j] & 0x7FFFFFFFu);
      return m;
    }
  }
  __device__ __forceinline__ void col_max(uint32_t (&m)[8]) const {
#pragma unroll
    for (int j = 0; j < kWords; ++j) {
      uint32_t v = raw[0][j];
      if constexpr (!kPacked) v &= 0x7FFFFFFFu;
#pragma unroll
      for (int i = 1; i < 8; ++i) {
        if constexpr (kPacked) v = absmax_nan_bf16x2(v, raw[i][j]);
        else v = max(v, raw[i][j] & 0x7FFFFFFFu);
      }
      if constexpr (kPacked) { m[2 * j] = v << 16; m[2 * j + 1] = v & 0xFFFF0000u; }
      else m[j] = v;
    }
  }
};

// Byte of the scale of (row r, block kb) of one quantized matrix.
__device__ __forceinline__ int64_t scale_at(int64_t r, int64_t kb, int64_t nb, int swizzled) {
  return swizzled ? sf_swizzled_offset(r, kb, (nb + 3) >> 2) : r * nb + kb;
}
// The scale of row r (of `rows`) in block kb, written by the thread that has it; tiles hold zero where there is no row or block.
__device__ __forceinline__ void store_scale(uint8_t* sf, int64_t r, int64_t rows, int64_t kb, int64_t nb, int swizzled, uint32_t code) {
  if (!swizzled) {
    if (r < rows) sf[r * nb + kb] = (uint8_t)code;
    return;
  }
  sf[scale_at(r, kb, nb, 1)] = r < rows ? (uint8_t)code : (uint8_t)0;
  if (kb == nb - 1)
    for (int64_t p = nb; p & 3; ++p) sf[scale_at(r, p, nb, 1)] = 0;
}

template <typename T, bool WEIGHTED>
__global__ void __launch_bounds__(256) quantize_fp8_kernel(const __grid_constant__ Fp8Ops ops) {
  __shared__ __align__(16) uint8_t turned[128 * 128];
  __shared__ uint32_t col_bits[8][128];
  __shared__ float col_inverse[128];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, half = lane >> 4, l16 = lane & 15;
  int w = 0;
  while (w + 1 < ops.n && (int64_t)blockIdx.x >= ops.op[w + 1].first) ++w;
  const Fp8Op& op = ops.op[w];
  const Fp8Operand& o = op.o;
  int64_t tile = (int64_t)blockIdx.x - op.first;
  const int64_t per_matrix = op.col_tiles * op.row_tiles, b = tile / per_matrix;
  tile -= b * per_matrix;
  const int64_t rt = tile / op.col_tiles, ct = tile - rt * op.col_tiles;
  const int64_t r0 = rt * 128, c0 = ct * 128;
  const int64_t row = r0 + warp * 16 + half * 8, col = c0 + l16 * 8;      // of this thread's first value

  grid_dependency_wait();
  grid_dependency_trigger();
  if (o.from.used && r0 >= *reinterpret_cast<const volatile int32_t*>(o.from.used)) return;

  Values<T, WEIGHTED> v;
  const T* const x = static_cast<const T*>(o.x) + b * o.rows * o.ld;
  const int left = (int)min((int64_t)8, o.cols - col);
  if (o.from.slot_of) {
    int slot[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      slot[i] = reinterpret_cast<const volatile int32_t*>(o.from.slot_of)[row + i];   // rows: a multiple of 128
      if (slot[i] >= o.from.slots) slot[i] = -1;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float weight = 1.0f;
      if (WEIGHTED && o.from.weights && slot[i] >= 0) weight = load_weight(o.from.weights, o.from.weights_dtype, slot[i]);
      const int64_t source = o.from.per_row ? slot[i] / o.from.per_row : row + i;
      v.load(i, slot[i] >= 0 && left > 0 ? x + source * o.ld + col : nullptr, left, weight);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v.load(i, row + i < o.rows && left > 0 ? x + (row + i) * o.ld + col : nullptr, left, 1.0f);
  }

  uint8_t* const codes_r = o.codes_r ? o.codes_r + (b * o.rows) * op.pitch_r : nullptr;
  uint8_t* const codes_t = o.codes_t ? o.codes_t + (b * o.cols) * op.pitch_t : nullptr;
  uint8_t* const scales_r = o.scales_r + b * op.sf_r;
  uint8_t* const scales_t = o.scales_t + b * op.sf_t;
  // codes of the thread's 8 rows x 8 columns go into shared memory as 8 columns x 8 rows; piece (8 rows) XOR column / 8, so that
  // the 16 lanes of a row, 8 columns apart, meet all banks
  const int piece = (warp * 2 + half) ^ l16;
  uint32_t square_code = 0u;

  if (o.square) {
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, v.row_max(i));
    m = __reduce_max_sync(0xFFFFFFFFu, m);
    if (lane == 0) col_bits[0][warp] = m;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 8; ++q) m = max(m, col_bits[0][q]);
    square_code = fp8_scale_code(m);
  }
  if (codes_r) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t code = square_code;
      if (!o.square) {
        uint32_t m = v.row_max(i);
#pragma unroll
        for (int d = 8; d; d >>= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
        code = fp8_scale_code(m);
      }
      const float inv = fp8_scale_inverse(code);
      const uint32_t lo = e4m3x4(v.get(i, 0) * inv, v.get(i, 1) * inv, v.get(i, 2) * inv, v.get(i, 3) * inv);
      const uint32_t hi = e4m3x4(v.get(i, 4) * inv, v.get(i, 5) * inv, v.get(i, 6) * inv, v.get(i, 7) * inv);
      if (row + i < o.rows && col < op.pitch_r) *reinterpret_cast<uint2*>(codes_r + (row + i) * op.pitch_r + col) = make_uint2(lo, hi);
      if (l16 == i) store_scale(scales_r, row + i, o.rows, ct, op.nb_r, ops.swizzled, code);
    }
  }
  if (codes_t) {
    if (!o.square) {
      uint32_t m[8];
      v.col_max(m);
#pragma unroll
      for (int j = 0; j < 8; ++j) m[j] = max(m[j], __shfl_xor_sync(0xFFFFFFFFu, m[j], 16));
      if (half == 0) {
#pragma unroll
        for (int j = 0; j < 8; j += 4)
          *reinterpret_cast<uint4*>(&col_bits[warp][l16 * 8 + j]) = make_uint4(m[j], m[j + 1], m[j + 2], m[j + 3]);
      }
      __syncthreads();
    }
    if (threadIdx.x < 128) {
      const int c = threadIdx.x;
      uint32_t code = square_code;
      if (!o.square) {
        uint32_t m = 0u;
#pragma unroll
        for (int q = 0; q < 8; ++q) m = max(m, col_bits[q][c]);
        code = fp8_scale_code(m);
      }
      col_inverse[c] = fp8_scale_inverse(code);
      store_scale(scales_t, c0 + c, o.cols, rt, op.nb_t, ops.swizzled, code);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float inv = col_inverse[l16 * 8 + j];
      const uint32_t lo = e4m3x4(v.get(0, j) * inv, v.get(1, j) * inv, v.get(2, j) * inv, v.get(3, j) * inv);
      const uint32_t hi = e4m3x4(v.get(4, j) * inv, v.get(5, j) * inv, v.get(6, j) * inv, v.get(7, j) * inv);
      *reinterpret_cast<uint2*>(turned + (l16 * 8 + j) * 128 + piece * 8) = make_uint2(lo, hi);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = i * 16 + warp * 2 + half;
      if (c0 + c < o.cols && r0 + l16 * 8 < op.pitch_t)
        *reinterpret_cast<uint2*>(codes_t + (c0 + c) * op.pitch_t + r0 + l16 * 8) =
            *reinterpret_cast<const uint2*>(turned + c * 128 + ((l16 ^ (c >> 3)) * 8));
    }
  }
}

template <typename T, bool WEIGHTED>
int launch(const Fp8Ops& ops, int64_t tiles, cudaStream_t s) {
  return launch_overlapped(quantize_fp8_kernel<T, WEIGHTED>, dim3((unsigned)tiles), 256, 0, s, ops) == cudaSuccess ? NVFP4_OK : NVFP4_ERR_CUDA;
}

}  // namespace

int quantize_fp8(const Fp8Operand* list, int n, int dtype, int sf_layout, cudaStream_t s) {
  Fp8Ops ops;
  ops.n = n;
  ops.swizzled = sf_layout == NVFP4_SF_SWIZZLED_128x4;
  int64_t tiles = 0;
  bool weighted = false;
  for (int i = 0; i < n; ++i) {
    Fp8Op& op = ops.op[i];
    const Fp8Operand& o = op.o = list[i];
    op.pitch_r = fp8_pitch(o.cols); op.pitch_t = fp8_pitch(o.rows);
    op.nb_r = fp8_blocks(o.cols); op.nb_t = fp8_blocks(o.rows);
    op.sf_r = (int64_t)nvfp4_sf_bytes_fp8(o.rows, o.cols, sf_layout); op.sf_t = (int64_t)nvfp4_sf_bytes_fp8(o.cols, o.rows, sf_layout);
    op.col_tiles = op.nb_r; op.row_tiles = op.nb_t;
    op.first = tiles;
    tiles += o.batch * op.col_tiles * op.row_tiles;
    weighted = weighted || o.from.weights;
  }
  if (tiles > 0x7FFFFFFFll) return NVFP4_ERR_SHAPE;
  if (dtype == NVFP4_BF16) return weighted ? launch<__nv_bfloat16, true>(ops, tiles, s) : launch<__nv_bfloat16, false>(ops, tiles, s);
  return weighted ? launch<float, true>(ops, tiles, s) : launch<float, false>(ops, tiles, s);
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
