// The 8-bit format of the FP8 operators, and the calls that its files share.
//
// Codes are E4M3, a block is 128 values along the contraction axis (or 128 x 128, for weights) and has one E8M0 scale:
// the smallest power of two 2^e with 448 * 2^e >= amax.  Multiplying by a power of two is exact, so a code is one rounding
// of the value itself, the tensor core applies the scales (kind::mxf8f6f4), and a square block quantized for the forward
// product is, transposed, the operand of the input gradient.
// A row of codes begins at a multiple of 16 bytes (what a tiled copy needs); its padding is never read.
#pragma once

#include "common.cuh"

namespace nvfp4 {

constexpr int kFp8Block = 128;

inline int64_t fp8_pitch(int64_t kq) { return (kq + 15) & ~(int64_t)15; }
inline int64_t fp8_blocks(int64_t kq) { return ceil_div(kq, kFp8Block); }
// 512-byte scale tiles of 128 rows x 4 blocks for one quantized matrix.
inline int64_t fp8_sf_tiles(int64_t rq, int64_t kq) { return ceil_div(rq, 128) * ceil_div(fp8_blocks(kq), 4); }

// Scale code of a block whose largest |x| has these bits: 448 = 1.75 * 2^8, so the exponent goes up by one where the
// mantissa is above 1.75.  255 (NaN) where the block holds a NaN or an infinity, which order above every finite value.
__device__ __forceinline__ uint32_t fp8_scale_code(uint32_t amax_bits) {
  if (amax_bits >= 0x7F800000u) return 255u;
  return (uint32_t)max((int)((amax_bits + 0x1FFFFFu) >> 23) - 8, 0);
}
// 2^(127 - code), by which a block's values are multiplied; NaN for code 255, so that its codes are NaN too.
__device__ __forceinline__ float fp8_scale_inverse(uint32_t code) {
  return __uint_as_float(code == 255u ? 0x7FFFFFFFu : (254u - code) << 23);
}
__device__ __forceinline__ uint32_t e4m3x4(float v0, float v1, float v2, float v3) {
  uint32_t r;
  asm("{\n\t.reg .b16 h0, h1;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 h0, %2, %1;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 h1, %4, %3;\n\t"
      "mov.b32 %0, {h0, h1};\n\t}"
      : "=r"(r) : "f"(v0), "f"(v1), "f"(v2), "f"(v3));
  return r;
}

// Which rows a gathered operand consists of: row r is source row slot_of[r] / per_row (or r itself where per_row is 0), times
// weights[slot_of[r]] where there are weights; zero where slot_of[r] is negative.  Rows from *used on are not quantized.
struct Fp8Rows {
  const int32_t* slot_of = nullptr;     // null: every row is its own source, all are used
  const int32_t* used = nullptr;
  int per_row = 0;
  const void* weights = nullptr;
  int weights_dtype = 0;
  int slots = 0;                        // slots from here on do not exist: such a row is zero
};
// An operand to quantize: `batch` matrices of rows x cols.  Null outputs are not written.
struct Fp8Operand {
  const void* x;
  int64_t batch, rows, cols, ld;
  int square;                           // blocks of 128 x 128
  uint8_t *codes_r, *scales_r;          // blocks along the columns: [batch, rows, pitch(cols)]
  uint8_t *codes_t, *scales_t;          // blocks along the rows: [batch, cols, pitch(rows)]
  Fp8Rows from;
};
constexpr int kMaxFp8Operands = 3;
// One launch for all of them, a second for those with weights (quantize_fp8.cu); the caller has checked the arguments.
int quantize_fp8(const Fp8Operand* ops, int n, int dtype, int sf_layout, cudaStream_t s);

// The products (gemm_fp8.cu); operands with swizzled scales.
//   experts == 0:  D[M, N] = A[M, K] . B[N, K]^T
//   by_rows:       rows of A and D in segments [offsets[e], offsets[e + 1]), multiples of 128; B [experts, N, K]
//   otherwise:     D[experts, M, N]: the contraction over segment e of K = offsets[experts] at most
struct Fp8Product {
  const uint8_t *a, *a_sf, *b, *b_sf;
  int64_t M, N, K;
  void* d;
  int d_dtype;
  int64_t ldd;
  int64_t experts = 0;
  const int32_t* offsets = nullptr;
  bool by_rows = false;
  const int32_t* counts = nullptr;      // by_rows: the rows of each segment that are no padding (null: unknown)
  int64_t slots = 0;                    // by_rows: the sum of the counts, at most
  bool late = false;                    // nothing that it reads or writes is the kernel before's, and that one has waited for all before it
};
int gemm_fp8(const Fp8Product& p, cudaStream_t s);
// The same for few rows (gemm_fp8_few.cu): one product, or by rows with their counts.  Padding rows of D are not written.
int gemm_fp8_few(const Fp8Product& p, cudaStream_t s);
// Two products of which the second needs nothing of the first's.
int gemm_fp8_two(const Fp8Product& a, const Fp8Product& b, cudaStream_t s);
int fp8_error_word(unsigned int* out);
int fp8_few_error_word(unsigned int* out);

constexpr int64_t kMaxExperts = 1024;

// The tensor core adds to its accumulator with truncation, so that an error grows with the number of additions: on normal values
// 7e-7 of the result at a contraction of 11008, over 1e-6 at 16384 (a sum in fp32 rounded at every step: 2e-7).  No accumulator takes
// more blocks than this; longer contractions are summed in parts, which are added with rounding.
constexpr int kMostBlocks = 96;

}  // namespace nvfp4
