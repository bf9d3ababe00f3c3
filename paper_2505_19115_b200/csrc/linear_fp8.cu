// Layer calls in 8-bit floating point with blocks of 128 (fp8.cuh): the linear layer and the layer of experts.
//   Y  = Q(X) . Q128(W)^T      blocks along K, weights in blocks of 128 x 128
//   dX = Q(dY) . Q128(W)       blocks along N; the same codes of W, transposed
//   dW = Q(dY^T) . Q(X^T)^T    blocks along the tokens
// Each call quantizes its operands in one launch (every tensor read once) and multiplies.  A layer of experts has W [experts, N, K]
// and takes its rows in the order of nvfp4_expert_sort; the quantizer gathers them, and applies the weights of the combination to
// the output gradient, on the way.
#include "fp8.cuh"

namespace nvfp4 {
namespace {

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

struct Place {
  size_t codes, sf;
};
void place(size_t& off, int64_t matrices, int64_t rq, int64_t kq, Place* at) {
  at->codes = off; off = align256(off + (size_t)(matrices * rq * fp8_pitch(kq)));
  at->sf = off;    off = align256(off + (size_t)(matrices * fp8_sf_tiles(rq, kq) * 512));
}
struct FwdLayout { Place x, w; size_t total; };
FwdLayout fwd_layout(int64_t E, int64_t M, int64_t N, int64_t K) {
  FwdLayout l; size_t off = 0;
  place(off, 1, M, K, &l.x);
  place(off, E, N, K, &l.w);
  l.total = off;
  return l;
}
struct BwdLayout { Place dy, dyt, xt, wt; size_t total; };
BwdLayout bwd_layout(int64_t E, int64_t M, int64_t N, int64_t K) {
  BwdLayout l; size_t off = 0;
  place(off, 1, M, N, &l.dy);
  place(off, 1, N, M, &l.dyt);
  place(off, 1, K, M, &l.xt);
  place(off, E, K, N, &l.wt);
  l.total = off;
  return l;
}
size_t workspace_bytes(int64_t E, int64_t M, int64_t N, int64_t K, int which) {
  switch (which) {
    case NVFP4_FP8_FWD: return fwd_layout(E, M, N, K).total;
    case NVFP4_FP8_BWD: return bwd_layout(E, M, N, K).total;
    default: return 0;
  }
}

bool dtype_ok(int dtype) { return dtype == NVFP4_BF16 || dtype == NVFP4_FP32; }
// N and K are the rows of dense tensors that are moved in 16-byte pieces; M is any.
bool sizes_ok(int64_t E, int64_t M, int64_t N, int64_t K) {
  constexpr int64_t kMost = (1ll << 31) - 512;
  if (E <= 0 || M <= 0 || N <= 0 || K <= 0 || N % 8 != 0 || K % 8 != 0) return false;
  if (M > kMost || N > kMost || K > kMost || E * N > kMost || E * K > kMost) return false;
  const int64_t m = fp8_blocks(M), n = fp8_blocks(N), k = fp8_blocks(K);
  return m * n + m * k + E * n * k <= 0x7FFFFFFFll;
}
bool buffer_ok(const void* p, size_t have, size_t need) { return p && have >= need && (reinterpret_cast<uintptr_t>(p) & 255u) == 0; }

}  // namespace
}  // namespace nvfp4

using namespace nvfp4;

extern "C" size_t nvfp4_linear_fp8_workspace_bytes(int64_t M, int64_t N, int64_t K, int which) {
  return sizes_ok(1, M, N, K) ? workspace_bytes(1, M, N, K, which) : 0;
}

extern "C" int nvfp4_linear_fp8_fwd(const void* X, const void* W, int dtype, int64_t M, int64_t N, int64_t K, void* Y, int y_dtype,
                                    void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (!X || !W || !Y) return NVFP4_ERR_NULL;
  if (!dtype_ok(dtype) || !dtype_ok(y_dtype)) return NVFP4_ERR_ENUM;
  if (!sizes_ok(1, M, N, K)) return NVFP4_ERR_SHAPE;
  if (!aligned16(X) || !aligned16(W) || !aligned16(Y)) return NVFP4_ERR_ALIGN;
  const FwdLayout l = fwd_layout(1, M, N, K);
  if (!buffer_ok(workspace, workspace_bytes, l.total)) return NVFP4_ERR_WORKSPACE;
  if (int st = check_arch()) return st;
  uint8_t* const ws = static_cast<uint8_t*>(workspace);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const Fp8Operand ops[2] = {{W, 1, N, K, K, 1, ws + l.w.codes, ws + l.w.sf, nullptr, nullptr, {}},
                             {X, 1, M, K, K, 0, ws + l.x.codes, ws + l.x.sf, nullptr, nullptr, {}}};
  if (int st = quantize_fp8(ops, 2, dtype, NVFP4_SF_SWIZZLED_128x4, s)) return st;
  return gemm_fp8({ws + l.x.codes, ws + l.x.sf, ws + l.w.codes, ws + l.w.sf, M, N, K, Y, y_dtype, N}, s);
}

extern "C" int nvfp4_linear_fp8_bwd(const void* dY, const void* W, const void* X, int dtype, int64_t M, int64_t N, int64_t K,
                                    void* dX, int dx_dtype, void* dW, int dw_dtype,
                                    void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (!dY || !W || !X || !dX || !dW) return NVFP4_ERR_NULL;
  if (!dtype_ok(dtype) || !dtype_ok(dx_dtype) || !dtype_ok(dw_dtype)) return NVFP4_ERR_ENUM;
  if (!sizes_ok(1, M, N, K)) return NVFP4_ERR_SHAPE;
  if (!aligned16(dY) || !aligned16(W) || !aligned16(X) || !aligned16(dX) || !aligned16(dW)) return NVFP4_ERR_ALIGN;
  const BwdLayout l = bwd_layout(1, M, N, K);
  if (!buffer_ok(workspace, workspace_bytes, l.total)) return NVFP4_ERR_WORKSPACE;
  if (int st = check_arch()) return st;
  uint8_t* const ws = static_cast<uint8_t*>(workspace);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const Fp8Operand ops[3] = {{W, 1, N, K, K, 1, nullptr, nullptr, ws + l.wt.codes, ws + l.wt.sf, {}},
                             {X, 1, M, K, K, 0, nullptr, nullptr, ws + l.xt.codes, ws + l.xt.sf, {}},
                             {dY, 1, M, N, N, 0, ws + l.dy.codes, ws + l.dy.sf, ws + l.dyt.codes, ws + l.dyt.sf, {}}};
  if (int st = quantize_fp8(ops, 3, dtype, NVFP4_SF_SWIZZLED_128x4, s)) return st;
  return gemm_fp8_two({ws + l.dy.codes, ws + l.dy.sf, ws + l.wt.codes, ws + l.wt.sf, M, K, N, dX, dx_dtype, K},
                      {ws + l.dyt.codes, ws + l.dyt.sf, ws + l.xt.codes, ws + l.xt.sf, N, K, M, dW, dw_dtype, K}, s);
}

extern "C" size_t nvfp4_experts_fp8_workspace_bytes(int64_t tokens, int64_t topk, int64_t experts, int64_t N, int64_t K, int which) {
  const int64_t rows = nvfp4_expert_rows(tokens, topk, experts);
  return rows && sizes_ok(experts, rows, N, K) ? workspace_bytes(experts, rows, N, K, which) : 0;
}

extern "C" int nvfp4_quantize_fp8_experts(const void* x, int dtype, int by_token, int64_t tokens, int64_t topk, int64_t experts, int64_t cols,
                                          int64_t ld, const int32_t* offsets, const int32_t* slot_of, const void* weights, int weights_dtype,
                                          uint8_t* codes_row, uint8_t* scales_row, uint8_t* codes_t, uint8_t* scales_t, void* cuda_stream) {
  if (!x || !offsets || !slot_of || (!codes_row && !codes_t) || (!codes_row != !scales_row) || (!codes_t != !scales_t)) return NVFP4_ERR_NULL;
  if (!dtype_ok(dtype) || !dtype_ok(weights_dtype) || (by_token != 0 && by_token != 1)) return NVFP4_ERR_ENUM;
  const int64_t rows = nvfp4_expert_rows(tokens, topk, experts);
  if (rows == 0 || cols <= 0 || ld < cols || cols > (1ll << 31) - 512 || fp8_blocks(rows) * fp8_blocks(cols) > 0x7FFFFFFFll) return NVFP4_ERR_SHAPE;
  if (!aligned16(x) || ld % 8 != 0 || !aligned16(codes_row) || !aligned16(codes_t) || !aligned16(scales_row) || !aligned16(scales_t) ||
      (reinterpret_cast<uintptr_t>(offsets) & 3u) || (reinterpret_cast<uintptr_t>(slot_of) & 3u) ||
      (reinterpret_cast<uintptr_t>(weights) & (weights_dtype == NVFP4_BF16 ? 1u : 3u)))
    return NVFP4_ERR_ALIGN;
  if (int st = check_arch()) return st;
  const Fp8Operand op = {x, 1, rows, cols, ld, 0, codes_row, scales_row, codes_t, scales_t,
                         {slot_of, offsets + experts, by_token ? (int)topk : 0, weights, weights_dtype, (int)(tokens * topk)}};
  return quantize_fp8(&op, 1, dtype, NVFP4_SF_SWIZZLED_128x4, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" int nvfp4_experts_fp8_fwd(const void* X, int x_by_token, const void* W, int dtype, int64_t tokens, int64_t topk, int64_t experts,
                                     int64_t N, int64_t K, const int32_t* offsets, const int32_t* slot_of, void* Y, int y_dtype,
                                     void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (!X || !W || !offsets || !slot_of || !Y) return NVFP4_ERR_NULL;
  if (!dtype_ok(dtype) || !dtype_ok(y_dtype) || (x_by_token != 0 && x_by_token != 1)) return NVFP4_ERR_ENUM;
  const int64_t R = nvfp4_expert_rows(tokens, topk, experts);
  if (R == 0 || !sizes_ok(experts, R, N, K)) return NVFP4_ERR_SHAPE;
  if (!aligned16(X) || !aligned16(W) || !aligned16(Y) || (reinterpret_cast<uintptr_t>(offsets) & 3u) || (reinterpret_cast<uintptr_t>(slot_of) & 3u))
    return NVFP4_ERR_ALIGN;
  const FwdLayout l = fwd_layout(experts, R, N, K);
  if (!buffer_ok(workspace, workspace_bytes, l.total)) return NVFP4_ERR_WORKSPACE;
  if (int st = check_arch()) return st;
  uint8_t* const ws = static_cast<uint8_t*>(workspace);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const Fp8Rows from = {slot_of, offsets + experts, x_by_token ? (int)topk : 0, nullptr, 0, (int)(tokens * topk)};
  const Fp8Operand ops[2] = {{W, experts, N, K, K, 1, ws + l.w.codes, ws + l.w.sf, nullptr, nullptr, {}},
                             {X, 1, R, K, K, 0, ws + l.x.codes, ws + l.x.sf, nullptr, nullptr, from}};
  if (int st = quantize_fp8(ops, 2, dtype, NVFP4_SF_SWIZZLED_128x4, s)) return st;
  return gemm_fp8({ws + l.x.codes, ws + l.x.sf, ws + l.w.codes, ws + l.w.sf, R, N, K, Y, y_dtype, N, experts, offsets, true, nullptr, tokens * topk}, s);
}

extern "C" int nvfp4_experts_fp8_bwd(const void* dY, int dy_by_token, const void* dy_weights, int weights_dtype, const void* W, const void* X,
                                     int x_by_token, int dtype, int64_t tokens, int64_t topk, int64_t experts, int64_t N, int64_t K,
                                     const int32_t* offsets, const int32_t* slot_of, void* dX, int dx_dtype, void* dW, int dw_dtype,
                                     void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (!dY || !W || !X || !offsets || !slot_of || !dX || !dW) return NVFP4_ERR_NULL;
  if (!dtype_ok(dtype) || !dtype_ok(dx_dtype) || !dtype_ok(dw_dtype) || !dtype_ok(weights_dtype) || (x_by_token != 0 && x_by_token != 1) ||
      (dy_by_token != 0 && dy_by_token != 1))
    return NVFP4_ERR_ENUM;
  const int64_t R = nvfp4_expert_rows(tokens, topk, experts);
  if (R == 0 || !sizes_ok(experts, R, N, K)) return NVFP4_ERR_SHAPE;
  if (!aligned16(dY) || !aligned16(W) || !aligned16(X) || !aligned16(dX) || !aligned16(dW) || (reinterpret_cast<uintptr_t>(offsets) & 3u) ||
      (reinterpret_cast<uintptr_t>(slot_of) & 3u) || (reinterpret_cast<uintptr_t>(dy_weights) & (weights_dtype == NVFP4_BF16 ? 1u : 3u)))
    return NVFP4_ERR_ALIGN;
  const BwdLayout l = bwd_layout(experts, R, N, K);
  if (!buffer_ok(workspace, workspace_bytes, l.total)) return NVFP4_ERR_WORKSPACE;
  if (int st = check_arch()) return st;
  uint8_t* const ws = static_cast<uint8_t*>(workspace);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const Fp8Rows x_from = {slot_of, offsets + experts, x_by_token ? (int)topk : 0, nullptr, 0, (int)(tokens * topk)};
  const Fp8Rows dy_from = {slot_of, offsets + experts, dy_by_token ? (int)topk : 0, dy_weights, weights_dtype, (int)(tokens * topk)};
  const Fp8Operand ops[3] = {{W, experts, N, K, K, 1, nullptr, nullptr, ws + l.wt.codes, ws + l.wt.sf, {}},
                             {X, 1, R, K, K, 0, nullptr, nullptr, ws + l.xt.codes, ws + l.xt.sf, x_from},
                             {dY, 1, R, N, N, 0, ws + l.dy.codes, ws + l.dy.sf, ws + l.dyt.codes, ws + l.dyt.sf, dy_from}};
  if (int st = quantize_fp8(ops, 3, dtype, NVFP4_SF_SWIZZLED_128x4, s)) return st;
  return gemm_fp8_two({ws + l.dy.codes, ws + l.dy.sf, ws + l.wt.codes, ws + l.wt.sf, R, K, N, dX, dx_dtype, K, experts, offsets, true, nullptr,
                       tokens * topk},
                      {ws + l.dyt.codes, ws + l.dyt.sf, ws + l.xt.codes, ws + l.xt.sf, N, K, R, dW, dw_dtype, K, experts, offsets, false}, s);
}
