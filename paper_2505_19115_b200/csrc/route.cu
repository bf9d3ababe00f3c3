// Tokens sorted by expert and back.  Slot s = token * topk + j carries the expert that the token's j-th choice names; an expert's
// rows are a segment that begins at a multiple of 128 rows (one row tile of the products, one block of the weight gradient's
// contraction), in the order of their slots, so that the result does not depend on how the work was split.
//   sort      counts, offsets, the row of every slot and the slot of every row (-1: dropped, padding)
//   gather    rows[r] = w[s] * x[token of s], s the slot of row r; zeros in padding rows
//   combine   y[t] = sum_j w[t,j] * rows[row of (t,j)], in the order of j, in fp32; the gradient of gather without weights too
//   combine's gradient: drows[r] = w[s] * dy[token of s] and dw[s] = <dy[token of s], rows[row of s]> from one read of both
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <type_traits>

#include "fp8.cuh"
#include "quantize_core.cuh"

namespace nvfp4 {
namespace {

namespace cg = cooperative_groups;

// ------------------------------------------------------------------------------------------------
// Sort.  Bound by latency: 4 or 8 bytes read and 8 written per slot.  One launch: a cluster of up to eight blocks (the slots cut
// into as many ranges, each cut into one per warp).  A warp counts its range per expert (lanes with the same expert find one
// another with a match), the counts become running sums over the warps, the blocks read one another's totals from shared
// memory, every block computes all offsets, and each warp goes over its range again and hands out rows.
// ------------------------------------------------------------------------------------------------
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32, kMaxCluster = 8;

struct SortParams {
  const void* expert_of;
  int wide;
  int n, experts;
  int per_warp;                 // slots of a warp, a multiple of 32
  int rows;                     // entries of slot_of
  int32_t *counts, *offsets, *row_of, *slot_of;
};

__global__ void __launch_bounds__(kSortThreads, 1) expert_sort_kernel(const SortParams p) {
  extern __shared__ int hist[];                      // [kSortWarps][experts], then totals[experts], base[experts], offset[experts + 1]
  __shared__ int warp_sum[kSortWarps];
  cg::cluster_group cluster = cg::this_cluster();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int E = p.experts;
  int* const totals = hist + kSortWarps * E;
  int* const base = totals + E;
  int* const offset = base + E;
  int* const mine = hist + warp * E;
  for (int e = lane; e < E; e += 32) mine[e] = 0;
  __syncwarp();
  grid_dependency_wait();
  grid_dependency_trigger();

  const int64_t first64 = ((int64_t)cluster.block_rank() * kSortWarps + warp) * p.per_warp;
  const int first = (int)min(first64, (int64_t)p.n), last = (int)min(first64 + p.per_warp, (int64_t)p.n);
  auto expert_at = [&](int s) {
    if (s >= last) return -1;
    const long long e = p.wide ? reinterpret_cast<const volatile long long*>(p.expert_of)[s] : reinterpret_cast<const volatile int32_t*>(p.expert_of)[s];
    return e >= 0 && e < E ? (int)e : -1;
  };
  int next = expert_at(first + lane);
  for (int s = first; s < last; s += 32) {
    const int e = next;
    next = expert_at(s + 32 + lane);
    const unsigned same = __match_any_sync(0xFFFFFFFFu, e);
    if (e >= 0 && lane == __ffs(same) - 1) mine[e] += __popc(same);
    __syncwarp();
  }
  __syncthreads();
  // running sums over the warps; this block's total of every expert
  for (int e = threadIdx.x; e < E; e += kSortThreads) {
    int sum = 0;
    for (int w = 0; w < kSortWarps; ++w) {
      const int c = hist[w * E + e];
      hist[w * E + e] = sum;
      sum += c;
    }
    totals[e] = sum;
  }
  cluster.sync();
  // offsets of all segments (an expert per thread), and where this block's rows of an expert begin
  const int e = threadIdx.x;
  int before = 0, count = 0;
  if (e < E) {
    for (unsigned c = 0; c < cluster.num_blocks(); ++c) {
      const int other = *cluster.map_shared_rank(totals + e, c);
      if (c < cluster.block_rank()) before += other;
      count += other;
    }
  }
  const int padded = (count + kFp8Block - 1) & ~(kFp8Block - 1);
  int sum = padded;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int up = __shfl_up_sync(0xFFFFFFFFu, sum, d);
    if (lane >= d) sum += up;
  }
  if (lane == 31) warp_sum[warp] = sum;
  __syncthreads();
  if (warp == 0) {
    int w = warp_sum[lane];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int up = __shfl_up_sync(0xFFFFFFFFu, w, d);
      if (lane >= d) w += up;
    }
    warp_sum[lane] = w;
  }
  __syncthreads();
  const int begin = sum - padded + (warp ? warp_sum[warp - 1] : 0);
  if (e < E) {
    offset[e] = begin;
    base[e] = begin + before;
    if (e == E - 1) offset[E] = begin + padded;
    if (cluster.block_rank() == 0) {
      p.counts[e] = count;
      p.offsets[e] = begin;
      if (e == E - 1) p.offsets[E] = begin + padded;
    }
    // padding of the segment: rows behind its last slot
    if (e % cluster.num_blocks() == cluster.block_rank())
      for (int r = begin + count; r < begin + padded; ++r) p.slot_of[r] = -1;
  }
  __syncthreads();
  next = expert_at(first + lane);
  for (int s = first; s < last; s += 32) {
    const int x = next;
    next = expert_at(s + 32 + lane);
    const unsigned same = __match_any_sync(0xFFFFFFFFu, x);
    int row = -1;
    if (x >= 0) row = base[x] + mine[x] + __popc(same & ((1u << lane) - 1u));
    __syncwarp();
    if (x >= 0 && lane == __ffs(same) - 1) mine[x] += __popc(same);
    __syncwarp();
    if (s + lane < last) {
      p.row_of[s + lane] = row;
      if (row >= 0) p.slot_of[row] = s + lane;
    }
  }
  for (int r = offset[E] + cluster.block_rank() * kSortThreads + threadIdx.x; r < p.rows; r += kSortThreads * cluster.num_blocks()) p.slot_of[r] = -1;
  cluster.sync();                                    // a block's totals are read until here
}

// ------------------------------------------------------------------------------------------------
// Moving rows.  All three are bound by memory; 8 values (16 or 32 bytes) of a row per lane and step.
// ------------------------------------------------------------------------------------------------
template <typename T>
struct Vec8 {
  float v[8];
  __device__ __forceinline__ void load(const T* src) {
    const uint4 a = load_vec16(src);
    if constexpr (std::is_same_v<T, float>) {
      const uint4 b = load_vec16(src + 4);
      const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
    } else {
      const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
    }
  }
  __device__ __forceinline__ void store(T* dst) const {
    if constexpr (std::is_same_v<T, float>) {
      reinterpret_cast<float4*>(dst)[0] = make_float4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<float4*>(dst)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
      }
      *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
};

// A weight that the kernel before this one may have written.
__device__ __forceinline__ float weight_at(const void* w, int dtype, int64_t i) {
  if (!w) return 1.0f;
  if (dtype == NVFP4_BF16) {
    const uint32_t bits = reinterpret_cast<const volatile uint16_t*>(w)[i];
    return __uint_as_float(bits << 16);
  }
  return reinterpret_cast<const volatile float*>(w)[i];
}
__device__ __forceinline__ int int_at(const int32_t* p, int64_t i) { return reinterpret_cast<const volatile int32_t*>(p)[i]; }

struct MoveParams {
  const void *x, *rows, *weights;
  void *out, *drows, *dweights;
  const int32_t *slot_of, *row_of, *used;
  int64_t tokens, n_rows, cols, ld;
  int topk, weights_dtype;
  int64_t pieces;               // per row
};

constexpr int kMoveWarps = 8;
constexpr int kGatherCols = 1024, kCombineCols = 256;

// One warp moves up to 1024 columns of a row.
template <typename T>
__global__ void __launch_bounds__(32 * kMoveWarps) expert_gather_kernel(const MoveParams p) {
  const int lane = threadIdx.x & 31;
  const int64_t item = (int64_t)blockIdx.x * kMoveWarps + (threadIdx.x >> 5);
  const int64_t r = item / p.pieces, c0 = (item - r * p.pieces) * kGatherCols + lane * 8;
  grid_dependency_wait();
  grid_dependency_trigger();
  if (r >= p.n_rows || r >= int_at(p.used, 0)) return;
  int slot = int_at(p.slot_of, r);
  if (slot >= p.tokens * p.topk) slot = -1;          // no such slot
  const float w = slot >= 0 ? weight_at(p.weights, p.weights_dtype, slot) : 0.0f;
  const T* const src = static_cast<const T*>(p.x) + (int64_t)(slot < 0 ? 0 : slot / p.topk) * p.ld + c0;
  T* const dst = static_cast<T*>(p.out) + r * p.cols + c0;
  Vec8<T> v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int q = 0; q < 8; ++q) v[i].v[q] = 0.0f;
    if (slot >= 0 && c0 + 256 * i < p.cols) v[i].load(src + 256 * i);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (c0 + 256 * i >= p.cols) break;
    if (p.weights) {
#pragma unroll
      for (int q = 0; q < 8; ++q) v[i].v[q] = slot >= 0 ? __fmul_rn(v[i].v[q], w) : 0.0f;
    }
    v[i].store(dst + 256 * i);
  }
}

// One warp computes 256 columns of a token.
template <typename T>
__global__ void __launch_bounds__(32 * kMoveWarps) expert_combine_kernel(const MoveParams p) {
  const int lane = threadIdx.x & 31;
  const int64_t item = (int64_t)blockIdx.x * kMoveWarps + (threadIdx.x >> 5);
  const int64_t t = item / p.pieces, c = (item - t * p.pieces) * kCombineCols + lane * 8;
  grid_dependency_wait();
  grid_dependency_trigger();
  if (t >= p.tokens || c >= p.cols) return;
  float sum[8] = {};
  for (int j0 = 0; j0 < p.topk; j0 += 4) {           // four rows in flight
    Vec8<T> v[4];
    float w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t s = t * p.topk + j0 + j;
      int r = j0 + j < p.topk ? int_at(p.row_of, s) : -1;
      if (r >= p.n_rows) r = -1;                     // no such row
      w[j] = r >= 0 ? weight_at(p.weights, p.weights_dtype, s) : 0.0f;
#pragma unroll
      for (int q = 0; q < 8; ++q) v[j].v[q] = 0.0f;
      if (r >= 0) v[j].load(static_cast<const T*>(p.rows) + (int64_t)r * p.cols + c);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int q = 0; q < 8; ++q) sum[q] = __fmaf_rn(w[j], v[j].v[q], sum[q]);
  }
  Vec8<T> out;
#pragma unroll
  for (int q = 0; q < 8; ++q) out.v[q] = sum[q];
  out.store(static_cast<T*>(p.out) + t * p.cols + c);
}

// One warp takes a slot (in the order of tokens: a token's row of dy comes from memory once); the warps behind those look at 32
// rows each and clear the padding rows among them.
template <typename T>
__global__ void __launch_bounds__(32 * kMoveWarps) expert_combine_bwd_kernel(const MoveParams p) {
  const int lane = threadIdx.x & 31;
  const int64_t slots = p.tokens * p.topk, item = (int64_t)blockIdx.x * kMoveWarps + (threadIdx.x >> 5);
  grid_dependency_wait();
  grid_dependency_trigger();
  if (item < slots) {
    int r = int_at(p.row_of, item);
    if (r >= p.n_rows) r = -1;                       // no such row
    float dot = 0.0f;
    if (r >= 0) {
      const float w = weight_at(p.weights, p.weights_dtype, item);
      const T* const dy = static_cast<const T*>(p.x) + item / p.topk * p.ld;
      const T* const row = static_cast<const T*>(p.rows) + (int64_t)r * p.cols;
      T* const drow = p.drows ? static_cast<T*>(p.drows) + (int64_t)r * p.cols : nullptr;
      for (int64_t c = lane * 8; c < p.cols; c += 1024) {
        Vec8<T> a[4], b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (c + 256 * i < p.cols) { a[i].load(dy + c + 256 * i); b[i].load(row + c + 256 * i); }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (c + 256 * i >= p.cols) break;
#pragma unroll
          for (int q = 0; q < 8; ++q) dot = __fmaf_rn(a[i].v[q], b[i].v[q], dot);
          if (drow) {
#pragma unroll
            for (int q = 0; q < 8; ++q) a[i].v[q] = __fmul_rn(a[i].v[q], w);
            a[i].store(drow + c + 256 * i);
          }
        }
      }
#pragma unroll
      for (int d = 16; d; d >>= 1) dot += __shfl_xor_sync(0xFFFFFFFFu, dot, d);
    }
    if (lane == 0) {
      if (p.weights_dtype == NVFP4_BF16) static_cast<__nv_bfloat16*>(p.dweights)[item] = __float2bfloat16_rn(dot);
      else static_cast<float*>(p.dweights)[item] = dot;
    }
    return;
  }
  if (!p.drows) return;
  const int64_t r0 = (item - slots) * 32;
  const int64_t used = min((int64_t)int_at(p.used, 0), p.n_rows);
  unsigned pads = __ballot_sync(0xFFFFFFFFu, r0 + lane < used && int_at(p.slot_of, min(r0 + lane, p.n_rows - 1)) < 0);
  Vec8<T> zero;
#pragma unroll
  for (int q = 0; q < 8; ++q) zero.v[q] = 0.0f;
  for (; pads; pads &= pads - 1) {
    T* const drow = static_cast<T*>(p.drows) + (r0 + __ffs(pads) - 1) * p.cols;
    for (int64_t c = lane * 8; c < p.cols; c += 256) zero.store(drow + c);
  }
}

template <typename Kernel>
int launch_warps(Kernel kernel, int64_t warps, const MoveParams& p, cudaStream_t s) {
  const int64_t blocks = ceil_div(warps, kMoveWarps);
  if (blocks > 0x7FFFFFFFll) return NVFP4_ERR_SHAPE;
  return launch_overlapped(kernel, dim3((unsigned)blocks), 32 * kMoveWarps, 0, s, p) == cudaSuccess ? NVFP4_OK : NVFP4_ERR_CUDA;
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
bool aligned_for(const void* p, int dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype == NVFP4_BF16 ? 1u : 3u)) == 0; }
bool dtype_ok(int dtype) { return dtype == NVFP4_BF16 || dtype == NVFP4_FP32; }

}  // namespace
}  // namespace nvfp4

using namespace nvfp4;

extern "C" int64_t nvfp4_expert_rows(int64_t tokens, int64_t topk, int64_t experts) {
  constexpr int64_t kMost = (1ll << 31) - 512;
  if (tokens <= 0 || topk <= 0 || experts <= 0 || experts > kMaxExperts || topk > kMost / tokens) return 0;
  const int64_t n = tokens * topk, rows = (n + (kFp8Block - 1) * std::min(n, experts)) / kFp8Block * kFp8Block;
  return rows <= kMost ? rows : 0;
}

extern "C" int nvfp4_expert_sort(const void* expert_of, int wide, int64_t tokens, int64_t topk, int64_t experts, int32_t* counts,
                                 int32_t* offsets, int32_t* row_of, int32_t* slot_of, void* cuda_stream) {
  if (!expert_of || !counts || !offsets || !row_of || !slot_of) return NVFP4_ERR_NULL;
  if (wide != 0 && wide != 1) return NVFP4_ERR_ENUM;
  const int64_t rows = nvfp4_expert_rows(tokens, topk, experts);
  if (rows == 0) return NVFP4_ERR_SHAPE;
  if (!aligned4(counts) || !aligned4(offsets) || !aligned4(row_of) || !aligned4(slot_of) ||
      (reinterpret_cast<uintptr_t>(expert_of) & (wide ? 7u : 3u)))
    return NVFP4_ERR_ALIGN;
  if (int st = check_arch()) return st;
  const int64_t n = tokens * topk;
  const int cluster = (int)std::clamp<int64_t>(ceil_div(n, 32 * kSortWarps), 1, kMaxCluster);
  SortParams p;
  p.expert_of = expert_of; p.wide = wide;
  p.n = (int)n; p.experts = (int)experts; p.rows = (int)rows;
  p.per_warp = (int)(ceil_div(n, 32 * kSortWarps * cluster) * 32);
  p.counts = counts; p.offsets = offsets; p.row_of = row_of; p.slot_of = slot_of;
  const size_t smem = sizeof(int) * ((kSortWarps + 3) * experts + 1);
  static DeviceFlags smem_set;
  if (set_max_dynamic_smem(smem_set, expert_sort_kernel, (int)(sizeof(int) * ((kSortWarps + 3) * kMaxExperts + 1))) != cudaSuccess) return NVFP4_ERR_CUDA;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(cluster); cfg.blockDim = dim3(kSortThreads); cfg.dynamicSmemBytes = smem;
  cfg.stream = static_cast<cudaStream_t>(cuda_stream);
  cfg.attrs = attr; cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, expert_sort_kernel, p) == cudaSuccess ? NVFP4_OK : NVFP4_ERR_CUDA;
}

extern "C" int nvfp4_expert_gather(const void* x, int dtype, int64_t tokens, int64_t topk, int64_t experts, int64_t cols, int64_t ld,
                                   const int32_t* offsets, const int32_t* slot_of, const void* weights, int weights_dtype, void* rows,
                                   void* cuda_stream) {
  if (!x || !offsets || !slot_of || !rows) return NVFP4_ERR_NULL;
  if (!dtype_ok(dtype) || !dtype_ok(weights_dtype)) return NVFP4_ERR_ENUM;
  const int64_t n_rows = nvfp4_expert_rows(tokens, topk, experts);
  if (n_rows == 0 || cols <= 0 || cols % 8 != 0 || ld < cols) return NVFP4_ERR_SHAPE;
  if (!aligned16(x) || !aligned16(rows) || ld % 8 != 0 || !aligned4(offsets) || !aligned4(slot_of) || !aligned_for(weights, weights_dtype))
    return NVFP4_ERR_ALIGN;
  if (int st = check_arch()) return st;
  MoveParams p = {};
  p.x = x; p.weights = weights; p.out = rows; p.slot_of = slot_of; p.used = offsets + experts;
  p.tokens = tokens; p.n_rows = n_rows; p.cols = cols; p.ld = ld; p.topk = (int)topk; p.weights_dtype = weights_dtype;
  p.pieces = ceil_div(cols, kGatherCols);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  return dtype == NVFP4_BF16 ? launch_warps(expert_gather_kernel<__nv_bfloat16>, n_rows * p.pieces, p, s)
                             : launch_warps(expert_gather_kernel<float>, n_rows * p.pieces, p, s);
}

extern "C" int nvfp4_expert_combine(const void* rows, int dtype, int64_t tokens, int64_t topk, int64_t experts, int64_t cols,
                                    const int32_t* row_of, const void* weights, int weights_dtype, void* y, void* cuda_stream) {
  if (!rows || !row_of || !y) return NVFP4_ERR_NULL;
  if (!dtype_ok(dtype) || !dtype_ok(weights_dtype)) return NVFP4_ERR_ENUM;
  const int64_t n_rows = nvfp4_expert_rows(tokens, topk, experts);
  if (n_rows == 0 || cols <= 0 || cols % 8 != 0) return NVFP4_ERR_SHAPE;
  if (!aligned16(rows) || !aligned16(y) || !aligned4(row_of) || !aligned_for(weights, weights_dtype)) return NVFP4_ERR_ALIGN;
  if (int st = check_arch()) return st;
  MoveParams p = {};
  p.rows = rows; p.weights = weights; p.out = y; p.row_of = row_of;
  p.tokens = tokens; p.n_rows = n_rows; p.cols = cols; p.topk = (int)topk; p.weights_dtype = weights_dtype;
  p.pieces = ceil_div(cols, kCombineCols);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  return dtype == NVFP4_BF16 ? launch_warps(expert_combine_kernel<__nv_bfloat16>, tokens * p.pieces, p, s)
                             : launch_warps(expert_combine_kernel<float>, tokens * p.pieces, p, s);
}

extern "C" int nvfp4_expert_combine_bwd(const void* dy, int dtype, int64_t tokens, int64_t topk, int64_t experts, int64_t cols, int64_t ld,
                                        const int32_t* offsets, const int32_t* slot_of, const int32_t* row_of, const void* rows,
                                        const void* weights, int weights_dtype, void* drows, void* dweights, void* cuda_stream) {
  if (!dy || !offsets || !slot_of || !row_of || !rows || !weights || !dweights) return NVFP4_ERR_NULL;
  if (!dtype_ok(dtype) || !dtype_ok(weights_dtype)) return NVFP4_ERR_ENUM;
  const int64_t n_rows = nvfp4_expert_rows(tokens, topk, experts);
  if (n_rows == 0 || cols <= 0 || cols % 8 != 0 || ld < cols) return NVFP4_ERR_SHAPE;
  if (!aligned16(dy) || !aligned16(rows) || !aligned16(drows) || ld % 8 != 0 || !aligned4(offsets) || !aligned4(slot_of) || !aligned4(row_of) ||
      !aligned_for(weights, weights_dtype) || !aligned_for(dweights, weights_dtype))
    return NVFP4_ERR_ALIGN;
  if (int st = check_arch()) return st;
  MoveParams p = {};
  p.x = dy; p.rows = rows; p.weights = weights; p.drows = drows; p.dweights = dweights;
  p.slot_of = slot_of; p.row_of = row_of; p.used = offsets + experts;
  p.tokens = tokens; p.n_rows = n_rows; p.cols = cols; p.ld = ld; p.topk = (int)topk; p.weights_dtype = weights_dtype;
  const int64_t warps = tokens * topk + (drows ? ceil_div(n_rows, 32) : 0);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  return dtype == NVFP4_BF16 ? launch_warps(expert_combine_bwd_kernel<__nv_bfloat16>, warps, p, s)
                             : launch_warps(expert_combine_bwd_kernel<float>, warps, p, s);
}
