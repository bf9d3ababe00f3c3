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
// another by votes), the counts become running sums over the warps, the blocks read one another's totals from shared
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

// The lanes that carry the same expert (meaningless for a dropped slot): a vote for each of its bits.  262144 slots, 64 experts, with one
// match instruction instead, of which a multiprocessor does one in about 60 cycles: 70 us; so: 50.
__device__ __forceinline__ unsigned same_expert(int e, int bits) {
  unsigned same = __ballot_sync(0xFFFFFFFFu, e >= 0);
  for (int b = 0; b < bits; ++b) {
    const bool bit = (e >> b) & 1;
    const unsigned set = __ballot_sync(0xFFFFFFFFu, bit);
    same &= bit ? set : ~set;
  }
  return same;
}

__global__ void __launch_bounds__(kSortThreads, 1) expert_sort_kernel(const SortParams p) {
  extern __shared__ int hist[];                      // [kSortWarps][stride], then totals, base, end [experts] and offset [experts + 1]
  __shared__ int warp_sum[kSortWarps];
  cg::cluster_group cluster = cg::this_cluster();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int E = p.experts, bits = 32 - __clz(E - 1);   // an expert's number
  const int stride = E | 1;                          // odd: 32 warps' counts of an expert lie in 32 banks
  int* const totals = hist + kSortWarps * stride;
  int* const base = totals + E;
  int* const end = base + E;
  int* const offset = end + E;
  int* const mine = hist + warp * stride;
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
  // four loads in flight; a range of up to 128 slots stays in registers for the second pass
  int at[4];
  auto fetch = [&](int s0) {
#pragma unroll
    for (int q = 0; q < 4; ++q) at[q] = expert_at(s0 + 32 * q + lane);
  };
  for (int s0 = first; s0 < last; s0 += 128) {
    fetch(s0);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (s0 + 32 * q >= last) break;
      const unsigned same = same_expert(at[q], bits);
      if (at[q] >= 0 && lane == __ffs(same) - 1) mine[at[q]] += __popc(same);
      __syncwarp();
    }
  }
  __syncthreads();
  // running sums over the warps (a lane each); this block's total of every expert
  for (int e = warp; e < E; e += kSortWarps) {
    const int c = hist[lane * stride + e];
    int sum = c;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int up = __shfl_up_sync(0xFFFFFFFFu, sum, d);
      if (lane >= d) sum += up;
    }
    hist[lane * stride + e] = sum - c;
    if (lane == 31) totals[e] = sum;
  }
  cluster.sync();
  // offsets of all segments (an expert per thread), and where this block's rows of an expert begin
  const int e = threadIdx.x;
  int before = 0, count = 0;
  if (e < E) {
#pragma unroll
    for (unsigned c = 0; c < kMaxCluster; ++c) {
      const int other = c < cluster.num_blocks() ? *cluster.map_shared_rank(totals + e, c) : 0;
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
    end[e] = begin + count;
  }
  __syncthreads();
  // padding of the segments: rows behind their last slots
  for (int s = cluster.block_rank() * kSortWarps + warp; s < E; s += kSortWarps * cluster.num_blocks())
    for (int r = end[s] + lane; r < offset[s + 1]; r += 32) p.slot_of[r] = -1;
  for (int s0 = first; s0 < last; s0 += 128) {
    if (last - first > 128) fetch(s0);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int s = s0 + 32 * q;
      if (s >= last) break;
      const int x = at[q];
      const unsigned same = same_expert(x, bits);
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
  }
  for (int r = offset[E] + cluster.block_rank() * kSortThreads + threadIdx.x; r < p.rows; r += kSortThreads * cluster.num_blocks()) p.slot_of[r] = -1;
  cluster.sync();                                    // a block's totals are read until here
}

// ------------------------------------------------------------------------------------------------
// Moving rows.  All three are bound by memory, in units of 16 bytes of a row.  What they read first are indices, so a warp fetches
// all that it needs at once (a lane each) and then has 4 to 12 units per lane in flight; it works in the order of tokens, so that a
// token's row is read once however many choices it has.
// 16384 tokens, two of 8 experts, bf16 (buffers in turn): 4096 columns gather 70 us = 5.8 TB/s (two thirds of it written), combine 61 =
// 6.6, its gradient 107 = 6.3, that of the weights alone 60 = 6.7; 2816 columns 50 / 45 / 76 / 43.  The sort 7 us (one token 3.7).
// ------------------------------------------------------------------------------------------------
template <typename T>
constexpr int kUnit = 16 / (int)sizeof(T);           // values per unit
template <typename T>
__device__ __forceinline__ void unpack(const uint4& u, float (&v)[kUnit<T>]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) v[i] = __uint_as_float(w[i]);
    else { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
  }
}
template <typename T>
__device__ __forceinline__ uint4 pack(const float (&v)[kUnit<T>]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(v[i]);
    else {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T>
__device__ __forceinline__ uint4 scaled(const uint4& u, float w) {
  float v[kUnit<T>];
  unpack<T>(u, v);
#pragma unroll
  for (int i = 0; i < kUnit<T>; ++i) v[i] = __fmul_rn(v[i], w);
  return pack<T>(v);
}

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
  int units;                    // of a row
  int item_blocks;              // blocks that move rows, in front of those that clear padding
  int piece_bits;               // gradient of the combination
};

constexpr int kMoveWarps = 8;

// Clears the padding rows among the eight that this warp looks at; gridDim.y warps share them.  block: among those that do this.
__device__ __forceinline__ void clear_padding(const MoveParams& p, void* rows, int64_t row_units, int64_t block) {
  const int lane = threadIdx.x & 31;
  const int64_t r0 = (block * kMoveWarps + (threadIdx.x >> 5)) * 8;
  const int64_t used = min((int64_t)int_at(p.used, 0), p.n_rows);
  unsigned pads = __ballot_sync(0xFFFFFFFFu, lane < 8 && r0 + lane < used && int_at(p.slot_of, min(r0 + lane, p.n_rows - 1)) < 0);
  for (; pads; pads &= pads - 1) {
    uint4* const row = static_cast<uint4*>(rows) + (r0 + __ffs(pads) - 1) * row_units;
    for (int u = blockIdx.y * 32 + lane; u < p.units; u += gridDim.y * 32) row[u] = make_uint4(0, 0, 0, 0);
  }
}

// A warp takes a token, so that its row is read once, and stores it to the rows of its choices, 32 * U units at a time; gridDim.y
// warps share it.  The blocks behind those clear padding rows.
template <typename T, int U>
__global__ void __launch_bounds__(32 * kMoveWarps, 4) expert_gather_kernel(const MoveParams p) {
  const int lane = threadIdx.x & 31;
  grid_dependency_wait();
  grid_dependency_trigger();
  if (blockIdx.x >= (unsigned)p.item_blocks) return clear_padding(p, p.out, p.units, blockIdx.x - p.item_blocks);
  const int64_t t = (int64_t)blockIdx.x * kMoveWarps + (threadIdx.x >> 5);
  if (t >= p.tokens) return;
  const uint4* const src = reinterpret_cast<const uint4*>(static_cast<const T*>(p.x) + t * p.ld);
  for (int u0 = blockIdx.y * 32 * U + lane; u0 - lane < p.units; u0 += gridDim.y * 32 * U) {
    uint4 v[U];
#pragma unroll
    for (int i = 0; i < U; ++i) v[i] = u0 + 32 * i < p.units ? load_vec16(src + u0 + 32 * i) : make_uint4(0, 0, 0, 0);
    for (int j0 = 0; j0 < p.topk; j0 += 32) {        // a lane fetches the row and the weight of a choice
      int row = -1;
      float weight = 1.0f;
      if (j0 + lane < p.topk) {
        const int64_t s = t * p.topk + j0 + lane;
        row = int_at(p.row_of, s);
        weight = weight_at(p.weights, p.weights_dtype, s);
        if (row >= p.n_rows) row = -1;               // no such row
      }
      const int n = min(32, p.topk - j0);
      for (int j = 0; j < n; ++j) {
        const int to = __shfl_sync(0xFFFFFFFFu, row, j);
        const float w = __shfl_sync(0xFFFFFFFFu, weight, j);
        if (to < 0) continue;
        uint4* const dst = static_cast<uint4*>(p.out) + (int64_t)to * p.units;
#pragma unroll
        for (int i = 0; i < U; ++i)
          if (u0 + 32 * i < p.units) dst[u0 + 32 * i] = p.weights ? scaled<T>(v[i], w) : v[i];
      }
    }
  }
}

// A warp computes a token, 32 * U units at a time of J rows at a time; gridDim.y warps share it.
template <typename T, int U, int J>
__global__ void __launch_bounds__(32 * kMoveWarps) expert_combine_kernel(const MoveParams p) {
  const int lane = threadIdx.x & 31;
  const int64_t t = (int64_t)blockIdx.x * kMoveWarps + (threadIdx.x >> 5);
  if (t >= p.tokens) return;
  grid_dependency_wait();
  grid_dependency_trigger();
  int row = -1;                                      // of the lane's choice, of 32 at a time
  float weight = 0.0f;
  auto fetch = [&](int j0) {
    row = -1;
    if (j0 + lane < p.topk) {
      const int64_t s = t * p.topk + j0 + lane;
      row = int_at(p.row_of, s);
      weight = weight_at(p.weights, p.weights_dtype, s);
      if (row >= p.n_rows) row = -1;                 // no such row
    }
  };
  fetch(0);
  uint4* const dst = reinterpret_cast<uint4*>(static_cast<T*>(p.out) + t * p.cols);
  for (int u = blockIdx.y * 32 * U; u < p.units; u += gridDim.y * 32 * U) {
    const int u0 = u + lane;
    float sum[U][kUnit<T>] = {};
    for (int j0 = 0; j0 < p.topk; j0 += 32) {
      if (p.topk > 32) fetch(j0);
      const int n = min(32, p.topk - j0);
      for (int j = 0; j < n; j += J) {
        uint4 v[J][U];
#pragma unroll
        for (int q = 0; q < J; ++q) {
          const int from = j + q < n ? __shfl_sync(0xFFFFFFFFu, row, j + q) : -1;
          const uint4* const src = reinterpret_cast<const uint4*>(static_cast<const T*>(p.rows) + (int64_t)max(from, 0) * p.cols);
#pragma unroll
          for (int i = 0; i < U; ++i) v[q][i] = from >= 0 && u0 + 32 * i < p.units ? load_vec16(src + u0 + 32 * i) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int q = 0; q < J; ++q) {
          if (j + q >= n || __shfl_sync(0xFFFFFFFFu, row, j + q) < 0) continue;
          const float w = __shfl_sync(0xFFFFFFFFu, weight, j + q);
#pragma unroll
          for (int i = 0; i < U; ++i) {
            float x[kUnit<T>];
            unpack<T>(v[q][i], x);
#pragma unroll
            for (int e = 0; e < kUnit<T>; ++e) sum[i][e] = __fmaf_rn(w, x[e], sum[i][e]);
          }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (u0 + 32 * i < p.units) dst[u0 + 32 * i] = pack<T>(sum[i]);
  }
}

// 2^piece_bits warps of a block take J choices of a token (in the order of tokens: a row of dy comes from memory once), 32 * U units of
// all rows each at a time, and join their parts of the products in shared memory; the blocks behind those look at eight rows a warp
// and clear the padding rows among them.
template <typename T, int J, int U>
__global__ void __launch_bounds__(32 * kMoveWarps, 3) expert_combine_bwd_kernel(const MoveParams p) {
  __shared__ float parts[J][kMoveWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const unsigned groups = (p.topk + J - 1) / J;
  grid_dependency_wait();
  grid_dependency_trigger();
  if (blockIdx.x < (unsigned)p.item_blocks) {
    const int piece = warp & ((1 << p.piece_bits) - 1);
    // items are fewer than slots: 32 bits
    const unsigned item = blockIdx.x * (kMoveWarps >> p.piece_bits) + (warp >> p.piece_bits), t = item / groups, j0 = (item - t * groups) * J;
    const int n = t < p.tokens ? min(J, (int)(p.topk - j0)) : 0;
    const int64_t s0 = (int64_t)t * p.topk + j0;
    const uint4* const dy = reinterpret_cast<const uint4*>(static_cast<const T*>(p.x) + (int64_t)(n ? t : 0) * p.ld);
    int r[J];
    float w[J], dot[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      r[j] = j < n ? int_at(p.row_of, s0 + j) : -1;
      w[j] = j < n ? weight_at(p.weights, p.weights_dtype, s0 + j) : 0.0f;
      if (r[j] >= p.n_rows) r[j] = -1;               // no such row
      dot[j] = 0.0f;
    }
    for (int u0 = piece * 32 * U + lane; u0 < p.units; u0 += (32 * U) << p.piece_bits) {
      uint4 a[U], b[J][U];
#pragma unroll
      for (int i = 0; i < U; ++i) a[i] = u0 + 32 * i < p.units ? load_vec16(dy + u0 + 32 * i) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const uint4* const row = reinterpret_cast<const uint4*>(static_cast<const T*>(p.rows) + (int64_t)max(r[j], 0) * p.cols);
#pragma unroll
        for (int i = 0; i < U; ++i) b[j][i] = r[j] >= 0 && u0 + 32 * i < p.units ? load_vec16(row + u0 + 32 * i) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int j = 0; j < J; ++j) {
        if (r[j] < 0) continue;
        uint4* const drow = p.drows ? reinterpret_cast<uint4*>(static_cast<T*>(p.drows) + (int64_t)r[j] * p.cols) : nullptr;
#pragma unroll
        for (int i = 0; i < U; ++i) {
          float x[kUnit<T>], y[kUnit<T>];
          unpack<T>(a[i], x);
          unpack<T>(b[j][i], y);
#pragma unroll
          for (int e = 0; e < kUnit<T>; ++e) dot[j] = __fmaf_rn(x[e], y[e], dot[j]);
          if (drow && u0 + 32 * i < p.units) drow[u0 + 32 * i] = scaled<T>(a[i], w[j]);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int d = 16; d; d >>= 1) dot[j] += __shfl_xor_sync(0xFFFFFFFFu, dot[j], d);
    if (p.piece_bits) {
      if (lane == 0)
#pragma unroll
        for (int j = 0; j < J; ++j) parts[j][warp] = dot[j];
      __syncthreads();
    }
    if (piece != 0 || lane >= n) return;
    float sum = dot[0];
#pragma unroll
    for (int j = 1; j < J; ++j)
      if (lane == j) sum = dot[j];
    for (int i = 1; i < 1 << p.piece_bits; ++i) sum += parts[lane][warp + i];
    if (p.weights_dtype == NVFP4_BF16) static_cast<__nv_bfloat16*>(p.dweights)[s0 + lane] = __float2bfloat16_rn(sum);
    else static_cast<float*>(p.dweights)[s0 + lane] = sum;
    return;
  }
  clear_padding(p, p.drows, p.units, blockIdx.x - p.item_blocks);
}

template <typename Kernel>
int launch_blocks(Kernel kernel, int64_t blocks, int64_t pieces, const MoveParams& p, cudaStream_t s) {
  if (blocks > 0x7FFFFFFFll || pieces > 65535) return NVFP4_ERR_SHAPE;
  return launch_overlapped(kernel, dim3((unsigned)blocks, (unsigned)pieces), 32 * kMoveWarps, 0, s, p) == cudaSuccess ? NVFP4_OK : NVFP4_ERR_CUDA;
}
// Warps that share a row of `units`, 32 * u at a time: one where there are rows enough to fill the multiprocessors, since its indices
// and addresses then cost least (16384 tokens, two choices, 2816 columns, us, eight warps -> one: combine 50 -> 45, gradient 104 -> 76).
int64_t row_pieces(int64_t rows, int64_t units, int64_t u) {
  return std::clamp<int64_t>(ceil_div(16 * sm_count(), rows), 1, std::min<int64_t>(ceil_div(units, 32 * u), 65535));
}
template <typename T>
int combine(MoveParams p, cudaStream_t s) {
  p.units = (int)(p.cols / kUnit<T>);
  const int64_t blocks = ceil_div(p.tokens, kMoveWarps);
  if (p.tokens < 16 * sm_count()) return launch_blocks(expert_combine_kernel<T, 1, 8>, blocks, row_pieces(p.tokens, p.units, 1), p, s);
  return launch_blocks(expert_combine_kernel<T, 4, 2>, blocks, 1, p, s);
}
template <typename T>
int gather(MoveParams p, cudaStream_t s) {
  p.units = (int)(p.cols / kUnit<T>);
  p.item_blocks = (int)ceil_div(p.tokens, kMoveWarps);
  const int64_t blocks = p.item_blocks + ceil_div(p.n_rows, 8 * kMoveWarps);
  if (p.tokens < 16 * sm_count()) return launch_blocks(expert_gather_kernel<T, 1>, blocks, row_pieces(p.tokens, p.units, 1), p, s);
  return launch_blocks(expert_gather_kernel<T, 4>, blocks, 1, p, s);
}
template <typename T, int J, int U>
int launch_combine_bwd(MoveParams p, cudaStream_t s) {
  const int64_t items = p.tokens * ceil_div(p.topk, J);
  // several warps for a row where there are few rows
  for (p.piece_bits = 0; p.piece_bits < 3 && (32 * U << p.piece_bits) < p.units && (items << p.piece_bits) < 8 * sm_count();) ++p.piece_bits;
  p.item_blocks = (int)ceil_div(items, kMoveWarps >> p.piece_bits);
  return launch_blocks(expert_combine_bwd_kernel<T, J, U>, p.item_blocks + (p.drows ? ceil_div(p.n_rows, 8 * kMoveWarps) : 0), 1, p, s);
}
template <typename T>
int combine_bwd(MoveParams p, cudaStream_t s) {
  p.units = (int)(p.cols / kUnit<T>);
  // two choices share a token's row of dy, once there are enough of them
  return p.topk > 1 && p.tokens * p.topk >= 32 * sm_count() ? launch_combine_bwd<T, 2, 4>(p, s) : launch_combine_bwd<T, 1, 4>(p, s);
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
bool aligned_for(const void* p, int dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype == NVFP4_BF16 ? 1u : 3u)) == 0; }
bool dtype_ok(int dtype) { return dtype == NVFP4_BF16 || dtype == NVFP4_FP32; }

}  // namespace
}  // namespace nvfp4

using namespace nvfp4;

extern "C" int64_t nvfp4_expert_rows(int64_t tokens, int64_t topk, int64_t experts) {
  constexpr int64_t kMost = (1ll << 31) - 65536;    // an index of a row or a slot, and the strides of the loops over them
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
  const size_t smem = sizeof(int) * (kSortWarps * (experts | 1) + 4 * experts + 1);
  static DeviceFlags smem_set;
  if (set_max_dynamic_smem(smem_set, expert_sort_kernel, (int)(sizeof(int) * (kSortWarps * (kMaxExperts | 1) + 4 * kMaxExperts + 1))) != cudaSuccess) return NVFP4_ERR_CUDA;
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
                                   const int32_t* offsets, const int32_t* slot_of, const int32_t* row_of, const void* weights,
                                   int weights_dtype, void* rows, void* cuda_stream) {
  if (!x || !offsets || !slot_of || !row_of || !rows) return NVFP4_ERR_NULL;
  if (!dtype_ok(dtype) || !dtype_ok(weights_dtype)) return NVFP4_ERR_ENUM;
  const int64_t n_rows = nvfp4_expert_rows(tokens, topk, experts);
  if (n_rows == 0 || cols <= 0 || cols % 8 != 0 || ld < cols || cols > (1ll << 31) - 512) return NVFP4_ERR_SHAPE;
  if (!aligned16(x) || !aligned16(rows) || ld % 8 != 0 || !aligned4(offsets) || !aligned4(slot_of) || !aligned4(row_of) ||
      !aligned_for(weights, weights_dtype))
    return NVFP4_ERR_ALIGN;
  if (int st = check_arch()) return st;
  MoveParams p = {};
  p.x = x; p.weights = weights; p.out = rows; p.slot_of = slot_of; p.row_of = row_of; p.used = offsets + experts;
  p.tokens = tokens; p.n_rows = n_rows; p.cols = cols; p.ld = ld; p.topk = (int)topk; p.weights_dtype = weights_dtype;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  return dtype == NVFP4_BF16 ? gather<__nv_bfloat16>(p, s) : gather<float>(p, s);
}

extern "C" int nvfp4_expert_combine(const void* rows, int dtype, int64_t tokens, int64_t topk, int64_t experts, int64_t cols,
                                    const int32_t* row_of, const void* weights, int weights_dtype, void* y, void* cuda_stream) {
  if (!rows || !row_of || !y) return NVFP4_ERR_NULL;
  if (!dtype_ok(dtype) || !dtype_ok(weights_dtype)) return NVFP4_ERR_ENUM;
  const int64_t n_rows = nvfp4_expert_rows(tokens, topk, experts);
  if (n_rows == 0 || cols <= 0 || cols % 8 != 0 || cols > (1ll << 31) - 512) return NVFP4_ERR_SHAPE;
  if (!aligned16(rows) || !aligned16(y) || !aligned4(row_of) || !aligned_for(weights, weights_dtype)) return NVFP4_ERR_ALIGN;
  if (int st = check_arch()) return st;
  MoveParams p = {};
  p.rows = rows; p.weights = weights; p.out = y; p.row_of = row_of;
  p.tokens = tokens; p.n_rows = n_rows; p.cols = cols; p.topk = (int)topk; p.weights_dtype = weights_dtype;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  return dtype == NVFP4_BF16 ? combine<__nv_bfloat16>(p, s) : combine<float>(p, s);
}

extern "C" int nvfp4_expert_combine_bwd(const void* dy, int dtype, int64_t tokens, int64_t topk, int64_t experts, int64_t cols, int64_t ld,
                                        const int32_t* offsets, const int32_t* slot_of, const int32_t* row_of, const void* rows,
                                        const void* weights, int weights_dtype, void* drows, void* dweights, void* cuda_stream) {
  if (!dy || !offsets || !slot_of || !row_of || !rows || !weights || !dweights) return NVFP4_ERR_NULL;
  if (!dtype_ok(dtype) || !dtype_ok(weights_dtype)) return NVFP4_ERR_ENUM;
  const int64_t n_rows = nvfp4_expert_rows(tokens, topk, experts);
  if (n_rows == 0 || cols <= 0 || cols % 8 != 0 || ld < cols || cols > (1ll << 31) - 512) return NVFP4_ERR_SHAPE;
  if (!aligned16(dy) || !aligned16(rows) || !aligned16(drows) || ld % 8 != 0 || !aligned4(offsets) || !aligned4(slot_of) || !aligned4(row_of) ||
      !aligned_for(weights, weights_dtype) || !aligned_for(dweights, weights_dtype))
    return NVFP4_ERR_ALIGN;
  if (int st = check_arch()) return st;
  MoveParams p = {};
  p.x = dy; p.rows = rows; p.weights = weights; p.drows = drows; p.dweights = dweights;
  p.slot_of = slot_of; p.row_of = row_of; p.used = offsets + experts;
  p.tokens = tokens; p.n_rows = n_rows; p.cols = cols; p.ld = ld; p.topk = (int)topk; p.weights_dtype = weights_dtype;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  return dtype == NVFP4_BF16 ? combine_bwd<__nv_bfloat16>(p, s) : combine_bwd<float>(p, s);
}
