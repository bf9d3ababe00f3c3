// Products of 8-bit operands with a power-of-two scale for each block of 128 (fp8.cuh has the format):
//   D[m,n] = sum_kb 2^(ea[m,kb] + eb[n,kb]) * sum_{k in kb} a[m,k]*b[n,k],  fp32 accumulation.
//
// Bound by the tensor cores for large M, N and K (one instruction, 256 x 256 x 32, takes a CTA pair 128 cycles), by the weights'
// bytes for few rows.  A cluster of two CTAs computes a 256 x BN tile with tcgen05.mma.cta_group::2.kind::mxf8f6f4, which applies
// the scales itself (the accumulator is never rescaled in registers); persistent, warp-specialised, roles and barriers as in the
// NVFP4 pair kernel (gemm.cu): operands by tiled copies into a ring of k-stages of 128 values (128 bytes a row, 128-byte
// swizzle), scales through registers into tensor memory, eight epilogue warps that move the accumulator out and store it by
// tiled copies.  A stage is one block of the scales: a 512-byte scale tile (128 rows x 4 blocks) serves four stages; it goes to
// tensor memory as it is, four columns per 128 rows, and an instruction's descriptor names the byte of the column that is its stage's block.
//
// One kernel, three forms (GROUPS):
//   0  one product
//   1  the rows of A and D lie in segments, one for each matrix of B (the layer of experts forward, and its input gradient)
//   2  the contraction axis lies in segments, one for each matrix of D (the weight gradient)
// Segments begin at multiples of 128 rows, which the host does not know: the blocks count tiles from the offsets in device memory.
#include <cuda.h>
#include <cuda_bf16.h>

#include <algorithm>

#include "bounded_waits.cuh"
#include "fp8.cuh"
#include "tc_ptx.cuh"
#include "tensor_map.cuh"

namespace nvfp4 {
namespace {

constexpr int kThreads = 512;
constexpr int kBK = 128;                           // values, and bytes of a row, per block of a k-stage
constexpr uint32_t kTmemCols = 512;
constexpr int kControlRegs = 72, kEpilogueRegs = 184;   // 256 x (72 + 184) = 65536, what the CTA is launched with

template <int BN>
struct Cfg {
  // Blocks per k-stage.  The roles' hand-over of a stage takes about as long as a block's instructions of 128 columns, so that narrow
  // tiles take two blocks at a time (us, one / two: 704 x 704 x 16384 35.0 / 30.3, 512 x 4096 x 11008 27.4 / 24.5; 192 columns 16384 x
  // 4096 x 4096 213 / 200); wide ones lose by it what the ring has in depth (16384 x 1024 x 2816 41.1 / 41.8).
  static constexpr int kSub = BN == 256 ? 1 : 2;
  static constexpr int kStages = BN == 128 ? 4 : BN == 192 ? 3 : 6;
  static constexpr int kAccStages = BN == 256 ? 1 : 2;
  static constexpr int kABytes = 128 * kBK;
  static constexpr int kBBytes = (BN / 2) * kBK;
  static constexpr int kSfbTiles = (BN + 127) / 128;   // a tile of 192 columns begins at the middle or at the beginning of one
  static constexpr int kSfBytes = (1 + kSfbTiles) * 512;
  static constexpr int kBlockBytes = kABytes + kBBytes;
  static constexpr int kStageBytes = kSub * kBlockBytes;
  static constexpr int kSfSlots = 4;               // of scale tiles, each for up to four stages
  static constexpr int kEpiWarpBytes = 2048;       // a 32-row x 64-byte staging buffer per epilogue warp
  static constexpr int kEpiBytes = 8 * kEpiWarpBytes;
  static constexpr int kBarrierBytes = 512;
  static constexpr int kTableBytes = (kMaxExperts + 1) * 8 + 8;      // per segment: its first tile and its offset
  static constexpr int kSmemBytes = kStages * kStageBytes + kEpiBytes + kSfSlots * kSfBytes + kBarrierBytes + kTableBytes + 1024 /*align*/;
  // tensor memory: accumulators, then 16 columns per slot of scales (4 for A, 4 per 128 rows of B)
  static constexpr uint32_t kSfCol = kAccStages * BN;
  static constexpr int kNumBarriers = 2 * kStages + 3 * kSfSlots + 2 * kAccStages;
  static_assert(kSmemBytes <= 232448, "shared memory overflow");
  static_assert(8 * kNumBarriers + 8 <= kBarrierBytes, "barrier area overflow");
  static_assert(kSfCol + 16 * kSfSlots <= kTmemCols, "tensor memory overflow");
};

struct Params {
  CUtensorMap a, b, sfa, sfb, d;
  const int32_t* offsets;           // of the segments (GROUPS != 0), experts + 1
  int experts, rows;                // rows: of all segments, at most
  int M, N;                         // GROUPS == 1: M = all rows
  int tiles_m, tiles_n;             // GROUPS == 1: tiles_m comes from the offsets
  int k_blocks, k_mmas;             // GROUPS == 2: from the offsets
  int sfa_ktiles, sfb_ktiles;       // scale tiles along a row of them
  int a_row_tiles, b_row_tiles;     // row tiles of one matrix
  int d_is_bf16;
  int late;                         // nothing that it reads or writes is the kernel before's (launch_overlapped)
  int ragged;                       // a row of D ends between two multiples of 16 bytes
  void* out;                        // D, for that case
  int64_t ldd;
};

// What a pair of CTAs computes at one time.
struct Tile {
  int m0, n0;                       // first row of A and of D, first row of B within its matrix = first column of D
  int e;                            // matrix of B (GROUPS 1) or of D (GROUPS 2)
  int kb0, blocks;                  // first block along the contraction axis, and how many
  int m_end;                        // rows from here on are not stored
};

constexpr int kPanel = 8;           // row tiles of a panel, as in gemm.cu: concurrent tiles share operands in the level-two cache
__device__ __forceinline__ void tile_coords(int tile, int tiles_m, int tiles_n, int& tm, int& tn) {
  const int per_panel = kPanel * tiles_n;
  const int panel = tile / per_panel, in_panel = tile - panel * per_panel;
  const int height = min(kPanel, tiles_m - panel * kPanel);
  tn = in_panel / height;
  tm = panel * kPanel + in_panel - tn * height;
}

// Contractions longer than kMostBlocks blocks are summed in equal parts, which the epilogue adds up in registers (LONG: a kernel of
// their own, since the others lose 2 % by the choice).  A part costs a turn-round of the accumulator.
template <bool LONG>
__device__ __forceinline__ int part_blocks(int blocks, int sub) {
  if (!LONG || blocks <= kMostBlocks) return blocks;
  const int parts = (blocks + kMostBlocks - 1) / kMostBlocks;
  return ((blocks + parts - 1) / parts + sub - 1) / sub * sub;
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr) : "memory");
  tmem_ld_wait();
#pragma unroll
  for (int i = 0; i < 16; i += 4) asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3])::"memory");
}

// The table of segments in shared memory: firsts[e] the first tile of segment e, offsets[e] its first row.
struct Segments {
  const int* firsts;
  const int* offsets;
};

template <int BN, int GROUPS>
__device__ __forceinline__ bool tile_at(const Params& p, const Segments& seg, int item, Tile& t) {
  int tm, tn;
  if constexpr (GROUPS == 0) {
    if (item >= p.tiles_m * p.tiles_n) return false;
    tile_coords(item, p.tiles_m, p.tiles_n, tm, tn);
    t.e = 0; t.kb0 = 0; t.blocks = p.k_blocks; t.m_end = p.M;
    t.m0 = tm * 256;
  } else if constexpr (GROUPS == 1) {
    if (item >= seg.firsts[p.experts]) return false;
    int lo = 0, hi = p.experts;                    // the last segment that begins at or before the item
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (seg.firsts[mid] <= item) lo = mid; else hi = mid;
    }
    t.e = lo;
    const int begin = seg.offsets[lo];
    t.m_end = seg.offsets[lo + 1];
    tile_coords(item - seg.firsts[lo], (t.m_end - begin + 255) >> 8, p.tiles_n, tm, tn);   // a segment with a tile has rows
    t.kb0 = 0; t.blocks = p.k_blocks;
    t.m0 = begin + tm * 256;
  } else {
    const int per = p.tiles_m * p.tiles_n;
    if (item >= per * p.experts) return false;
    t.e = item / per;
    tile_coords(item - t.e * per, p.tiles_m, p.tiles_n, tm, tn);
    t.kb0 = seg.offsets[t.e] >> 7;
    t.blocks = max((seg.offsets[t.e + 1] >> 7) - t.kb0, 0);
    t.m0 = tm * 256; t.m_end = p.M;
  }
  t.n0 = tn * BN;
  return true;
}

// A pair's tiles of one product: pair, pair + num_pairs, ...
template <int BN, int GROUPS, bool LONG>
__device__ __forceinline__ void gemm_fp8_tiles(const Params& p, const int pair, const int num_pairs) {
  using C = Cfg<BN>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem_gen = smem_raw + (smem_base - smem_u32(smem_raw));
  const uint32_t epi_base = smem_base + C::kStages * C::kStageBytes;
  const uint32_t sf_base = epi_base + C::kEpiBytes, bar_base = sf_base + C::kSfSlots * C::kSfBytes;
  uint8_t* sf_gen = smem_gen + C::kStages * C::kStageBytes + C::kEpiBytes;
  uint8_t* bar_gen = sf_gen + C::kSfSlots * C::kSfBytes;
  // full: operands of both CTAs landed (leader's)         empty: the stage's MMAs are done (both)
  // sfl: this CTA's scale tiles landed   sfr: they are in tensor memory in both CTAs (leader's)   sfe: the MMAs of their stages are done (both)
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (C::kStages + s); };
  auto sfl_bar = [&](int q) { return bar_base + 8u * (2 * C::kStages + q); };
  auto sfr_bar = [&](int q) { return bar_base + 8u * (2 * C::kStages + C::kSfSlots + q); };
  auto sfe_bar = [&](int q) { return bar_base + 8u * (2 * C::kStages + 2 * C::kSfSlots + q); };
  auto tfull_bar = [&](int a) { return bar_base + 8u * (2 * C::kStages + 3 * C::kSfSlots + a); };
  auto tempty_bar = [&](int a) { return bar_base + 8u * (2 * C::kStages + 3 * C::kSfSlots + C::kAccStages + a); };
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(bar_gen + 8 * C::kNumBarriers);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  int* const offsets = reinterpret_cast<int*>(bar_gen + C::kBarrierBytes);
  int* const firsts = offsets + kMaxExperts + 1;
  const Segments seg = {firsts, offsets};
  const int warp = __shfl_sync(0xFFFFFFFFu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();          // 0 = leader of the pair

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int q = 0; q < C::kSfSlots; ++q) { mbar_init(sfl_bar(q), 1); mbar_init(sfr_bar(q), 8); mbar_init(sfe_bar(q), 1); }
    for (int a = 0; a < C::kAccStages; ++a) { mbar_init(tfull_bar(a), 1); mbar_init(tempty_bar(a), 16); }
    *abort_flag = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
    prefetch_map(&p.a); prefetch_map(&p.b); prefetch_map(&p.sfa); prefetch_map(&p.sfb); prefetch_map(&p.d);
  }
  if (warp == 1) tmem_alloc_pair(smem_u32((const void*)tmem_slot), kTmemCols);
  if constexpr (GROUPS != 0) {
    // the segments' table, by one warp: a running sum of the tiles of 32 segments at a time
    if (warp == 2) {
      if (!p.late) grid_dependency_wait();
      int tiles = 0;
      for (int e0 = 0; e0 <= p.experts; e0 += 32) {
        const int e = e0 + lane;
        // an offset is a multiple of 128 and at most all rows; what is not becomes one, so that no copy leaves the tensors
        auto at = [&](int i) { return min(max(*reinterpret_cast<const volatile int32_t*>(p.offsets + i), 0), p.rows) & ~127; };
        const int begin = e <= p.experts ? at(e) : 0;
        const int end = e < p.experts ? at(e + 1) : begin;
        const int mine = max((end - begin + 255) >> 8, 0) * p.tiles_n;
        int sum = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const int up = __shfl_up_sync(0xFFFFFFFFu, sum, d);
          if (lane >= d) sum += up;
        }
        if (e <= p.experts) { offsets[e] = begin; firsts[e] = tiles + sum - mine; }
        tiles += __shfl_sync(0xFFFFFFFFu, sum, 31);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                               // both CTAs' barriers exist before any remote signal
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  // As in gemm.cu, each role waits for the kernel before this one directly before its first copy or bounded wait; a late product waits
  // at its end.
  auto follow = [&] {
    if (!p.late) grid_dependency_wait();
  };

  if (warp < 8) {
    regs_release<kControlRegs>();
    if (warp == 0) {
      // ------------------------------- operand producer (both CTAs) -------------------------------
      const bool issuer = elect_one();
      int s = 0;
      uint32_t ph = 0;
      bool ok = true, first = true;
      Tile t;
      for (int item = pair; ok && tile_at<BN, GROUPS>(p, seg, item, t); item += num_pairs) {
        const int a_row = t.m0 + (int)rank * 128;
        const int b_row = (GROUPS == 1 ? t.e * p.N : 0) + t.n0 + (int)rank * (BN / 2);
        for (int kb = 0; kb < t.blocks; kb += C::kSub) {
          ok = mbar_wait_issuer(empty_bar(s), ph ^ 1u, abort_flag, 0x41);
          if (!ok) break;
          const uint32_t st = smem_base + s * C::kStageBytes;
          const uint32_t lead_full = map_to_cta(full_bar(s), 0);
          if (first) {
            follow();
            if (!p.late) grid_dependency_trigger();
            first = false;
          }
          if (issuer) {
            const int n = min(C::kSub, t.blocks - kb);
            if (rank == 0) mbar_arrive_expect_tx(full_bar(s), 2u * C::kBlockBytes * n);   // of both CTAs
#pragma unroll
            for (int u = 0; u < C::kSub; ++u) {
              if (u >= n) break;
              tma_load_2d_pair(st + u * C::kBlockBytes, &p.a, lead_full, (t.kb0 + kb + u) * kBK, a_row);
              tma_load_2d_pair(st + u * C::kBlockBytes + C::kABytes, &p.b, lead_full, (t.kb0 + kb + u) * kBK, b_row);
            }
          }
          if (++s == C::kStages) { s = 0; ph ^= 1u; }
        }
      }
      if (!ok && issuer) {                          // give copies in flight a bounded time to land
        const unsigned long long t0 = global_timer_ns();
        while (global_timer_ns() - t0 < 200000ull) {}
      }
    } else if (warp == 2) {
      // ------------------------------- scale producer (both CTAs) -------------------------------
      const bool issuer = elect_one();
      int q = 0;
      uint32_t ph = 0;
      bool ok = true, first = true;
      Tile t;
      for (int item = pair; ok && tile_at<BN, GROUPS>(p, seg, item, t); item += num_pairs) {
        const int a_tile = min((t.m0 >> 7) + (int)rank, p.a_row_tiles - 1) * p.sfa_ktiles;
        int b_tile[C::kSfbTiles];
#pragma unroll
        for (int h = 0; h < C::kSfbTiles; ++h)      // rows past N are never stored
          b_tile[h] = ((GROUPS == 1 ? t.e * p.b_row_tiles : 0) + min((t.n0 >> 7) + h, p.b_row_tiles - 1)) * p.sfb_ktiles;
        for (int kt = t.kb0 >> 2; kt < (t.kb0 + t.blocks + 3) >> 2; ++kt) {
          if (GROUPS == 2 && t.blocks == 0) break;
          ok = mbar_wait_relaxed(sfe_bar(q), ph ^ 1u, abort_flag, 0x48);
          if (!ok) break;
          const uint32_t sf = sf_base + q * C::kSfBytes;
          if (first) { follow(); first = false; }
          if (issuer) {
            mbar_arrive_expect_tx(sfl_bar(q), C::kSfBytes);
            tma_load_2d(sf, &p.sfa, sfl_bar(q), 0, a_tile + kt);
#pragma unroll
            for (int h = 0; h < C::kSfbTiles; ++h) tma_load_2d(sf + 512 + h * 512, &p.sfb, sfl_bar(q), 0, b_tile[h] + kt);
          }
          if (++q == C::kSfSlots) { q = 0; ph ^= 1u; }
        }
      }
      if (!ok && issuer) {
        const unsigned long long t0 = global_timer_ns();
        while (global_timer_ns() - t0 < 200000ull) {}
      }
    } else if (warp == 1) {
      // ------------------------------- MMA issuer (leader CTA only) -------------------------------
      if (rank == 0) {
        const bool issuer = elect_one();
        int s = 0, q = 0, acc = 0;
        uint32_t ph = 0, q_ph = 0, acc_ph = 0;
        bool ok = true, first = true;
        Tile t;
        for (int item = pair; ok && tile_at<BN, GROUPS>(p, seg, item, t); item += num_pairs) {
          if (first) { follow(); first = false; }
          ok = mbar_wait_issuer(tempty_bar(acc), acc_ph ^ 1u, abort_flag, 0x42);
          if (!ok) break;
          const uint32_t sfb_off = BN % 128 ? (uint32_t)(t.n0 & 127) / 32 : 0u;   // first scale column of the tile
          const int part = part_blocks<LONG>(t.blocks, C::kSub);
          int begin = 0;                            // of the part
          for (int kb = 0; kb < t.blocks; kb += C::kSub) {
            if (LONG && kb == begin + part) {
              begin = kb;
              if (issuer) tc_commit_pair(tfull_bar(acc));
              if (++acc == C::kAccStages) { acc = 0; acc_ph ^= 1u; }
              ok = mbar_wait_issuer(tempty_bar(acc), acc_ph ^ 1u, abort_flag, 0x42);
              if (!ok) break;
            }
            const uint32_t d_tmem = tmem_base + acc * BN;
            ok = mbar_wait_issuer(full_bar(s), ph, abort_flag, 0x43);
            if (!ok) break;
            const uint32_t st = smem_base + s * C::kStageBytes;
#pragma unroll
            for (int u = 0; u < C::kSub; ++u) {
              if (kb + u >= t.blocks) break;
              const uint32_t byte = (uint32_t)(t.kb0 + kb + u) & 3u;
              if (kb + u == 0 || byte == 0u) ok = mbar_wait_issuer(sfr_bar(q), q_ph, abort_flag, 0x45);
              if (!ok) break;
              tc_fence_after();
              const uint32_t idesc = instr_desc_mxf8(256, BN, 0) | byte << 4 | byte << 29;
              const uint32_t sfa_t = tmem_base + C::kSfCol + q * 16, sfb_t = sfa_t + 4 + sfb_off;
              const uint64_t adesc = operand_desc(st + u * C::kBlockBytes), bdesc = operand_desc(st + u * C::kBlockBytes + C::kABytes);
              const int n = GROUPS == 2 ? 4 : min(4, p.k_mmas - (kb + u) * 4);
              const bool last_of_slot = byte == 3u || kb + u == t.blocks - 1;
              if (issuer) {
                if (n == 4) {
#pragma unroll
                  for (int j = 0; j < 4; ++j) tc_mma_mxf8_pair(d_tmem, adesc + 2u * j, bdesc + 2u * j, idesc, sfa_t, sfb_t, (kb > begin || u || j) ? 1u : 0u);
                } else {
                  for (int j = 0; j < n; ++j) tc_mma_mxf8_pair(d_tmem, adesc + 2u * j, bdesc + 2u * j, idesc, sfa_t, sfb_t, (kb > begin || u || j) ? 1u : 0u);
                }
                if (last_of_slot) tc_commit_pair(sfe_bar(q));
              }
              if (last_of_slot)
                if (++q == C::kSfSlots) { q = 0; q_ph ^= 1u; }
            }
            if (!ok) break;
            if (issuer) tc_commit_pair(empty_bar(s));   // the stage is free in both CTAs
            if (++s == C::kStages) { s = 0; ph ^= 1u; }
          }
          if (!ok) break;
          if (issuer) tc_commit_pair(tfull_bar(acc));
          if (++acc == C::kAccStages) { acc = 0; acc_ph ^= 1u; }
        }
      }
    } else if (warp >= 4) {
      // ------------------------------- scale movers (both CTAs) -------------------------------
      // Row l of a scale tile (16 bytes) = four 32-row groups x four blocks: that word in lane l of every 32-lane quarter,
      // one column per group.
      const uint32_t lane_field = (uint32_t)((warp & 3) * 32) << 16;
      const uint32_t lead_sfr0 = map_to_cta(sfr_bar(0), 0);
      int q = 0;
      uint32_t ph = 0;
      bool ok = true, first = true;
      Tile t;
      for (int item = pair; ok && tile_at<BN, GROUPS>(p, seg, item, t); item += num_pairs) {
        if (first) { follow(); first = false; }
        for (int kt = t.kb0 >> 2; kt < (t.kb0 + t.blocks + 3) >> 2; ++kt) {
          if (GROUPS == 2 && t.blocks == 0) break;
          // the MMAs that read the slot's columns before are done: its copies were issued behind them
          if (!(ok = warp_acquire(mbar_wait_issuer(sfl_bar(q), ph, abort_flag, 0x46)))) break;
          tc_fence_after();
          const uint8_t* sf = sf_gen + q * C::kSfBytes + lane * 16;
          uint32_t r[16];
#pragma unroll
          for (int j = 0; j < 1 + C::kSfbTiles; ++j) {
            const uint4 v = *reinterpret_cast<const uint4*>(sf + j * 512);
            r[4 * j] = v.x; r[4 * j + 1] = v.y; r[4 * j + 2] = v.z; r[4 * j + 3] = v.w;
          }
#pragma unroll
          for (int j = 4 * (1 + C::kSfbTiles); j < 16; ++j) r[j] = 0u;
          tmem_st16(tmem_base + C::kSfCol + q * 16 + lane_field, r);
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(lead_sfr0 + 8u * q);
          if (++q == C::kSfSlots) { q = 0; ph ^= 1u; }
        }
      }
    }
  } else {
    regs_acquire<kEpilogueRegs>();
    // ------------------------------- epilogue (both CTAs, warps 8-15) -------------------------------
    // Two warps share each 32-lane quarter, every warp moves its half of the columns into registers, hands the accumulator
    // back, and converts, stages and stores it while the next tile's MMAs run.
    const int quarter = warp & 3, half = (warp >> 2) & 1;
    constexpr int kWarpCols = BN / 2, kLoads = kWarpCols / 32;
    const uint32_t buf = epi_base + (warp - 8) * C::kEpiWarpBytes;
    const uint32_t lead_tempty0 = map_to_cta(tempty_bar(0), 0);
    int acc = 0;
    uint32_t acc_ph = 0;
    bool ok = true, first = true;
    Tile t;
    for (int item = pair; ok && tile_at<BN, GROUPS>(p, seg, item, t); item += num_pairs) {
      if (first) { follow(); first = false; }
      auto begin_part = [&] {                        // the address of this warp's share of the finished accumulator
        ok = mbar_wait_warp_spin(tfull_bar(acc), acc_ph, abort_flag, 0x44);
        tc_fence_after();
        return tmem_base + acc * BN + half * kWarpCols + ((uint32_t)(quarter * 32) << 16);
      };
      auto end_part = [&] {                          // accumulator fully read: hand it back to the leader
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(lead_tempty0 + 8u * acc);
        if (++acc == C::kAccStages) { acc = 0; acc_ph ^= 1u; }
      };
      uint32_t t_row = begin_part();
      if (!ok) break;
      uint32_t r[kLoads][32];
#pragma unroll
      for (int l = 0; l < kLoads; ++l) tmem_ld32(t_row + 32 * l, r[l]);
      tmem_ld_wait();
#pragma unroll
      for (int l = 0; l < kLoads; ++l) tmem_ld_pin(r[l]);
      end_part();
      if constexpr (LONG) {
        const int part = part_blocks<LONG>(t.blocks, C::kSub);
        for (int kb = part; kb < t.blocks; kb += part) {
          t_row = begin_part();
          if (!ok) break;
#pragma unroll
          for (int l = 0; l < 2 * kLoads; ++l) {
            uint32_t more[16];
            tmem_ld16(t_row + 16 * l, more);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              uint32_t& sum = r[l / 2][16 * (l & 1) + e];
              sum = __float_as_uint(__uint_as_float(sum) + __uint_as_float(more[e]));
            }
          }
          end_part();
        }
        if (!ok) break;
      }
      if (GROUPS == 2 && t.blocks == 0) {            // an empty segment: nothing was accumulated
#pragma unroll
        for (int l = 0; l < kLoads; ++l)
#pragma unroll
          for (int e = 0; e < 32; ++e) r[l][e] = 0u;
      }
      const int row0 = t.m0 + (int)rank * 128 + quarter * 32, col0 = t.n0 + half * kWarpCols;
      if (row0 >= t.m_end) continue;                 // rows of the next segment, or past the last
      auto store_chunks = [&](auto bf16) {
        constexpr bool BF16_OUT = decltype(bf16)::value;
        constexpr int kChunkCols = BF16_OUT ? 32 : 16;             // accumulator columns per 64 bytes of output row
#pragma unroll
        for (int c = 0; c < kWarpCols; c += kChunkCols) {
          if (col0 + c >= p.N) break;
          uint32_t v[16];
          if constexpr (BF16_OUT) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const uint32_t* x = r[(c + 2 * e) / 32] + (2 * e) % 32;
              const __nv_bfloat162 h2 = __floats2bfloat162_rn(__uint_as_float(x[0]), __uint_as_float(x[1]));
              v[e] = *reinterpret_cast<const uint32_t*>(&h2);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = r[c / 32][c % 32 + e];
          }
          if (p.ragged && col0 + c + kChunkCols > p.N) {
            // a tiled store clips at 16 bytes: where the rows of D end between, the last columns are stored one by one
            const int row = row0 + lane, n = p.N - (col0 + c);
            const int64_t at = ((GROUPS == 2 ? (int64_t)t.e * p.M : 0) + row) * p.ldd + col0 + c;
            if (row < t.m_end && row < p.M) {
#pragma unroll
              for (int e = 0; e < kChunkCols; ++e) {
                if (e >= n) break;
                if constexpr (BF16_OUT) static_cast<uint16_t*>(p.out)[at + e] = (uint16_t)(v[e / 2] >> (16 * (e & 1)));
                else static_cast<uint32_t*>(p.out)[at + e] = v[e];
              }
            }
            break;
          }
          if (lane == 0) tma_store_wait_read<0>();  // the chunk stored before this one has left the buffer
          __syncwarp();
#pragma unroll
          for (int e = 0; e < 4; ++e) {              // row = lane, 16-byte pieces, piece XOR bits 7-8 of the row's offset: the 64-byte swizzle
            const uint32_t dst = buf + lane * 64 + ((e ^ ((lane >> 1) & 3)) << 4);
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(v[4 * e]), "r"(v[4 * e + 1]),
                         "r"(v[4 * e + 2]), "r"(v[4 * e + 3]) : "memory");
          }
          fence_async_smem();
          __syncwarp();
          if (lane == 0) {
            tma_store_3d(&p.d, buf, col0 + c, row0, GROUPS == 2 ? t.e : 0);
            tma_store_commit();
          }
        }
      };
      if (p.d_is_bf16) store_chunks(std::true_type{});
      else store_chunks(std::false_type{});
    }
    if (lane == 0) tma_store_wait_all();
  }

  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                               // the peer's MMAs and loads are done before anyone frees or exits
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem_base, kTmemCols);
  }
  grid_dependency_wait();                           // a pair without a tile, or of a late product, has not waited: "finished" keeps meaning "and all before"
}

template <int BN, int GROUPS, bool LONG>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) gemm_fp8_kernel(const __grid_constant__ Params p) {
  gemm_fp8_tiles<BN, GROUPS, LONG>(p, blockIdx.x >> 1, gridDim.x >> 1);
}
// Two products at once, a pair of CTAs for every tile of either.
struct TwoParams {
  Params p[2];
  int first;                        // pairs of the first
};
template <int BN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) gemm_fp8_two_kernel(const __grid_constant__ TwoParams two) {
  const int pair = blockIdx.x >> 1, second = pair >= two.first;
  gemm_fp8_tiles<BN, 0, false>(two.p[second], second ? pair - two.first : pair, second ? (gridDim.x >> 1) - two.first : two.first);
}

// ------------------------------------------------------------------------------------------------
// Host side
// ------------------------------------------------------------------------------------------------
// Codes [rows, width] with a pitch -> boxes of 128 bytes x box_rows, 128-byte swizzle, zero fill.
bool codes_map(CUtensorMap* map, const uint8_t* base, int64_t rows, int64_t width, int box_rows) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)width, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)fp8_pitch(width)};
  const cuuint32_t box[2] = {kBK, (cuuint32_t)box_rows};
  const cuuint32_t estr[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Scale tiles, one of 512 bytes per row of the map.
bool scales_map(CUtensorMap* map, const uint8_t* base, int64_t tiles) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {128, (cuuint64_t)tiles};
  const cuuint64_t strides[1] = {512};
  const cuuint32_t box[2] = {128, 1};
  const cuuint32_t estr[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, const_cast<uint8_t*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Output [matrices, rows, cols] -> boxes of 32 rows x 64 bytes of one matrix.
bool out_map(CUtensorMap* map, void* base, int64_t matrices, int64_t rows, int64_t cols, int64_t ldd, bool bf16) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const cuuint64_t esz = bf16 ? 2 : 4;
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)matrices};
  const cuuint64_t strides[2] = {(cuuint64_t)ldd * esz, (cuuint64_t)(rows * ldd) * esz};
  const cuuint32_t box[3] = {(cuuint32_t)(64 / esz), 32, 1};
  const cuuint32_t estr[3] = {1, 1, 1};
  return fn(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, base, dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int BN, int GROUPS>
bool fill(Params& p, const Fp8Product& c) {
  const int64_t experts = GROUPS ? c.experts : 1;
  const int64_t b_matrices = GROUPS == 1 ? experts : 1, d_matrices = GROUPS == 2 ? experts : 1;
  p.offsets = c.offsets;
  p.experts = (int)experts;
  p.rows = (int)(GROUPS == 1 ? c.M : c.K);
  p.M = (int)c.M; p.N = (int)c.N;
  p.tiles_m = (int)ceil_div(c.M, 256); p.tiles_n = (int)ceil_div(c.N, BN);
  p.k_blocks = (int)ceil_div(c.K, kBK); p.k_mmas = (int)ceil_div(c.K, 32);
  p.sfa_ktiles = p.sfb_ktiles = (int)ceil_div(fp8_blocks(c.K), 4);
  p.a_row_tiles = (int)ceil_div(c.M, 128); p.b_row_tiles = (int)ceil_div(c.N, 128);
  p.d_is_bf16 = c.d_dtype == NVFP4_BF16; p.late = c.late;
  p.ragged = c.N * (p.d_is_bf16 ? 2 : 4) % 16 != 0; p.out = c.d; p.ldd = c.ldd;
  return codes_map(&p.a, c.a, c.M, c.K, 128) && codes_map(&p.b, c.b, b_matrices * c.N, c.K, BN / 2) &&
         scales_map(&p.sfa, c.a_sf, fp8_sf_tiles(c.M, c.K)) && scales_map(&p.sfb, c.b_sf, b_matrices * fp8_sf_tiles(c.N, c.K)) &&
         out_map(&p.d, c.d, d_matrices, c.M, c.N, c.ldd, p.d_is_bf16 != 0);
}

template <int BN, int GROUPS, bool LONG>
int launch(const Fp8Product& c, cudaStream_t s) {
  using C = Cfg<BN>;
  Params p;
  if (!fill<BN, GROUPS>(p, c)) return NVFP4_ERR_CUDA;
  // GROUPS 1: a segment's last tile may be half empty
  const int64_t tiles = GROUPS == 1 ? (ceil_div(c.M, 256) + c.experts) * p.tiles_n : (GROUPS == 2 ? c.experts : 1) * p.tiles_m * (int64_t)p.tiles_n;
  const int64_t pairs = std::min<int64_t>(tiles, sm_count() / 2);
  static DeviceFlags smem_set;                         // per instantiation, per device
  if (set_max_dynamic_smem(smem_set, gemm_fp8_kernel<BN, GROUPS, LONG>, C::kSmemBytes) != cudaSuccess) return NVFP4_ERR_CUDA;
  return launch_overlapped(gemm_fp8_kernel<BN, GROUPS, LONG>, (unsigned)(2 * pairs), kThreads, C::kSmemBytes, s, p) == cudaSuccess ? NVFP4_OK
                                                                                                                            : NVFP4_ERR_CUDA;
}

template <int BN>
int launch_two(const Fp8Product& a, const Fp8Product& b, cudaStream_t s) {
  using C = Cfg<BN>;
  TwoParams two;
  if (!fill<BN, 0>(two.p[0], a) || !fill<BN, 0>(two.p[1], b)) return NVFP4_ERR_CUDA;
  two.first = two.p[0].tiles_m * two.p[0].tiles_n;
  const int pairs = two.first + two.p[1].tiles_m * two.p[1].tiles_n;
  static DeviceFlags smem_set;
  if (set_max_dynamic_smem(smem_set, gemm_fp8_two_kernel<BN>, C::kSmemBytes) != cudaSuccess) return NVFP4_ERR_CUDA;
  return launch_overlapped(gemm_fp8_two_kernel<BN>, (unsigned)(2 * pairs), kThreads, C::kSmemBytes, s, two) == cudaSuccess ? NVFP4_OK : NVFP4_ERR_CUDA;
}

template <int BN, int GROUPS>
int launch(const Fp8Product& c, cudaStream_t s) {
  return fp8_blocks(c.K) > kMostBlocks ? launch<BN, GROUPS, true>(c, s) : launch<BN, GROUPS, false>(c, s);
}

template <int GROUPS>
int launch_width(int width, const Fp8Product& c, cudaStream_t s) {
  return width == 128 ? launch<128, GROUPS>(c, s) : width == 192 ? launch<192, GROUPS>(c, s) : launch<256, GROUPS>(c, s);
}

// Columns of a tile: the width whose waves of pairs take the least, a tile of 192 columns taking 0.83 and one of 128 0.68 of one of 256
// (which alone has no second accumulator).  us, 256 / 192 columns: 2077 x 2840 x 1064 14.3 / 13.0, 2077 x 1064 x 2840 12.8 / 11.1, 8192 x 1064
// x 712 16.4 / 14.7; with more waves 4096 x 2816 x 1024 16.2 / 16.9, 16384 x 4096 x 4096 197 / 219.  256 / 128: 1024 x 1024 x 1024 7.2 / 5.4,
// 512 x 4096 x 11008 30.8 / 24.5; with two waves instead of one 2077 x 1064 x 2840 12.7 / 14.0.
int tile_width(int64_t tiles_m, int64_t N) {
  const int64_t pairs = sm_count() / 2;
  auto cost = [&](int64_t width, int64_t per_tile) { return ceil_div(tiles_m * ceil_div(N, width), pairs) * per_tile; };
  const int64_t wide = cost(256, 100), middle = cost(192, 83), narrow = cost(128, 68);
  return wide <= middle && wide <= narrow ? 256 : middle <= narrow ? 192 : 128;
}

}  // namespace

// Rows of A (of a segment, on average) up to which the product goes to gemm_fp8_few.cu: those that it takes at one time.  us, there / here:
// 128 rows 11008 x 4096 13.7 / 15.9, 4096 x 11008 14.9 / 23.4, 4096 x 4096 10.3 / 11.3, 2816 x 1024 5.1 / 5.0; 64 experts of 2816 x 1024 with 8
// rows each 34.5 / 47.6, with 128 each 43.3 / 48.6, 4 with 128 each 7.0 / 8.8.  The host knows the average alone: the same 8192 rows all in one
// segment take 40.9 / 22.0, in eight 41.0 / 22.7.
constexpr int64_t kFewRows = 128;

int gemm_fp8(const Fp8Product& p, cudaStream_t s) {
  if (!p.experts && p.M <= kFewRows) return gemm_fp8_few(p, s);
  if (p.by_rows && p.counts && p.slots <= kFewRows * p.experts) return gemm_fp8_few(p, s);
  const int groups = p.experts == 0 ? 0 : p.by_rows ? 1 : 2;
  // rows of tiles; a segment's last tile is half empty on average
  const int64_t tiles_m = groups == 0 ? ceil_div(p.M, 256) : groups == 2 ? p.experts * ceil_div(p.M, 256)
                                                                      : ceil_div(p.slots ? std::min(p.slots, p.M) : p.M, 256) + p.experts / 2;
  const int width = tile_width(tiles_m, p.N);
  switch (groups) {
    case 0: return launch_width<0>(width, p, s);
    case 1: return launch_width<1>(width, p, s);
    default: return launch_width<2>(width, p, s);
  }
}

// The second depends on nothing of the first.  Where every tile of both has a pair of its own they take one launch; otherwise the second begins
// where multiprocessors are done with the first.  A step of a layer in a graph, us, two launches / one: M 256, N and K 512 (tiles of 128
// columns) 15.6 / 13.9; 777 x 720 x 1160 22.6 / 22.7; 700 x 704 x 2048 (192) 26.5 / 23.0; 1024 x 1024 x 2048 (256) 28.1 / 24.2.
int gemm_fp8_two(const Fp8Product& a, const Fp8Product& b, cudaStream_t s) {
  auto tiles = [](const Fp8Product& c, int64_t width) { return ceil_div(c.M, 256) * ceil_div(c.N, width); };
  if (!a.experts && !b.experts && std::min(a.M, b.M) > kFewRows && std::max(fp8_blocks(a.K), fp8_blocks(b.K)) <= kMostBlocks) {
    for (int width : {128, 192, 256})
      if (tiles(a, width) + tiles(b, width) <= sm_count() / 2) return width == 128 ? launch_two<128>(a, b, s) : width == 192 ? launch_two<192>(a, b, s) : launch_two<256>(a, b, s);
  }
  if (int st = gemm_fp8(a, s)) return st;
  Fp8Product late = b;
  late.late = true;
  return gemm_fp8(late, s);
}

int fp8_error_word(unsigned int* out) {
  unsigned int w = 0, zero = 0;
  if (cudaMemcpyFromSymbol(&w, g_error_word, sizeof(w)) != cudaSuccess) return NVFP4_ERR_CUDA;
  if (w != 0 && cudaMemcpyToSymbol(g_error_word, &zero, sizeof(zero)) != cudaSuccess) return NVFP4_ERR_CUDA;
  *out = w;
  return NVFP4_OK;
}

}  // namespace nvfp4

using namespace nvfp4;

namespace {
constexpr int64_t kMost = (1ll << 31) - 512;
// The checks that the products share; N: columns of D, which limit its rows' pitch.
int check_product(const void* a, const void* a_sf, const void* b, const void* b_sf, const void* d, int64_t M, int64_t N, int64_t K,
                  int d_dtype, int64_t ldd) {
  if (!a || !a_sf || !b || !b_sf || !d) return NVFP4_ERR_NULL;
  if (d_dtype != NVFP4_BF16 && d_dtype != NVFP4_FP32) return NVFP4_ERR_ENUM;
  if (M <= 0 || N <= 0 || K <= 0 || ldd < N || M > kMost || N > kMost || K > kMost) return NVFP4_ERR_SHAPE;
  if (ceil_div(M, 128) * ceil_div(N, 128) > kMost || fp8_sf_tiles(M, K) > kMost || fp8_sf_tiles(N, K) > kMost) return NVFP4_ERR_SHAPE;
  if (!aligned16(a) || !aligned16(a_sf) || !aligned16(b) || !aligned16(b_sf) || !aligned16(d) ||
      (ldd * (d_dtype == NVFP4_BF16 ? 2 : 4)) % 16 != 0)
    return NVFP4_ERR_ALIGN;
  return NVFP4_OK;
}
int check_experts(int64_t experts, const void* offsets, int64_t N, int64_t K) {
  if (!offsets) return NVFP4_ERR_NULL;
  if (experts <= 0 || experts > kMaxExperts) return NVFP4_ERR_SHAPE;
  if (N > 0 && K > 0 && (experts * N > kMost || experts * fp8_sf_tiles(N, K) > kMost)) return NVFP4_ERR_SHAPE;
  return (reinterpret_cast<uintptr_t>(offsets) & 3u) ? NVFP4_ERR_ALIGN : NVFP4_OK;
}
}  // namespace

extern "C" int nvfp4_gemm_fp8(const uint8_t* a_codes, const uint8_t* a_sf, const uint8_t* b_codes, const uint8_t* b_sf,
                              int64_t M, int64_t N, int64_t K, void* d, int d_dtype, int64_t ldd, void* cuda_stream) {
  if (int st = check_product(a_codes, a_sf, b_codes, b_sf, d, M, N, K, d_dtype, ldd)) return st;
  if (int st = check_arch()) return st;
  return gemm_fp8({a_codes, a_sf, b_codes, b_sf, M, N, K, d, d_dtype, ldd}, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" int nvfp4_gemm_fp8_experts(const uint8_t* a_codes, const uint8_t* a_sf, const uint8_t* b_codes, const uint8_t* b_sf,
                                      int64_t tokens, int64_t topk, int64_t experts, const int32_t* counts, const int32_t* offsets,
                                      int64_t N, int64_t K, void* d, int d_dtype, int64_t ldd, void* cuda_stream) {
  const int64_t rows = nvfp4_expert_rows(tokens, topk, experts);
  if (int st = check_product(a_codes, a_sf, b_codes, b_sf, d, rows, N, K, d_dtype, ldd)) return st;
  if (int st = check_experts(experts, offsets, N, K)) return st;
  if (reinterpret_cast<uintptr_t>(counts) & 3u) return NVFP4_ERR_ALIGN;
  if ((ceil_div(rows, 256) + experts) * ceil_div(N, 128) > kMost) return NVFP4_ERR_SHAPE;
  if (int st = check_arch()) return st;
  return gemm_fp8({a_codes, a_sf, b_codes, b_sf, rows, N, K, d, d_dtype, ldd, experts, offsets, true, counts, tokens * topk},
                  static_cast<cudaStream_t>(cuda_stream));
}

extern "C" int nvfp4_gemm_fp8_experts_dw(const uint8_t* a_codes, const uint8_t* a_sf, const uint8_t* b_codes, const uint8_t* b_sf,
                                         int64_t tokens, int64_t topk, int64_t experts, const int32_t* offsets, int64_t N, int64_t K,
                                         void* d, int d_dtype, void* cuda_stream) {
  const int64_t rows = nvfp4_expert_rows(tokens, topk, experts);
  if (int st = check_product(a_codes, a_sf, b_codes, b_sf, d, N, K, rows, d_dtype, K)) return st;
  if (int st = check_experts(experts, offsets, N, K)) return st;
  if (experts * ceil_div(N, 256) * ceil_div(K, 128) > kMost) return NVFP4_ERR_SHAPE;
  if (int st = check_arch()) return st;
  return gemm_fp8({a_codes, a_sf, b_codes, b_sf, N, K, rows, d, d_dtype, K, experts, offsets, false}, static_cast<cudaStream_t>(cuda_stream));
}
