// Products of FP8 operands (fp8.cuh) with few rows of A: tokens on weights that are kept, and experts with few tokens each.
//
// Its floor is the bytes of B, each read once.  gemm_fp8.cu's tiles would leave most multiprocessors idle (a CTA pair takes 256 columns of
// D) and fill half of their rings with rows that do not exist.  Here the operands change places: 128 rows of B (weights) are the
// instruction's 128 rows, up to 128 rows of A (tokens), in steps of 16, its columns, so that nearly all of a k-stage of 128 values is
// weights, of which a block keeps 160-190 KB in flight.  tcgen05.mma.cta_group::1.kind::mxf8f6f4, scales through
// registers into tensor memory, a tile for four stages; a lane of the accumulator is a column of D, so that a warp stores 32 of a row at a
// time.  us, weights that are in no cache (floor: their bytes at the rate of a copy): 11008 x 4096 (7.0) 1 row 12.0, 67 rows 13.0, 128 rows
// 13.7; 4096 x 11008 (7.0) 11.6, 13.3, 14.9; 4096 x 4096 (2.6) 6.8, 8.9, 10.3.  With gemm_fp8.cu's kernel 15-16, 23, 11; with dot products by
// mma.sync, 16 rows of B a block, 11.0, 15.2 and 7.3 for up to 8 rows, and twice that for 16.  3-4 us are a launch and the first and
// last latencies.  The rest is the chain of a block's stages: an instruction of 128 rows takes about 115 cycles however few its columns, four of
// them 0.25 us, and 11008 columns are 86 tiles, so that 86 of 148 multiprocessors go through 32 stages one after the other (8 us; two blocks
// for a tile would be 172).  Pairs of CTAs, whose instructions of 256 rows take 40 to 64 cycles, gain nothing in all (11.8) and lose where
// clusters of eight blocks do not all find room (4096 x 11008 19.8).
//
// One product: with few tiles of B a cluster of 2, 4 or 8 blocks shares one along the contraction axis; each then sums a share of
// the tokens over all blocks' accumulators, which they write into one another's shared memory, in the order of the blocks.
// Segments (experts): the blocks go over the tiles of all segments with rows, one tile at a time.
// A block whose contraction is longer than kMostBlocks stages sums it in equal parts: the epilogue adds up the accumulators in columns
// of tensor memory of their own, which takes no more registers.  us, one accumulator for all of it / in parts: 1 x 9600 x 28672 66.6 / 68.8,
// 128 rows 71.8 / 75.6, 64 x 8192 x 28672 (two parts) 43.1 / 43.5.
#include <cuda.h>
#include <cuda_bf16.h>

#include <algorithm>

#include "bounded_waits.cuh"
#include "fp8.cuh"
#include "tc_ptx.cuh"
#include "tensor_map.cuh"

namespace nvfp4 {
namespace {

constexpr int kThreads = 384;                       // warps: 0 operands, 1 issuer, 2 table of segments and scales, 4-7 scale movers, 8-11 epilogue
constexpr int kBK = 128;                            // values, and bytes of a row, per k-stage
constexpr int kMaxTokens = 128;
constexpr int kWBytes = 128 * kBK;
constexpr int kSfBytes = 2 * 512;                   // a scale tile of B's rows and one of A's
constexpr int kMaxStages = 12;
constexpr int kSfSlots = 4;                         // scale tiles of four stages each
constexpr int kRingBytes = 200 * 1024;
template <bool LONG>
constexpr uint32_t kTmemCols = LONG ? 512 : 256;
constexpr uint32_t kSfCol = 128;                    // accumulators: columns 0-127; then 8 columns of scales per slot
constexpr uint32_t kSumCol = 256;                   // LONG: sums of the parts so far, 128 columns
constexpr int kTableBytes = 3 * (int)(kMaxExperts + 1) * 4 + 4;
constexpr int kBarrierBytes = 512;
constexpr int kSmemBytes = 1024 /*align*/ + kRingBytes + kSfSlots * kSfBytes + kBarrierBytes + kTableBytes;
static_assert(kSmemBytes <= 232448, "shared memory overflow");
static_assert(kSfCol + 8 * kSfSlots <= kTmemCols<false> && kTmemCols<false> <= kSumCol && kSumCol + kMaxTokens <= kTmemCols<true>, "tensor memory overflow");
static_assert(8 * (2 * kMaxStages + 3 * kSfSlots + 4) + 8 <= kBarrierBytes, "barrier area overflow");
static_assert(kMaxTokens * 128 * 4 <= kRingBytes, "the ring holds a share of all blocks' accumulators");

struct Params {
  CUtensorMap w, x, sfw, sfx;
  const int32_t *offsets, *counts;  // of the segments; null: one product
  void* d;
  int64_t ldd;
  int M, N;                         // rows of A in all, columns of D
  int experts, tiles;               // tiles of 128 columns of D
  int slots;                        // rows of all segments together, padding aside, at most
  int k_stages, k_mmas, k_tiles;
  int w_row_tiles;                  // scale row tiles of one matrix of B
  int tokens, box;                  // a stage holds `tokens` rows of A (a multiple of 16), fetched `box` at a time
  int stages;
  int split;                        // blocks of a cluster
  int d_is_bf16, late;
};
struct Item {
  int row, rows, n0, e;             // rows of A [row, row + rows), first column of D, matrix of B
};
struct Table {
  int *firsts, *rows, *counts;
};

__device__ __forceinline__ bool item_at(const Params& p, const Table& tab, int i, Item& t) {
  if (!p.offsets) {
    if (i >= p.tiles) return false;
    t = {0, p.M, i * 128, 0};
    return true;
  }
  if (i >= tab.firsts[p.experts]) return false;
  int lo = 0, hi = p.experts;                       // the last segment that begins at or before the item
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (tab.firsts[mid] <= i) lo = mid; else hi = mid;
  }
  const int groups = (tab.counts[lo] + kMaxTokens - 1) / kMaxTokens, local = i - tab.firsts[lo], tile = local / groups, m = (local - tile * groups) * kMaxTokens;
  t = {tab.rows[lo] + m, min(tab.counts[lo] - m, kMaxTokens), tile * 128, lo};
  return true;
}

__device__ __forceinline__ void tc_mma_mxf8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa_tmem,
                                            uint32_t sfb_tmem, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\t"
               "setp.ne.b32 p, %4, 0;\n\t"
               "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
               ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(sfa_tmem), "r"(sfb_tmem)
               : "memory");
}
// A box on its way into the level-two cache, whatever is written to it until it is loaded.
__device__ __forceinline__ void prefetch_2d(const CUtensorMap* map, int x, int y) {
  asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global [%0, {%1, %2}];" ::"l"(map), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
// 32 columns of an accumulator, plus those of the parts before it where there are any.
template <bool LONG>
__device__ __forceinline__ void load_sums(uint32_t acc, uint32_t sums, bool more, uint32_t (&r)[32]) {
  tmem_ld32(acc, r);
  tmem_ld_wait();
  tmem_ld_pin(r);
  if (LONG && more) {
    uint32_t s[32];
    tmem_ld32(sums, s);
    tmem_ld_wait();
    tmem_ld_pin(s);
#pragma unroll
    for (int c = 0; c < 32; ++c) r[c] = __float_as_uint(__uint_as_float(r[c]) + __uint_as_float(s[c]));
  }
}
__device__ __forceinline__ void store_as(__nv_bfloat16* d, float v) { *d = __float2bfloat16_rn(v); }
__device__ __forceinline__ void store_as(float* d, float v) { *d = v; }
// Up to 32 values of a column of D, one below the other.
template <typename D>
__device__ __forceinline__ void store_column(D* d, int64_t ldd, const uint32_t (&r)[32], int n) {
#pragma unroll
  for (int c = 0; c < 32; ++c) {
    if (c < n) store_as(d, __uint_as_float(r[c]));
    d += ldd;
  }
}

// LONG: a block's contraction may be longer than kMostBlocks.  The choice takes 2-3 % of the others' time (1 x 11008 x 4096 13.3 -> 13.6 us).
template <bool LONG>
__global__ void __launch_bounds__(kThreads, 1) gemm_fp8_few_kernel(const __grid_constant__ Params p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem_gen = smem_raw + (smem_base - smem_u32(smem_raw));
  const uint32_t sf_base = smem_base + kRingBytes, bar_base = sf_base + kSfSlots * kSfBytes;
  uint8_t* bar_gen = smem_gen + kRingBytes + kSfSlots * kSfBytes;
  // full: operands landed   empty: the stage's MMAs are done
  // sfl: scale tiles landed   sfr: they are in tensor memory   sfe: the MMAs of their (up to) four stages are done
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (kMaxStages + s); };
  auto sfl_bar = [&](int q) { return bar_base + 8u * (2 * kMaxStages + q); };
  auto sfr_bar = [&](int q) { return bar_base + 8u * (2 * kMaxStages + kSfSlots + q); };
  auto sfe_bar = [&](int q) { return bar_base + 8u * (2 * kMaxStages + 2 * kSfSlots + q); };
  auto tfull_bar = [&](int a) { return bar_base + 8u * (2 * kMaxStages + 3 * kSfSlots + a); };
  auto tempty_bar = [&](int a) { return bar_base + 8u * (2 * kMaxStages + 3 * kSfSlots + 2 + a); };
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(bar_gen + 8 * (2 * kMaxStages + 3 * kSfSlots + 4));
  volatile uint32_t* abort_flag = tmem_slot + 1;
  int* const table = reinterpret_cast<int*>(bar_gen + kBarrierBytes);
  const Table tab = {table, table + kMaxExperts + 1, table + 2 * (kMaxExperts + 1)};
  const int warp = __shfl_sync(0xFFFFFFFFu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const int x_bytes = p.tokens * kBK, stage_bytes = kWBytes + x_bytes;
  const int acc_stages = p.tokens <= 64 ? 2 : 1;
  // the blocks of a cluster share the k-stages of an item
  const int rank = p.split > 1 ? (int)cluster_ctarank() : 0;
  const int first_item = blockIdx.x / p.split, items_step = gridDim.x / p.split;
  const int ks0 = p.k_stages * rank / p.split, ks1 = p.k_stages * (rank + 1) / p.split;
  // an accumulator takes a part of the block's contraction at a time
  int part = ks1 - ks0, parts = 1;
  if constexpr (LONG) {
    parts = (part + kMostBlocks - 1) / kMostBlocks;
    part = (part + parts - 1) / parts;
    parts = (ks1 - ks0 + part - 1) / part;          // fewer where there are very many
  }

  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int q = 0; q < kSfSlots; ++q) { mbar_init(sfl_bar(q), 1); mbar_init(sfr_bar(q), 4); mbar_init(sfe_bar(q), 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(tfull_bar(a), 1); mbar_init(tempty_bar(a), 4); }
    *abort_flag = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
    prefetch_map(&p.w); prefetch_map(&p.x); prefetch_map(&p.sfw); prefetch_map(&p.sfx);
  }
  if (warp == 1) tmem_alloc(smem_u32((const void*)tmem_slot), kTmemCols<LONG>);
  if (warp == 2 && p.offsets) {
    // the segments' table: a running sum of the items of 32 segments at a time; what is no plan is cut to the rows that there are
    if (!p.late) grid_dependency_wait();
    int items = 0;
    for (int e0 = 0; e0 <= p.experts; e0 += 32) {
      const int e = e0 + lane;
      const int row = e < p.experts ? min(max(reinterpret_cast<const volatile int32_t*>(p.offsets)[e], 0), p.M) & ~127 : 0;
      const int count = e < p.experts ? min(max(reinterpret_cast<const volatile int32_t*>(p.counts)[e], 0), min(p.M - row, p.slots)) : 0;
      const int mine = (count + kMaxTokens - 1) / kMaxTokens * p.tiles;
      int sum = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int up = __shfl_up_sync(0xFFFFFFFFu, sum, d);
        if (lane >= d) sum += up;
      }
      if (e <= p.experts) { tab.firsts[e] = items + sum - mine; tab.rows[e] = row; tab.counts[e] = count; }
      items += __shfl_sync(0xFFFFFFFFu, sum, 31);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  auto follow = [&] {                               // a late product waits at its end
    if (!p.late) grid_dependency_wait();
  };

  if (warp == 0) {
    // ------------------------------- operand producer -------------------------------
    const bool issuer = elect_one();
    int s = 0;
    uint32_t ph = 0;
    bool ok = true, first = true;
    Item t;
    // One product knows its first weights before the kernel ahead is done, the quantizer of its rows as a rule: into the level-two cache,
    // which that kernel's writes go through as well, they may come early (both calls, 11008 x 4096 and one row: 15.5 -> 15.2 us).
    if (!p.offsets && issuer && item_at(p, tab, first_item, t))
      for (int ks = ks0; ks < min(ks1, ks0 + p.stages); ++ks) prefetch_2d(&p.w, ks * kBK, t.n0);
    for (int i = first_item; ok && item_at(p, tab, i, t); i += items_step) {
      const int w_row = t.e * p.N + t.n0;
      const int boxes = (t.rows + p.box - 1) / p.box;
      const uint32_t bytes = kWBytes + boxes * p.box * kBK;
      for (int ks = ks0; ks < ks1; ++ks) {
        ok = mbar_wait_issuer(empty_bar(s), ph ^ 1u, abort_flag, 0x61);
        if (!ok) break;
        const uint32_t st = smem_base + s * stage_bytes;
        if (first) {
          follow();
          if (!p.late) grid_dependency_trigger();
          first = false;
        }
        if (issuer) {
          mbar_arrive_expect_tx(full_bar(s), bytes);
          tma_load_2d(st, &p.w, full_bar(s), ks * kBK, w_row);
          for (int b = 0; b < boxes; ++b) tma_load_2d(st + kWBytes + b * p.box * kBK, &p.x, full_bar(s), ks * kBK, t.row + b * p.box);
        }
        if (++s == p.stages) { s = 0; ph ^= 1u; }
      }
    }
    if (!ok && issuer) {                            // give copies in flight a bounded time to land
      const unsigned long long t0 = global_timer_ns();
      while (global_timer_ns() - t0 < 200000ull) {}
    }
  } else if (warp == 2) {
    // ------------------------------- scale producer -------------------------------
    const bool issuer = elect_one();
    int q = 0;
    uint32_t ph = 0;
    bool ok = true, first = true;
    Item t;
    for (int i = first_item; ok && item_at(p, tab, i, t); i += items_step) {
      const int sfw_row = (t.e * p.w_row_tiles + (t.n0 >> 7)) * p.k_tiles, sfx_row = (t.row >> 7) * p.k_tiles;
      for (int kt = ks0 >> 2; kt <= (ks1 - 1) >> 2; ++kt) {
        ok = mbar_wait_relaxed(sfe_bar(q), ph ^ 1u, abort_flag, 0x68);
        if (!ok) break;
        if (first) { follow(); first = false; }
        if (issuer) {
          mbar_arrive_expect_tx(sfl_bar(q), kSfBytes);
          tma_load_2d(sf_base + q * kSfBytes, &p.sfw, sfl_bar(q), 0, sfw_row + kt);
          tma_load_2d(sf_base + q * kSfBytes + 512, &p.sfx, sfl_bar(q), 0, sfx_row + kt);
        }
        if (++q == kSfSlots) { q = 0; ph ^= 1u; }
      }
    }
    if (!ok && issuer) {
      const unsigned long long t0 = global_timer_ns();
      while (global_timer_ns() - t0 < 200000ull) {}
    }
  } else if (warp == 1) {
    // ------------------------------- MMA issuer -------------------------------
    const bool issuer = elect_one();
    int s = 0, q = 0, acc = 0;
    uint32_t ph = 0, q_ph = 0, acc_ph = 0;
    bool ok = true, first = true;
    Item t;
    for (int i = first_item; ok && item_at(p, tab, i, t); i += items_step) {
      if (first) { follow(); first = false; }
      ok = mbar_wait_issuer(tempty_bar(acc), acc_ph ^ 1u, abort_flag, 0x62);
      if (!ok) break;
      uint32_t d_tmem = tmem_base + acc * 64;
      const uint32_t idesc0 = instr_desc_mxf8(128, (t.rows + 15) & ~15, 0);
      int begin = ks0;                              // of the part
      for (int ks = ks0; ks < ks1; ++ks) {
        if (LONG && ks == begin + part) {
          begin = ks;
          if (issuer) tc_commit(tfull_bar(acc));
          if (++acc == acc_stages) { acc = 0; acc_ph ^= 1u; }
          ok = mbar_wait_issuer(tempty_bar(acc), acc_ph ^ 1u, abort_flag, 0x62);
          if (!ok) break;
          d_tmem = tmem_base + acc * 64;
        }
        if (ks == ks0 || !(ks & 3)) ok = mbar_wait_issuer(sfr_bar(q), q_ph, abort_flag, 0x65);
        ok = ok && mbar_wait_issuer(full_bar(s), ph, abort_flag, 0x63);
        if (!ok) break;
        tc_fence_after();
        const uint32_t st = smem_base + s * stage_bytes;
        const uint32_t byte = (uint32_t)ks & 3u, idesc = idesc0 | byte << 4 | byte << 29;
        const uint32_t sfw_t = tmem_base + kSfCol + q * 8, sfx_t = sfw_t + 4;
        const uint64_t wdesc = operand_desc(st), xdesc = operand_desc(st + kWBytes);
        const int n = min(4, p.k_mmas - ks * 4);
        if (issuer) {
          for (int j = 0; j < n; ++j) tc_mma_mxf8(d_tmem, wdesc + 2u * j, xdesc + 2u * j, idesc, sfw_t, sfx_t, (ks > begin || j) ? 1u : 0u);
          tc_commit(empty_bar(s));
          if ((ks & 3) == 3 || ks == ks1 - 1) tc_commit(sfe_bar(q));
        }
        if ((ks & 3) == 3 || ks == ks1 - 1)
          if (++q == kSfSlots) { q = 0; q_ph ^= 1u; }
        if (++s == p.stages) { s = 0; ph ^= 1u; }
      }
      if (!ok) break;
      if (issuer) tc_commit(tfull_bar(acc));
      if (++acc == acc_stages) { acc = 0; acc_ph ^= 1u; }
    }
  } else if (warp >= 4 && warp < 8) {
    // ------------------------------- scale movers -------------------------------
    // Row l of a scale tile (16 bytes) = four 32-row groups x four blocks: that word in lane l of every 32-lane quarter, one column per group.
    const uint32_t lane_field = (uint32_t)((warp & 3) * 32) << 16;
    int q = 0;
    uint32_t ph = 0;
    bool ok = true, first = true;
    Item t;
    for (int i = first_item; ok && item_at(p, tab, i, t); i += items_step) {
      if (first) { follow(); first = false; }
      for (int kt = ks0 >> 2; kt <= (ks1 - 1) >> 2; ++kt) {
        // the MMAs that read the slot's columns before are done: its copies were issued behind them
        if (!(ok = warp_acquire(mbar_wait_issuer(sfl_bar(q), ph, abort_flag, 0x66)))) break;
        tc_fence_after();
        const uint8_t* sf = smem_gen + kRingBytes + q * kSfBytes + lane * 16;
        const uint4 a = *reinterpret_cast<const uint4*>(sf), b = *reinterpret_cast<const uint4*>(sf + 512);
        const uint32_t r[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        tmem_st8(tmem_base + kSfCol + q * 8 + lane_field, r);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(sfr_bar(q));
        if (++q == kSfSlots) { q = 0; ph ^= 1u; }
      }
    }
  } else if (warp >= 8) {
    // ------------------------------- epilogue -------------------------------
    const int quarter = warp & 3;
    int acc = 0;
    uint32_t acc_ph = 0;
    bool ok = true, first = true;
    Item t;
    for (int i = first_item; ok && item_at(p, tab, i, t); i += items_step) {
      if (first) { follow(); first = false; }
      const uint32_t sum_row = tmem_base + kSumCol + ((uint32_t)(quarter * 32) << 16);
      for (int n = 1; LONG && n < parts; ++n) {     // all parts but the last go into the sums
        ok = mbar_wait_warp_spin(tfull_bar(acc), acc_ph, abort_flag, 0x64);
        if (!ok) break;
        tc_fence_after();
        const uint32_t t_row = tmem_base + acc * 64 + ((uint32_t)(quarter * 32) << 16);
        for (int c0 = 0; c0 < t.rows; c0 += 32) {
          uint32_t r[32];
          load_sums<LONG>(t_row + c0, sum_row + c0, n > 1, r);
          tmem_st16(sum_row + c0, *reinterpret_cast<const uint32_t(*)[16]>(r));
          tmem_st16(sum_row + c0 + 16, *reinterpret_cast<const uint32_t(*)[16]>(r + 16));
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(tempty_bar(acc));
        if (++acc == acc_stages) { acc = 0; acc_ph ^= 1u; }
      }
      ok = ok && mbar_wait_warp_spin(tfull_bar(acc), acc_ph, abort_flag, 0x64);
      if (!ok || p.split > 1) break;                // one item: the sums over the cluster follow below
      tc_fence_after();
      const uint32_t t_row = tmem_base + acc * 64 + ((uint32_t)(quarter * 32) << 16);
      const int n = t.n0 + quarter * 32 + lane;
      for (int c0 = 0; c0 < t.rows; c0 += 32) {
        uint32_t r[32];
        load_sums<LONG>(t_row + c0, sum_row + c0, parts > 1, r);
        if (c0 + 32 >= t.rows) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(tempty_bar(acc));   // accumulator read: the next item's MMAs may begin
        }
        if (n < p.N) {
          const int64_t at = (int64_t)(t.row + c0) * p.ldd + n;
          if (p.d_is_bf16) store_column(static_cast<__nv_bfloat16*>(p.d) + at, p.ldd, r, t.rows - c0);
          else store_column(static_cast<float*>(p.d) + at, p.ldd, r, t.rows - c0);
        }
      }
      if (++acc == acc_stages) { acc = 0; acc_ph ^= 1u; }
    }
  }

  __syncwarp();
  if (p.split > 1) {
    // One item per cluster.  Its blocks are done with their rings when all have come here: block q then gets columns
    // [q * share, (q + 1) * share) of everyone's accumulator, adds them up and stores them.
    tc_fence_before();
    cluster_sync_all();
    tc_fence_after();
    // (in steps of eight, so that a lane's eight stores go to one block: a block and an address for every column cost 75 cycles each)
    const int share = ((p.M + 7) / 8 + p.split - 1) / p.split * 8, tile = first_item;
    if (warp >= 8) {
      const uint32_t quarter_row = tmem_base + ((uint32_t)((warp & 3) * 32) << 16);
      const uint32_t t_row = quarter_row + (LONG ? (parts - 1) % acc_stages * 64 : 0), sum_row = quarter_row + kSumCol;
      const uint32_t mine = smem_base + (uint32_t)(rank * share * 128 + (warp & 3) * 32 + lane) * 4u;
      for (int c0 = 0; c0 < p.M; c0 += 32) {
        uint32_t r[32];
        load_sums<LONG>(t_row + c0, sum_row + c0, parts > 1, r);
#pragma unroll
        for (int c = 0; c < 32; c += 8) {
          if (c0 + c >= p.M) break;
          const int owner = (c0 + c) / share;
          const uint32_t at = map_to_cta(mine + (uint32_t)(c0 + c - owner * share) * 512u, owner);
#pragma unroll
          for (int e = 0; e < 8; ++e) asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(at + 512u * e), "r"(r[c + e]) : "memory");
        }
      }
    }
    tc_fence_before();
    cluster_sync_all();
    tc_fence_after();
    const float* const parts = reinterpret_cast<const float*>(smem_gen);
    const int c1 = min(share, p.M - rank * share);
    const bool fine = !*abort_flag;
#pragma unroll 4
    for (int i = threadIdx.x; i < (fine ? c1 * 128 : 0); i += kThreads) {
      const int c = i >> 7, n = tile * 128 + (i & 127);
      float v = parts[i] + parts[share * 128 + i];
#pragma unroll
      for (int q = 2; q < 8; ++q)
        if (q < p.split) v += parts[q * share * 128 + i];
      if (n >= p.N) continue;
      const int64_t at = (int64_t)(rank * share + c) * p.ldd + n;
      if (p.d_is_bf16) store_as(static_cast<__nv_bfloat16*>(p.d) + at, v);
      else store_as(static_cast<float*>(p.d) + at, v);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, kTmemCols<LONG>);
  }
  grid_dependency_wait();                           // a block without an item has not waited: "finished" keeps meaning "and all before"
}

// ------------------------------------------------------------------------------------------------
// Host side
// ------------------------------------------------------------------------------------------------
bool byte_map(CUtensorMap* map, const uint8_t* base, int64_t rows, int64_t width, int64_t pitch, int box_width, int box_rows, bool swizzled) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)width, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)pitch};
  const cuuint32_t box[2] = {(cuuint32_t)box_width, (cuuint32_t)box_rows};
  const cuuint32_t estr[2] = {1, 1};
  return fn(map, swizzled ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, const_cast<uint8_t*>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, swizzled ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool LONG>
int launch(const Params& p, int64_t blocks, cudaStream_t s) {
  static DeviceFlags smem_set;                      // per instantiation, per device
  if (set_max_dynamic_smem(smem_set, gemm_fp8_few_kernel<LONG>, kSmemBytes) != cudaSuccess) return NVFP4_ERR_CUDA;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = p.split; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = kSmemBytes; cfg.stream = s;
  cfg.attrs = attr; cfg.numAttrs = p.split > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, gemm_fp8_few_kernel<LONG>, p) == cudaSuccess ? NVFP4_OK : NVFP4_ERR_CUDA;
}

}  // namespace

int gemm_fp8_few(const Fp8Product& c, cudaStream_t s) {
  Params p;
  const int64_t experts = c.experts ? c.experts : 1;
  p.offsets = c.experts ? c.offsets : nullptr; p.counts = c.counts;
  p.d = c.d; p.ldd = c.ldd; p.d_is_bf16 = c.d_dtype == NVFP4_BF16; p.late = c.late;
  p.M = (int)c.M; p.N = (int)c.N; p.experts = (int)experts;
  p.tiles = (int)ceil_div(c.N, 128);
  p.slots = (int)c.slots;
  p.k_stages = (int)ceil_div(c.K, kBK); p.k_mmas = (int)ceil_div(c.K, 32); p.k_tiles = (int)ceil_div(fp8_blocks(c.K), 4);
  p.w_row_tiles = (int)ceil_div(c.N, 128);
  // one product: a stage has room for just its rows; segments: for any number, fetched 16 at a time
  const int64_t most = c.experts ? std::min<int64_t>(c.slots, kMaxTokens) : c.M;
  p.tokens = (int)ceil_div(most, 16) * 16;
  p.box = c.experts ? 16 : p.tokens;
  p.stages = std::min(kMaxStages, kRingBytes / (kWBytes + p.tokens * kBK));
  if (!byte_map(&p.w, c.b, experts * c.N, c.K, fp8_pitch(c.K), kBK, 128, true) || !byte_map(&p.x, c.a, c.M, c.K, fp8_pitch(c.K), kBK, p.box, true) ||
      !byte_map(&p.sfw, c.b_sf, experts * fp8_sf_tiles(c.N, c.K), 128, 512, 128, 1, false) ||
      !byte_map(&p.sfx, c.a_sf, fp8_sf_tiles(c.M, c.K), 128, 512, 128, 1, false))
    return NVFP4_ERR_CUDA;
  p.split = 1;
  int64_t blocks;
  if (c.experts) {
    blocks = std::min<int64_t>((c.slots / kMaxTokens + std::min(c.slots, experts)) * p.tiles, sm_count());
  } else {
    // As many blocks as there are multiprocessors for them, each with four k-stages or more.  A stage takes 0.25 us, so that sharing
    // saves that much for every stage less; the exchange costs 0.3 us and 0.018 for every row (us, one block / shared: 2816 x 1024, 1 row
    // 4.2 / 3.8, 128 rows 5.1 / 7.5; 1024 x 2816, 128 rows, two / four blocks 11.1 / 7.6).
    while (p.split < 8 && (int64_t)p.tiles * p.split * 2 <= sm_count() && p.k_stages >= 8 * p.split) p.split *= 2;
    if ((p.k_stages - p.k_stages / p.split) * 14 <= 16 + p.M) p.split = 1;
    blocks = p.split > 1 ? (int64_t)p.tiles * p.split : std::min<int64_t>(p.tiles, sm_count());
  }
  return ceil_div(p.k_stages, p.split) > kMostBlocks ? launch<true>(p, blocks, s) : launch<false>(p, blocks, s);
}

int fp8_few_error_word(unsigned int* out) {
  unsigned int w = 0, zero = 0;
  if (cudaMemcpyFromSymbol(&w, g_error_word, sizeof(w)) != cudaSuccess) return NVFP4_ERR_CUDA;
  if (w != 0 && cudaMemcpyToSymbol(g_error_word, &zero, sizeof(zero)) != cudaSuccess) return NVFP4_ERR_CUDA;
  *out = w;
  return NVFP4_OK;
}

}  // namespace nvfp4
