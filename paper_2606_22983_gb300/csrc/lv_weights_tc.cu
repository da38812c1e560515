// Attention weights added up for the cached tokens, on the fifth-generation tensor cores (lv_weights.cuh has
// how the work is cut).
#include <climits>

#include "lv_tc.cuh"
#include "lv_weights.cuh"

namespace lv {

namespace {

// Roles of a CTA's twenty warps.
constexpr int kSumWarps = 16;             // a warpgroup for each buffer of scores and half of a unit's keys
constexpr int kWarpK = 16, kWarpQ = 17, kWarpMma = 18, kWarpUnits = 19;
constexpr int kThreads = 640;
constexpr int kHalf = 128, kUnitKeys = 2 * kHalf;
constexpr int kCols = 128;                // rows of the step (packed) a product has as columns
constexpr int kIndexThreads = 64;
constexpr int kUnits = 8;                 // found ahead at most,
constexpr int kAhead = 5;                 // where no more products than this are left to be issued
constexpr long long kUnitWaits = 64;      // a wait for a unit, in those for copies: millions of rows may come before it
constexpr float kLog2e = 1.44269504088896341f;

template <int DP>
struct WShape {
  static constexpr int kBlocks = DP / 64;                  // 128-byte wide column blocks
  static constexpr int kTile = kHalf * DP * 2;             // bytes of half a unit's K, and of a tile of queries
  static constexpr int kKStages = DP == 128 ? 4 : 6;
  static constexpr int kQStages = DP == 128 ? 2 : 4;
  static constexpr int kQ = kKStages * kTile;
  static constexpr int kMisc = kQ + kQStages * kTile;
};

struct WBars {
  uint64_t k_full[8], k_empty[8], q_full[4], q_empty[4];
  uint64_t s_full[2][2], s_empty[2][2];    // a buffer of scores, a half
  // Sums of a unit's second buffer.  part_full by turns: threads that leave their sums go on without a wait for the
  // others that do, and may take the next ones before those have come; one barrier for both would look full to them.
  uint64_t part_full[2], part_empty;
  uint64_t unit_full[kUnits], unit_empty[kUnits];
  uint64_t drain;
  uint32_t tmem;
  volatile int bad;
};

struct Misc {
  WBars bars;
  alignas(16) float b[kSumWarps][kCols];      // the rows' terms, a copy a warp, read by 16 bytes
  float part[kUnitKeys];
  volatile int issued;            // tiles of queries
  Unit units[kUnits];
  int pieces[kUnits];             // find_unit's
  SegmentIndex<kIndexThreads> index;
};
static_assert(WShape<128>::kMisc % 16 == 0 && WShape<64>::kMisc % 16 == 0, "its place in shared memory");
static_assert(WShape<128>::kMisc + sizeof(Misc) <= 227 * 1024, "shared memory of a CTA");
static_assert(WShape<64>::kMisc + sizeof(Misc) <= 227 * 1024, "shared memory of a CTA");

// The n lowest bits, all of them from 32 on, none below 1.
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }
__device__ __forceinline__ int clamp_col(int x) { return min(max(x, 0), kCols); }

// A unit's products: its packed rows [begin, end) in tiles of `step`.
struct Chunks {
  int begin, end, step, count, halves;
  __device__ __forceinline__ Chunks(const WeightArgs& a, const Unit& u, int step_)
      : begin(u.t0 * a.G), end(u.t1 * a.G), step(step_), count(u.products), halves(u.g.keys - u.key0 > kHalf ? 2 : 1) {}
  __device__ __forceinline__ int rows(int i) const { return min(step, end - begin - i * step); }
};

// w[j] += sum_r 2^(c q_r.k_j + b_r), b_r = -lse_r log2(e): S = K Q^T with a unit's keys as the product's rows, 128
// and 128 of them, and the step's rows as its columns, so that a thread has a key, adds up its row of S
// as it reads it from TMEM, and writes one word at the end.  No maximum is needed, as the sums are known, and no V.
//
// What bounds it: few rows, the bytes of K: 61 single tokens over 2 to 16 k keys, 0.42 GB in 80 us, 5.3 TB/s.  Many
// rows, products and sums that wait for one another, a product of 256 keys and 128 rows some 2100 cycles (the tensor
// pipe active 49 % of them, issue 53 %, shared memory by the tensor core 46 % and by threads 41 %): 4 prompts of 4096, 32
// query heads of 128, 270 us, 1.02 PFLOP/s.  These have 8 heads a KV head.  Groups that do not divide 128 have fewer rows a
// product (7 heads: 126) and take the columns one by one under a mask in all of them, not beside the diagonal alone: 4
// prompts with 28 query heads 292 us, where an eighth less work than 32 is asked.  Terms read for a key of each half at once (a thread 64 columns of both)
// took a tenth more, as a half's scores then wait for the other's.
//
// kCut: units may come in pieces, some of a unit's rows each, whose sums k_weights_join adds up.  (A kernel of its own
// for steps without: finding their units took 4 us more of 58 otherwise.)
// One CTA an SM; units are taken in order from a counter, long ones (the first keys of a context, which
// all rows see) first.
//   warp 19  finds units ahead
//   warp 16  K of a unit's first half into a ring of shared memory, by TMA: a box a page and 64 columns
//   warp 17  K of its second half, and queries into a ring of their own
//   warp 18  products into two buffers of TMEM for each half
//   0 .. 15  the rows' terms, exponentials and sums, a thread a key in every second product
template <int DP, bool kBf16, bool kCut>
__global__ void __launch_bounds__(kThreads, 1)
k_weights_tc(const __grid_constant__ WeightArgs a, const __grid_constant__ CUtensorMap kmap,
             const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap q_few, int box_rows, int few_rows,
             int q_tma) {
  using S = WShape<DP>;
  extern __shared__ __align__(1024) unsigned char dyn[];
  Misc& m = *reinterpret_cast<Misc*>(dyn + S::kMisc);
  WBars& bars = m.bars;
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const uint32_t k_s = smem_u32(dyn), q_s = k_s + S::kQ;
  if (k_s & 1023u) {      // (the swizzle's pattern starts at multiples of 1024 bytes)
    if (threadIdx.x == 0) report(a.ctl, LV_ERR_CUDA, blockIdx.x);
    return;
  }
  if (threadIdx.x == 0) {
    const uint32_t copies = a.hold == LV_HOLD_COPIES ? 1u + (blockIdx.x & 1u) : 1u;
    const uint32_t products = a.hold == LV_HOLD_PRODUCTS ? 1u + (blockIdx.x & 1u) : 1u;
    for (int i = 0; i < S::kKStages; ++i) {
      bar_init(&bars.k_full[i], copies);
      bar_init(&bars.k_empty[i], 1);
    }
    for (int i = 0; i < S::kQStages; ++i) {
      bar_init(&bars.q_full[i], 1);
      bar_init(&bars.q_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      for (int h = 0; h < 2; ++h) {
        bar_init(&bars.s_full[i][h], products);
        bar_init(&bars.s_empty[i][h], 4);
      }
    }
    for (int i = 0; i < 2; ++i) bar_init(&bars.part_full[i], kSumWarps / 2);
    bar_init(&bars.part_empty, kSumWarps / 2);
    for (int i = 0; i < kUnits; ++i) {
      bar_init(&bars.unit_full[i], 1);
      bar_init(&bars.unit_empty[i], kSumWarps + 3);
    }
    bar_init(&bars.drain, 1);
    bars.bad = 0;
    m.issued = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (wid == kWarpMma) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&bars.tmem))
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bars.tmem;
  dep_wait();

  const StepHead step = load_words(a.head);
  const bool fits = weights_fit(a, step);
  if (!fits && blockIdx.x == 0 && threadIdx.x == 0) report(a.ctl, LV_ERR_STATE, -1);
  const int n = step.requests & (kSharedStep - 1);
  // (the sessions' words are in what the copies fill later)
  const int step_rows = product_rows(a.G);
  const int units =
      fits ? index_segments<kIndexThreads, kUnitKeys, kCut>(a, step, m.index, reinterpret_cast<int*>(dyn), step_rows) : 0;
  fence_async();
  __syncthreads();

  // the units of the CTA in order, for a role: false at the end or where a wait ran out
  int unit_at = 0;
  uint32_t unit_par = 0;
  bool ok = true;
  Unit u;
  int piece = -1;
  auto next_unit = [&]() -> bool {
    if (!(ok = bar_wait(&bars, &bars.unit_full[unit_at], unit_par, kUnitWaits * a.wait_ns))) return false;
    u = m.units[unit_at];
    if constexpr (kCut) piece = m.pieces[unit_at];
    warp_arrive(&bars.unit_empty[unit_at]);
    if (++unit_at == kUnits) {
      unit_at = 0;
      unit_par ^= 1;
    }
    return u.t0 < u.t1;
  };

  // K of a half of each unit, for a warp: lane i finds the page of box i of its keys; one thread then issues the
  // copies.  (Half the 64 boxes of a unit of 16-token pages took 1200 cycles to issue, by one warp all of them 2400,
  // which is nearly what their bytes take.)
  struct KHalf {
    int of, slot, page, off;      // which half; tiles of K before it
  } k_half{0, 0, -1, 0};
  const int boxes = kHalf / box_rows;
  auto find = [&](KHalf& x) {
    const int key = u.key0 + kHalf * x.of + lane * box_rows;
    const int32_t* table = u.g.req < 0 ? a.pool_table + (size_t)u.g.sid * a.maxB : a.tables + (size_t)u.g.req * a.maxB;
    const int b = a.t_shift >= 0 ? key >> a.t_shift : key / a.T;
    x.off = key - b * a.T;
    x.page = lane < boxes && key < u.g.keys ? table[b] : -1;
  };
  auto load = [&](KHalf& x, const Unit& v, int page, int off) -> bool {
    const int halves = v.g.keys - v.key0 > kHalf ? 2 : 1;
    if (x.of < halves) {
      const int at = x.slot + x.of, stage = at % S::kKStages;
      if (!bar_wait(&bars, &bars.k_empty[stage], ~(at / S::kKStages) & 1u, a.wait_ns)) return false;
      if ((uint32_t)page >= a.hbm_pages) page = (int)a.hbm_pages;      // none: outside the array, zeros
      uint64_t* full = &bars.k_full[stage];
      const uint32_t dst = k_s + stage * S::kTile;
      if (elected()) bar_expect(full, S::kTile);
#pragma unroll 1
      for (int i = 0; i < boxes; i += 4) {
        int pg[4], of[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          pg[e] = __shfl_sync(0xffffffffu, page, (i + e) & 31);
          of[e] = __shfl_sync(0xffffffffu, off, (i + e) & 31);
        }
        if (elected()) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (i + e >= boxes) break;
#pragma unroll
            for (int y = 0; y < S::kBlocks; ++y)
              tma_box(dst + y * kHalf * 128 + (i + e) * box_rows * 128, &kmap, 64 * y, v.head, of[e], pg[e], full);
          }
        }
        __syncwarp();
      }
    }
    x.slot += halves;
    return true;
  };
  // after a wait that ran out: what is on its way lands before the shared memory is given up
  auto drain = [&](const KHalf& x) {
    for (int i = max(0, x.slot - S::kKStages); i < x.slot; ++i) {
      const unsigned long long t0 = now_ns();
      while (!bar_try(&bars.k_full[i % S::kKStages], (uint32_t)(i / S::kKStages) & 1u))
        if ((long long)(now_ns() - t0) > a.wait_ns) break;
    }
  };

  if (wid < kSumWarps) {
    const int buf = wid >> 3, half = wid >> 2 & 1, row = threadIdx.x & 127;
    // this warp's 32 lanes of its buffer and half in TMEM
    const uint32_t s_at = tmem + ((uint32_t)(wid & 3) << 21) + kCols * (2 * buf + half);
    const float2 c2 = make_float2(a.scale, a.scale);
    uint32_t s_par = 0, parts = 0;      // parts: units whose sums were joined
    int turn = 0;           // the buffer of the next product
    const int Hq = a.H * a.G;
    float* const b = m.b[wid];
    int in_col[kCols / 32];      // where the sums of this lane's columns lie, from a product's first
#pragma unroll
    for (int k = 0; k < kCols / 32; ++k) {
      const int c = 32 * k + lane, token = c / a.G;
      in_col[k] = token * Hq + c - token * a.G;
    }
    const int step_words = a.G > kCols ? 0 : kCols / a.G * Hq;      // and the next product's
    // the sums of four columns' rows, asked for a product ahead
    float z[kCols / 32];
    bool asked = false;      // for the unit to come
    auto ask = [&](const Unit& v, const Chunks& c_of, int i) {
      const int rows = i < c_of.count ? c_of.rows(i) : 0;
      const float* const lse = a.lse + (int64_t)(v.g.qrow + v.t0) * Hq + v.head * a.G;
      const float* at = lse + (int64_t)i * step_words;
      const bool odd = a.G > kCols || (v.g.req < 0 && a.last > 0);
#pragma unroll
      for (int k = 0; k < kCols / 32; ++k) {
        z[k] = -INFINITY;
        const int c = 32 * k + lane;
        if (c >= rows) continue;
        if (odd) {      // (a product need not begin at a token's first head; rows that do not count)
          const int R = c_of.begin + i * c_of.step + c, token = R / a.G;
          if (counts(a, v.g, n, token)) z[k] = lse[(int64_t)(token - v.t0) * Hq + (R - token * a.G)];
        } else {
          z[k] = at[in_col[k]];
        }
      }
    };
    while (ok && next_unit()) {
      const Chunks ch(a, u, step_rows);
      const int key = u.key0 + kHalf * half + row;
      const bool there = half < ch.halves, mine = key < u.g.keys;
      // the threads of the unit's last product write; those of the other buffer, which have the products before
      // it and every second one from there, leave theirs
      const int next_turn = turn ^ (ch.count & 1);
      const bool joins = ch.count > 1, writes = buf != next_turn;
      // (a piece's sums are added to the weights by k_weights_join)
      const bool whole = !kCut || piece < 0;
      float* w = whole ? a.w + u.g.sid * a.w_session + u.head * a.w_head + key : a.pieces + (int64_t)piece * kUnitKeys + kHalf * half + row;
      // the packed rows that see the key: from its own position on, to the window's end
      const bool all_see = u.g.req < 0, no_end = all_see || a.window == 0 || key < a.sinks, check_b = all_see && a.last > 0;
      auto row_of = [&](long long token) { return (int)(token < 0 ? 0 : token > u.g.tokens ? u.g.tokens : token) * a.G; };
      const int from = all_see ? 0 : row_of((long long)key - u.g.first);
      // a product whose rows lie between these all see all keys of the half
      const int key_lo = u.key0 + kHalf * half, key_hi = key_lo + kHalf - 1;
      const int open_lo = all_see ? 0 : row_of((long long)key_hi - u.g.first);
      const int open_hi = all_see || a.window == 0 || key_hi < a.sinks ? INT_MAX : row_of((long long)key_lo - u.g.first + a.window);
      LongSum all;
      if (!asked && there) ask(u, ch, turn ^ buf);
      asked = false;
      for (int i = turn ^ buf; i < ch.count; i += 2) {
        if (there) {
#pragma unroll
          for (int k = 0; k < kCols / 32; ++k) b[32 * k + lane] = z[k] == -INFINITY ? z[k] : -z[k] * kLog2e;
          __syncwarp();
          if (i + 2 < ch.count) {
            ask(u, ch, i + 2);
          } else if (__all_sync(0xffffffffu, bar_try(&bars.unit_full[unit_at], unit_par))) {
            // the next unit's first ones, where it is known: they would be waited for at its begin
            const Unit v = m.units[unit_at];
            const Chunks next(a, v, step_rows);
            asked = v.t0 < v.t1 && half < next.halves;
            if (asked) ask(v, next, turn ^ (ch.count & 1) ^ buf);
          }
          if (!(ok = bar_wait(&bars, &bars.s_full[buf][half], s_par, a.wait_ns))) break;
          s_par ^= 1;
          tc_fence_after();
          const int R0 = ch.begin + i * ch.step, rows = ch.rows(i);
          float2 acc0 = make_float2(0.f, 0.f), acc1 = acc0;
          if (rows == kCols && R0 >= open_lo && R0 <= open_hi - kCols && !check_b) {
            // (keys past the end have sums of whatever the page holds, which nobody takes)
#pragma unroll 1
            for (int c0 = 0; c0 < kCols; c0 += 32) {
              uint32_t x[32];
              tc_ld32(x, s_at + c0);
              tc_wait_ld();
              tc_loaded<32>(x);
              const float* s = reinterpret_cast<const float*>(x);
#pragma unroll
              for (int j = 0; j < 32; j += 4) {
                const float4 bb = *reinterpret_cast<const float4*>(b + c0 + j);
                float2 y0 = fma2(make_float2(s[j], s[j + 1]), c2, make_float2(bb.x, bb.y));
                float2 y1 = fma2(make_float2(s[j + 2], s[j + 3]), c2, make_float2(bb.z, bb.w));
                y0.x = exp2_fast(y0.x);
                y0.y = exp2_fast(y0.y);
                y1.x = exp2_fast(y1.x);
                y1.y = exp2_fast(y1.y);
                acc0 = add2(acc0, y0);
                acc1 = add2(acc1, y1);
              }
            }
          } else {
            const int c_lo = clamp_col(from - R0);
            const int c_hi = !mine ? 0 : no_end ? rows
                             : min(rows, clamp_col(row_of((long long)key - u.g.first + a.window) - R0));
#pragma unroll 1
            for (int c0 = 0; c0 < rows; c0 += 32) {
              uint32_t seen = low_bits(c_hi - c0) & ~low_bits(c_lo - c0);
              if (check_b) seen &= __ballot_sync(0xffffffffu, b[c0 + lane] != -INFINITY);
              if (!__any_sync(0xffffffffu, seen != 0)) continue;
              uint32_t x[32];
              tc_ld32(x, s_at + c0);
              tc_wait_ld();
              tc_loaded<32>(x);
              const float* s = reinterpret_cast<const float*>(x);
#pragma unroll
              for (int j = 0; j < 32; j += 2) {
                const float2 bb = *reinterpret_cast<const float2*>(b + c0 + j);
                float2 y = fma2(make_float2(s[j], s[j + 1]), c2, bb);
                y.x = exp2_fast(seen >> j & 1u ? y.x : -INFINITY);
                y.y = exp2_fast(seen >> (j + 1) & 1u ? y.y : -INFINITY);
                acc0 = add2(acc0, y);
              }
            }
          }
          tc_fence_before();
          warp_arrive(&bars.s_empty[buf][half]);
          acc0 = add2(acc0, acc1);
          all.add(acc0.x + acc0.y);
        }
      }
      turn = next_turn;
      if (!ok) break;
      float sum = all.sum;
      if (joins) {
        float* part = m.part + kHalf * half + row;
        if (!writes) {
          if (!(ok = bar_wait(&bars, &bars.part_empty, ~parts & 1u, a.wait_ns))) break;
          *part = sum;
          warp_arrive(&bars.part_full[parts & 1]);
        } else {
          if (!(ok = bar_wait(&bars, &bars.part_full[parts & 1], parts >> 1 & 1u, a.wait_ns))) break;
          sum += *part;      // (the same whichever of the two is whose)
          warp_arrive(&bars.part_empty);
        }
        ++parts;
      }
      // (one addition to the word in this call; nothing waits for it)
      if (!whole && writes && mine) __stcg(w, sum);
      else if (writes && mine && sum != 0.f) asm volatile("red.global.add.f32 [%0], %1;" ::"l"(w), "f"(sum) : "memory");
    }
    tc_fence_before();
  } else if (wid == kWarpK) {
    k_half.of = 0;
    bool more = next_unit();
    if (more) find(k_half);
    while (more) {
      const Unit now = u;
      // (the next unit's pages are looked up before this one's copies may wait)
      const int page = k_half.page, off = k_half.off;
      if (!(ok = load(k_half, now, page, off))) break;
      more = next_unit();
      if (more) find(k_half);
    }
    if (LV_RARE(bars.bad)) drain(k_half);
  } else if (wid == kWarpQ) {
    int stage = 0, issued = 0;
    uint32_t par = 0;
    long long tiles = 0;
    k_half.of = 1;
    while (ok && next_unit()) {
      const Chunks ch(a, u, step_rows);
      find(k_half);
      if (!(ok = load(k_half, u, k_half.page, k_half.off))) break;
      for (int i = 0; ok && i < ch.count; ++i) {
        const int R0 = ch.begin + i * ch.step, rows = ch.rows(i);
        if (!(ok = bar_wait(&bars, &bars.q_empty[stage], ~par & 1u, a.wait_ns))) break;
        const uint32_t dst = q_s + stage * S::kTile;
        uint64_t* full = &bars.q_full[stage];
        if (q_tma) {
          const bool few = rows <= few_rows * a.G;
          if (elected()) {
            bar_expect(full, (few ? few_rows * a.G : ch.step) * 128 * S::kBlocks);
#pragma unroll
            for (int x = 0; x < S::kBlocks; ++x)
              tma_box(dst + x * kHalf * 128, few ? &q_few : &qmap, 64 * x, 0, u.head, u.g.qrow + R0 / a.G, full);
          }
          __syncwarp();
          ++tiles;
        } else {
          // lane i finds rows i, 32 + i, ...; a step copies kStep rows, kChunks lanes a row
          constexpr int kChunks = DP / 8, kStep = 32 / kChunks;
          const int c = lane % kChunks, sub = lane / kChunks;
          const bool col = c * 8 < a.D;
          for (int r0 = 0; r0 < rows; r0 += 32) {
            const int R = R0 + min(r0 + lane, rows - 1), token = R / a.G;
            const int64_t at = (u.g.qrow + token) * a.q_row + (int64_t)(u.head * a.G + (R - token * a.G)) * a.q_head;
#pragma unroll 4
            for (int k = 0; k < 32 / kStep; ++k) {
              const int r = r0 + kStep * k + sub;
              const uint16_t* src =
                  reinterpret_cast<const uint16_t*>(a.q) + __shfl_sync(0xffffffffu, at, kStep * k + sub) + c * 8;
              uint32_t w[4] = {0, 0, 0, 0};
              if (col) {
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = (uint32_t)src[2 * e] | (uint32_t)src[2 * e + 1] << 16;
              }
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + (c / 8) * (kHalf * 128) + r * 128 +
                                                                           (((c % 8) ^ (r & 7)) << 4)),
                           "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3])
                           : "memory");
            }
          }
          fence_async();
          __syncwarp();
          if (elected()) bar_arrive(full);
          __syncwarp();
        }
        ++issued;
        if (lane == 0) m.issued = issued;
        if (++stage == S::kQStages) {
          stage = 0;
          par ^= 1;
        }
      }
    }
    if (LV_RARE(bars.bad)) drain(k_half);
    if (LV_RARE(bars.bad) && q_tma) {
      for (long long i = tiles < S::kQStages ? 0 : tiles - S::kQStages; i < tiles; ++i) {
        const unsigned long long t0 = now_ns();
        while (!bar_try(&bars.q_full[i % S::kQStages], (uint32_t)(i / S::kQStages) & 1u))
          if ((long long)(now_ns() - t0) > a.wait_ns) break;
      }
    }
  } else if (wid == kWarpMma) {
    // by one thread (a warp that votes at each wait took some 200 cycles for it, four times a product)
    if (elected()) {
      const uint32_t kd0 = desc_low(k_s, 16), qd0 = desc_low(q_s, 16);
      int ks = 0, qs = 0, buf = 0;
      uint32_t k_par = 0, q_par = 0, s_par = 0;      // s_par: a bit for (buffer, half)
      auto products = [&]() -> bool {
        for (;;) {
          if (!bar_wait1(&bars, &bars.unit_full[unit_at], unit_par, kUnitWaits * a.wait_ns)) return false;
          u = m.units[unit_at];
          bar_arrive(&bars.unit_empty[unit_at]);
          if (++unit_at == kUnits) {
            unit_at = 0;
            unit_par ^= 1;
          }
          if (u.t0 >= u.t1) return true;
          const Chunks ch(a, u, step_rows);
          int at[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            at[h] = ks;
            if (h >= ch.halves) break;
            if (!bar_wait1(&bars, &bars.k_full[ks], k_par, a.wait_ns)) return false;
            if (++ks == S::kKStages) {
              ks = 0;
              k_par ^= 1;
            }
          }
          // a product's barriers are asked while the products before it are still being issued: the answers of
          // three asked one after the other as each is needed took as long as half a product
          bool q_in = bar_try(&bars.q_full[qs], q_par);
          bool s_out[2];
          auto ask = [&](int bf) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
              s_out[h] = h >= ch.halves || bar_try(&bars.s_empty[bf][h], ~(s_par >> (2 * bf + h)) & 1u);
          };
          ask(buf);
#pragma unroll 1
          for (int i = 0; i < ch.count; ++i) {
            const int cols = (ch.rows(i) + 15) & ~15;
            const uint32_t desc = mma_desc<kBf16>(kHalf, cols, false), qd = qd0 + qs * (S::kTile >> 4);
            const int q_now = qs;
            if (LV_RARE(!q_in) && !bar_wait_slow(&bars, &bars.q_full[qs], q_par, a.wait_ns)) return false;
            if (++qs == S::kQStages) {
              qs = 0;
              q_par ^= 1;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              if (h >= ch.halves) break;
              if (LV_RARE(!s_out[h]) &&
                  !bar_wait_slow(&bars, &bars.s_empty[buf][h], ~(s_par >> (2 * buf + h)) & 1u, a.wait_ns))
                return false;
              s_par ^= 1u << (2 * buf + h);
              tc_fence_after();
              const uint32_t kd = kd0 + at[h] * (S::kTile >> 4);
#pragma unroll
              for (int k = 0; k < DP / 16; ++k) {
                const uint32_t o = ((k / 4) * (kHalf * 128) + (k % 4) * 32) >> 4;
                tc_mma_ss(tmem + kCols * (2 * buf + h), kd + o, qd + o, desc, k > 0);
              }
              tc_commit(&bars.s_full[buf][h]);
              if (i + 1 == ch.count) tc_commit(&bars.k_empty[at[h]]);
              if (h + 1 == ch.halves) tc_commit(&bars.q_empty[q_now]);
              if (h == 0 && i + 1 < ch.count) q_in = bar_try(&bars.q_full[qs], q_par);
            }
            buf ^= 1;
            if (i + 1 < ch.count) ask(buf);
          }
        }
      };
      if (!products()) {      // let the products under way end
        tc_commit(&bars.drain);
        const unsigned long long t0 = now_ns();
        while (!bar_try(&bars.drain, 0))
          if ((long long)(now_ns() - t0) > a.wait_ns) break;
      }
    }
    __syncwarp();
  } else {
    // Units are taken when few products of those before are left to be issued: a CTA that held long ones ahead
    // would end last.  Short ones come four at a time until few are left, a lane finding each, as a
    // ticket and its unit take some two microseconds and the copies of one 1.4.
    int at = 0;
    uint32_t par = 0;
    int handed = 0;
    const bool brief = (long long)m.index.most * a.G <= 2 * kCols;
    int taken = 0;
    for (bool end = false; !end;) {
      while (handed - m.issued > kAhead && !bars.bad) __nanosleep(100);
      const int batch = brief && units - taken > 8 * (int)gridDim.x ? 4 : 1;
      int t = 0;
      if (lane == 0) t = atomicAdd(&a.tickets[0], batch);
      taken = __shfl_sync(0xffffffffu, t, 0);
      t = taken + lane;
      Unit x{};
      int of = -1;
      if (lane < batch && t < units) x = find_unit<kIndexThreads, kUnitKeys, kCut>(a, step, m.index, t, step_rows, of);
      end = taken + batch > units || units == 0;
      const int products = x.t0 < x.t1 ? ((x.t1 - x.t0) * a.G + step_rows - 1) / step_rows : 0;
      x.products = products;
      for (int j = 0; j <= batch; ++j) {      // (the last: the end, where it is)
        const bool marker = j == batch;
        const int some = marker ? (int)end : __shfl_sync(0xffffffffu, products, j & 31);
        if (!some) continue;
        if (!(ok = bar_wait(&bars, &bars.unit_empty[at], ~par & 1u, a.wait_ns))) break;
        if (lane == (marker ? 0 : j)) {
          m.units[at] = marker ? Unit{} : x;
          if constexpr (kCut) m.pieces[at] = of;
        }
        warp_arrive(&bars.unit_full[at]);
        handed += marker ? 0 : some;
        if (++at == kUnits) {
          at = 0;
          par ^= 1;
        }
      }
      if (!ok || bars.bad) break;
    }
    // the last CTA that has taken its last unit sets the counters back
    if (lane == 0) {
      __threadfence();
      if (atomicAdd(&a.tickets[1], 1) == (int)gridDim.x - 1) {
        a.tickets[0] = 0;
        a.tickets[1] = 0;
      }
    }
    __syncwarp();
  }
  __syncthreads();
  if (threadIdx.x == 0 && LV_RARE(bars.bad)) {
    report(a.ctl, LV_ERR_TIMEOUT, blockIdx.x);
    a.head_out->kind = -1;
  }
  if (wid == kWarpMma) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

template <int DP, bool kBf16>
cudaError_t run(const WeightArgs& a, const WeightMaps& m, int ctas, cudaStream_t s) {
  static const CUtensorMap none{};
  return launch_dependent(a.cut_units ? k_weights_tc<DP, kBf16, true> : k_weights_tc<DP, kBf16, false>, dim3(ctas), kThreads, WShape<DP>::kMisc + sizeof(Misc), s, a, *m.k,
                          m.q ? *m.q : none, m.q_few ? *m.q_few : none, m.box_rows, m.few_rows, m.q ? 1 : 0);
}

template <int DP>
cudaError_t set() {
  for (auto k : {k_weights_tc<DP, true, true>, k_weights_tc<DP, true, false>, k_weights_tc<DP, false, true>,
                 k_weights_tc<DP, false, false>}) {
    const cudaError_t e =
        cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, WShape<DP>::kMisc + (int)sizeof(Misc));
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

// w[j] += the sums of a cut unit's pieces, in their order: a CTA a unit, a thread a key.
__global__ void __launch_bounds__(kUnitKeys) k_weights_join(const __grid_constant__ WeightArgs a) {
  dep_wait();
  const StepHead step = load_words(a.head);
  if (!weights_fit(a, step) || (int)blockIdx.x >= *a.cut_count) return;
  const CutUnit c = load_words(&a.cuts[blockIdx.x]);
  if ((int)threadIdx.x >= c.keys) return;
  const float* x = a.pieces + (int64_t)c.piece0 * kUnitKeys + threadIdx.x;
  LongSum sum;
#pragma unroll 4
  for (int i = 0; i < c.pieces; ++i) sum.add(__ldcg(x + (int64_t)i * kUnitKeys));
  if (sum.sum != 0.f) c.w[threadIdx.x] += sum.sum;
}

}  // namespace

cudaError_t configure_weights_tc() {
  const cudaError_t e = set<64>();
  return e != cudaSuccess ? e : set<128>();
}

cudaError_t launch_weights_tc(const WeightArgs& a, const WeightMaps& m, bool bf16, int dp, int num_sms, cudaStream_t s) {
  const cudaError_t e = dp == 64 ? (bf16 ? run<64, true>(a, m, num_sms, s) : run<64, false>(a, m, num_sms, s))
                                 : (bf16 ? run<128, true>(a, m, num_sms, s) : run<128, false>(a, m, num_sms, s));
  if (e != cudaSuccess || !a.cut_units) return e;
  return launch_dependent(k_weights_join, dim3(a.cut_units), kUnitKeys, 0, s, a);
}

}  // namespace lv
