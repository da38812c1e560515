// Attention weights added up for the cached tokens, on the fifth-generation tensor cores (lv_weights.cuh has
// how the work is cut).
#include "lv_tc.cuh"
#include "lv_weights.cuh"

namespace lv {

namespace {

// Roles of a CTA's thirteen warps.
constexpr int kSumWarps = 8;              // two warpgroups, one for each half of a unit's keys
constexpr int kWarpK = 8, kWarpQ = 9, kWarpMma = 10, kWarpRows = 11, kWarpUnits = 12;
constexpr int kThreads = 416;
constexpr int kHalf = 128, kUnitKeys = 2 * kHalf;
constexpr int kCols = 128;                // rows of the step (packed) a product has as columns
constexpr int kIndexThreads = 64;
constexpr int kUnits = 4;                 // found ahead
constexpr float kLog2e = 1.44269504088896341f;

template <int DP>
struct WShape {
  static constexpr int kBlocks = DP / 64;                  // 128-byte wide column blocks
  static constexpr int kTile = kHalf * DP * 2;             // bytes of half a unit's K, and of a tile of queries
  static constexpr int kKStages = DP == 128 ? 4 : 8;
  static constexpr int kQStages = DP == 128 ? 3 : 4;
  static constexpr int kQ = kKStages * kTile;
  static constexpr int kMisc = kQ + kQStages * kTile;
};

struct WBars {
  uint64_t k_full[8], k_empty[8], q_full[4], q_empty[4];
  uint64_t s_full[2][2], s_empty[2][2];    // a buffer of scores, a half
  uint64_t b_full[2], b_empty[2];          // the rows' terms beside it
  uint64_t unit_full[kUnits], unit_empty[kUnits];
  uint64_t drain;
  uint32_t tmem;
  volatile int bad;
};

struct Misc {
  WBars bars;
  float b[2][kCols];
  Unit units[kUnits];
  SegmentIndex<kIndexThreads> index;
};
static_assert(WShape<128>::kMisc + sizeof(Misc) <= 227 * 1024, "shared memory of a CTA");
static_assert(WShape<64>::kMisc + sizeof(Misc) <= 227 * 1024, "shared memory of a CTA");

// The n lowest bits, all of them from 32 on, none below 1.
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }
__device__ __forceinline__ int clamp_col(long long x) { return (int)(x < 0 ? 0 : x > kCols ? kCols : x); }

// A unit's products: its packed rows [begin, end) in tiles of `step`.
struct Chunks {
  int begin, end, step, count, halves;
  __device__ __forceinline__ Chunks(const WeightArgs& a, const Unit& u) {
    begin = u.t0 * a.G;
    end = u.t1 * a.G;
    step = a.G > kCols ? kCols : kCols / a.G * a.G;
    count = (end - begin + step - 1) / step;
    halves = u.g.keys - u.key0 > kHalf ? 2 : 1;
  }
  __device__ __forceinline__ int rows(int i) const { return min(step, end - begin - i * step); }
};

// w[j] += sum_r 2^(c q_r.k_j + b_r), b_r = -lse_r log2(e): S = K Q^T with a unit's keys as the product's rows, 128
// and 128 of them, and the step's rows as its columns, so that a thread has a key, adds up its row of S
// as it reads it from TMEM, and writes one word at the end.
//
// One CTA an SM; units are taken in order from a counter, long ones (the first keys of a context, which
// all rows see) first.
//   warp 12  finds units ahead
//   warp 8   K of a unit into a ring of shared memory, by TMA: a box a page and 64 columns
//   warp 9   queries into a ring of their own, by TMA
//   warp 11  the rows' terms b
//   warp 10  products into two buffers of TMEM for each half
//   0 .. 7   exponentials and sums, a thread a key
template <int DP, bool kBf16>
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
      bar_init(&bars.b_full[i], 1);
      bar_init(&bars.b_empty[i], kSumWarps);
    }
    for (int i = 0; i < kUnits; ++i) {
      bar_init(&bars.unit_full[i], 1);
      bar_init(&bars.unit_empty[i], kSumWarps + 4);
    }
    bar_init(&bars.drain, 1);
    bars.bad = 0;
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
  const bool fits = step.kind >= 0 && step.num_tokens <= a.num_tokens;
  if (!fits && blockIdx.x == 0 && threadIdx.x == 0) report(a.ctl, LV_ERR_STATE, -1);
  const int n = step.requests & (kSharedStep - 1);
  // (the sessions' words are in what the copies fill later)
  const int units = fits ? index_segments<kIndexThreads, kUnitKeys>(a, step, m.index, reinterpret_cast<int*>(dyn)) : 0;
  fence_async();
  __syncthreads();

  // the units of the CTA in order, for a role: false at the end or where a wait ran out
  int unit_at = 0;
  uint32_t unit_par = 0;
  bool ok = true;
  Unit u;
  auto next_unit = [&]() -> bool {
    if (!(ok = bar_wait(&bars, &bars.unit_full[unit_at], unit_par, a.wait_ns))) return false;
    u = m.units[unit_at];
    warp_arrive(&bars.unit_empty[unit_at]);
    if (++unit_at == kUnits) {
      unit_at = 0;
      unit_par ^= 1;
    }
    return u.t0 < u.t1;
  };

  if (wid < kSumWarps) {
    const int half = wid >> 2, row = threadIdx.x & 127;
    const uint32_t s_at = tmem + ((uint32_t)(wid & 3) << 21) + kCols * half;      // this warp's 32 lanes of TMEM
    uint32_t b_par = 0, s_par = 0;      // a bit a buffer
    int buf = 0;
    const float2 c2 = make_float2(a.scale, a.scale);
    while (ok && next_unit()) {
      const Chunks ch(a, u);
      const int key = u.key0 + kHalf * half + row;
      const bool there = half < ch.halves, mine = key < u.g.keys;
      float* w = a.w + u.g.sid * a.w_session + u.head * a.w_head + key;
      const float before = mine ? *w : 0.f;
      // the packed rows that see the key: from its own position on, to the window's end
      const long long from = u.g.req < 0 ? 0 : (long long)(key - u.g.first) * a.G;
      const long long to = u.g.req < 0 || a.window == 0 || key < a.sinks ? 1ll << 40 : from + (long long)a.window * a.G;
      const bool check_b = u.g.req < 0 && a.last > 0;
      LongSum all;
      for (int i = 0; i < ch.count; ++i) {
        if (!(ok = bar_wait(&bars, &bars.b_full[buf], b_par >> buf & 1, a.wait_ns))) break;
        b_par ^= 1u << buf;
        if (there) {
          if (!(ok = bar_wait(&bars, &bars.s_full[buf][half], s_par >> buf & 1, a.wait_ns))) break;
          s_par ^= 1u << buf;
          tc_fence_after();
          const int R0 = ch.begin + i * ch.step, rows = ch.rows(i);
          const int c_lo = clamp_col(from - R0), c_hi = mine ? min(rows, clamp_col(to - R0)) : 0;
          const uint32_t at = s_at + 2 * kCols * buf;
          const float* b = m.b[buf];
          float2 acc0 = make_float2(0.f, 0.f), acc1 = acc0;
#pragma unroll 1
          for (int c0 = 0; c0 < rows; c0 += 32) {
            uint32_t x[32];
            tc_ld32(x, at + c0);
            const uint32_t seen = low_bits(c_hi - c0) & ~low_bits(c_lo - c0);
            const bool open = __all_sync(0xffffffffu, seen == ~0u) && !check_b;
            tc_wait_ld();
            tc_loaded<32>(x);
            const float* s = reinterpret_cast<const float*>(x);
            if (open) {
#pragma unroll
              for (int j = 0; j < 32; j += 4) {
                const float4 bb = *reinterpret_cast<const float4*>(b + c0 + j);
                float2 y = fma2(make_float2(s[j], s[j + 1]), c2, make_float2(bb.x, bb.y));
                float2 z = fma2(make_float2(s[j + 2], s[j + 3]), c2, make_float2(bb.z, bb.w));
                y.x = exp2_fast(y.x);
                y.y = exp2_fast(y.y);
                z.x = exp2_fast(z.x);
                z.y = exp2_fast(z.y);
                acc0 = add2(acc0, y);
                acc1 = add2(acc1, z);
              }
            } else if (__any_sync(0xffffffffu, seen != 0)) {
#pragma unroll
              for (int j = 0; j < 32; ++j) {
                const float bb = b[c0 + j];
                const float y = seen >> j & 1u && bb != -INFINITY ? exp2_fast(fmaf(s[j], a.scale, bb)) : 0.f;
                if (j & 1) acc1.x += y;
                else acc0.x += y;
              }
            }
          }
          tc_fence_before();
          warp_arrive(&bars.s_empty[buf][half]);
          acc0 = add2(acc0, acc1);
          all.add(acc0.x + acc0.y);
        }
        warp_arrive(&bars.b_empty[buf]);
        buf ^= 1;
      }
      if (ok && mine && all.sum != 0.f) *w = before + all.sum;
    }
    tc_fence_before();
  } else if (wid == kWarpK) {
    // lane i finds the page of box i of half a unit's keys; one thread then issues the copies
    const int boxes = kHalf / box_rows;
    int stage = 0;
    uint32_t par = 0;
    long long halves = 0;
    while (ok && next_unit()) {
      const Chunks ch(a, u);
      const int32_t* table = u.g.req < 0 ? a.pool_table + (size_t)u.g.sid * a.maxB : a.tables + (size_t)u.g.req * a.maxB;
      for (int h = 0; ok && h < ch.halves; ++h) {
        const int key = u.key0 + kHalf * h + lane * box_rows;
        const int b = a.t_shift >= 0 ? key >> a.t_shift : key / a.T, off = key - b * a.T;
        int page = -1;
        if (lane < boxes && key < u.g.keys) page = table[b];
        if ((uint32_t)page >= a.hbm_pages) page = (int)a.hbm_pages;      // outside the array: zeros
        if (!(ok = bar_wait(&bars, &bars.k_empty[stage], ~par & 1u, a.wait_ns))) break;
        uint64_t* full = &bars.k_full[stage];
        const uint32_t dst = k_s + stage * S::kTile;
        if (elected()) bar_expect(full, S::kTile);
#pragma unroll 1
        for (int i = 0; i < boxes; ++i) {
          const int pg = __shfl_sync(0xffffffffu, page, i), of = __shfl_sync(0xffffffffu, off, i);
          if (elected()) {
#pragma unroll
            for (int x = 0; x < S::kBlocks; ++x)
              tma_box(dst + x * kHalf * 128 + i * box_rows * 128, &kmap, 64 * x, u.head, of, pg, full);
          }
          __syncwarp();
        }
        ++halves;
        if (++stage == S::kKStages) {
          stage = 0;
          par ^= 1;
        }
      }
    }
    if (LV_RARE(bars.bad)) {      // let what is on its way land before the shared memory is given up
      for (long long i = halves < S::kKStages ? 0 : halves - S::kKStages; i < halves; ++i) {
        const unsigned long long t0 = now_ns();
        while (!bar_try(&bars.k_full[i % S::kKStages], (uint32_t)(i / S::kKStages) & 1u))
          if ((long long)(now_ns() - t0) > a.wait_ns) break;
      }
    }
  } else if (wid == kWarpQ) {
    int stage = 0;
    uint32_t par = 0;
    long long tiles = 0;
    while (ok && next_unit()) {
      const Chunks ch(a, u);
      for (int i = 0; ok && i < ch.count; ++i) {
        if (!(ok = bar_wait(&bars, &bars.q_empty[stage], ~par & 1u, a.wait_ns))) break;
        const uint32_t dst = q_s + stage * S::kTile;
        uint64_t* full = &bars.q_full[stage];
        const int R0 = ch.begin + i * ch.step, rows = ch.rows(i);
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
        if (++stage == S::kQStages) {
          stage = 0;
          par ^= 1;
        }
      }
    }
    if (LV_RARE(bars.bad) && q_tma) {
      for (long long i = tiles < S::kQStages ? 0 : tiles - S::kQStages; i < tiles; ++i) {
        const unsigned long long t0 = now_ns();
        while (!bar_try(&bars.q_full[i % S::kQStages], (uint32_t)(i / S::kQStages) & 1u))
          if ((long long)(now_ns() - t0) > a.wait_ns) break;
      }
    }
  } else if (wid == kWarpMma) {
    const uint32_t kd0 = desc_low(k_s, 16), qd0 = desc_low(q_s, 16);
    int ks = 0, qs = 0, buf = 0;
    uint32_t k_par = 0, q_par = 0, s_par = 0;      // s_par: a bit for (buffer, half)
    while (ok && next_unit()) {
      const Chunks ch(a, u);
      int at[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        at[h] = ks;
        if (h >= ch.halves) break;
        if (!(ok = bar_wait(&bars, &bars.k_full[ks], k_par, a.wait_ns))) break;
        if (++ks == S::kKStages) {
          ks = 0;
          k_par ^= 1;
        }
      }
      for (int i = 0; ok && i < ch.count; ++i) {
        if (!(ok = bar_wait(&bars, &bars.q_full[qs], q_par, a.wait_ns))) break;
        const int cols = (ch.rows(i) + 15) & ~15;
        const uint32_t desc = mma_desc<kBf16>(kHalf, cols, false), qd = qd0 + qs * (S::kTile >> 4);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (h >= ch.halves) break;
          if (!(ok = bar_wait(&bars, &bars.s_empty[buf][h], ~(s_par >> (2 * buf + h)) & 1u, a.wait_ns))) break;
          s_par ^= 1u << (2 * buf + h);
          tc_fence_after();
          if (elected()) {
            const uint32_t kd = kd0 + at[h] * (S::kTile >> 4);
#pragma unroll
            for (int k = 0; k < DP / 16; ++k) {
              const uint32_t o = ((k / 4) * (kHalf * 128) + (k % 4) * 32) >> 4;
              tc_mma_ss(tmem + kCols * (2 * buf + h), kd + o, qd + o, desc, k > 0);
            }
            tc_commit(&bars.s_full[buf][h]);
            if (i + 1 == ch.count) tc_commit(&bars.k_empty[at[h]]);
            if (h + 1 == ch.halves) tc_commit(&bars.q_empty[qs]);
          }
          __syncwarp();
        }
        buf ^= 1;
        if (++qs == S::kQStages) {
          qs = 0;
          q_par ^= 1;
        }
      }
    }
    if (LV_RARE(bars.bad)) {      // let the products under way end
      if (elected()) tc_commit(&bars.drain);
      const unsigned long long t0 = now_ns();
      while (!bar_try(&bars.drain, 0))
        if ((long long)(now_ns() - t0) > a.wait_ns) break;
      __syncwarp();
    }
  } else if (wid == kWarpRows) {
    uint32_t par = 0;      // a bit a buffer
    int buf = 0;
    const int Hq = a.H * a.G;
    while (ok && next_unit()) {
      const Chunks ch(a, u);
      for (int i = 0; ok && i < ch.count; ++i) {
        const int R0 = ch.begin + i * ch.step, rows = ch.rows(i);
        float b[kCols / 32];
#pragma unroll
        for (int k = 0; k < kCols / 32; ++k) {
          const int c = 32 * k + lane, R = R0 + c, token = R / a.G;
          float z = -INFINITY;
          if (c < rows && counts(a, u.g, n, token))
            z = a.lse[(int64_t)(u.g.qrow + token) * Hq + u.head * a.G + (R - token * a.G)];
          b[k] = z == -INFINITY ? z : -z * kLog2e;
        }
        if (!(ok = bar_wait(&bars, &bars.b_empty[buf], ~(par >> buf) & 1u, a.wait_ns))) break;
        par ^= 1u << buf;
#pragma unroll
        for (int k = 0; k < kCols / 32; ++k) m.b[buf][32 * k + lane] = b[k];
        warp_arrive(&bars.b_full[buf]);
        buf ^= 1;
      }
    }
  } else {
    int at = 0;
    uint32_t par = 0;
    int t = blockIdx.x, following = 0;
    auto ask = [&]() {
      if (lane == 0) following = gridDim.x + atomicAdd(&a.tickets[0], 1);
    };
    for (;;) {
      ask();
      Unit x{};
      if (t < units) x = find_unit<kIndexThreads, kUnitKeys>(a, step, m.index, t);
      const bool end = t >= units;
      if (end || x.t0 < x.t1) {
        if (!bar_wait(&bars, &bars.unit_empty[at], ~par & 1u, a.wait_ns)) break;
        if (lane == 0) m.units[at] = x;
        warp_arrive(&bars.unit_full[at]);
        if (++at == kUnits) {
          at = 0;
          par ^= 1;
        }
      }
      if (end) break;
      t = __shfl_sync(0xffffffffu, following, 0);
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
  return launch_dependent(k_weights_tc<DP, kBf16>, dim3(ctas), kThreads, WShape<DP>::kMisc + sizeof(Misc), s, a, *m.k,
                          m.q ? *m.q : none, m.q_few ? *m.q_few : none, m.box_rows, m.few_rows, m.q ? 1 : 0);
}

template <int DP>
cudaError_t set() {
  for (auto k : {k_weights_tc<DP, true>, k_weights_tc<DP, false>}) {
    const cudaError_t e =
        cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, WShape<DP>::kMisc + (int)sizeof(Misc));
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace

cudaError_t configure_weights_tc() {
  const cudaError_t e = set<64>();
  return e != cudaSuccess ? e : set<128>();
}

cudaError_t launch_weights_tc(const WeightArgs& a, const WeightMaps& m, bool bf16, int dp, int num_sms, cudaStream_t s) {
  if (dp == 64) return bf16 ? run<64, true>(a, m, num_sms, s) : run<64, false>(a, m, num_sms, s);
  return bf16 ? run<128, true>(a, m, num_sms, s) : run<128, false>(a, m, num_sms, s);
}

}  // namespace lv
