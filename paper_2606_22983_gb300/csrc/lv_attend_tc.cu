// Attention of requests with many rows (chunks of user input, prompts, and single tokens beside
// them) over the paged context, on the fifth-generation tensor cores.
#include "lv_batch.cuh"

namespace lv {

namespace {

// Roles of a CTA's twelve warps.
constexpr int kSoftWarps = 8;             // two warpgroups, one for each tile of 128 rows
constexpr int kWarpKv = 8, kWarpMma = 9, kWarpQ = 10;   // and 11: queries of tile 0 and 1
constexpr int kThreads = 384;
constexpr int kKeys = kTcUnit;            // keys of a unit
// registers a thread: 168 at launch (384 * 168 = 64 512), then 208 for the softmax warps and 88
// for the others (256 * 208 + 128 * 88 = 64 512)
constexpr int kRegsSoft = 208, kRegsOther = 88;
constexpr long long kWaitLimitNs = 1000000000ll;   // one second a wait

template <int DP>
struct TcShape {
  static constexpr int kHalves = DP / 64;                  // 128-byte wide column blocks
  static constexpr int kBlock = kKeys * DP * 2;            // bytes of a K or V unit, and of a Q tile
  static constexpr int kStages = DP == 128 ? 5 : 8;
  static constexpr int kSmem = 2 * kBlock + kStages * kBlock + 1024;
  static constexpr int kColO = 256;                        // S0 at column 0, S1 at 128, O0, O1
};

struct Bars {
  uint64_t kv_full[8], kv_empty[8];
  uint64_t q_full[2], q_empty[2], s_full[2], p_full[2], o_full[2];
  uint64_t drain;
  uint32_t tmem;
  volatile int bad;
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint64_t* b, uint32_t n) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(b)), "r"(n) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t* b) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(b)) : "memory");
}
__device__ __forceinline__ void bar_expect(uint64_t* b, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(b)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint64_t* b, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done)
      : "r"(smem_u32(b)), "r"(parity)
      : "memory");
  return done != 0;
}
__device__ __forceinline__ unsigned long long now_ns() {
  unsigned long long t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}
// False once the limit has passed, here or in another role: every role then leaves its loop.
__device__ __forceinline__ bool bar_wait_slow(Bars* b, uint64_t* bar, uint32_t parity) {
  const unsigned long long t0 = now_ns();
  for (;;) {
    if (bar_try(bar, parity)) return true;
    if (b->bad) return false;
    if ((long long)(now_ns() - t0) > kWaitLimitNs) {
      b->bad = 1;
      return false;
    }
  }
}
// For a whole warp, whose lanes leave it together with one answer (what follows is .aligned).
__device__ __forceinline__ bool bar_wait(Bars* b, uint64_t* bar, uint32_t parity) {
  bool ok = bar_try(bar, parity);
  if (!ok) ok = bar_wait_slow(b, bar, parity);
  return __all_sync(0xffffffffu, ok);
}

// ---- tcgen05
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar))
               : "memory");
}
// D[tmem] (+)= A[smem] B[smem]
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(desc), "r"((uint32_t)add)
      : "memory");
}
// D[tmem] (+)= A[tmem] B[smem]
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t desc, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(desc), "r"((uint32_t)add)
      : "memory");
}
#define LV_R8(x, i) "=r"(x[i]), "=r"(x[i + 1]), "=r"(x[i + 2]), "=r"(x[i + 3]), "=r"(x[i + 4]), "=r"(x[i + 5]), \
                    "=r"(x[i + 6]), "=r"(x[i + 7])
#define LV_W8(x, i) "r"(x[i]), "r"(x[i + 1]), "r"(x[i + 2]), "r"(x[i + 3]), "r"(x[i + 4]), "r"(x[i + 5]), \
                    "r"(x[i + 6]), "r"(x[i + 7])
// 32 columns of this warp's 32 lanes, a lane a row
__device__ __forceinline__ void tc_ld32(uint32_t* x, uint32_t at) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,"
      "%30,%31}, [%32];"
      : LV_R8(x, 0), LV_R8(x, 8), LV_R8(x, 16), LV_R8(x, 24)
      : "r"(at));
}
__device__ __forceinline__ void tc_ld16(uint32_t* x, uint32_t at) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : LV_R8(x, 0), LV_R8(x, 8)
      : "r"(at));
}
__device__ __forceinline__ void tc_st16(uint32_t at, const uint32_t* x) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::LV_W8(
          x, 0),
      LV_W8(x, 8), "r"(at)
      : "memory");
}
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// The loaded values as of now: nothing that reads them moves above the wait before this.
template <int N>
__device__ __forceinline__ void tc_loaded(uint32_t* x) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+r"(x[i]));
}
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// Shared-memory matrix descriptors, 128-byte swizzle (rows of 128 bytes, the pattern repeating
// every 8 rows = 1024 bytes).  K-major (Q, K): stride between 8-row groups 1024 bytes.
// MN-major (V: rows are keys, columns are O's): 64 columns a block, blocks kKeys * 128 bytes
// apart (leading offset), groups of 8 keys 1024 bytes apart (stride offset).
__device__ __forceinline__ uint64_t smem_desc(uint32_t at, uint32_t lead, uint32_t stride) {
  return (uint64_t)((at & 0x3ffffu) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(stride >> 4) << 32 | 1ull << 46 |
         2ull << 61;
}
// Instruction descriptor of kind::f16: 32-bit accumulation, A and B of one 16-bit type.
template <bool kBf16>
__device__ __forceinline__ constexpr uint32_t mma_desc(int m, int n, bool b_mn_major) {
  return 1u << 4 | (kBf16 ? 1u : 0u) << 7 | (kBf16 ? 1u : 0u) << 10 | (b_mn_major ? 1u : 0u) << 16 |
         (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}

__device__ __forceinline__ void tma_box(uint32_t dst, const CUtensorMap* map, int x, int head, int row, int page,
                                        uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::
          "r"(dst),
      "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(head), "r"(row), "r"(page)
      : "memory");
}

__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(reinterpret_cast<unsigned long long&>(d))
      : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)),
        "l"(reinterpret_cast<unsigned long long&>(c)));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("add.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<unsigned long long&>(d))
      : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
  return d;
}

// The pairs (tile, head) of a CTA's share, one after the other.
struct Pairs {
  long long w, end;
  AttnTile t;
  int tile, head, u0, u1;
  bool started;
  __device__ __forceinline__ void init(const AttnArgs& a) {
    const long long units = a.head->units, share = a.head->share;
    w = blockIdx.x * share;
    end = min(units, w + share);
    started = false;
  }
  __device__ __forceinline__ bool next(const AttnArgs& a) {
    if (w >= end) return false;
    if (!started) {
      started = true;
      tile = a.cta_tile[blockIdx.x];
      t = load_tile(&a.tiles[tile]);
    } else if (w >= t.before + (long long)t.units * a.groups) {
      t = load_tile(&a.tiles[++tile]);
    }
    const long long off = w - t.before;
    head = (int)(off / t.units);
    u0 = (int)(off - (long long)head * t.units);
    u1 = (int)min((long long)t.units, u0 + (end - w));
    w += u1 - u0;
    return true;
  }
  __device__ __forceinline__ int key_of(int u) const {
    return (u < t.sink_units ? u : t.win_unit + u - t.sink_units) * kKeys;
  }
};

// Weights of one tile's rows for one unit: a thread a row.  S is read from TMEM, and the weights
// replace it there in 16 bits, two to a column, as the left operand of the product with V.
template <int DP, bool kBf16>
struct Softmax {
  float top, sum;      // of the raw scores; sum of the weights
  __device__ __forceinline__ void step(const AttnArgs& a, uint32_t s_at, uint32_t o_at, bool fresh, bool open, int key0,
                                       int pos, float c) {
    uint32_t x[128];
#pragma unroll
    for (int i = 0; i < 4; ++i) tc_ld32(x + 32 * i, s_at + 32 * i);
    tc_wait_ld();
    tc_loaded<128>(x);
    float* s = reinterpret_cast<float*>(x);
    if (!open) {
      // keys key0 + i: seen up to pos, from the window's start or among the sinks
      const int hi = pos - key0, lo = a.window > 0 ? pos - a.window - key0 : -1, sk = a.sinks - key0;
#pragma unroll
      for (int i = 0; i < 128; ++i)
        if (i > hi || (i <= lo && i >= sk)) s[i] = -INFINITY;
    }
    float m0 = fmaxf(s[0], s[1]), m1 = fmaxf(s[2], s[3]);
#pragma unroll
    for (int i = 4; i < 128; i += 4) {
      m0 = fmaxf(fmaxf(m0, s[i]), s[i + 1]);
      m1 = fmaxf(fmaxf(m1, s[i + 2]), s[i + 3]);
    }
    const float high = fmaxf(fmaxf(m0, m1), top);
    const bool raise = (high - top) * c > kLazy;      // (NaN from -inf - -inf: no)
    if (fresh) {
      top = high;
    } else if (__any_sync(0xffffffffu, raise)) {
      // S of this unit follows the previous unit's product with V: O is at rest
      const float f = high == top ? 1.f : exp2_fast((top - high) * c);
      top = high;
      sum *= f;
#pragma unroll
      for (int i = 0; i < DP; i += 16) {
        uint32_t o[16];
        tc_ld16(o, o_at + i);
        tc_wait_ld();
        tc_loaded<16>(o);
#pragma unroll
        for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
        tc_st16(o_at + i, o);
      }
    }
    const float b = weight_bias<kBf16>() - (top == -INFINITY ? 0.f : top * c);
    const float2 c2 = make_float2(c, c), b2 = make_float2(b, b);
    float2 acc0 = make_float2(0.f, 0.f), acc1 = acc0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t w[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int k = 32 * i + 2 * j;
        float2 y = fma2(make_float2(s[k], s[k + 1]), c2, b2);
        y.x = exp2_fast(y.x);
        y.y = exp2_fast(y.y);
        if (j & 1) acc1 = add2(acc1, y);
        else acc0 = add2(acc0, y);
        w[j] = pack16<kBf16>(y.x, y.y);
      }
      tc_st16(s_at + 16 * i, w);
    }
    acc0 = add2(acc0, acc1);
    sum += acc0.x + acc0.y;
    tc_wait_st();
  }
};

// One CTA an SM: its share of the line of units.  A tile is 256 packed rows, two halves of 128
// (an M = 128 tile of the tensor core each) whose softmaxes take turns: while one half's
// weights are computed, the tensor core runs the other half's products.
//   warp 8   K and V units into a ring of shared memory, by TMA: a box a page and 64 columns;
//            what the table has no page for, and rows past a tile's keys, reads as zeros
//   warp 9   S = Q K^T (tcgen05, operands in shared memory), O += P V (P in TMEM)
//   10, 11   queries of the two halves, when the previous pair's last S has been issued
//   0 .. 7   softmax, a thread a row, and the pair's end: O / sum, or the sums of a cut pair
template <int DP, bool kBf16>
__global__ void __launch_bounds__(kThreads, 1)
k_attend_tc(const __grid_constant__ AttnArgs a, const __grid_constant__ CUtensorMap kmap,
            const __grid_constant__ CUtensorMap vmap, int box_rows) {
  using S = TcShape<DP>;
  extern __shared__ __align__(1024) unsigned char dyn[];
  __shared__ Bars bars;
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const uint32_t base = (smem_u32(dyn) + 1023u) & ~1023u;
  const uint32_t q_s = base, ring_s = base + 2 * S::kBlock;
  if (threadIdx.x == 0) {
    for (int i = 0; i < S::kStages; ++i) {
      bar_init(&bars.kv_full[i], 1);
      bar_init(&bars.kv_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      bar_init(&bars.q_full[i], 32);
      bar_init(&bars.q_empty[i], 1);
      bar_init(&bars.s_full[i], 1);
      bar_init(&bars.p_full[i], 128);
      bar_init(&bars.o_full[i], 1);
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

  if (wid < kSoftWarps) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoft));
    const int half = wid >> 2;
    const int row = 128 * half + (threadIdx.x & 127);       // of the tile
    const uint32_t lanes = (uint32_t)(wid & 3) << 21;       // this warp's 32 lanes of TMEM
    const uint32_t s_at = tmem + lanes + 128 * half, o_at = tmem + lanes + S::kColO + DP * half;
    uint32_t s_par = 0, o_par = 0;
    Pairs pr;
    pr.init(a);
    bool ok = true;
    while (ok && pr.next(a)) {
      if (pr.t.rows <= 128 * half) continue;                // nothing in this half
      const bool live = pr.t.rows > (row & ~31);            // rows in this warp
      const int R = pr.t.row0 + min(row, pr.t.rows - 1), token = R / a.G;
      const int pos = pr.t.first + token;
      const int p_lo = pr.t.first + (pr.t.row0 + 128 * half) / a.G;
      const int p_hi = pr.t.first + (pr.t.row0 + min(128 * half + 127, pr.t.rows - 1)) / a.G;
      Softmax<DP, kBf16> sm{-INFINITY, 0.f};
      for (int u = pr.u0; u < pr.u1; ++u) {
        if (!bar_wait(&bars, &bars.s_full[half], s_par)) {
          ok = false;
          break;
        }
        s_par ^= 1;
        if (live) {
          tc_fence_after();
          const int key0 = pr.key_of(u);
          const bool open =
              key0 + kKeys - 1 <= p_lo && (a.window == 0 || key0 > p_hi - a.window || key0 + kKeys <= a.sinks);
          sm.step(a, s_at, o_at, u == pr.u0, open, key0, pos, a.scale);
          tc_fence_before();
        }
        bar_arrive(&bars.p_full[half]);
      }
      if (!ok || !bar_wait(&bars, &bars.o_full[half], o_par)) break;
      o_par ^= 1;
      if (!live) continue;
      tc_fence_after();
      const bool whole = pr.u0 == 0 && pr.u1 == pr.t.units;
      const int h = pr.head * a.G + (R - token * a.G);
      const int64_t r = pr.t.qrow + token;
      const bool mine = row < pr.t.rows;
      const float inv = !whole ? 1.f : sm.sum > 0.f || sm.sum != sm.sum ? 1.f / sm.sum : 0.f;
      const int64_t slot = part_slot(blockIdx.x, pr.u0 == 0) * a.tile_rows + row;
      uint16_t* out = reinterpret_cast<uint16_t*>(a.out) + r * a.o_row + h * a.o_head;
#pragma unroll
      for (int i = 0; i < DP; i += 32) {
        uint32_t o[32];
        tc_ld32(o, o_at + i);
        tc_wait_ld();
        tc_loaded<32>(o);
        if (mine && whole) {
#pragma unroll
          for (int j = 0; j < 32; j += 8) {
            if (i + j >= a.D) continue;
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
              w[e] = pack16<kBf16>(__uint_as_float(o[j + 2 * e]) * inv, __uint_as_float(o[j + 2 * e + 1]) * inv);
            if (a.o_vec) {
              *reinterpret_cast<uint4*>(out + i + j) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                out[i + j + 2 * e] = (uint16_t)w[e];
                out[i + j + 2 * e + 1] = (uint16_t)(w[e] >> 16);
              }
            }
          }
        } else if (mine) {
          float4* po = reinterpret_cast<float4*>(a.part_o + slot * DP + i);
#pragma unroll
          for (int j = 0; j < 32; j += 4)
            po[j / 4] = make_float4(__uint_as_float(o[j]), __uint_as_float(o[j + 1]), __uint_as_float(o[j + 2]),
                                    __uint_as_float(o[j + 3]));
        }
        __syncwarp();
      }
      const float top2 = sm.top * a.scale;      // in log2
      if (mine && !whole) {
        a.part_ml[slot] = make_float2(top2, sm.sum);
      } else if (mine && a.lse) {
        a.lse[r * (a.H * a.G) + h] =
            sm.sum == 0.f ? -INFINITY : (top2 - weight_bias<kBf16>()) * 0.693147180559945f + logf(sm.sum);
      }
    }
    tc_fence_before();
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
    Pairs pr;
    pr.init(a);
    if (wid == kWarpKv) {
      // ---- K and V
      int stage = 0;
      uint32_t par = 0;               // of the ring's current round
      long long loads = 0;
      bool ok = true;
      auto unit = [&](const CUtensorMap* map, int key0) -> bool {
        if (!bar_wait(&bars, &bars.kv_empty[stage], par ^ 1)) return false;
        if (lane == 0) bar_expect(&bars.kv_full[stage], S::kBlock);
        __syncwarp();
        const uint32_t dst = ring_s + stage * S::kBlock;
        for (int i = lane; i < kKeys / box_rows * S::kHalves; i += 32) {
          const int box = i / S::kHalves, x = i % S::kHalves;
          const int key = key0 + box * box_rows;
          const int b = key / a.T;
          int page = -1;
          if (key < pr.t.kv_hi && (key + box_rows > pr.t.kv_lo || key < a.sinks))
            page = a.tables[(size_t)pr.t.req * a.maxB + b];
          // no page: a box outside the array, which reads as zeros
          if ((uint32_t)page >= a.hbm_pages) page = (int)a.hbm_pages;
          tma_box(dst + x * kKeys * 128 + box * box_rows * 128, map, 64 * x, pr.head, key - b * a.T, page,
                  &bars.kv_full[stage]);
        }
        ++loads;
        if (++stage == S::kStages) {
          stage = 0;
          par ^= 1;
        }
        return true;
      };
      while (ok && pr.next(a))
        for (int u = pr.u0; ok && u < pr.u1; ++u) {
          const int key0 = pr.key_of(u);
          ok = unit(&kmap, key0) && unit(&vmap, key0);
        }
      if (!ok) {      // let what is on its way land before the shared memory is given up
        const long long n = loads < S::kStages ? loads : S::kStages;
        for (long long i = loads - n; i < loads; ++i) {
          const unsigned long long t0 = now_ns();
          while (!bar_try(&bars.kv_full[i % S::kStages], (uint32_t)(i / S::kStages) & 1u))
            if ((long long)(now_ns() - t0) > kWaitLimitNs) break;
        }
      }
    } else if (wid == kWarpMma) {
      // ---- products
      constexpr uint32_t kDescS = mma_desc<kBf16>(128, kKeys, false), kDescO = mma_desc<kBf16>(128, DP, true);
      uint32_t par = 0, p_par[2] = {0, 0}, q_par[2] = {0, 0};
      int stage = 0;
      bool ok = true;
      auto step = [&]() {
        if (++stage == S::kStages) {
          stage = 0;
          par ^= 1;
        }
      };
      auto scores = [&](int half, int st) {      // S_half = Q_half K^T
        if (lane == 0) {
#pragma unroll
          for (int k = 0; k < DP / 16; ++k) {
            const uint32_t at = (k / 4) * (kKeys * 128) + (k % 4) * 32;
            tc_mma_ss(tmem + 128 * half, smem_desc(q_s + half * S::kBlock + at, 16, 1024),
                      smem_desc(ring_s + st * S::kBlock + at, 16, 1024), kDescS, k > 0);
          }
          tc_commit(&bars.s_full[half]);
        }
        __syncwarp();
      };
      auto values = [&](int half, int st, bool add) {      // O_half (+)= P_half V
        if (lane == 0) {
#pragma unroll
          for (int k = 0; k < kKeys / 16; ++k)
            tc_mma_ts(tmem + S::kColO + DP * half, tmem + 128 * half + 8 * k,
                      smem_desc(ring_s + st * S::kBlock + k * 2048, kKeys * 128, 1024), kDescO, add || k > 0);
        }
        __syncwarp();
      };
      auto release = [&](uint64_t* bar) {
        if (lane == 0) tc_commit(bar);
        __syncwarp();
      };
      while (ok && pr.next(a)) {
        const int halves = pr.t.rows > 128 ? 2 : 1;
        // the first unit's scores
        if (!(ok = bar_wait(&bars, &bars.kv_full[stage], par))) break;
        for (int h = 0; h < halves && ok; ++h) {
          if (!(ok = bar_wait(&bars, &bars.q_full[h], q_par[h]))) break;
          q_par[h] ^= 1;
          tc_fence_after();
          scores(h, stage);
          if (pr.u1 - pr.u0 == 1) release(&bars.q_empty[h]);
        }
        if (!ok) break;
        release(&bars.kv_empty[stage]);
        step();
        for (int u = pr.u0; ok && u < pr.u1; ++u) {
          const int vs = stage;
          if (!(ok = bar_wait(&bars, &bars.kv_full[vs], par))) break;
          step();
          // rows of V that no row of the tile sees hold whatever the page does: zeros, since a
          // weight of zero does not cancel a NaN
          const int key0 = pr.key_of(u);
          if (key0 + kKeys > pr.t.kv_hi || (key0 < pr.t.kv_lo && key0 + kKeys > a.sinks)) {
            for (int i = lane; i < kKeys * 8; i += 32) {
              const int key = key0 + i / 8;
              if (key < pr.t.kv_hi && (key >= pr.t.kv_lo || key < a.sinks)) continue;
#pragma unroll
              for (int x = 0; x < S::kHalves; ++x)
                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(ring_s + vs * S::kBlock + x * kKeys * 128 +
                                                                             (i / 8) * 128 + (i % 8) * 16),
                             "r"(0)
                             : "memory");
            }
            fence_async();
            __syncwarp();
          }
          const bool more = u + 1 < pr.u1;
          const int ks = stage;
          for (int h = 0; h < halves && ok; ++h) {
            if (!(ok = bar_wait(&bars, &bars.p_full[h], p_par[h]))) break;
            p_par[h] ^= 1;
            tc_fence_after();
            values(h, vs, u > pr.u0);
            if (h == halves - 1) release(&bars.kv_empty[vs]);
            if (!more) {
              release(&bars.o_full[h]);
              continue;
            }
            if (h == 0 && !(ok = bar_wait(&bars, &bars.kv_full[ks], par))) break;
            scores(h, ks);
            if (u + 2 == pr.u1) release(&bars.q_empty[h]);
          }
          if (ok && more) {
            release(&bars.kv_empty[ks]);
            step();
          }
        }
      }
      if (!ok) {      // let the products under way end
        release(&bars.drain);
        const unsigned long long t0 = now_ns();
        while (!bar_try(&bars.drain, 0))
          if ((long long)(now_ns() - t0) > kWaitLimitNs) break;
        if (lane == 0) report(a.ctl, LV_ERR_TIMEOUT, blockIdx.x);
      }
    } else {
      // ---- queries of one half
      const int half = wid - kWarpQ;
      uint32_t par = 0;
      bool ok = true;
      constexpr int kChunks = DP / 8;
      while (ok && pr.next(a)) {
        const int rows = min(128, pr.t.rows - 128 * half);
        if (rows <= 0) continue;
        if (!(ok = bar_wait(&bars, &bars.q_empty[half], par ^ 1))) break;
        par ^= 1;
        const uint16_t* q = reinterpret_cast<const uint16_t*>(a.q);
#pragma unroll 4
        for (int i = lane; i < 128 * kChunks; i += 32) {
          const int row = i / kChunks, c = i % kChunks;
          const bool in = row < rows && c * 8 < a.D;
          const int R = pr.t.row0 + 128 * half + (row < rows ? row : 0), token = R / a.G, g = R - token * a.G;
          const uint16_t* src = q + (pr.t.qrow + token) * a.q_row + (int64_t)(pr.head * a.G + g) * a.q_head + c * 8;
          const uint32_t dst = q_s + half * S::kBlock + (c / 8) * (kKeys * 128) + row * 128 + (((c % 8) ^ (row & 7)) << 4);
          if (a.q_vec || !in) {
            const int n = in ? 16 : 0;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(in ? (const void*)src : a.q), "r"(n)
                         : "memory");
          } else {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = (uint32_t)src[2 * e] | (uint32_t)src[2 * e + 1] << 16;
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3])
                         : "memory");
          }
        }
        asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 0;" ::: "memory");
        fence_async();
        bar_arrive(&bars.q_full[half]);
      }
      // rows of no request
      if (ok && a.head->dead > 0) {
        const int Hq = a.H * a.G;
        for (int r = blockIdx.x * 2 + half; r < a.num_tokens; r += gridDim.x * 2) {
          if (a.positions[r] >= 0) continue;
          for (int h = 0; h < Hq; ++h) {
            uint16_t* o = reinterpret_cast<uint16_t*>(a.out) + r * a.o_row + h * a.o_head;
            for (int d = lane; d < a.D; d += 32) o[d] = 0;
          }
          if (a.lse)
            for (int h = lane; h < Hq; h += 32) a.lse[(size_t)r * Hq + h] = -INFINITY;
        }
      }
    }
    tc_fence_before();
  }
  __syncthreads();
  if (wid == kWarpMma) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

template <int DP, bool kBf16>
cudaError_t run(const AttnArgs& a, const CUtensorMap& k, const CUtensorMap& v, int box_rows, int ctas, cudaStream_t s) {
  return launch_dependent(k_attend_tc<DP, kBf16>, dim3(ctas), kThreads, TcShape<DP>::kSmem, s, a, k, v, box_rows);
}

}  // namespace

cudaError_t configure_attend_tc() {
  for (auto k : {k_attend_tc<64, true>, k_attend_tc<64, false>}) {
    const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, TcShape<64>::kSmem);
    if (e != cudaSuccess) return e;
  }
  for (auto k : {k_attend_tc<128, true>, k_attend_tc<128, false>}) {
    const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, TcShape<128>::kSmem);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_attend_tc(const AttnArgs& a, const CUtensorMap& k, const CUtensorMap& v, int box_rows, bool bf16,
                             int ctas, cudaStream_t s) {
  if (a.dp == 64) return bf16 ? run<64, true>(a, k, v, box_rows, ctas, s) : run<64, false>(a, k, v, box_rows, ctas, s);
  return bf16 ? run<128, true>(a, k, v, box_rows, ctas, s) : run<128, false>(a, k, v, box_rows, ctas, s);
}

}  // namespace lv
