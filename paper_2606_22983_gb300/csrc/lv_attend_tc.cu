// Attention of requests with many rows (chunks of user input, prompts, and single tokens beside
// them) over the paged context, on the fifth-generation tensor cores.
#include <type_traits>

#include "lv_batch.cuh"

namespace lv {

namespace {

// Roles of a CTA's twelve warps.
constexpr int kSoftWarps = 8;             // two warpgroups, one for each half of a tile
constexpr int kWarpK = 8, kWarpV = 9, kWarpMma = 10;    // and 11: queries and zeros
constexpr int kThreads = 384;
constexpr int kKeys = kTcUnit;            // keys of a unit
// registers a thread: 168 at launch (384 * 168 = 64 512), then 208 for the softmax warps and 88
// for the others (256 * 208 + 128 * 88 = 64 512)
constexpr int kRegsSoft = 208, kRegsOther = 88;

template <int DP>
struct TcShape {
  static constexpr int kHalves = DP / 64;                  // 128-byte wide column blocks
  static constexpr int kBlock = kKeys * DP * 2;            // bytes of a K or V unit, and of a Q tile
  static constexpr int kStages = DP == 128 ? 5 : 8;
  static constexpr int kData = 2 * kBlock + kStages * kBlock;
  static constexpr int kSmem = kData + 512;                // then the barriers
  static constexpr int kColO = 256;                        // S0 at column 0, S1 at 128, O0, O1
  static_assert(kSmem + 1024 <= 227 * 1024, "shared memory of a CTA");
};

struct Bars {
  uint64_t kv_full[8], kv_empty[8];
  uint64_t q_full[2], q_empty[2], s_full[2], p_full[2][3], o_full[2];
  uint64_t clean_ask, clean_done, drain;
  uint32_t tmem;
  volatile int bad;
};
static_assert(sizeof(Bars) <= 512, "its room in shared memory");

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint64_t* b, uint32_t n) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(b)), "r"(n) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t* b) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(b)) : "memory");
}
// Once for a warp, after what its lanes did before.
__device__ __forceinline__ void warp_arrive(uint64_t* b) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) bar_arrive(b);
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
// False once the limit has passed, here or in another role: every role then leaves its loop.  (The limit is
// a kernel argument: kept in shared memory beside the barriers, it cost 8 prompts of 4096 742 us for 718.)
__device__ __forceinline__ bool bar_wait_slow(Bars* b, uint64_t* bar, uint32_t parity, long long limit) {
  const unsigned long long t0 = now_ns();
  for (;;) {
    if (bar_try(bar, parity)) return true;
    if (b->bad) return false;
    if ((long long)(now_ns() - t0) > limit) {
      b->bad = 1;
      return false;
    }
  }
}
// For one thread.
__device__ __forceinline__ bool bar_wait1(Bars* b, uint64_t* bar, uint32_t parity, long long limit) {
  if (LV_MOSTLY(bar_try(bar, parity))) return true;
  return bar_wait_slow(b, bar, parity, limit);
}
// For a whole warp, whose lanes leave it together with one answer (what follows is .aligned).
__device__ __forceinline__ bool bar_wait(Bars* b, uint64_t* bar, uint32_t parity, long long limit) {
  bool ok = bar_try(bar, parity);
  if (LV_RARE(!ok)) ok = bar_wait_slow(b, bar, parity, limit);
  return __all_sync(0xffffffffu, ok);
}

// ---- tcgen05
// Shared-memory matrix descriptors, 128-byte swizzle (rows of 128 bytes, the pattern repeating
// every 8 rows = 1024 bytes).  K-major (Q, K): stride between 8-row groups 1024 bytes.
// MN-major (V: rows are keys, columns are O's): 64 columns a block, blocks kKeys * 128 bytes
// apart (leading offset), groups of 8 keys 1024 bytes apart (stride offset).
constexpr uint32_t kDescHigh = 1024u >> 4 | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint32_t desc_low(uint32_t at, uint32_t lead) { return (at & 0x3ffffu) >> 4 | (lead >> 4) << 16; }
// One lane of the warp, always the same.  (With a test of the lane number in its place the
// compiler cannot tell that one thread issues, and a product took 109 cycles to issue, not 64.)
__device__ __forceinline__ bool elected() {
  uint32_t e;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(e)
      :
      : "memory");
  return e != 0;
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar))
               : "memory");
}
// Matrix descriptors by their low words (address and leading offset); the high one is the same
// for all operands here.
// D[tmem] (+)= A[smem] B[smem]
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t desc, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
      "mov.b64 da, {%1, %5};\n\t"
      "mov.b64 db, {%2, %5};\n\t"
      "setp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}" ::"r"(d),
      "r"(a), "r"(b), "r"(desc), "r"((uint32_t)add), "n"(kDescHigh)
      : "memory");
}
// D[tmem] (+)= A[tmem] B[smem]
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t desc, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\t"
      "mov.b64 db, {%2, %5};\n\t"
      "setp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}" ::"r"(d),
      "r"(a), "r"(b), "r"(desc), "r"((uint32_t)add), "n"(kDescHigh)
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
__device__ __forceinline__ void tc_st32(uint32_t at, const uint32_t* x) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,"
      "%30,%31};" ::LV_W8(x, 0),
      LV_W8(x, 8), LV_W8(x, 16), LV_W8(x, 24), "r"(at)
      : "memory");
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

// A piece's sums lie [4 columns][row of the tile][4], so that a warp, a lane a row, writes and reads
// 512 bytes at once.
template <int DP>
__device__ __forceinline__ float4* part_at(const AttnArgs& a, int64_t slot, int col, int row) {
  return reinterpret_cast<float4*>(a.part_o) + (slot * (DP / 4) + col / 4) * a.tile_rows + row;
}

// Pieces p0, p0 + step, ... (count of them) of a cut pair joined by one warp, a lane a row of the
// tile: every piece's sums weighted by its maximum against the largest, in the pieces' order.  To
// the output, or (not last) to the first of the pieces' own slots.
template <int DP, bool kBf16>
__device__ __forceinline__ void join_rows(const AttnArgs& a, int64_t first, int p0, int step, int count, bool last,
                                          int row, bool mine, uint16_t* out, int64_t r, int hq) {
  auto slot = [&](int i) {
    const int p = p0 + min(i, count - 1) * step;
    return part_slot(first + p, p == 0);
  };
  auto ml_of = [&](int i) { return __ldcg(&a.part_ml[slot(i) * a.tile_rows + row]); };
  float top = -INFINITY, sum = 0.f;
  if (mine) {
    for (int i = 0; i < count; i += 4) {
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = ml_of(i + e).x;
      top = fmaxf(fmaxf(fmaxf(top, x[0]), fmaxf(x[1], x[2])), x[3]);
    }
#pragma unroll 1
    for (int c0 = 0; c0 < DP; c0 += 64) {
      float4 acc[16];
#pragma unroll
      for (int c = 0; c < 16; ++c) acc[c] = make_float4(0.f, 0.f, 0.f, 0.f);
      float2 next = ml_of(0);
      sum = 0.f;
#pragma unroll 1
      for (int p = 0; p < count; ++p) {
        const float2 ml = next;
        next = ml_of(p + 1);
        const float f = ml.x == top ? 1.f : exp2_fast(ml.x - top);
        sum += ml.y * f;
        const float4* o = part_at<DP>(a, slot(p), c0, row);
#pragma unroll
        for (int c = 0; c < 16; ++c) {
          const float4 v = __ldcg(o + c * a.tile_rows);
          acc[c].x += v.x * f;
          acc[c].y += v.y * f;
          acc[c].z += v.z * f;
          acc[c].w += v.w * f;
        }
      }
      if (!last) {
        float4* o = part_at<DP>(a, slot(0), c0, row);
#pragma unroll
        for (int c = 0; c < 16; ++c) o[c * a.tile_rows] = acc[c];
        continue;
      }
      const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
#pragma unroll
      for (int c = 0; c < 16; c += 2) {
        if (c0 + 4 * c >= a.D) break;
        const uint4 w = make_uint4(pack16<kBf16>(acc[c].x * inv, acc[c].y * inv), pack16<kBf16>(acc[c].z * inv, acc[c].w * inv),
                                   pack16<kBf16>(acc[c + 1].x * inv, acc[c + 1].y * inv),
                                   pack16<kBf16>(acc[c + 1].z * inv, acc[c + 1].w * inv));
        uint16_t* to = out + c0 + 4 * c;
        if (a.o_vec) {
          *reinterpret_cast<uint4*>(to) = w;
        } else {
          const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            to[2 * e] = (uint16_t)x[e];
            to[2 * e + 1] = (uint16_t)(x[e] >> 16);
          }
        }
      }
    }
    if (!last)
      a.part_ml[slot(0) * a.tile_rows + row] = make_float2(top, sum);
    else if (a.lse)
      a.lse[r * (a.H * a.G) + hq] =
          sum == 0.f ? -INFINITY : (top - weight_bias<kBf16>()) * 0.693147180559945f + logf(sum);
  }
  __syncwarp();
}

// A pair of more than kAlone pieces is joined in two steps, groups of kGroup pieces first: the last
// warp of a group joins the group, the last of those the groups.
constexpr int kAlone = 6, kGroup = 5;

// The pairs (tile, head) of a CTA's share, one after the other.
struct Pairs {
  long long w, end;
  int share, lead;
  AttnTile t;
  int tile, head, u0, u1;
  // (no pairs where the step is not one that this call may work on)
  __device__ __forceinline__ void init(const AttnArgs& a) {
    const StepHead step = load_words(a.head);
    const CtaWork x = load_words(&a.work[blockIdx.x]);
    w = x.begin;
    end = step_fits(step, ATTN_TC, a.num_tokens) ? x.end : x.begin;
    share = x.share;
    lead = x.lead;
    t = x.t;
    tile = x.tile;
  }
  __device__ __forceinline__ bool next(const AttnArgs& a) {
    while (w < end) {
      if (w >= t.before + (long long)stretch_of(t.units, lead, share) * a.H) t = load_words(&a.tiles[++tile]);
      const int len = stretch_of(t.units, lead, share);
      const long long off = w - t.before;
      head = (int)(off / len);
      const int o0 = (int)(off - (long long)head * len), o1 = (int)min((long long)len, o0 + (end - w));
      w += o1 - o0;
      const int2 u = units_of(o0, o1, t.units, lead);
      u0 = u.x;
      u1 = u.y;
      if (u1 > u0) return true;
    }
    return false;
  }
  __device__ __forceinline__ int key_of(int u) const {
    return (u < t.sink_units ? u : t.win_unit + u - t.sink_units) * kKeys;
  }
  // keys of unit u that no row of the tile sees
  __device__ __forceinline__ bool hidden(int key, int sinks) const {
    return key >= t.kv_hi || (key < t.kv_lo && key >= sinks);
  }
  __device__ __forceinline__ bool ragged(int u, int sinks) const {
    const int key0 = key_of(u);
    return key0 + kKeys > t.kv_hi || (key0 < t.kv_lo && key0 + kKeys > sinks);
  }
};

// The n lowest bits, all of them from 32 on, none below 1.
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }

__device__ __forceinline__ void store32(void* p, const uint32_t* w) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]),
               "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}
// Two 32-byte halves of each lane's row to halves of the rows of its pair of lanes: an even lane has the
// first half of either row afterwards (the even lane's row in w[0..8)), an odd one the second, so that a
// store of one half a lane covers 64 consecutive bytes of sixteen rows.  (8 prompts of 4096: 715 us, with
// four 16-byte pieces passed round among four lanes 721.  With each lane storing its own row, a store
// touched 32 lines.)
__device__ __forceinline__ void rows_to_halves(uint32_t (&w)[16], int lane) {
  const bool odd = lane & 1;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    uint32_t &lo = w[e], &hi = w[8 + e];
    const uint32_t got = __shfl_xor_sync(0xffffffffu, odd ? lo : hi, 1);
    if (odd) lo = got;
    else hi = got;
  }
}

// Weights of N keys, s[0..N) scaled by c and moved by b, in 16 bits; returns their sum.
template <int N, bool kBf16>
__device__ __forceinline__ float weights(const float* s, float c, float b, uint32_t* w) {
  const float2 c2 = make_float2(c, c), b2 = make_float2(b, b);
  float2 acc0 = make_float2(0.f, 0.f), acc1 = acc0;
#pragma unroll
  for (int j = 0; j < N / 2; ++j) {
    float2 y = fma2(make_float2(s[2 * j], s[2 * j + 1]), c2, b2);
    y.x = exp2_fast(y.x);
    y.y = exp2_fast(y.y);
    if (j & 1) acc1 = add2(acc1, y);
    else acc0 = add2(acc0, y);
    w[j] = pack16<kBf16>(y.x, y.y);
  }
  acc0 = add2(acc0, acc1);
  return acc0.x + acc0.y;
}

__device__ __forceinline__ float max128(const float* s) {
  float m0 = fmaxf(s[0], s[1]), m1 = fmaxf(s[2], s[3]);
#pragma unroll
  for (int i = 4; i < 128; i += 4) {
    m0 = fmaxf(fmaxf(m0, s[i]), s[i + 1]);
    m1 = fmaxf(fmaxf(m1, s[i + 2]), s[i + 3]);
  }
  return fmaxf(m0, m1);
}

// One unit's weights of one half of a tile: a thread a row.  S is read from TMEM, and the weights
// replace it there in 16 bits, two to a column, as the left operand of the product with V, which
// starts on the first 64 keys while the others' weights are computed, and on the next 32 (prompts 798 us
// with 96 and 32 keys, 754 with three pieces).  The first are taken
// against the maximum so far, beside the search for this unit's; only where that shows a row to
// have outgrown it are they taken again (and in a pair's first unit).
constexpr int kFirst = 64;
template <int DP, bool kBf16>
struct Softmax {
  float top = -INFINITY, b = weight_bias<kBf16>(), sum = 0.f;      // of the raw scores; what is added to scaled ones; of the weights
  __device__ __forceinline__ void step(const AttnArgs& a, uint32_t s_at, uint32_t o_at, bool fresh, bool open, int key0,
                                       int pos, uint64_t* ready) {
    const float c = a.scale;
    uint32_t x[128];
    float* s = reinterpret_cast<float*>(x);
#pragma unroll
    for (int i = 0; i < 4; ++i) tc_ld32(x + 32 * i, s_at + 32 * i);
    tc_wait_ld();
    tc_loaded<128>(x);
    if (!open) {
      // keys key0 + i: seen up to pos, from the window's start or among the sinks
      const int upto = pos + 1 - key0, before = a.window > 0 ? upto - a.window : 0, sinks = a.sinks - key0;
#pragma unroll
      for (int i = 0; i < 128; i += 32) {
        const uint32_t m = low_bits(upto - i) & (~low_bits(before - i) | low_bits(sinks - i));
#pragma unroll
        for (int j = 0; j < 32; ++j) s[i + j] = m >> j & 1u ? s[i + j] : -INFINITY;
      }
    }
    // (one copy of the first weights' code: a second one for the second take, seldom run, was
    // fetched anew in every pair)
    uint32_t w[kFirst / 2];
    float part, high = -INFINITY;
    if (fresh) high = max128(s);
#pragma unroll 1
    for (bool again = fresh;; again = true) {
      if (again) {
        const float f = high == top ? 1.f : exp2_fast((top - high) * c);
        top = high;
        sum *= f;
        if (!fresh) {
          // S of this unit follows the previous unit's product with V: O is at rest
#pragma unroll 1
          for (int i = 0; i < DP; i += 32) {
            uint32_t o[32];
            tc_ld32(o, o_at + i);
            tc_wait_ld();
            tc_loaded<32>(o);
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
            tc_st32(o_at + i, o);
          }
        }
        if (top != -INFINITY) b = weight_bias<kBf16>() - top * c;
      }
      part = weights<kFirst, kBf16>(s, c, b, w);
      high = fmaxf(max128(s), top);
      if (!__any_sync(0xffffffffu, !again && (high - top) * c > kLazy)) break;      // (yes from -inf; no from there to there)
    }
    tc_st32(s_at, w);
    tc_wait_st();
    tc_fence_before();
    warp_arrive(ready);
    part += weights<32, kBf16>(s + 64, c, b, w);
    tc_st16(s_at + 32, w);
    tc_wait_st();
    tc_fence_before();
    warp_arrive(ready + 1);
    sum += part + weights<32, kBf16>(s + 96, c, b, w);
    tc_st16(s_at + 48, w);
    tc_wait_st();
  }
};

// o = sum_j w_j v_j / sum_j w_j with w_j = 2^(c q.k_j - m), c = scale log2(e), m the maximum so far (raised only
// when a row outgrows it by 2^kLazy), over units of 128 keys; pieces of a cut pair join as in the
// kernel for few rows.
// What bounds it: in a long context the tensor core and the softmax that feeds it.  A unit of both halves
// is 2048 cycles of products at the tensor core's rate and took 2850: a half's chain of products (some 1400) and
// softmax (1500) is as long as both halves' products, which hides in two halves' turns but for the waits.  500 tokens at 64 000
// keys, 32 query heads of 128: 334 to 353 us over boxes, 1.49 to 1.57 PFLOP/s (the pipe is active 74 % of the
// time); 8 prompts of 4096 from nothing 715 to 727 us, 1.54; 5 chunks of 1500 to 2100 under a window of 1024
// 145 us, 0.9.  These are launches in a graph after a pause; calls one after another take 388, 780 and 150.
// Of a pair's time some 6000 cycles lie between its last weights and the next pair's first, some 3000 more
// than between units.  Under a steady load the power limit lowers the clock, and all of this by 3 to 8 %.
//
// One CTA an SM: its share of the line of units.  A tile is two halves of half_rows packed rows
// (whole tokens; an M = 128 tile of the tensor core each) that take turns: while one half's weights are
// computed, the tensor core runs the other half's products.
//   8, 9     K and V units into a ring of shared memory, by TMA: a box a page and 64 columns;
//            what the table has no page for reads as zeros
//   warp 10  S = Q K^T (tcgen05, operands in shared memory), O += P V (P in TMEM)
//   warp 11  queries, and zeros in the rows of V units that no row of the tile sees
//   0 .. 7   softmax, a thread a row, and the pair's end: O / sum, or the sums of a cut pair
template <int DP, bool kBf16>
__global__ void __launch_bounds__(kThreads, 1)
k_attend_tc(const __grid_constant__ AttnArgs a, const __grid_constant__ CUtensorMap kmap,
            const __grid_constant__ CUtensorMap vmap, const __grid_constant__ CUtensorMap qmap, int box_rows,
            int half_rows, int q_tma) {
  using S = TcShape<DP>;
  extern __shared__ __align__(1024) unsigned char dyn[];
  Bars& bars = *reinterpret_cast<Bars*>(dyn + S::kData);
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const uint32_t q_s = smem_u32(dyn), ring_s = q_s + 2 * S::kBlock;
  if (q_s & 1023u) {      // (the swizzle's pattern starts at multiples of 1024 bytes)
    if (threadIdx.x == 0) report(a.ctl, LV_ERR_CUDA, blockIdx.x);
    return;
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < S::kStages; ++i) {
      bar_init(&bars.kv_full[i], arrivals_of(a, LV_HOLD_COPIES));
      bar_init(&bars.kv_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      bar_init(&bars.q_full[i], 1);
      bar_init(&bars.q_empty[i], 1);
      bar_init(&bars.s_full[i], 1);
      for (int k = 0; k < 3; ++k) bar_init(&bars.p_full[i][k], 4);
      bar_init(&bars.o_full[i], arrivals_of(a, LV_HOLD_PRODUCTS));
    }
    bar_init(&bars.clean_ask, 1);
    bar_init(&bars.clean_done, 32);
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
    const int half = wid >> 2, row = threadIdx.x & 127;                   // of the half
    const uint32_t lanes = tmem + ((uint32_t)(wid & 3) << 21);            // this warp's 32 lanes of TMEM
    const uint32_t s_at = lanes + 128 * half, o_at = lanes + S::kColO + DP * half;
    uint32_t s_par = 0, o_par = 0;
    Pairs pr;
    pr.init(a);
    bool ok = true;
    Pairs nx = pr;
    bool has = nx.next(a);
    while (ok && has) {
      pr = nx;
      const int rows = min(half_rows, pr.t.rows - half * half_rows);
      if (rows <= 0) {                                      // nothing in this half
        has = nx.next(a);
        continue;
      }
      const bool live = rows > (row & ~31);                 // rows in this warp
      const int R0 = pr.t.row0 + half * half_rows;
      const int R = R0 + min(row, rows - 1), token = R / a.G;
      const int pos = pr.t.first + token;
      const int p_lo = pr.t.first + R0 / a.G, p_hi = pr.t.first + (R0 + rows - 1) / a.G;
      Softmax<DP, kBf16> sm;
      for (int u = pr.u0; u < pr.u1; ++u) {
        if (!(ok = bar_wait(&bars, &bars.s_full[half], s_par, a.wait_ns))) break;
        s_par ^= 1;
        if (live) {
          tc_fence_after();
          const int key0 = pr.key_of(u);
          const bool open =
              key0 + kKeys - 1 <= p_lo && (a.window == 0 || key0 > p_hi - a.window || key0 + kKeys <= a.sinks);
          sm.step(a, s_at, o_at, u == pr.u0, open, key0, pos, &bars.p_full[half][0]);
          tc_fence_before();
        } else {
          warp_arrive(&bars.p_full[half][0]);
          warp_arrive(&bars.p_full[half][1]);
        }
        warp_arrive(&bars.p_full[half][2]);
      }
      has = nx.next(a);
      if (!ok || !(ok = bar_wait(&bars, &bars.o_full[half], o_par, a.wait_ns))) break;
      o_par ^= 1;
      if (!live) continue;
      // the pair's end
      tc_fence_after();
      const bool whole = pr.u0 == 0 && pr.u1 == pr.t.units;
      const int hq = pr.head * a.G + (R - token * a.G);
      const int64_t r = pr.t.qrow + token;
      const bool mine = row < rows;
      const float inv = !whole ? 1.f : sm.sum > 0.f || sm.sum != sm.sum ? 1.f / sm.sum : 0.f;
      const int64_t slot = part_slot(blockIdx.x, pr.u0 == 0);
      const int t_row = half * half_rows + row;
      uint16_t* out = reinterpret_cast<uint16_t*>(a.out) + r * a.o_row + hq * a.o_head;
      // the rows of this lane's pair, null where there is none
      uint16_t* to[2];
#pragma unroll
      for (int t = 0; t < 2; ++t)
        to[t] = reinterpret_cast<uint16_t*>(
                    __shfl_sync(0xffffffffu, mine ? reinterpret_cast<uint64_t>(out) : 0ull, (lane & 30) + t));
      const int side = 16 * (lane & 1);
#pragma unroll 1
      for (int col = 0; col < DP; col += 32) {
        uint32_t o[32];
        tc_ld32(o, o_at + col);
        tc_wait_ld();
        tc_loaded<32>(o);
        uint32_t w[16];
        if (whole) {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            w[e] = pack16<kBf16>(__uint_as_float(o[2 * e]) * inv, __uint_as_float(o[2 * e + 1]) * inv);
          if (a.o_vec) {
            rows_to_halves(w, lane);
#pragma unroll
            for (int t = 0; t < 2; ++t)
              if (to[t] && col + side < a.D) {
                uint16_t* at = to[t] + col + side;
                if (a.o_vec == 2) {
                  store32(at, &w[8 * t]);
                } else {
                  *reinterpret_cast<uint4*>(at) = make_uint4(w[8 * t], w[8 * t + 1], w[8 * t + 2], w[8 * t + 3]);
                  if (col + side + 8 < a.D)
                    *reinterpret_cast<uint4*>(at + 8) = make_uint4(w[8 * t + 4], w[8 * t + 5], w[8 * t + 6], w[8 * t + 7]);
                }
              }
          } else if (mine) {
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (col + 2 * e < a.D) {
                out[col + 2 * e] = (uint16_t)w[e];
                out[col + 2 * e + 1] = (uint16_t)(w[e] >> 16);
              }
          }
        } else if (mine) {
          float4* po = part_at<DP>(a, slot, col, t_row);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            po[e * a.tile_rows] = make_float4(__uint_as_float(o[4 * e]), __uint_as_float(o[4 * e + 1]),
                                              __uint_as_float(o[4 * e + 2]), __uint_as_float(o[4 * e + 3]));
        }
        __syncwarp();
      }
      const float top2 = sm.top * a.scale;      // in log2
      if (!whole) {
        if (mine) a.part_ml[slot * a.tile_rows + t_row] = make_float2(top2, sm.sum);
        // (a warp writes, counts and joins its own 32 rows of the pair's pieces)
        const Pieces ps = pieces_of(pr.t, pr.head, pr.lead, pr.share);
        // true when `count` warps have come to set `set` of piece `of`, this one last
        auto last = [&](int of, int count, int set) {
          __syncwarp();
          int was = 0;
          if (lane == 0) {
            int32_t* at = &a.arrived[(ps.first + of) * kArriveWords + set * kArriveSet + wid];
            was = add_release(at, 1);
            if (was == count - 1) *at = 0;
          }
          was = __shfl_sync(0xffffffffu, was, 0);
          if (was != count - 1) return false;
          __threadfence();
          return true;
        };
        if (ps.count <= kAlone) {
          if (last(0, ps.count, 0))
            join_rows<DP, kBf16>(a, ps.first, 0, 1, ps.count, true, t_row, mine, out, r, hq);
        } else {
          const int g0 = (int)(blockIdx.x - ps.first) / kGroup * kGroup, n = min(kGroup, ps.count - g0);
          const int groups = (ps.count + kGroup - 1) / kGroup;
          if (last(g0, n, g0 ? 2 : 1)) {
#pragma unroll 1
            for (int step = 0; step < 2; ++step) {
              join_rows<DP, kBf16>(a, ps.first, step ? 0 : g0, step ? kGroup : 1, step ? groups : n, step == 1, t_row, mine,
                                   out, r, hq);
              if (step || !last(0, groups, 0)) break;
            }
          }
        }
      } else if (mine && a.lse) {
        a.lse[r * (a.H * a.G) + hq] =
            sm.sum == 0.f ? -INFINITY : (top2 - weight_bias<kBf16>()) * 0.693147180559945f + logf(sm.sum);
      }
      __syncwarp();
    }
    tc_fence_before();
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
    Pairs pr;
    pr.init(a);
    if (wid == kWarpK || wid == kWarpV) {
      // ---- K (or V): lane i finds the page of a unit's box of box_rows keys; one thread then
      // issues the copies.  (With each lane issuing its own, a unit's 16 took 1300 cycles.)
      const int kv = wid == kWarpV;
      const CUtensorMap* map = kv ? &vmap : &kmap;
      const int boxes = kKeys / box_rows;
      long long unit = 0;
      bool ok = true;
      auto page_of = [&](int u) {
        const int key = pr.key_of(u) + lane * box_rows;
        if (lane >= boxes || u >= pr.u1 || key >= pr.t.kv_hi || (key + box_rows <= pr.t.kv_lo && key >= a.sinks)) return -1;
        return a.tables[(size_t)pr.t.req * a.maxB + key / a.T];
      };
      while (ok && pr.next(a)) {
        int next = page_of(pr.u0);
        for (int u = pr.u0; ok && u < pr.u1; ++u, ++unit) {
          // no page: a box outside the array, which reads as zeros
          const int page = (uint32_t)next < a.hbm_pages ? next : (int)a.hbm_pages;
          const int off = (pr.key_of(u) + lane * box_rows) % a.T;
          next = page_of(u + 1);
          const int n = (int)((2 * unit + kv) % S::kStages);
          const uint32_t round = (uint32_t)((2 * unit + kv) / S::kStages);
          if (!(ok = bar_wait(&bars, &bars.kv_empty[n], ~round & 1u, a.wait_ns))) break;
          uint64_t* full = &bars.kv_full[n];
          const uint32_t dst = ring_s + n * S::kBlock;
          if (elected()) bar_expect(full, S::kBlock);
#pragma unroll 1
          for (int i = 0; i < boxes; i += 4) {
            int pages[4], offs[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              pages[e] = __shfl_sync(0xffffffffu, page, (i + e) & 31);
              offs[e] = __shfl_sync(0xffffffffu, off, (i + e) & 31);
            }
            if (elected()) {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                if (i + e >= boxes) break;
#pragma unroll
                for (int x = 0; x < S::kHalves; ++x)
                  tma_box(dst + x * kKeys * 128 + (i + e) * box_rows * 128, map, 64 * x, pr.head, offs[e], pages[e], full);
              }
            }
            __syncwarp();
          }
        }
      }
      if (!ok) {      // let what is on its way land before the shared memory is given up
        for (long long i = unit < S::kStages ? 0 : unit - S::kStages; i < unit; ++i) {
          const unsigned long long t0 = now_ns();
          while (!bar_try(&bars.kv_full[(2 * i + kv) % S::kStages], (uint32_t)((2 * i + kv) / S::kStages) & 1u))
            if ((long long)(now_ns() - t0) > a.wait_ns) break;
        }
      }
    } else if (wid == kWarpMma) {
      // ---- products, by one thread (a warp that votes at each wait took some 200 cycles for it)
      if (elected()) {
        constexpr uint32_t kDescS = mma_desc<kBf16>(128, kKeys, false), kDescO = mma_desc<kBf16>(128, DP, true);
        const uint32_t kd0 = desc_low(ring_s, 16), vd0 = desc_low(ring_s, kKeys * 128), qd0 = desc_low(q_s, 16);
        uint32_t par = 0, p_par = 0, q_par = 0, clean_par = 0;      // (the last three: a bit a half)
        int stage = 0;
        auto step = [&]() {
          if (++stage == S::kStages) {
            stage = 0;
            par ^= 1;
          }
        };
        auto scores = [&](int half, int st) {      // S_half = Q_half K^T
          const uint32_t qd = qd0 + half * (S::kBlock >> 4), kd = kd0 + st * (S::kBlock >> 4);
#pragma unroll
          for (int k = 0; k < DP / 16; ++k) {
            const uint32_t at = ((k / 4) * (kKeys * 128) + (k % 4) * 32) >> 4;
            tc_mma_ss(tmem + 128 * half, qd + at, kd + at, kDescS, k > 0);
          }
          tc_commit(&bars.s_full[half]);
        };
        // O_half (+)= P_half V, steps of 16 keys from k0 to k1
        auto values = [&](int half, int st, int k0, int k1, bool add) {
          const uint32_t vd = vd0 + st * (S::kBlock >> 4);
#pragma unroll
          for (int k = k0; k < k1; ++k)
            tc_mma_ts(tmem + S::kColO + DP * half, tmem + 128 * half + 8 * k, vd + k * (2048 >> 4), kDescO, add || k > k0);
        };
        // a pair's units; false when a wait ran out.  nx: the pair after it, found meanwhile
        Pairs nx = pr;
        bool has = nx.next(a);
        auto pair = [&](auto halves_of) -> bool {
          constexpr int kHalves = decltype(halves_of)::value;
          pr = nx;
          if (!bar_wait1(&bars, &bars.kv_full[stage], par, a.wait_ns)) return false;
#pragma unroll
          for (int h = 0; h < kHalves; ++h) {      // the first unit's scores
            if (!bar_wait1(&bars, &bars.q_full[h], q_par >> h & 1, a.wait_ns)) return false;
            q_par ^= 1u << h;
            tc_fence_after();
            scores(h, stage);
            if (pr.u1 - pr.u0 == 1) tc_commit(&bars.q_empty[h]);
          }
          tc_commit(&bars.kv_empty[stage]);
          step();
          has = nx.next(a);
#pragma unroll 1
          for (int u = pr.u0; u < pr.u1; ++u) {
            const int vs = stage;
            const bool ragged = pr.ragged(u, a.sinks), more = u + 1 < pr.u1;
            if (LV_RARE(!bar_wait1(&bars, &bars.kv_full[vs], par, a.wait_ns))) return false;
            step();
            if (LV_RARE(ragged)) bar_arrive(&bars.clean_ask);
            const int ks = stage;
            if (LV_MOSTLY(more)) {
              if (LV_RARE(!bar_wait1(&bars, &bars.kv_full[ks], par, a.wait_ns))) return false;
            }
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
              if (LV_RARE(!bar_wait1(&bars, &bars.p_full[h][0], p_par >> h & 1, a.wait_ns))) return false;
              if (h == 0 && LV_RARE(ragged)) {
                if (!bar_wait1(&bars, &bars.clean_done, clean_par, a.wait_ns)) return false;
                clean_par ^= 1;
              }
              tc_fence_after();
              values(h, vs, 0, 4, u > pr.u0);
              if (LV_RARE(!bar_wait1(&bars, &bars.p_full[h][1], p_par >> h & 1, a.wait_ns))) return false;
              tc_fence_after();
              values(h, vs, 4, 6, true);
              if (LV_RARE(!bar_wait1(&bars, &bars.p_full[h][2], p_par >> h & 1, a.wait_ns))) return false;
              tc_fence_after();
              values(h, vs, 6, 8, true);
              if (LV_MOSTLY(more)) {
                scores(h, ks);
                if (LV_RARE(u + 2 == pr.u1)) tc_commit(&bars.q_empty[h]);
              } else {
                tc_commit(&bars.o_full[h]);
              }
            }
            p_par ^= kHalves == 2 ? 3u : 1u;
            tc_commit(&bars.kv_empty[vs]);
            if (LV_MOSTLY(more)) {
              tc_commit(&bars.kv_empty[ks]);
              step();
            }
          }
          return true;
        };
        bool ok = true;
        while (ok && has)
          ok = nx.t.rows > half_rows ? pair(std::integral_constant<int, 2>()) : pair(std::integral_constant<int, 1>());
        if (!ok) {      // let the products under way end
          tc_commit(&bars.drain);
          const unsigned long long t0 = now_ns();
          while (!bar_try(&bars.drain, 0))
            if ((long long)(now_ns() - t0) > a.wait_ns) break;
        }
      }
      __syncwarp();
    } else {
      // ---- queries of each pair, when the S of the pair before it has been computed; and zeros
      // in the rows of V that no row of the tile sees, which hold whatever the page does (a weight
      // of zero does not cancel a NaN): the products ask for each such unit, in order
      uint32_t par = 0;      // a bit a half
      uint32_t z_par = 0;
      long long units = 0;
      bool ok = true;
      while (ok && pr.next(a)) {
        for (int half = 0; half < 2; ++half) {
          const int rows = min(half_rows, pr.t.rows - half * half_rows);
          if (rows <= 0) break;
          if (!(ok = bar_wait(&bars, &bars.q_empty[half], ~par >> half & 1, a.wait_ns))) break;
          par ^= 1u << half;
          const uint32_t to = q_s + half * S::kBlock;
          const int R0 = pr.t.row0 + half * half_rows;
          if (q_tma) {
            if (elected()) {
              bar_expect(&bars.q_full[half], half_rows * 128 * S::kHalves);
#pragma unroll
              for (int x = 0; x < S::kHalves; ++x)
                tma_box(to + x * kKeys * 128, &qmap, 64 * x, 0, pr.head, pr.t.qrow + R0 / a.G, &bars.q_full[half]);
            }
            __syncwarp();
          } else {
            // lane i finds rows i, 32 + i, ...; a step copies kStep rows, kChunks lanes a row
            constexpr int kChunks = DP / 8, kStep = 32 / kChunks;
            const int c = lane % kChunks, sub = lane / kChunks;
            const bool col = c * 8 < a.D;
            for (int r0 = 0; r0 < rows; r0 += 32) {
              const int R = R0 + min(r0 + lane, rows - 1), token = R / a.G;
              const int64_t at =
                  (pr.t.qrow + token) * a.q_row + (int64_t)(pr.head * a.G + (R - token * a.G)) * a.q_head;
#pragma unroll 4
              for (int i = 0; i < 32 / kStep; ++i) {
                const int row = r0 + kStep * i + sub;
                const uint16_t* src =
                    reinterpret_cast<const uint16_t*>(a.q) + __shfl_sync(0xffffffffu, at, kStep * i + sub) + c * 8;
                uint32_t w[4] = {0, 0, 0, 0};
                if (col) {
#pragma unroll
                  for (int e = 0; e < 4; ++e) w[e] = (uint32_t)src[2 * e] | (uint32_t)src[2 * e + 1] << 16;
                }
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + (c / 8) * (kKeys * 128) + row * 128 +
                                                                             (((c % 8) ^ (row & 7)) << 4)),
                             "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3])
                             : "memory");
              }
            }
            fence_async();
            __syncwarp();
            if (elected()) bar_arrive(&bars.q_full[half]);
            __syncwarp();
          }
        }
        for (int u = pr.u0; ok && u < pr.u1; ++u, ++units) {
          if (!pr.ragged(u, a.sinks)) continue;
          if (!(ok = bar_wait(&bars, &bars.clean_ask, z_par, a.wait_ns))) break;
          z_par ^= 1;
          const uint32_t v = ring_s + (uint32_t)((2 * units + 1) % S::kStages) * S::kBlock;
          const int key0 = pr.key_of(u);
          for (int i = lane; i < kKeys * 8; i += 32) {
            if (!pr.hidden(key0 + i / 8, a.sinks)) continue;
#pragma unroll
            for (int x = 0; x < S::kHalves; ++x)
              asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(v + x * kKeys * 128 + i * 16), "r"(0)
                           : "memory");
          }
          fence_async();
          bar_arrive(&bars.clean_done);
        }
      }
      if (!ok && q_tma) {      // as above: the last queries asked for
        for (int half = 0; half < 2; ++half) {
          const unsigned long long t0 = now_ns();
          while (!bar_try(&bars.q_full[half], ~par >> half & 1))
            if ((long long)(now_ns() - t0) > a.wait_ns) break;
        }
      }
      // rows of no request
      const StepHead step = load_words(a.head);
      const bool fits = step_fits(step, ATTN_TC, a.num_tokens);
      if (LV_RARE(!fits) && blockIdx.x == 0 && lane == 0) report(a.ctl, LV_ERR_STATE, -1);
      if (ok && fits && step.live < a.num_tokens) {
        const int Hq = a.H * a.G;
        for (int r = blockIdx.x; r < a.num_tokens; r += gridDim.x) {
          if (r < step.num_tokens && a.positions[r] >= 0) continue;
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
  // (whichever role's wait it was: the products' thread may have ended well before)
  if (threadIdx.x == 0 && LV_RARE(bars.bad)) give_up(a);
  if (wid == kWarpMma) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

template <int DP, bool kBf16>
cudaError_t run(const AttnArgs& a, const TcMaps& m, int ctas, cudaStream_t s) {
  static const CUtensorMap none{};
  return launch_dependent(k_attend_tc<DP, kBf16>, dim3(ctas), kThreads, TcShape<DP>::kSmem, s, a, *m.k, *m.v,
                          m.q ? *m.q : none, m.box_rows, a.tile_rows / 2, m.q ? 1 : 0);
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

cudaError_t launch_attend_tc(const AttnArgs& a, const TcMaps& m, bool bf16, int ctas, cudaStream_t s) {
  if (a.dp == 64) return bf16 ? run<64, true>(a, m, ctas, s) : run<64, false>(a, m, ctas, s);
  return bf16 ? run<128, true>(a, m, ctas, s) : run<128, false>(a, m, ctas, s);
}

}  // namespace lv
