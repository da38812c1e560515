// Attention of requests with few rows (single tokens of a reply, drafts to verify) over the
// paged context (see lv_batch.cuh for how the work is cut).
#include "lv_batch.cuh"

namespace lv {

namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kU = kRowsUnit;

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// 16 bytes to shared memory, zeros where ok is false (nothing is read then).
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool ok) {
  const int n = ok ? 16 : 0;
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done)
      : "r"(bar), "r"(parity)
      : "memory");
  return done != 0;
}
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
__device__ __forceinline__ void tma_box(uint32_t dst, const CUtensorMap* map, int x, int head, int row, int page,
                                        uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::
          "r"(dst),
      "l"(map), "r"(bar), "r"(x), "r"(head), "r"(row), "r"(page)
      : "memory");
}
__device__ __forceinline__ unsigned long long now_ns() {
  unsigned long long t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
template <bool kBf16>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (kBf16)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Rows of no request: out = 0, lse = -inf.  Thread i of `of` threads.
__device__ __forceinline__ void clear_dead(const AttnArgs& a, int i, int of) {
  const int Hq = a.H * a.G, planned = a.head->num_tokens;
  for (int r = i >> 5; r < a.num_tokens; r += of >> 5) {
    if (r < planned && a.positions[r] >= 0) continue;
    for (int h = 0; h < Hq; ++h) {
      uint16_t* o = reinterpret_cast<uint16_t*>(a.out) + r * a.o_row + h * a.o_head;
      for (int d = i & 31; d < a.D; d += 32) o[d] = 0;
    }
    if (a.lse)
      for (int h = i & 31; h < Hq; h += 32) a.lse[(size_t)r * Hq + h] = -INFINITY;
  }
}

// A walk over the units of a CTA's share that one warp takes: of each tile the units
// first + wid, first + wid + kWarps, ...
struct Walk {
  int64_t w, end;          // the next tile's first place; the share's end
  AttnTile t;
  int tile;
  int u, u_end;            // units of the pair, this warp's next and the CTA's end
  int u_begin;
  int32_t page, off;       // of unit u (where a unit lies in one page)
};

struct CutTile {
  AttnTile t;
  int last, pad[3];        // this CTA's was its last piece to arrive
};

template <int DP>
struct RowsShape {
  static constexpr int kStages = DP == 64 ? 4 : 2;
  static constexpr int kCtas = DP == 256 ? 1 : 3;            // in an SM: 228 KiB, 64 K registers
  static constexpr int kBlocks = DP / 64;                    // of 64 columns, 128 bytes
  static constexpr int kTile = kU * DP * 2;                  // bytes of a unit's K (or V) in a stage
  static constexpr int kRing = kStages * 2 * kTile;          // of a warp
  static constexpr int kJoin = kRowsRows * (DP * 4 + 8);     // what a warp hands over: sums; maxima and weights
  static constexpr int kBars = 8 * kWarps * kStages + 2 * (int)sizeof(CutTile);      // a barrier a stage and warp
  static constexpr int kSmem = kWarps * kRing + kJoin + kBars;
  static_assert(kCtas * (kSmem + 1024) <= 228 * 1024, "shared memory of an SM");
};

// Pieces p0, p0 + step, ... (count of them) of a cut pair joined by a CTA, a warp a row: every piece's
// sums weighted by its maximum against the largest, in the pieces' order.  To the output, or
// (not kLast) to the first of the pieces' own slots.
template <int DP, bool kBf16, bool kLast>
__device__ __forceinline__ void join_rows(const AttnArgs& a, const AttnTile& t, int head, int64_t first, int p0,
                                          int step, int count) {
  const int lane = threadIdx.x & 31;
  constexpr int kCols = DP / 32;
  constexpr int kBatch = 8;
  for (int row = threadIdx.x >> 5; row < t.rows; row += kWarps) {
    auto at = [&](int i) {
      const int p = p0 + i * step;
      return part_slot((first + p) * a.H + head, p == 0) * kRowsRows + row;
    };
    float top = -INFINITY;
    for (int i = lane; i < count; i += 32) top = fmaxf(top, __ldcg(&a.part_ml[at(i)]).x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    float sum = 0.f, acc[kCols];
#pragma unroll
    for (int e = 0; e < kCols; ++e) acc[e] = 0.f;
    for (int i0 = 0; i0 < count; i0 += 32) {
      float f = 0.f;
      if (i0 + lane < count) {
        const float2 ml = __ldcg(&a.part_ml[at(i0 + lane)]);
        f = ml.x == top ? 1.f : exp2_fast(ml.x - top);
        sum += ml.y * f;
      }
      for (int i = i0; i < min(i0 + 32, count); i += kBatch) {
        float v[kBatch][kCols];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
          const float* o = a.part_o + at(min(i + b, count - 1)) * DP + kCols * lane;
#pragma unroll
          for (int e = 0; e < kCols; e += 2)
            *reinterpret_cast<float2*>(&v[b][e]) = __ldcg(reinterpret_cast<const float2*>(o + e));
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
          const float g = __shfl_sync(0xffffffffu, f, (i - i0 + b) & 31);
          if (i + b < count) {
#pragma unroll
            for (int e = 0; e < kCols; ++e) acc[e] += v[b][e] * g;
          }
        }
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if constexpr (!kLast) {
      float* o = a.part_o + at(0) * DP + kCols * lane;
#pragma unroll
      for (int e = 0; e < kCols; e += 2) *reinterpret_cast<float2*>(o + e) = make_float2(acc[e], acc[e + 1]);
      if (lane == 0) a.part_ml[at(0)] = make_float2(top, sum);
      continue;
    }
    const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
    const int R = t.row0 + row, token = R / a.G, g = R - token * a.G;
    const int64_t r = t.qrow + token;
    const int h = head * a.G + g;
    uint16_t* out = reinterpret_cast<uint16_t*>(a.out) + r * a.o_row + h * a.o_head + kCols * lane;
    if (kCols * lane < a.D) {
#pragma unroll
      for (int e = 0; e < kCols; e += 2) {
        const uint32_t w = pack16<kBf16>(acc[e] * inv, acc[e + 1] * inv);
        if (a.o_vec) {
          *reinterpret_cast<uint32_t*>(out + e) = w;
        } else {
          out[e] = (uint16_t)w;
          out[e + 1] = (uint16_t)(w >> 16);
        }
      }
    }
    if (a.lse && lane == 0)
      a.lse[r * (a.H * a.G) + h] =
          sum == 0.f ? -INFINITY : (top - weight_bias<kBf16>()) * 0.693147180559945f + logf(sum);
  }
}

// A pair of more than kAlone pieces is joined in two steps, groups of kGroup pieces first: the last CTA
// of a group joins the group, the last of those the groups (one CTA alone took some 25 us for the
// 114 pieces of a context of 60 000 keys).
constexpr int kAlone = 32, kGroup = 12;

// o = sum_j w_j v_j / sum_j w_j with w_j = 2^(c q.k_j - m), c = scale log2(e): over each unit of 16 keys with
// the maximum m so far, the sums rescaled when it grows; pieces with sums (O, l) and maximum m join as
// sum 2^(m_i - M) O_i / sum 2^(m_i - M) l_i.
// What bounds it: the cache's bytes (16 flops a byte with 8 heads a KV head).  61 tokens over 2 to 16 k keys
// each, 4 KV heads of 128: 0.82 GB in 139 us, 5.9 TB/s; 16 tokens over 33 to 65 k: 1.5 GB in 233 to 242 us, 6.3 to 6.5.
// Some SMs read at a rate up to 15 % below others'; twice to four times as many shares, for CTAs to even that out,
// took more for their begins and ends (64 tokens of a 4000-key window 80 us, 89 to 99).  Three CTAs of
// four warps an SM: 61 tokens 202 us with one of them, 141 with three.
//
// One CTA: its share of one KV head's line.  Its four warps take a tile's units in turn and are joined at the
// tile's end; each streams its units' K and V rows through a ring of its own, so no barrier of the
// CTA lies in the loop.  S = Q K^T (16 rows x 16 keys a step), the running maximum and sum of the
// softmax, O += P V, all in registers, by mma.sync: the rows are few, the work is reading the
// cache, and m16n8k16 wastes half its rows where a 128-row tcgen05 tile would waste 15 of 16.
//
// kTma: a unit's K and V come by TMA, a box of 16 keys and 64 columns each, where pages hold whole
// units (T a multiple of 16); else by 16-byte copies, a key at a time from its page.  In shared
// memory a unit is [64-column block][key][128 bytes], swizzled as TMA does it.
template <int DP, bool kBf16, bool kTma>
__global__ void __launch_bounds__(kThreads, RowsShape<DP>::kCtas)
k_attend_rows(const __grid_constant__ AttnArgs a, const __grid_constant__ CUtensorMap kmap,
              const __grid_constant__ CUtensorMap vmap) {
  using S = RowsShape<DP>;
  extern __shared__ __align__(1024) unsigned char dyn[];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const uint32_t ring_s = smem_u32(dyn) + wid * S::kRing;
  float* join = reinterpret_cast<float*>(dyn + kWarps * S::kRing);
  uint64_t* bars = reinterpret_cast<uint64_t*>(dyn + kWarps * S::kRing + S::kJoin);
  CutTile* cut = reinterpret_cast<CutTile*>(bars + kWarps * S::kStages);      // [2]
  const uint32_t bar_s = smem_u32(bars + wid * S::kStages);
  const uint32_t tok = (uint32_t)a.H * a.D * 2;     // bytes from a token's row to the next
  if (kTma) {
    if (lane < S::kStages)
      asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar_s + 8 * lane),
                   "r"(arrivals_of(a, LV_HOLD_COPIES))
                   : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncwarp();
  }
  dep_wait();
  dep_trigger();

  const int group = blockIdx.x / a.H, head = blockIdx.x - group * a.H;
  const CtaWork work = load_words(&a.work[group]);
  const StepHead step = load_words(a.head);
  if (LV_RARE(!step_fits(step, ATTN_ROWS, a.num_tokens))) {
    if (blockIdx.x == 0 && threadIdx.x == 0) report(a.ctl, LV_ERR_STATE, -1);
    return;
  }
  const bool dead = step.live < a.num_tokens;
  auto key_of = [&](const AttnTile& t, int u) { return (u < t.sink_units ? u : t.win_unit + u - t.sink_units) * kU; };
  auto hidden = [&](const AttnTile& t, int key) { return key >= t.kv_hi || (key < t.kv_lo && key >= a.sinks); };
  auto find_page = [&](Walk& x) {
    if (kTma && x.u < x.u_end) {
      const uint32_t key = key_of(x.t, x.u), b = a.t_shift >= 0 ? key >> a.t_shift : key / (uint32_t)a.T;
      x.page = a.tables[(size_t)x.t.req * a.maxB + b];
      x.off = key - b * a.T;
    }
  };
  auto next_pair = [&](Walk& x) -> bool {
    while (x.w < x.end) {
      const int len = stretch_of(x.t.units, work.lead, work.share);
      if (x.w >= x.t.before + len) {
        x.t = load_words(&a.tiles[++x.tile]);
        continue;
      }
      const int o0 = (int)(x.w - x.t.before), o1 = (int)min((int64_t)len, o0 + (x.end - x.w));
      x.w += o1 - o0;
      const int2 in = units_of(o0, o1, x.t.units, work.lead);
      x.u_begin = in.x;
      x.u_end = in.y;
      x.u = x.u_begin + wid;
      if (x.u_end > x.u_begin) {
        find_page(x);
        return true;
      }
    }
    return false;
  };
  Walk L;
  L.w = work.begin;
  L.end = work.end;
  L.t = work.t;
  L.tile = work.tile;
  bool more = next_pair(L);
  const bool any = more;
  Walk C = L;
  while (more && L.u >= L.u_end) more = next_pair(L);

  long long loads = 0;
  // unit L.u of L's pair into stage s
  auto load = [&](int s) {
    const uint32_t dst = ring_s + s * 2 * S::kTile;
    if constexpr (kTma) {
      const int page = (uint32_t)L.page < a.hbm_pages ? L.page : (int)a.hbm_pages;      // none: zeros
      if (elected()) {
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar_s + 8 * s), "r"(2 * S::kTile)
                     : "memory");
#pragma unroll
        for (int x = 0; x < S::kBlocks; ++x) {
          tma_box(dst + x * kU * 128, &kmap, 64 * x, head, L.off, page, bar_s + 8 * s);
          tma_box(dst + S::kTile + x * kU * 128, &vmap, 64 * x, head, L.off, page, bar_s + 8 * s);
        }
      }
      __syncwarp();
    } else {
      const int key0 = key_of(L.t, L.u);
      const uint32_t head_at = (uint32_t)head * (uint32_t)a.D * 2;
      constexpr int kChunks = DP / 8;               // 16-byte pieces of a row
#pragma unroll
      for (int n = 0; n < kU * kChunks / 32; ++n) {
        const int idx = n * 32 + lane;
        const int r = idx / kChunks, c = idx % kChunks;
        const int key = key0 + r;
        bool ok = !hidden(L.t, key) && c * 8 < a.D;
        int32_t page = -1;
        const uint32_t b = (uint32_t)key / (uint32_t)a.T;
        if (ok) page = a.tables[(size_t)L.t.req * a.maxB + b];
        ok = ok && (uint32_t)page < a.hbm_pages;
        const size_t off = ok ? (size_t)page * a.P + (size_t)(key - b * a.T) * tok + head_at + c * 16 : 0;
        const uint32_t to = dst + (c >> 3) * kU * 128 + r * 128 + (((c & 7) ^ (r & 7)) << 4);
        copy16(to, a.kv[0] + off, ok);
        copy16(to + S::kTile, a.kv[1] + off, ok);
      }
    }
    ++loads;
    L.u += kWarps;
    if (L.u < L.u_end) find_page(L);
    else
      while (more && L.u >= L.u_end) more = next_pair(L);
  };
#pragma unroll
  for (int s = 0; s < S::kStages - 1; ++s) {
    if (more) load(s);
    if (!kTma) copy_commit();
  }
  int stage = 0;
  uint32_t par = 0;
  int cuts = 0, was_first = 0, was_last = 0;      // (counts: thread 0's)
  bool bad = false;          // a wait ran out: the rest is done without copies and waits, and reported

  for (bool go = any; go; go = next_pair(C)) {
    // ---- queries of this pair's head: packed rows lane / 4 + 8 i
    int pos[2];
    uint32_t qr[DP / 16][4];
    const uint16_t* q = reinterpret_cast<const uint16_t*>(a.q);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = lane / 4 + 8 * i, R = C.t.row0 + min(row, C.t.rows - 1), token = R / a.G;
      pos[i] = C.t.first + token;
      const uint16_t* x = q + (C.t.qrow + token) * a.q_row + (int64_t)(head * a.G + (R - token * a.G)) * a.q_head;
      auto two = [&](int d) -> uint32_t {      // elements d, d + 1; zeros past the rows and columns
        if (row >= C.t.rows || d >= a.D) return 0u;
        if (a.q_vec) return *reinterpret_cast<const uint32_t*>(x + d);
        return (uint32_t)x[d] | (uint32_t)x[d + 1] << 16;
      };
#pragma unroll
      for (int k = 0; k < DP / 16; ++k) {
        qr[k][i] = two(16 * k + 2 * (lane & 3));
        qr[k][i + 2] = two(16 * k + 2 * (lane & 3) + 8);
      }
    }
    float o[DP / 8][4];
    float top[2], sum[2];      // per row: maximum in log2 (the scale folded in), the lane's weights
#pragma unroll
    for (int n = 0; n < DP / 8; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[n][e] = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) top[i] = -INFINITY, sum[i] = 0.f;
    const int p_lo = C.t.first + C.t.row0 / a.G, p_hi = C.t.kv_hi - 1;

#pragma unroll 1
    for (int u = C.u; u < C.u_end; u += kWarps) {
      const uint32_t ks = ring_s + stage * 2 * S::kTile, vs = ks + S::kTile;
      const int key0 = key_of(C.t, u);
      if constexpr (kTma) {
        {
          int s = stage + S::kStages - 1;
          if (s >= S::kStages) s -= S::kStages;
          if (more) load(s);      // (its last reads were before the end of the step before)
        }
        bool ok = bad || bar_try(bar_s + 8 * stage, par);
        if (!ok) {
          const unsigned long long t0 = now_ns();
          while (!(ok = bar_try(bar_s + 8 * stage, par)))
            if ((long long)(now_ns() - t0) > a.wait_ns) break;
        }
        bad = bad || !__all_sync(0xffffffffu, ok);
        more = more && !bad;      // (the stage's barrier is still in its old phase)
        if (key0 + kU > C.t.kv_hi || (key0 < C.t.kv_lo && key0 + kU > a.sinks)) {
          // V rows that no row sees hold whatever the page does: zeros, since a weight of zero does
          // not cancel a NaN
          for (int i = lane; i < kU * 8; i += 32)
            if (hidden(C.t, key0 + i / 8)) {
#pragma unroll
              for (int x = 0; x < S::kBlocks; ++x)
                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(vs + x * kU * 128 + i * 16), "r"(0)
                             : "memory");
            }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
        }
      } else {
        copy_wait<S::kStages - 2>();
        __syncwarp();
        int s = stage + S::kStages - 1;
        if (s >= S::kStages) s -= S::kStages;
        if (more) load(s);
        copy_commit();
      }
      if (++stage == S::kStages) {
        stage = 0;
        par ^= 1;
      }
      float s[2][4];
#pragma unroll
      for (int e = 0; e < 4; ++e) s[0][e] = s[1][e] = 0.f;
      {
        const int key = (lane & 7) + ((lane >> 4) << 3), half = (lane >> 3) & 1;
        const uint32_t row = ks + key * 128;
#pragma unroll
        for (int k = 0; k < DP / 16; ++k) {
          uint32_t b[4];
          ldsm4(b, row + (k >> 2) * kU * 128 + (((2 * (k & 3) + half) ^ (key & 7)) << 4));
          mma<kBf16>(s[0], qr[k], b[0], b[1]);
          mma<kBf16>(s[1], qr[k], b[2], b[3]);
        }
      }
      const bool open = key0 + kU - 1 <= p_lo && (a.window == 0 || key0 > p_hi - a.window || key0 + kU <= a.sinks);
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[n][e] *= a.scale;
          if (!open) {
            const int key = key0 + 8 * n + 2 * (lane & 3) + (e & 1), p = pos[e >> 1];
            const bool seen = key <= p && (a.window == 0 || key > p - a.window || key < a.sinks);
            if (!seen) s[n][e] = -INFINITY;
          }
        }
      float top_new[2];
      bool raise = false;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float x = fmaxf(fmaxf(s[0][2 * i], s[0][2 * i + 1]), fmaxf(s[1][2 * i], s[1][2 * i + 1]));
        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
        top_new[i] = fmaxf(x, top[i]);
        raise |= top_new[i] > top[i] + kLazy;      // also from -inf; not from -inf to -inf
      }
      if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float f = top_new[i] == top[i] ? 1.f : exp2_fast(top[i] - top_new[i]);
          top[i] = top_new[i];
          sum[i] *= f;
#pragma unroll
          for (int n = 0; n < DP / 8; ++n) {
            o[n][2 * i] *= f;
            o[n][2 * i + 1] *= f;
          }
        }
      }
      uint32_t pa[4];
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float at = (top[i] == -INFINITY ? 0.f : top[i]) - weight_bias<kBf16>();
          const float x = exp2_fast(s[n][2 * i] - at), y = exp2_fast(s[n][2 * i + 1] - at);
          sum[i] += x + y;
          pa[2 * n + i] = pack16<kBf16>(x, y);
        }
      {
        const int key = (lane & 7) + (((lane >> 3) & 1) << 3);
        const uint32_t row = vs + key * 128;
#pragma unroll
        for (int d = 0; d < DP / 16; ++d) {
          uint32_t b[4];
          ldsm4t(b, row + (d >> 2) * kU * 128 + (((2 * (d & 3) + (lane >> 4)) ^ (key & 7)) << 4));
          mma<kBf16>(o[2 * d], pa, b[0], b[1]);
          mma<kBf16>(o[2 * d + 1], pa, b[2], b[3]);
        }
      }
      __syncwarp();
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 1);
      sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 2);
    }
    // ---- the warps that had a unit joined, one after the other, by the first
    const int have = min(C.u_end - C.u_begin, kWarps);
#pragma unroll 1
    for (int n = 1; n < have; ++n) {
      float* box = join + lane;
      float2* ml = reinterpret_cast<float2*>(join + kRowsRows * DP) + lane / 4;
      __syncthreads();
      if (wid == n) {
#pragma unroll
        for (int d = 0; d < DP / 8; ++d)
#pragma unroll
          for (int e = 0; e < 4; ++e) box[(d * 4 + e) * 32] = o[d][e];
        if ((lane & 3) == 0) {
#pragma unroll
          for (int i = 0; i < 2; ++i) ml[8 * i] = make_float2(top[i], sum[i]);
        }
      }
      __syncthreads();
      if (wid == 0) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float2 x = ml[8 * i];
          const float t = fmaxf(top[i], x.x);
          const float f = top[i] == t ? 1.f : exp2_fast(top[i] - t), f2 = x.x == t ? 1.f : exp2_fast(x.x - t);
          top[i] = t;
          sum[i] = sum[i] * f + x.y * f2;
#pragma unroll
          for (int d = 0; d < DP / 8; ++d)
#pragma unroll
            for (int e = 2 * i; e < 2 * i + 2; ++e) o[d][e] = o[d][e] * f + box[(d * 4 + e) * 32] * f2;
        }
      }
    }
    const bool whole = C.u_begin == 0 && C.u_end == C.t.units;
    if (wid == 0) {
      const int64_t slot = part_slot(blockIdx.x, C.u_begin == 0);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int row = lane / 4 + 8 * i;
        if (row >= C.t.rows) continue;
        if (whole) {
          const int R = C.t.row0 + row, token = R / a.G, g = R - token * a.G;
          const int64_t r = C.t.qrow + token;
          const int h = head * a.G + g;
          const float inv = sum[i] > 0.f || sum[i] != sum[i] ? 1.f / sum[i] : 0.f;
          uint16_t* out = reinterpret_cast<uint16_t*>(a.out) + r * a.o_row + h * a.o_head;
#pragma unroll
          for (int d = 0; d < DP / 8; ++d) {
            const int col = 8 * d + 2 * (lane & 3);
            if (col >= a.D) break;
            const uint32_t w = pack16<kBf16>(o[d][2 * i] * inv, o[d][2 * i + 1] * inv);
            if (a.o_vec) {
              *reinterpret_cast<uint32_t*>(out + col) = w;
            } else {
              out[col] = (uint16_t)w;
              out[col + 1] = (uint16_t)(w >> 16);
            }
          }
          if (a.lse && (lane & 3) == 0)
            a.lse[r * (a.H * a.G) + h] =
                sum[i] == 0.f ? -INFINITY : (top[i] - weight_bias<kBf16>()) * 0.693147180559945f + logf(sum[i]);
        } else {
          float* po = a.part_o + (slot * kRowsRows + row) * DP;
#pragma unroll
          for (int d = 0; d < DP / 8; ++d)
            *reinterpret_cast<float2*>(po + 8 * d + 2 * (lane & 3)) = make_float2(o[d][2 * i], o[d][2 * i + 1]);
          if ((lane & 3) == 0) a.part_ml[slot * kRowsRows + row] = make_float2(top[i], sum[i]);
        }
      }
    }
    if (!whole) {
      const Pieces ps = pieces_of(C.t, 0, work.lead, work.share);
      const int n = C.w < C.end ? 0 : 1;      // a cut first tile, then the share's last
      if (wid == 0) {
        if (lane == 0) cut[n].t = C.t;
        // the other lanes' sums, then the count: it is asked for here and looked at after the share,
        // so that what it takes (some microseconds beside a cache read at full rate) is not waited for
        __syncwarp();
        if (lane == 0) {
          const int p = (int)(group - ps.first), g0 = ps.count > kAlone ? p / kGroup * kGroup : 0;
          const int set = ps.count <= kAlone ? 0 : g0 ? 2 : 1;
          const int was =
              add_release(&a.arrived[((ps.first + g0) * a.H + head) * kArriveWords + set * kArriveSet], 1);
          if (n == 0) was_first = was;
          else was_last = was;
        }
      }
      cuts |= 1 << n;
    }
  }
  if (cuts) {
    __syncthreads();
#pragma unroll 1
    for (int n = 0; n < 2; ++n) {
      if (!(cuts >> n & 1)) continue;
      const AttnTile t = cut[n].t;
      const Pieces ps = pieces_of(t, 0, work.lead, work.share);
      const int p = (int)(group - ps.first), g0 = p / kGroup * kGroup, g_count = min(kGroup, ps.count - g0);
      const bool grouped = ps.count > kAlone;
      // true in the whole CTA when its piece (or its group) was the last to arrive
      auto last = [&](int was, int of, int count, int set) {
        if (threadIdx.x == 0) {
          const bool yes = was == count - 1;
          if (yes) a.arrived[((ps.first + of) * a.H + head) * kArriveWords + set * kArriveSet] = 0;
          cut[n].last = yes;
          __threadfence();
        }
        __syncthreads();
        const bool yes = cut[n].last;
        __syncthreads();
        return yes;
      };
      const int was = n == 0 ? was_first : was_last;
      if (!grouped) {
        if (last(was, 0, ps.count, 0)) join_rows<DP, kBf16, true>(a, t, head, ps.first, 0, 1, ps.count);
        continue;
      }
      if (!last(was, g0, g_count, g0 ? 2 : 1)) continue;
      join_rows<DP, kBf16, false>(a, t, head, ps.first, g0, 1, g_count);
      const int groups = (ps.count + kGroup - 1) / kGroup;
      __syncthreads();
      int was2 = 0;
      if (threadIdx.x == 0) was2 = add_release(&a.arrived[(ps.first * a.H + head) * kArriveWords], 1);
      if (last(was2, 0, groups, 0)) join_rows<DP, kBf16, true>(a, t, head, ps.first, 0, kGroup, groups);
    }
  }
  if (!kTma) copy_wait<0>();
  if (LV_RARE(bad)) {      // let what is on its way land before the shared memory is given up
    for (long long i = loads < S::kStages ? 0 : loads - S::kStages; i < loads; ++i) {
      const unsigned long long t0 = now_ns();
      while (!bar_try(bar_s + 8 * (int)(i % S::kStages), (uint32_t)(i / S::kStages) & 1u))
        if ((long long)(now_ns() - t0) > a.wait_ns) break;
    }
    if (lane == 0) give_up(a);
  }
  if (dead) clear_dead(a, blockIdx.x * kThreads + threadIdx.x, gridDim.x * kThreads);
}

template <int DP, bool kTma>
cudaError_t set_rows() {
  for (auto k : {k_attend_rows<DP, true, kTma>, k_attend_rows<DP, false, kTma>}) {
    cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, RowsShape<DP>::kSmem);
    // (the default split leaves room for one CTA)
    if (e == cudaSuccess)
      e = cudaFuncSetAttribute(k, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

template <int DP, bool kTma>
cudaError_t run_rows(const AttnArgs& a, const CUtensorMap* k, const CUtensorMap* v, bool bf16, int ctas, cudaStream_t s) {
  static const CUtensorMap none{};
  return launch_dependent(bf16 ? k_attend_rows<DP, true, kTma> : k_attend_rows<DP, false, kTma>, dim3(ctas), kThreads,
                          RowsShape<DP>::kSmem, s, a, k ? *k : none, v ? *v : none);
}

}  // namespace

cudaError_t configure_attend() {
  for (cudaError_t e : {set_rows<64, true>(), set_rows<128, true>(), set_rows<64, false>(), set_rows<128, false>(),
                        set_rows<256, false>()})
    if (e != cudaSuccess) return e;
  return cudaSuccess;
}

// CTAs of the kernel that an SM holds
int attend_rows_ctas(int dp) { return dp == 256 ? RowsShape<256>::kCtas : RowsShape<128>::kCtas; }

cudaError_t launch_attend_rows(const AttnArgs& a, const CUtensorMap* k, const CUtensorMap* v, bool bf16, int ctas,
                               cudaStream_t s) {
  if (a.dp == 256) return run_rows<256, false>(a, k, v, bf16, ctas, s);
  if (a.dp == 64) return k ? run_rows<64, true>(a, k, v, bf16, ctas, s) : run_rows<64, false>(a, k, v, bf16, ctas, s);
  return k ? run_rows<128, true>(a, k, v, bf16, ctas, s) : run_rows<128, false>(a, k, v, bf16, ctas, s);
}

}  // namespace lv
