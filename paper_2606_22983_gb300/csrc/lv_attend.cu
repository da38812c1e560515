// Attention of requests with few rows (single tokens of a reply, drafts to verify) over the
// paged context, and the join of work that was cut (see lv_batch.cuh for the cutting).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

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
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
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
  const int Hq = a.H * a.G;
  for (int r = i >> 5; r < a.num_tokens; r += of >> 5) {
    if (a.positions[r] >= 0) continue;
    for (int h = 0; h < Hq; ++h) {
      uint16_t* o = reinterpret_cast<uint16_t*>(a.out) + r * a.o_row + h * a.o_head;
      for (int d = i & 31; d < a.D; d += 32) o[d] = 0;
    }
    if (a.lse)
      for (int h = i & 31; h < Hq; h += 32) a.lse[(size_t)r * Hq + h] = -INFINITY;
  }
}

// A walk over the units of a CTA's share that one warp takes: of each (tile, head group) the
// units first + ki, first + ki + KI, ...
struct Walk {
  long long w, end;        // the current pair's next unit after this CTA's part; the share's end
  AttnTile t;
  int tile, group;
  int u, u_end;            // units of the pair, this warp's next and the CTA's end
  int u_begin;
  int32_t page;            // of unit u (pages a multiple of the unit long)
};

template <int DP, int MT>
struct RowsShape {
  static constexpr int kM = 16 * MT;
  static constexpr int kStages = MT == 1 && DP <= 128 ? 3 : 2;
  static constexpr int kTile = kU * DP * 2;                  // bytes of a unit's K (or V) in a stage
  static constexpr int kRing = kStages * 2 * kTile;          // of a warp
  static constexpr int kRegs = MT * DP / 2 + 4 * MT;         // floats a lane hands over: sums, maxima, weights
  static constexpr bool kQInRegs = MT * DP <= 128;
  static constexpr int kQ = kQInRegs ? 0 : kM * DP * 2;      // a warp's queries
  static constexpr int kJoin = 2 * kRegs * 32 * 4;
  static constexpr int kSmem = kWarps * (kRing + kQ) + kJoin;
  static_assert(kSmem <= 227 * 1024, "shared memory of a CTA");
};

// One CTA: its share of the line of units, a warp a KV head of the group (and KI = 4 / hg warps
// a head, which take units in turn and are joined at each pair's end).  A warp streams its
// units' K and V rows through a ring of its own, so no barrier of the CTA lies in the loop.
// S = Q K^T (16 x 16 keys a step), the running maximum and sum of the softmax, O += P V, all in
// registers, by mma.sync: the rows are few, the work is reading the cache, and m16n8k16 wastes
// half its rows where a 128-row tcgen05 tile would waste 15 of 16.
template <int DP, int MT, bool kBf16>
__global__ void __launch_bounds__(kThreads) k_attend_rows(const __grid_constant__ AttnArgs a) {
  using S = RowsShape<DP, MT>;
  extern __shared__ __align__(128) unsigned char dyn[];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const int KI = kWarps / a.hg;
  const int hh = wid % a.hg, ki = wid / a.hg;
  unsigned char* ring = dyn + wid * S::kRing;
  const uint32_t ring_s = smem_u32(ring);
  unsigned char* qbuf = dyn + kWarps * S::kRing + wid * S::kQ;
  float* join = reinterpret_cast<float*>(dyn + kWarps * (S::kRing + S::kQ));
  const uint32_t tok = (uint32_t)a.H * a.D * 2;     // bytes from a token's row to the next
  const bool whole = a.T % kU == 0;                 // a unit lies in one page
  dep_wait();
  const long long units = a.head->units, share = a.head->share;

  auto key_of = [&](const AttnTile& t, int u) { return (u < t.sink_units ? u : t.win_unit + u - t.sink_units) * kU; };
  auto find_page = [&](Walk& x) {
    if (whole && x.u < x.u_end)
      x.page = a.tables[(size_t)x.t.req * a.maxB + (uint32_t)key_of(x.t, x.u) / (uint32_t)a.T];
  };
  auto enter = [&](Walk& x) -> bool {      // the pair that x.w is in; false where no unit of it is the CTA's
    const int len = x.t.units + a.lead;
    const long long off = x.w - x.t.before;
    x.group = (int)(off / len);
    const int o0 = (int)(off - (long long)x.group * len), o1 = (int)min((long long)len, o0 + (x.end - x.w));
    x.w += o1 - o0;
    x.u_begin = max(o0 - a.lead, 0);
    x.u_end = o1 - a.lead;
    x.u = x.u_begin + ki;
    find_page(x);
    return x.u_end > x.u_begin;
  };
  auto next_pair = [&](Walk& x) -> bool {
    while (x.w < x.end) {
      if (x.w >= x.t.before + (long long)(x.t.units + a.lead) * a.groups) x.t = load_tile(&a.tiles[++x.tile]);
      if (enter(x)) return true;
    }
    return false;
  };
  Walk L;
  L.w = blockIdx.x * share;
  L.end = min(units, L.w + share);
  bool any = L.w < L.end;
  if (any) {
    L.tile = a.cta_tile[blockIdx.x];
    L.t = load_tile(&a.tiles[L.tile]);
    any = enter(L) || next_pair(L);
  }
  Walk C = L;
  bool more = any;
  while (more && L.u >= L.u_end) more = next_pair(L);

  // unit L.u of L's pair into stage s
  auto load = [&](int s) {
    const int key0 = key_of(L.t, L.u);
    const uint32_t head = (uint32_t)(L.group * a.hg + hh) * (uint32_t)a.D * 2;
    constexpr int kChunks = DP / 8;               // 16-byte pieces of a row
    const uint32_t dst = ring_s + s * 2 * S::kTile;
    const uint8_t* kp = nullptr;
    const uint8_t* vp = nullptr;
    if (whole) {
      const uint32_t page = (uint32_t)L.page < a.hbm_pages ? (uint32_t)L.page : 0u;
      const size_t off = (size_t)page * a.P + (size_t)(key0 % a.T) * tok + head;
      kp = a.kv[0] + off;
      vp = a.kv[1] + off;
    }
#pragma unroll
    for (int n = 0; n < kU * kChunks / 32; ++n) {
      const int idx = n * 32 + lane;
      const int r = idx / kChunks, c = idx % kChunks;
      const int key = key0 + r;
      bool ok = key < L.t.kv_hi && (key >= L.t.kv_lo || key < a.sinks) && c * 8 < a.D;
      size_t off;
      const uint8_t *ks, *vs;
      if (whole) {
        ok = ok && (uint32_t)L.page < a.hbm_pages;
        off = (size_t)r * tok + c * 16;
        ks = kp + off;
        vs = vp + off;
      } else {
        int32_t page = -1;
        const uint32_t b = (uint32_t)key / (uint32_t)a.T;
        if (ok) page = a.tables[(size_t)L.t.req * a.maxB + b];
        ok = ok && (uint32_t)page < a.hbm_pages;
        off = ok ? (size_t)page * a.P + (size_t)(key - b * a.T) * tok + head + c * 16 : 0;
        ks = a.kv[0] + off;
        vs = a.kv[1] + off;
      }
      if (!ok) ks = a.kv[0], vs = a.kv[1];
      const uint32_t to = dst + r * DP * 2 + ((c ^ (r & 7)) << 4);
      copy16(to, ks, ok);
      copy16(to + S::kTile, vs, ok);
    }
    L.u += KI;
    if (L.u < L.u_end) find_page(L);
    else
      while (more && L.u >= L.u_end) more = next_pair(L);
  };
#pragma unroll
  for (int s = 0; s < S::kStages - 1; ++s) {
    if (more) load(s);
    copy_commit();
  }
  int stage = 0;

  for (bool go = any; go; go = next_pair(C)) {
    // ---- queries of this pair's head: packed rows lane / 4 + 8 i
    const int head = C.group * a.hg + hh;
    int pos[2 * MT];
    uint32_t qr[S::kQInRegs ? MT : 1][S::kQInRegs ? DP / 16 : 1][4];
    const uint16_t* q = reinterpret_cast<const uint16_t*>(a.q);
    auto q_at = [&](int row, int d) -> uint32_t {     // two elements, zeros past the rows and columns
      if (row >= C.t.rows || d >= a.D) return 0u;
      const int R = C.t.row0 + row, token = R / a.G, g = R - token * a.G;
      const uint16_t* x = q + (C.t.qrow + token) * a.q_row + (int64_t)(head * a.G + g) * a.q_head + d;
      if (a.q_vec) return *reinterpret_cast<const uint32_t*>(x);
      return (uint32_t)x[0] | (uint32_t)x[1] << 16;
    };
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) pos[i] = C.t.first + (C.t.row0 + min(lane / 4 + 8 * i, C.t.rows - 1)) / a.G;
    if constexpr (S::kQInRegs) {
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            qr[m][k][e] = q_at(16 * m + lane / 4 + 8 * (e & 1), 16 * k + 2 * (lane & 3) + 8 * (e >> 1));
    } else {
      __syncwarp();
      for (int i = lane; i < S::kM * DP / 2; i += 32) {
        const int row = i / (DP / 2), d = 2 * (i % (DP / 2));
        *reinterpret_cast<uint32_t*>(qbuf + row * DP * 2 + (((d >> 3) ^ (row & 7)) << 4) + (d & 7) * 2) = q_at(row, d);
      }
      __syncwarp();
    }
    float o[MT][DP / 8][4];
    float top[2 * MT], sum[2 * MT];      // per row: maximum in log2 (the scale folded in), the lane's weights
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int n = 0; n < DP / 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[m][n][e] = 0.f;
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) top[i] = -INFINITY, sum[i] = 0.f;
    const int p_lo = C.t.first + C.t.row0 / a.G, p_hi = C.t.kv_hi - 1;

#pragma unroll 1
    for (int u = C.u; u < C.u_end; u += KI) {
      copy_wait<S::kStages - 2>();
      __syncwarp();
      {
        int s = stage + S::kStages - 1;
        if (s >= S::kStages) s -= S::kStages;
        if (more) load(s);
        copy_commit();
      }
      const uint32_t ks = ring_s + stage * 2 * S::kTile, vs = ks + S::kTile;
      if (++stage == S::kStages) stage = 0;
      float s[MT][2][4];
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[m][0][e] = s[m][1][e] = 0.f;
      {
        const int key = (lane & 7) + ((lane >> 4) << 3), half = (lane >> 3) & 1;
        const uint32_t row = ks + key * DP * 2;
#pragma unroll
        for (int k = 0; k < DP / 16; ++k) {
          uint32_t b[4];
          ldsm4(b, row + (((2 * k + half) ^ (key & 7)) << 4));
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            uint32_t qa[4];
            if constexpr (S::kQInRegs) {
#pragma unroll
              for (int e = 0; e < 4; ++e) qa[e] = qr[m][k][e];
            } else {
              const int r = 16 * m + (lane & 15);
              ldsm4(qa, smem_u32(qbuf) + r * DP * 2 + (((2 * k + (lane >> 4)) ^ (r & 7)) << 4));
            }
            mma<kBf16>(s[m][0], qa, b[0], b[1]);
            mma<kBf16>(s[m][1], qa, b[2], b[3]);
          }
        }
      }
      const int key0 = key_of(C.t, u);
      const bool open = key0 + kU - 1 <= p_lo && (a.window == 0 || key0 > p_hi - a.window || key0 + kU <= a.sinks);
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[m][n][e] *= a.scale;
            if (!open) {
              const int key = key0 + 8 * n + 2 * (lane & 3) + (e & 1), p = pos[2 * m + (e >> 1)];
              const bool seen = key <= p && (a.window == 0 || key > p - a.window || key < a.sinks);
              if (!seen) s[m][n][e] = -INFINITY;
            }
          }
      float top_new[2 * MT];
      bool raise = false;
#pragma unroll
      for (int i = 0; i < 2 * MT; ++i) {
        const int m = i >> 1, e = 2 * (i & 1);
        float x = fmaxf(fmaxf(s[m][0][e], s[m][0][e + 1]), fmaxf(s[m][1][e], s[m][1][e + 1]));
        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
        top_new[i] = fmaxf(x, top[i]);
        raise |= top_new[i] > top[i] + kLazy;      // also from -inf; not from -inf to -inf
      }
      if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
        for (int i = 0; i < 2 * MT; ++i) {
          const float f = top_new[i] == top[i] ? 1.f : exp2_fast(top[i] - top_new[i]);
          top[i] = top_new[i];
          sum[i] *= f;
#pragma unroll
          for (int n = 0; n < DP / 8; ++n) {
            o[i >> 1][n][2 * (i & 1)] *= f;
            o[i >> 1][n][2 * (i & 1) + 1] *= f;
          }
        }
      }
      uint32_t pa[MT][4];
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const int i = 2 * m + hf;
            const float at = (top[i] == -INFINITY ? 0.f : top[i]) - weight_bias<kBf16>();
            const float x = exp2_fast(s[m][n][2 * hf] - at), y = exp2_fast(s[m][n][2 * hf + 1] - at);
            sum[i] += x + y;
            pa[m][2 * n + hf] = pack16<kBf16>(x, y);
          }
      {
        const int key = (lane & 7) + (((lane >> 3) & 1) << 3);
        const uint32_t row = vs + key * DP * 2;
#pragma unroll
        for (int d = 0; d < DP / 16; ++d) {
          uint32_t b[4];
          ldsm4t(b, row + (((2 * d + (lane >> 4)) ^ (key & 7)) << 4));
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            mma<kBf16>(o[m][2 * d], pa[m], b[0], b[1]);
            mma<kBf16>(o[m][2 * d + 1], pa[m], b[2], b[3]);
          }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) {
      sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 1);
      sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 2);
    }
    // ---- the warps of a head joined, pair by pair
    for (int n = KI; n > 1; n >>= 1) {
      // warps ki in [n / 2, n) hand over to ki - n / 2
      const bool give = ki >= n / 2 && ki < n;
      float* box = join + ((ki % (n / 2)) * a.hg + hh) * S::kRegs * 32 + lane;
      __syncthreads();
      if (give) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int d = 0; d < DP / 8; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) box[((m * (DP / 8) + d) * 4 + e) * 32] = o[m][d][e];
#pragma unroll
        for (int i = 0; i < 2 * MT; ++i) {
          box[(MT * DP / 2 + i) * 32] = top[i];
          box[(MT * DP / 2 + 2 * MT + i) * 32] = sum[i];
        }
      }
      __syncthreads();
      if (ki < n / 2) {
#pragma unroll
        for (int i = 0; i < 2 * MT; ++i) {
          const float t2 = box[(MT * DP / 2 + i) * 32];
          const float t = fmaxf(top[i], t2);
          const float f = top[i] == t ? 1.f : exp2_fast(top[i] - t), f2 = t2 == t ? 1.f : exp2_fast(t2 - t);
          top[i] = t;
          sum[i] = sum[i] * f + box[(MT * DP / 2 + 2 * MT + i) * 32] * f2;
#pragma unroll
          for (int d = 0; d < DP / 8; ++d)
#pragma unroll
            for (int e = 2 * (i & 1); e < 2 * (i & 1) + 2; ++e)
              o[i >> 1][d][e] = o[i >> 1][d][e] * f + box[(((i >> 1) * (DP / 8) + d) * 4 + e) * 32] * f2;
        }
      }
    }
    if (ki != 0) continue;
    const bool whole_pair = C.u_begin == 0 && C.u_end == C.t.units;
    const int64_t slot = part_slot(blockIdx.x, C.u_begin == 0) * a.hg + hh;
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) {
      const int row = lane / 4 + 8 * i;
      if (row >= C.t.rows) continue;
      if (whole_pair) {
        const int R = C.t.row0 + row, token = R / a.G, g = R - token * a.G;
        const int64_t r = C.t.qrow + token;
        const int h = head * a.G + g;
        const float inv = sum[i] > 0.f || sum[i] != sum[i] ? 1.f / sum[i] : 0.f;
        uint16_t* out = reinterpret_cast<uint16_t*>(a.out) + r * a.o_row + h * a.o_head;
#pragma unroll
        for (int d = 0; d < DP / 8; ++d) {
          const int col = 8 * d + 2 * (lane & 3);
          if (col >= a.D) break;
          const uint32_t w = pack16<kBf16>(o[i >> 1][d][2 * (i & 1)] * inv, o[i >> 1][d][2 * (i & 1) + 1] * inv);
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
        float* po = a.part_o + (slot * a.tile_rows + row) * DP;
#pragma unroll
        for (int d = 0; d < DP / 8; ++d)
          *reinterpret_cast<float2*>(po + 8 * d + 2 * (lane & 3)) =
              make_float2(o[i >> 1][d][2 * (i & 1)], o[i >> 1][d][2 * (i & 1) + 1]);
        if ((lane & 3) == 0) a.part_ml[slot * a.tile_rows + row] = make_float2(top[i], sum[i]);
      }
    }
  }
  copy_wait<0>();
  if (a.head->dead > 0) clear_dead(a, blockIdx.x * kThreads + threadIdx.x, gridDim.x * kThreads);
}

// Joins the pieces of the pair that CTA c of the attention began and did not end: its own last
// piece and the first pieces of the CTAs after it, added in their order.  A warp a row.
constexpr int kJoinThreads = 256;

template <bool kBf16>
__global__ void __launch_bounds__(kJoinThreads) k_attend_join(const __grid_constant__ AttnArgs a) {
  dep_wait();
  const long long units = a.head->units, share = a.head->share;
  const long long c = blockIdx.x, edge = (c + 1) * share;
  if (edge >= units) return;
  const AttnTile t = load_tile(&a.tiles[a.cta_tile[c + 1]]);
  const int group = (int)((edge - t.before) / (t.units + a.lead));
  const long long start = t.before + (long long)group * (t.units + a.lead) + a.lead;      // of its first unit
  if (start >= edge || start < c * share) return;
  const int pieces = (int)((start + t.units - 1) / share - c) + 1;
  const int lane = threadIdx.x & 31;
  const int rows = t.rows * a.hg;
  for (int x = blockIdx.y * (kJoinThreads / 32) + (threadIdx.x >> 5); x < rows; x += gridDim.y * (kJoinThreads / 32)) {
    const int hh = x / t.rows, row = x - hh * t.rows;
    auto at = [&](int p) { return (part_slot(c + p, p == 0) * a.hg + hh) * a.tile_rows + row; };
    float top = -INFINITY;
    for (int p = lane; p < pieces; p += 32) top = fmaxf(top, __ldcg(&a.part_ml[at(p)]).x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    float sum = 0.f;
    for (int p = lane; p < pieces; p += 32) {
      const float2 ml = __ldcg(&a.part_ml[at(p)]);
      sum += ml.x == top ? ml.y : ml.y * exp2_fast(ml.x - top);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
    const int R = t.row0 + row, token = R / a.G, g = R - token * a.G;
    const int64_t r = t.qrow + token;
    const int h = (group * a.hg + hh) * a.G + g;
    uint16_t* out = reinterpret_cast<uint16_t*>(a.out) + r * a.o_row + h * a.o_head;
    for (int d = lane * 4; d < a.D; d += 128) {
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
      for (int p = 0; p < pieces; ++p) {
        const int64_t q = at(p);
        const float m = __ldcg(&a.part_ml[q]).x;
        const float f = m == top ? 1.f : exp2_fast(m - top);
        const float4 v = __ldcg(reinterpret_cast<const float4*>(a.part_o + q * a.dp + d));
        acc.x += v.x * f;
        acc.y += v.y * f;
        acc.z += v.z * f;
        acc.w += v.w * f;
      }
      const uint2 w = make_uint2(pack16<kBf16>(acc.x * inv, acc.y * inv), pack16<kBf16>(acc.z * inv, acc.w * inv));
      if (a.o_vec) {
        *reinterpret_cast<uint2*>(out + d) = w;
      } else {
        out[d] = (uint16_t)w.x;
        out[d + 1] = (uint16_t)(w.x >> 16);
        out[d + 2] = (uint16_t)w.y;
        out[d + 3] = (uint16_t)(w.y >> 16);
      }
    }
    if (a.lse && lane == 0)
      a.lse[r * (a.H * a.G) + h] =
          sum == 0.f ? -INFINITY : (top - weight_bias<kBf16>()) * 0.693147180559945f + logf(sum);
  }
}

template <int DP, int MT>
cudaError_t set_rows() {
  for (void (*k)(AttnArgs) : {k_attend_rows<DP, MT, true>, k_attend_rows<DP, MT, false>}) {
    const cudaError_t e =
        cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, RowsShape<DP, MT>::kSmem);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

template <int DP, int MT>
cudaError_t run_rows(const AttnArgs& a, bool bf16, int ctas, cudaStream_t s) {
  return launch_dependent(bf16 ? k_attend_rows<DP, MT, true> : k_attend_rows<DP, MT, false>, dim3(ctas), kThreads,
                          RowsShape<DP, MT>::kSmem, s, a);
}

}  // namespace

cudaError_t configure_attend() {
  for (cudaError_t e : {set_rows<64, 1>(), set_rows<64, 2>(), set_rows<128, 1>(), set_rows<128, 2>(), set_rows<256, 1>()})
    if (e != cudaSuccess) return e;
  return cudaSuccess;
}

// CTAs that fit in an SM's 227 KiB of shared memory (and its registers)
int attend_rows_ctas(int dp, bool wide) {
  const int bytes = dp == 64 ? (wide ? RowsShape<64, 2>::kSmem : RowsShape<64, 1>::kSmem)
                    : dp == 128 ? (wide ? RowsShape<128, 2>::kSmem : RowsShape<128, 1>::kSmem)
                                : RowsShape<256, 1>::kSmem;
  const int fit = 227 * 1024 / (bytes + 1024);
  const int most = wide ? 2 : dp == 64 ? 4 : 2;
  return fit < 1 ? 1 : fit > most ? most : fit;
}

cudaError_t launch_attend_rows(const AttnArgs& a, bool wide, bool bf16, int ctas, cudaStream_t s) {
  if (a.dp == 64) return wide ? run_rows<64, 2>(a, bf16, ctas, s) : run_rows<64, 1>(a, bf16, ctas, s);
  if (a.dp == 128) return wide ? run_rows<128, 2>(a, bf16, ctas, s) : run_rows<128, 1>(a, bf16, ctas, s);
  return run_rows<256, 1>(a, bf16, ctas, s);
}

cudaError_t launch_attend_join(const AttnArgs& a, bool bf16, int ctas, cudaStream_t s) {
  const int rows = a.tile_rows * a.hg;
  const int y = rows / (kJoinThreads / 32) < 8 ? rows / (kJoinThreads / 32) : 8;
  return launch_dependent(bf16 ? k_attend_join<true> : k_attend_join<false>, dim3(ctas, y < 1 ? 1 : y), kJoinThreads, 0,
                          s, a);
}

}  // namespace lv
