// The plan of a serving step and the write of its K and V rows (include/lv.h, "a serving step
// on resident KV").
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "lv_batch.cuh"

namespace lv {

namespace {

constexpr int kPlanThreads = 256;
constexpr long long kManyShares = (1 << 11) - 1;   // more than there are CTAs, in 11 bits
constexpr int kMaxRequests = 4096;      // lv_batch_create's limit

// Sum over the CTA, to every thread.  ws: one word a warp; a barrier lies between its uses.
__device__ __forceinline__ long long cta_sum(long long v, long long* ws) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) ws[threadIdx.x >> 5] = v;
  __syncthreads();
  long long s = 0;
  for (int w = 0; w < kPlanThreads / 32; ++w) s += ws[w];
  return s;
}

// Exclusive prefix over the CTA; *total receives the sum.
__device__ __forceinline__ long long cta_scan(long long v, long long* ws, long long* total) {
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  long long x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) ws[wid] = x;
  __syncthreads();
  long long before = 0, sum = 0;
  for (int w = 0; w < kPlanThreads / 32; ++w) {
    if (w < wid) before += ws[w];
    sum += ws[w];
  }
  *total = sum;
  return before + x - v;
}

__device__ __forceinline__ int tiles_of(const PlanArgs& a, int len) {
  return len > 0 ? (int)(((long long)len * a.G + a.tile_rows - 1) / a.tile_rows) : 0;
}

__device__ __forceinline__ AttnTile make_tile(const PlanArgs& a, const PlanReq& r, int req, int k) {
  AttnTile t;
  t.before = 0;
  t.req = req;
  t.row0 = k * a.tile_rows;
  const int all = r.len * a.G;
  t.rows = min(a.tile_rows, all - t.row0);
  t.first = r.first;
  t.qrow = r.qrow;
  t.kv_hi = r.first + (t.row0 + t.rows - 1) / a.G + 1;
  const int p0 = r.first + t.row0 / a.G;
  t.kv_lo = a.window > 0 ? max(0, p0 - a.window + 1) : 0;
  const int hi = (t.kv_hi + a.unit - 1) / a.unit;
  t.sink_units = min((min(a.sinks, t.kv_lo) + a.unit - 1) / a.unit, hi);
  t.win_unit = max(t.kv_lo / a.unit, t.sink_units);
  t.units = t.sink_units + hi - t.win_unit;
  return t;
}

// CTA i < n: request i's rows, table row and checks; CTA n: the rows of no request.  Every CTA
// sums the lengths before its own (at most 16 KiB that stay in L2: less than a launch between
// a scan and the rest would cost).  The CTA that finishes last cuts the requests into tiles
// and the tiles' units into equal shares.
__global__ void __launch_bounds__(kPlanThreads) k_batch_plan(PlanArgs a) {
  __shared__ long long ws[kPlanThreads / 32];
  __shared__ int last;
  __shared__ int first_tile[kMaxRequests];
  dep_wait();
  dep_trigger();
  const int i = blockIdx.x;
  const DevPool& p = a.p;
  long long mine = 0;
  for (int j = threadIdx.x; j < i; j += kPlanThreads) mine += max(a.lens[j], 0);
  const long long start = cta_sum(mine, ws);
  const int row0 = (int)min(start, (long long)a.num_tokens);
  if (threadIdx.x == 0) a.row_starts[i] = row0;
  if (i == a.n) {
    for (int r = row0 + threadIdx.x; r < a.num_tokens; r += kPlanThreads) {
      a.positions[r] = -1;
      a.slots[r] = -1;
    }
  } else {
    const int sid = a.sids[i];
    const int asked = a.lens[i];
    const int len = max(asked, 0);
    int err = 0;
    int first = 0;
    const bool known = sid >= 0 && sid < p.S;
    if (!known || asked < 0 || asked > a.max_len || start + len > a.num_tokens) {
      err = LV_ERR_BOUNDS;
    } else {
      const int ctx = p.sess[sid].ctx_tokens;
      first = a.firsts ? a.firsts[i] : -1;
      if (first < 0) first = ctx - len;
      // (positions stay far enough below 2^31 for a unit's keys past them)
      if (first < 0 || (long long)first + len > ctx || (long long)first + len > 0x7ffff000ll ||
          ((long long)first + len + p.T - 1) / p.T > p.maxB)
        err = LV_ERR_BOUNDS;
    }
    const int32_t* row = p.table + (size_t)(known ? sid : 0) * p.maxB;
    int32_t* out = a.tables + (size_t)i * p.maxB;
    const int kv_len = err ? 0 : first + len;
    const int nb = (int)(((uint32_t)kv_len + (uint32_t)p.T - 1u) / (uint32_t)p.T);
    // blocks that some row sees: from the first row's window on, and the sinks
    const int lo = a.window > 0 ? max(0, first - a.window + 1) : 0;
    const int lo_blk = lo / p.T;
    const int sink_blk = (int)(((uint32_t)min(a.sinks, kv_len) + (uint32_t)p.T - 1u) / (uint32_t)p.T);
    bool absent = false;
#pragma unroll 4
    for (int b = threadIdx.x; b < p.maxB; b += kPlanThreads) {
      int e = -1;
      if (b < nb) {
        e = row[b];
        if (e < 0 || e >= p.hbm_pages) {
          e = -1;
          absent |= len > 0 && (b >= lo_blk || b < sink_blk);
        }
      }
      out[b] = e;
    }
    if (__syncthreads_or(absent)) {
      err = LV_ERR_STATE;
      for (int b = threadIdx.x; b < nb; b += kPlanThreads) out[b] = -1;   // its own entries again
    }
    if (threadIdx.x == 0) {
      if (err) report(p.ctl, err, i);
      a.kv_lens[i] = err ? 0 : kv_len;
      a.reqs[i] = PlanReq{first, err ? 0 : len, row0, 0};
    }
    const int rows = (int)min((long long)len, a.num_tokens - (long long)row0);
    for (int r = threadIdx.x; r < rows; r += kPlanThreads) {
      int pos = -1;
      long long slot = -1;
      if (!err) {
        pos = first + r;
        const int b = (int)((uint32_t)pos / (uint32_t)p.T);
        slot = (long long)row[b] * p.T + (pos - b * p.T);
        if (p.incl && p.shadow[(size_t)sid * p.maxB + b] >= 0) slot = -slot - 2;
      }
      a.positions[row0 + r] = pos;
      a.slots[row0 + r] = slot;
    }
  }

  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(&a.head->ticket, 1) == (int)gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  // each request's first tile: a scan over the requests
  long long tiles = 0, live = 0;
  for (int base = 0; base < a.n; base += kPlanThreads) {
    const int q = base + threadIdx.x;
    const int len = q < a.n ? __ldcg(&a.reqs[q].len) : 0;
    long long total;
    const long long at = cta_scan(tiles_of(a, len), ws, &total);
    if (q < a.n) first_tile[q] = (int)min(tiles + at, (long long)a.max_tiles);
    tiles += total;
    live += len;
  }
  live = cta_sum(live, ws);
  const int n_tiles = (int)min(tiles, (long long)a.max_tiles);
  // the tiles, a thread each (its request found by bisection), and where they lie on the line
  long long units = 0, shorts = 0, longs = 0;
  bool cut_free = true;      // no pair has more units than one CTA may well take
  for (int base = 0; base < n_tiles; base += kPlanThreads) {
    const int t = base + threadIdx.x;
    AttnTile tile{};
    if (t < n_tiles) {
      int lo = 0, hi = a.n - 1;      // the last request whose first tile is not after t
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first_tile[mid] <= t) lo = mid;
        else hi = mid - 1;
      }
      const int4 r = __ldcg(reinterpret_cast<const int4*>(&a.reqs[lo]));
      tile = make_tile(a, PlanReq{r.x, r.y, r.z, 0}, lo, t - first_tile[lo]);
    }
    long long total;
    const long long at = cta_scan(t < n_tiles ? tile.units : 0, ws, &total);
    long long total_short, total_long;
    const long long at_short =
        cta_scan(t < n_tiles ? (tile.units + a.min_share - 1) / a.min_share : 0, ws, &total_short);
    const long long at_long = cta_scan(t < n_tiles ? (tile.units + a.uncut - 1) / a.uncut : 0, ws, &total_long);
    if (t < n_tiles) {
      // what comes before it, in units, in short shares (from bit 40 on) and in long ones (from 51)
      tile.before = units + at + (min(shorts + at_short, kManyShares) << 40) + (min(longs + at_long, kManyShares) << 51);
      a.tiles[t] = tile;
      cut_free &= tile.units <= a.uncut;
    }
    units += total;
    shorts += total_short;
    longs += total_long;
  }
  // Pairs apart in shares of their own: uncut ones of up to `uncut` units where that holds them all,
  // else cut short (a cut costs what some 8 units of a warp do, so in the middle there is nothing).
  cut_free = __syncthreads_and(cut_free);
  const long long needed = cut_free ? longs : shorts;
  const bool apart = needed * a.line_heads <= a.shares;
  const int lead = apart ? -1 : a.lead, size = cut_free ? a.uncut : a.min_share;
  units = apart ? needed * size * a.line_heads : (units + (long long)n_tiles * lead) * a.line_heads;
  const long long share = apart ? size : max((units + a.shares - 1) / a.shares, (long long)a.min_share);
  const int dead = a.num_tokens - (int)live;
  if (threadIdx.x == 0) a.head->ticket = 0;
  // (zero already but after an attention that ran out of a wait)
  static_assert(kArriveWords % 4 == 0, "cleared by 16 bytes");
  for (int i = threadIdx.x; i < a.ctas * (kArriveWords / 4); i += kPlanThreads)
    reinterpret_cast<int4*>(a.arrived)[i] = make_int4(0, 0, 0, 0);
  __syncthreads();
  for (int t = threadIdx.x; t < n_tiles; t += kPlanThreads) {
    AttnTile tile = a.tiles[t];      // (this thread's own)
    tile.before = apart ? (tile.before >> (cut_free ? 51 : 40) & kManyShares) * size * a.line_heads
                        : ((tile.before & ((1ll << 40) - 1)) + (long long)t * lead) * a.line_heads;
    a.tiles[t].before = tile.before;
    const long long lo = tile.before, hi = lo + (long long)stretch_of(tile.units, lead, (int)share) * a.line_heads;
    for (long long c = (lo + share - 1) / share; c * share < hi; ++c)
      a.work[c] = CtaWork{tile, c * share, min(units, (c + 1) * share), (int)share, lead, t, dead};
  }
  for (long long c = (units + share - 1) / share + threadIdx.x; c < a.shares; c += kPlanThreads)
    a.work[c] = CtaWork{AttnTile{}, 0, 0, (int)share, lead, 0, dead};
}

// ---------------------------------------------------------------- KV write
// A unit is 8 elements, out[slot][h][8c..] <- src[r][h][8c..]; a row's are those of K, then V's.  A
// CTA takes kWriteThreads * U of them in a row, a thread U with all its loads on their way before
// the first store.
// What bounds it: the launch for a decode step; HBM for prompts' rows.
constexpr int kWriteThreads = 256;

template <bool kBf16>
__device__ __forceinline__ uint4 load8(const uint8_t* src, int64_t at, int type, bool vec) {
  if (type == LV_F32) {
    const float* f = reinterpret_cast<const float*>(src) + at;
    float x[8];
    if (vec) {
      const float4 lo = __ldcs(reinterpret_cast<const float4*>(f)), hi = __ldcs(reinterpret_cast<const float4*>(f) + 1);
      x[0] = lo.x; x[1] = lo.y; x[2] = lo.z; x[3] = lo.w;
      x[4] = hi.x; x[5] = hi.y; x[6] = hi.z; x[7] = hi.w;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = f[e];
    }
    return make_uint4(pack16<kBf16>(x[0], x[1]), pack16<kBf16>(x[2], x[3]), pack16<kBf16>(x[4], x[5]),
                      pack16<kBf16>(x[6], x[7]));
  }
  const uint16_t* h = reinterpret_cast<const uint16_t*>(src) + at;
  uint4 w;
  if (vec) {
    w = __ldcs(reinterpret_cast<const uint4*>(h));
  } else {
    uint32_t y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (uint32_t)h[2 * e] | (uint32_t)h[2 * e + 1] << 16;
    w = make_uint4(y[0], y[1], y[2], y[3]);
  }
  if ((type == LV_BF16) == kBf16) return w;
  // the other 16-bit type: through 32 bits, which hold both exactly
  uint32_t* y = &w.x;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float2 f;
    if (kBf16) f = __half22float2(*reinterpret_cast<const __half2*>(&y[e]));
    else f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&y[e]));
    y[e] = pack16<kBf16>(f.x, f.y);
  }
  return w;
}

template <bool kBf16, int U>
__global__ void __launch_bounds__(kWriteThreads) k_kv_write(const __grid_constant__ WriteArgs a) {
  dep_wait();
  dep_trigger();
  const uint32_t cols = (uint32_t)a.D / 8u, per_kv = (uint32_t)a.H * cols, per_row = 2u * per_kv;
  const uint64_t base = (uint64_t)blockIdx.x * (kWriteThreads * U);
  const uint32_t r0 = (uint32_t)(base / per_row), off0 = (uint32_t)(base - (uint64_t)r0 * per_row);
  uint4 w[U];
  uint8_t* to[U];
#pragma unroll
  for (int k = 0; k < U; ++k) {
    const uint32_t off = off0 + k * kWriteThreads + threadIdx.x;
    const uint32_t up = off / per_row, r = r0 + up, x = off - up * per_row;
    to[k] = nullptr;
    if (r >= (uint32_t)a.num_tokens) continue;
    const bool kv = x >= per_kv;
    const uint32_t y = kv ? x - per_kv : x;
    const uint32_t h = y / cols, c = y - h * cols;
    const int64_t slot = a.slots[r];
    if (slot < 0 || slot >= a.num_slots) {
      if (x == 0 && slot != -1) report(a.ctl, slot < 0 ? LV_ERR_STATE : LV_ERR_BOUNDS, r);
      continue;
    }
    const int64_t at = r * (kv ? a.row_stride[1] : a.row_stride[0]) + h * (kv ? a.head_stride[1] : a.head_stride[0]) + 8 * c;
    w[k] = load8<kBf16>(kv ? a.src[1] : a.src[0], at, kv ? a.src_type[1] : a.src_type[0],
                        (kv ? a.vec[1] : a.vec[0]) != 0);
    to[k] = (kv ? a.dst[1] : a.dst[0]) + ((uint64_t)slot * per_kv + y) * 16u;
  }
#pragma unroll
  for (int k = 0; k < U; ++k)
    if (to[k]) *reinterpret_cast<uint4*>(to[k]) = w[k];
}

}  // namespace

cudaError_t launch_plan(const PlanArgs& a, cudaStream_t s) {
  return launch_dependent(k_batch_plan, dim3(a.n + 1), kPlanThreads, 0, s, a);
}

// One unit a thread while the GPU holds all of them at once, else two: 64 rows of 4 heads of 128
// 1.8 us and 2.3; 13706 such rows from f32 (84 MB in and out) 11.7 us and 10.7 (7.9 TB/s, part of
// it from L2), and 11.8 with four.
cudaError_t launch_kv_write(const WriteArgs& a, cudaStream_t s, int num_sms) {
  const uint64_t units = (uint64_t)a.num_tokens * 2 * a.H * (a.D / 8);
  const int U = units <= (uint64_t)num_sms * 2048 ? 1 : 2;
  const uint64_t ctas = (units + kWriteThreads * U - 1) / (kWriteThreads * U);
  if (ctas > 0x7fffffffull) return cudaErrorInvalidValue;
  const bool bf16 = a.dtype == LV_BF16;
  return launch_dependent(U == 1 ? (bf16 ? k_kv_write<true, 1> : k_kv_write<false, 1>)
                                 : (bf16 ? k_kv_write<true, 2> : k_kv_write<false, 2>),
                          dim3((unsigned)ctas), kWriteThreads, 0, s, a);
}

}  // namespace lv
