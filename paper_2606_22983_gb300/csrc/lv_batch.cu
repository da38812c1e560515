// The plan of a serving step and the write of its K and V rows (include/lv.h, "a serving step
// on resident KV").
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "lv_batch.cuh"

namespace lv {

namespace {

constexpr int kPlanThreads = 256, kCutThreads = 1024;
constexpr int kMaxRequests = 4096;      // lv_batch_create's limit
constexpr int kOneLaunch = kPlanOneLaunch;

// Exclusive prefix over the CTA of NT threads; *total receives the sum.  ws: a word a warp; a barrier
// lies between its uses.
template <int NT>
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
  // every warp scans the warps' sums
  const long long own = lane < NT / 32 ? ws[lane] : 0;
  long long y = own;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long z = __shfl_up_sync(0xffffffffu, y, o);
    if (lane >= o) y += z;
  }
  *total = __shfl_sync(0xffffffffu, y, 31);
  return __shfl_sync(0xffffffffu, y - own, wid) + x - v;
}
template <int NT>
__device__ __forceinline__ long long cta_sum(long long v, long long* ws) {
  long long total;
  cta_scan<NT>(v, ws, &total);
  return total;
}

// (32-bit divisions: len * G is below 2^31)
__device__ __forceinline__ int tiles_of(const PlanArgs& a, int len) {
  return len > 0 ? (int)(((uint32_t)len * (uint32_t)a.G + (uint32_t)a.tile_rows - 1u) / (uint32_t)a.tile_rows) : 0;
}

__device__ __forceinline__ AttnTile make_tile(const PlanArgs& a, const PlanReq& r, int req, int k) {
  const int up = (1 << a.unit_shift) - 1;
  AttnTile t;
  t.before = 0;
  t.req = req;
  t.row0 = k * a.tile_rows;
  t.rows = min(a.tile_rows, r.len * a.G - t.row0);
  t.first = r.first;
  t.qrow = r.qrow;
  t.kv_hi = r.first + (int)((uint32_t)(t.row0 + t.rows - 1) / (uint32_t)a.G) + 1;
  const int p0 = r.first + (int)((uint32_t)t.row0 / (uint32_t)a.G);
  t.kv_lo = a.window > 0 ? max(0, p0 - a.window + 1) : 0;
  const int hi = (t.kv_hi + up) >> a.unit_shift;
  t.sink_units = min((min(a.sinks, t.kv_lo) + up) >> a.unit_shift, hi);
  t.win_unit = max(t.kv_lo >> a.unit_shift, t.sink_units);
  t.units = t.sink_units + hi - t.win_unit;
  return t;
}

// One CTA of NT threads cuts the requests into tiles and the tiles' units into shares: prefix sums over
// the requests' tiles and over the tiles' units, a thread taking several in a row, so that a tile is made
// twice (once to be counted, once to be written) rather than kept.  What bounds it is the chain: five
// scans of two barriers each (tiles, owned rows, units, shares of either size; the last two and a vote only
// where there may be pairs apart), some 5 us for 64 requests of one tile and 10 for 1024.
template <int NT>
__device__ __forceinline__ void cut_line(const PlanArgs& a, long long* ws, int* first_tile) {
  // each request's first tile: a scan over the requests, a thread taking several in a row
  const int per = (a.n + NT - 1) / NT, q0 = min((int)threadIdx.x * per, a.n), q1 = min(q0 + per, a.n);
  long long own = 0, tiles, live = 0;
  for (int q = q0; q < q1; ++q) {
    const int len = __ldcg(&a.reqs[q].len);
    first_tile[q] = tiles_of(a, len);
    own += first_tile[q];
    live += len;
  }
  long long at_tile = cta_scan<NT>(own, ws, &tiles);
  for (int q = q0; q < q1; ++q) {
    const int m = first_tile[q];
    first_tile[q] = (int)min(at_tile, (long long)a.max_tiles);
    at_tile += m;
  }
  live = cta_sum<NT>(live, ws);      // (with a barrier after the writes above)
  const int n_tiles = (int)min(tiles, (long long)a.max_tiles);
  // the tiles, a thread several in a row (its first one's request found by bisection), and where
  // they lie on the line: what comes before each in units, and in short and long shares
  const int per_tile = (n_tiles + NT - 1) / NT;
  const int t0 = min((int)threadIdx.x * per_tile, n_tiles), t1 = min(t0 + per_tile, n_tiles);
  int req0 = 0;
  if (t0 < t1) {
    int hi = a.n - 1;      // the last request whose first tile is not after t0
    while (req0 < hi) {
      const int mid = (req0 + hi + 1) >> 1;
      if (first_tile[mid] <= t0) req0 = mid;
      else hi = mid - 1;
    }
  }
  auto each_tile = [&](auto&& f) {
    int q = req0, loaded = -1;
    PlanReq r{};
    for (int t = t0; t < t1; ++t) {
      while (q + 1 < a.n && first_tile[q + 1] <= t) ++q;
      if (q != loaded) {
        const int4 w = __ldcg(reinterpret_cast<const int4*>(&a.reqs[q]));
        r = PlanReq{w.x, w.y, w.z, 0};
        loaded = q;
      }
      f(t, make_tile(a, r, q, t - first_tile[q]));
    }
  };
  long long my_units = 0, my_short = 0, my_long = 0;
  bool cut_free = true;      // no pair has more units than one CTA may well take
  each_tile([&](int, const AttnTile& t) {
    my_units += t.units;
    my_short += (uint32_t)(t.units + a.min_share - 1) / (uint32_t)a.min_share;
    my_long += (uint32_t)(t.units + a.uncut - 1) / (uint32_t)a.uncut;
    cut_free &= t.units <= a.uncut;
  });
  long long units, shorts = 0, longs = 0, at_short = 0, at_long = 0;
  const long long at_unit = cta_scan<NT>(my_units, ws, &units);
  const bool few = (long long)n_tiles * a.line_heads <= a.shares;      // (or no pair has shares of its own)
  if (few) {
    at_short = cta_scan<NT>(my_short, ws, &shorts);
    at_long = cta_scan<NT>(my_long, ws, &longs);
    cut_free = __syncthreads_and(cut_free);
  }
  // Pairs apart in shares of their own: uncut ones of up to `uncut` units where that holds them all,
  // else cut short (a cut costs what some 8 units of a warp do, so in the middle there is nothing).
  const long long needed = cut_free ? longs : shorts;
  const bool apart = few && needed * a.line_heads <= a.shares;
  const int lead = apart ? -1 : a.lead, size = cut_free ? a.uncut : a.min_share;
  units = apart ? needed * size * a.line_heads : (units + (long long)n_tiles * lead) * a.line_heads;
  const long long share = apart ? size : max((units + a.shares - 1) / a.shares, (long long)a.min_share);
  if (threadIdx.x == 0) *a.head = StepHead{a.kind, a.num_tokens, (int)live, 0};
  // (zero already but after an attention that ran out of a wait)
  static_assert(kArriveWords % 4 == 0, "cleared by 16 bytes");
  for (int i = threadIdx.x; i < a.ctas * (kArriveWords / 4); i += NT)
    reinterpret_cast<int4*>(a.arrived)[i] = make_int4(0, 0, 0, 0);
  long long before = apart ? (cut_free ? at_long : at_short) * size : at_unit + (long long)t0 * lead;
  long long c = -1;      // the next share to begin
  each_tile([&](int t, AttnTile tile) {
    const int stretch = stretch_of(tile.units, lead, (int)share);
    tile.before = before * a.line_heads;
    a.tiles[t] = tile;
    const long long hi = tile.before + (long long)stretch * a.line_heads;
    if (c < 0) c = (tile.before + share - 1) / share;
    for (; c * share < hi; ++c)
      a.work[c] = CtaWork{tile, c * share, min(units, (c + 1) * share), (int)share, lead, t, 0};
    before += stretch;
  });
  for (c = (units + share - 1) / share + threadIdx.x; c < a.shares; c += NT)
    a.work[c] = CtaWork{AttnTile{}, 0, 0, (int)share, lead, 0, 0};
}

// CTA i < n: request i's rows, table row and checks; CTA n: the rows of no request.
//   row_start_i = sum of len_j over j < i;  position of row r: first_i + r - row_start_i;
//   slot: table[sid][position / T] * T + position % T
// It reads the tables once and writes them once, 8 KiB a request of 16 000 tokens, and 12 bytes a row:
// latency bounds it, not bytes (64 requests with the cut of their work 9.2 us, 1024 in two launches 17.4).
// Every CTA
// sums the lengths before its own (at most 16 KiB that stay in L2: less than a launch between
// a scan and the rest would cost).  kCut: the CTA that finishes last cuts the line too.
template <bool kCut>
__global__ void __launch_bounds__(kPlanThreads) k_batch_rows(const __grid_constant__ PlanArgs a) {
  __shared__ long long ws[kPlanThreads / 32];
  dep_wait();
  dep_trigger();
  const int i = blockIdx.x;
  const DevPool& p = a.p;
  long long mine = 0;
  for (int j = threadIdx.x; j < i; j += kPlanThreads) mine += max(a.lens[j], 0);
  const long long start = cta_sum<kPlanThreads>(mine, ws);
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
  if constexpr (kCut) {
    __shared__ int last;
    __shared__ int first_tile[kOneLaunch];
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
      last = atomicAdd(a.ticket, 1) == (int)gridDim.x - 1;
      if (last) *a.ticket = 0;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    cut_line<kPlanThreads>(a, ws, first_tile);
  }
}

__global__ void __launch_bounds__(kCutThreads) k_batch_cut(const __grid_constant__ PlanArgs a) {
  __shared__ long long ws[kCutThreads / 32];
  __shared__ int first_tile[kMaxRequests];
  dep_wait();
  dep_trigger();
  cut_line<kCutThreads>(a, ws, first_tile);
}

// ---------------------------------------------------------------- KV write
// A unit is 8 elements, out[slot][h][8c..] <- src[r][h][8c..]; a row's are those of K, then V's.  A
// CTA takes kWriteThreads * U of them in a row, a thread U with all its loads on their way before
// the first store.
// What bounds it: the launch for a decode step (64 rows of 4 heads of 128, 1.9 us); HBM for prompts' rows
// (13 706 of them from 32 to 16 bits, 84 MB in and out, 10.9 us, some of it from L2).  Each row's K and V are
// read and written once: 2 H D (source bytes + 2), and the 8 bytes of its slot.  Rounding is to nearest even.
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
  const StepHead head = load_words(a.head);
  // rows of the planned step, none where it has more than this call's tensors
  const int rows = head.num_tokens <= a.num_tokens ? head.num_tokens : 0;
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
    const int64_t slot = a.slots[r];      // (asked for beside the step's head)
    if (r >= (uint32_t)rows) continue;
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
  if (LV_RARE(head.num_tokens > a.num_tokens) && blockIdx.x == 0 && threadIdx.x == 0) report(a.ctl, LV_ERR_STATE, -1);
}

}  // namespace

// One launch up to kOneLaunch requests (64 decoding sessions: 8.8 us, in two 10.2), else one CTA of
// 1024 threads cuts the line by itself (1024 requests: 17 us; by the last CTA of the rows' 24).
cudaError_t launch_plan(const PlanArgs& a, cudaStream_t s) {
  if (a.n <= kOneLaunch) return launch_dependent(k_batch_rows<true>, dim3(a.n + 1), kPlanThreads, 0, s, a);
  const cudaError_t e = launch_dependent(k_batch_rows<false>, dim3(a.n + 1), kPlanThreads, 0, s, a);
  if (e != cudaSuccess) return e;
  return launch_dependent(k_batch_cut, dim3(1), kCutThreads, 0, s, a);
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
