// Eviction of tokens from sessions' caches by what they weigh (include/lv.h, "keeping a part of the cache"): the
// choice of the tokens to keep, their K and V moved to the front of the sessions' pages, and the
// pages behind them given back.
#include <cooperative_groups.h>

#include "lv_batch.cuh"
#include "lv_keep.cuh"

namespace lv {

namespace {

__device__ __forceinline__ uint32_t blocks_of(int32_t tokens, int32_t T) {
  return tokens <= 0 ? 0u : ((uint32_t)tokens + (uint32_t)T - 1u) / (uint32_t)T;
}

// ---------------------------------------------------------------- choice
// A weight's place in the order of the numbers: larger for larger ones, equal for the two zeros, and the
// largest for every NaN.
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x);
  if (x != x) return 0xffffffffu;
  if (x == 0.f) return 0x80000000u;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int kSelThreads = 512, kSelWarps = kSelThreads / 32;
constexpr int kBins = 2048;      // 11 bits of the key at a time: 11, 11 and 10

// One list: request blockIdx.y's tokens in (layer, head) blockIdx.x.  Tokens before lo and from hi on
// stay; of those between, the `need` of largest key.  The key of the last of them is found by its digits
// from above, a histogram of the candidates each; then the tokens are gone through in order, those above it
// kept and of those equal to it the first.
__global__ void __launch_bounds__(kSelThreads) k_select_kept(const __grid_constant__ SelectArgs a) {
  __shared__ int bins[kBins];
  __shared__ int sums[2][kSelWarps];
  __shared__ uint32_t s_digit;
  __shared__ int s_above;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int i = blockIdx.y, layer = blockIdx.x / a.H, head = blockIdx.x - layer * a.H;
  dep_wait();
  dep_trigger();
  const int sid = a.sids[i];
  int32_t* out = a.kept + ((int64_t)i * gridDim.x + blockIdx.x) * a.most;
  int keep = a.keeps[i], c = 0;
  bool bad = sid < 0 || sid >= a.p.S || keep < 0 || keep > a.most;
  if (!bad) {
    c = a.p.sess[sid].ctx_tokens;
    bad = c > a.w.tokens;
  }
  if (bad) {
    if (blockIdx.x == 0 && tid == 0) report(a.p.ctl, LV_ERR_BOUNDS, i);
    keep = 0;
  }
  keep = min(keep, c);
  const float* w = a.w.data + layer * a.w.layer_stride + (bad ? 0 : sid) * a.w.session_stride + head * a.w.head_stride;
  const int lo = min(a.first, keep), hi = max(c - min(a.last, keep - lo), lo);
  int need = keep - lo - (c - hi);
  uint32_t last = 0xffffffffu;      // the last kept key, with `need` of its equals
  int ties = 0;
  if (keep == 0) {
  } else if (need == hi - lo) {
    last = 0;
    ties = need;
  } else if (need > 0) {
    uint32_t have = 0;
    int shift = 32;
    while (shift > 0) {
      const int bits = shift > 11 ? 11 : shift;      // 11, 11, 10
      shift -= bits;
      for (int b = tid; b < kBins; b += kSelThreads) bins[b] = 0;
      __syncthreads();
      for (int j = lo + tid; j < hi; j += kSelThreads) {
        const uint32_t k = order_key(w[j]);
        if (shift + bits == 32 || (k >> (shift + bits)) == (have >> (shift + bits)))
          atomicAdd(&bins[k >> shift & ((1u << bits) - 1u)], 1);
      }
      __syncthreads();
      // from the top bin down: the bin in which `need` is reached
      constexpr int kPer = kBins / kSelThreads;
      int mine[kPer], sum = 0;
#pragma unroll
      for (int e = 0; e < kPer; ++e) sum += mine[e] = bins[kBins - 1 - (tid * kPer + e)];
      int x = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
      }
      if (lane == 31) sums[0][wid] = x;
      __syncthreads();
      int above = x - sum;
      for (int v = 0; v < wid; ++v) above += sums[0][v];
      if (above < need && above + sum >= need) {
        int e = 0;
        while (above + mine[e] < need) above += mine[e++];
        s_digit = kBins - 1 - (tid * kPer + e);
        s_above = above;
      }
      __syncthreads();
      have |= s_digit << shift;
      need -= s_above;
    }
    last = have;
    ties = need;
  }
  // the kept ones, in order
  int kept_before = 0, ties_before = 0;
  for (int j0 = 0; j0 < c && keep > 0; j0 += kSelThreads) {
    const int j = j0 + tid;
    const bool between = j >= lo && j < hi;
    const uint32_t k = between ? order_key(w[j]) : 0;
    const bool tie = between && (k == last || need == hi - lo);
    const uint32_t tie_votes = __ballot_sync(0xffffffffu, tie);
    if (lane == 0) sums[0][wid] = __popc(tie_votes);
    __syncthreads();
    int t = ties_before + __popc(tie_votes & ((1u << lane) - 1u)), all_ties = 0;
    for (int v = 0; v < kSelWarps; ++v) {
      if (v < wid) t += sums[0][v];
      all_ties += sums[0][v];
    }
    ties_before += all_ties;
    const bool stay = j < c && (!between || (tie ? t < ties : k > last));
    const uint32_t votes = __ballot_sync(0xffffffffu, stay);
    if (lane == 0) sums[1][wid] = __popc(votes);
    __syncthreads();
    int at = kept_before + __popc(votes & ((1u << lane) - 1u)), all = 0;
    for (int v = 0; v < kSelWarps; ++v) {
      if (v < wid) at += sums[1][v];
      all += sums[1][v];
    }
    kept_before += all;
    if (stay && at < keep) out[at] = j;
  }
  for (int j = keep + tid; j < a.most; j += kSelThreads) out[j] = -1;
}

// ---------------------------------------------------------------- compaction
constexpr int kCheckThreads = 512, kCheckCtas = 8;

// Request blockIdx.x / kCheckCtas by a cluster: its session, that its blocks are in HBM, and its lists, which
// have to ascend within the context.  lens[i] receives what it may be cut to, or -1 where nothing moves.
__global__ void __cluster_dims__(kCheckCtas, 1, 1) __launch_bounds__(kCheckThreads)
    k_compact_check(const __grid_constant__ CompactArgs a) {
  namespace cg = cooperative_groups;
  __shared__ int s_bad;
  const cg::cluster_group cluster = cg::this_cluster();
  const int i = blockIdx.x / kCheckCtas, rank = cluster.block_rank(), tid = threadIdx.x;
  dep_wait();
  dep_trigger();
  if (tid == 0) s_bad = 0;
  __syncthreads();
  const int sid = a.sids[i], asked = a.keeps[i];
  int bad = sid < 0 || sid >= a.p.S || asked < 0 || asked > a.most ? LV_ERR_BOUNDS : 0;
  const int c = bad ? 0 : a.p.sess[sid].ctx_tokens, keep = min(asked, c);
  if (!bad && a.w.data && c > a.w.tokens) bad = LV_ERR_BOUNDS;
  if (!bad) {
    const int at = rank * kCheckThreads + tid, step = kCheckCtas * kCheckThreads;
    for (int j = at; j < i; j += step)
      if (a.sids[j] == sid) bad = LV_ERR_DOUBLE_MAP;
    const int nb = (int)blocks_of(c, a.p.T);
    for (int b = at; b < nb; b += step) {
      const int e = a.p.table[(size_t)sid * a.p.maxB + b];
      if (e < 0 || e >= a.p.hbm_pages) bad = LV_ERR_STATE;
    }
    if (keep < c) {
      const int lists = a.p.J / 2 * a.H;
      for (int l = rank; l < lists; l += kCheckCtas) {
        const int32_t* x = a.kept + ((int64_t)i * lists + l) * a.most;
        for (int j = tid; j < keep; j += kCheckThreads) {
          const int v = x[j], before = j > 0 ? x[j - 1] : -1;
          if (v <= before || v >= c) bad = LV_ERR_BOUNDS;
        }
      }
    }
  }
  if (bad) atomicMax(&s_bad, bad);
  cluster.sync();
  if (rank == 0 && tid == 0) {
    int worst = 0;
    for (int r = 0; r < kCheckCtas; ++r) worst = max(worst, *cluster.map_shared_rank(&s_bad, r));
    if (worst) report(a.p.ctl, worst, i);
    a.lens[i] = worst ? -1 : keep;
  }
  cluster.sync();      // (the others' shared memory is read until here)
}

// Moves rows [0, keep) of one list's K or V: row j of the head from the slot of token kept[j], in chunks of
// rows in order: as the lists ascend, kept[j] >= j, so a chunk whose loads come before its stores reads
// nothing that an earlier one wrote over.  A row's vectors lie together; `parts` CTAs share them.
template <typename V, int U>
__global__ void __launch_bounds__(kMoveThreads) k_compact(const __grid_constant__ CompactArgs a, int vecs, int part_vecs) {
  dep_wait();
  dep_trigger();
  const int i = blockIdx.y, tid = threadIdx.x;
  const int lists = a.p.J / 2 * a.H, parts = (vecs + part_vecs - 1) / part_vecs;
  const int part = blockIdx.x % parts, kv = blockIdx.x / parts % 2, list = blockIdx.x / parts / 2;
  const int layer = list / a.H, head = list - layer * a.H;
  const int keep = a.lens[i];
  if (keep < 0) return;
  const int sid = a.sids[i], c = a.p.sess[sid].ctx_tokens;
  if (keep >= c) return;
  const int32_t* kept = a.kept + ((int64_t)i * lists + list) * a.most;
  const int32_t* table = a.p.table + (size_t)sid * a.p.maxB;
  V* base = reinterpret_cast<V*>(a.p.kv[2 * layer + kv]);
  const uint64_t page_vecs = (uint64_t)a.p.P / sizeof(V);
  const uint32_t T = a.p.T, token_vecs = (uint32_t)a.H * vecs;
  const int v0 = part * part_vecs, mine = min(part_vecs, vecs - v0);
  auto slot = [&](int token) -> V* {
    const uint32_t b = a.t_shift >= 0 ? (uint32_t)token >> a.t_shift : (uint32_t)token / T;
    return base + (uint64_t)table[b] * page_vecs + (uint64_t)((uint32_t)token - b * T) * token_vecs + head * vecs + v0;
  };
  const int rows = kMoveThreads * U / part_vecs;      // of a chunk
  for (int j0 = 0; j0 < keep; j0 += rows) {
    V x[U];
    V* to[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = u * kMoveThreads + tid, r = at / part_vecs, v = at - r * part_vecs, j = j0 + r;
      to[u] = nullptr;
      if (r >= rows || j >= keep || v >= mine) continue;
      const int from = kept[j];
      if (from == j) continue;
      x[u] = slot(from)[v];
      to[u] = slot(j) + v;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (to[u]) *to[u] = x[u];
  }
  if (part || kv) return;
  if (a.w.data) {
    float* w = a.w.data + layer * a.w.layer_stride + sid * a.w.session_stride + head * a.w.head_stride;
    for (int j0 = 0; j0 < keep; j0 += kMoveThreads) {
      const int j = j0 + tid;
      const float y = j < keep ? w[kept[j]] : 0.f;
      __syncthreads();
      if (j < keep) w[j] = y;
    }
    __syncthreads();
    for (int j = keep + tid; j < c; j += kMoveThreads) w[j] = 0.f;
  }
  // the blocks' rows are others now: what the host tier holds of them is no copy any more
  if (a.p.incl && list == 0) {
    const int nb = (int)blocks_of(keep, a.p.T);
    for (int b = tid; b < nb; b += kMoveThreads) drop_clean(a.p, (size_t)sid * a.p.maxB + b);
  }
}

// ---------------------------------------------------------------- the context's end
constexpr int kCutThreads = 256;

// Request blockIdx.x: session sids[i] keeps its first lens[i] tokens; the blocks behind them are freed, in
// either tier.
__global__ void __launch_bounds__(kCutThreads) k_truncate(DevPool p, const int32_t* sids, const int32_t* lens) {
  dep_wait();
  const int i = blockIdx.x, tid = threadIdx.x;
  const int sid = sids[i], len = lens[i];
  if (len < 0) return;
  if (sid < 0 || sid >= p.S) {
    if (tid == 0) report(p.ctl, LV_ERR_BOUNDS, i);
    return;
  }
  bool again = false;
  for (int j = tid; j < i; j += kCutThreads) again |= sids[j] == sid && lens[j] >= 0;
  const int c = p.sess[sid].ctx_tokens;
  if (__syncthreads_or(again)) {      // (and every thread has read the context's length)
    if (tid == 0) report(p.ctl, LV_ERR_DOUBLE_MAP, i);
    return;
  }
  if (len >= c) return;
  const int nb = (int)blocks_of(len, p.T), end = min((int)blocks_of(c, p.T), p.maxB);
  int in_hbm = 0, in_host = 0;
  for (int b = nb + tid; b < end; b += kCutThreads) {
    const size_t at = (size_t)sid * p.maxB + b;
    const int e = p.table[at];
    p.table[at] = -1;
    if (p.incl) drop_clean(p, at);
    if (e >= 0 && e < p.hbm_pages) {
      p.own_hbm[e] = kOwnerNone;
      atomicAnd(&p.bits_hbm[e >> 5], ~(1u << (e & 31)));
      ++in_hbm;
    } else if (e <= -2 && -(long long)e - 2 < p.host_pages) {
      const int s = -e - 2;
      p.own_host[s] = kOwnerNone;
      atomicAnd(&p.bits_host[s >> 5], ~(1u << (s & 31)));
      ++in_host;
    }
  }
  in_hbm = __reduce_add_sync(0xffffffffu, in_hbm);
  in_host = __reduce_add_sync(0xffffffffu, in_host);
  if ((tid & 31) == 0 && (in_hbm || in_host)) {
    atomicAdd(reinterpret_cast<unsigned long long*>(&p.cnt[sid]),
              ((unsigned long long)(unsigned)-in_host << 32) + (unsigned long long)(long long)-in_hbm);
    if (in_hbm) atomicAdd(reinterpret_cast<unsigned long long*>(&p.ctl[C_HBM_ALLOC]), (unsigned long long)(long long)-in_hbm);
    if (in_host) atomicAdd(reinterpret_cast<unsigned long long*>(&p.ctl[C_HOST_ALLOC]), (unsigned long long)(long long)-in_host);
  }
  if (tid == 0) p.sess[sid].ctx_tokens = len;
}

}  // namespace

cudaError_t launch_select_kept(const SelectArgs& a, int n, cudaStream_t s) {
  return launch_dependent(k_select_kept, dim3(a.p.J / 2 * a.H, n), kSelThreads, 0, s, a);
}

cudaError_t launch_compact(const CompactArgs& a, int n, int row_bytes, int num_sms, cudaStream_t s) {
  const cudaError_t e = launch_dependent(k_compact_check, dim3(n * kCheckCtas), kCheckThreads, 0, s, a);
  if (e != cudaSuccess) return e;
  const int lists = a.p.J / 2 * a.H;
  const int vecs = row_bytes % 16 == 0 ? row_bytes / 16 : row_bytes;
  // rows shared by several CTAs, down to 32 bytes of each, where there are few lists
  int part = vecs;
  if (row_bytes % 16 == 0)
    while (part > 2 && (int64_t)2 * lists * n * ((vecs + part - 1) / part) < 2 * num_sms) part = (part + 1) / 2;
  part = part < kMoveThreads ? part : kMoveThreads;
  const dim3 grid(lists * 2 * ((vecs + part - 1) / part), n);
  if (row_bytes % 16 == 0) return launch_dependent(k_compact<uint4, 8>, grid, kMoveThreads, 0, s, a, vecs, part);
  return launch_dependent(k_compact<uint8_t, 8>, grid, kMoveThreads, 0, s, a, vecs, part);
}

cudaError_t launch_truncate(const DevPool& p, const int32_t* sids, const int32_t* lens, int n, cudaStream_t s) {
  return launch_dependent(k_truncate, dim3(n), kCutThreads, 0, s, p, sids, lens);
}

}  // namespace lv
