// Eviction of tokens from sessions' caches by what they weigh (include/lv.h, "keeping a part of the cache"): the
// choice of the tokens to keep, their K and V moved to the front of the sessions' pages, and the
// pages behind them given back.
#include <cooperative_groups.h>

#include <type_traits>

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
__device__ __forceinline__ uint32_t order_key(uint32_t bits) {
  if ((bits << 1) > 0xff000000u) return 0xffffffffu;      // a NaN
  if ((bits << 1) == 0) return 0x80000000u;
  return bits ^ ((uint32_t)((int32_t)bits >> 31) | 0x80000000u);
}

// The number whose key it is, the nearest infinity where that is a NaN's.
__device__ __forceinline__ float number_of(uint32_t key) {
  if (key >= 0xff800000u) return INFINITY;
  if (key <= 0x007fffffu) return -INFINITY;
  return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

constexpr int kSelThreads = 256, kSelWarps = kSelThreads / 32;
constexpr int kStepBits = 8;           // log2(kSelThreads): steps between the bounds
static_assert(1 << kStepBits == kSelThreads, "a thread a step");
constexpr int kBins = 2048;            // 11 bits of the key, or 12 in halves of words
constexpr int kSample = 2048;
constexpr int kTurns = 64;             // requests whose lists are taken by their lengths
constexpr int kMostWords = 2048;       // of 32 tokens, in a list that is read once

// Keys near the border between kept and not that are gathered: an eighth of the longest list, which the bounds
// by the sample hold where its weights spread over some octaves.
__host__ __device__ constexpr int few_of(int words) { return words * 4 > 2048 ? words * 4 : 2048; }

struct SelectShared {
  int* bins;                   // [kBins]
  int steps[kSelThreads];      // a histogram of those near the border
  int sums[2][kSelWarps];
  int few, above, low;         // tokens near the border, above it, and of the lowest key there
  int digit, before, inside;
  int turn, ctx[kTurns];
  uint32_t lo_key, hi_key;
  uint32_t last_key[32];
  int last_at[32];
  int last;
};

// What select_once keeps beside it, for lists of `words` words of 32 tokens, a multiple of 32.  (The first histogram,
// and at the end the kept ones' numbers, lie where the keys near the border do.)
struct OnceShared {
  uint32_t* key;       // of those near the border, [few_of(words)]
  uint4* word;         // [words]: which of 32 tokens are above the bounds, have the lowest key in them, lie between;
                       // and a word that makes it one store of 16 bytes
  int* batch;          // [words / 32] kept ones of 1024 tokens
  uint16_t* at;        // [few_of(words)]
  static size_t bytes(int words) { return (size_t)words * 16 + words / 8 + (size_t)few_of(words) * 6; }
  __device__ OnceShared(uint32_t* p, int words)
      : key(p), word(reinterpret_cast<uint4*>(p + few_of(words))), batch(reinterpret_cast<int*>(word + words)),
        at(reinterpret_cast<uint16_t*>(batch + words / 32)) {}
};
static_assert(few_of(0) >= kBins && 4 * few_of(0) >= 1024 * kSelWarps, "the histogram's room, and a KiB for each warp");
static_assert(few_of(0) % 4 == 0 && few_of(kMostWords) % 4 == 0 && few_of(32) % 4 == 0, "words of 16 bytes lie behind them");

// A list's tokens lo..hi, of which `need` of the largest keys are to be found.
struct List {
  const float* w;      // of token lo
  int n, need;
  int32_t* out;
  int lo;
};

// Inclusive sums over the CTA; *all receives the total.  A barrier lies between its uses.
__device__ __forceinline__ int scan_up(int v, int* sums, int* all) {
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) sums[wid] = x;
  __syncthreads();
  int total = 0, before = 0;
#pragma unroll
  for (int k = 0; k < kSelWarps; ++k) {
    if (k == wid) before = total;
    total += sums[k];
  }
  *all = total;
  return before + x;
}

// Any list: the key of the last kept token by its digits from above, a histogram of the candidates each; then
// the tokens in order, those above it kept and of those equal to it the first.  The list is read four times by
// one CTA: 4 sessions of 70 000 tokens in 48 layers and heads take 485 us, of 60 000 (select_once) 67.
__device__ __noinline__ void select_by_digits(const List& t, SelectShared& sh) {
  const int tid = threadIdx.x, lane = tid & 31;
  uint32_t have = 0;
  int need = t.need, shift = 32;
  while (shift > 0) {
    const int bits = shift > 11 ? 11 : shift;      // 11, 11, 10
    shift -= bits;
    __syncthreads();
    for (int b = tid; b < kBins; b += kSelThreads) sh.bins[b] = 0;
    __syncthreads();
    for (uint32_t j = tid; j < (uint32_t)t.n; j += kSelThreads) {
      const uint32_t k = order_key(__float_as_uint(t.w[j]));
      if (shift + bits == 32 || (k >> (shift + bits)) == (have >> (shift + bits)))
        atomicAdd(&sh.bins[k >> shift & ((1u << bits) - 1u)], 1);
    }
    __syncthreads();
    // from the top bin down: the bin in which `need` is reached
    constexpr int kPer = kBins / kSelThreads;
    int mine[kPer], sum = 0, all;
#pragma unroll
    for (int e = 0; e < kPer; ++e) sum += mine[e] = sh.bins[kBins - 1 - (tid * kPer + e)];
    int above = scan_up(sum, sh.sums[0], &all) - sum;
    if (above < need && above + sum >= need) {
      int e = 0;
      while (above + mine[e] < need) above += mine[e++];
      sh.digit = kBins - 1 - (tid * kPer + e);
      sh.before = above;
    }
    __syncthreads();
    have |= (uint32_t)sh.digit << shift;
    need -= sh.before;
  }
  int kept = 0, ties = 0;
  for (uint32_t j0 = 0; j0 < (uint32_t)t.n; j0 += kSelThreads) {
    const uint32_t j = j0 + tid;
    const uint32_t k = j < (uint32_t)t.n ? order_key(__float_as_uint(t.w[j])) : 0;
    const bool tie = k == have;
    int all;
    __syncthreads();
    const int rank = ties + scan_up(tie, sh.sums[0], &all);
    ties += all;
    const bool stay = k > have || (tie && rank <= need);
    const int at = kept + scan_up(stay, sh.sums[1], &all);
    kept += all;
    if (stay) t.out[at - 1] = t.lo + (int)j;
  }
}

// The bounds between which the border lies by a sample of the list, as bins of the key's first 12 bits (an
// eighth of an octave): at 3.5 deviations of the sample's rank, so that it lies outside in some 1 of 2000 lists.
__device__ __forceinline__ void bounds_by_sample(const List& t, SelectShared& sh) {
  const int tid = threadIdx.x;
  float x[kSample / kSelThreads];
#pragma unroll
  for (int e = 0; e < kSample / kSelThreads; ++e)
    x[e] = t.w[(uint32_t)(e * kSelThreads + tid) * (uint32_t)t.n / kSample];      // (n is at most 2^16)
  for (int b = tid; b < kBins / 4; b += kSelThreads) reinterpret_cast<int4*>(sh.bins)[b] = make_int4(0, 0, 0, 0);
  if (tid == 0) {
    sh.lo_key = 0;
    sh.hi_key = 0xffffffffu;
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < kSample / kSelThreads; ++e) {
    const uint32_t k = order_key(__float_as_uint(x[e]));
    atomicAdd(&sh.bins[k >> 21], k >> 20 & 1u ? 1 << 16 : 1);
  }
  __syncthreads();
  const float p = (float)t.need / (float)t.n, margin = 3.5f * sqrtf(p * (1.f - p) * kSample) + 1.f;
  const int r_hi = (int)(p * kSample - margin), r_lo = (int)(p * kSample + margin) + 1;
  constexpr int kPer = kBins / kSelThreads;
  uint32_t mine[kPer];
  int sum = 0, all;
#pragma unroll
  for (int e = 0; e < kPer; e += 4) {      // (a thread's bins downward)
    const int4 x = reinterpret_cast<const int4*>(sh.bins)[(kBins - (tid * kPer + e)) / 4 - 1];
    mine[e] = x.w, mine[e + 1] = x.z, mine[e + 2] = x.y, mine[e + 3] = x.x;
  }
#pragma unroll
  for (int e = 0; e < kPer; ++e) sum += (mine[e] & 0xffffu) + (mine[e] >> 16);
  int above = scan_up(sum, sh.sums[0], &all) - sum;
  if (above < r_lo && above + sum >= min(max(r_hi, 1), r_lo)) {
#pragma unroll
    for (int e = 0; e < 2 * kPer; ++e) {
      const uint32_t bin = (uint32_t)(2 * (kBins - 1 - (tid * kPer + e / 2)) + (e & 1 ? 0 : 1)) << 20;
      const int upto = above + (e & 1 ? mine[e / 2] & 0xffffu : mine[e / 2] >> 16);
      if (above < r_hi && upto >= r_hi) sh.hi_key = bin | 0xfffffu;
      if (above < r_lo && upto >= r_lo) sh.lo_key = bin;
      above = upto;
    }
  }
  __syncthreads();
}

// Inclusive sums over the warp.
__device__ __forceinline__ int warp_up(int x) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if ((int)(threadIdx.x & 31) >= o) x += y;
  }
  return x;
}

// A list of up to 32 * kMostWords tokens, read once: a word a 32 tokens says which are above the bounds, which
// have the lowest key in them (zeros do, where the border is among them), and which lie between; these are
// listed.  The border is then found among them: by their place between the bounds in kSelThreads steps, finer
// until at most 32 share one, which a warp ranks.  False where it is not found so: the bounds do not hold it,
// too many keys lie in them, or too many are equal at the border.
//
// What bounds it is instructions and the chain of barriers, not the list's bytes: so tokens are compared as numbers
// and told apart by votes (some nine instructions for 32 of them), and a lane goes through the few set bits of a
// word by itself.  12 sessions of 4000 to 30 000 tokens, 48 layers of 4 heads: 142 MB in 83 us in a graph, 1.7 TB/s, by
// digits 296.  Samples of 1024 and 512: 91 and 113, as more lies between the bounds.
__device__ __forceinline__ bool select_once(const List& t, SelectShared& sh, const OnceShared& o, int room) {
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int words = (t.n + 31) >> 5, batches = (t.n + 1023) >> 10;
  __syncthreads();
  if (tid == 0) sh.few = sh.above = sh.low = sh.last = 0;
  // (the two zeros are equal, and a NaN is not at or below any bound)
  float lo_x = -INFINITY, hi_x = INFINITY;
  if (t.n > room) {
    bounds_by_sample(t, sh);
    lo_x = number_of(sh.lo_key);
    hi_x = number_of(sh.hi_key);
  } else {
    __syncthreads();
  }
  constexpr int kUnroll = 8;
  int n_above = 0, n_low = 0;
  auto some_words = [&](int w0, auto full) {
    constexpr bool kFull = decltype(full)::value;
    float x[kUnroll];
    const float* from = t.w + 32 * w0 + lane;
    const int end = t.n - 32 * w0 - lane;
#pragma unroll
    for (int e = 0; e < kUnroll; ++e) x[e] = kFull || 32 * e < end ? __ldcs(from + 32 * e) : 0.f;
#pragma unroll
    for (int e = 0; e < kUnroll; ++e) {
      const bool there = kFull || 32 * e < end, to_hi = x[e] <= hi_x;
      uint4 v;
      v.x = __ballot_sync(0xffffffffu, there && !to_hi);
      v.y = __ballot_sync(0xffffffffu, there && x[e] == lo_x);
      v.z = __ballot_sync(0xffffffffu, there && x[e] > lo_x && to_hi);
      v.w = 0;
      if (lane == 0) o.word[w0 + e] = v;
    }
  };
  for (int b = wid; b < batches; b += kSelWarps) {
#pragma unroll 1
    for (int g = 0; g < 32; g += kUnroll) {
      if (1024 * b + 32 * (g + kUnroll) <= t.n) some_words(32 * b + g, std::true_type());
      else some_words(32 * b + g, std::false_type());
    }
    __syncwarp();
    // a lane a word: those between are listed, in any order
    const uint4 v = o.word[32 * b + lane];
    n_above += __popc(v.x);
    n_low += __popc(v.y);
    const int mine = __popc(v.z), upto = warp_up(mine);
    int at = 0;
    if (lane == 31 && upto) at = atomicAdd(&sh.few, upto);
    at = __shfl_sync(0xffffffffu, at, 31) + upto - mine;
    for (uint32_t m = v.z; m; m &= m - 1, ++at)
      if (at < room) o.at[at] = (uint16_t)(1024 * b + 32 * lane + __ffs(m) - 1);
    __syncwarp();
  }
  n_above = __reduce_add_sync(0xffffffffu, n_above);
  n_low = __reduce_add_sync(0xffffffffu, n_low);
  if (lane == 0) {
    atomicAdd(&sh.above, n_above);
    atomicAdd(&sh.low, n_low);
  }
  __syncthreads();
  const int few = sh.few;
  int r = t.need - sh.above;      // of those in the bounds
  if (few > room || r < 0 || r > few + sh.low) return false;
  auto keep = [&](int j) { atomicOr(&o.word[j >> 5].x, 1u << (j & 31)); };
  if (r >= few) {
    // all between, and of the lowest ones the first
    for (int j = tid; j < few; j += kSelThreads) keep(o.at[j]);
    if (r > few) {
      const int per = (words + kSelThreads - 1) / kSelThreads;
      const int w0 = min(tid * per, words), w1 = min(w0 + per, words);
      int mine = 0, all;
      for (int w = w0; w < w1; ++w) mine += __popc(o.word[w].y);
      int left = r - few - (scan_up(mine, sh.sums[0], &all) - mine);
      for (int w = w0; w < w1 && left > 0; ++w) {
        uint32_t x = o.word[w].y;
        const int have = __popc(x);
        if (have > left) {
          uint32_t rest = x;
          for (int k = 0; k < left; ++k) rest &= rest - 1;
          x ^= rest;
        }
        atomicOr(&o.word[w].x, x);
        left -= have;
      }
    }
  } else if (r > 0) {
    const uint32_t lo_key = order_key(__float_as_uint(lo_x)), hi_key = order_key(__float_as_uint(hi_x));
    const uint32_t width = hi_key - lo_key - 1;      // of key - lo_key - 1 at most
    int shift = max(0, 32 - kStepBits - __clz(width | 1u)), up = 32;
    uint32_t at = 0;      // (key - lo_key - 1) >> up of the border
    for (;;) {
      sh.steps[tid] = 0;
      __syncthreads();
      const uint32_t digits = up - shift >= 32 ? ~0u : (1u << (up - shift)) - 1u;
      for (int j = tid; j < few; j += kSelThreads) {
        uint32_t d;
        if (up == 32) {
          d = order_key(__float_as_uint(t.w[o.at[j]])) - lo_key - 1;
          o.key[j] = d;
        } else {
          d = o.key[j];
        }
        if (up == 32 || d >> up == at) atomicAdd(&sh.steps[d >> shift & digits], 1);
      }
      __syncthreads();
      const int mine = sh.steps[kSelThreads - 1 - tid];
      int all;
      const int upto = scan_up(mine, sh.sums[0], &all);
      if (upto - mine < r && upto >= r) {
        sh.digit = kSelThreads - 1 - tid;
        sh.before = upto - mine;
        sh.inside = mine;
      }
      __syncthreads();
      at = (up == 32 ? 0u : at << (up - shift)) + (uint32_t)sh.digit;
      r -= sh.before;
      up = shift;
      if (sh.inside <= 32) break;
      if (shift == 0) return false;
      shift = max(0, shift - kStepBits);
    }
    for (int j = tid; j < few; j += kSelThreads) {
      const uint32_t d = o.key[j] >> up;
      if (d > at) {
        keep(o.at[j]);
      } else if (d == at) {
        const int k = atomicAdd(&sh.last, 1);
        sh.last_key[k] = o.key[j];
        sh.last_at[k] = o.at[j];
      }
    }
    __syncthreads();
    if (wid == 0) {
      const int count = sh.last;
      const uint32_t k = lane < count ? sh.last_key[lane] : 0u;
      const int where = lane < count ? sh.last_at[lane] : 0;
      int rank = 0;
      for (int j = 0; j < count; ++j) {
        const uint32_t kj = __shfl_sync(0xffffffffu, k, j);
        const int wj = __shfl_sync(0xffffffffu, where, j);
        rank += kj > k || (kj == k && wj < where);
      }
      if (lane < count && rank < r) keep(where);
    }
  }
  __syncthreads();
  // how many each 1024 tokens keep; then what comes before them, and their numbers through shared memory
  for (int b = wid; b < batches; b += kSelWarps) {
    const int all = __reduce_add_sync(0xffffffffu, __popc(o.word[32 * b + lane].x));
    if (lane == 0) o.batch[b] = all;
  }
  __syncthreads();
  uint16_t* const numbers = reinterpret_cast<uint16_t*>(o.key) + 512 * wid;
  for (int b = wid; b < batches; b += kSelWarps) {
    int before = 0;
    for (int k = lane; k < b; k += 32) before += o.batch[k];
    int32_t* out = t.out + __reduce_add_sync(0xffffffffu, before);
    const uint32_t mine = o.word[32 * b + lane].x;
#pragma unroll 1
    for (int half = 0; half < 2; ++half) {      // (512 tokens' numbers at once)
      const uint32_t x = lane >> 4 == half ? mine : 0u;
      const int upto = warp_up(__popc(x)), all = __shfl_sync(0xffffffffu, upto, 31);
      int at = upto - __popc(x);
      for (uint32_t m = x; m; m &= m - 1) numbers[at++] = (uint16_t)(32 * lane + __ffs(m) - 1);
      __syncwarp();
      const int from = t.lo + 1024 * b;
      for (int k = lane; k < all; k += 32) out[k] = from + numbers[k];
      out += all;
      __syncwarp();
    }
  }
  return true;
}

// One list: a request's tokens in a layer and head.  Tokens before lo and from hi on stay,
// and of those between the `need` of largest key.
// 256 threads, and six CTAs an SM where contexts hold up to some 29 000 tokens: with 128, 512 and 64 threads a list the
// same lists took 96, 104 and 129 us.  Shared memory is sized by the longest context that the pool and the weights have
// room for, as the lengths are on the device: 82 KB from 65 536 tokens on, two CTAs an SM, where 12 lists of 6000 to
// 29 000 tokens in 192 layers and heads take 196 us in place of 110.
__global__ void __launch_bounds__(kSelThreads, 6) k_select_kept(const __grid_constant__ SelectArgs a, int n, int words) {
  __shared__ SelectShared sh;
  extern __shared__ __align__(16) uint32_t dyn[];
  const int tid = threadIdx.x;
  const int lists = a.p.J / 2 * a.H, turn = blockIdx.x / lists, list = blockIdx.x - turn * lists;
  const int layer = list / a.H, head = list - layer * a.H;
  if (tid == 0) sh.bins = reinterpret_cast<int*>(dyn);
  dep_wait();
  int i = turn;
  if (n > 1 && n <= kTurns) {
    // the longest first, so that none of them ends last
    if (tid < n) {
      const int sid = a.sids[tid];
      sh.ctx[tid] = sid >= 0 && sid < a.p.S ? a.p.sess[sid].ctx_tokens : -1;
    }
    __syncthreads();
    if (tid < n) {
      const int mine = sh.ctx[tid];
      int before = 0;
      for (int j = 0; j < n; ++j) before += sh.ctx[j] > mine || (sh.ctx[j] == mine && j < tid);
      if (before == turn) sh.turn = tid;
    }
    __syncthreads();
    i = sh.turn;
  }
  const int sid = a.sids[i];
  int32_t* out = a.kept + ((int64_t)i * lists + list) * a.most;
  int keep = a.keeps[i], c = 0;
  bool bad = sid < 0 || sid >= a.p.S || keep < 0 || keep > a.most;
  if (!bad) {
    c = a.p.sess[sid].ctx_tokens;
    bad = c > a.w.tokens;
  }
  if (bad) {
    if (list == 0 && tid == 0) report(a.p.ctl, LV_ERR_BOUNDS, i);
    keep = 0;
  }
  keep = min(keep, c);
  const int lo = min(a.first, keep), hi = max(c - min(a.last, keep - lo), lo);
  List t;
  t.n = hi - lo;
  t.need = keep - lo - (c - hi);
  t.lo = lo;
  t.out = out + lo;
  t.w = a.w.data + layer * a.w.layer_stride + (bad ? 0 : sid) * a.w.session_stride + head * a.w.head_stride + lo;
  // the first and last ones, and what is behind the list.  (Unsigned here and below: the step past the end of a list
  // of 2^31 - 1 leaves 31 bits.)
  for (uint32_t j = tid; j < (uint32_t)lo; j += kSelThreads) out[j] = (int)j;
  if (keep > 0)
    for (uint32_t j = tid; j < (uint32_t)(c - hi); j += kSelThreads) out[lo + t.need + j] = hi + (int)j;
  for (uint32_t j = (uint32_t)keep + tid; j < (uint32_t)a.most; j += kSelThreads) out[j] = -1;
  if (t.need == 0) return;
  if (t.need == t.n) {
    for (uint32_t j = tid; j < (uint32_t)t.n; j += kSelThreads) t.out[j] = lo + (int)j;
    return;
  }
  if (t.n > 32 * words || !select_once(t, sh, OnceShared(dyn, words), few_of(words)))
    select_by_digits(t, sh);
}

// ---------------------------------------------------------------- compaction
constexpr int kCheckThreads = 1024, kCheckCtas = 16;

// Request blockIdx.x / kCheckCtas by a cluster: its session, that its blocks are in HBM, and its lists, which
// have to ascend within the context.  lens[i] receives what it may be cut to, or -1 where nothing moves.
// The lists are read once here and once by k_compact: a kernel that moved rows while it checked could stop half-way.
__global__ void __cluster_dims__(kCheckCtas, 1, 1) __launch_bounds__(kCheckThreads, 1)
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
#pragma unroll 4
        for (uint32_t j = tid; j < (uint32_t)keep; j += kCheckThreads) {
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
// nothing that an earlier one wrote over.  A row's vectors lie together; `parts` CTAs share them.  A chunk's
// places are looked up (list, then table) while the chunk before it is on its way.
// What bounds it: HBM, both ways.  4 sessions of 6000 to 14 000 tokens cut to a quarter in 48 layers of 4 heads of
// 128, bf16: 1.9 GB in 329 us with the checks, 5.8 TB/s, 410 before the look-ups were taken ahead.
constexpr int kMoveRows = 256;      // of a chunk at most
template <typename V, int U>
__global__ void __launch_bounds__(kMoveThreads, 4) k_compact(const __grid_constant__ CompactArgs a, int vecs, int part_vecs) {
  // of a chunk's rows: where from, where to (null: it stays); three chunks', as a thread may write the next one's
  // while another stores by the one's before
  __shared__ V* place[3][2][kMoveRows];
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
  const int v0 = part * part_vecs, mine = min(part_vecs, vecs - v0);
  V* const base = reinterpret_cast<V*>(a.p.kv[2 * layer + kv]) + head * vecs + v0;
  const uint64_t page_vecs = (uint64_t)a.p.P / sizeof(V);
  const uint32_t T = a.p.T, token_vecs = (uint32_t)a.H * vecs;
  auto slot = [&](int token) -> V* {
    const uint32_t b = a.t_shift >= 0 ? (uint32_t)token >> a.t_shift : (uint32_t)token / T;
    return base + (uint64_t)table[b] * page_vecs + (uint64_t)((uint32_t)token - b * T) * token_vecs;
  };
  const int rows = min(kMoveThreads * U / part_vecs, kMoveRows);      // of a chunk
  V *from = nullptr, *to = nullptr;
  auto look = [&](uint32_t j) {      // thread j's row of the next chunk
    from = to = nullptr;
    if (tid >= rows || j >= (uint32_t)keep) return;
    const int token = kept[j];
    if (token == (int)j) return;
    from = slot(token);
    to = slot((int)j);
  };
  look(tid);
  int buf = 0;
  if (tid < rows) {
    place[0][0][tid] = from;
    place[0][1][tid] = to;
  }
  __syncthreads();
  // this thread's vectors: the same rows and columns of every chunk
  int row[U], col[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int at = u * kMoveThreads + tid;
    row[u] = at / part_vecs;
    col[u] = at - row[u] * part_vecs;
    if (row[u] >= rows || col[u] >= mine) row[u] = -1;
  }
  for (uint32_t j0 = 0; j0 < (uint32_t)keep; j0 += rows) {
    const int next = buf == 2 ? 0 : buf + 1;
    V x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const V* p = row[u] >= 0 ? place[buf][0][row[u]] : nullptr;
      if (p) x[u] = p[col[u]];
    }
    look(j0 + rows + tid);
    if (tid < rows) {
      place[next][0][tid] = from;
      place[next][1][tid] = to;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u) {
      V* p = row[u] >= 0 ? place[buf][1][row[u]] : nullptr;
      if (p) p[col[u]] = x[u];
    }
    buf = next;
  }
  if (part || kv) return;
  if (a.w.data) {
    float* w = a.w.data + layer * a.w.layer_stride + sid * a.w.session_stride + head * a.w.head_stride;
    for (uint32_t j0 = 0; j0 < (uint32_t)keep; j0 += kMoveThreads) {
      const uint32_t j = j0 + tid;
      const float y = j < (uint32_t)keep ? w[kept[j]] : 0.f;
      __syncthreads();
      if (j < (uint32_t)keep) w[j] = y;
    }
    __syncthreads();
    for (uint32_t j = (uint32_t)keep + tid; j < (uint32_t)c; j += kMoveThreads) w[j] = 0.f;
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
    if (p.incl) drop_clean(p, at);
    if (e >= 0 && e < p.hbm_pages) {
      p.own_hbm[e] = kOwnerNone;
      ++in_hbm;
    } else if (e <= -2 && -(long long)e - 2 < p.host_pages) {
      p.own_host[-e - 2] = kOwnerNone;
      ++in_host;
    }
  }
  // (an allocation may run beside this one, and takes a page as soon as its bit is clear: the owner that it then
  // writes comes after the word above)
  __threadfence();
  for (int b = nb + tid; b < end; b += kCutThreads) {
    const size_t at = (size_t)sid * p.maxB + b;
    const int e = p.table[at];
    p.table[at] = -1;
    if (e >= 0 && e < p.hbm_pages) {
      atomicAnd(&p.bits_hbm[e >> 5], ~(1u << (e & 31)));
    } else if (e <= -2 && -(long long)e - 2 < p.host_pages) {
      const int s = -e - 2;
      atomicAnd(&p.bits_host[s >> 5], ~(1u << (s & 31)));
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

cudaError_t configure_keep() {
  const cudaError_t e = cudaFuncSetAttribute(k_compact_check, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e != cudaSuccess) return e;
  return cudaFuncSetAttribute(k_select_kept, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)OnceShared::bytes(kMostWords));
}

cudaError_t launch_select_kept(const SelectArgs& a, int n, cudaStream_t s) {
  // words for the longest context that there may be
  const int64_t tokens = (int64_t)a.p.maxB * a.p.T < a.w.tokens ? (int64_t)a.p.maxB * a.p.T : a.w.tokens;
  const int words = (int)((tokens + 1023) / 1024 * 32 < kMostWords ? (tokens + 1023) / 1024 * 32 : kMostWords);
  return launch_dependent(k_select_kept, dim3(a.p.J / 2 * a.H * n), kSelThreads, OnceShared::bytes(words), s, a, n, words);
}

cudaError_t launch_compact(const CompactArgs& a, int n, int row_bytes, int num_sms, cudaStream_t s) {
  const cudaError_t e = launch_dependent(k_compact_check, dim3(n * kCheckCtas), kCheckThreads, 0, s, a);
  if (e != cudaSuccess) return e;
  const int lists = a.p.J / 2 * a.H;
  const int vecs = row_bytes % 16 == 0 ? row_bytes / 16 : row_bytes;
  // rows shared by several CTAs, down to 32 bytes of each, where there are few lists: the lists of one layer do not
  // fill the SMs, and a list's rows have to be moved in order
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
