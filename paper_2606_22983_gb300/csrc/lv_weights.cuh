// Attention weights added up for the cached tokens: the launches of lv_weights.cu, and how its kernels find
// their work.
#pragma once

#include "lv_batch.cuh"

namespace lv {

// A unit whose rows several CTAs share: where its pieces' sums lie, and the weights that they go to.
struct alignas(16) CutUnit {
  float* w;
  int32_t keys, pieces, piece0, pad[3];
};

struct WeightArgs {
  const uint8_t* k;        // the layer's K sub-page array
  int64_t P;
  uint32_t hbm_pages;
  int32_t T, t_shift, H, D, G, S;
  int32_t maxB;
  const int32_t* tables;       // the step's, by request
  const int32_t* pool_table;   // the pool's, by session
  const int32_t* row_starts;
  const PlanReq* reqs;
  const PlanReq* pre_reqs;     // of the prefixes, where the step has some
  const StepHead* head;
  int32_t* tickets;            // units given out, CTAs done; zero between calls
  uint32_t* refused;           // [kMostSegments / 32] a bit a segment (every CTA writes the same)
  CutUnit* cuts;               // [cut_units]
  int32_t* cut_count;          // of them
  float* pieces;               // [cut_pieces][256] their sums
  int32_t cut_units, cut_pieces;      // 0: none is cut
  const uint8_t* q;
  int64_t q_row, q_head;       // in elements
  const float* lse;            // [num_tokens][Hq]
  float* w;                    // of the layer
  int64_t w_session, w_head;
  int32_t w_tokens;
  int32_t num_tokens, last;
  int32_t window, sinks;
  float scale;                 // scale * log2(e)
  long long* ctl;
  long long wait_ns;
  int32_t hold;                // LV_HOLD_NONE but in a self-test
  StepHead* head_out;          // the same head, for a wait that ran out
  const int32_t* no_lse;       // one where the last attention on the step did nothing
};

// Sums of many terms in 32 bits: what the additions lose is kept beside them (Kahan), so that the sum's error
// does not grow with a prompt's length (32 768 rows of a key added one after the other were off by 1.6e-6).
struct LongSum {
  float sum = 0.f, lost = 0.f;
#ifdef __CUDACC__
  __device__ __forceinline__ void add(float x) {
    const float y = x - lost, t = sum + y;
    lost = fabsf(t) < INFINITY ? (t - sum) - y : 0.f;      // (an infinite sum loses nothing, and stays)
    sum = t;
  }
#endif
};

// The tensor-core kernel's maps: K in boxes of 64 columns and box_rows keys; the queries in boxes of 64 columns,
// G heads and 128 / G rows, or few_rows of them (null: plain loads).
struct WeightMaps {
  const CUtensorMap* k;
  const CUtensorMap* q;
  const CUtensorMap* q_few;
  int box_rows, few_rows;
};
cudaError_t launch_weights_tc(const WeightArgs& a, const WeightMaps& m, bool bf16, int dp, int num_sms, cudaStream_t s);
cudaError_t configure_weights_tc();
cudaError_t launch_weights_plain(const WeightArgs& a, bool bf16, int dp, int num_sms, cudaStream_t s);
cudaError_t configure_weights();
constexpr int kMostSegments = 2 * 4096;

// The tensor-core kernel's units have pieces of about a kGoes-th of what a CTA has to do in all, and of kMinPiece
// products at least.
// One prompt of 4096 with 4 KV heads is 64 units, of which the longest has 256 products and an SM 57 in all: 260 us
// whole, 89 cut; 4 of them 283 and 264, 500 tokens at 16 000 keys 73 either way.  2 and 4 goes: 293 and 267 for the 4; with
// 16 products at least 86 for the one at 4 goes, with 4 no change.
constexpr int kGoes = 8, kMinPiece = 8, kCutUnits = 512;
// Packed rows of a product, whole tokens of G.
__host__ __device__ constexpr int product_rows(int G) { return G > 128 ? 128 : 128 / G * G; }

#ifdef __CUDACC__
// The weights' work: a segment is the context of one request with the request's rows, or a prefix with the rows
// of all that continue it; a unit is kKeys keys of a segment for one KV head, with all rows that see some of
// them.  So every word of the weights belongs to one unit, whose sums are made in one order.  Long units are cut into
// pieces by rows, whose sums a second kernel adds up in their order.
struct Segment {
  int first, tokens, qrow;     // position of its first row; its rows' tokens; the first of them in the step
  int keys;
  int sid, req;                // req: -1 for a prefix
};

struct Unit {
  Segment g;
  int head, key0;
  int t0, t1;                  // tokens [t0, t1) of the segment see some of its keys
  int products;                // the tensor-core kernel's
};

// Units are taken in kClasses goes, those that most rows see first, so that no long one begins last: a
// segment's keys are seen by the fewer rows the later they are, so a class is a stretch of them.  (In the order of the
// keys the last CTA of 4 prompts of 4096 had 1.66 times the mean's products.)
constexpr int kClasses = 4;

// What a CTA knows of the segments, divided among NT of its threads.
template <int NT>
struct SegmentIndex {
  int before[kClasses * NT + 1];             // units before thread t's segments in class c
  int ws[NT / 32];
  int most, seen;                            // rows' tokens of a segment, and that see a unit's keys
  int cuts[kClasses];                        // pieces of a unit of the class at most
  int tickets[kClasses + 1];                 // pieces before the class
  unsigned long long products;               // in all, about
};

// Whether the step on the device is one that the call may work on, and its last attention ran (one that was refused, or
// that gave up over the prefixes, has left the lse of another step or none).
__device__ __forceinline__ bool weights_fit(const WeightArgs& a, const StepHead& step) {
  return step.kind >= 0 && step.num_tokens <= a.num_tokens && *a.no_lse == 0;
}

__device__ __forceinline__ Segment segment_of(const WeightArgs& a, int n, int s) {
  const bool pre = s >= n;
  const PlanReq r = load_words(pre ? &a.pre_reqs[s - n] : &a.reqs[s]);
  Segment g;
  g.first = r.first;
  g.tokens = r.len;
  g.qrow = r.qrow;
  g.keys = r.len == 0 ? 0 : r.first + (pre ? 1 : r.len);
  g.sid = r.sid & (kSharedReq - 1);
  g.req = pre ? -1 : s;
  return g;
}

// Which tokens of g see keys of [key0, key0 + keys): those from the first key's position on, and under a
// window up to where it has left the last one.
__device__ __forceinline__ Unit unit_of(const WeightArgs& a, const Segment& g, int head, int key0, int keys) {
  Unit u{g, head, key0, 0, g.tokens, 0};
  if (g.req < 0) return u;
  if (a.last > 0) u.t0 = max(0, g.tokens - a.last);
  u.t0 = max(u.t0, key0 - g.first);
  if (a.window > 0 && key0 >= a.sinks)
    u.t1 = (int)min((long long)u.t1, (long long)key0 + keys - 1 + a.window - g.first);
  return u;
}

// Whether a token of a segment counts, and whether it sees a key.
__device__ __forceinline__ bool sees(const WeightArgs& a, const Segment& g, int token, int key) {
  if (g.req < 0) return key < g.keys;
  const int p = g.first + token;
  return key <= p && (a.window == 0 || key > p - a.window || key < a.sinks);
}
__device__ __forceinline__ bool counts(const WeightArgs& a, const Segment& g, int n, int token) {
  if (a.last <= 0) return true;
  if (g.req >= 0) return token >= g.tokens - a.last;
  // the request of this row: the last one that does not begin after it and has rows
  const int r = g.qrow + token;
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.row_starts[mid] <= r) lo = mid;
    else hi = mid - 1;
  }
  return r >= a.row_starts[lo + 1] - a.last;
}

// Tiles of kKeys keys of g before the end of class c.
template <int kKeys>
__device__ __forceinline__ int class_end(const Segment& g, int c, int most) {
  const int all = (g.keys + kKeys - 1) / kKeys;
  if (c == kClasses - 1) return all;
  const int more_than = (int)((long long)most * (kClasses - 1 - c) / kClasses);      // tokens see its keys
  if (g.tokens <= more_than) return 0;
  return g.req < 0 ? all : min(all, (int)(((long long)g.first + g.tokens - more_than + kKeys - 1) / kKeys));
}

// How many tokens see some of `keys` keys, behind the sinks.
__device__ __forceinline__ int most_seen(const WeightArgs& a, const Segment& g, int keys) {
  if (g.req < 0) return g.tokens;
  const int rows = a.last > 0 ? min(a.last, g.tokens) : g.tokens;
  return a.window > 0 ? (int)min((long long)rows, (long long)a.window + keys) : rows;
}
// About how many products of step_rows rows a segment has.
__device__ __forceinline__ unsigned long long products_of(const WeightArgs& a, const Segment& g, int rows, int keys, int step_rows) {
  const float seen = (float)rows * (g.keys - (g.req < 0 || a.window > 0 ? 0.f : 0.5f * rows));
  return (unsigned long long)(seen * a.H * a.G / ((float)keys * step_rows));
}

// Every thread of the CTA (whole warps) calls it: fills x and returns the units in all, or with kCut the pieces, of
// products of step_rows rows.  first_of: room for a word a session.
// The segments whose session an earlier one has, or that the weights have no room for, are refused (their
// units are empty).
template <int NT, int kKeys, bool kCut>
__device__ int index_segments(const WeightArgs& a, const StepHead& step, SegmentIndex<NT>& x, int* first_of, int step_rows) {
  const int n = step.requests & (kSharedStep - 1), count = step.requests >= kSharedStep ? 2 * n : n;
  const int tid = threadIdx.x, lane = tid & 31;
  for (int s = tid; s < a.S; s += blockDim.x) first_of[s] = kMostSegments;
  if (tid == 0) {
    x.most = x.seen = 0;
    x.products = 0;
  }
  __syncthreads();
  for (int s = tid; s < count; s += blockDim.x) {
    const Segment g = segment_of(a, n, s);
    if (g.keys > 0) atomicMin(&first_of[g.sid], s);
  }
  __syncthreads();
  for (int s0 = tid - lane; s0 < count; s0 += blockDim.x) {
    const int s = s0 + lane;
    bool again = false, far = false;
    if (s < count) {
      const Segment g = segment_of(a, n, s);
      again = g.keys > 0 && first_of[g.sid] != s;
      far = g.keys > a.w_tokens;
      if ((again || far) && blockIdx.x == 0) report(a.ctl, again ? LV_ERR_DOUBLE_MAP : LV_ERR_BOUNDS, s < n ? s : s - n);
    }
    const uint32_t votes = __ballot_sync(0xffffffffu, again || far);
    if (lane == 0) a.refused[s0 >> 5] = votes;
  }
  const int per = (count + NT - 1) / NT, s0 = min(tid * per, count), s1 = tid < NT ? min(s0 + per, count) : s0;
  int longest = 0;
  [[maybe_unused]] int seen = 0;
  for (int s = s0; s < s1; ++s) {
    const Segment g = segment_of(a, n, s);
    longest = max(longest, g.tokens);
    if constexpr (kCut) seen = max(seen, most_seen(a, g, kKeys));
  }
  longest = __reduce_max_sync(0xffffffffu, longest);
  if (lane == 0 && longest) atomicMax(&x.most, longest);
  if constexpr (kCut) {
    seen = __reduce_max_sync(0xffffffffu, seen);
    if (lane == 0 && seen) atomicMax(&x.seen, seen);
  }
  __syncthreads();
  const int most = x.most;
  const bool cuts = kCut && (long long)x.seen * a.G > (long long)step_rows * kMinPiece;
  if (cuts) {
    unsigned long long products = 0;
    for (int s = s0; s < s1; ++s) {
      const Segment g = segment_of(a, n, s);
      products += products_of(a, g, most_seen(a, g, kKeys), kKeys, step_rows);
    }
    if (products) atomicAdd(&x.products, products);
  }
  int total = 0;
#pragma unroll 1
  for (int c = 0; c < kClasses; ++c) {
    int mine = 0;
    for (int s = s0; s < s1; ++s) {
      const Segment g = segment_of(a, n, s);
      mine += a.H * (class_end<kKeys>(g, c, most) - (c ? class_end<kKeys>(g, c - 1, most) : 0));
    }
    int sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += y;
    }
    if (lane == 31 && tid < NT) x.ws[tid >> 5] = sum;
    __syncthreads();
    int before = total;
    for (int v = 0; v < NT / 32; ++v) {
      if (v < tid >> 5) before += x.ws[v];
      total += x.ws[v];
    }
    if (tid < NT) x.before[c * NT + tid + 1] = before + sum;
    __syncthreads();
  }
  if (tid == 0) x.before[0] = 0;
  if (kCut && tid == 0) {
    // the pieces of a class's longest unit, for all of them: a class that finds no room is left whole, as those behind
    // it are, which are shorter
    x.cuts[0] = 1;
    x.tickets[kClasses] = total;
    if (blockIdx.x == 0) *a.cut_count = 0;
  }
  if (tid == 0 && cuts) {
    const long long goal = max((long long)kMinPiece, (long long)x.products / ((long long)gridDim.x * kGoes));
    bool cut = true;
    int units = 0, tickets = 0;
    for (int c = 0; c < kClasses; ++c) {
      const int here = x.before[(c + 1) * NT] - x.before[c * NT];
      int cuts = 1;
      if (cut) {
        const long long rows = min((long long)most * (kClasses - c) / kClasses, (long long)x.seen) * a.G;
        cuts = (int)min((rows + step_rows * goal - 1) / (step_rows * goal), 1024ll);
        cut = cuts > 1 && units + here <= a.cut_units && tickets + (long long)here * cuts <= a.cut_pieces;
        if (!cut) cuts = 1;
      }
      x.cuts[c] = cuts;
      x.tickets[c] = tickets;
      units += here;
      if (cut && blockIdx.x == 0) *a.cut_count = units;
      tickets += here * cuts;
    }
    x.tickets[kClasses] = tickets;
  }
  __syncthreads();
  return kCut ? x.tickets[kClasses] : total;
}

// Unit or piece `ticket` of all; no tokens where there is nothing to do.  of: the piece of a cut unit, -1 of a whole one.
template <int NT, int kKeys, bool kCut>
__device__ __forceinline__ Unit find_unit(const WeightArgs& a, const StepHead& step, const SegmentIndex<NT>& x, int ticket,
                                          int step_rows, int& of) {
  of = -1;
  int in = 0, cuts = kCut ? x.cuts[0] : 1, piece = 0, u = ticket;
  if (kCut && cuts > 1) {
    while (in + 1 < kClasses && ticket >= x.tickets[in + 1]) ++in;
    cuts = x.cuts[in];
    u = (ticket - x.tickets[in]) / cuts;
    piece = ticket - x.tickets[in] - u * cuts;
    u += x.before[in * NT];
  }
  const int n = step.requests & (kSharedStep - 1), count = step.requests >= kSharedStep ? 2 * n : n;
  const int per = (count + NT - 1) / NT;
  int lo = 0, hi = kClasses * NT - 1;      // the last thread and class whose segments do not begin after u
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (x.before[mid] <= u) lo = mid;
    else hi = mid - 1;
  }
  const int c = lo / NT, most = x.most;
  int s = (lo - c * NT) * per, off = u - x.before[lo], t0;
  Segment g = segment_of(a, n, s);
  for (;;) {
    t0 = c ? class_end<kKeys>(g, c - 1, most) : 0;
    const int units = a.H * (class_end<kKeys>(g, c, most) - t0);
    if (off < units) break;
    off -= units;
    g = segment_of(a, n, ++s);
  }
  const int tile = off / a.H;
  Unit out = unit_of(a, g, off - tile * a.H, (t0 + tile) * kKeys, kKeys);
  if (a.refused[s >> 5] >> (s & 31) & 1u) out.t1 = out.t0;
  if (kCut && cuts > 1) {      // (its rows in pieces of whole products; the last ones may be none)
    const int tokens = step_rows / a.G, products = max(0, out.t1 - out.t0 + tokens - 1) / tokens;
    const int size = max((products + cuts - 1) / cuts, kMinPiece), pieces = (products + size - 1) / size;
    if (piece == 0)
      a.cuts[u] = CutUnit{a.w + g.sid * a.w_session + out.head * a.w_head + out.key0, min(kKeys, g.keys - out.key0),
                          pieces > 1 ? pieces : 0, ticket, {}};
    if (pieces > 1) of = ticket;
    const long long t0 = out.t0 + (long long)piece * size * tokens;
    out.t1 = (int)min((long long)out.t1, t0 + (long long)size * tokens);
    out.t0 = (int)min(t0, (long long)out.t1);
  }
  return out;
}
#endif

}  // namespace lv
