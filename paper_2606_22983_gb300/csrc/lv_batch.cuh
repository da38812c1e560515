// A serving step on resident KV: what its plan leaves on the device, and the launches of
// lv_batch.cu (plan, KV write), lv_attend.cu (attention of few rows a request, join of split
// work) and lv_attend_tc.cu (attention of many rows, tcgen05).
#pragma once

#include <cuda.h>
#include <utility>

#include "lv_internal.cuh"

namespace lv {

// The rows of one request in one tile of the attention's work: up to the kernel's tile height
// of packed rows, packed row R of a request being query head R % G (of its KV head) of new
// token R / G, so that the G heads that share a KV head read it once.  Its keys are cut into
// units of the kernel's size: first the units that hold sinks, then those from the window on.
struct AttnTile {
  int64_t before;       // where it starts on the line
  int32_t req;
  int32_t row0;         // its first packed row
  int32_t rows;         // its packed rows
  int32_t units;        // units a head group
  int32_t sink_units;   // unit u < sink_units starts at key u * unit,
  int32_t win_unit;     // the others at key (win_unit + u - sink_units) * unit
  int32_t first;        // position of the request's first new token
  int32_t qrow;         // its row in the step's tensors
  int32_t kv_lo;        // first key in the window of the tile's first row
  int32_t kv_hi;        // keys up to the tile's last row
};
static_assert(sizeof(AttnTile) == 48, "read as three 16-byte words");

// A pair of a tile and a KV head takes a stretch of a line: `lead` places for what it costs to begin
// and end it, then one for each of its units.  A CTA takes `share` places on, whatever pairs that
// cuts; the one that finishes the last piece of a cut pair joins its pieces, in their order.  Where
// there are CTAs enough that each pair may begin one of its own, the stretches are whole shares
// instead, with empty places at their ends (lead -1), and short pairs are not cut.
// The kernel for many rows has one line of all pairs, tile after tile and head after head in it.
// The one for few rows has a line of the tiles for each KV head, and H CTAs beside one another take
// the same places of theirs: they read the same pages, whose H rows of a token lie together, at
// about the same time.
struct CtaWork {        // what a CTA starts from
  AttnTile t;           // of its first place
  int64_t begin, end;   // its places; begin == end: none
  int32_t share, lead;
  int32_t tile;
  int32_t pad;
};
static_assert(sizeof(CtaWork) == 80, "read as five 16-byte words");

// What the step's tables and work list are for, written by the plan after them.  The calls that use them
// take their kernel and their rows from the plan that the host made last, which in a replayed graph need
// not be the plan that the device made last: they compare, and do nothing where a list of the other
// kernel's units or a step of more rows than their tensors have would be read.
struct StepHead {
  int32_t kind;         // AttnKind of the work list; -1: none (nothing planned, or a wait ran out: the pieces
                        // that came are counted, and another call on the list would join them as its own)
  int32_t num_tokens;   // the plan's; rows past it are of no request whatever positions and slots hold
  int32_t live;         // rows of requests
  int32_t pad;
};
static_assert(sizeof(StepHead) == 16, "read as one word");

struct PlanReq {        // per request, from the plan's first kernel to its second
  int32_t first, len, qrow, pad;   // len 0: left out
};

struct PlanArgs {
  DevPool p;
  const int32_t* sids;
  const int32_t* firsts;   // or null
  const int32_t* lens;
  int32_t n, num_tokens, max_len;
  int32_t G;               // query heads a KV head
  int32_t line_heads;      // KV heads in a line: all, or 1
  int32_t tile_rows, unit_shift;   // of the attention kernel that will run (its unit's log2)
  int32_t lead;            // places of the line ahead of a pair's units
  int32_t min_share;       // places a CTA takes at least
  int32_t uncut;           // units of a pair that is better not cut
  int32_t shares;          // of a line
  int32_t ctas;            // of the attention
  int32_t window, sinks;
  int32_t* row_starts;
  int32_t* kv_lens;
  int32_t* tables;
  int32_t* positions;
  int64_t* slots;
  PlanReq* reqs;
  AttnTile* tiles;
  int32_t max_tiles;
  CtaWork* work;           // [shares]
  int32_t* arrived;        // [ctas][kArriveWords] pieces of cut pairs that are done, all zero between calls
  int32_t* ticket;         // CTAs of the plan that are done, zero between calls
  int32_t kind;            // AttnKind
  StepHead* head;
};

struct WriteArgs {
  uint8_t* dst[2];         // the layer's K and V sub-page arrays
  const uint8_t* src[2];
  int64_t row_stride[2], head_stride[2];
  int32_t src_type[2];
  int32_t vec[2];          // 16-byte loads allowed
  const int64_t* slots;
  const StepHead* head;
  int32_t num_tokens, H, D, dtype;
  int64_t num_slots;       // hbm_pages * T
  long long* ctl;
};

struct AttnArgs {
  const uint8_t* kv[2];    // the layer's K and V sub-page arrays
  int64_t P;
  uint32_t hbm_pages;
  int32_t T, H, D, G;
  int32_t t_shift;         // log2(T), -1 where T is no power of two
  int32_t maxB;
  const int32_t* tables;
  const int32_t* positions;
  const AttnTile* tiles;
  const CtaWork* work;
  StepHead* head;
  int32_t* arrived;
  const uint8_t* q;
  uint8_t* out;
  float* lse;
  int64_t q_row, q_head, o_row, o_head;   // strides in elements
  int32_t q_vec, o_vec;    // 16-byte accesses allowed (o_vec 2: of 32 bytes, D a multiple of 16)
  int32_t num_tokens;
  int32_t window, sinks;
  int32_t tile_rows;       // rows of a partial result's slot
  int32_t dp;              // columns of a partial result
  float scale;             // scale * log2(e)
  float* part_o;           // [2 * ctas][tile_rows][dp] sums, and
  float2* part_ml;         // [2 * ctas][tile_rows] their maximum (in log2) and weight
  long long* ctl;
  long long wait_ns;       // of each wait on a copy or a product
  int32_t hold;            // LV_HOLD_NONE but in a self-test
};

constexpr long long kAttnWaitNs = 1000000000ll;   // one second a wait

// Words of AttnArgs.arrived a CTA, in sets of kArriveSet (a warp's rows each, where warps count for
// themselves).  The pieces of a cut pair, or their groups, are counted at the CTA of its first piece,
// in set 0; the pieces of a group at the CTA of the group's first piece, in set 1 for a pair's first
// group and in set 2 for another (which may begin with the pair's last piece, in a CTA where the
// next pair begins too).
constexpr int kArriveSet = 8, kArriveWords = 3 * kArriveSet;

// CTA c's slot for a piece of a (tile, head) pair that it holds only part of: a piece
// that does not start the pair is the first that the CTA does, one that starts it the last.
__host__ __device__ inline int64_t part_slot(int64_t cta, bool starts) { return 2 * cta + (starts ? 1 : 0); }

enum AttnKind : int { ATTN_ROWS = 0, ATTN_TC = 1 };

constexpr int kPlanOneLaunch = 256;      // requests up to which a plan is one launch
cudaError_t launch_plan(const PlanArgs& a, cudaStream_t s);
cudaError_t launch_kv_write(const WriteArgs& a, cudaStream_t s, int num_sms);
cudaError_t configure_attend();
cudaError_t configure_attend_tc();
// keys of a unit, and CTAs that an SM holds, of the rows kernel
constexpr int kRowsUnitShift = 4, kRowsUnit = 1 << kRowsUnitShift, kRowsRows = 16;
int attend_rows_ctas(int dp);
cudaError_t launch_attend_rows(const AttnArgs& a, const CUtensorMap* k, const CUtensorMap* v, bool bf16,
                               int ctas, cudaStream_t s);      // maps: boxes of 64 columns and a unit's keys, or null
constexpr int kTcUnitShift = 7, kTcUnit = 1 << kTcUnitShift, kTcRows = 256;
// places ahead of a pair's units: what a pair costs besides its units, in units (8 prompts of 4096: 722 us
// with 2, 794 with 1, 739 with 4; 20 single tokens over 2000 to 4000 keys: 31.2 with 16, 33.8 with 8, 30 to
// 31.2 with 32, which longer contexts did not gain from)
constexpr int kRowsLead = 16, kTcLead = 2;
// packed rows of a tile: two halves of whole tokens
inline int tc_tile_rows(int G) { return G > 128 ? kTcRows : 2 * (128 / G * G); }
struct TcMaps {
  const CUtensorMap* k;    // the layer's, in boxes of 64 columns and box_rows keys
  const CUtensorMap* v;
  const CUtensorMap* q;    // boxes of 64 columns, G heads and 128 / G rows; null: plain loads
  int box_rows;
};
cudaError_t launch_attend_tc(const AttnArgs& a, const TcMaps& m, bool bf16, int ctas, cudaStream_t s);

// A launch that may be scheduled while the previous kernel on `s` still runs; the kernel waits
// (pdl_wait) before it reads anything that kernel may have written.
template <typename... KArgs, typename... Args>
cudaError_t launch_dependent(void (*kernel)(KArgs...), dim3 grid, unsigned block, size_t smem, cudaStream_t s,
                             Args&&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
}

#ifdef __CUDACC__
// A warp that runs alone pays some 110 cycles for a taken branch: what is rare is laid out of line.
#define LV_RARE(x) __builtin_expect(!!(x), 0)
#define LV_MOSTLY(x) __builtin_expect(!!(x), 1)
__device__ __forceinline__ void report(long long* ctl, int code, long long detail) {
  if (atomicCAS(reinterpret_cast<unsigned long long*>(&ctl[C_ERR]), 0ull, (unsigned long long)code) == 0ull)
    ctl[C_ERR_DETAIL] = detail;
}
// The sum before, and what this warp wrote visible with it.
__device__ __forceinline__ int add_release(int32_t* p, int v) {
  int was;
  asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], %2;" : "=r"(was) : "l"(p), "r"(v) : "memory");
  return was;
}
// True where the step on the device is one that an attention over num_tokens rows may work on.
__device__ __forceinline__ bool step_fits(const StepHead& head, int kind, int num_tokens) {
  return head.kind == kind && head.num_tokens <= num_tokens;
}
// Arrivals that a barrier of kind `what` waits for: one more than come, in every second CTA, where a
// self-test holds them.
__device__ __forceinline__ uint32_t arrivals_of(const AttnArgs& a, int what) {
  return a.hold == what ? 1u + (blockIdx.x & 1u) : 1u;
}
// A wait ran out: later calls on the step are refused until it is planned again.
__device__ __forceinline__ void give_up(const AttnArgs& a) {
  report(a.ctl, LV_ERR_TIMEOUT, blockIdx.x);
  a.head->kind = -1;
}
__device__ __forceinline__ void dep_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void dep_trigger() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
template <typename T>
__device__ __forceinline__ T load_words(const T* p) {
  union {
    int4 w[sizeof(T) / 16];
    T t;
  } x;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(T) / 16); ++i) x.w[i] = reinterpret_cast<const int4*>(p)[i];
  return x.t;
}
// Places of a pair's stretch.
__device__ __forceinline__ int stretch_of(int units, int lead, int share) {
  return lead < 0 ? (units + share - 1) / share * share : units + lead;
}
// Units [u0, u1) of a pair that places [o0, o1) of its stretch hold.
__device__ __forceinline__ int2 units_of(int o0, int o1, int units, int lead) {
  const int ahead = max(lead, 0);
  return make_int2(max(o0 - ahead, 0), min(o1 - ahead, units));
}
// The pieces of a pair (head: its head's number in the line): shares first .. first + count - 1.
struct Pieces {
  int64_t first;
  int count;
};
__device__ __forceinline__ Pieces pieces_of(const AttnTile& t, int head, int lead, int share) {
  const int64_t start = t.before + (int64_t)head * stretch_of(t.units, lead, share) + max(lead, 0);
  const int64_t first = start / share;
  return {first, (int)((start + t.units - 1) / share - first) + 1};
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Two floats rounded to 16 bits, the first in the low half.
template <bool kBf16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  uint32_t r;
  if (kBf16)
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// A weight is at most 2^(kLazy + bias) times its row's true one: the running maximum is only
// raised when a row outgrows it by 2^kLazy, so that the sums are seldom rescaled.  In f16 the
// weights are kept near the top of the type's range (2^15 at most): the row's largest is 2^7 at least,
// so that one of 2^-21 of it still has full precision, where 2^-14 would be the end without the bias.
// Weights are rounded to the pool's 16-bit type for the product with V, whose operands the tensor
// cores take in one type: by at most 2^-8 (bf16) or 2^-11 (f16) of each.  Their sum is taken before
// that, and it, the maxima and the products' sums are in 32 bits.
constexpr float kLazy = 8.0f;
template <bool kBf16>
__device__ __forceinline__ constexpr float weight_bias() {
  return kBf16 ? 0.0f : 7.0f;
}
#endif

}  // namespace lv
