// Keeping a part of sessions' caches: the launches of lv_keep.cu.
#pragma once

#include "lv_internal.cuh"

namespace lv {

constexpr int kMoveThreads = 256;

struct SelectArgs {
  DevPool p;
  lv_weights w;
  const int32_t* sids;
  const int32_t* keeps;
  int32_t H, first, last, most;
  int32_t* kept;           // [n][L][H][most]
};

struct CompactArgs {
  DevPool p;
  lv_weights w;            // data null: none
  const int32_t* sids;
  const int32_t* keeps;
  int32_t H, most, t_shift;
  const int32_t* kept;     // [n][L][H][most]
  int32_t* lens;           // [n]
};

cudaError_t configure_keep();
cudaError_t launch_select_kept(const SelectArgs& a, int n, cudaStream_t s);
cudaError_t launch_compact(const CompactArgs& a, int n, int row_bytes, int num_sms, cudaStream_t s);
cudaError_t launch_truncate(const DevPool& p, const int32_t* sids, const int32_t* lens, int n, cudaStream_t s);

#ifdef __CUDACC__
// The clean host copy of the block at place `at` of the tables is given up, where it has one.
__device__ __forceinline__ void drop_clean(const DevPool& p, size_t at) {
  const int32_t g = p.shadow[at];
  if (g < 0 || g >= p.host_pages) return;
  p.shadow[at] = -1;
  p.own_host[g] = kOwnerNone;
  __threadfence();      // (as soon as the bit is clear an allocation beside this may give the slot an owner)
  atomicAnd(&p.bits_host[g >> 5], ~(1u << (g & 31)));
  atomicAdd(reinterpret_cast<unsigned long long*>(&p.ctl[C_HOST_ALLOC]), (unsigned long long)-1ll);
  atomicAdd(reinterpret_cast<unsigned long long*>(&p.ctl[C_CLEAN]), (unsigned long long)-1ll);
  atomicAdd(reinterpret_cast<unsigned long long*>(&p.ctl[C_CLEAN_DROPPED]), 1ull);
}
#endif

}  // namespace lv
