// Barriers, TMA copies and tcgen05 products for the kernels on the fifth-generation tensor cores.
#pragma once

#include "lv_batch.cuh"

namespace lv {

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
// False once the limit has passed, here or in another role (b->bad, volatile): every role then leaves its loop.  (The limit is
// a kernel argument: kept in shared memory beside the barriers, it cost 8 prompts of 4096 742 us for 718.)
template <typename B>
__device__ __forceinline__ bool bar_wait_slow(B* b, uint64_t* bar, uint32_t parity, long long limit) {
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
template <typename B>
__device__ __forceinline__ bool bar_wait1(B* b, uint64_t* bar, uint32_t parity, long long limit) {
  if (LV_MOSTLY(bar_try(bar, parity))) return true;
  return bar_wait_slow(b, bar, parity, limit);
}
// For a whole warp, whose lanes leave it together with one answer (what follows is .aligned).
template <typename B>
__device__ __forceinline__ bool bar_wait(B* b, uint64_t* bar, uint32_t parity, long long limit) {
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

}  // namespace lv
