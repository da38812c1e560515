// Attention weights of a step's rows, added up for the cached tokens (include/lv.h, lv_attention_weights):
//   w[s][h][j] += sum over rows r and heads g of 2^(c q_rg.k_j - lse_rg log2(e)), c = scale log2(e),
// over the rows that see key j.  The attention has left the rows' normalisers, so no maximum and no
// rescaling is needed, and no V is read.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "lv_weights.cuh"

namespace lv {

namespace {

constexpr float kLog2e = 1.44269504088896341f;

// ---------------------------------------------------------------- any shape
constexpr int kPlainThreads = 128, kPlainKeys = 64, kPlainRows = 16;

template <bool kBf16>
__device__ __forceinline__ float to_float(uint16_t x) {
  if (kBf16) return __uint_as_float((uint32_t)x << 16);
  return __half2float(__ushort_as_half(x));
}

// For shapes that the tensor-core kernel does not take (heads of over 128, pages of no whole 8 tokens): a unit
// of 64 keys in shared memory in 32 bits, the rows 16 at a time beside them, a thread 8 rows of a key.
template <bool kBf16>
__global__ void __launch_bounds__(kPlainThreads) k_weights_plain(const __grid_constant__ WeightArgs a) {
  extern __shared__ __align__(16) unsigned char dyn[];
  __shared__ SegmentIndex<kPlainThreads> x;
  __shared__ float s_b[kPlainRows], s_sum[kPlainKeys];
  __shared__ int s_token[kPlainRows];
  const int ld = a.D + 1, tid = threadIdx.x;
  float* ks = reinterpret_cast<float*>(dyn);              // [kPlainKeys][D + 1]
  float* qs = ks + kPlainKeys * ld;                       // [kPlainRows][D]
  dep_wait();
  dep_trigger();
  const StepHead step = load_words(a.head);
  if (step.kind < 0 || step.num_tokens > a.num_tokens) {
    if (blockIdx.x == 0 && tid == 0) report(a.ctl, LV_ERR_STATE, -1);
    return;
  }
  const int n = step.requests & (kSharedStep - 1);
  const int units = index_segments<kPlainThreads, kPlainKeys>(a, step, x, reinterpret_cast<int*>(dyn));
  const int key = tid % kPlainKeys, half = tid / kPlainKeys;
  for (int i = blockIdx.x; i < units; i += gridDim.x) {
    const Unit u = find_unit<kPlainThreads, kPlainKeys>(a, step, x, i);
    if (u.t0 >= u.t1) continue;
    __syncthreads();
    for (int e = tid; e < kPlainKeys * a.D; e += kPlainThreads) {
      const int r = e / a.D, d = e - r * a.D, j = u.key0 + r;
      float v = 0.f;
      if (j < u.g.keys) {
        const uint32_t b = (uint32_t)j / (uint32_t)a.T;
        const int page = u.g.req < 0 ? a.pool_table[(size_t)u.g.sid * a.maxB + b] : a.tables[(size_t)u.g.req * a.maxB + b];
        if ((uint32_t)page < a.hbm_pages)
          v = to_float<kBf16>(reinterpret_cast<const uint16_t*>(a.k + (size_t)page * a.P)[((size_t)(j - b * a.T) * a.H + u.head) * a.D + d]);
      }
      ks[r * ld + d] = v;
    }
    LongSum all;
    for (int R0 = u.t0 * a.G; R0 < u.t1 * a.G; R0 += kPlainRows) {
      __syncthreads();
      for (int e = tid; e < kPlainRows * a.D; e += kPlainThreads) {
        const int r = e / a.D, d = e - r * a.D, R = R0 + r;
        if (R >= u.t1 * a.G) break;
        const int token = R / a.G;
        qs[r * a.D + d] = to_float<kBf16>(reinterpret_cast<const uint16_t*>(a.q)[(u.g.qrow + token) * a.q_row +
                                                                                 (int64_t)(u.head * a.G + R - token * a.G) * a.q_head + d]);
      }
      if (tid < kPlainRows) {
        const int R = R0 + tid, token = R / a.G;
        float z = -INFINITY;
        if (R < u.t1 * a.G && counts(a, u.g, n, token))
          z = a.lse[(int64_t)(u.g.qrow + token) * (a.H * a.G) + u.head * a.G + R - token * a.G];
        s_b[tid] = -z * kLog2e;
        s_token[tid] = z == -INFINITY ? -1 : token;
      }
      __syncthreads();
      float s[kPlainRows / 2];
#pragma unroll
      for (int r = 0; r < kPlainRows / 2; ++r) s[r] = 0.f;
      const float *kk = ks + key * ld, *qq = qs + half * (kPlainRows / 2) * a.D;
      for (int d = 0; d < a.D; ++d) {
        const float v = kk[d];
#pragma unroll
        for (int r = 0; r < kPlainRows / 2; ++r) s[r] += v * qq[r * a.D + d];
      }
      float sum = 0.f;
#pragma unroll
      for (int r = 0; r < kPlainRows / 2; ++r) {
        const int at = half * (kPlainRows / 2) + r, token = s_token[at];
        if (token >= 0 && sees(a, u.g, token, u.key0 + key)) sum += exp2_fast(s[r] * a.scale + s_b[at]);
      }
      all.add(sum);
    }
    float sum = all.sum;
    if (half == 1) s_sum[key] = sum;
    __syncthreads();
    if (half == 0 && u.key0 + key < u.g.keys) {
      sum += s_sum[key];
      float* to = a.w + u.g.sid * a.w_session + u.head * a.w_head + u.key0 + key;
      if (sum != 0.f) *to += sum;
    }
  }
}

size_t plain_smem(int D) {
  const size_t tile = (size_t)kPlainKeys * (D + 1) * 4 + (size_t)kPlainRows * D * 4;
  return tile > 4096 * 4 ? tile : 4096 * 4;      // (sessions' words before the first tile)
}

}  // namespace

cudaError_t configure_weights() {
  for (auto k : {k_weights_plain<true>, k_weights_plain<false>}) {
    const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)plain_smem(256));
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_weights_plain(const WeightArgs& a, bool bf16, int num_sms, cudaStream_t s) {
  return launch_dependent(bf16 ? k_weights_plain<true> : k_weights_plain<false>, dim3(2 * num_sms), kPlainThreads,
                          plain_smem(a.D), s, a);
}

}  // namespace lv
