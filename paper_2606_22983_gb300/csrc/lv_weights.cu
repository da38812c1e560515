// Attention weights of a step's rows, added up for the cached tokens (include/lv.h, lv_attention_weights):
//   w[s][h][j] += sum over rows r and heads g of 2^(c q_rg.k_j - lse_rg log2(e)), c = scale log2(e),
// over the rows that see key j.  The attention has left the rows' normalisers, so no maximum and no
// rescaling is needed, and no V is read.
#include "lv_weights.cuh"

namespace lv {

namespace {

constexpr float kLog2e = 1.44269504088896341f;

// ---------------------------------------------------------------- any shape
constexpr int kPlainThreads = 128, kPlainKeys = 64, kPlainRows = 16;

// For shapes that the tensor-core kernel does not take (heads of over 128, pages of no whole 8 tokens): a unit
// of 64 keys in shared memory, 16 of them a warp, held in registers as the left operand of mma.sync; the rows 16
// at a time beside them.  DP: head_dim rounded up to 64, 128 or 256, with zeros.  Rows of shared memory are 16
// bytes longer than that, so that the eight rows of an ldmatrix lie in different banks.
// 16 single tokens over 4 to 16 k keys, 4 KV heads of 256: 208 us (32-bit products in their place 2890); 500 tokens at
// 16 000 keys 1590, as each 16 rows are read from L2 again for every 64 keys.
template <int DP, bool kBf16>
__global__ void __launch_bounds__(kPlainThreads) k_weights_plain(const __grid_constant__ WeightArgs a) {
  extern __shared__ __align__(16) unsigned char dyn[];
  __shared__ SegmentIndex<kPlainThreads> x;
  __shared__ float s_b[kPlainRows];
  __shared__ int s_token[kPlainRows];
  constexpr int kLd = DP + 8, kChunks = DP / 8;           // elements and 16-byte pieces of a row
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  uint4* const ks = reinterpret_cast<uint4*>(dyn);                                  // [kPlainKeys][kLd]
  uint4* const qs = ks + kPlainKeys * kLd / 8;                                      // [kPlainRows][kLd]
  const uint32_t k_s = (uint32_t)__cvta_generic_to_shared(ks), q_s = (uint32_t)__cvta_generic_to_shared(qs);
  dep_wait();
  dep_trigger();
  const StepHead step = load_words(a.head);
  if (!weights_fit(a, step)) {
    if (blockIdx.x == 0 && tid == 0) report(a.ctl, LV_ERR_STATE, -1);
    return;
  }
  const int n = step.requests & (kSharedStep - 1);
  const int units = index_segments<kPlainThreads, kPlainKeys, false>(a, step, x, reinterpret_cast<int*>(dyn), 0);
  const uint4 zero = make_uint4(0, 0, 0, 0);
  for (int i = blockIdx.x; i < units; i += gridDim.x) {
    int piece;
    const Unit u = find_unit<kPlainThreads, kPlainKeys, false>(a, step, x, i, 0, piece);
    if (u.t0 >= u.t1) continue;
    __syncthreads();
#pragma unroll 4
    for (int e = tid; e < kPlainKeys * kChunks; e += kPlainThreads) {
      const int r = e / kChunks, c = e % kChunks, j = u.key0 + r;
      uint4 v = zero;
      if (j < u.g.keys && c * 8 < a.D) {
        const uint32_t b = (uint32_t)j / (uint32_t)a.T;
        const int page = u.g.req < 0 ? a.pool_table[(size_t)u.g.sid * a.maxB + b] : a.tables[(size_t)u.g.req * a.maxB + b];
        if ((uint32_t)page < a.hbm_pages)
          v = *reinterpret_cast<const uint4*>(a.k + (size_t)page * a.P + (((size_t)(j - b * a.T) * a.H + u.head) * a.D + c * 8) * 2);
      }
      ks[r * (kLd / 8) + c] = v;
    }
    __syncthreads();
    uint32_t k_of[DP / 16][4];
    {
      const uint32_t at = k_s + ((16 * wid + (lane & 15)) * kLd + (lane >> 4) * 8) * 2;
#pragma unroll
      for (int d = 0; d < DP / 16; ++d) ldsm4(k_of[d], at + 32 * d);
    }
    // this lane's keys: lane / 4 of the warp's 16 and 8 on, summed over its columns of the rows
    const int key = u.key0 + 16 * wid + lane / 4;
    LongSum all[2];
    for (int R0 = u.t0 * a.G; R0 < u.t1 * a.G; R0 += kPlainRows) {
      __syncthreads();
      for (int e = tid; e < kPlainRows * kChunks; e += kPlainThreads) {
        const int r = e / kChunks, c = e % kChunks, R = R0 + r, token = R / a.G;
        uint32_t w[4] = {0, 0, 0, 0};
        if (R < u.t1 * a.G && c * 8 < a.D) {
          const uint16_t* q = reinterpret_cast<const uint16_t*>(a.q) + (u.g.qrow + token) * a.q_row +
                              (int64_t)(u.head * a.G + R - token * a.G) * a.q_head + c * 8;
#pragma unroll
          for (int k = 0; k < 4; ++k) w[k] = (uint32_t)q[2 * k] | (uint32_t)q[2 * k + 1] << 16;
        }
        qs[r * (kLd / 8) + c] = make_uint4(w[0], w[1], w[2], w[3]);
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
      float c[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
      const uint32_t at = q_s + (((lane & 7) + (lane >> 4) * 8) * kLd + (lane >> 3 & 1) * 8) * 2;
#pragma unroll
      for (int d = 0; d < DP / 16; ++d) {
        uint32_t b[4];
        ldsm4(b, at + 32 * d);
        mma<kBf16>(c[0], k_of[d], b[0], b[1]);
        mma<kBf16>(c[1], k_of[d], b[2], b[3]);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 8 * (e >> 1) + 2 * (lane & 3) + (e & 1), token = s_token[r];
          if (token >= 0 && sees(a, u.g, token, key + 8 * h)) sum += exp2_fast(c[e >> 1][2 * h + (e & 1)] * a.scale + s_b[r]);
        }
        all[h].add(sum);
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float sum = all[h].sum;
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      const int j = key + 8 * h;
      if ((lane & 3) == 0 && j < u.g.keys && sum != 0.f) a.w[u.g.sid * a.w_session + u.head * a.w_head + j] += sum;
    }
  }
}

template <int DP>
constexpr int plain_smem() {
  constexpr int tile = (kPlainKeys + kPlainRows) * (DP + 8) * 2;
  return tile > 4096 * 4 ? tile : 4096 * 4;      // (sessions' words before the first tile)
}

template <int DP>
cudaError_t set_plain() {
  for (auto k : {k_weights_plain<DP, true>, k_weights_plain<DP, false>}) {
    const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, plain_smem<DP>());
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

template <int DP>
cudaError_t run_plain(const WeightArgs& a, bool bf16, int num_sms, cudaStream_t s) {
  return launch_dependent(bf16 ? k_weights_plain<DP, true> : k_weights_plain<DP, false>, dim3(4 * num_sms), kPlainThreads,
                          plain_smem<DP>(), s, a);
}

}  // namespace

cudaError_t configure_weights() {
  for (cudaError_t e : {set_plain<64>(), set_plain<128>(), set_plain<256>()})
    if (e != cudaSuccess) return e;
  return cudaSuccess;
}

cudaError_t launch_weights_plain(const WeightArgs& a, bool bf16, int dp, int num_sms, cudaStream_t s) {
  if (dp == 64) return run_plain<64>(a, bf16, num_sms, s);
  return dp == 128 ? run_plain<128>(a, bf16, num_sms, s) : run_plain<256>(a, bf16, num_sms, s);
}

}  // namespace lv
