// The product of the router: logits [tokens][experts] = X W^T + bias, from X as it is.
//
// Two logits decide by their order, so their sums are held in more than 32 bits: a block of 32 channels in fp32 (eight 16x16x4 matrix instructions; bf16
// operands are widened, which is exact), the blocks in fp64, one rounding at the end.
#include "stamp_fp8.h"

namespace {
using namespace f8;

constexpr int kWaves = 8;

// 8 channels of a row from c on as fp32, zeros from d on
template <bool BF16>
__device__ __forceinline__ void load8(float (&v)[8], const void* row, int c, int d) {
  if (c + 8 <= d) {
    if constexpr (BF16) {
      const u4 w = *reinterpret_cast<const u4_any*>(static_cast<const uint16_t*>(row) + c);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = (j & 1) ? bf16_hi(w[j >> 1]) : bf16_lo(w[j >> 1]);
    } else {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const f4 w = reinterpret_cast<const f4_any*>(static_cast<const float*>(row) + c)[q];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[4 * q + j] = w[j];
      }
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    v[j] = 0.0f;
    if (c + j < d) v[j] = BF16 ? bf16_lo(static_cast<const uint16_t*>(row)[c + j]) : static_cast<const float*>(row)[c + j];
  }
}

// A workgroup has 16 experts and 16 tokens; its waves take blocks of 32 channels in turn.
template <bool XBF16, bool WBF16>
__global__ __launch_bounds__(kWaves * 64) void k_router(const void* W, const float* bias, const void* X, int64_t ld_x, int tokens, int experts, int d,
                                                        float* logits) {
  __shared__ double red[kWaves][256];
  const int t = threadIdx.x, lane = t & 63, f = lane >> 4, i = lane & 15, wave = t >> 6;
  const int e0 = blockIdx.x * 16, t0 = blockIdx.y * 16;
  const char* const w = static_cast<const char*>(W) + (int64_t)min(e0 + i, experts - 1) * d * (WBF16 ? 2 : 4);
  const char* const x = static_cast<const char*>(X) + (int64_t)min(t0 + i, tokens - 1) * ld_x * (XBF16 ? 2 : 4);
  double sum[4] = {0, 0, 0, 0};
  for (int c = wave * 32; c < d; c += kWaves * 32) {
    float wv[8], xv[8];
    load8<WBF16>(wv, w, c + 8 * f, d);
    load8<XBF16>(xv, x, c + 8 * f, d);
    f4 p = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j) p = __builtin_amdgcn_mfma_f32_16x16x4f32(wv[j], xv[j], p, 0, 0, 0);
#pragma unroll
    for (int r = 0; r < 4; ++r) sum[r] += (double)p[r];
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) red[wave][i * 16 + 4 * f + r] = sum[r];  // token i, expert 4 f + r
  __syncthreads();
  if (t < 256) {
    double s = red[0][t];
#pragma unroll
    for (int q = 1; q < kWaves; ++q) s += red[q][t];
    const int e = e0 + (t & 15), tok = t0 + (t >> 4);
    if (e < experts && tok < tokens) logits[(int64_t)tok * experts + e] = (float)(bias != nullptr ? s + (double)bias[e] : s);
  }
}
}  // namespace

hipError_t stamp_launch_router(const stamp_router_t& router, const void* X, int x_bf16, int64_t ld_x, int tokens, int experts, int d, float* logits,
                               hipStream_t st) {
  const bool wb = router.w_dtype == STAMP_BF16;
  auto* const k = x_bf16 ? (wb ? k_router<true, true> : k_router<true, false>) : (wb ? k_router<false, true> : k_router<false, false>);
  // up to 2^22 tokens are 2^18 rows of workgroups: a grid's second axis holds 65535
  for (int t0 = 0; t0 < tokens; t0 += 65535 * 16) {
    const int n = tokens - t0 < 65535 * 16 ? tokens - t0 : 65535 * 16;
    k<<<dim3((experts + 15) / 16, (n + 15) / 16), kWaves * 64, 0, st>>>(router.W_dev, router.bias_dev_or_null,
                                                                        static_cast<const char*>(X) + (int64_t)t0 * ld_x * (x_bf16 ? 2 : 4), ld_x, n, experts, d,
                                                                        logits + (int64_t)t0 * experts);
  }
  return hipGetLastError();
}
