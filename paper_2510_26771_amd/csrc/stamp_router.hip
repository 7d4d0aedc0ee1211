// First launch of the layer of experts: the router's product, and what else needs X alone.
//
// The product: 16 experts x 16 tokens of logits = X W^T + bias by a workgroup, from X as it is.
//
// Two logits decide by their order, so their sums are held in more than 32 bits: a block of 32 channels in fp32 (one matrix instruction of bf16
// operands, or eight of fp32 ones, a bf16 operand widened), the blocks in fp64, one rounding at the end.
// 1 token, 64 experts, 2048 channels (with Q8 of X beside it) 4.5 us; 16 tokens, 256 experts, 4096 channels 10.5; 512 tokens, 64 experts, 2048 channels, fp32 9.  Narrower
// tiles on more workgroups: 6, 10 and 11.  Made for few tokens: 8192 tokens, 256 experts, 4096 channels take 306, as each of 16 tiles side by side reads X again.
#include "stamp_fp8.h"

namespace {
using namespace f8;

struct RouterArgs {
  const void* W;
  const float* bias;  // or nullptr
  const void* X;
  int64_t ld_x;
  int32_t tokens, experts, d;
  float* logits;  // [tokens][experts]
};

constexpr int kRouterWaves = 16;

// 8 channels of a row from c on as they are stored, zeros from d on
template <bool BF16>
struct Raw8 {
  u4 w[BF16 ? 1 : 2];
  __device__ __forceinline__ void load(const char* row, int c, int d) {
    if (c + 8 <= d) {
      const u4_any* s = reinterpret_cast<const u4_any*>(row + (int64_t)c * (BF16 ? 2 : 4));
#pragma unroll
      for (int q = 0; q < (BF16 ? 1 : 2); ++q) w[q] = s[q];
      return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (BF16) {
        const uint32_t x = c + j < d ? reinterpret_cast<const uint16_t*>(row)[c + j] : 0u;
        if (j & 1) w[0][j >> 1] |= x << 16;
        else w[0][j >> 1] = x;
      } else {
        w[j >> 2][j & 3] = c + j < d ? reinterpret_cast<const uint32_t*>(row)[c + j] : 0u;
      }
    }
  }
  __device__ __forceinline__ float at(int j) const {
    if constexpr (BF16) return (j & 1) ? bf16_hi(w[0][j >> 1]) : bf16_lo(w[0][j >> 1]);
    else return __uint_as_float(w[j >> 2][j & 3]);
  }
};

// Experts e0 .. e0 + 15, tokens t0 .. t0 + 15.  The 16 waves take blocks of 32 channels in turn and ask for several at once: the time is the loads' way, one or
// two of them.
template <bool XBF16, bool WBF16>
__device__ __forceinline__ void router_tile(const RouterArgs& a, int e0, int t0, double (*red)[256]) {
  constexpr int kAtOnce = XBF16 && WBF16 ? 8 : 4;
  const int t = threadIdx.x, lane = t & 63, f = lane >> 4, i = lane & 15, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const char* const w = static_cast<const char*>(a.W) + (int64_t)min(e0 + i, a.experts - 1) * a.d * (WBF16 ? 2 : 4);
  const char* const x = static_cast<const char*>(a.X) + (int64_t)min(t0 + i, a.tokens - 1) * a.ld_x * (XBF16 ? 2 : 4);
  double sum[4] = {0, 0, 0, 0};
  for (int c0 = wave * 32; c0 < a.d; c0 += kAtOnce * kRouterWaves * 32) {
    Raw8<WBF16> wv[kAtOnce];
    Raw8<XBF16> xv[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int c = c0 + u * kRouterWaves * 32;
      if (c >= a.d) break;
      wv[u].load(w, c + 8 * f, a.d);
      xv[u].load(x, c + 8 * f, a.d);
    }
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      if (c0 + u * kRouterWaves * 32 >= a.d) break;
      f4 p = {0, 0, 0, 0};
      if constexpr (XBF16 && WBF16) {
        p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, wv[u].w[0]), __builtin_bit_cast(b8, xv[u].w[0]), p, 0, 0, 0);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) p = __builtin_amdgcn_mfma_f32_16x16x4f32(wv[u].at(j), xv[u].at(j), p, 0, 0, 0);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) sum[r] += (double)p[r];
    }
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) red[wave][i * 16 + 4 * f + r] = sum[r];  // token i, expert 4 f + r
  __syncthreads();
  if (t < 256) {
    double s = red[0][t];
#pragma unroll
    for (int q = 1; q < kRouterWaves; ++q) s += red[q][t];
    const int e = e0 + (t & 15), tok = t0 + (t >> 4);
    if (e < a.experts && tok < a.tokens) a.logits[(int64_t)tok * a.experts + e] = (float)(a.bias != nullptr ? s + (double)a.bias[e] : s);
  }
}

constexpr int kThreads = kRouterWaves * 64;

// Workgroups 0 .. tiles - 1: 16 experts x 16 tokens of the logits; the others: Q8 of X as in k_f8_quant, 16 channels of a row a thread, 8 lanes a block.
template <bool XBF16, bool WBF16>
__global__ __launch_bounds__(kThreads) void k_router(RouterArgs a, RouterQ8 q, int64_t tiles, int64_t first) {
  __shared__ double red[kRouterWaves][256];
  const int64_t block = first + blockIdx.x;
  const int t = threadIdx.x, across = (a.experts + 15) / 16;
  if (block < tiles) {
    router_tile<XBF16, WBF16>(a, (int)(block % across) * 16, (int)(block / across) * 16, red);
    return;
  }
  if (block == tiles)
    for (int i = t; i < q.zeros; i += kThreads) q.zero[i] = 0;
  if (q.codes == nullptr) return;
  const int Kp = (a.d + 127) / 128 * 128, per = Kp / 16;
  const int64_t u = (block - tiles) * kThreads + t, m = u / per;
  const int c = (int)(u - m * per) * 16;
  if (m >= a.tokens) return;  // whole groups of 8 lanes
  Raw16<XBF16> x;
  x.load(static_cast<const char*>(a.X) + m * a.ld_x * (XBF16 ? 2 : 4), c, a.d);
  float scale, inv;
  scale_of(max8(x.amax()), q.pow2, &scale, &inv);
  const u4 o = x.codes(inv);
  put_codes(q.codes, m * Kp + c, u2{o[0], o[1]}, q.wide);
  put_codes(q.codes, m * Kp + c + 8, u2{o[2], o[3]}, q.wide);
  if ((t & 7) == 0) q.scales[(int64_t)(c >> 7) * q.ld_s + m] = scale;
}
}  // namespace

hipError_t stamp_launch_router(const stamp_router_t& router, const void* X, int x_bf16, int64_t ld_x, int tokens, int experts, int d, const RouterQ8& q,
                               float* logits, hipStream_t st) {
  const bool wb = router.w_dtype == STAMP_BF16;
  auto* const k = x_bf16 ? (wb ? k_router<true, true> : k_router<true, false>) : (wb ? k_router<false, true> : k_router<false, false>);
  const RouterArgs a = {router.W_dev, router.bias_dev_or_null, X, ld_x, tokens, experts, d, logits};
  const int64_t tiles = (int64_t)((experts + 15) / 16) * ((tokens + 15) / 16), units = (int64_t)tokens * ((d + 127) / 128) * 8;
  const int64_t others = q.codes != nullptr ? (units + kThreads - 1) / kThreads : q.zeros > 0;
  return f8_launches(tiles + others, kThreads, [&](int64_t first, uint32_t n) { k<<<n, kThreads, 0, st>>>(a, q, tiles, first); });
}
