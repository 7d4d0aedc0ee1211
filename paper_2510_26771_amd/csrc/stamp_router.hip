// First launch of the layer of experts: the router's product, and what else needs X alone.
#include "stamp_router.h"

namespace {
using namespace f8;

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
