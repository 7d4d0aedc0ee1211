// The router's product for any number of tokens.
#include "stamp_router.h"

namespace {
using namespace f8;

template <bool XBF16, bool WBF16>
__global__ __launch_bounds__(kRouterWaves * 64) void k_router(RouterArgs a) {
  __shared__ double red[kRouterWaves][256];
  router_tile<XBF16, WBF16>(a, blockIdx.x * 16, blockIdx.y * 16, red);
}
}  // namespace

hipError_t stamp_launch_router(const stamp_router_t& router, const void* X, int x_bf16, int64_t ld_x, int tokens, int experts, int d, float* logits,
                               hipStream_t st) {
  const bool wb = router.w_dtype == STAMP_BF16;
  auto* const k = x_bf16 ? (wb ? k_router<true, true> : k_router<true, false>) : (wb ? k_router<false, true> : k_router<false, false>);
  // up to 2^22 tokens are 2^18 rows of workgroups: a grid's second axis holds 65535
  for (int t0 = 0; t0 < tokens; t0 += 65535 * 16) {
    const int n = tokens - t0 < 65535 * 16 ? tokens - t0 : 65535 * 16;
    const RouterArgs a = {router.W_dev, router.bias_dev_or_null, static_cast<const char*>(X) + (int64_t)t0 * ld_x * (x_bf16 ? 2 : 4), ld_x, n, experts, d,
                          logits + (int64_t)t0 * experts};
    k<<<dim3((experts + 15) / 16, (n + 15) / 16), kRouterWaves * 64, 0, st>>>(a);
  }
  return hipGetLastError();
}
