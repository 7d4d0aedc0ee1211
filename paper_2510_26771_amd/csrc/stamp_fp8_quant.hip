// Quantizers of the 8-bit floating point layers: activations by row and block of 128 channels, weights by block of 128 x 128.
#include "stamp_fp8.h"

namespace {
using namespace f8;

// A thread has 16 channels, 8 lanes a block: the largest magnitude takes three steps over lanes, and loads and stores are 16 bytes.  Bound by memory:
// 2 (4) bytes read, 1.03 written per element (2.03 as bf16).  32768 x 4096 from bf16 66 us, 6.1 TB/s; 1 to 100 rows 3 to 5 us, the launch.
template <bool BF16, bool WIDE>
__global__ __launch_bounds__(256) void k_f8_quant(const void* X, int64_t ld_x, int rows, int d, int Kp, int pow2, uint8_t* codes, float* scales,
                                                  int64_t ld_s, int64_t first) {
  const int per = Kp >> 4;
  const int64_t u = (first + blockIdx.x) * 256 + threadIdx.x;
  const int64_t m = u / per;
  const int c = (int)(u - m * per) * 16;
  if (m >= rows) return;  // whole groups of 8 lanes: per is a multiple of 8
  Raw16<BF16> x;
  x.load(static_cast<const char*>(X) + m * ld_x * (BF16 ? 2 : 4), c, d);
  float scale, inv;
  scale_of(max8(x.amax()), pow2, &scale, &inv);
  const u4 o = x.codes(inv);
  if constexpr (WIDE) {
    b8* p = reinterpret_cast<b8*>(codes + (m * Kp + c) * 2);
    p[0] = widen8((int)o[0], (int)o[1]);
    p[1] = widen8((int)o[2], (int)o[3]);
  } else {
    *reinterpret_cast<u4*>(codes + m * Kp + c) = o;
  }
  if ((threadIdx.x & 7) == 0) scales[(int64_t)(c >> 7) * ld_s + m] = scale;
}

// ---- weights, once per plan ----
__device__ __forceinline__ float w_value(const void* W, int dtype, int out_by_in, int64_t mat, int n, int c, int N, int d) {
  const int64_t o = mat * N * d + (out_by_in ? (int64_t)n * d + c : (int64_t)c * N + n);
  return dtype == STAMP_BF16 ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(W)[o] << 16) : static_cast<const float*>(W)[o];
}

// one workgroup per block of 128 x 128: the bits of its largest magnitude
__global__ __launch_bounds__(256) void k_f8_w_amax(const void* W, int dtype, int out_by_in, int N, int d, int nblk, int Kb, uint32_t* SW) {
  const int kb = blockIdx.x % Kb, nb = blockIdx.x / Kb;
  const int64_t mat = blockIdx.y;
  uint32_t a = 0;
  for (int i = threadIdx.x; i < 128 * 128; i += 256) {
    const int n = nb * 128 + (out_by_in ? i >> 7 : i & 127), c = kb * 128 + (out_by_in ? i & 127 : i >> 7);
    if (n < N && c < d) a = max(a, abs_bits(w_value(W, dtype, out_by_in, mat, n, c, N, d)));
  }
  __shared__ uint32_t red[256];
  red[threadIdx.x] = a;
  __syncthreads();
  for (int s = 128; s > 0; s >>= 1) {
    if ((int)threadIdx.x < s) red[threadIdx.x] = max(red[threadIdx.x], red[threadIdx.x + s]);
    __syncthreads();
  }
  if (threadIdx.x == 0) SW[(mat * nblk + nb) * Kb + kb] = red[0];
}

__global__ __launch_bounds__(256) void k_f8_w_scale(float* SW, int64_t n, int pow2) {
  const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (u >= n) return;
  float scale, inv;
  scale_of(__float_as_uint(SW[u]), pow2, &scale, &inv);
  SW[u] = scale;
}

// one thread per 16 bytes of the operand image; SW: the blocks' largest magnitudes, unless W holds codes
__global__ __launch_bounds__(256) void k_f8_w_image(const void* W, int dtype, int out_by_in, int N, int d, int nblk, int Kb, int groups, int gated, int pow2,
                                                    const float* SW, uint8_t* image, int64_t total, int64_t first) {
  const int64_t u = (first + blockIdx.x) * 256 + threadIdx.x;
  if (u >= total) return;
  const int lane = (int)(u & 63), h = (int)(u >> 6) & 1, b = (int)(u >> 7) & 3;
  const int64_t gk = u >> 9;
  const int kb = (int)(gk % Kb);
  const int64_t sg = gk / Kb;
  const int g = (int)(sg % groups);
  const int64_t set = sg / groups, mat = gated ? 2 * set + (b & 1) : set;
  const int n = f8_column(gated, g, b, lane & 15), c0 = kb * 128 + 64 * h + 16 * (lane >> 4);
  u4 o = {0, 0, 0, 0};
  if (n < N && c0 < d) {
    if (dtype == STAMP_E4M3) {
      const uint8_t* s = static_cast<const uint8_t*>(W) + (mat * N + n) * d + c0;
      for (int j = 0; j < 16 && c0 + j < d; ++j) o[j >> 2] |= (uint32_t)s[j] << 8 * (j & 3);
    } else {
      float scale, inv;
      scale_of(__float_as_uint(SW[(mat * nblk + (n >> 7)) * Kb + kb]), pow2, &scale, &inv);
      float v[16];
      for (int j = 0; j < 16; ++j) v[j] = c0 + j < d ? __fmul_rn(w_value(W, dtype, out_by_in, mat, n, c0 + j, N, d), inv) : 0.0f;
      for (int j = 0; j < 4; ++j) o[j] = pack4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
    }
  }
  *reinterpret_cast<u4*>(image + u * 16) = o;
}

// flag: set where a scale is no normal power of two
__global__ __launch_bounds__(256) void k_f8_check_pow2(const float* s, int64_t n, uint32_t* flag) {
  const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (u >= n) return;
  const uint32_t b = __float_as_uint(s[u]);
  if ((b & 0x807fffffu) != 0 || b == 0 || b == kInfBits) *flag = 1;
}
}  // namespace

hipError_t stamp_launch_f8_quant(const void* X, int x_bf16, int64_t ld_x, int rows, int d, int pow2, int wide, uint8_t* codes, float* scales, int64_t ld_s,
                                 hipStream_t st) {
  const int Kp = (d + 127) / 128 * 128;
  auto* kernel = x_bf16 ? (wide ? k_f8_quant<true, true> : k_f8_quant<true, false>) : (wide ? k_f8_quant<false, true> : k_f8_quant<false, false>);
  return f8_launches(((int64_t)rows * (Kp / 16) + 255) / 256, 256, [&](int64_t first, uint32_t n) {
    kernel<<<n, 256, 0, st>>>(X, ld_x, rows, d, Kp, pow2, codes, scales, ld_s, first);
  });
}

hipError_t stamp_launch_f8_weights(stamp_fp8_plan* p, const void* W, const float* w_scales, hipStream_t st, uint32_t* flag) {
  const stamp_fp8_desc_t& d = p->desc;
  const int mats = p->sets * (d.gated ? 2 : 1), pow2 = d.scale_format == STAMP_SCALE_POW2;
  const int64_t ns = (int64_t)mats * p->nblk * p->Kb;
  if (d.w_dtype == STAMP_E4M3) {
    hipError_t e = hipMemcpyAsync(p->sw_dev, w_scales, ns * sizeof(float), hipMemcpyDeviceToDevice, st);
    if (e != hipSuccess) return e;
    if (flag != nullptr) k_f8_check_pow2<<<(uint32_t)((ns + 255) / 256), 256, 0, st>>>(p->sw_dev, ns, flag);
  } else {
    k_f8_w_amax<<<dim3(p->nblk * p->Kb, mats), 256, 0, st>>>(W, d.w_dtype, d.w_is_out_by_in, d.d_out, d.d_in, p->nblk, p->Kb,
                                                             reinterpret_cast<uint32_t*>(p->sw_dev));
  }
  const int64_t total = (int64_t)p->sets * p->groups * p->Kb * (kF8GroupBytes / 16);
  const hipError_t e = f8_launches((total + 255) / 256, 256, [&](int64_t first, uint32_t n) {
    k_f8_w_image<<<n, 256, 0, st>>>(W, d.w_dtype, d.w_is_out_by_in, d.d_out, d.d_in, p->nblk, p->Kb, p->groups, d.gated, pow2, p->sw_dev, p->w_dev, total, first);
  });
  if (e != hipSuccess) return e;
  if (d.w_dtype != STAMP_E4M3) k_f8_w_scale<<<(uint32_t)((ns + 255) / 256), 256, 0, st>>>(p->sw_dev, ns, pow2);
  return hipGetLastError();
}
