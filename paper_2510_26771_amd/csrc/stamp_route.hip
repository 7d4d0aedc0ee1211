// The router of the expert layers: top-k experts of every token, their weights, the rows' order by expert; and the weighted sum of the
// experts' rows.
#include "stamp_fp8.h"

namespace {
using namespace f8;

constexpr int kRtWaves = 8;
constexpr int kRtMaxBlocks = 256;

struct RouteArgs {
  stamp_routing_t r;
  const void* logits;
  int64_t ld;
  int32_t bf16, renorm;
  int32_t per_block;   // tokens of a workgroup
  uint16_t* hist;      // [workgroups][experts] rows that a workgroup's tokens give an expert
};

// order of floats as unsigned integers; 0 for what is masked.  -0 counts as 0.
__device__ __forceinline__ uint32_t order_key(float l) {
  if (!(l > -__builtin_inff())) return 0;
  const uint32_t b = __float_as_uint(l + 0.0f);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k); }
// exp(l - top), where both may be +infinity: then they are equal
__device__ __forceinline__ float share(float l, float top) { return l == top ? 1.0f : expf(l - top); }

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  return v;
}

// One wave per token at a time, lane l has experts l + 64 j.  The largest (key, lower index first) is taken k times.
template <int NV>
__device__ void top_tokens(const RouteArgs& a, int tok0, int tok1, int wave, int lane, uint32_t* count) {
  const int E = a.r.experts, K = a.r.top_k;
  for (int t = tok0 + wave; t < tok1; t += kRtWaves) {
    uint32_t key[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int e = lane + 64 * j;
      float l = -__builtin_inff();
      if (e < E)
        l = a.bf16 ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(a.logits)[(int64_t)t * a.ld + e] << 16)
                   : static_cast<const float*>(a.logits)[(int64_t)t * a.ld + e];
      key[j] = order_key(l);
    }
    uint32_t mine = 0;  // lane j: key of the j-th chosen
    int id = -1;
    float top = 0.0f, sum = 0.0f;
    for (int k = 0; k < K; ++k) {
      uint64_t best = 0;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const uint64_t c = (uint64_t)key[j] << 32 | (uint32_t)~(lane + 64 * j);
        best = c > best ? c : best;
      }
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const uint64_t o = __shfl_xor((unsigned long long)best, d);
        best = o > best ? o : best;
      }
      const uint32_t bk = (uint32_t)(best >> 32);
      if (bk == 0) break;
      const int e = (int)~(uint32_t)best;
      if (k == 0) {
        top = key_value(bk);
        if (!a.renorm) {
          float s = 0.0f;
#pragma unroll
          for (int j = 0; j < NV; ++j) s += key[j] != 0 ? share(key_value(key[j]), top) : 0.0f;
          sum = wave_sum(s);
        }
      }
      if (lane == k) mine = bk, id = e;
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (e == lane + 64 * j) key[j] = 0;
    }
    const float sh = id >= 0 ? share(key_value(mine), top) : 0.0f;
    if (a.renorm) sum = wave_sum(sh);
    if (lane < K) {
      a.r.ids_dev[(int64_t)t * K + lane] = id;
      a.r.weights_dev[(int64_t)t * K + lane] = id >= 0 ? sh / sum : 0.0f;
      if (id >= 0) atomicAdd(&count[id], 1u);
    }
  }
}
__device__ __forceinline__ void top_tokens_of(const RouteArgs& a, int tok0, int tok1, int wave, int lane, uint32_t* count) {
  const int E = a.r.experts;
  if (E <= 64) top_tokens<1>(a, tok0, tok1, wave, lane, count);
  else if (E <= 128) top_tokens<2>(a, tok0, tok1, wave, lane, count);
  else if (E <= 256) top_tokens<4>(a, tok0, tok1, wave, lane, count);
  else if (E <= 512) top_tokens<8>(a, tok0, tok1, wave, lane, count);
  else top_tokens<16>(a, tok0, tok1, wave, lane, count);
}

// Order of the workgroup's slots by expert: every wave has a run of them.  cnt [waves][E].
__device__ void place_rows(const RouteArgs& a, int tok0, int tok1, int wave, int lane, uint32_t (*cnt)[kF8MaxExperts], const uint32_t* base) {
  const int E = a.r.experts, K = a.r.top_k, t = threadIdx.x;
  const int64_t s0 = (int64_t)tok0 * K;
  const int n = (tok1 - tok0) * K;
  const int run = ((n + kRtWaves - 1) / kRtWaves + 63) / 64 * 64;
  for (int i = t; i < kRtWaves * kF8MaxExperts; i += kRtWaves * 64) (&cnt[0][0])[i] = 0;
  __syncthreads();
  const int r0 = min(wave * run, n), r1 = min(r0 + run, n);
  for (int i = r0 + lane; i < r1; i += 64) {
    const int e = a.r.ids_dev[s0 + i];
    if (e >= 0) atomicAdd(&cnt[wave][e], 1u);
  }
  __syncthreads();
  for (int e = t; e < E; e += kRtWaves * 64) {
    uint32_t b = base[e];
    for (int w = 0; w < kRtWaves; ++w) {
      const uint32_t c = cnt[w][e];
      cnt[w][e] = b;
      b += c;
    }
  }
  __syncthreads();
  const int bits = 32 - __builtin_clz((unsigned)E);
  for (int i0 = r0; i0 < r1; i0 += 64) {
    const int i = i0 + lane;
    const int e = i < r1 ? a.r.ids_dev[s0 + i] : -1;
    uint64_t same = ~0ull;
    for (int b = 0; b <= bits; ++b) {  // one bit more: -1 has none in common with the others
      const bool on = (e >> b) & 1;
      const uint64_t m = __ballot(on);
      same &= on ? m : ~m;
    }
    int row = -1;
    volatile uint32_t* c = cnt[wave];
    if (e >= 0) row = (int)(c[e] + __popcll(same & ((1ull << lane) - 1)));
    __builtin_amdgcn_wave_barrier();
    if (e >= 0 && (same >> lane) == 1) c[e] = (uint32_t)row + 1;  // the last of its expert
    __builtin_amdgcn_wave_barrier();
    if (i < r1) a.r.row_of_slot_dev[s0 + i] = row;
    if (row >= 0) a.r.token_of_row_dev[row] = (int)((s0 + i) / K);
  }
}

// Exclusive sums of total[0 .. E) -> base; returns the whole.  E <= 1024 = 2 * threads.
__device__ uint32_t scan_experts(const uint32_t* total, uint32_t* base, int E, uint32_t* tmp) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const uint32_t x = 2 * t < E ? total[2 * t] : 0, y = 2 * t + 1 < E ? total[2 * t + 1] : 0;
  uint32_t incl = x + y;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_up(incl, d);
    if (lane >= d) incl += o;
  }
  if (lane == 63) tmp[wave] = incl;
  __syncthreads();
  uint32_t before = 0, all = 0;
  for (int w = 0; w < kRtWaves; ++w) {
    before += w < wave ? tmp[w] : 0;
    all += tmp[w];
  }
  const uint32_t b = before + incl - x - y;
  if (2 * t < E) base[2 * t] = b;
  if (2 * t + 1 < E) base[2 * t + 1] = b + x;
  __syncthreads();
  return all;
}

// ONE: a single workgroup does all.
template <bool ONE>
__global__ __launch_bounds__(kRtWaves * 64) void k_route_top(RouteArgs a) {
  __shared__ uint32_t count[kF8MaxExperts];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, E = a.r.experts;
  const int tok0 = min((int)blockIdx.x * a.per_block, a.r.tokens), tok1 = min(tok0 + a.per_block, a.r.tokens);
  for (int e = t; e < E; e += kRtWaves * 64) count[e] = 0;
  __syncthreads();
  top_tokens_of(a, tok0, tok1, wave, lane, count);
  __threadfence_block();
  __syncthreads();
  if constexpr (!ONE) {
    for (int e = t; e < E; e += kRtWaves * 64) a.hist[(size_t)blockIdx.x * E + e] = (uint16_t)count[e];
  } else {
    __shared__ uint32_t cnt[kRtWaves][kF8MaxExperts];
    __shared__ uint32_t base[kF8MaxExperts];
    __shared__ uint32_t tmp[kRtWaves];
    const uint32_t all = scan_experts(count, base, E, tmp);
    for (int e = t; e <= E; e += kRtWaves * 64) a.r.offsets_dev[e] = (int)(e < E ? base[e] : all);
    place_rows(a, tok0, tok1, wave, lane, cnt, base);
    for (int i = (int)all + t; i < a.r.tokens * a.r.top_k; i += kRtWaves * 64) a.r.token_of_row_dev[i] = -1;
  }
}

__global__ __launch_bounds__(kRtWaves * 64) void k_route_place(RouteArgs a) {
  __shared__ uint32_t cnt[kRtWaves][kF8MaxExperts];
  __shared__ uint32_t total[kF8MaxExperts], base[kF8MaxExperts], mine[kF8MaxExperts];
  __shared__ uint32_t tmp[kRtWaves];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, E = a.r.experts, nb = gridDim.x;
  const int tok0 = min((int)blockIdx.x * a.per_block, a.r.tokens), tok1 = min(tok0 + a.per_block, a.r.tokens);
  for (int e = t; e < E; e += kRtWaves * 64) {
    uint32_t all = 0, before = 0;
    for (int b = 0; b < nb; ++b) {
      const uint32_t h = a.hist[(size_t)b * E + e];
      all += h;
      before += b < (int)blockIdx.x ? h : 0;
    }
    total[e] = all;
    mine[e] = before;
  }
  __syncthreads();
  const uint32_t all = scan_experts(total, base, E, tmp);
  if (blockIdx.x == 0)
    for (int e = t; e <= E; e += kRtWaves * 64) a.r.offsets_dev[e] = (int)(e < E ? base[e] : all);
  __syncthreads();
  for (int e = t; e < E; e += kRtWaves * 64) base[e] += mine[e];
  __syncthreads();
  place_rows(a, tok0, tok1, wave, lane, cnt, base);
  const int64_t slots = (int64_t)a.r.tokens * a.r.top_k;
  for (int64_t i = (int64_t)all + (int64_t)blockIdx.x * (kRtWaves * 64) + t; i < slots; i += (int64_t)nb * (kRtWaves * 64)) a.r.token_of_row_dev[i] = -1;
}

int tokens_per_block(int tokens) {
  const int per = (tokens + kRtMaxBlocks - 1) / kRtMaxBlocks;
  return per < 128 ? 128 : per;
}

// Y[t] = sum of a token's rows times their weights, slots in order.  A thread has 8 columns.
template <bool BF16>
__global__ __launch_bounds__(256) void k_combine(stamp_routing_t r, const void* rows, int64_t ld_rows, int nrows, void* Y, int64_t ld_y, int d, int wide) {
  const int per = (d + 7) / 8;
  const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t t = u / per;
  const int c = (int)(u - t * per) * 8;
  if (t >= r.tokens) return;
  float y[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int j = 0; j < r.top_k; ++j) {
    const int row = r.row_of_slot_dev[t * r.top_k + j];
    if ((uint32_t)row >= (uint32_t)nrows) continue;
    const float w = r.weights_dev[t * r.top_k + j];
    if constexpr (BF16) {
      const u4 v = *reinterpret_cast<const u4*>(static_cast<const uint16_t*>(rows) + row * ld_rows + c);
#pragma unroll
      for (int i = 0; i < 4; ++i) y[2 * i] = __builtin_fmaf(w, bf16_lo(v[i]), y[2 * i]), y[2 * i + 1] = __builtin_fmaf(w, bf16_hi(v[i]), y[2 * i + 1]);
    } else {
      const f4* s = reinterpret_cast<const f4*>(static_cast<const float*>(rows) + row * ld_rows + c);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = __builtin_fmaf(w, s[i >> 2][i & 3], y[i]);
    }
  }
  const int64_t o = t * ld_y + c;
  if constexpr (BF16) {
    uint16_t* p = static_cast<uint16_t*>(Y) + o;
    if (wide && c + 8 <= d) {
      *reinterpret_cast<u4*>(p) = u4{to_bf16x2(y[0], y[1]), to_bf16x2(y[2], y[3]), to_bf16x2(y[4], y[5]), to_bf16x2(y[6], y[7])};
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < d) p[i] = to_bf16(y[i]);
    }
  } else {
    float* p = static_cast<float*>(Y) + o;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < d) p[i] = y[i];
  }
}
}  // namespace

size_t stamp_route_ws(int tokens, int experts, int) {
  const int per = tokens_per_block(tokens);
  const size_t nb = ((size_t)tokens + per - 1) / per;
  return (nb * experts * sizeof(uint16_t) + 255) / 256 * 256 + 256;
}

hipError_t stamp_launch_route(const stamp_routing_t& r, const void* logits, int bf16, int64_t ld, int renorm, void* ws, hipStream_t st) {
  RouteArgs a;
  a.r = r;
  a.logits = logits;
  a.ld = ld;
  a.bf16 = bf16;
  a.renorm = renorm;
  a.per_block = tokens_per_block(r.tokens);
  a.hist = static_cast<uint16_t*>(ws);
  const int nb = (r.tokens + a.per_block - 1) / a.per_block;
  if (nb <= 1) {
    k_route_top<true><<<1, kRtWaves * 64, 0, st>>>(a);
  } else {
    k_route_top<false><<<nb, kRtWaves * 64, 0, st>>>(a);
    k_route_place<<<nb, kRtWaves * 64, 0, st>>>(a);
  }
  return hipGetLastError();
}

hipError_t stamp_launch_combine(const stamp_routing_t& r, const void* rows, int y_bf16, int64_t ld_rows, int nrows, void* Y, int64_t ld_y, int d,
                                hipStream_t st) {
  const int64_t blocks = ((int64_t)r.tokens * ((d + 7) / 8) + 255) / 256;
  const int wide = (reinterpret_cast<uintptr_t>(Y) | (uintptr_t)(ld_y * (y_bf16 ? 2 : 4))) % 16 == 0;
  if (y_bf16) k_combine<true><<<(uint32_t)blocks, 256, 0, st>>>(r, rows, ld_rows, nrows, Y, ld_y, d, wide);
  else k_combine<false><<<(uint32_t)blocks, 256, 0, st>>>(r, rows, ld_rows, nrows, Y, ld_y, d, wide);
  return hipGetLastError();
}
