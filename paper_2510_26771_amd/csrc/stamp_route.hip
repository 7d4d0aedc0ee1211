// The router of the expert layers: top-k experts of every token, their weights, the rows' order by expert; and the weighted sum of the
// experts' rows.
#include "stamp_route.h"

namespace {
using namespace f8;

constexpr int kTopWaves = 16, kPlaceWaves = 8;  // of a workgroup
constexpr int kRtMaxBlocks = 256;

struct RouteArgs {
  stamp_routing_t r;
  const void* logits;
  int64_t ld;
  int32_t renorm;
  int32_t per_block;   // tokens of a workgroup
  uint16_t* hist;      // [workgroups][experts, an even number] rows that a workgroup's tokens give an expert
};

// slot_id: where not nullptr, the ids go there as well.
template <bool BF16>
__device__ __forceinline__ void top_tokens_of(const RouteArgs& a, int tok0, int tok1, int wave, int lane, uint32_t* count, int* slot_id) {
  const TopArgs top = {a.logits, a.ld, a.r.experts, a.r.top_k, a.renorm};
  const int E = a.r.experts, K = a.r.top_k;
  auto put = [&](int t, int k, int id, float weight) __attribute__((always_inline)) {
    a.r.ids_dev[(int64_t)t * K + k] = id;
    a.r.weights_dev[(int64_t)t * K + k] = weight;
    if (slot_id != nullptr) slot_id[(t - tok0) * K + k] = id;
    if (id >= 0) atomicAdd(&count[id], 1u);
  };
  if (E <= 32) top_tokens<kTopWaves, 16, 2, BF16>(top, tok0, tok1, wave, lane, put);
  else if (E <= 64) top_tokens<kTopWaves, 16, 4, BF16>(top, tok0, tok1, wave, lane, put);
  else if (E <= 128) top_tokens<kTopWaves, 16, 8, BF16>(top, tok0, tok1, wave, lane, put);
  else if (E <= 256) top_tokens<kTopWaves, 16, 16, BF16>(top, tok0, tok1, wave, lane, put);
  else if (E <= 512) top_tokens<kTopWaves, 64, 8, BF16>(top, tok0, tok1, wave, lane, put);
  else top_tokens<kTopWaves, 64, 16, BF16>(top, tok0, tok1, wave, lane, put);
}

template <int W>
__device__ void place_rows(const RouteArgs& a, const int* ids, int tok0, int tok1, int wave, int lane, uint32_t (*cnt)[kF8MaxExperts], const uint32_t* base) {
  const int E = a.r.experts, K = a.r.top_k, t = threadIdx.x;
  const int64_t s0 = (int64_t)tok0 * K;
  const int n = (tok1 - tok0) * K;
  const int run = ((n + W - 1) / W + 63) / 64 * 64;
  for (int e = lane; e < E; e += 64) cnt[wave][e] = 0;
  __syncthreads();
  const int r0 = min(wave * run, n), r1 = min(r0 + run, n);
  for (int i = r0 + lane; i < r1; i += 64) {
    const int e = ids[i];
    if (e >= 0) atomicAdd(&cnt[wave][e], 1u);
  }
  __syncthreads();
  for (int e = t; e < E; e += W * 64) {
    uint32_t b = base[e];
    for (int w = 0; w < W; ++w) {
      const uint32_t c = cnt[w][e];
      cnt[w][e] = b;
      b += c;
    }
  }
  __syncthreads();
  const int bits = 32 - __builtin_clz((unsigned)E);
  for (int i0 = r0; i0 < r1; i0 += 64) {
    const int i = i0 + lane;
    const int e = i < r1 ? ids[i] : -1;
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

// Exclusive sums of total[0 .. E) -> base; returns the whole.  E <= 1024, two experts a thread (512 threads or more).
template <int W>
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
  for (int w = 0; w < W; ++w) {
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
template <bool ONE, bool BF16>
__global__ __launch_bounds__(kTopWaves * 64) void k_route_top(RouteArgs a) {
  __shared__ uint32_t count[kF8MaxExperts];
  __shared__ int slot_id[ONE ? kTopWaves * 4 * 32 : 1];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, E = a.r.experts;
  const int tok0 = min((int)blockIdx.x * a.per_block, a.r.tokens), tok1 = min(tok0 + a.per_block, a.r.tokens);
  for (int e = t; e < E; e += kTopWaves * 64) count[e] = 0;
  __syncthreads();
  top_tokens_of<BF16>(a, tok0, tok1, wave, lane, count, ONE ? slot_id : nullptr);
  __syncthreads();
  if constexpr (!ONE) {
    const int stride = (E + 1) & ~1;
    for (int e = t; e < stride; e += kTopWaves * 64) a.hist[(size_t)blockIdx.x * stride + e] = e < E ? (uint16_t)count[e] : (uint16_t)0;
  } else {
    __shared__ uint32_t cnt[kTopWaves][kF8MaxExperts];
    __shared__ uint32_t base[kF8MaxExperts];
    __shared__ uint32_t tmp[kTopWaves];
    const uint32_t all = scan_experts<kTopWaves>(count, base, E, tmp);
    for (int e = t; e <= E; e += kTopWaves * 64) a.r.offsets_dev[e] = (int)(e < E ? base[e] : all);
    place_rows<kTopWaves>(a, slot_id, tok0, tok1, wave, lane, cnt, base);
    for (int i = (int)all + t; i < a.r.tokens * a.r.top_k; i += kTopWaves * 64) a.r.token_of_row_dev[i] = -1;
  }
}

// Rows of several workgroups' tokens: each adds up the counts of all (integers, in any order) and places its own.  32768 tokens, 8 of 256 experts: 9.7 us,
// the counts' two trips through the L2s.
__global__ __launch_bounds__(kPlaceWaves * 64) void k_route_place(RouteArgs a) {
  __shared__ uint32_t cnt[kPlaceWaves][kF8MaxExperts];
  __shared__ uint32_t total[kF8MaxExperts], base[kF8MaxExperts], mine[kF8MaxExperts];
  __shared__ uint32_t tmp[kPlaceWaves];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, E = a.r.experts, nb = gridDim.x;
  const int tok0 = min((int)blockIdx.x * a.per_block, a.r.tokens), tok1 = min(tok0 + a.per_block, a.r.tokens);
  // all workgroups' counts, two experts and a part of the workgroups a thread: `parts` threads side by side have the same experts
  const int pairs = (E + 1) / 2, parts = max(1, kPlaceWaves * 64 / pairs), stride = (E + 1) & ~1;
  for (int e = t; e < E; e += kPlaceWaves * 64) total[e] = mine[e] = 0;
  __syncthreads();
  for (int u = t; u < pairs * parts; u += kPlaceWaves * 64) {
    const int pair = u % pairs, part = u / pairs, b1 = nb * (part + 1) / parts;
    const uint32_t* h = reinterpret_cast<const uint32_t*>(a.hist) + pair;
    uint32_t all0 = 0, all1 = 0, before0 = 0, before1 = 0;
#pragma unroll 16
    for (int b = nb * part / parts; b < b1; ++b) {
      const uint32_t v = h[(size_t)b * (stride / 2)];
      const uint32_t mask = b < (int)blockIdx.x ? 0xffffffffu : 0;
      all0 += v & 0xffff;
      all1 += v >> 16;
      before0 += v & 0xffff & mask;
      before1 += (v & mask) >> 16;
    }
    atomicAdd(&total[2 * pair], all0);
    atomicAdd(&mine[2 * pair], before0);
    if (2 * pair + 1 < E) {
      atomicAdd(&total[2 * pair + 1], all1);
      atomicAdd(&mine[2 * pair + 1], before1);
    }
  }
  __syncthreads();
  const uint32_t all = scan_experts<kPlaceWaves>(total, base, E, tmp);
  if (blockIdx.x == 0)
    for (int e = t; e <= E; e += kPlaceWaves * 64) a.r.offsets_dev[e] = (int)(e < E ? base[e] : all);
  __syncthreads();
  for (int e = t; e < E; e += kPlaceWaves * 64) base[e] += mine[e];
  __syncthreads();
  place_rows<kPlaceWaves>(a, a.r.ids_dev + (int64_t)tok0 * a.r.top_k, tok0, tok1, wave, lane, cnt, base);
  const int64_t slots = (int64_t)a.r.tokens * a.r.top_k;
  for (int64_t i = (int64_t)all + (int64_t)blockIdx.x * (kPlaceWaves * 64) + t; i < slots; i += (int64_t)nb * (kPlaceWaves * 64)) a.r.token_of_row_dev[i] = -1;
}

// Tokens of a workgroup: what its waves take at once, or more where that would be over 256 workgroups (each of which adds up the counts of
// all).  One workgroup does all in one launch.
int tokens_at_once(int experts) { return kTopWaves * (experts <= 256 ? 4 : 1); }
int tokens_per_block(int tokens, int experts) {
  const int once = tokens_at_once(experts), per = (tokens + kRtMaxBlocks - 1) / kRtMaxBlocks;
  return per < once ? once : per;
}

// Y[t] = sum of a token's rows times their weights, slots in order.  A thread has 8 columns and 8 rows in flight.  Bound by memory: 8192 tokens of
// 4096 columns, 8 rows each, bf16: 122 us, 5 TB/s.
// ROWS16, BF16: rows and Y in bf16.
template <bool ROWS16, bool BF16>
__global__ __launch_bounds__(256) void k_combine(stamp_routing_t r, const void* rows, int64_t ld_rows, int nrows, const void* R, int64_t ld_r, void* Y, int64_t ld_y,
                                                 int d) {
  const int per = (d + 7) / 8;
  const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t t = u / per;
  const int c = (int)(u - t * per) * 8;
  if (t >= r.tokens) return;
  float y[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  const int32_t* slot = r.row_of_slot_dev + t * r.top_k;
  const float* weight = r.weights_dev + t * r.top_k;
  for (int j0 = 0; j0 < r.top_k; j0 += 8) {  // 8 rows in flight
    int row[8];
    float w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int jj = min(j0 + j, r.top_k - 1);
      row[j] = slot[jj];
      w[j] = weight[jj];
      if (j0 + j >= r.top_k) row[j] = -1;
    }
    if constexpr (ROWS16) {
      u4 v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        v[j] = (uint32_t)row[j] < (uint32_t)nrows ? *reinterpret_cast<const u4*>(static_cast<const uint16_t*>(rows) + row[j] * ld_rows + c) : u4{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float f = (uint32_t)row[j] < (uint32_t)nrows ? w[j] : 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[2 * i] = __builtin_fmaf(f, bf16_lo(v[j][i]), y[2 * i]), y[2 * i + 1] = __builtin_fmaf(f, bf16_hi(v[j][i]), y[2 * i + 1]);
      }
    } else {
      f4 v[8][2];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const f4* s = reinterpret_cast<const f4*>(static_cast<const float*>(rows) + row[j] * ld_rows + c);
        const bool on = (uint32_t)row[j] < (uint32_t)nrows;
        v[j][0] = on ? s[0] : f4{0, 0, 0, 0};
        v[j][1] = on ? s[1] : f4{0, 0, 0, 0};
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float f = (uint32_t)row[j] < (uint32_t)nrows ? w[j] : 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = __builtin_fmaf(f, v[j][i >> 2][i & 3], y[i]);
      }
    }
  }
  if (R != nullptr) {
    Residual8<BF16> res;
    res.load(static_cast<const char*>(R) + (t * ld_r + c) * (BF16 ? 2 : 4), d - c);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] += res.at(i);
  }
  const int64_t o = t * ld_y + c;
  if constexpr (BF16) {
    uint16_t* p = static_cast<uint16_t*>(Y) + o;
    if (c + 8 <= d) {
      *reinterpret_cast<u4_any*>(p) = u4{to_bf16x2(y[0], y[1]), to_bf16x2(y[2], y[3]), to_bf16x2(y[4], y[5]), to_bf16x2(y[6], y[7])};
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < d) p[i] = to_bf16(y[i]);
    }
  } else {
    float* p = static_cast<float*>(Y) + o;
    if (c + 8 <= d) {
      reinterpret_cast<f4_any*>(p)[0] = f4{y[0], y[1], y[2], y[3]};
      reinterpret_cast<f4_any*>(p)[1] = f4{y[4], y[5], y[6], y[7]};
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < d) p[i] = y[i];
    }
  }
}
}  // namespace

// The counts of as many workgroups as any call of up to `tokens` tokens has: beyond 256 times the tokens at once a workgroup takes more, and
// their number falls and rises again.
size_t stamp_route_ws(int tokens, int experts, int) {
  const int once = tokens_at_once(experts), blocks = (tokens + once - 1) / once;
  const size_t nb = blocks < kRtMaxBlocks ? blocks : kRtMaxBlocks;
  return (nb * ((size_t)experts + 1) * sizeof(uint16_t) + 255) / 256 * 256 + 256;
}

hipError_t stamp_launch_route(const stamp_routing_t& r, const void* logits, int bf16, int64_t ld, int renorm, void* ws, hipStream_t st) {
  RouteArgs a;
  a.r = r;
  a.logits = logits;
  a.ld = ld;
  a.renorm = renorm;
  a.per_block = tokens_per_block(r.tokens, r.experts);
  a.hist = static_cast<uint16_t*>(ws);
  const int nb = (r.tokens + a.per_block - 1) / a.per_block;
  if (nb <= 1) {
    if (bf16) k_route_top<true, true><<<1, kTopWaves * 64, 0, st>>>(a);
    else k_route_top<true, false><<<1, kTopWaves * 64, 0, st>>>(a);
  } else {
    if (bf16) k_route_top<false, true><<<nb, kTopWaves * 64, 0, st>>>(a);
    else k_route_top<false, false><<<nb, kTopWaves * 64, 0, st>>>(a);
    k_route_place<<<nb, kPlaceWaves * 64, 0, st>>>(a);
  }
  return hipGetLastError();
}

hipError_t stamp_launch_combine(const stamp_routing_t& r, const void* rows, int rows_bf16, int y_bf16, int64_t ld_rows, int nrows, const void* R, int64_t ld_r,
                                void* Y, int64_t ld_y, int d, hipStream_t st) {
  const int64_t blocks = ((int64_t)r.tokens * ((d + 7) / 8) + 255) / 256;
  auto* const k = !y_bf16 ? k_combine<false, false> : rows_bf16 ? k_combine<true, true> : k_combine<false, true>;
  k<<<(uint32_t)blocks, 256, 0, st>>>(r, rows, ld_rows, nrows, R, ld_r, Y, ld_y, d);
  return hipGetLastError();
}
