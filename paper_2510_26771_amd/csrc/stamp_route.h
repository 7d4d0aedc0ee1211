// Choosing experts: the k largest logits of a token and their weights, by the lanes of a wave.
#ifndef STAMP_ROUTE_H_
#define STAMP_ROUTE_H_

#include "stamp_fp8.h"

struct TopArgs {
  const void* logits;
  int64_t ld;
  int32_t experts, top_k, renorm;
};

#ifdef __HIPCC__
namespace f8 {

// order of floats as unsigned integers; 0 for what is masked.  -0 counts as 0.
__device__ __forceinline__ uint32_t order_key(float l) {
  if (!(l > -__builtin_inff())) return 0;
  const uint32_t b = __float_as_uint(l + 0.0f);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
// exp(l - top) to 2 ulp, where both may be +infinity: then they are equal.  The product with log2 e in two parts.
__device__ __forceinline__ float share(float l, float top) {
  if (l == top) return 1.0f;
  const float x = l - top, t = x * 1.44269502162933349609f;
  const float rest = __builtin_fmaf(x, 1.44269502162933349609f, -t) + x * 1.92596299112661746887e-8f;
  const float p = __builtin_amdgcn_exp2f(t);
  return p > 0.0f ? __builtin_fmaf(p, rest * 0.693147180559945f, p) : 0.0f;  // (rest is no number where x is -infinity)
}

// over the LANES lanes of a token, in all of them
template <int CTRL>
__device__ __forceinline__ uint32_t turn(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xf, 0xf, false);
}
template <int LANES, typename F>
__device__ __forceinline__ uint32_t over_lanes(uint32_t v, F f) {
  v = f(v, turn<0x128>(v));  // the row of 16 turned by 8, 4, 2, 1
  v = f(v, turn<0x124>(v));
  v = f(v, turn<0x122>(v));
  v = f(v, turn<0x121>(v));
  if constexpr (LANES == 64) {
    v = f(v, (uint32_t)__shfl_xor((int)v, 16));
    v = f(v, (uint32_t)__shfl_xor((int)v, 32));
  }
  return v;
}
template <int LANES>
__device__ __forceinline__ float sum_lanes(float v) {
  return __uint_as_float(over_lanes<LANES>(__float_as_uint(v), [](uint32_t x, uint32_t y) { return __float_as_uint(__uint_as_float(x) + __uint_as_float(y)); }));
}

// LANES lanes have a token, lane l of them experts NV l + j: 4 tokens a wave up to 256 experts (the vector ALU is the bound, and the
// steps over lanes cost the same for 1 and for 4 tokens).  The largest key, of the lowest expert, is taken top_k times.  A bf16 logit's key
// has 16 bits: with the expert below it in one word the largest word is the choice, and no two are equal.
// 32768 tokens, 8 of 256 experts: 18 us (the logits alone 3); 64 tokens, 6 of 64, with the sort in the same workgroup 6.5.
// put(t, k, id, weight) gets the choices of tokens tok0 .. tok1 - 1; id -1: none.
template <int W, int LANES, int NV, bool BF16, typename Put>
__device__ void top_tokens(const TopArgs& a, int tok0, int tok1, int wave, int lane, Put put) {
  constexpr int kTokens = 64 / LANES, kMine = LANES == 16 ? 2 : 1;  // top_k <= 32 = kMine * LANES (or less)
  const int E = a.experts, K = a.top_k, l0 = lane % LANES;
  auto value = [](uint32_t k) {
    if constexpr (BF16) return __uint_as_float(((k & 0x80000000u) ? k & 0x7fff0000u : ~k & 0xffff0000u));
    else return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k);
  };
  for (int tb = tok0 + wave * kTokens; tb < tok1; tb += W * kTokens) {
    const int t = tb + lane / LANES;
    const bool in = t < tok1;
    uint32_t key[NV];
    constexpr int kSize = BF16 ? 2 : 4, kWords = NV * kSize / 16;
    const char* const row = static_cast<const char*>(a.logits) + ((int64_t)(in ? t : tok0) * a.ld + l0 * NV) * kSize;
    uint32_t raw[NV];  // the logits as fp32
    if (kWords > 0 && (l0 + 1) * NV <= E) {
#pragma unroll
      for (int w = 0; w < kWords; ++w) {
        const u4 v = reinterpret_cast<const u4_any*>(row)[w];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (BF16) raw[8 * w + 2 * i] = v[i] << 16, raw[8 * w + 2 * i + 1] = v[i] & 0xffff0000u;
          else raw[4 * w + i] = v[i];
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        raw[j] = 0xff800000u;
        if (l0 * NV + j < E) raw[j] = BF16 ? (uint32_t)reinterpret_cast<const uint16_t*>(row)[j] << 16 : reinterpret_cast<const uint32_t*>(row)[j];
      }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      key[j] = in ? order_key(__uint_as_float(raw[j])) : 0;
      if constexpr (BF16) key[j] = key[j] == 0 ? 0 : (key[j] & 0xffff0000u) | (uint32_t)(0xffff - (l0 * NV + j));
    }
    uint32_t mine[kMine] = {};  // lane l: key of the chosen l, l + 16
    int id[kMine];
#pragma unroll
    for (int q = 0; q < kMine; ++q) id[q] = -1;
    float top = 0.0f, sum = 0.0f;
    for (int k = 0; k < K; ++k) {
      uint32_t best = key[0];
#pragma unroll
      for (int j = 1; j < NV; ++j) best = max(best, key[j]);
      best = over_lanes<LANES>(best, [](uint32_t x, uint32_t y) { return max(x, y); });
      uint32_t e;
      if constexpr (BF16) {
        e = 0xffffu - (best & 0xffffu);
      } else {
        uint32_t at = 0xffffffffu;
#pragma unroll
        for (int j = NV - 1; j >= 0; --j) at = key[j] == best ? (uint32_t)j : at;
        e = over_lanes<LANES>(at == 0xffffffffu ? at : at + l0 * NV, [](uint32_t x, uint32_t y) { return min(x, y); });
      }
      if (k == 0) {
        top = value(best);
        if (!a.renorm) {
          float s = 0.0f;
#pragma unroll
          for (int j = 0; j < NV; ++j) s += key[j] != 0 ? share(value(key[j]), top) : 0.0f;
          sum = sum_lanes<LANES>(s);
        }
      }
      if (best == 0) continue;  // nothing left of this token (the wave's others may go on)
      if (l0 == k % LANES) {
#pragma unroll
        for (int q = 0; q < kMine; ++q)
          if (k / LANES == q) mine[q] = best, id[q] = (int)e;
      }
      const uint32_t gone = e - l0 * NV;  // j where the chosen one is this lane's
#pragma unroll
      for (int j = 0; j < NV; ++j) key[j] = (BF16 ? key[j] == best : gone == (uint32_t)j) ? 0 : key[j];
    }
    float sh[kMine], s = 0.0f;
#pragma unroll
    for (int q = 0; q < kMine; ++q) {
      sh[q] = id[q] >= 0 ? share(value(mine[q]), top) : 0.0f;
      s += sh[q];
    }
    if (a.renorm) sum = sum_lanes<LANES>(s);
#pragma unroll
    for (int q = 0; q < kMine; ++q) {
      const int k = l0 + q * LANES;
      if (in && k < K) put(t, k, id[q], id[q] >= 0 ? sh[q] / sum : 0.0f);
    }
  }
}

}  // namespace f8
#endif
#endif  // STAMP_ROUTE_H_
