// Product of the 8-bit floating point layers in tiles of BM rows x 256 places.
//
// Eight waves, 2 x 4, of BM / 2 x 64 each; the operands of a block of 128 channels are one stage in LDS, two stages, the next one filled
// by asynchronous 16-byte loads while this one is multiplied.  The weights' stage is a copy of the operand image.  The rows' stage is
// [row][8 pieces of 16 bytes], piece p at p ^ (row / 2 % 8): the 16 lanes of a read then hit all 64 banks once.
#include "stamp_fp8.h"

namespace {
using namespace f8;

typedef __attribute__((address_space(3))) void* LdsPtr;
typedef const __attribute__((address_space(1))) void* GlobalPtr;

template <int BM, bool POW2, bool GATED>
__global__ __launch_bounds__(512) void k_f8_tiles(StampF8Gemm a) {
  constexpr int kStageA = BM * 128, kStageB = 4 * kF8GroupBytes;
  constexpr int MI = BM / 32;  // instructions along the rows, per wave
  constexpr int LA = BM / 64;  // 16-byte pieces of the rows' stage per thread
  // two variables, not one array of two: the compiler then knows that a read of one stage does not wait for the loads into the other
  __shared__ __attribute__((aligned(1024))) uint8_t stage0[kStageA + kStageB + BM * 4];
  __shared__ __attribute__((aligned(1024))) uint8_t stage1[kStageA + kStageB + BM * 4];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = wave >> 2, wn = wave & 3;
  const int ncol = (a.groups + 3) / 4, col = blockIdx.x % ncol;  // consecutive workgroups share the rows' operand
  int set, row0, nrows;
  if (!find_tile(a, BM, blockIdx.x / ncol, &set, &row0, &nrows)) return;
  const int g0 = col * 4, Kb = a.Kb, Kp = Kb * 128;

  const uint8_t* asrc[LA];
#pragma unroll
  for (int i = 0; i < LA; ++i) {
    const int p = i * 512 + t, row = p >> 3, piece = (p & 7) ^ ((row >> 1) & 7);
    int r = row0 + min(row, nrows - 1);
    if (a.index != nullptr) r = min(max(a.index[r], 0), a.a_rows - 1);
    asrc[i] = a.A + (size_t)r * Kp + piece * 16;
  }
  const uint8_t* bsrc[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) bsrc[i] = a.W + ((size_t)set * a.groups + min(g0 + i, a.groups - 1)) * Kb * kF8GroupBytes + t * 16;
  const float* ssrc = a.SA + row0 + min(t, nrows - 1);

  auto load = [&](uint8_t* S, int kb) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < LA; ++i)
      __builtin_amdgcn_global_load_lds((GlobalPtr)(asrc[i] + (size_t)kb * 128), (LdsPtr)(S + i * 8192 + wave * 1024), 16, 0, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      __builtin_amdgcn_global_load_lds((GlobalPtr)(bsrc[i] + (size_t)kb * kF8GroupBytes), (LdsPtr)(S + kStageA + i * 8192 + wave * 1024), 16, 0, 0);
    if (wave < BM / 64)
      __builtin_amdgcn_global_load_lds((GlobalPtr)(ssrc + (int64_t)kb * a.ld_sa), (LdsPtr)(S + kStageA + kStageB + wave * 256), 4, 0, 0);
  };

  f4 acc[MI][4];
#pragma unroll
  for (int mi = 0; mi < MI; ++mi)
#pragma unroll
    for (int b = 0; b < 4; ++b) acc[mi][b] = f4{0, 0, 0, 0};
  const int gw = min(g0 + wn, a.groups - 1);
  const float* sw0 = a.SW + (size_t)set * (GATED ? 2 : 1) * a.nblk * Kb + (size_t)(GATED ? gw >> 2 : gw >> 1) * Kb;
  const int x = ((lane & 15) >> 1) & 7, f = lane >> 4;
  const int abase = (wm * (BM / 2) + (lane & 15)) * 128, p0 = ((2 * f) ^ x) * 16, p1 = ((2 * f + 1) ^ x) * 16;

  auto multiply = [&](const uint8_t* S, int kb) __attribute__((always_inline)) {
    v8i W[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const uint8_t* s = S + kStageA + wn * kF8GroupBytes + b * 2048 + lane * 16;
      W[b] = __builtin_shufflevector(*reinterpret_cast<const v4i*>(s), *reinterpret_cast<const v4i*>(s + 1024), 0, 1, 2, 3, 4, 5, 6, 7);
    }
    const float sw = sw0[kb], su = GATED ? sw0[(size_t)a.nblk * Kb + kb] : 0.0f;
    const float* SA = reinterpret_cast<const float*>(S + kStageA + kStageB) + wm * (BM / 2) + (lane & 15);
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
      const uint8_t* s = S + abase + mi * 2048;
      const v8i X = __builtin_shufflevector(*reinterpret_cast<const v4i*>(s + p0), *reinterpret_cast<const v4i*>(s + p1), 0, 1, 2, 3, 4, 5, 6, 7);
      const float sx = SA[16 * mi];
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const float sc = GATED && (b & 1) ? su : sw;
        if constexpr (POW2) {
          acc[mi][b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(W[b], X, acc[mi][b], 0, 0, 0, (int)(__float_as_uint(sc) >> 23), 0,
                                                                       (int)(__float_as_uint(sx) >> 23));
        } else {
          const f4 z = {0, 0, 0, 0};
          const f4 p = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(W[b], X, z, 0, 0, 0, 0, 0, 0);
          const float fs = sx * sc;
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[mi][b][r] = __builtin_fmaf(p[r], fs, acc[mi][b][r]);
        }
      }
    }
  };
  // the own loads have landed, the own reads returned; then everyone's
  auto turn = [&]() __attribute__((always_inline)) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  load(stage0, 0);
  for (int kb = 0; kb < Kb; kb += 2) {
    turn();
    if (kb + 1 < Kb) load(stage1, kb + 1);
    multiply(stage0, kb);
    if (kb + 1 >= Kb) break;
    turn();
    if (kb + 2 < Kb) load(stage0, kb + 2);
    multiply(stage1, kb + 1);
  }

  const int g = g0 + wn;
  if constexpr (!GATED) {
    const int n0 = 64 * g + 16 * f;
    float bias[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) bias[j] = a.bias != nullptr && n0 + j < a.N ? a.bias[(size_t)set * a.N + n0 + j] : 0.0f;
    const int size = a.y_bf16 ? 2 : 4;
    const bool wide = n0 + 16 <= a.N && (reinterpret_cast<uintptr_t>(a.Y) | (uintptr_t)(a.ld_y * size)) % 16 == 0;
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
      const int m = wm * (BM / 2) + 16 * mi + (lane & 15);
      if (m >= nrows) continue;
      const int64_t o = (int64_t)(row0 + m) * a.ld_y + n0;
      float v[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] = acc[mi][j >> 2][j & 3] + bias[j];
      if (a.y_bf16) {
        uint16_t* y = static_cast<uint16_t*>(a.Y) + o;
        if (wide) {
          u4 w[2];
#pragma unroll
          for (int j = 0; j < 8; ++j) w[j >> 2][j & 3] = to_bf16x2(v[2 * j], v[2 * j + 1]);
          reinterpret_cast<u4*>(y)[0] = w[0];
          reinterpret_cast<u4*>(y)[1] = w[1];
        } else {
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (n0 + j < a.N) y[j] = to_bf16(v[j]);
        }
      } else {
        float* y = static_cast<float*>(a.Y) + o;
        if (wide) {
#pragma unroll
          for (int j = 0; j < 4; ++j) reinterpret_cast<f4*>(y)[j] = f4{v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]};
        } else {
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (n0 + j < a.N) y[j] = v[j];
        }
      }
    }
  } else {
    // a lane has 8 neighbouring columns of gate and up; the tile's 128 columns are a block of the next layer's input
    float* part = reinterpret_cast<float*>(stage0);  // [4][BM] largest magnitudes of the waves' 32 columns, as bits
    const int n0 = 32 * g + 8 * f;
    turn();
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
      uint32_t amax = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int b = 2 * (j >> 2), r = j & 3;
        const float h = n0 + j < a.N ? silu(acc[mi][b][r]) * acc[mi][b + 1][r] : 0.0f;
        acc[mi][b][r] = h;
        amax = max(amax, abs_bits(h));
      }
      amax = max(amax, (uint32_t)__shfl_xor((int)amax, 16));
      amax = max(amax, (uint32_t)__shfl_xor((int)amax, 32));
      if (f == 0) part[wn * BM + wm * (BM / 2) + 16 * mi + lane] = __uint_as_float(amax);
    }
    turn();
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
      const int m = wm * (BM / 2) + 16 * mi + (lane & 15);
      uint32_t amax = 0;
#pragma unroll
      for (int w = 0; w < 4; ++w) amax = max(amax, __float_as_uint(part[w * BM + m]));
      float scale, inv;
      scale_of(amax, POW2, &scale, &inv);
      if (m >= nrows) continue;
      u2 o;
      o[0] = pack4(acc[mi][0][0] * inv, acc[mi][0][1] * inv, acc[mi][0][2] * inv, acc[mi][0][3] * inv);
      o[1] = pack4(acc[mi][2][0] * inv, acc[mi][2][1] * inv, acc[mi][2][2] * inv, acc[mi][2][3] * inv);
      *reinterpret_cast<u2*>(static_cast<uint8_t*>(a.Y) + (int64_t)(row0 + m) * a.ld_y + 32 * g + 8 * f) = o;
      if (wn == 0 && f == 0) a.SH[(int64_t)col * a.ld_sh + row0 + m] = scale;
    }
  }
}

template <int BM>
hipError_t go(const StampF8Gemm& a, hipStream_t st) {
  const int64_t tiles = a.offsets == nullptr ? ((int64_t)a.rows + BM - 1) / BM : (int64_t)a.rows / BM + (a.sets < a.rows ? a.sets : a.rows);
  const uint32_t grid = (uint32_t)(tiles * ((a.groups + 3) / 4));
  if (a.gated) {
    if (a.pow2) k_f8_tiles<BM, true, true><<<grid, 512, 0, st>>>(a);
    else k_f8_tiles<BM, false, true><<<grid, 512, 0, st>>>(a);
  } else {
    if (a.pow2) k_f8_tiles<BM, true, false><<<grid, 512, 0, st>>>(a);
    else k_f8_tiles<BM, false, false><<<grid, 512, 0, st>>>(a);
  }
  return hipGetLastError();
}
}  // namespace

hipError_t stamp_launch_f8_tiles(const StampF8Gemm& a, int bm, hipStream_t st) {
  return bm == 64 ? go<64>(a, st) : bm == 128 ? go<128>(a, st) : go<256>(a, st);
}
