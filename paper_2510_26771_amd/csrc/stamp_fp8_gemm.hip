// Product of the 8-bit floating point layers in tiles of BM rows x 256 places.
//
// Eight waves, 2 x 4, of BM / 2 x 64 each; the operands of a block of 128 channels are one stage in LDS, two stages of 256 rows or three of
// fewer (a step of 64 or 128 rows takes 0.4 to 0.9 us, which a load asked for one step ahead does not always meet).  The weights' stage is
// a copy of the operand image.  The rows' stage is [row][8 pieces of 16 bytes], piece p at p ^ (row / 2 % 8): the 16 lanes that are
// read at a time then hit all 64 banks once (also where they are lanes 0-3, 12-15 and 20-27, which take pieces f and f + 1 of 8 rows each).
//
// A wave's turn from one stage to the next lies before its last row block of the stage: all its reads of this stage have returned, its
// loads into the next have landed; behind the barrier it asks for the stage that takes this one's place and reads the next one's first
// operands under the last block's matrix instructions.
//
// Sums in fp32 (kWide): the rows come as bf16 (the quantizer widens the codes, or k_f8_widen: half of the kernel's conversions otherwise, and
// the vector ALU its bound), 256 bytes a row, piece p of 16 at p ^ (row % 16); the weights are widened once per step and wave
// (conversions among the matrix instructions, see wide_step: in a row of their own they leave the matrix pipe idle in both waves of a SIMD).
//
// Bound: the clock under the matrix load (1.8 to 1.9 of 2.4 GHz) and the matrix pipe's pauses (busy in 61 to 71 % of those cycles; counters at
// 8192 x 8192 -> 8192).  There 425 to 448 us, 2.45 to 2.59 PFLOP/s (the instructions alone, operands constant: 4.25; with zeros as operands this
// kernel 3.05); scales that are powers of two 2.76 to 2.85; sums in fp32 900 us, 1.22 PFLOP/s (instructions with their conversions and additions alone
// 1.65).  Short depths add a tile's start and end, 3 to 9 us.
//
// Few tiles: the depth in parts, each tile by as many workgroups, whose fp32 rows k_f8_join adds up in order.
//
// STAMP_SCALE_F32: an instruction's sum over the block of channels (its addend is 0) goes to the accumulators by a multiplication with
// both scales, 4 fused multiply-adds per instruction, one row block behind, so that the matrix pipe (32 cycles an instruction) runs on.
#include <type_traits>

#include "stamp_fp8.h"

namespace {
using namespace f8;

typedef __attribute__((address_space(3))) void* LdsPtr;

#if defined(__HIP_DEVICE_COMPILE__)
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }
// buffer over 4 GB from a uniform address on
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void* p) {
  const uint64_t u = reinterpret_cast<uint64_t>(p);
  const uint64_t v = (uint64_t)uniform((uint32_t)(u >> 32)) << 32 | uniform((uint32_t)u);
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(v), 0, (int)0xfffffff0u, 0x00027000);
}
#endif

// How the products are summed: FP8 instructions with the scales by multiplication or as their own, or bf16 instructions (f8_wide_sums).
enum Sums { kScaled, kPow2, kWide };

[[maybe_unused]] constexpr int kMaxBlocks = 65536 / kF8Block;

template <int BM, Sums SUMS, bool GATED>
__global__ __launch_bounds__(512) void k_f8_tiles(StampF8Gemm a) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr bool POW2 = SUMS == kPow2, WIDE = SUMS == kWide;
  constexpr int kRowBytes = WIDE ? 256 : 128;
  constexpr int kStageA = BM * kRowBytes, kStageB = 4 * kF8GroupBytes;
  constexpr int MI = BM / 32;         // row blocks of 16 per wave
  constexpr int LA = kStageA / 8192;  // 16-byte pieces of the rows' stage per thread
  constexpr int NS = kStageA > 16384 ? 2 : 3;                 // stages
  constexpr int kStage = kStageA + kStageB + 8 * 256;         // with 64 row scales per wave (those of the first BM / 64 waves are used)
  // variables of their own, not one array: the compiler then knows that a read of one stage does not wait for the loads into the others
  __shared__ __attribute__((aligned(1024))) uint8_t stage0[kStage];
  __shared__ __attribute__((aligned(1024))) uint8_t stage1[kStage];
  __shared__ __attribute__((aligned(1024))) uint8_t stage2[NS > 2 ? kStage : 16];
  __shared__ float wscale[2][kMaxBlocks];
  __shared__ float bias_of[GATED ? 1 : 256];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = wave >> 2, wn = wave & 3;
  // Workgroups go to the 8 XCDs in turn: an XCD takes a run of the tiles in an order in which 32 neighbours (its CUs) are 8 x 4 tiles, so
  // that its L2 has 12 panels of operands to fetch for them and not 33.
  constexpr int kXcd = 8, kBand = 8;
  const Tiles tiles = count_tiles(a, BM);
  const int ncol = (a.groups + 3) / 4, nrow = tiles.total, ntile = nrow * ncol, run = (ntile + kXcd - 1) / kXcd;
  const uint32_t group = a.first + blockIdx.x;
  const int order = (int)(group % kXcd) * run + (int)(group / kXcd);
  if ((int)(group / kXcd) >= run || order >= ntile) return;
  const int band = order / (kBand * ncol), in_band = order - band * kBand * ncol, height = min(kBand, nrow - band * kBand);
  const int col = in_band / height;
  int set, row0, nrows;
  find_tile(a, tiles, BM, band * kBand + in_band % height, &set, &row0, &nrows);
  set = __builtin_amdgcn_readfirstlane(set);
  row0 = __builtin_amdgcn_readfirstlane(row0);
  nrows = __builtin_amdgcn_readfirstlane(nrows);
  // its part of the depth: blocks kb0 .. kb0 + Kb - 1
  const int g0 = col * 4, depth = a.Kb, parts = gridDim.y, part_no = blockIdx.y;
  const int kb0 = depth * part_no / parts, Kb = depth * (part_no + 1) / parts - kb0;

  // 32-bit offsets from a scalar base: the tile's first row, or (gated, by index) all rows of A, below 4 GB
  uint32_t aoff[LA], boff[4], soff;
#pragma unroll
  for (int i = 0; i < 4; ++i) boff[i] = uniform((uint32_t)(min(g0 + i, a.groups - 1) - g0) * (uint32_t)depth * kF8GroupBytes);
  const __amdgpu_buffer_rsrc_t ra = buffer(a.A + (GATED ? (size_t)0 : (size_t)row0 * depth * kRowBytes) + (size_t)kb0 * kRowBytes);
  const __amdgpu_buffer_rsrc_t rb = buffer(a.W + (((size_t)set * a.groups + g0) * depth + kb0) * kF8GroupBytes);
  const float* const sa = a.SA + (GATED ? 0 : row0) + (int64_t)kb0 * a.ld_sa;

  // the q-th of a stage's loads; behind the last block of channels that one again, which nobody reads
  constexpr int kLoads = 4 + LA + 1;
  auto load = [&](uint8_t* S, int kb, int q) __attribute__((always_inline)) {
    kb = min(kb, Kb - 1);
    if (q < 4) {
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (LdsPtr)(S + kStageA + q * 8192 + wave * 1024), 16, t * 16, boff[q] + kb * kF8GroupBytes, 0, 0);
    } else if (q < 4 + LA) {
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (LdsPtr)(S + (q - 4) * 8192 + wave * 1024), 16, aoff[q - 4], kb * kRowBytes, 0, 0);
    } else {
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(sa + (int64_t)kb * a.ld_sa + soff),
                                       (LdsPtr)(S + kStageA + kStageB + wave * 256), 4, 0, 0);
    }
  };

  f4 acc[MI][4], P[4];
#pragma unroll
  for (int mi = 0; mi < MI; ++mi)
#pragma unroll
    for (int b = 0; b < 4; ++b) acc[mi][b] = f4{0, 0, 0, 0};
#pragma unroll
  for (int b = 0; b < 4; ++b) P[b] = f4{0, 0, 0, 0};
  const int x = ((lane & 15) >> 1) & 7, f = lane >> 4;
  const int abase = (wm * (BM / 2) + (lane & 15)) * kRowBytes, p0 = abase + (f ^ x) * 16, p1 = abase + ((f + 4) ^ x) * 16;
  const int wbase = kStageA + wn * kF8GroupBytes + lane * 16, sbase = kStageA + kStageB + (wm * (BM / 2) + (lane & 15)) * 4;

  // weight scales of the tile's two blocks of 128 columns (gated: of its gate and up columns): a register that now and then is loaded
  // anew would make every use of it wait for the loads in flight
  const float* const sw_of = wscale[GATED ? 0 : wn >> 1];
  auto read_w = [&](const uint8_t* S, int b) __attribute__((always_inline)) -> v8i {
    const uint8_t* s = S + wbase + b * 2048;
    return __builtin_shufflevector(*reinterpret_cast<const v4i*>(s), *reinterpret_cast<const v4i*>(s + 1024), 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto read_x1 = [&](const uint8_t* S, int mi, int k) __attribute__((always_inline)) -> b8 {
    return *reinterpret_cast<const b8*>(S + abase + mi * 16 * kRowBytes + ((8 * (k >> 1) + 2 * f + (k & 1)) ^ (lane & 15)) * 16);
  };
  auto read_x = [&](const uint8_t* S, int mi) __attribute__((always_inline)) -> v8i {
    return __builtin_shufflevector(*reinterpret_cast<const v4i*>(S + p0 + mi * 2048), *reinterpret_cast<const v4i*>(S + p1 + mi * 2048), 0, 1, 2, 3, 4, 5, 6,
                                   7);
  };
  auto read_s = [&](const uint8_t* S, int mi) __attribute__((always_inline)) { return *reinterpret_cast<const float*>(S + sbase + mi * 64); };
  // all but the youngest `left` of the own loads have landed and the own reads returned; then everyone's
  auto turn = [&](auto left) __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(0x0070 | decltype(left)::value);  // vmcnt(left) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  auto add = [&](f4& c, const f4& p, float fs) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < 4; ++r) c[r] = __builtin_fmaf(p[r], fs, c[r]);
    asm volatile("" : "+v"(c));  // here, not where the value is next used: the products would pile up
  };

  v8i W[4], X;
  float sx, sw, su, fg = 0.0f, fu = 0.0f;  // fg, fu: factors of the row block before
  constexpr std::integral_constant<int, 0> none;
  constexpr std::integral_constant<int, (NS - 2) * kLoads> later;  // the loads of the stages behind the next
  static_assert(later <= 15, "one field of the wait");
  // the step of stage S; N: the next one's stage; B: the one of the step before, which is being filled again
  auto step = [&](uint8_t* S, uint8_t* N, uint8_t* B, int kb) __attribute__((always_inline)) {
    float next_w = 0.0f, next_u = 0.0f;
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
      if constexpr (POW2) {
#pragma unroll
        for (int b = 0; b < 4; ++b) asm volatile("" : "+v"(acc[(mi + MI / 2) % MI][b]));
      }
      v8i Xn;
      float sn;
      if (mi < MI - 1) {
        Xn = read_x(S, mi + 1);
        sn = read_s(S, mi + 1);
      } else {
        turn(later);
        Xn = read_x(N, 0);
        sn = read_s(N, 0);
        next_w = sw_of[min(kb + 1, Kb - 1)];
        if (GATED) next_u = wscale[1][min(kb + 1, Kb - 1)];
      }
      const float f0 = sx * sw, f1 = GATED ? sx * su : 0.0f;
      const int before = mi == 0 ? MI - 1 : mi - 1;
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        if constexpr (POW2) {
          acc[mi][b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(W[b], X, acc[mi][b], 0, 0, 0, (int)(__float_as_uint(GATED && (b & 1) ? su : sw) >> 23),
                                                                       0, (int)(__float_as_uint(sx) >> 23));
        } else {
          add(acc[before][b], P[b], GATED && (b & 1) ? fu : fg);
          const f4 z = {0, 0, 0, 0};
          P[b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(W[b], X, z, 0, 0, 0, 0, 0, 0);
        }
        // the stage's loads one by one: all at once they would keep the address unit busy, and the matrix pipe waiting
        if (mi == MI - 1) {
          W[b] = read_w(N, b);
          load(S, kb + NS, b);
        }
        if (mi == 0) {
#pragma unroll
          for (int q = 4 + b; q < kLoads; q += 4) load(B, kb - 1 + NS, q);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      X = Xn;
      sx = sn;
      fg = f0;
      fu = f1;
    }
    sw = next_w;
    su = next_u;
  };

  // kWide: by blocks of 16 places, so that the conversions of a block's weights lie among the 4 MI matrix instructions of the block before;
  // all rows of the stage are in registers, and the turn lies before the last block.
  b8 XW[MI][4];
  b8 Wb[2][4];
  v8i raw;
  f4 PW[MI];
  float sxw[MI], f0[MI], f1[MI];  // f0, f1: this step's factors (of the gate and the up columns)
  float fold[MI];                 // of the block before
  auto widen_w = [&](b8(&w)[4], const v8i& r) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = widen8(r[2 * k], r[2 * k + 1]);
  };
  auto wide_step = [&](uint8_t* S, uint8_t* N, uint8_t* B, int kb) __attribute__((always_inline)) {
    float next_w = 0.0f, next_u = 0.0f, sn[MI];
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
      f0[mi] = sxw[mi] * sw;
      f1[mi] = GATED ? sxw[mi] * su : 0.0f;
    }
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      if (b == 3) {
        turn(later);
        next_w = sw_of[min(kb + 1, Kb - 1)];
        if (GATED) next_u = wscale[1][min(kb + 1, Kb - 1)];
      }
      raw = b < 3 ? read_w(S, b + 1) : read_w(N, 0);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) {
          if (k == 0) add(acc[mi][(b + 3) & 3], PW[mi], fold[mi]);
          const f4 z = {0, 0, 0, 0};
          PW[mi] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(Wb[b & 1][k], XW[mi][k], k == 0 ? z : PW[mi], 0, 0, 0);
          if (b == 3) XW[mi][k] = read_x1(N, mi, k);
        }
        if (b == 3) {
          load(S, kb + NS, k);
          if (k == 0) {
#pragma unroll
            for (int mi = 0; mi < MI; ++mi) sn[mi] = read_s(N, mi);
          }
        }
        if (b == 0) {
#pragma unroll
          for (int q = 4 + k; q < kLoads; q += 4) load(B, kb - 1 + NS, q);
        }
        if (k == 1) widen_w(Wb[(b + 1) & 1], raw);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int mi = 0; mi < MI; ++mi) fold[mi] = GATED && (b & 1) ? f1[mi] : f0[mi];
    }
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) sxw[mi] = sn[mi];
    sw = next_w;
    su = next_u;
  };
  auto any_step = [&](uint8_t* S, uint8_t* N, uint8_t* B, int kb) __attribute__((always_inline)) {
    if constexpr (WIDE) wide_step(S, N, B, kb);
    else step(S, N, B, kb);
  };

  // The start: the small loads first (they return in order), so that the rows' numbers (GATED) are there before the weights, which wait for
  // nothing; and the steps begin while the second stage is on its way.  191 experts of 896 -> 1054, gated, 200 rows each: 419 -> 411 us of the whole MLP.
  auto scale_at = [&](int i) __attribute__((always_inline)) {
    const int which = i >= Kb, kb = i - which * Kb;
    const int blk = GATED ? which * a.nblk + (min(g0, a.groups - 1) >> 2) : min((g0 >> 1) + which, a.nblk - 1);
    return a.SW[((size_t)set * (GATED ? 2 : 1) * a.nblk + blk) * depth + kb0 + kb];
  };
  const float scale0 = t < 2 * Kb ? scale_at(t) : 0.0f;
  float bias0 = 0.0f;
  if constexpr (!GATED) {
    const int n = g0 * 64 + t;
    if (t < 256 && a.bias != nullptr && n < a.N && part_no == 0) bias0 = a.bias[(size_t)set * a.N + n];
  }
  int from[LA + 1];  // rows of A: of the thread's pieces, and of its scale
#pragma unroll
  for (int i = 0; i <= LA; ++i) {
    from[i] = min(i < LA ? (WIDE ? (i * 512 + t) >> 4 : (i * 512 + t) >> 3) : t, nrows - 1);
    if constexpr (GATED) from[i] = a.index[row0 + from[i]];
  }
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int q = 0; q < 4; ++q) load(stage0, 0, q);
  if constexpr (NS == 3) {
#pragma unroll
    for (int q = 0; q < 4; ++q) load(stage1, 1, q);
  }
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int i = 0; i < LA; ++i) {
    const int p = i * 512 + t, row = WIDE ? p >> 4 : p >> 3, piece = WIDE ? (p & 15) ^ (row & 15) : (p & 7) ^ ((row >> 1) & 7);
    if constexpr (GATED) from[i] = min(max(from[i], 0), a.a_rows - 1);
    aoff[i] = (uint32_t)from[i] * (uint32_t)(depth * kRowBytes) + piece * 16;
  }
  soff = (uint32_t)(GATED ? min(max(from[LA], 0), a.a_rows - 1) : from[LA]);
#pragma unroll
  for (int q = 4; q < kLoads; ++q) load(stage0, 0, q);
  __builtin_amdgcn_sched_barrier(0);
  if constexpr (NS == 3) {
#pragma unroll
    for (int q = 4; q < kLoads; ++q) load(stage1, 1, q);
  }
  __builtin_amdgcn_sched_barrier(0);
  if (t < 2 * Kb) wscale[t >= Kb][t >= Kb ? t - Kb : t] = scale0;
  for (int i = t + 512; i < 2 * Kb; i += 512) wscale[i >= Kb][i >= Kb ? i - Kb : i] = scale_at(i);
  if constexpr (!GATED) {
    if (t < 256) bias_of[t] = bias0;
  }
  turn(std::integral_constant<int, (NS - 2) * (kLoads - 4)>());
#pragma unroll
  for (int q = 0; q < 4; ++q) load(NS == 3 ? stage2 : stage1, NS - 1, q);
  if constexpr (WIDE) {
    widen_w(Wb[0], read_w(stage0, 0));
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
#pragma unroll
      for (int k = 0; k < 4; ++k) XW[mi][k] = read_x1(stage0, mi, k);
      sxw[mi] = read_s(stage0, mi);
      PW[mi] = f4{0, 0, 0, 0};
      fold[mi] = 0.0f;
    }
  } else {
#pragma unroll
    for (int b = 0; b < 4; ++b) W[b] = read_w(stage0, b);
    X = read_x(stage0, 0);
    sx = read_s(stage0, 0);
  }
  sw = sw_of[0];
  su = wscale[1][0];
  int kb = 0;
  if constexpr (NS == 2) {
    for (; kb + 1 < Kb; kb += 2) {
      any_step(stage0, stage1, stage1, kb);
      any_step(stage1, stage0, stage0, kb + 1);
    }
    if (kb < Kb) any_step(stage0, stage1, stage1, kb);
  } else {
    for (; kb + 2 < Kb; kb += 3) {
      any_step(stage0, stage1, stage2, kb);
      any_step(stage1, stage2, stage0, kb + 1);
      any_step(stage2, stage0, stage1, kb + 2);
    }
    if (kb < Kb) any_step(stage0, stage1, stage2, kb);
    if (kb + 1 < Kb) any_step(stage1, stage2, stage0, kb + 1);
  }
  if constexpr (WIDE) {
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) add(acc[mi][3], PW[mi], fold[mi]);
  } else if constexpr (!POW2) {
#pragma unroll
    for (int b = 0; b < 4; ++b) add(acc[MI - 1][b], P[b], GATED && (b & 1) ? fu : fg);
  }

  __builtin_amdgcn_s_waitcnt(0x0070);  // no load into LDS may outlive the workgroup

  const int g = g0 + wn;
  if constexpr (!GATED) {
    const int n0 = 64 * g + 8 * f;  // and 32 further on
    float bias[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) bias[j] = bias_of[64 * wn + 32 * (j >> 3) + 8 * f + (j & 7)];
    // one of several parts: fp32 rows of all places into its own piece of the scratch memory, for k_f8_join
    const bool whole = parts == 1, bf16 = whole && a.y_bf16;
    const int N = whole ? a.N : a.groups * 64;
    const int64_t ld_y = whole ? a.ld_y : N;
    const uint32_t size = bf16 ? 2 : 4, ld = (uint32_t)ld_y * size;
    char* const base = whole ? static_cast<char*>(a.Y) : reinterpret_cast<char*>(a.partial + (int64_t)part_no * a.rows * N);
    char* const y = base + ((int64_t)row0 * ld_y) * size;  // 256 rows are below 4 GB, checked by the host
    // 8 columns at a time wherever the row begins, element by element in the last 8 only: 4742 x 576 -> 7644 (rows 8 bytes off the grid of 16)
    // took 108 us with elements throughout, 44 so, and 7680 columns take 43.  bf16 rows that begin between two words are slow to store all the same
    // (8192 x 1152 -> 4607 79 us, rows 4608 apart 58): there a lane stores its words from the second element on, the last one with the next lane's
    // first element, and the ends of the wave's 64 columns one by one.
    const bool between = bf16 && ((reinterpret_cast<uintptr_t>(base) | ld) & 2) != 0 && 64 * g + 64 <= N;
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
      const int m = wm * (BM / 2) + 16 * mi + (lane & 15);
      char* const o = y + ((uint32_t)m * ld + (uint32_t)n0 * size);
      float v[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] = acc[mi][j >> 2][j & 3] + bias[j];
      u4 w[2];
      if (bf16) {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j >> 2][j & 3] = to_bf16x2(v[2 * j], v[2 * j + 1]);
      }
      if (between) {
        // lanes f = 1, 2, 3 give their first word, f = 0 that of the second 32 columns
        const uint32_t next0 = (uint32_t)__shfl((int)(f == 0 ? w[1][0] : w[0][0]), (lane + 16) & 63);
        const uint32_t next1 = (uint32_t)__shfl((int)w[1][0], (lane + 16) & 63);
        if (m >= nrows) continue;
        const bool odd = (reinterpret_cast<uintptr_t>(o) & 2) != 0;
        const uint16_t first = (uint16_t)w[0][0], last = (uint16_t)(w[1][3] >> 16);
        if (odd) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j) w[h][j] = __builtin_amdgcn_alignbit(j < 3 ? w[h][j + 1] : h == 0 ? next0 : next1, w[h][j], 16);
        }
        char* const p = o + (odd ? 2 : 0);
        *reinterpret_cast<u4_any*>(p) = w[0];
        if (odd && f == 3) {
          *reinterpret_cast<u2_any*>(p + 64) = u2{w[1][0], w[1][1]};
          *reinterpret_cast<uint32_t*>(p + 72) = w[1][2];
          *reinterpret_cast<uint16_t*>(p + 76) = last;
        } else {
          *reinterpret_cast<u4_any*>(p + 64) = w[1];
        }
        if (odd && f == 0) *reinterpret_cast<uint16_t*>(o) = first;
        continue;
      }
      if (m >= nrows) continue;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int left = N - n0 - 32 * h;
        char* const p = o + 32 * h * size;
        if (bf16) {
          if (left >= 8) {
            *reinterpret_cast<u4_any*>(p) = w[h];
          } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (j < left) reinterpret_cast<uint16_t*>(p)[j] = (uint16_t)(w[h][j >> 1] >> (16 * (j & 1)));
          }
        } else if (left >= 8) {
#pragma unroll
          for (int q = 0; q < 2; ++q)
            reinterpret_cast<u4_any*>(p)[q] = u4{__float_as_uint(v[8 * h + 4 * q]), __float_as_uint(v[8 * h + 4 * q + 1]), __float_as_uint(v[8 * h + 4 * q + 2]),
                                                 __float_as_uint(v[8 * h + 4 * q + 3])};
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (j < left) reinterpret_cast<float*>(p)[j] = v[8 * h + j];
        }
      }
    }
  } else {
    // a lane has 8 neighbouring columns of gate and up; the tile's 128 columns are a block of the next layer's input
    float* part = reinterpret_cast<float*>(stage0);  // [4][BM] largest magnitudes of the waves' 32 columns, as bits
    const int n0 = 32 * g + 8 * f;
    turn(none);
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
    turn(none);
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
      const int m = wm * (BM / 2) + 16 * mi + (lane & 15);
      uint32_t amax = 0;
#pragma unroll
      for (int w = 0; w < 4; ++w) amax = max(amax, __float_as_uint(part[w * BM + m]));
      float scale, inv;
      scale_of(amax, a.pow2, &scale, &inv);
      if (m >= nrows) continue;
      u2 o;
      o[0] = pack4(acc[mi][0][0] * inv, acc[mi][0][1] * inv, acc[mi][0][2] * inv, acc[mi][0][3] * inv);
      o[1] = pack4(acc[mi][2][0] * inv, acc[mi][2][1] * inv, acc[mi][2][2] * inv, acc[mi][2][3] * inv);
      *reinterpret_cast<u2*>(static_cast<uint8_t*>(a.Y) + (int64_t)(row0 + m) * a.ld_y + 32 * g + 8 * f) = o;
      if (wn == 0 && f == 0) a.SH[(int64_t)col * a.ld_sh + row0 + m] = scale;
    }
  }
#endif
}

__global__ __launch_bounds__(256) void k_f8_widen(const uint8_t* codes, int64_t n16, uint8_t* out, int64_t first) {
  const int64_t u = (first + blockIdx.x) * 256 + threadIdx.x;
  if (u >= n16) return;
  const u4 c = reinterpret_cast<const u4*>(codes)[u];
  reinterpret_cast<b8*>(out)[2 * u] = widen8((int)c[0], (int)c[1]);
  reinterpret_cast<b8*>(out)[2 * u + 1] = widen8((int)c[2], (int)c[3]);
}

// Y = sum of the parts, in order.  A thread has 4 columns of a row and all parts in flight.  Bound by its launch: 4 parts of 1310 x 384 4.3 us.
template <int PARTS>
__global__ __launch_bounds__(256) void k_f8_join(StampF8Gemm a) {
  const int N = a.groups * 64, per = (a.N + 3) / 4;
  const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x, m = u / per;
  const int c = (int)(u - m * per) * 4;
  const int rows = a.offsets == nullptr ? a.rows : min(max(a.offsets[a.sets], 0), a.rows);
  if (m >= rows) return;
  const f4* p = reinterpret_cast<const f4*>(a.partial + m * N + c);
  f4 v[PARTS];
#pragma unroll
  for (int i = 0; i < PARTS; ++i) v[i] = p[(int64_t)i * a.rows * (N / 4)];
  f4 s = v[0];
#pragma unroll
  for (int i = 1; i < PARTS; ++i) s += v[i];
  if (a.y_bf16) {
    uint16_t* y = static_cast<uint16_t*>(a.Y) + m * a.ld_y + c;
    if (c + 4 <= a.N) {
      *reinterpret_cast<u2_any*>(y) = u2{to_bf16x2(s[0], s[1]), to_bf16x2(s[2], s[3])};
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (c + j < a.N) y[j] = to_bf16(s[j]);
    }
  } else {
    float* y = static_cast<float*>(a.Y) + m * a.ld_y + c;
    if (c + 4 <= a.N) {
      *reinterpret_cast<f4_any*>(y) = s;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (c + j < a.N) y[j] = s[j];
    }
  }
}

template <int BM>
hipError_t go(const StampF8Gemm& a, int parts, hipStream_t st) {
  const int64_t tiles = a.offsets == nullptr ? ((int64_t)a.rows + BM - 1) / BM : (int64_t)a.rows / BM + (a.sets < a.rows ? a.sets : a.rows);
  if (BM == 256 && a.wide_sums) return hipErrorInvalidValue;  // its registers do not hold the bf16 operands: never chosen
  // a launch's first workgroup is a multiple of 8: the XCDs keep their turn
  const hipError_t e = f8_launches((tiles * ((a.groups + 3) / 4) + 7) / 8 * 8, 512, [&](int64_t first, uint32_t n) {
    const dim3 grid(n, parts);
    StampF8Gemm part = a;
    part.first = (uint32_t)first;
    if constexpr (BM == 256) {
      if (a.pow2) k_f8_tiles<BM, kPow2, false><<<grid, 512, 0, st>>>(part);
      else k_f8_tiles<BM, kScaled, false><<<grid, 512, 0, st>>>(part);
    } else {
      if (a.gated) k_f8_tiles<BM, kWide, true><<<grid, 512, 0, st>>>(part);
      else if (a.wide_sums) k_f8_tiles<BM, kWide, false><<<grid, 512, 0, st>>>(part);
      else if (a.pow2) k_f8_tiles<BM, kPow2, false><<<grid, 512, 0, st>>>(part);
      else k_f8_tiles<BM, kScaled, false><<<grid, 512, 0, st>>>(part);
    }
  });
  if (e != hipSuccess) return e;
  if (parts > 1) {
    const int64_t n = (int64_t)a.rows * ((a.N + 3) / 4);
    static_assert(kF8MaxParts == 8, "a kernel for every number of parts");
    auto* const join = parts == 2   ? k_f8_join<2>
                       : parts == 3 ? k_f8_join<3>
                       : parts == 4 ? k_f8_join<4>
                       : parts == 5 ? k_f8_join<5>
                       : parts == 6 ? k_f8_join<6>
                       : parts == 7 ? k_f8_join<7>
                                    : k_f8_join<8>;
    join<<<(uint32_t)((n + 255) / 256), 256, 0, st>>>(a);
  }
  return hipGetLastError();
}
}  // namespace

hipError_t stamp_launch_f8_widen(const uint8_t* codes, int64_t bytes, uint8_t* out, hipStream_t st) {
  return f8_launches((bytes / 16 + 255) / 256, 256,
                     [&](int64_t first, uint32_t n) { k_f8_widen<<<n, 256, 0, st>>>(codes, bytes / 16, out, first); });
}

hipError_t stamp_launch_f8_tiles(const StampF8Gemm& a, int bm, int parts, hipStream_t st) {
  return bm == 64 ? go<64>(a, parts, st) : bm == 128 ? go<128>(a, parts, st) : go<256>(a, parts, st);
}
