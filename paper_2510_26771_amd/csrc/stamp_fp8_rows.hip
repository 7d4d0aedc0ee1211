// Product of the 8-bit floating point layers for few rows (on average per expert).
//
// Bound by the weights' bytes: every byte is read once and feeds one matrix instruction per 16 rows.  So nothing is staged: a wave takes
// blocks of 16 places and a part of the depth, and reads its operand straight into registers in runs of 1 KB; the parts of the depth
// are summed in LDS in a fixed order.  Always on the bf16 matrix instructions (f8_wide_sums): the pipe is idle most of the time.
//
// 1 x 4096 -> 11008: 9.9 us, 4.5 TB/s of weights; 96 rows over 27 of 32 experts, 4096 -> 1536: 27 us, 6.2 TB/s.
//
// Few rows the kernel quantizes itself, into LDS: X is asked for first, then the weights, and the codes are made while those are on their
// way (loads return in order).  Every workgroup does that again for its rows; a launch of its own is saved (2.6 us for one row, more than a
// quarter of the product).
#include "stamp_fp8.h"

namespace {
using namespace f8;

// where the rows come from: codes, or X in its type
enum Rows { kCodes, kBf16, kF32 };

// MT: tiles of 16 rows held at once.  NB: blocks of 16 places per wave.  S: parts of the depth; kWaves / S waves lie side by side.
template <int MT, int NB, int S, int kWaves, bool GATED, Rows IN>
__global__ __launch_bounds__(kWaves * 64, IN == kCodes ? 2 : 4) void k_f8_rows(StampF8Gemm a) {
  constexpr int kSide = kWaves / S;             // waves side by side
  constexpr int kPlaces = kSide * NB * 16;      // places of the workgroup
  constexpr int kLd = kPlaces + 4;              // floats of a row of partial sums
  constexpr int kRows = 16 * MT;
  // blocks of channels whose weights are asked for at once: 64 registers, 32 beside the rows' (two workgroups a CU then)
  constexpr int U = MT > 1 ? 1 : IN == kCodes ? 8 / NB : 4 / NB;
  // one after the other: codes [rows][Kp + 16] and scales [rows][Kb] of the rows quantized here; partial sums
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  float(*red)[kRows][kLd] = reinterpret_cast<float(*)[kRows][kLd]>(lds);
  const int chunk = IN == kCodes ? kRows : a.chunk;
  const int ldc = a.Kb * 128 + 16;
  float* lds_scale = reinterpret_cast<float*>(lds + chunk * ldc);
  const int t = threadIdx.x, lane = t & 63, f = lane >> 4, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int side = wave % kSide, part = wave / kSide;
  const int set = blockIdx.y;
  int lo, hi;
  rows_of(a, set, &lo, &hi);
  lo = __builtin_amdgcn_readfirstlane(lo);
  hi = __builtin_amdgcn_readfirstlane(hi);
  if (lo >= hi) return;
  const int blk0 = (blockIdx.x * kSide + side) * NB;  // first of the wave's blocks, counted over the groups
  const int g = blk0 >> 2, b0 = blk0 & 3;
  const bool in = g < a.groups;
  const int kb0 = (int)((int64_t)a.Kb * part / S), kb1 = in ? (int)((int64_t)a.Kb * (part + 1) / S) : kb0;
  const uint8_t* w0 = a.W + (((size_t)set * a.groups + (in ? g : 0)) * a.Kb) * kF8GroupBytes + b0 * 2048 + lane * 16;
  const float* sw0 = a.SW + (size_t)set * (GATED ? 2 : 1) * a.nblk * a.Kb + (size_t)(GATED ? (in ? g : 0) >> 2 : (in ? g : 0) >> 1) * a.Kb;
  const int Kp = a.Kb * 128;

  for (int r0 = lo; r0 < hi; r0 += chunk) {
    const int nr = min(chunk, hi - r0);
    f4 acc[MT][NB];
#pragma unroll
    for (int mi = 0; mi < MT; ++mi)
#pragma unroll
      for (int b = 0; b < NB; ++b) acc[mi][b] = f4{0, 0, 0, 0};
    const uint8_t* arow[MT];
    int srow[MT];
#pragma unroll
    for (int mi = 0; mi < MT; ++mi) {
      const int m = min(16 * mi + (lane & 15), nr - 1);
      if constexpr (IN == kCodes) {
        int ar = r0 + m;
        if constexpr (GATED) ar = min(max(a.index[ar], 0), a.a_rows - 1);
        arow[mi] = a.A + (size_t)ar * Kp + 16 * f;
        srow[mi] = ar;
      } else {
        arow[mi] = lds + m * ldc + 16 * f;
        srow[mi] = m * a.Kb;
      }
    }

    struct Step {
      v8i W[NB];
      v8i X[MT];
      float sx[MT], sw, su;
    };
    auto fetch_rows = [&](Step& s, int kb) __attribute__((always_inline)) {
#pragma unroll
      for (int mi = 0; mi < MT; ++mi) {
        const v4i* p = reinterpret_cast<const v4i*>(arow[mi] + (size_t)kb * 128);
        s.X[mi] = __builtin_shufflevector(p[0], p[4], 0, 1, 2, 3, 4, 5, 6, 7);
        s.sx[mi] = IN == kCodes ? a.SA[(int64_t)kb * a.ld_sa + srow[mi]] : lds_scale[srow[mi] + kb];
      }
    };
    auto fetch = [&](Step& s, int kb) __attribute__((always_inline)) {
      const uint8_t* w = w0 + (size_t)kb * kF8GroupBytes;
#pragma unroll
      for (int b = 0; b < NB; ++b)
        s.W[b] = __builtin_shufflevector(*reinterpret_cast<const v4i*>(w + b * 2048), *reinterpret_cast<const v4i*>(w + b * 2048 + 1024), 0, 1, 2, 3, 4, 5, 6, 7);
      if constexpr (IN == kCodes) fetch_rows(s, kb);
      s.sw = sw0[kb];
      s.su = GATED ? sw0[(size_t)a.nblk * a.Kb + kb] : 0.0f;
    };
    auto multiply = [&](Step& s, int kb) __attribute__((always_inline)) {
      if constexpr (IN != kCodes) fetch_rows(s, kb);
      b8 X[MT][4];
#pragma unroll
      for (int mi = 0; mi < MT; ++mi)
#pragma unroll
        for (int k = 0; k < 4; ++k) X[mi][k] = widen8(s.X[mi][2 * k], s.X[mi][2 * k + 1]);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        f4 p[MT];
#pragma unroll
        for (int mi = 0; mi < MT; ++mi) p[mi] = f4{0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const b8 w = widen8(s.W[b][2 * k], s.W[b][2 * k + 1]);
#pragma unroll
          for (int mi = 0; mi < MT; ++mi) p[mi] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, X[mi][k], p[mi], 0, 0, 0);
        }
#pragma unroll
        for (int mi = 0; mi < MT; ++mi) {
          const float fs = s.sx[mi] * (GATED && ((b0 + b) & 1) ? s.su : s.sw);
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[mi][b][r] = __builtin_fmaf(p[mi][r], fs, acc[mi][b][r]);
        }
      }
    };
    if constexpr (MT == 1) {
      Step s[U];
      if constexpr (IN != kCodes) {
        // a unit: 16 channels of a row, 8 lanes a block
        const int units = nr * a.Kb * 8, per = a.Kb * 8;
        auto row_of = [&](int u) __attribute__((always_inline)) {
          const int r = r0 + u / per;
          const int ar = GATED ? min(max(a.index[r], 0), a.a_rows - 1) : r;
          return static_cast<const char*>(a.X) + (int64_t)ar * a.ld_x * (IN == kBf16 ? 2 : 4);
        };
        auto make = [&](int u, const Raw16<IN == kBf16>& x) __attribute__((always_inline)) {
          float scale, inv;
          scale_of(max8(x.amax()), a.pow2, &scale, &inv);
          const int m = u / per, c = (u - m * per) * 16;
          *reinterpret_cast<u4*>(lds + m * ldc + c) = x.codes(inv);
          if ((t & 7) == 0) lds_scale[m * a.Kb + (c >> 7)] = scale;
        };
        Raw16<IN == kBf16> x0, x1;
        const bool two = t + kWaves * 64 < units;
        if (t < units) x0.load(row_of(t), t % per * 16, a.d);
        if (two) x1.load(row_of(t + kWaves * 64), (t + kWaves * 64) % per * 16, a.d);
        if (kb0 < kb1) {
#pragma unroll
          for (int u = 0; u < U; ++u) fetch(s[u], min(kb0 + u, kb1 - 1));
        }
        __syncthreads();  // the partial sums of the rows before have been read
        if (t < units) make(t, x0);
        if (two) make(t + kWaves * 64, x1);
        for (int u = t + 2 * kWaves * 64; u < units; u += kWaves * 64) {
          x0.load(row_of(u), u % per * 16, a.d);
          make(u, x0);
        }
        __syncthreads();
      }
      for (int kb = kb0; kb < kb1; kb += U) {
        if (IN == kCodes || kb > kb0) {
#pragma unroll
          for (int u = 0; u < U; ++u) fetch(s[u], min(kb + u, kb1 - 1));
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (kb + u < kb1) multiply(s[u], kb + u);
      }
    } else if (kb0 < kb1) {
      Step s, n;
      fetch(s, kb0);
      for (int kb = kb0; kb < kb1; ++kb) {
        fetch(n, min(kb + 1, kb1 - 1));
        multiply(s, kb);
        s = n;
      }
    }
    // partial sums: element r of block b is row 4 f + r of the instruction, token lane % 16
    __syncthreads();
#pragma unroll
    for (int mi = 0; mi < MT; ++mi)
#pragma unroll
      for (int b = 0; b < NB; ++b) *reinterpret_cast<f4*>(&red[part][16 * mi + (lane & 15)][(side * NB + b) * 16 + 4 * f]) = acc[mi][b];
    __syncthreads();
    if constexpr (!GATED) {
      for (int u = t; u < nr * kPlaces; u += kWaves * 64) {
        const int m = u / kPlaces, pl = u % kPlaces;
        const int blk = blockIdx.x * (kSide * NB) + (pl >> 4);
        const int n = f8_column(0, blk >> 2, blk & 3, pl & 15);
        if (n >= a.N) continue;
        float v = red[0][m][pl];
#pragma unroll
        for (int s = 1; s < S; ++s) v += red[s][m][pl];
        if (a.bias != nullptr) v += a.bias[(size_t)set * a.N + n];
        const int64_t o = (int64_t)(r0 + m) * a.ld_y + n;
        if (a.y_bf16) static_cast<uint16_t*>(a.Y)[o] = to_bf16(v);
        else static_cast<float*>(a.Y)[o] = v;
      }
    } else {
      // 256 places are a block of 128 columns: 8 lanes of 16 columns each take a row
      static_assert(kPlaces == 256, "a block of the next layer's input in one workgroup");
      for (int u = t; u < kRows * 8; u += kWaves * 64) {
        const int m = u >> 3, c0 = (u & 7) * 16;
        float hv[16];
        uint32_t amax = 0;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int c = c0 + j, ch = blockIdx.x * 128 + c;  // of group c / 32: lanes c / 8 % 4, pair c / 4 % 2
          const int pl = (c >> 5) * 64 + ((c >> 2) & 1) * 32 + ((c >> 3) & 3) * 4 + (c & 3);
          float gt = red[0][m][pl], up = red[0][m][pl + 16];
#pragma unroll
          for (int s = 1; s < S; ++s) gt += red[s][m][pl], up += red[s][m][pl + 16];
          hv[j] = ch < a.N ? silu(gt) * up : 0.0f;
          amax = max(amax, abs_bits(hv[j]));
        }
        amax = max8(amax);
        float scale, inv;
        scale_of(amax, a.pow2, &scale, &inv);
        u4 o;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = pack4(hv[4 * j] * inv, hv[4 * j + 1] * inv, hv[4 * j + 2] * inv, hv[4 * j + 3] * inv);
        if (m < nr) {
          *reinterpret_cast<u4*>(static_cast<uint8_t*>(a.Y) + (int64_t)(r0 + m) * a.ld_y + blockIdx.x * 128 + c0) = o;
          if ((u & 7) == 0) a.SH[(int64_t)blockIdx.x * a.ld_sh + r0 + m] = scale;
        }
      }
    }
  }
}

int row_bytes(int Kb) { return Kb * 128 + 16 + Kb * 4; }  // of a row quantized here
constexpr int kCodesLds = 68 << 10;                       // 16 rows of 4096 channels, two workgroups a CU

template <int MT, int NB, int S, int WV, bool GATED, Rows IN>
hipError_t go(const StampF8Gemm& a, hipStream_t st) {
  const int places = WV / S * NB * 16, sums = S * 16 * MT * (places + 4) * 4, codes = IN == kCodes ? 0 : a.chunk * row_bytes(a.Kb);
  const int lds = codes > sums ? codes : sums;
  static size_t done[kStampMaxDevices];
  const hipError_t e = stamp_allow_lds(reinterpret_cast<const void*>(&k_f8_rows<MT, NB, S, WV, GATED, IN>), (size_t)lds, done);
  if (e != hipSuccess) return e;
  k_f8_rows<MT, NB, S, WV, GATED, IN><<<dim3((a.groups * 64 + places - 1) / places, a.sets), WV * 64, lds, st>>>(a);
  return hipGetLastError();
}
template <Rows IN>
hipError_t quantizing(const StampF8Gemm& a, int nb, hipStream_t st) {
  if (a.gated) return go<1, 2, 2, 16, true, IN>(a, st);
  return nb >= 2 ? go<1, 2, 8, 8, false, IN>(a, st) : go<1, 1, 8, 8, false, IN>(a, st);
}
int average(const StampF8Gemm& a, int rows) { return (int)(((int64_t)rows + a.sets - 1) / a.sets); }
}  // namespace

// Where all workgroups run at once and the rows are few: 1 x 4096 -> 11008 9.9 us, with a launch for the codes 12.1; with more workgroups
// than that the registers of the quantizer cost more than the launch (1 x 8192 -> 28672: 49 us and 38.5; 96 rows over 24 of 32 experts,
// 4096 -> 1536: 29.9 and 29.8; 24 rows over 24 experts, gated 2048 -> 1408: 33 and 29).
int stamp_f8_rows_quantize(const StampF8Gemm& a, int rows) {
  const int fit = kCodesLds / row_bytes(a.Kb), busy = a.sets < rows ? a.sets : rows;
  const int chunk = fit > 16 ? 16 : fit;  // 65536 channels: one row
  const int64_t workgroups = (int64_t)busy * (a.gated ? (a.groups + 3) / 4 : a.groups);  // gated: one a CU; else two, of half a group at least
  return workgroups <= stamp_device_cus() && average(a, rows) <= (chunk < 4 ? chunk : 4) ? chunk : 0;
}

hipError_t stamp_launch_f8_rows(const StampF8Gemm& a, hipStream_t st) {
  const int avg = average(a, a.rows), busy = a.sets < a.rows ? a.sets : a.rows;
  // blocks per wave: as many as leave a workgroup for every CU; fewer workgroups read (and quantize) the rows less often.  Four do not fit
  // the registers beside the quantizer's.
  const int64_t groups = (int64_t)a.groups * busy;
  const int cus = stamp_device_cus();
  const int nb = groups >= cus ? 4 : 2 * groups >= cus ? 2 : 1;
  if (a.X != nullptr) return a.x_bf16 ? quantizing<kBf16>(a, nb, st) : quantizing<kF32>(a, nb, st);
  if (a.gated) return avg <= 16 ? go<1, 4, 2, 8, true, kCodes>(a, st) : go<2, 4, 2, 8, true, kCodes>(a, st);
  if (avg <= 16)
    return nb == 4 ? go<1, 4, 8, 8, false, kCodes>(a, st) : nb == 2 ? go<1, 2, 8, 8, false, kCodes>(a, st) : go<1, 1, 8, 8, false, kCodes>(a, st);
  if (avg <= 32)
    return nb == 4 ? go<2, 4, 8, 8, false, kCodes>(a, st) : nb == 2 ? go<2, 2, 8, 8, false, kCodes>(a, st) : go<2, 1, 8, 8, false, kCodes>(a, st);
  return nb >= 2 ? go<4, 2, 8, 8, false, kCodes>(a, st) : go<4, 1, 8, 8, false, kCodes>(a, st);
}
