// 8-bit floating point layers with block scales: plan, layouts and launchers (gfx950).
//
// Places: a plan's output columns are dealt to groups of 64, so that after the matrix instructions a lane holds neighbouring columns of
// one row.  The weights are the first operand of v_mfma_f32_16x16x128_f8f6f4, a block of 128 input channels in one instruction: lane
// 16 f + i gives row i of it, and element r of lane 16 f + m of the result is row 4 f + r of column m.  With the tokens as columns a lane
// has one token, whose scale it then needs once, and rows 4 f .. 4 f + 3 of every instruction b = 0 .. 3 of a group:
//   plain  column 64 g + 32 (b / 2) + 8 f + 4 (b % 2) + r: twice 8 neighbours; the 4 lanes of a row have 32, stored at once
//   gated  column 32 g + 8 f + 4 (b / 2) + r of the gate (b even) or the up matrix (b odd): 8 neighbours of both; four groups are a block
//          of 128 of the next layer's input
//
// Operand image of the weights, [matrix set e][group][block of 128 channels][b][h][lane][16 bytes]: lane 16 f + i's parts h = 0, 1 are
// channels 64 h + 16 f .. + 15 of row i (any dealing of the channels is right that is the same for both operands).  A wave reads 1 KB of
// consecutive addresses, from memory or LDS.  Activations stay in rows: [row][Kp] bytes (or bf16).
#ifndef STAMP_FP8_H_
#define STAMP_FP8_H_

#include "stamp_internal.h"

constexpr int kF8Block = 128;
constexpr int kF8Group = 64;                        // places of a group
constexpr int kF8GroupBytes = kF8Group * kF8Block;  // of a group and block of channels
constexpr int kF8MaxExperts = 1024;
constexpr int kF8DividedSilu = 16;  // beside stamp_activation_t, for gated products

struct stamp_fp8_plan {
  stamp_fp8_desc_t desc;
  int32_t sets;        // experts, or 1
  int32_t Kb, Kp;      // blocks of the input channels, bytes of a row of codes
  int32_t groups;      // of a set
  int32_t nblk;        // blocks of 128 output columns of one matrix
  int32_t forced;      // stamp_fp8_debug_set_route
  int32_t looks;       // stamp_moe_debug_set_looks
  uint8_t* w_dev;      // operand image
  float* sw_dev;       // [sets][2 if gated][nblk][Kb]
  float* bias_dev;     // [sets][d_out] or nullptr
};

// column of place (b, row i of the instruction) in group g; gated: of the gate matrix for even b
STAMP_HD int f8_column(int gated, int g, int b, int i) {
  return gated ? 32 * g + 8 * (i >> 2) + 4 * (b >> 1) + (i & 3) : 64 * g + 32 * (b >> 1) + 8 * (i >> 2) + 4 * (b & 1) + (i & 3);
}
STAMP_HD size_t f8_w_offset(int groups, int Kb, int set, int g, int kb, int b, int h, int lane) {
  return ((((size_t)set * groups + g) * Kb + kb) * 8 + b * 2 + h) * 1024 + (size_t)lane * 16;
}

// The product's arguments.
struct StampF8Gemm {
  const uint8_t* A;        // codes [a_rows][Kp], for tiles of wide_sums as bf16
  const float* SA;         // scales [Kb][ld_sa], by row of A
  int64_t ld_sa;
  const int32_t* index;    // gated: row of A of every row of the product, nullptr: the same (and so it is where not gated)
  int32_t a_rows;
  const void* X;           // not nullptr: A's rows before Q8, quantized by the product itself (few rows)
  int64_t ld_x;
  int32_t x_bf16, d;       // channels
  int32_t chunk;           // rows quantized at a time
  int32_t rows;
  const int32_t* offsets;  // [sets + 1] or nullptr (one set)
  const uint8_t* W;
  const float* SW;
  const float* bias;
  int32_t sets, groups, Kb, nblk, N, pow2, gated, y_bf16;
  int32_t forced;          // stamp_fp8_route_t, 0: by rule
  int32_t wide_sums;       // products on the bf16 matrix instructions (f8_wide_sums)
  void* Y;                 // rows of N values; gated, codes: codes [rows][ld_y] and scales [ld_y / 128][ld_sh]
  int64_t ld_y;
  int32_t codes;           // not gated: Y as codes (in tiles alone)
  int32_t h_wide;          // codes of Y as bf16
  int32_t h_rows;          // gated, few rows: Y as rows of N values in fp32 instead of codes
  int32_t act;             // stamp_activation_t, of the gate where gated (or kF8DividedSilu)
  const void* R;           // residual rows in Y's type, or nullptr
  int64_t ld_r;
  float* SH;
  int64_t ld_sh;
  float* partial;          // [parts][rows][groups * 64] where the depth is split
  uint32_t first;          // workgroups of the launches before this one (tiles)
};

inline bool f8_has_epilogue(const StampF8Gemm& a) { return !a.gated && (a.act != STAMP_ACT_NONE || a.R != nullptr); }

// A launch of 2^32 threads or more is refused: units beyond that many workgroups are taken by further launches.
constexpr int64_t kF8MaxThreads = (int64_t)1 << 31;
template <typename F>
hipError_t f8_launches(int64_t workgroups, int threads, F launch) {
  const int64_t most = kF8MaxThreads / threads;
  for (int64_t first = 0; first < workgroups; first += most) {
    launch(first, (uint32_t)(workgroups - first < most ? workgroups - first : most));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// stamp_fp8_route_t of a product of `rows` rows over `sets` weights
int stamp_f8_route(int sets, int groups, int Kb, int rows, int wide_sums, int gated, int forced);
// its tiles: 64 << size rows and the parts of the depth, of the first `groups` groups (0: of all), and of the rest
struct F8Cut {
  int groups, size, parts, rest_size, rest_parts;
};
F8Cut stamp_f8_cut(int sets, int groups, int Kb, int rows, int wide_sums, int gated, int forced);
// an up product's rows as codes, straight from tiles (quantized_below: the down product would quantize fp32 rows itself)
int stamp_f8_codes_pay(int groups, int Kb, int rows, int quantized_below);
int stamp_f8_codes_route(int groups, int Kb, int rows);
constexpr int kF8MaxParts = 8;
// bytes of the parts' rows, at most
size_t stamp_f8_partial_bytes(int groups, int rows);
hipError_t stamp_launch_f8_weights(stamp_fp8_plan* p, const void* W, const float* w_scales, hipStream_t st, uint32_t* flag);
// wide: the codes as bf16
hipError_t stamp_launch_f8_widen(const uint8_t* codes, int64_t bytes, uint8_t* out, hipStream_t st);
hipError_t stamp_launch_f8_quant(const void* X, int x_bf16, int64_t ld_x, int rows, int d, int pow2, int wide, uint8_t* codes, float* scales, int64_t ld_s,
                                 hipStream_t st);
int stamp_f8_rows_quantize(const StampF8Gemm& a, int rows);  // rows that the kernel for few rows quantizes at a time, 0: it takes codes
hipError_t stamp_launch_f8_rows(const StampF8Gemm& a, hipStream_t st);
hipError_t stamp_launch_f8_tiles(const StampF8Gemm& a, int bm, int parts, hipStream_t st);

// The FP8 matrix instructions align the 8 products of neighbouring channels to the largest of them and drop what lies 14 bits and more
// below it (2^16 + 2^3 comes out, 2^16 + 2^2 does not): a product of random codes is 1e-5 to 6e-5 of its size off, while the bf16
// instructions, which the codes fit exactly, keep 4e-8 at half the rate.  A bf16 Y cannot tell (its own rounding is 2e-3), so its layers
// take the FP8 instructions.  An fp32 Y and the codes of the next layer (an error of 6e-5 moves one in 1000 of them to its neighbour) take
// the bf16 instructions.
inline int f8_wide_sums(const StampF8Gemm& a) { return a.gated || a.codes || !a.y_bf16; }
hipError_t stamp_launch_route(const stamp_routing_t& r, const void* logits, int bf16, int64_t ld, int renorm, void* ws, hipStream_t st);
size_t stamp_route_ws(int tokens, int experts, int top_k);
hipError_t stamp_launch_combine(const stamp_routing_t& r, const void* rows, int rows_bf16, int y_bf16, int64_t ld_rows, int nrows, const void* R, int64_t ld_r,
                                void* Y, int64_t ld_y, int d, hipStream_t st);

// logits [tokens][experts] = X W^T + bias; in the same launch Q8 of X (codes nullptr: not wanted; wide: as bf16) and zeros to `zeros` words
struct RouterQ8 {
  uint8_t* codes;
  float* scales;
  int64_t ld_s;
  int32_t pow2, wide;
  uint32_t* zero;
  int32_t zeros;
};
hipError_t stamp_launch_router(const stamp_router_t& router, const void* X, int x_bf16, int64_t ld_x, int tokens, int experts, int d, const RouterQ8& q,
                               float* logits, hipStream_t st);

// The whole layer in two kernels for few tokens and few rows, as long as a token's h for every token fits the LDS beside each other; else the kernels of the
// other calls one after the other.  us, two kernels / the others (weights not in the cache):
//                               1 token     2           4            8            16
//   6 of 64,  2048 -> 1408        29 / 37     39 / 49     50 / 59      73 / 79      99 / 106
//   8 of 256, 4096 -> 1536        49 / 59     69 / 107    119 / 152    202 / 227    336 / 358
//   2 of 16,  1024 -> 512         14 / 25     16 / 26     17 / 26      22 / 28      25 / 29
//   2 of 8,   4096 -> 2048        30 / 50     35 / 54     52 / 61      57 / 66      64 / 70
//   16 of 64, 2048 -> 1408        48 / 62     66 / 74     82 / 91      113 / 119    142 / 126
//   32 of 128, 1024 -> 512        40 / 48     48 / 64     56 / 60      67 / 67      80 / 71
//   6 of 64,  6144 -> 1536        55 / 76     77 / 95     120 / 137    194 / 214    260 / 274
//   4 of 128, 7168 -> 2048        53 / 87     84 / 112    140 / 181    231 / 250    404 / 413
//   8 of 256, 7168 -> 2048        82 / 114    140 / 197   249 / 275    453 / 463    765 / 769
//   2 of 8,   6144 -> 4096        44 / 69     71 / 84     95 / 107     117 / 138    132 / 153
//   2 of 16,  8192 -> 2048        45 / 74     54 / 87     85 / 105     123 / 145    150 / 171
// Beyond 128 rows Q8 of h, which every workgroup does again for its part of the rows, is what loses.
constexpr int kMoeTokens = 16, kMoeSlots = 128;
constexpr int kMoeChunkBytes = 96 << 10;
// workgroups that share 64 columns of Y, at most: as many as fit the CUs
inline int stamp_moe_parts(int groups) {
  const int fit = stamp_device_cus() / groups;
  return fit < 1 ? 1 : fit > 16 ? 16 : fit;
}
inline size_t stamp_moe_sync_bytes(int groups) { return (size_t)(1 + kMoeSlots + groups) * 4; }
inline bool stamp_moe_fits(int tokens, int top_k, int Kb_down) {
  return tokens <= kMoeTokens && tokens * top_k <= kMoeSlots && (int64_t)tokens * (Kb_down * 132 + 16) <= kMoeChunkBytes;
}
// up: act, Y for h in fp32 (ld_y whole blocks); down: R, Y.  sync: stamp_moe_sync_bytes of any content; sums: parts * tokens * groups * 64.  looks: of a wait, -1: as many as ever needed.
hipError_t stamp_launch_moe(const stamp_router_t& router, const stamp_routing_t& r, const void* X, int x_bf16, int64_t ld_x, const StampF8Gemm& up,
                            const StampF8Gemm& down, uint8_t* codes, float* scales, float* logits, uint32_t* sync, float* sums,
                            int32_t looks, hipStream_t st);

// ---- device helpers ----
#ifdef __HIPCC__
namespace f8 {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
// in rows of any stride and alignment: loads and stores of 8 and 16 bytes need none
typedef f4 f4_any __attribute__((aligned(4)));
typedef u4 u4_any __attribute__((aligned(2)));
typedef u2 u2_any __attribute__((aligned(2)));

constexpr uint32_t kSmallest = (127u - 118u) << 23 | 0x600000u;  // 1.75 * 2^-118
constexpr uint32_t kInfBits = 0x7f800000u;

// Scale and multiplier of a block from the bits of its largest magnitude: as bits, magnitudes compare as integers, and infinities and NaN
// are above all numbers.
__device__ __forceinline__ void scale_of(uint32_t amax, int pow2, float* scale, float* inv) {
  const uint32_t a = amax > kSmallest ? amax : kSmallest;
  if (a >= kInfBits) {
    *scale = *inv = __uint_as_float(0x7fc00000u);
  } else if (pow2) {
    const uint32_t e = (a >> 23) - 8 + ((a & 0x7fffffu) > 0x600000u ? 1 : 0);  // 448 = 1.75 * 2^8
    *scale = __uint_as_float(e << 23);
    *inv = __uint_as_float((254 - e) << 23);
  } else {
    *scale = __fdiv_rn(__uint_as_float(a), 448.0f);
    *inv = __fdiv_rn(448.0f, __uint_as_float(a));
  }
}
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
}
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xf, 0xf, false);
  return v > o ? v : o;
}
// largest of 8 neighbouring lanes, in all of them: pairs, quads, the mirrored half row
__device__ __forceinline__ uint32_t max8(uint32_t v) { return dpp_max<0x141>(dpp_max<0x4e>(dpp_max<0xb1>(v))); }

__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }
__device__ __forceinline__ float bf16_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
__device__ __forceinline__ uint16_t to_bf16(float x) {
  const __bf16 b = (__bf16)x;
  return __builtin_bit_cast(uint16_t, b);
}
__device__ __forceinline__ uint32_t to_bf16x2(float x, float y) {
  typedef __bf16 bb __attribute__((ext_vector_type(2)));
  const bb v = {(__bf16)x, (__bf16)y};
  return __builtin_bit_cast(uint32_t, v);
}

// Rows of set e, cut to 0 .. rows.
__device__ __forceinline__ void rows_of(const StampF8Gemm& a, int e, int* lo, int* hi) {
  if (a.offsets == nullptr) {
    *lo = 0;
    *hi = a.rows;
    return;
  }
  const int l = min(max(a.offsets[e], 0), a.rows);
  *lo = l;
  *hi = min(max(a.offsets[e + 1], l), a.rows);
}

// Tiles of BM rows, counted over the sets.  Every wave counts by itself.
__device__ __forceinline__ int tiles_of(const StampF8Gemm& a, int e, int BM, int* lo, int* hi) {
  *lo = *hi = 0;
  if (e < a.sets) rows_of(a, e, lo, hi);
  return (*hi - *lo + BM - 1) / BM;
}
__device__ __forceinline__ int wave_scan(int v) {  // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}
// The sets 0 .. 63 stay in the lanes: their rows and the tiles up to and including theirs.
struct Tiles {
  int lo, hi, incl, total;
};
__device__ __forceinline__ Tiles count_tiles(const StampF8Gemm& a, int BM) {
  Tiles t;
  t.lo = t.hi = t.incl = 0;
  t.total = (a.rows + BM - 1) / BM;
  if (a.offsets == nullptr) return t;
  t.incl = wave_scan(tiles_of(a, threadIdx.x & 63, BM, &t.lo, &t.hi));
  int n = __shfl(t.incl, 63), more = 0, lo, hi;
  if (a.sets > 64) {
    for (int e = 64 + (threadIdx.x & 63); e < a.sets; e += 64) more += tiles_of(a, e, BM, &lo, &hi);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) more += __shfl_xor(more, d);
  }
  t.total = __builtin_amdgcn_readfirstlane(n + more);
  return t;
}
// set and rows of a tile below total
__device__ __forceinline__ void find_tile(const StampF8Gemm& a, const Tiles& t, int BM, int tile, int* set, int* row0, int* nrows) {
  *set = 0;
  *row0 = tile * BM;
  *nrows = min(BM, a.rows - *row0);
  if (a.offsets == nullptr) return;
  int base = 0;
  for (int e0 = 0; e0 < a.sets; e0 += 64) {
    int lo = t.lo, hi = t.hi, incl = t.incl;
    if (e0 > 0) incl = wave_scan(tiles_of(a, e0 + (threadIdx.x & 63), BM, &lo, &hi));
    const uint64_t past = __ballot(base + incl > tile);
    if (past != 0) {
      const int src = __builtin_ctzll(past), first = base + __shfl(incl, src) - (__shfl(hi, src) - __shfl(lo, src) + BM - 1) / BM;
      const int l = __shfl(lo, src), h = __shfl(hi, src);
      *set = __builtin_amdgcn_readfirstlane(e0 + src);
      *row0 = __builtin_amdgcn_readfirstlane(l + (tile - first) * BM);
      *nrows = __builtin_amdgcn_readfirstlane(min(BM, h - *row0));
      return;
    }
    base += __shfl(incl, 63);
  }
}

// 16 channels of a row from c on as they are stored, zeros from d on
template <bool BF16>
struct Raw16 {
  u4 w[BF16 ? 2 : 4];
  __device__ __forceinline__ void load(const void* row, int c, int d) {
    if (c + 16 <= d) {
      const u4_any* s = reinterpret_cast<const u4_any*>(static_cast<const char*>(row) + (size_t)c * (BF16 ? 2 : 4));
#pragma unroll
      for (int q = 0; q < (BF16 ? 2 : 4); ++q) w[q] = s[q];
      return;
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      if constexpr (BF16) {
        const uint32_t x = c + j < d ? static_cast<const uint16_t*>(row)[c + j] : 0u;
        if (j & 1) w[j >> 3][(j >> 1) & 3] |= x << 16;
        else w[j >> 3][(j >> 1) & 3] = x;
      } else {
        w[j >> 2][j & 3] = c + j < d ? static_cast<const uint32_t*>(row)[c + j] : 0u;
      }
    }
  }
  __device__ __forceinline__ float at(int j) const {
    if constexpr (BF16) return (j & 1) ? bf16_hi(w[j >> 3][(j >> 1) & 3]) : bf16_lo(w[j >> 3][(j >> 1) & 3]);
    else return __uint_as_float(w[j >> 2][j & 3]);
  }
  __device__ __forceinline__ uint32_t amax() const {
    uint32_t a = 0;
#pragma unroll
    for (int j = 0; j < 16; ++j) a = max(a, abs_bits(at(j)));
    return a;
  }
  __device__ __forceinline__ u4 codes(float inv) const {
    u4 o;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      o[j] = pack4(__fmul_rn(at(4 * j), inv), __fmul_rn(at(4 * j + 1), inv), __fmul_rn(at(4 * j + 2), inv), __fmul_rn(at(4 * j + 3), inv));
    return o;
  }
};

// Residual of 8 columns of a row, p + column: as they are stored, zeros from `left` columns on.
template <bool BF16>
struct Residual8 {
  u4 w[BF16 ? 1 : 2];
  __device__ __forceinline__ void load(const char* p, int left) {
#pragma unroll
    for (int q = 0; q < (BF16 ? 1 : 2); ++q) w[q] = u4{0, 0, 0, 0};
    if (left >= 8) {
#pragma unroll
      for (int q = 0; q < (BF16 ? 1 : 2); ++q) w[q] = reinterpret_cast<const u4_any*>(p)[q];
      return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (j >= left) continue;
      if constexpr (BF16) w[0][j >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[j] << (16 * (j & 1));
      else w[j >> 2][j & 3] = reinterpret_cast<const uint32_t*>(p)[j];
    }
  }
  __device__ __forceinline__ float at(int j) const {
    if constexpr (BF16) return (j & 1) ? bf16_hi(w[0][j >> 1]) : bf16_lo(w[0][j >> 1]);
    else return __uint_as_float(w[j >> 2][j & 3]);
  }
};

typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
// 8 codes as bf16: exact
__device__ __forceinline__ b8 widen8(int lo, int hi) {
  const b2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
  const b2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  return b8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// 8 codes at element o of a row's codes, as bytes or as bf16
__device__ __forceinline__ void put_codes(void* base, int64_t o, const u2& c, int wide) {
  if (wide) reinterpret_cast<b8*>(base)[o >> 3] = widen8((int)c[0], (int)c[1]);
  else reinterpret_cast<u2*>(base)[o >> 3] = c;
}

__device__ __forceinline__ float silu(float g) { return g / (1.0f + __expf(-g)); }

// x / (1 + exp(-y)) by the reciprocal instruction, one rounding more than a division
__device__ __forceinline__ float logistic_times(float x, float y) {
  return x * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(y * -1.44269504088896341f));
}
// x Phi(x) as max(x, 0) - |x| Q(|x|), Q(t) = 1 - Phi(t) = exp(-t^2 / 2) r(t): r falls slowly (as 1 / t) and is a polynomial of degree 7 in 1 / (1 + t / 4), fitted for t up to 10 by
// least squares of its relative error with weights raised where that is largest (1.6e-7; beyond 10 gelu is below 1e-22).  So the tail keeps its own digits: 6e-7 of the value down to x = -3, 2e-6
// to -6 (0.5 x (1 + erf) has none left below -5.5), and 2.7e-7 of |x| at most.  An fp32 Y shows them, and so do codes of h: with x normal, deviation 3, 13 of 5.2 million values came to a code
// beside their own, 464 by the shorter form below, 318 by erf in fp32.  It takes 18 instructions: an MLP of 8192 x 1152 -> 4608 -> 1152 167 us, with the shorter form 163.5.
__device__ __forceinline__ float gelu(float x) {
  const float t = __builtin_fabsf(__builtin_fminf(x, 20.0f));  // infinity times Q's zero would be NaN; minus infinity's is meant to be
  const float u = __builtin_amdgcn_rcpf(__builtin_fmaf(0.25f, t, 1.0f));
  float r = -0.09756410121917725f;
  r = __builtin_fmaf(r, u, 0.37102118134498596f);
  r = __builtin_fmaf(r, u, -0.32742080092430115f);
  r = __builtin_fmaf(r, u, 0.3479419946670532f);
  r = __builtin_fmaf(r, u, -0.017856374382972717f);
  r = __builtin_fmaf(r, u, 0.12785829603672028f);
  r = __builtin_fmaf(r, u, 0.09578244388103485f);
  r = __builtin_fmaf(r, u, 0.0002374343603150919f);
  const float q = r * __builtin_amdgcn_exp2f(t * t * -0.72134752044448170f);
  return __builtin_fmaf(-t, q, x < 0.0f ? 0.0f : x);
}
// The same for rows of a bf16 Y in tiles, whose end the matrix pipe waits for: x / (1 + 2^y), y = x p(x^2): log2 of (1 - Phi) / Phi is odd in x, and its quotient by x a polynomial of
// degree 7 in x^2, fitted for |x| up to sqrt(30) by least squares with weights raised where Phi's error is largest, and held beyond.  2.0e-7 of |x| at most, measured over -100 .. 100, a
// step of bf16 of the value itself down to x = -5 (3.3e-4; 2^-8 is 3.9e-3); 6 % off at -5.5, where gelu is 1e-7, four times it at -6, zero beyond.  14 instructions, two of them of a
// quarter rate: 8192 x 1152 -> 4608, bf16: 68 us without, 75 with gelu_tanh, 80 so, 85 with the form above.
__device__ __forceinline__ float gelu_bf16(float x) {
  const float s = __builtin_fminf(x * x, 30.0f);
  float p = 7.60429497148607e-11f;
  p = __builtin_fmaf(p, s, -9.219624175216268e-09f);
  p = __builtin_fmaf(p, s, 4.6102681494630815e-07f);
  p = __builtin_fmaf(p, s, -1.2103833796572872e-05f);
  p = __builtin_fmaf(p, s, 0.0001620831899344921f);
  p = __builtin_fmaf(p, s, 9.015658724820241e-05f);
  p = __builtin_fmaf(p, s, -0.10483329743146896f);
  p = __builtin_fmaf(p, s, -2.3022093772888184f);
  return x * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * p));
}
__device__ __forceinline__ float gelu_tanh(float x) {
  const float c = 1.59576912160573071f;  // 2 sqrt(2 / pi)
  return logistic_times(x, x * __builtin_fmaf(x * x, c * 0.044715f, c));
}
__device__ __forceinline__ float relu(float x) { return x < 0.0f ? 0.0f : x; }
// one choice for N values: act is the same in all lanes.  BF16: the results are rounded to bf16
template <int N, bool BF16 = false>
__device__ __forceinline__ void activate(float (&v)[N], int act) {
  if (act == STAMP_ACT_RELU) {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = relu(v[j]);
  } else if (act == STAMP_ACT_SILU) {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = logistic_times(v[j], v[j]);
  } else if (act == STAMP_ACT_GELU) {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = BF16 ? gelu_bf16(v[j]) : gelu(v[j]);
  } else if (act == STAMP_ACT_GELU_TANH) {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = gelu_tanh(v[j]);
  }
}
// act(g) u; kF8DividedSilu: silu by a division, as stamp_experts_forward has had it (8192 x 4096 -> 11008, gated: 1260 us of tiles by the reciprocal, 1294 so)
template <int N>
__device__ __forceinline__ void gate(float (&g)[N], const float (&u)[N], int act) {
  if (act == kF8DividedSilu) {
#pragma unroll
    for (int j = 0; j < N; ++j) g[j] = silu(g[j]);
  } else {
    activate(g, act);
  }
#pragma unroll
  for (int j = 0; j < N; ++j) g[j] *= u[j];
}

}  // namespace f8
#endif
#endif  // STAMP_FP8_H_
