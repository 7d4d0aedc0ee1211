// The layer of experts for few tokens in two kernels: what is left of the time beside the chosen experts' weights is launches and waits.
//
// First kernel (k_router): logits, codes of X, and zeros in the counters of the second.  Second kernel: every workgroup chooses the experts from the logits by
// itself (2 to 4 us; a launch of its own would take as long, and its results as long again to arrive), then takes products of 32 columns of h of an expert from a
// counter until none is left, then has 64 columns of Y for a part of the experts.
//
// The down product reads all columns of h, so it waits for its experts' rows, each counted by those who finish a piece of it, and not before its first weights
// are on their way.  The wait ends: up products are taken in order by workgroups that run already, so whoever waits, waits for products that are being worked on, and
// those wait for nobody.  That holds for any number of workgroups on the chip, other kernels' among them.  (Two calls that use one workspace at once, against the rules, may
// take a counter back under a waiter: so it gives up after some seconds, and what it would have added to Y becomes NaN.)
//
// h passes between workgroups in fp32: whoever reads it makes Q8 of it (few rows; a block of 128 columns would be four workgroups' otherwise).  Y's sum over a token's
// experts stays in the accumulators: a column of the down product's matrix instruction is a token (one that has not chosen the expert takes nothing from it), and its
// factor carries the router's weight.  So there are no rows to be written; the parts of a column are added up by the last of its workgroups, in the parts' order, and
// nothing depends on the order of workgroups.
//
// Bound by the weights' bytes where they are many: 16 tokens, 8 of 256 experts, 4096 -> 1536: 312 us, 6.1 TB/s (up products 5.8).  Else by the chain of steps: 1 token, 6 of
// 64, 2048 -> 1408 (52 MB) 24 us: chosen after 4.5, up products 7 more and, as 264 of them are one round of the CUs and 8 more, 6 for those; down product and sum of the
// parts 7.  What a CU gets from memory is what counts (20 to 30 KB a us): runs of 8 KB of a weight matrix, one after the other, with the next ones on their way; in pieces of
// 2 or 4 KB of every 8 the same bytes take 1.3 times as long.
#include "stamp_route.h"

namespace {
using namespace f8;

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * 64;
constexpr int kMaxSlots = kMoeSlots;
constexpr int kMaxLooks = 1 << 22;     // at a counter behind the first, some 0.7 us each: more than all weights that the memory holds take
constexpr int kUpLd = kF8Group + 4;    // floats of a row of an up product's partial sums
constexpr int kRoom = kWaves * 16 * kUpLd * 4 > kMoeChunkBytes ? kWaves * 16 * kUpLd * 4 : kMoeChunkBytes;

struct MoeArgs {
  const float* logits;
  stamp_routing_t r;
  int32_t renorm;
  StampF8Gemm up, down;  // h in up.Y
  uint8_t* codes;        // Q8 of X
  float* scales;
  int32_t parts;         // workgroups that share 64 columns of Y
  int32_t looks;         // kMaxLooks, or a test's
  float* sums;           // [parts][tokens][down.groups * 64]
  // [0] up products taken; [1 + i] of the i-th expert with rows: rows of h finished, 32 columns each; [1 + kMaxSlots + g] parts of 64 columns of Y finished
  uint32_t* sync;
};

struct Chosen {
  uint32_t mask[kF8MaxExperts];      // tokens of an expert
  int32_t base[kF8MaxExperts];       // its first row
  uint16_t expert[kMaxSlots + 1];    // experts with rows, in order; their first rows, and behind the last the number of rows
  uint16_t first[kMaxSlots + 1];
  uint8_t token[kMaxSlots];          // of a row
  float weight[kMaxSlots];           // of a row; NaN where a wait for it gave up
  int32_t id[kMaxSlots];             // of a slot
  float slot_weight[kMaxSlots];
  uint32_t wave_sum[kWaves];
  int32_t experts;
  uint32_t ticket;
};

__device__ __forceinline__ v8i load_w(const uint8_t* w) {
  return __builtin_shufflevector(*reinterpret_cast<const v4i*>(w), *reinterpret_cast<const v4i*>(w + 1024), 0, 1, 2, 3, 4, 5, 6, 7);
}

__device__ void choose(const MoeArgs& a, Chosen& s) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, E = a.r.experts, K = a.r.top_k, T = a.r.tokens;
  for (int e = t; e < kF8MaxExperts; e += kThreads) s.mask[e] = 0;
  __syncthreads();
  const TopArgs top = {a.logits, E, E, K, a.renorm};
  auto put = [&](int tok, int k, int id, float weight) __attribute__((always_inline)) {
    s.id[tok * K + k] = id;
    s.slot_weight[tok * K + k] = weight;
    if (id >= 0) atomicOr(&s.mask[id], 1u << tok);
  };
  if (E <= 32) top_tokens<kWaves, 16, 2, false>(top, 0, T, wave, lane, put);
  else if (E <= 64) top_tokens<kWaves, 16, 4, false>(top, 0, T, wave, lane, put);
  else if (E <= 128) top_tokens<kWaves, 16, 8, false>(top, 0, T, wave, lane, put);
  else if (E <= 256) top_tokens<kWaves, 16, 16, false>(top, 0, T, wave, lane, put);
  else top_tokens<kWaves, 64, 16, false>(top, 0, T, wave, lane, put);
  __syncthreads();
  // first rows and places among the experts with rows: one sum of both over the experts, two experts a thread
  static_assert(2 * kThreads >= kF8MaxExperts, "two experts a thread");
  uint32_t rows[2], mine[2];
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    rows[q] = __popc(s.mask[2 * t + q]);
    mine[q] = rows[q] | (rows[q] > 0 ? 0x10000u : 0u);
  }
  uint32_t incl = mine[0] + mine[1];
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_up(incl, d);
    if (lane >= d) incl += o;
  }
  if (lane == 63) s.wave_sum[wave] = incl;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    before += w < wave ? s.wave_sum[w] : 0;
    all += s.wave_sum[w];
  }
  uint32_t excl = before + incl - mine[0] - mine[1];
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    s.base[2 * t + q] = excl & 0xffff;
    if (rows[q] > 0) {
      s.expert[excl >> 16] = (uint16_t)(2 * t + q);
      s.first[excl >> 16] = (uint16_t)excl;
    }
    excl += mine[q];
  }
  if (t == 0) {
    s.experts = (int)(all >> 16);
    s.first[all >> 16] = (uint16_t)all;
  }
  __syncthreads();
  const bool writes = blockIdx.x == 0;
  if (t < T * K) {
    const int e = s.id[t], tok = t / K;
    const int row = e >= 0 ? s.base[e] + __popc(s.mask[e] & ((1u << tok) - 1)) : -1;
    if (row >= 0) {
      s.token[row] = (uint8_t)tok;
      s.weight[row] = s.slot_weight[t];
    }
    if (writes) {
      a.r.ids_dev[t] = e;
      a.r.weights_dev[t] = s.slot_weight[t];
      a.r.row_of_slot_dev[t] = row;
      if (row >= 0) a.r.token_of_row_dev[row] = tok;
      if (t >= (int)(all & 0xffff)) a.r.token_of_row_dev[t] = -1;
    }
  }
  if (writes) {
    for (int e = t; e < E; e += kThreads) a.r.offsets_dev[e] = s.base[e];
    if (t == 0) a.r.offsets_dev[E] = (int)(all & 0xffff);
  }
  __syncthreads();
}

// v[i] as a load of the vector unit: scalar loads return in any order, so a wait for one is a wait for all that were asked for since
__device__ __forceinline__ float vector_load(const float* v, int64_t i) {
  int zero = 0;
  asm volatile("" : "+v"(zero));
  return v[i + zero];
}

// h of 32 columns (a group) of an expert: the depth over the waves.  A wave has the weights of U blocks of channels in registers, and behind its last ones the first
// of its next product.
struct UpProduct {
  static constexpr int U = 4;
  int kb0, kb1, index, r0, nr, g, tok;
  const uint8_t *w0, *x0;
  const float* sw0;
  v8i W[U][4], X[U];
  float sx[U], sw[U], su[U];

  __device__ __forceinline__ void begin(const MoeArgs& a, const Chosen& s, int place, int group) {
    const StampF8Gemm& p = a.up;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int e = __builtin_amdgcn_readfirstlane(s.expert[place]);
    index = place;
    g = group;
    r0 = __builtin_amdgcn_readfirstlane(s.first[place]);
    nr = __builtin_amdgcn_readfirstlane(s.first[place + 1]) - r0;
    kb0 = p.Kb * wave / kWaves;
    kb1 = p.Kb * (wave + 1) / kWaves;
    w0 = p.W + ((int64_t)e * p.groups + g) * p.Kb * kF8GroupBytes + lane * 16;
    sw0 = p.SW + ((int64_t)e * 2 * p.nblk + (g >> 2)) * p.Kb;
    tok = s.token[r0 + min(lane & 15, nr - 1)];
    x0 = a.codes + (int64_t)tok * p.Kb * 128 + 16 * (lane >> 4);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (kb0 + u < kb1) ask(a, u, kb0 + u);
  }
  __device__ __forceinline__ void ask(const MoeArgs& a, int u, int kb) {
#pragma unroll
    for (int b = 0; b < 4; ++b) W[u][b] = load_w(w0 + (int64_t)kb * kF8GroupBytes + b * 2048);
    const v4i* const x = reinterpret_cast<const v4i*>(x0 + (int64_t)kb * 128);
    X[u] = __builtin_shufflevector(x[0], x[4], 0, 1, 2, 3, 4, 5, 6, 7);
    sx[u] = a.scales[kb * a.up.ld_sa + tok];
    sw[u] = vector_load(sw0, kb);
    su[u] = vector_load(sw0, (int64_t)a.up.nblk * a.up.Kb + kb);
  }
  __device__ __forceinline__ void multiply(const MoeArgs& a, f4 (&acc)[4]) {
    for (int kb = kb0; kb < kb1; kb += U) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (kb + u < kb1) {
          b8 x[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) x[k] = widen8(X[u][2 * k], X[u][2 * k + 1]);
          const float f0 = sx[u] * sw[u], f1 = sx[u] * su[u];
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            f4 q = {0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < 4; ++k) q = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(W[u][b][2 * k], W[u][b][2 * k + 1]), x[k], q, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[b][r] = __builtin_fmaf(q[r], (b & 1) ? f1 : f0, acc[b][r]);
          }
          __builtin_amdgcn_sched_barrier(0);
          if (kb + u + U < kb1) ask(a, u, kb + u + U);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  }
};

// act(gate) * up of the product's rows: a thread a value.
__device__ __forceinline__ void finish_h(const MoeArgs& a, float (*red)[16][kUpLd], int index, int r0, int nr, int g) {
  static_assert(kThreads == 16 * 32, "a thread a value");
  const StampF8Gemm& p = a.up;
  const int t = threadIdx.x, m = t >> 5, c = t & 31, pl = ((c >> 2) & 1) * 32 + (c >> 3) * 4 + (c & 3);  // lanes c / 8, pair c / 4 % 2
  const int first = 2 * __builtin_amdgcn_readfirstlane(t >> 6);  // of the wave's two rows
  if (first >= nr) return;
  float h[1] = {0}, u[1] = {0};
#pragma unroll
  for (int q = 0; q < kWaves; ++q) h[0] += red[q][m][pl], u[0] += red[q][m][pl + 16];
  gate(h, u, p.act);
  // stores that go through to where the whole chip looks: a release fence would write the L2's changed lines back, 45 us for 16 tokens and 8 of 256 experts
  if (m < nr)
    __hip_atomic_store(static_cast<float*>(p.Y) + (int64_t)(r0 + m) * p.ld_y + g * 32 + c, g * 32 + c < p.N ? h[0] : 0.0f, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  // the rows are there before they are counted
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  if ((t & 63) == 0) __hip_atomic_fetch_add(&a.sync[1 + index], (uint32_t)min(nr - first, 2), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <bool YBF16>
__global__ __launch_bounds__(kThreads) void k_moe_few(MoeArgs a) {
  __shared__ Chosen s;
  __shared__ __attribute__((aligned(16))) uint8_t lds[kRoom];
  const int t = threadIdx.x, lane = t & 63, f = lane >> 4, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  uint32_t ticket = 0;
  if (t == 0) ticket = __hip_atomic_fetch_add(&a.sync[0], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  choose(a, s);

  const int nact = __builtin_amdgcn_readfirstlane(s.experts), groups = a.up.groups;
  float(*const up_red)[16][kUpLd] = reinterpret_cast<float(*)[16][kUpLd]>(lds);
  auto take = [&]() __attribute__((always_inline)) {  // the next up product; the one after it is asked for
    if (t == 0) s.ticket = ticket;
    __syncthreads();
    const uint32_t item = __builtin_amdgcn_readfirstlane(s.ticket);
    if (t == 0 && item < (uint32_t)(nact * groups)) ticket = __hip_atomic_fetch_add(&a.sync[0], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return item;
  };
  uint32_t item = take();
  if (item < (uint32_t)(nact * groups)) {
    UpProduct up;
    up.begin(a, s, item / groups, item % groups);
    for (;;) {
      f4 acc[4];
#pragma unroll
      for (int b = 0; b < 4; ++b) acc[b] = f4{0, 0, 0, 0};
      up.multiply(a, acc);
      __syncthreads();  // the sums of the product before have been read
#pragma unroll
      for (int b = 0; b < 4; ++b) *reinterpret_cast<f4*>(&up_red[wave][lane & 15][b * 16 + 4 * f]) = acc[b];
      const int index = up.index, r0 = up.r0, nr = up.nr, g = up.g;
      item = take();
      const bool more = item < (uint32_t)(nact * groups);
      if (more) up.begin(a, s, item / groups, item % groups);
      finish_h(a, up_red, index, r0, nr, g);
      if (!more) break;
    }
  }

  const StampF8Gemm& p = a.down;
  const int Kb = p.Kb, ld_row = Kb * 128 + 16, row_bytes = ld_row + Kb * 4;
  const int most = kMoeChunkBytes / row_bytes;  // rows of h held at a time: at least a token's for every token
  const int tok = lane & 15, all_units = nact * Kb;
  for (int item = blockIdx.x; item < p.groups * a.parts; item += gridDim.x) {
    const int part = item / p.groups, g = item - part * p.groups;
    const int ua = (int)((int64_t)all_units * part / a.parts), ub = (int)((int64_t)all_units * (part + 1) / a.parts);  // units: 128 channels of an expert
    const uint8_t* const w0 = p.W + (int64_t)g * Kb * kF8GroupBytes + lane * 16;
    const float* const sw0 = p.SW + (int64_t)(g >> 1) * Kb;
    f4 acc[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) acc[b] = f4{0, 0, 0, 0};
    const int end = ua < ub ? (ub - 1) / Kb + 1 : 0;
    for (int i0 = ua < ub ? ua / Kb : 0; i0 < end;) {
      const int r0 = s.first[i0];
      int i1 = end;
      if (s.first[end] - r0 > most) {
        i1 = i0 + 1;
        while (s.first[i1 + 1] - r0 <= most) ++i1;  // not up to the last: with its rows they are more than that
      }
      const int nr = s.first[i1] - r0, v0 = max(ua, i0 * Kb), nv = min(ub, i1 * Kb) - v0;
      const int u0 = v0 + nv * wave / kWaves, u1 = v0 + nv * (wave + 1) / kWaves;
      constexpr int U = 4;
      v8i W[U][4];
      float sw[U];
      // lane l: where the weights of the wave's unit u + l are, and which rows it has
      struct Units {
        uint32_t w, sw, rows, kb;
      };
      auto units_from = [&](int u) __attribute__((always_inline)) {
        const int v = min(u + lane, u1 - 1), i = v / Kb, e = s.expert[i];
        Units n;
        n.kb = v - i * Kb;
        n.w = (uint32_t)(e * p.groups) * Kb + n.kb;
        n.sw = (uint32_t)(e * p.nblk) * Kb + n.kb;
        n.rows = s.mask[e] | (uint32_t)(s.first[i] - r0) << 16;
        return n;
      };
      auto fetch = [&](int j, const Units& n, int l) __attribute__((always_inline)) {
        const uint8_t* const w = w0 + (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)n.w, l) * kF8GroupBytes;
#pragma unroll
        for (int b = 0; b < 4; ++b) W[j][b] = load_w(w + b * 2048);
        sw[j] = vector_load(sw0, (uint32_t)__builtin_amdgcn_readlane((int)n.sw, l));
      };
      Units now{}, next{};
      if (u0 < u1) {
        now = units_from(u0);
        next = units_from(u0 + 64);
      }
#pragma unroll
      for (int j = 0; j < U; ++j)
        if (u0 + j < u1) fetch(j, now, j);
      if (wave == 0) {  // the experts' rows of h; one wave looks, and drops what its CU and L2 hold of before, for all
        for (int i = i0 + lane; i < i1; i += 64) {
          const uint32_t all = (uint32_t)((s.first[i + 1] - s.first[i]) * groups);
          for (int look = 0; __hip_atomic_load(&a.sync[1 + i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) < all; ++look) {
            if (look >= a.looks) {  // in vain: its rows count as NaN from here on
              for (int r = s.first[i]; r < s.first[i + 1]; ++r) s.weight[r] = __builtin_nanf("");
              break;
            }
            __builtin_amdgcn_s_sleep(1);
          }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
      }
      __syncthreads();  // and the rows before have been read
      uint8_t* const h = lds;
      float* const sh = reinterpret_cast<float*>(lds + nr * ld_row);
      constexpr int kAtOnce = 2;  // loads on their way
      for (int v1 = t; v1 < nr * Kb * 8; v1 += kAtOnce * kThreads) {  // Q8 of h: 16 channels of a row, 8 lanes a block
        Raw16<false> x[kAtOnce];
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) {
          const int v = v1 + q * kThreads, m = v / (Kb * 8), c = (v - m * Kb * 8) * 16;
          if (v < nr * Kb * 8) x[q].load(static_cast<const float*>(a.up.Y) + (int64_t)(r0 + m) * a.up.ld_y, c, a.up.groups * 32);
        }
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) {
          const int v = v1 + q * kThreads, m = v / (Kb * 8), c = (v - m * Kb * 8) * 16;
          if (v < nr * Kb * 8) {
            float scale, inv;
            scale_of(max8(x[q].amax()), p.pow2, &scale, &inv);
            *reinterpret_cast<u4*>(h + m * ld_row + c) = x[q].codes(inv);
            if ((t & 7) == 0) sh[m * Kb + (c >> 7)] = scale * s.weight[r0 + m];
          }
        }
      }
      __syncthreads();
      for (int u = u0; u < u1; u += U) {
        const int l0 = (u - u0) & 63, l1 = (l0 + U) & 63;
        const Units after = l1 == 0 ? next : now;
#pragma unroll
        for (int j = 0; j < U; ++j) {
          if (u + j < u1) {
            // the row of the lane's token among the expert's
            const uint32_t list = (uint32_t)__builtin_amdgcn_readlane((int)now.rows, l0 + j);
            const int kb = __builtin_amdgcn_readlane((int)now.kb, l0 + j);
            const bool has = (list >> tok) & 1;
            const int m = has ? (int)(list >> 16) + __popc(list & ((1u << tok) - 1)) : 0;
            const v4i* const x = reinterpret_cast<const v4i*>(h + m * ld_row + kb * 128 + 16 * f);
            const v8i X = __builtin_shufflevector(x[0], x[4], 0, 1, 2, 3, 4, 5, 6, 7);
            const float fs = sh[m * Kb + kb] * sw[j];
            b8 xw[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) xw[k] = widen8(X[2 * k], X[2 * k + 1]);
#pragma unroll
            for (int b = 0; b < 4; ++b) {
              f4 q = {0, 0, 0, 0};
#pragma unroll
              for (int k = 0; k < 4; ++k) q = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(W[j][b][2 * k], W[j][b][2 * k + 1]), xw[k], q, 0, 0, 0);
#pragma unroll
              for (int r = 0; r < 4; ++r) acc[b][r] = has ? __builtin_fmaf(q[r], fs, acc[b][r]) : acc[b][r];
            }
            __builtin_amdgcn_sched_barrier(0);
            if (u + U + j < u1) fetch(j, after, l1 + j);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        if (l1 == 0) {
          now = next;
          if (u + U + 64 < u1) next = units_from(u + U + 64);
        }
      }
      i0 = i1;
    }
    // the waves' sums: element r of block b is place 16 b + 4 f + r, token lane % 16
    __syncthreads();
    float(*red)[16][kUpLd] = reinterpret_cast<float(*)[16][kUpLd]>(lds);
#pragma unroll
    for (int b = 0; b < 4; ++b) *reinterpret_cast<f4*>(&red[wave][tok][16 * b + 4 * f]) = acc[b];
    __syncthreads();
    // a thread has one column for the tokens of its wave and of that plus 8
    const int c = lane, pl = (2 * (c >> 5) + ((c >> 2) & 1)) * 16 + ((c >> 3) & 3) * 4 + (c & 3), n = 64 * g + c;
    float v[2] = {0, 0};
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int m = wave + 8 * q;
      if (m >= a.r.tokens) continue;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) v[q] += red[w][m][pl];
    }
    if (a.parts > 1) {
      // the last of the column's workgroups adds the parts up, in order
      float* const sums = a.sums + (int64_t)g * 64 + c;
      const int64_t ld = (int64_t)p.groups * 64;
#pragma unroll
      for (int q = 0; q < 2; ++q)
        if (wave + 8 * q < a.r.tokens)
          __hip_atomic_store(sums + ((int64_t)part * a.r.tokens + wave + 8 * q) * ld, v[q], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      if (t == 0) s.ticket = __hip_atomic_fetch_add(&a.sync[1 + kMaxSlots + g], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __syncthreads();
      if (s.ticket != (uint32_t)a.parts - 1) continue;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        v[q] = 0.0f;
        if (wave + 8 * q >= a.r.tokens) continue;
        for (int i = 0; i < a.parts; i += 8) {
          float w[8];
#pragma unroll
          for (int k = 0; k < 8; ++k)
            w[k] = i + k < a.parts ? __hip_atomic_load(sums + ((int64_t)(i + k) * a.r.tokens + wave + 8 * q) * ld, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0f;
#pragma unroll
          for (int k = 0; k < 8; ++k) v[q] += w[k];
        }
      }
    }
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int m = wave + 8 * q;
      if (m >= a.r.tokens || n >= p.N) continue;
      if (p.bias != nullptr) {
        for (int k = 0; k < a.r.top_k; ++k) {
          const int e = s.id[m * a.r.top_k + k];
          if (e >= 0) v[q] = __builtin_fmaf(s.slot_weight[m * a.r.top_k + k], p.bias[(int64_t)e * p.N + n], v[q]);
        }
      }
      if (p.R != nullptr) v[q] += YBF16 ? bf16_lo(static_cast<const uint16_t*>(p.R)[m * p.ld_r + n]) : static_cast<const float*>(p.R)[m * p.ld_r + n];
      if constexpr (YBF16) static_cast<uint16_t*>(p.Y)[m * p.ld_y + n] = to_bf16(v[q]);
      else static_cast<float*>(p.Y)[m * p.ld_y + n] = v[q];
    }
  }
}
}  // namespace

hipError_t stamp_launch_moe(const stamp_router_t& router, const stamp_routing_t& r, const void* X, int x_bf16, int64_t ld_x, const StampF8Gemm& up,
                            const StampF8Gemm& down, uint8_t* codes, float* scales, float* logits, uint32_t* sync, float* sums,
                            int32_t looks, hipStream_t st) {
  MoeArgs a;
  a.looks = looks < 0 ? kMaxLooks : looks;
  a.logits = logits;
  a.r = r;
  a.renorm = router.renormalize;
  a.up = up;
  a.down = down;
  a.codes = codes;
  a.scales = scales;
  a.sync = sync;
  a.sums = sums;
  // a unit (128 channels of an expert) for each of a workgroup's waves at least, if every row has an expert of its own: one token, 2 of 16 experts,
  // 1024 -> 512 take 14 us in one part and 18 in 16
  const int64_t slots = (int64_t)r.tokens * r.top_k, units = (slots < r.experts ? slots : r.experts) * down.Kb;
  const int most_parts = stamp_moe_parts(down.groups), busy = (int)(units / kWaves);
  a.parts = busy < 1 ? 1 : busy < most_parts ? busy : most_parts;
  const RouterQ8 q = {codes, scales, up.ld_sa, up.pow2, 0, sync, (int32_t)(stamp_moe_sync_bytes(down.groups) / 4)};
  const hipError_t e = stamp_launch_router(router, X, x_bf16, ld_x, r.tokens, r.experts, up.d, q, logits, st);
  if (e != hipSuccess) return e;
  const int64_t products = (slots < r.experts ? slots : r.experts) * up.groups, columns = (int64_t)down.groups * a.parts;
  const int64_t most = products > columns ? products : columns, cus = stamp_device_cus();
  const uint32_t grid = (uint32_t)(most < cus ? most : cus);
  if (down.y_bf16) k_moe_few<true><<<grid, kThreads, 0, st>>>(a);
  else k_moe_few<false><<<grid, kThreads, 0, st>>>(a);
  return hipGetLastError();
}
