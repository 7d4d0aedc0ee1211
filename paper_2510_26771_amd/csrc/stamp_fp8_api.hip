// C entry points of the 8-bit floating point layers, the router and the experts.
#include <stdlib.h>
#include <string.h>

#include <new>

#include "stamp_fp8.h"

namespace {

constexpr int32_t kMaxRows = 1 << 24;

size_t align256(size_t n) { return (n + 255) / 256 * 256; }
int64_t scales_ld(int32_t rows) { return ((int64_t)rows + 3) / 4 * 4; }
int type_size(int32_t dtype) { return dtype == STAMP_BF16 ? 2 : 4; }
bool is_float_type(int32_t t) { return t == STAMP_F32 || t == STAMP_BF16; }

stamp_status_t validate(const stamp_fp8_desc_t* d) {
  if (d->d_in < 1 || d->d_out < 1 || d->experts < 0) return STAMP_ERR_SHAPE;
  if (d->gated < 0 || d->gated > 1 || d->w_is_out_by_in < 0 || d->w_is_out_by_in > 1) return STAMP_ERR_SHAPE;
  if (!is_float_type(d->x_dtype) || !is_float_type(d->y_dtype)) return STAMP_ERR_SHAPE;
  if (!is_float_type(d->w_dtype) && d->w_dtype != STAMP_E4M3) return STAMP_ERR_SHAPE;
  if (d->scale_format != STAMP_SCALE_F32 && d->scale_format != STAMP_SCALE_POW2) return STAMP_ERR_SHAPE;
  if (d->gated && d->experts == 0) return STAMP_ERR_SHAPE;
  if (d->d_in > 65536 || d->d_out > (1 << 20) || d->experts > kF8MaxExperts) return STAMP_ERR_UNSUPPORTED;
  if (d->w_dtype == STAMP_E4M3 && !d->w_is_out_by_in) return STAMP_ERR_UNSUPPORTED;
  return STAMP_OK;
}

StampF8Gemm gemm_args(const stamp_fp8_plan* p) {
  StampF8Gemm a;
  memset(&a, 0, sizeof(a));
  a.W = p->w_dev;
  a.SW = p->sw_dev;
  a.bias = p->bias_dev;
  a.sets = p->sets;
  a.groups = p->groups;
  a.Kb = p->Kb;
  a.nblk = p->nblk;
  a.N = p->desc.d_out;
  a.pow2 = p->desc.scale_format == STAMP_SCALE_POW2;
  a.gated = p->desc.gated;
  a.y_bf16 = p->desc.y_dtype == STAMP_BF16;
  a.wide_sums = f8_wide_sums(a);
  a.forced = p->forced;
  return a;
}

int route_of(const StampF8Gemm& a, int rows) { return stamp_f8_route(a.sets, a.groups, a.Kb, rows, a.wide_sums, a.gated, a.forced); }
// the codes are wanted as bf16
bool wide_codes(const StampF8Gemm& a, int rows) { return a.wide_sums && route_of(a, rows) != STAMP_FP8_ROUTE_ROWS; }

// the kernel quantizes the rows itself
bool takes_x(const StampF8Gemm& a, int rows) { return route_of(a, rows) == STAMP_FP8_ROUTE_ROWS && stamp_f8_rows_quantize(a, rows) > 0; }
void give_x(StampF8Gemm* a, const stamp_fp8_desc_t& d, int rows, const void* X, int64_t ld_x) {
  a->X = X;
  a->chunk = stamp_f8_rows_quantize(*a, rows);
  a->ld_x = ld_x;
  a->x_bf16 = d.x_dtype == STAMP_BF16;
  a->d = d.d_in;
}

hipError_t product(const StampF8Gemm& a, hipStream_t st) {
  if (route_of(a, a.rows) == STAMP_FP8_ROUTE_ROWS) return stamp_launch_f8_rows(a, st);
  const F8Cut cut = stamp_f8_cut(a.sets, a.groups, a.Kb, a.rows, a.wide_sums, a.gated, a.forced);
  if (cut.groups == 0) return stamp_launch_f8_tiles(a, 64 << cut.size, cut.parts, st);
  StampF8Gemm first = a, rest = a;
  const int columns = cut.groups * kF8Group;
  first.groups = cut.groups;
  first.nblk = cut.groups / 2;
  first.N = columns;
  rest.groups -= cut.groups;
  rest.nblk -= cut.groups / 2;
  rest.N -= columns;
  rest.W += (size_t)cut.groups * a.Kb * kF8GroupBytes;
  rest.SW += (size_t)(cut.groups / 2) * a.Kb;
  if (a.bias != nullptr) rest.bias += columns;
  rest.Y = static_cast<char*>(a.Y) + (size_t)columns * (a.y_bf16 ? 2 : 4);
  const hipError_t e = stamp_launch_f8_tiles(first, 64 << cut.size, cut.parts, st);
  return e != hipSuccess ? e : stamp_launch_f8_tiles(rest, 64 << cut.rest_size, cut.rest_parts, st);
}

// room for a code of the activations: as bf16 where some route wants that
int code_bytes(const stamp_fp8_plan* p) { return gemm_args(p).wide_sums ? 2 : 1; }

struct LinearWs {
  size_t codes, scales, partial, total;
};
LinearWs linear_ws(const stamp_fp8_plan* p, int32_t rows) {
  LinearWs w;
  w.codes = 0;
  w.scales = align256((size_t)rows * p->Kp * code_bytes(p));
  w.partial = w.scales + align256((size_t)p->Kb * scales_ld(rows) * sizeof(float));
  w.total = w.partial + align256(stamp_f8_partial_bytes(p->groups, rows));
  return w;
}

struct ExpertsWs {
  size_t codes, scales, h, sh, rows, wide, partial, total;
  int64_t ld_rows;
};
ExpertsWs experts_ws(const stamp_fp8_plan* up, const stamp_fp8_plan* down, int32_t tokens, int32_t top_k) {
  ExpertsWs w;
  const int64_t slots = (int64_t)tokens * top_k, ld = scales_ld((int32_t)slots);
  w.codes = 0;
  w.scales = align256((size_t)tokens * up->Kp * code_bytes(up));
  w.h = w.scales + align256((size_t)up->Kb * scales_ld(tokens) * sizeof(float));
  w.sh = w.h + align256((size_t)slots * down->Kp);
  w.rows = w.sh + align256((size_t)down->Kb * ld * sizeof(float));
  w.ld_rows = (down->desc.d_out + 7) / 8 * 8;
  // Rows in Y's type: a bf16 Y is a sum of terms rounded once each, 2.3e-3 off where rows in fp32 give 1.7e-3, which is Y's own rounding; but
  // they are the most bytes of the call (8192 tokens, 8 of 64 experts, 4096 -> 1536: down product 529 -> 647 us, weighted sum 122 -> 242, the whole
  // 2200 -> 2447).  An fp32 Y has them in fp32.
  // The up product writes codes of one byte; a down product that wants them as bf16 has them widened here
  w.wide = w.rows + align256((size_t)slots * w.ld_rows * type_size(down->desc.y_dtype));
  w.partial = w.wide + (code_bytes(down) == 2 ? align256((size_t)slots * down->Kp * 2) : 0);
  w.total = w.partial + align256(stamp_f8_partial_bytes(down->groups, (int32_t)slots));
  return w;
}

stamp_status_t check_ws(const void* ws, size_t bytes, size_t need) {
  if (need == 0) return STAMP_OK;
  return ws == nullptr || reinterpret_cast<uintptr_t>(ws) % 256 != 0 || bytes < need ? STAMP_ERR_WORKSPACE : STAMP_OK;
}

// a matrix of `rows` rows of n elements, ld apart: element-aligned
stamp_status_t check_matrix(const void* p, int32_t dtype, int64_t ld, int64_t n) {
  if (p == nullptr) return STAMP_ERR_NULL;
  if (ld < n || reinterpret_cast<uintptr_t>(p) % type_size(dtype) != 0) return STAMP_ERR_SHAPE;
  return ld > (1 << 21) ? STAMP_ERR_UNSUPPORTED : STAMP_OK;  // 256 rows within 32-bit offsets
}

stamp_status_t check_routing(const stamp_routing_t* r) {
  if (r->tokens < 0 || r->experts < 1 || r->top_k < 1) return STAMP_ERR_SHAPE;
  if (r->experts > kF8MaxExperts || r->top_k > 32 || r->tokens > (1 << 22)) return STAMP_ERR_UNSUPPORTED;
  if (r->offsets_dev == nullptr) return STAMP_ERR_NULL;
  if (r->tokens > 0 && (r->ids_dev == nullptr || r->weights_dev == nullptr || r->token_of_row_dev == nullptr || r->row_of_slot_dev == nullptr))
    return STAMP_ERR_NULL;
  return STAMP_OK;
}

stamp_status_t done(hipError_t e) { return e == hipSuccess ? STAMP_OK : STAMP_ERR_DEVICE; }

// linear_forward, grouped_forward
stamp_status_t forward(const stamp_fp8_plan* p, int32_t rows, const int32_t* offsets, bool grouped, const void* X, int64_t ld_x, void* Y, int64_t ld_y,
                       void* ws, size_t ws_bytes, hipStream_t st) {
  if (p == nullptr) return STAMP_ERR_NULL;
  if (p->desc.gated || (p->desc.experts > 0) != grouped) return STAMP_ERR_UNSUPPORTED;
  if (rows < 0 || rows > kMaxRows) return STAMP_ERR_SHAPE;
  if (grouped && offsets == nullptr) return STAMP_ERR_NULL;
  if (rows == 0) return STAMP_OK;
  stamp_status_t s = check_matrix(X, p->desc.x_dtype, ld_x, p->desc.d_in);
  if (s == STAMP_OK) s = check_matrix(Y, p->desc.y_dtype, ld_y, p->desc.d_out);
  const LinearWs w = linear_ws(p, rows);
  if (s == STAMP_OK) s = check_ws(ws, ws_bytes, w.total);
  if (s != STAMP_OK) return s;
  uint8_t* codes = static_cast<uint8_t*>(ws) + w.codes;
  float* scales = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + w.scales);
  StampF8Gemm a = gemm_args(p);
  if (takes_x(a, rows)) {
    give_x(&a, p->desc, rows, X, ld_x);
  } else if (stamp_launch_f8_quant(X, p->desc.x_dtype == STAMP_BF16, ld_x, rows, p->desc.d_in, a.pow2, wide_codes(a, rows), codes, scales, scales_ld(rows),
                                   st) != hipSuccess) {
    return STAMP_ERR_DEVICE;
  }
  a.A = codes;
  a.partial = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + w.partial);
  a.SA = scales;
  a.ld_sa = scales_ld(rows);
  a.a_rows = a.rows = rows;
  a.offsets = offsets;
  a.Y = Y;
  a.ld_y = ld_y;
  return done(product(a, st));
}

}  // namespace

// Kernel for a product of `rows` rows over `sets` weights, by estimates in us.
//
// The host knows rows and sets, not how the rows lie on the sets: the estimates take them as even (the last paragraph: where they are not).
//
// Few rows: up to 12 a set always the rows kernel, which reads the weights at up to 6 TB/s; beyond that its pass over 16 rows is the bound, and
// a set's last pass half empty.  Tiles of 64, 128, 256 rows: a workgroup a CU, so rounds of `cus` tiles, each of Kb steps and a start and end.
// us per step and per round, measured on full rounds: 0.53 + 3.5, 0.9 + 4.5, 1.45 + 6; with sums in fp32 1.05 + 4, 1.75 + 6.  (2048 x 4096 -> 11008:
// 120, 98 and 100 us; 8192 x 1152 -> 4608: 77, 64 and 60; 512 x 4096 -> 11008: 39, 30 and 45.)  Over several sets the tiles' ends take 2 to 5 more,
// as neighbours read other weights; and the weights have to come from memory.
// Few tiles: the depth in up to 8 parts, at least 4 blocks each, while the workgroups fit the CUs; 3.5 us for the pass that adds them up,
// and the parts' rows at 3 TB/s.  A step takes 0.43, 0.7, 1.1 us while most CUs are idle (sums in fp32: 0.9, 1.3).
//
// Whole calls, us (rows kernel / tiles of 64 / of 128), 85 sets of 1024 -> 2944, bf16 Y: 16 rows a set 52 / 53 / 57, 24: 74 / 56 / 59, 48: 145 / 62 / 66;
// fp32 Y 16: 56 / 62 / 76, 24: 76 / 66 / 80, 64: 196 / 105 / 97.  8 sets of 2048 -> 2048, fp32 Y 32: 15.3 / 21.2 / 22.3, 64: 27 / 25 / 28.  One of 4096 -> 11008,
// bf16 Y 32: 17.9 / 17.4, 48: 24.1 / 18.2; of 1152 -> 4608 32: 8.8 / 9.4, 48: 11.7 / 9.8, fp32 Y 64: 13.5 / 15.1, 96: 19.1 / 15.2; of 8192 -> 1024 64: 22.4 / 18.4;
// of 590 -> 7231 58: 11.2 / 13.2.  Over 88 layers of 13 to 16000 rows, 100 to 9000 channels and 100 to 15000 columns the choice takes 0.3 % more than the
// best on average, 6 % at worst.
// Over 120 products of 8 to 191 sets with 4 to 96 rows a set, gated ones among them, rows dealt at random with all sets alike, the choice takes
// 0.6 % more than the best on average, 17 % at worst.
//
// Rows that lie unevenly: the rows kernel walks a set's rows 16 by 16 in that set's workgroups alone, while tiles of 64 rows spread over the CUs.
// us, rows kernel (the choice) / tiles of 64; "falling": shares 1, 1/2, 1/3, ...; two, one: sets that have all rows.
//                                     even          half of the sets  falling      two          one
//   96 over 32 sets, 4096 -> 1536    37 / 36        21 / 23           31 / 28      20 / 21      34 / 21
//   760 over 64, 4096 -> 1536        80 / 85        72 / 37          117 / 85     142 / 24     236 / 24
//   1500 over 128, 2048 -> 2048     100 / 112       84 / 55          143 / 120    205 / 21     284 / 22
//   3000 over 256, 2048 -> 768       81 / 90        71 / 48          171 / 99     302 / 22     561 / 22
// A rule on rows and sets alone has to lose on one side; this one is right for even loads and loses most where few of many sets are busy.
namespace {
constexpr float kStep[2][3] = {{0.53f, 0.9f, 1.45f}, {1.05f, 1.75f, 0.0f}}, kIdle[2][3] = {{0.43f, 0.7f, 1.1f}, {0.9f, 1.3f, 0.0f}},
                kEnds[2][3] = {{3.5f, 4.5f, 6.0f}, {4.0f, 6.0f, 0.0f}}, kSetEnds[2][3] = {{7.5f, 7.5f, 9.0f}, {9.0f, 8.0f, 0.0f}};
constexpr float kBytesPerUs = 6e6f;
constexpr int kAlwaysRows = 12;  // a set
struct TileChoice {
  int size, parts;  // tiles of 64 << size rows, parts of the depth
  float us;
};
int busy_sets(int sets, int rows) { return sets < rows ? sets : rows > 0 ? rows : 1; }
float weight_bytes(int sets, int groups, int Kb, int rows) { return (float)busy_sets(sets, rows) * groups * Kb * kF8GroupBytes; }

TileChoice best_tiles(int sets, int groups, int Kb, int rows, int wide_sums, int gated, int forced) {
  const int busy = busy_sets(sets, rows), cus = stamp_device_cus(), w = wide_sums != 0;
  const int64_t ncol = (groups + 3) / 4;
  const float read = weight_bytes(sets, groups, Kb, rows) / kBytesPerUs;
  TileChoice best = {-1, 1, 0.0f};
  for (int i = 0; i < (w ? 2 : 3); ++i) {  // the bf16 operands of 256 rows do not fit the registers
    if (forced != 0 && forced != STAMP_FP8_ROUTE_TILES_64 + i) continue;
    const int bm = 64 << i, many = rows / bm + (busy + 1) / 2;  // half of the last tile of a set is empty
    const int64_t tiles = (sets == 1 ? (rows + bm - 1) / bm : many > busy ? many : busy) * ncol;
    const float ends = (sets > 1 ? kSetEnds : kEnds)[w][i];
    TileChoice c = {i, 1, (float)((tiles + cus - 1) / cus) * ((float)Kb * (2 * tiles <= cus ? kIdle : kStep)[w][i] + ends)};
    const float least = read + (sets > 1 ? 6.0f : ends);  // the weights' way from memory
    if (c.us < least) c.us = least;
    for (int n = 2; !gated && n <= kF8MaxParts && n * tiles <= cus && 4 * n <= Kb; ++n) {
      const float steps = (float)((Kb + n - 1) / n) * kIdle[w][i] + ends;
      const float us = (steps > least ? steps : least) + 3.5f + (float)n * rows * groups * 64 * 8 * 1e-6f / 3.0f;
      if (us < c.us) c.us = us, c.parts = n;
    }
    if (best.size < 0 || c.us < best.us) best = c;
  }
  return best;
}

float rows_us(int sets, int groups, int Kb, int rows) {
  const float read = weight_bytes(sets, groups, Kb, rows) / kBytesPerUs;
  const float passes = sets == 1 ? (float)((rows + 15) / 16) : (float)rows / busy_sets(sets, rows) / 16.0f + 0.5f;
  const float work = read * 0.84f * passes;
  const float pass = 0.3f + 0.09f * Kb, deep = 0.8f + 0.025f * Kb;  // its own chain of steps
  return 2.5f + (read > work ? read : work) + passes * (pass < deep ? pass : deep);
}
}  // namespace

int stamp_f8_route(int sets, int groups, int Kb, int rows, int wide_sums, int gated, int forced) {
  if (forced == STAMP_FP8_ROUTE_ROWS || (forced == 0 && (int64_t)rows <= (int64_t)kAlwaysRows * sets)) return STAMP_FP8_ROUTE_ROWS;
  const TileChoice tiles = best_tiles(sets, groups, Kb, rows, wide_sums, gated, forced);
  return forced == 0 && rows_us(sets, groups, Kb, rows) <= tiles.us ? STAMP_FP8_ROUTE_ROWS : STAMP_FP8_ROUTE_TILES_64 + tiles.size;
}

// Tiles that leave most CUs idle in their last round: of one layer, the columns of the whole rounds first, the others in a launch of their own
// in the tiles that suit them.  2048 x 4096 -> 11008: 344 tiles of 256 rows x 256 columns are 1.34 rounds, 100.7 us; 256 such tiles, then the
// other columns as 176 tiles of 128 rows 95.7.  8192 x 1152 -> 4608 (powers of two): 60.0 -> 56.7.  Over 44 drawn sizes where the estimate fell by 5 % or more the
// two launches took 0.78 to 1.04 of the one's time; where it fell by 10 % or more 0.78 to 1.04 as well, by 5 to 10 % mostly nothing: the line.
F8Cut stamp_f8_cut(int sets, int groups, int Kb, int rows, int wide_sums, int gated, int forced) {
  const TileChoice all = best_tiles(sets, groups, Kb, rows, wide_sums, gated, forced);
  F8Cut cut = {0, all.size, all.parts, 0, 1};
  if (sets > 1 || gated || forced != 0 || all.parts > 1) return cut;
  const int cus = stamp_device_cus(), ncol = (groups + 3) / 4, w = wide_sums != 0;
  float best = 0.9f * all.us;  // the second launch has to pay
  for (int i = 0; i < (w ? 2 : 3); ++i) {
    const int high = (rows + (64 << i) - 1) / (64 << i), rounds = (int)((int64_t)high * ncol / cus);
    const int cols = high > 0 ? (int)((int64_t)rounds * cus / high) : 0;
    if (rounds < 1 || cols < 1 || cols >= ncol) continue;
    const TileChoice rest = best_tiles(1, groups - 4 * cols, Kb, rows, wide_sums, 0, 0);
    const float us = (float)rounds * ((float)Kb * kStep[w][i] + kEnds[w][i]) + rest.us;
    if (us < best) best = us, cut = F8Cut{cols * 4, i, 1, rest.size, rest.parts};
  }
  return cut;
}

// parts * tiles <= CUs, and the rows are at most the tiles' (a set's half tile is counted, and one more)
size_t stamp_f8_partial_bytes(int groups, int rows) {
  const size_t whole = (size_t)kF8MaxParts * rows * groups * 64, fit = (size_t)stamp_device_cus() * 256 * 256;
  return (whole < fit ? whole : fit) * sizeof(float);
}

extern "C" {

stamp_status_t stamp_fp8_plan_create(const stamp_fp8_desc_t* desc, const void* W_dev, const float* w_scales_dev, const float* bias_dev, void* hip_stream,
                                     stamp_fp8_plan_t** out) {
  if (desc == nullptr || out == nullptr) return STAMP_ERR_NULL;
  *out = nullptr;
  const stamp_status_t vs = validate(desc);
  if (vs != STAMP_OK) return vs;
  if (W_dev == nullptr || (desc->w_dtype == STAMP_E4M3) != (w_scales_dev != nullptr)) return STAMP_ERR_NULL;
  if (desc->gated && bias_dev != nullptr) return STAMP_ERR_UNSUPPORTED;
  stamp_fp8_plan* p = new (std::nothrow) stamp_fp8_plan;
  if (p == nullptr) return STAMP_ERR_ALLOC;
  p->desc = *desc;
  p->sets = desc->experts > 0 ? desc->experts : 1;
  p->Kb = (desc->d_in + kF8Block - 1) / kF8Block;
  p->Kp = p->Kb * kF8Block;
  const int per_group = desc->gated ? kF8Group / 2 : kF8Group;
  p->groups = (desc->d_out + per_group - 1) / per_group;
  p->nblk = (desc->d_out + kF8Block - 1) / kF8Block;
  p->forced = 0;
  p->w_dev = nullptr;
  p->sw_dev = p->bias_dev = nullptr;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  const size_t image = (size_t)p->sets * p->groups * p->Kb * kF8GroupBytes;
  const size_t nscales = (size_t)p->sets * (desc->gated ? 2 : 1) * p->nblk * p->Kb, nbias = (size_t)p->sets * desc->d_out;
  const bool look = desc->w_dtype == STAMP_E4M3 && desc->scale_format == STAMP_SCALE_POW2;
  uint32_t* flag = nullptr;
  bool ok = hipMalloc(reinterpret_cast<void**>(&p->w_dev), image) == hipSuccess &&
            hipMalloc(reinterpret_cast<void**>(&p->sw_dev), nscales * sizeof(float)) == hipSuccess;
  if (ok && bias_dev != nullptr) ok = hipMalloc(reinterpret_cast<void**>(&p->bias_dev), nbias * sizeof(float)) == hipSuccess;
  if (ok && look) ok = hipMalloc(reinterpret_cast<void**>(&flag), sizeof(uint32_t)) == hipSuccess;
  if (!ok) {
    (void)hipGetLastError();
    (void)stamp_fp8_plan_destroy(p);
    return STAMP_ERR_ALLOC;
  }
  uint32_t found = 0;
  if (look) ok = hipMemcpyAsync(flag, &found, sizeof(found), hipMemcpyHostToDevice, st) == hipSuccess;
  if (ok) ok = stamp_launch_f8_weights(p, W_dev, w_scales_dev, st, flag) == hipSuccess;
  if (ok && bias_dev != nullptr) ok = hipMemcpyAsync(p->bias_dev, bias_dev, nbias * sizeof(float), hipMemcpyDeviceToDevice, st) == hipSuccess;
  if (ok && look) ok = hipMemcpyAsync(&found, flag, sizeof(found), hipMemcpyDeviceToHost, st) == hipSuccess && hipStreamSynchronize(st) == hipSuccess;
  if (flag != nullptr) (void)hipFree(flag);
  if (!ok || found != 0) {
    (void)hipStreamSynchronize(st);
    (void)hipGetLastError();
    (void)stamp_fp8_plan_destroy(p);
    return ok ? STAMP_ERR_UNSUPPORTED : STAMP_ERR_DEVICE;
  }
  *out = p;
  return STAMP_OK;
}

stamp_status_t stamp_fp8_plan_destroy(stamp_fp8_plan_t* p) {
  if (p == nullptr) return STAMP_ERR_NULL;
  if (p->w_dev) (void)hipFree(p->w_dev);
  if (p->sw_dev) (void)hipFree(p->sw_dev);
  if (p->bias_dev) (void)hipFree(p->bias_dev);
  delete p;
  return STAMP_OK;
}

size_t stamp_fp8_workspace_bytes(const stamp_fp8_plan_t* p, int32_t rows) {
  if (p == nullptr || rows < 0 || rows > kMaxRows) return 0;
  return linear_ws(p, rows).total;
}

stamp_status_t stamp_fp8_quantize_act(const stamp_fp8_plan_t* p, int32_t rows, const void* X_dev, int64_t ld_x, uint8_t* codes_dev, float* scales_dev,
                                      int64_t ld_scales, void* hip_stream) {
  if (p == nullptr) return STAMP_ERR_NULL;
  if (rows < 0 || rows > kMaxRows) return STAMP_ERR_SHAPE;
  if (rows == 0) return STAMP_OK;
  const stamp_status_t s = check_matrix(X_dev, p->desc.x_dtype, ld_x, p->desc.d_in);
  if (s != STAMP_OK) return s;
  if (codes_dev == nullptr || scales_dev == nullptr) return STAMP_ERR_NULL;
  if (ld_scales < rows || ld_scales % 4 != 0 || (reinterpret_cast<uintptr_t>(codes_dev) | reinterpret_cast<uintptr_t>(scales_dev)) % 16 != 0) return STAMP_ERR_SHAPE;
  return done(stamp_launch_f8_quant(X_dev, p->desc.x_dtype == STAMP_BF16, ld_x, rows, p->desc.d_in, p->desc.scale_format == STAMP_SCALE_POW2, 0, codes_dev,
                                    scales_dev, ld_scales, reinterpret_cast<hipStream_t>(hip_stream)));
}

stamp_status_t stamp_fp8_linear_forward(const stamp_fp8_plan_t* p, int32_t rows, const void* X_dev, int64_t ld_x, void* Y_dev, int64_t ld_y,
                                        void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  return forward(p, rows, nullptr, false, X_dev, ld_x, Y_dev, ld_y, workspace_dev, workspace_bytes, reinterpret_cast<hipStream_t>(hip_stream));
}

stamp_status_t stamp_fp8_linear_forward_q(const stamp_fp8_plan_t* p, int32_t rows, const uint8_t* codes_dev, const float* scales_dev, int64_t ld_scales,
                                          void* Y_dev, int64_t ld_y, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  if (p == nullptr) return STAMP_ERR_NULL;
  if (p->desc.experts > 0) return STAMP_ERR_UNSUPPORTED;
  if (rows < 0 || rows > kMaxRows) return STAMP_ERR_SHAPE;
  if (rows == 0) return STAMP_OK;
  if (codes_dev == nullptr || scales_dev == nullptr) return STAMP_ERR_NULL;
  if (ld_scales < rows || ld_scales % 4 != 0 || (reinterpret_cast<uintptr_t>(codes_dev) | reinterpret_cast<uintptr_t>(scales_dev)) % 16 != 0) return STAMP_ERR_SHAPE;
  stamp_status_t s = check_matrix(Y_dev, p->desc.y_dtype, ld_y, p->desc.d_out);
  if (s == STAMP_OK) s = check_ws(workspace_dev, workspace_bytes, linear_ws(p, rows).total);
  if (s != STAMP_OK) return s;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  StampF8Gemm a = gemm_args(p);
  a.partial = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace_dev) + linear_ws(p, rows).partial);
  a.A = codes_dev;
  if (wide_codes(a, rows)) {
    uint8_t* wide = static_cast<uint8_t*>(workspace_dev);
    if (stamp_launch_f8_widen(codes_dev, (int64_t)rows * p->Kp, wide, st) != hipSuccess) return STAMP_ERR_DEVICE;
    a.A = wide;
  }
  a.SA = scales_dev;
  a.ld_sa = ld_scales;
  a.a_rows = a.rows = rows;
  a.Y = Y_dev;
  a.ld_y = ld_y;
  return done(product(a, st));
}

stamp_status_t stamp_fp8_grouped_forward(const stamp_fp8_plan_t* p, int32_t rows, const int32_t* offsets_dev, const void* X_dev, int64_t ld_x, void* Y_dev,
                                         int64_t ld_y, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  return forward(p, rows, offsets_dev, true, X_dev, ld_x, Y_dev, ld_y, workspace_dev, workspace_bytes, reinterpret_cast<hipStream_t>(hip_stream));
}

size_t stamp_route_workspace_bytes(int32_t tokens, int32_t experts, int32_t top_k) {
  if (tokens < 0 || tokens > (1 << 22) || experts < 1 || experts > kF8MaxExperts || top_k < 1 || top_k > 32) return 0;
  return stamp_route_ws(tokens, experts, top_k);
}

stamp_status_t stamp_route_topk(const stamp_routing_t* r, const void* logits_dev, int32_t logits_dtype, int64_t ld, int32_t renormalize, void* workspace_dev,
                                size_t workspace_bytes, void* hip_stream) {
  if (r == nullptr) return STAMP_ERR_NULL;
  stamp_status_t s = check_routing(r);
  if (s != STAMP_OK) return s;
  if (!is_float_type(logits_dtype) || renormalize < 0 || renormalize > 1) return STAMP_ERR_SHAPE;
  if (r->tokens > 0) s = check_matrix(logits_dev, logits_dtype, ld, r->experts);
  if (s == STAMP_OK) s = check_ws(workspace_dev, workspace_bytes, stamp_route_ws(r->tokens, r->experts, r->top_k));
  if (s != STAMP_OK) return s;
  return done(stamp_launch_route(*r, logits_dev, logits_dtype == STAMP_BF16, ld, renormalize, workspace_dev, reinterpret_cast<hipStream_t>(hip_stream)));
}

size_t stamp_experts_workspace_bytes(const stamp_fp8_plan_t* up, const stamp_fp8_plan_t* down, int32_t tokens, int32_t top_k) {
  if (up == nullptr || down == nullptr || tokens < 0 || top_k < 1 || (int64_t)tokens * top_k > kMaxRows) return 0;
  return experts_ws(up, down, tokens, top_k).total;
}

stamp_status_t stamp_experts_forward(const stamp_fp8_plan_t* up, const stamp_fp8_plan_t* down, const stamp_routing_t* r, const void* X_dev, int64_t ld_x,
                                     void* Y_dev, int64_t ld_y, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  if (up == nullptr || down == nullptr || r == nullptr) return STAMP_ERR_NULL;
  if (!up->desc.gated || down->desc.gated || down->desc.experts == 0) return STAMP_ERR_UNSUPPORTED;
  if (up->desc.experts != down->desc.experts || up->desc.d_out != down->desc.d_in || up->desc.d_in != down->desc.d_out ||
      up->desc.scale_format != down->desc.scale_format || r->experts != up->desc.experts)
    return STAMP_ERR_SHAPE;
  stamp_status_t s = check_routing(r);
  if (s != STAMP_OK) return s;
  if ((int64_t)r->tokens * r->top_k > kMaxRows || (int64_t)r->tokens * up->Kp * 2 >= (int64_t)0xfffffff0u) return STAMP_ERR_UNSUPPORTED;
  if (r->tokens == 0) return STAMP_OK;
  s = check_matrix(X_dev, up->desc.x_dtype, ld_x, up->desc.d_in);
  if (s == STAMP_OK) s = check_matrix(Y_dev, down->desc.y_dtype, ld_y, down->desc.d_out);
  const ExpertsWs w = experts_ws(up, down, r->tokens, r->top_k);
  if (s == STAMP_OK) s = check_ws(workspace_dev, workspace_bytes, w.total);
  if (s != STAMP_OK) return s;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  uint8_t* ws = static_cast<uint8_t*>(workspace_dev);
  const int32_t slots = r->tokens * r->top_k;
  const int64_t ld = scales_ld(slots);

  StampF8Gemm a = gemm_args(up);
  float* scales = reinterpret_cast<float*>(ws + w.scales);
  if (takes_x(a, slots)) {
    give_x(&a, up->desc, slots, X_dev, ld_x);
  } else if (stamp_launch_f8_quant(X_dev, up->desc.x_dtype == STAMP_BF16, ld_x, r->tokens, up->desc.d_in, a.pow2, wide_codes(a, slots), ws + w.codes, scales,
                                   scales_ld(r->tokens), st) != hipSuccess) {
    return STAMP_ERR_DEVICE;
  }
  a.A = ws + w.codes;
  a.SA = scales;
  a.ld_sa = scales_ld(r->tokens);
  a.index = r->token_of_row_dev;
  a.a_rows = r->tokens;
  a.rows = slots;
  a.offsets = r->offsets_dev;
  a.Y = ws + w.h;
  a.ld_y = down->Kp;
  a.SH = reinterpret_cast<float*>(ws + w.sh);
  a.ld_sh = ld;
  if (product(a, st) != hipSuccess) return STAMP_ERR_DEVICE;

  StampF8Gemm b = gemm_args(down);
  b.partial = reinterpret_cast<float*>(ws + w.partial);
  b.A = ws + w.h;
  if (wide_codes(b, slots)) {
    if (stamp_launch_f8_widen(b.A, (int64_t)slots * down->Kp, ws + w.wide, st) != hipSuccess) return STAMP_ERR_DEVICE;
    b.A = ws + w.wide;
  }
  b.SA = a.SH;
  b.ld_sa = ld;
  b.a_rows = b.rows = slots;
  b.offsets = r->offsets_dev;
  b.Y = ws + w.rows;
  b.ld_y = w.ld_rows;
  if (product(b, st) != hipSuccess) return STAMP_ERR_DEVICE;
  return done(stamp_launch_combine(*r, b.Y, b.y_bf16, w.ld_rows, slots, Y_dev, ld_y, down->desc.d_out, st));
}

stamp_status_t stamp_fp8_debug_weight_codes(const stamp_fp8_plan_t* p, uint8_t* codes_host, float* scales_host) {
  if (p == nullptr || codes_host == nullptr || scales_host == nullptr) return STAMP_ERR_NULL;
  const stamp_fp8_desc_t& d = p->desc;
  const size_t image = (size_t)p->sets * p->groups * p->Kb * kF8GroupBytes;
  uint8_t* h = static_cast<uint8_t*>(malloc(image));
  if (h == nullptr) return STAMP_ERR_ALLOC;
  if (hipDeviceSynchronize() != hipSuccess || hipMemcpy(h, p->w_dev, image, hipMemcpyDeviceToHost) != hipSuccess ||
      hipMemcpy(scales_host, p->sw_dev, (size_t)p->sets * (d.gated ? 2 : 1) * p->nblk * p->Kb * sizeof(float), hipMemcpyDeviceToHost) != hipSuccess) {
    free(h);
    return STAMP_ERR_DEVICE;
  }
  for (int set = 0; set < p->sets; ++set)
    for (int g = 0; g < p->groups; ++g)
      for (int b = 0; b < 4; ++b)
        for (int i = 0; i < 16; ++i) {
          const int n = f8_column(d.gated, g, b, i);
          if (n >= d.d_out) continue;
          const size_t mat = d.gated ? 2 * (size_t)set + (b & 1) : (size_t)set;
          uint8_t* row = codes_host + (mat * d.d_out + n) * d.d_in;
          for (int c = 0; c < d.d_in; c += 16) {
            const uint8_t* s = h + f8_w_offset(p->groups, p->Kb, set, g, c >> 7, b, (c >> 6) & 1, 16 * ((c >> 4) & 3) + i);
            memcpy(row + c, s, d.d_in - c < 16 ? d.d_in - c : 16);
          }
        }
  free(h);
  return STAMP_OK;
}

int32_t stamp_fp8_debug_route(const stamp_fp8_plan_t* p, int32_t rows) {
  if (p == nullptr || rows < 0) return 0;
  return route_of(gemm_args(p), rows);
}

stamp_status_t stamp_fp8_debug_cut(const stamp_fp8_plan_t* p, int32_t rows, int32_t* cut_host) {
  if (p == nullptr || cut_host == nullptr) return STAMP_ERR_NULL;
  if (rows < 0 || rows > kMaxRows) return STAMP_ERR_SHAPE;
  const StampF8Gemm a = gemm_args(p);
  cut_host[0] = cut_host[1] = cut_host[2] = 0;
  if (route_of(a, rows) == STAMP_FP8_ROUTE_ROWS) return STAMP_OK;
  const F8Cut cut = stamp_f8_cut(a.sets, a.groups, a.Kb, rows, a.wide_sums, a.gated, a.forced);
  cut_host[0] = cut.groups * kF8Group;
  cut_host[1] = cut.parts;
  cut_host[2] = cut.groups > 0 ? cut.rest_parts : 0;
  return STAMP_OK;
}

stamp_status_t stamp_fp8_debug_set_route(stamp_fp8_plan_t* p, int32_t route) {
  if (p == nullptr) return STAMP_ERR_NULL;
  if (route < 0 || route > STAMP_FP8_ROUTE_TILES_256) return STAMP_ERR_SHAPE;
  if (route == STAMP_FP8_ROUTE_TILES_256 && gemm_args(p).wide_sums) return STAMP_ERR_UNSUPPORTED;
  p->forced = route;
  return STAMP_OK;
}

}  // extern "C"
