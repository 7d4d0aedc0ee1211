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
  a.act = p->desc.gated ? kF8DividedSilu : STAMP_ACT_NONE;
  a.wide_sums = f8_wide_sums(a);
  a.forced = p->forced;
  return a;
}

// products whose results become codes have their depth in one piece
bool in_one(const StampF8Gemm& a) { return a.gated || a.codes; }
int route_of(const StampF8Gemm& a, int rows) { return stamp_f8_route(a.sets, a.groups, a.Kb, rows, a.wide_sums, in_one(a), a.forced); }
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
  const F8Cut cut = stamp_f8_cut(a.sets, a.groups, a.Kb, a.rows, a.wide_sums, in_one(a), a.forced);
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
  if (a.R != nullptr) rest.R = static_cast<const char*>(a.R) + (size_t)columns * (a.y_bf16 ? 2 : 4);
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
  size_t codes, scales, h, sh, rows, partial, total;
  int64_t ld_rows;
};
ExpertsWs experts_ws(const stamp_fp8_plan* up, const stamp_fp8_plan* down, int32_t tokens, int32_t top_k, bool wide_rows = false) {
  ExpertsWs w;
  const int64_t slots = (int64_t)tokens * top_k, ld = scales_ld((int32_t)slots);
  w.codes = 0;
  w.scales = align256((size_t)tokens * up->Kp * code_bytes(up));
  w.h = w.scales + align256((size_t)up->Kb * scales_ld(tokens) * sizeof(float));
  w.sh = w.h + align256((size_t)slots * down->Kp * code_bytes(down));
  w.rows = w.sh + align256((size_t)down->Kb * ld * sizeof(float));
  w.ld_rows = (down->desc.d_out + 7) / 8 * 8;
  // Rows in Y's type: a bf16 Y is a sum of terms rounded once each, 2.3e-3 off where rows in fp32 give 1.7e-3, which is Y's own rounding; but
  // they are the most bytes of the call (8192 tokens, 8 of 64 experts, 4096 -> 1536: down product 529 -> 647 us, weighted sum 122 -> 242, the whole
  // 2200 -> 2447).  An fp32 Y has them in fp32.
  w.partial = w.rows + align256((size_t)slots * w.ld_rows * (wide_rows ? 4 : type_size(down->desc.y_dtype)));
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

// nullptr: no epilogue.  in_place: X may be Y (it is not read any more where Y is written).
stamp_status_t check_epilogue(const stamp_epilogue_t* e, int32_t rows, int32_t y_dtype, int32_t d_out, const void* Y, int64_t ld_y, const void* X, bool in_place) {
  if (e == nullptr) return STAMP_OK;
  if (e->activation < STAMP_ACT_NONE || e->activation > STAMP_ACT_GELU_TANH) return STAMP_ERR_SHAPE;
  if (!in_place && X != nullptr && X == Y) return STAMP_ERR_SHAPE;
  if (e->residual_dev == nullptr) return STAMP_OK;
  const stamp_status_t s = check_matrix(e->residual_dev, y_dtype, e->ld_residual, d_out);
  if (s != STAMP_OK) return s;
  return e->residual_dev == Y && rows > 1 && e->ld_residual != ld_y ? STAMP_ERR_SHAPE : STAMP_OK;
}
void give_epilogue(StampF8Gemm* a, const stamp_epilogue_t* e) {
  if (e == nullptr) return;
  a->act = e->activation;
  a->R = e->residual_dev;
  a->ld_r = e->ld_residual;
}

// linear_forward, grouped_forward
stamp_status_t forward(const stamp_fp8_plan* p, int32_t rows, const int32_t* offsets, bool grouped, const void* X, int64_t ld_x, const stamp_epilogue_t* ep,
                       void* Y, int64_t ld_y, void* ws, size_t ws_bytes, hipStream_t st) {
  if (p == nullptr) return STAMP_ERR_NULL;
  if (p->desc.gated || (p->desc.experts > 0) != grouped) return STAMP_ERR_UNSUPPORTED;
  if (rows < 0 || rows > kMaxRows) return STAMP_ERR_SHAPE;
  if (grouped && offsets == nullptr) return STAMP_ERR_NULL;
  if (rows == 0) return STAMP_OK;
  stamp_status_t s = check_matrix(X, p->desc.x_dtype, ld_x, p->desc.d_in);
  if (s == STAMP_OK) s = check_matrix(Y, p->desc.y_dtype, ld_y, p->desc.d_out);
  if (s == STAMP_OK) s = check_epilogue(ep, rows, p->desc.y_dtype, p->desc.d_out, Y, ld_y, X, false);
  const LinearWs w = linear_ws(p, rows);
  if (s == STAMP_OK) s = check_ws(ws, ws_bytes, w.total);
  if (s != STAMP_OK) return s;
  uint8_t* codes = static_cast<uint8_t*>(ws) + w.codes;
  float* scales = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + w.scales);
  StampF8Gemm a = gemm_args(p);
  give_epilogue(&a, ep);
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

stamp_status_t forward_q(const stamp_fp8_plan* p, int32_t rows, const uint8_t* codes, const float* scales, int64_t ld_scales, const stamp_epilogue_t* ep,
                         void* Y, int64_t ld_y, void* ws, size_t ws_bytes, hipStream_t st) {
  if (p == nullptr) return STAMP_ERR_NULL;
  if (p->desc.experts > 0) return STAMP_ERR_UNSUPPORTED;
  if (rows < 0 || rows > kMaxRows) return STAMP_ERR_SHAPE;
  if (rows == 0) return STAMP_OK;
  if (codes == nullptr || scales == nullptr) return STAMP_ERR_NULL;
  if (ld_scales < rows || ld_scales % 4 != 0 || (reinterpret_cast<uintptr_t>(codes) | reinterpret_cast<uintptr_t>(scales)) % 16 != 0) return STAMP_ERR_SHAPE;
  stamp_status_t s = check_matrix(Y, p->desc.y_dtype, ld_y, p->desc.d_out);
  if (s == STAMP_OK) s = check_epilogue(ep, rows, p->desc.y_dtype, p->desc.d_out, Y, ld_y, nullptr, true);
  const LinearWs w = linear_ws(p, rows);
  if (s == STAMP_OK) s = check_ws(ws, ws_bytes, w.total);
  if (s != STAMP_OK) return s;
  StampF8Gemm a = gemm_args(p);
  give_epilogue(&a, ep);
  a.partial = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + w.partial);
  a.A = codes;
  if (wide_codes(a, rows)) {
    uint8_t* wide = static_cast<uint8_t*>(ws);
    if (stamp_launch_f8_widen(codes, (int64_t)rows * p->Kp, wide, st) != hipSuccess) return STAMP_ERR_DEVICE;
    a.A = wide;
  }
  a.SA = scales;
  a.ld_sa = ld_scales;
  a.a_rows = a.rows = rows;
  a.Y = Y;
  a.ld_y = ld_y;
  return done(product(a, st));
}

// Places of the experts' MLP: the up product's rows of X, its results as codes, the rows behind the down product.
struct ExpertsRun {
  const stamp_fp8_plan *up, *down;
  const stamp_routing_t* r;
  const void* X;
  int64_t ld_x;
  stamp_epilogue_t ep;
  void* Y;
  int64_t ld_y;
  bool wide_rows;  // the rows behind the down product in fp32 whatever Y's type
  bool coded;      // Q8 of X is there, where run_experts would put it
};
stamp_status_t check_experts(const ExpertsRun& e) {
  const stamp_fp8_plan *up = e.up, *down = e.down;
  if (!up->desc.gated || down->desc.gated || down->desc.experts == 0) return STAMP_ERR_UNSUPPORTED;
  if (up->desc.experts != down->desc.experts || up->desc.d_out != down->desc.d_in || up->desc.d_in != down->desc.d_out ||
      up->desc.scale_format != down->desc.scale_format || e.r->experts != up->desc.experts)
    return STAMP_ERR_SHAPE;
  const stamp_status_t s = check_routing(e.r);
  if (s != STAMP_OK) return s;
  if ((int64_t)e.r->tokens * e.r->top_k > kMaxRows || (int64_t)e.r->tokens * up->Kp * 2 >= (int64_t)0xfffffff0u) return STAMP_ERR_UNSUPPORTED;
  return STAMP_OK;
}
stamp_status_t check_experts_rows(const ExpertsRun& e) {
  const stamp_status_t s = check_matrix(e.X, e.up->desc.x_dtype, e.ld_x, e.up->desc.d_in);
  return s == STAMP_OK ? check_matrix(e.Y, e.down->desc.y_dtype, e.ld_y, e.down->desc.d_out) : s;
}
// up product, down product, weighted sum, for a routing that is there
stamp_status_t run_experts(const ExpertsRun& e, uint8_t* ws, hipStream_t st) {
  const stamp_fp8_plan *up = e.up, *down = e.down;
  const stamp_routing_t* r = e.r;
  const ExpertsWs w = experts_ws(up, down, r->tokens, r->top_k, e.wide_rows);
  const int32_t slots = r->tokens * r->top_k;
  const int64_t ld = scales_ld(slots);

  StampF8Gemm a = gemm_args(up);
  a.act = e.ep.activation;
  float* scales = reinterpret_cast<float*>(ws + w.scales);
  if (takes_x(a, slots)) {
    give_x(&a, up->desc, slots, e.X, e.ld_x);
  } else if (!e.coded && stamp_launch_f8_quant(e.X, up->desc.x_dtype == STAMP_BF16, e.ld_x, r->tokens, up->desc.d_in, a.pow2, wide_codes(a, slots), ws + w.codes, scales,
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
  StampF8Gemm b = gemm_args(down);
  a.h_wide = wide_codes(b, slots);
  if (product(a, st) != hipSuccess) return STAMP_ERR_DEVICE;

  b.partial = reinterpret_cast<float*>(ws + w.partial);
  b.A = ws + w.h;
  b.SA = a.SH;
  b.ld_sa = ld;
  b.a_rows = b.rows = slots;
  b.offsets = r->offsets_dev;
  b.Y = ws + w.rows;
  b.ld_y = w.ld_rows;
  if (e.wide_rows) b.y_bf16 = 0;  // the instructions stay those of Y's type
  if (product(b, st) != hipSuccess) return STAMP_ERR_DEVICE;
  return done(stamp_launch_combine(*r, b.Y, b.y_bf16, down->desc.y_dtype == STAMP_BF16, w.ld_rows, slots, e.ep.residual_dev, e.ep.ld_residual, e.Y, e.ld_y, down->desc.d_out, st));
}

// The dense MLP's places: the rows of X as codes, h in fp32 or as codes, parts of the depth.
struct MlpWs {
  size_t codes, scales, h, hcodes, hscales, partial, total;
};
// Up to so many rows h may lie in fp32: beyond, codes straight from the tiles are as fast or faster (stamp_f8_codes_pay).  Of a gated layer up to 16 rows; us, rows in fp32 by
// workgroups of 32 places / codes by workgroups of 256:
//                               1 row         2            4            6            8            12           16
//   4096 -> 11008 -> 4096         34 / 47       36 / 48      39 / 49      37 / 44      38 / 45      40 / 47      42 / 50
//   2048 -> 5632 -> 2048          17 / 26       18 / 27      20 / 27      22 / 25      23 / 25      24 / 27      26 / 28
//   1024 -> 2816 -> 1024          10 / 16       11 / 17      11 / 18      17 / 16      17 / 16      17 / 18      17 / 18
//   8192 -> 28672 -> 8192         133 / 148     135 / 149    131 / 150    130 / 127    130 / 127    133 / 127    149 / 149
constexpr int32_t kMlpRowsInFp32 = 1024, kMlpGatedRows = 16;
MlpWs mlp_ws(const stamp_fp8_plan* up, const stamp_fp8_plan* down, int32_t rows) {
  MlpWs w;
  w.codes = 0;
  w.scales = align256((size_t)rows * up->Kp * 2);  // bf16 codes: h is a sum in fp32
  w.h = w.scales + align256((size_t)up->Kb * scales_ld(rows) * sizeof(float));
  const int32_t most = up->desc.gated ? kMlpGatedRows : kMlpRowsInFp32;
  w.hcodes = w.h + align256((size_t)(rows < most ? rows : most) * up->desc.d_out * sizeof(float));
  w.hscales = w.hcodes + align256((size_t)rows * down->Kp * code_bytes(down));
  w.partial = w.hscales + align256((size_t)down->Kb * scales_ld(rows) * sizeof(float));
  const size_t pu = up->desc.gated ? 0 : stamp_f8_partial_bytes(up->groups, rows), pd = stamp_f8_partial_bytes(down->groups, rows);
  w.total = w.partial + align256(pu > pd ? pu : pd);
  return w;
}
stamp_status_t check_mlp(const stamp_fp8_plan* up, const stamp_fp8_plan* down) {
  if (up == nullptr || down == nullptr) return STAMP_ERR_NULL;
  if (down->desc.gated || up->desc.experts != (up->desc.gated ? 1 : 0) || down->desc.experts > up->desc.experts) return STAMP_ERR_UNSUPPORTED;
  if (up->desc.d_out != down->desc.d_in || up->desc.scale_format != down->desc.scale_format) return STAMP_ERR_SHAPE;
  return STAMP_OK;
}

// h straight to codes, in tiles, or in fp32 and by the quantizer: see stamp_f8_codes_pay
bool mlp_codes_in_tiles(const StampF8Gemm& up, const StampF8Gemm& down, int rows) {
  if (rows > kMlpRowsInFp32) return true;
  if (up.forced != 0) return up.forced != STAMP_FP8_ROUTE_ROWS;
  return stamp_f8_codes_pay(up.groups, up.Kb, rows, takes_x(down, rows));
}

struct MlpProducts {
  StampF8Gemm up, down;
  bool coded;  // the up product's results are codes, else rows in fp32
};
MlpProducts mlp_products(const stamp_fp8_plan* up, const stamp_fp8_plan* down, int32_t rows) {
  MlpProducts p = {gemm_args(up), gemm_args(down), false};
  StampF8Gemm& a = p.up;
  a.y_bf16 = 0;
  a.wide_sums = f8_wide_sums(a);
  if (a.forced == STAMP_FP8_ROUTE_TILES_256) a.forced = 0;
  a.codes = !a.gated && mlp_codes_in_tiles(a, p.down, rows);
  if (a.codes && a.forced <= STAMP_FP8_ROUTE_ROWS) a.forced = stamp_f8_codes_route(a.groups, a.Kb, rows);
  a.h_rows = a.gated && rows <= kMlpGatedRows && route_of(a, rows) == STAMP_FP8_ROUTE_ROWS;
  p.coded = (a.gated || a.codes) && !a.h_rows;
  return p;
}

// The layer of experts' places: logits and the router's, then those of the experts.
struct MoeWs {
  size_t logits, sync, h, sums, route, experts, total;
};
bool moe_few(const stamp_fp8_plan* up, const stamp_fp8_plan* down, int32_t tokens, int32_t top_k) {
  return stamp_moe_fits(tokens, top_k, down->Kb) && up->forced == 0 && down->forced == 0;  // a plan's forced kernel is one of the others
}
MoeWs moe_ws(const stamp_fp8_plan* up, const stamp_fp8_plan* down, int32_t tokens, int32_t top_k) {
  MoeWs w;
  w.logits = 0;
  w.sync = align256((size_t)tokens * up->desc.experts * sizeof(float));
  // for the two kernels of few tokens: h in fp32, parts of Y
  w.h = w.sync + align256(stamp_moe_sync_bytes(down->groups));
  const int few = tokens < kMoeTokens ? tokens : kMoeTokens, slots = few * top_k;
  w.sums = w.h + align256((size_t)(slots < kMoeSlots ? slots : kMoeSlots) * down->Kp * sizeof(float));
  w.route = w.sums + align256((size_t)stamp_moe_parts(down->groups) * few * down->groups * 64 * sizeof(float));
  w.experts = w.route + align256(stamp_route_ws(tokens, up->desc.experts, top_k));
  w.total = w.experts + experts_ws(up, down, tokens, top_k, true).total;
  return w;
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

// An up product of tiles whose results become codes has its depth in one piece; with rows in fp32 it may have parts or be the rows kernel's, but they
// are written and, unless the down product does it (few rows), quantized by a launch of 3.5 us: 4 + 4 + 1 bytes for 1.
// us, rows in fp32 / codes, bf16 Y, the first the choice up to the bar, the second behind it:
//   rows                         1           16          32          64          100           200           400           1024
//   1152 -> 4608 -> 1152         13 / 21     25 / 24     21 / 25     29 / 30  |  34 / 32       37 / 34       41 / 37       63 / 55
//   4096 -> 11008 -> 4096        28 / 52     35 / 57     47 / 63     54 / 67     60 / 66  |    73 / 69       104 / 99      175 / 175
//   590 -> 1185 -> 590           11 / 18     18 / 21     16 / 20  |  20 / 23     28 / 26       28 / 26       29 / 26       33 / 27
// Over 88 sizes the choice takes 1 % more than the better one on average, 16 % at worst (64 rows).
int stamp_f8_codes_route(int groups, int Kb, int rows) { return STAMP_FP8_ROUTE_TILES_64 + best_tiles(1, groups, Kb, rows, 1, 1, 0).size; }
int stamp_f8_codes_pay(int groups, int Kb, int rows, int quantized_below) {
  const float codes = best_tiles(1, groups, Kb, rows, 1, 1, 0).us;
  const float tiles = best_tiles(1, groups, Kb, rows, 1, 0, 0).us, few = rows_us(1, groups, Kb, rows), elements = (float)rows * groups * 64;
  return codes < (tiles < few ? tiles : few) + (quantized_below ? 0.0f : 3.5f + elements * 8.0f / kBytesPerUs);
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
  p->looks = -1;
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
  return forward(p, rows, nullptr, false, X_dev, ld_x, nullptr, Y_dev, ld_y, workspace_dev, workspace_bytes, reinterpret_cast<hipStream_t>(hip_stream));
}
stamp_status_t stamp_fp8_linear_forward_act(const stamp_fp8_plan_t* p, int32_t rows, const void* X_dev, int64_t ld_x, const stamp_epilogue_t* epilogue,
                                            void* Y_dev, int64_t ld_y, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  if (epilogue == nullptr) return STAMP_ERR_NULL;
  return forward(p, rows, nullptr, false, X_dev, ld_x, epilogue, Y_dev, ld_y, workspace_dev, workspace_bytes, reinterpret_cast<hipStream_t>(hip_stream));
}

stamp_status_t stamp_fp8_linear_forward_q(const stamp_fp8_plan_t* p, int32_t rows, const uint8_t* codes_dev, const float* scales_dev, int64_t ld_scales,
                                          void* Y_dev, int64_t ld_y, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  return forward_q(p, rows, codes_dev, scales_dev, ld_scales, nullptr, Y_dev, ld_y, workspace_dev, workspace_bytes, reinterpret_cast<hipStream_t>(hip_stream));
}
stamp_status_t stamp_fp8_linear_forward_q_act(const stamp_fp8_plan_t* p, int32_t rows, const uint8_t* codes_dev, const float* scales_dev, int64_t ld_scales,
                                              const stamp_epilogue_t* epilogue, void* Y_dev, int64_t ld_y, void* workspace_dev, size_t workspace_bytes,
                                              void* hip_stream) {
  if (epilogue == nullptr) return STAMP_ERR_NULL;
  return forward_q(p, rows, codes_dev, scales_dev, ld_scales, epilogue, Y_dev, ld_y, workspace_dev, workspace_bytes, reinterpret_cast<hipStream_t>(hip_stream));
}

stamp_status_t stamp_fp8_grouped_forward(const stamp_fp8_plan_t* p, int32_t rows, const int32_t* offsets_dev, const void* X_dev, int64_t ld_x, void* Y_dev,
                                         int64_t ld_y, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  return forward(p, rows, offsets_dev, true, X_dev, ld_x, nullptr, Y_dev, ld_y, workspace_dev, workspace_bytes, reinterpret_cast<hipStream_t>(hip_stream));
}
stamp_status_t stamp_fp8_grouped_forward_act(const stamp_fp8_plan_t* p, int32_t rows, const int32_t* offsets_dev, const void* X_dev, int64_t ld_x,
                                             const stamp_epilogue_t* epilogue, void* Y_dev, int64_t ld_y, void* workspace_dev, size_t workspace_bytes,
                                             void* hip_stream) {
  if (epilogue == nullptr) return STAMP_ERR_NULL;
  return forward(p, rows, offsets_dev, true, X_dev, ld_x, epilogue, Y_dev, ld_y, workspace_dev, workspace_bytes, reinterpret_cast<hipStream_t>(hip_stream));
}

size_t stamp_mlp_workspace_bytes(const stamp_fp8_plan_t* up, const stamp_fp8_plan_t* down, int32_t rows) {
  if (check_mlp(up, down) != STAMP_OK || rows < 0 || rows > kMaxRows) return 0;
  return mlp_ws(up, down, rows).total;
}

stamp_status_t stamp_mlp_forward(const stamp_fp8_plan_t* up, const stamp_fp8_plan_t* down, int32_t rows, const void* X_dev, int64_t ld_x,
                                 const stamp_epilogue_t* epilogue, void* Y_dev, int64_t ld_y, void* workspace_dev, size_t workspace_bytes,
                                 void* hip_stream) {
  if (epilogue == nullptr) return STAMP_ERR_NULL;
  stamp_status_t s = check_mlp(up, down);
  if (s != STAMP_OK) return s;
  if (rows < 0 || rows > kMaxRows) return STAMP_ERR_SHAPE;
  if (up->desc.gated && (int64_t)rows * up->Kp * 2 >= (int64_t)0xfffffff0u) return STAMP_ERR_UNSUPPORTED;
  if (rows == 0) return STAMP_OK;
  s = check_matrix(X_dev, up->desc.x_dtype, ld_x, up->desc.d_in);
  if (s == STAMP_OK) s = check_matrix(Y_dev, down->desc.y_dtype, ld_y, down->desc.d_out);
  if (s == STAMP_OK) s = check_epilogue(epilogue, rows, down->desc.y_dtype, down->desc.d_out, Y_dev, ld_y, X_dev, true);
  const MlpWs w = mlp_ws(up, down, rows);
  if (s == STAMP_OK) s = check_ws(workspace_dev, workspace_bytes, w.total);
  if (s != STAMP_OK) return s;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  uint8_t* ws = static_cast<uint8_t*>(workspace_dev);

  const MlpProducts products = mlp_products(up, down, rows);
  StampF8Gemm a = products.up, b = products.down;
  const bool coded = products.coded;
  a.act = epilogue->activation;
  b.R = epilogue->residual_dev;
  b.ld_r = epilogue->ld_residual;
  float* scales = reinterpret_cast<float*>(ws + w.scales);
  if (takes_x(a, rows)) {
    give_x(&a, up->desc, rows, X_dev, ld_x);
  } else if (stamp_launch_f8_quant(X_dev, up->desc.x_dtype == STAMP_BF16, ld_x, rows, up->desc.d_in, a.pow2, wide_codes(a, rows), ws + w.codes, scales,
                                   scales_ld(rows), st) != hipSuccess) {
    return STAMP_ERR_DEVICE;
  }
  a.A = ws + w.codes;
  a.SA = scales;
  a.ld_sa = scales_ld(rows);
  a.a_rows = a.rows = rows;
  a.partial = b.partial = reinterpret_cast<float*>(ws + w.partial);
  float* const hscales = reinterpret_cast<float*>(ws + w.hscales);
  if (coded) {
    a.Y = ws + w.hcodes;
    a.ld_y = down->Kp;
    a.SH = hscales;
    a.ld_sh = scales_ld(rows);
    a.h_wide = wide_codes(b, rows);
  } else {
    a.Y = ws + w.h;
    a.ld_y = up->desc.d_out;
  }
  if (product(a, st) != hipSuccess) return STAMP_ERR_DEVICE;
  if (!coded) {
    stamp_fp8_desc_t h = down->desc;
    h.x_dtype = STAMP_F32;
    if (takes_x(b, rows)) give_x(&b, h, rows, a.Y, a.ld_y);
    else if (stamp_launch_f8_quant(a.Y, 0, a.ld_y, rows, h.d_in, b.pow2, wide_codes(b, rows), ws + w.hcodes, hscales, scales_ld(rows), st) != hipSuccess)
      return STAMP_ERR_DEVICE;
  }
  b.A = ws + w.hcodes;
  b.SA = hscales;
  b.ld_sa = scales_ld(rows);
  b.a_rows = b.rows = rows;
  b.Y = Y_dev;
  b.ld_y = ld_y;
  return done(product(b, st));
}

stamp_status_t stamp_mlp_debug_route(const stamp_fp8_plan_t* up, const stamp_fp8_plan_t* down, int32_t rows, int32_t* route_host) {
  if (route_host == nullptr) return STAMP_ERR_NULL;
  const stamp_status_t s = check_mlp(up, down);
  if (s != STAMP_OK) return s;
  if (rows < 1 || rows > kMaxRows) return STAMP_ERR_SHAPE;
  const MlpProducts p = mlp_products(up, down, rows);
  route_host[0] = route_of(p.up, rows);
  route_host[1] = route_of(p.down, rows);
  route_host[2] = p.coded;
  return STAMP_OK;
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
  const ExpertsRun e = {up, down, r, X_dev, ld_x, {kF8DividedSilu, nullptr, 0}, Y_dev, ld_y, false, false};
  stamp_status_t s = check_experts(e);
  if (s != STAMP_OK) return s;
  if (r->tokens == 0) return STAMP_OK;
  s = check_experts_rows(e);
  if (s == STAMP_OK) s = check_ws(workspace_dev, workspace_bytes, experts_ws(up, down, r->tokens, r->top_k).total);
  if (s != STAMP_OK) return s;
  return run_experts(e, static_cast<uint8_t*>(workspace_dev), reinterpret_cast<hipStream_t>(hip_stream));
}

size_t stamp_moe_workspace_bytes(const stamp_fp8_plan_t* up, const stamp_fp8_plan_t* down, int32_t tokens, int32_t top_k) {
  if (up == nullptr || down == nullptr) return 0;
  int32_t some = 0;  // an address, for the checks
  const stamp_routing_t r = {tokens, up->desc.experts, top_k, &some, reinterpret_cast<float*>(&some), &some, &some, &some};
  const ExpertsRun e = {up, down, &r, nullptr, 0, {STAMP_ACT_SILU, nullptr, 0}, nullptr, 0, true, true};
  return check_experts(e) == STAMP_OK ? moe_ws(up, down, tokens, top_k).total : 0;
}

int32_t stamp_moe_debug_route(const stamp_fp8_plan_t* up, const stamp_fp8_plan_t* down, int32_t tokens, int32_t top_k) {
  return stamp_moe_workspace_bytes(up, down, tokens, top_k) > 0 && tokens > 0 && moe_few(up, down, tokens, top_k);
}

stamp_status_t stamp_moe_debug_set_looks(stamp_fp8_plan_t* up, int32_t looks) {
  if (up == nullptr) return STAMP_ERR_NULL;
  if (looks < -1) return STAMP_ERR_SHAPE;
  up->looks = looks;
  return STAMP_OK;
}

stamp_status_t stamp_moe_forward(const stamp_router_t* router, const stamp_fp8_plan_t* up, const stamp_fp8_plan_t* down, const stamp_routing_t* r,
                                 const void* X_dev, int64_t ld_x, const stamp_epilogue_t* epilogue, void* Y_dev, int64_t ld_y, void* workspace_dev,
                                 size_t workspace_bytes, void* hip_stream) {
  if (router == nullptr || up == nullptr || down == nullptr || r == nullptr || epilogue == nullptr) return STAMP_ERR_NULL;
  const ExpertsRun e = {up, down, r, X_dev, ld_x, *epilogue, Y_dev, ld_y, true, true};
  stamp_status_t s = check_experts(e);
  if (s != STAMP_OK) return s;
  if (!is_float_type(router->w_dtype) || router->renormalize < 0 || router->renormalize > 1) return STAMP_ERR_SHAPE;
  if (epilogue->activation < STAMP_ACT_NONE || epilogue->activation > STAMP_ACT_GELU_TANH) return STAMP_ERR_SHAPE;
  if (r->tokens > 0) {
    s = check_matrix(router->W_dev, router->w_dtype, up->desc.d_in, up->desc.d_in);
    if (s == STAMP_OK) s = check_experts_rows(e);
    if (s == STAMP_OK) s = check_epilogue(epilogue, r->tokens, down->desc.y_dtype, down->desc.d_out, Y_dev, ld_y, X_dev, true);
  }
  const MoeWs w = moe_ws(up, down, r->tokens, r->top_k);
  if (s == STAMP_OK) s = check_ws(workspace_dev, workspace_bytes, w.total);
  if (s != STAMP_OK) return s;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  uint8_t* ws = static_cast<uint8_t*>(workspace_dev);
  float* logits = reinterpret_cast<float*>(ws + w.logits);
  if (r->tokens > 0 && moe_few(up, down, r->tokens, r->top_k)) {
    // the places of the experts' rows serve here, too
    const ExpertsWs v = experts_ws(up, down, r->tokens, r->top_k, true);
    uint8_t* const rows = ws + w.experts;
    StampF8Gemm a = gemm_args(up), b = gemm_args(down);
    a.d = up->desc.d_in;
    a.act = epilogue->activation;
    a.ld_sa = scales_ld(r->tokens);
    a.Y = ws + w.h;
    a.ld_y = down->Kp;
    b.R = epilogue->residual_dev;
    b.ld_r = epilogue->ld_residual;
    b.Y = Y_dev;
    b.ld_y = ld_y;
    return done(stamp_launch_moe(*router, *r, X_dev, up->desc.x_dtype == STAMP_BF16, ld_x, a, b, rows + v.codes, reinterpret_cast<float*>(rows + v.scales), logits,
                                 reinterpret_cast<uint32_t*>(ws + w.sync), reinterpret_cast<float*>(ws + w.sums), up->looks, st));
  }
  if (r->tokens > 0) {
    const ExpertsWs v = experts_ws(up, down, r->tokens, r->top_k, true);
    StampF8Gemm a = gemm_args(up);
    const int slots = r->tokens * r->top_k;
    RouterQ8 q = {ws + w.experts + v.codes, reinterpret_cast<float*>(ws + w.experts + v.scales), scales_ld(r->tokens), a.pow2, wide_codes(a, slots), nullptr, 0};
    if (takes_x(a, slots)) q.codes = nullptr;
    if (stamp_launch_router(*router, X_dev, up->desc.x_dtype == STAMP_BF16, ld_x, r->tokens, r->experts, up->desc.d_in, q, logits, st) != hipSuccess)
      return STAMP_ERR_DEVICE;
  }
  if (stamp_launch_route(*r, logits, 0, r->experts, router->renormalize, ws + w.route, st) != hipSuccess) return STAMP_ERR_DEVICE;
  return r->tokens > 0 ? run_experts(e, ws + w.experts, st) : STAMP_OK;
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
