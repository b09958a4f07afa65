// Launch planning of a decoder's blocks: rotary positions, the norms around a residual sum, the gated
// half of a feed-forward block, attention (host only, no HIP calls).
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>
#include <cstring>
#include "opara_internal.h"

namespace opara {
namespace {

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
int fail(const char *what, const opara_op_desc &op) {
  set_error("operator type %d: %s", op.op_type, what);
  return OPARA_EINVAL;
}
int too_large(const char *what, const opara_op_desc &op) {
  set_error("operator type %d: %s", op.op_type, what);
  return OPARA_EUNSUPPORTED;
}
constexpr int64_t kInt = INT32_MAX;

int plan_rotary(const opara_op_desc &op, const opara_op_more &q, const void *const *in, KernelPlan *out) {
  const opara_op_params &p = op.params;
  const bool f16 = op.dtype == OPARA_F16;
  const int ve = f16 ? 8 : 4;
  if (op.n_inputs > 2 || !op.weight) return fail("rotary positions take one or two inputs and a table of frequencies", op);
  if (p.m <= 0 || q.heads <= 0 || q.width <= 0 || q.width > 4096 || q.rotated < 2 || q.rotated > q.width || q.rotated % 2)
    return fail("bad rotary shape", op);
  const int64_t cols = (int64_t)q.heads * q.width;
  if (cols > kInt) return fail("bad rotary shape", op);
  if ((p.a_row_stride != 0 && p.a_row_stride < cols) || (p.c_row_stride != 0 && p.c_row_stride < cols))
    return fail("row stride below heads * width", op);
  RotaryArgs a;
  std::memset(&a, 0, sizeof a);
  a.x = in[0]; a.y = op.out; a.turns = (const uint64_t *)op.weight;
  a.positions = op.n_inputs > 1 ? (const int32_t *)in[1] : nullptr;
  a.ldx = p.a_row_stride ? p.a_row_stride : cols;
  a.ldy = p.c_row_stride ? p.c_row_stride : cols;
  a.heads = q.heads; a.width = q.width; a.rotated = q.rotated; a.first = q.first;
  a.interleaved = (p.flags & OPARA_FLAG_INTERLEAVED) ? 1 : 0;
  a.rotated_units = (int32_t)cdiv(q.rotated / 2, ve);
  a.units = (int32_t)(a.interleaved ? cdiv(q.width, ve) : a.rotated_units + cdiv(q.width - q.rotated, ve));
  const int64_t items = (int64_t)p.m * a.units;
  if (items > kInt) return too_large("more rows than one launch holds", op);
  a.items = (uint32_t)items;
  a.div_units = div_magic(a.units);
  a.amplitude = p.alpha;
  a.heads_each = q.heads;
  const int64_t blocks = cdiv(items, 256);
  a.heads_each = (int32_t)std::max<int64_t>(1, std::min<int64_t>(8, blocks * q.heads / 1024));
  a.heads_each = (int32_t)std::max<int64_t>(a.heads_each, cdiv(q.heads, 65535));
  out->kernel = f16 ? K_rotary_f16 : K_rotary_f32;
  out->gx = (uint32_t)blocks; out->gy = (uint32_t)cdiv(q.heads, a.heads_each); out->gz = 1; out->block = 256;
  out->args.rotary = a;
  return OPARA_OK;
}

int plan_norm(const opara_op_desc &op, const opara_op_more &q, const void *const *in, KernelPlan *out) {
  const opara_op_params &p = op.params;
  const bool f16 = op.dtype == OPARA_F16;
  const int ve = f16 ? 8 : 4;
  if (op.n_inputs > 3) return fail("residual norm takes a block result, a residual and a gate", op);
  if (p.m <= 0 || p.n <= 0) return fail("bad residual norm shape", op);
  // A workgroup's row counter steps past the last row, by at most four rows of 1024 workgroups, in 32 bits.
  if (p.m > kInt - 4 * 1024) return too_large("more rows than a kernel counts", op);
  if (p.n > (1 << 30)) return too_large("more columns than a kernel counts", op);   // the weights of both norms are one row
  if (p.batch < 0 || (p.batch > 0 && p.m % p.batch)) return fail("rows must be a multiple of the gate's rows", op);
  if (op.n_inputs < 3 && p.batch > 0) return fail("gate rows without a gate", op);
  if (!(p.eps >= 0.f)) return fail("negative eps", op);
  const bool after = p.flags & OPARA_FLAG_NORM_AFTER, before = p.flags & OPARA_FLAG_NORM_BEFORE;
  if (q.out2 && !before) return fail("a second result goes with a norm of the sum", op);
  if (q.out2 && q.out2 == op.out) return fail("both results in one buffer", op);
  if ((op.weight || op.bias) && !after && !before) return fail("weights without a norm", op);
  NormArgs a;
  std::memset(&a, 0, sizeof a);
  a.x = in[0];
  a.r = op.n_inputs > 1 ? in[1] : nullptr;
  a.g = op.n_inputs > 2 ? in[2] : nullptr;
  a.w = op.weight; a.b = op.bias;
  a.y = before ? op.out : nullptr;
  a.s = before ? q.out2 : op.out;
  a.rows = p.m; a.cols = p.n;
  a.gate_rows = p.batch > 0 ? p.m / p.batch : 1;
  a.div_gate = div_magic(a.gate_rows);
  a.rms = (p.flags & OPARA_FLAG_RMS) ? 1 : 0;
  a.after = after; a.before = before;
  a.eps = p.eps; a.alpha = a.r ? p.alpha : 0.f; a.beta = q.beta;
  const bool vec = p.n % ve == 0 && aligned16(a.x) && aligned16(a.r) && aligned16(a.g) && aligned16(a.w) && aligned16(a.b) && aligned16(a.y) &&
                   aligned16(a.s);
  enum { kWave, kBlock, kLarge, kHuge, kOdd, kOddLarge, kWide };
  static const int ids[2][7] = {
      {K_resnorm_f32_wave, K_resnorm_f32_block, K_resnorm_f32_large, K_resnorm_f32_huge, K_resnorm_f32_odd, K_resnorm_f32_oddlarge, K_resnorm_f32_wide},
      {K_resnorm_f16_wave, K_resnorm_f16_block, K_resnorm_f16_large, K_resnorm_f16_huge, K_resnorm_f16_odd, K_resnorm_f16_oddlarge, K_resnorm_f16_wide}};
  int form = kWide;
  if (vec) form = p.n <= 64 * ve * kNormWavePieces ? kWave : p.n <= 256 * ve * kNormBlockPieces ? kBlock
                : p.n <= 256 * ve * kNormLargePieces ? kLarge : p.n <= 256 * ve * kNormHugePieces ? kHuge : kWide;
  else form = p.n <= 256 * kNormOddPieces ? kOdd : p.n <= 512 * kNormOddPieces ? kOddLarge : kWide;
  out->kernel = ids[f16][form];
  // Workgroups that the chip holds at once; with more rows than that a workgroup takes several.
  static const int64_t resident[7] = {1024, 1024, 512, 256, 1024, 1024, kInt};
  out->gx = (uint32_t)std::min(form == kWave ? cdiv(p.m, 4) : (int64_t)p.m, resident[form]);
  out->gy = out->gz = 1; out->block = 256;
  out->args.norm = a;
  return OPARA_OK;
}

// The forms of the gated block that are fed through workgroup memory, and what one workgroup costs in
// microseconds, in fp32 and in fp16: a 128-byte step of K with a compute unit to itself (`alone`) and in a full
// launch (`busy`), and everything outside the K walk (`fixed`).  Fitted to 115 products of each type (1..2048 rows,
// 256..4096 -> 512..12288, weights in no cache) within 12 %; the form it picks is 2 % slower than the best in the mean
// and 25 % at worst, most of all at 64 to 200 rows of the largest (192 rows of 4096 -> 12288 in fp32: 64 x 32 tiles
// 375 us, 32 x 32 ones 300; 128 rows in fp16: 128 x 64 tiles 68, 64 x 32 ones 58).
struct GatedCost { double alone, busy, fixed; };
struct GatedForm { int ids[2], rows, cols, threads; GatedCost cost[2]; };            // f32, f16
const GatedForm kGatedForms[] = {
    {{K_gated_f32_split16, K_gated_f16_split16}, 16, 16, 256, {{0.103, 0.091, 0.9}, {0.06, 0.066, 0.5}}},
    {{K_gated_f32_split32, K_gated_f16_split32}, 32, 32, 256, {{0.28, 0.29, 1.2}, {0.14, 0.14, 0.5}}},
    {{K_gated_f32_split64, K_gated_f16_split64}, 64, 32, 256, {{0.51, 0.52, 2.1}, {0.165, 0.21, 1.4}}},
    {{-1, K_gated_f16_tile64}, 64, 64, 256, {{0.0, 0.0, 0.0}, {0.56, 0.39, 0.45}}},
    {{K_gated_f32_tile128, K_gated_f16_tile128}, 128, 64, 256, {{2.03, 1.88, 5.0}, {0.66, 0.56, 2.0}}},
    {{-1, K_gated_f16_tile256}, 256, 128, 512, {{0.0, 0.0, 0.0}, {1.25, 1.83, 7.0}}},
};
double gated_cost(const GatedForm &f, double m, double n, double k, bool f16) {
  const double es = f16 ? 2.0 : 4.0, steps = std::ceil(k * es / 128.0), tiles = std::ceil(m / f.rows) * std::ceil(n / f.cols);
  const GatedCost &c = f.cost[f16];
  double work = tiles * (steps * c.busy + c.fixed) / 256.0;
  if (tiles > 256.0 && tiles < 1024.0) work *= std::ceil(tiles / 256.0) * 256.0 / tiles;     // whole rounds over the CUs
  const double bytes = (2.0 * n * k + m * k + m * n) * es / 5.8e6;                           // 5.8 TB/s
  return std::max({steps * c.alone + c.fixed, work, bytes});
}

int plan_gated(const opara_op_desc &op, const opara_op_more &q, const void *const *in, KernelPlan *out) {
  const opara_op_params &p = op.params;
  const bool f16 = op.dtype == OPARA_F16;
  if (op.n_inputs != 1 || !op.weight) return fail("the gated block takes one input and a weight", op);
  if (p.m <= 0 || p.n <= 0 || p.k <= 0 || p.n > kInt / 2) return fail("bad shape of a gated block", op);
  if (q.activation < 0 || q.activation >= OPARA_N_ACTIVATIONS) return fail("unknown activation", op);
  if ((p.a_row_stride != 0 && p.a_row_stride < p.k) || (p.c_row_stride != 0 && p.c_row_stride < p.n))
    return fail("row stride below the row", op);
  IgemmArgs a;
  std::memset(&a, 0, sizeof a);
  a.x = in[0]; a.w = op.weight; a.bias = op.bias; a.y = op.out;
  a.M = p.m; a.N = p.n; a.K = p.k;
  a.lda = p.a_row_stride ? p.a_row_stride : p.k;
  a.ldb = p.k;
  a.ldy = p.c_row_stride ? p.c_row_stride : p.n;
  a.relu = q.activation;
  a.alpha = 1.0f;
  a.HoWo = a.Wo = a.Cin = a.kw = 1;
  // Kernels count K past its end in 32 bits: to the end of a tile, with one row to the end of two wavefronts' vectors.
  if (p.m > kInt - 64 || p.k > kInt - 2048) return too_large("more rows or columns than one launch holds", op);
  auto set = [&](int kernel, int rows, int cols, int threads) {
    out->kernel = kernel;
    out->gx = (uint32_t)cdiv(p.m, rows); out->gy = (uint32_t)cdiv(p.n, cols); out->gz = 1; out->block = threads;
  };
  const int64_t es = f16 ? 2 : 4, x_bytes = es * ((int64_t)(p.m - 1) * a.lda + p.k), w_bytes = es * 2 * (int64_t)p.n * p.k;
  // Loads straight into workgroup memory need aligned 16-byte pieces and 32-bit offsets.
  const bool vec = p.k % (16 / es) == 0 && a.lda % (16 / es) == 0 && aligned16(a.x) && aligned16(a.w) && x_bytes < kOperandMaxBytes &&
                   w_bytes < kOperandMaxBytes && p.k * es < 1 << 29;
  a.x_bytes = vec ? (uint32_t)x_bytes : 0;
  a.w_bytes = vec ? (uint32_t)w_bytes : 0;
  if (p.m == 1 && (!vec || p.n <= kGatedRowMaxCols)) {
    set(f16 ? K_gated_f16_row : K_gated_f32_row, 1, 4, 256);
    std::swap(out->gx, out->gy);
  } else if (!vec) {
    set(f16 ? K_gated_f16_any : K_gated_f32_any, kGatedAnyRows, kGatedAnyCols, 256);
  } else {
    const GatedForm *best = nullptr;
    double least = 0.0;
    for (const GatedForm &f : kGatedForms) {
      if (f.ids[f16] < 0) continue;
      const double cost = gated_cost(f, p.m, p.n, p.k, f16);
      if (!best || cost < least) { best = &f; least = cost; }
    }
    set(best->ids[f16], best->rows, best->cols, best->threads);
  }
  if ((int64_t)out->gx * out->gy > kInt) return too_large("more rows or columns than one launch holds", op);
  a.div_gx = div_magic(out->gx);
  out->args.igemm = a;
  return OPARA_OK;
}

// ---- attention
struct AttendShape {
  int64_t batch, heads, kv_heads, share, width, v_width, strides[4][3];
  int dp;                                  // both widths padded: 64, 128 or 256
  double keys;                             // what a query row sees of n in the mean, as far as the host knows
};

int attend_shape(const opara_op_desc &op, const opara_op_more &q, AttendShape *s) {
  const opara_op_params &p = op.params;
  s->batch = p.batch ? p.batch : 1;
  s->heads = q.heads;
  s->kv_heads = q.kv_heads ? q.kv_heads : q.heads;
  s->width = q.width;
  s->v_width = q.v_width ? q.v_width : q.width;
  if (s->batch < 1 || s->batch > 65535 || p.m <= 0 || p.n <= 0 || s->heads <= 0 || s->kv_heads <= 0 || s->heads % s->kv_heads)
    return fail("bad attention shape", op);
  if (q.width < 1 || q.width > kAttendMaxWidth || s->v_width < 1 || s->v_width > kAttendMaxWidth) return fail("head width outside 1..256", op);
  if ((p.flags & OPARA_FLAG_CAUSAL) && (p.flags & OPARA_FLAG_CAUSAL_END)) return fail("one kind of causal mask", op);
  s->share = s->heads / s->kv_heads;
  if (s->kv_heads > 65535 || p.n > (1 << 30) || (int64_t)p.m * s->share > (1 << 30)) return too_large("more rows or heads than one launch holds", op);
  const int64_t rows[4] = {p.m, p.n, p.n, p.m}, heads[4] = {s->heads, s->kv_heads, s->kv_heads, s->heads},
                width[4] = {q.width, q.width, s->v_width, s->v_width};
  for (int i = 0; i < 4; ++i) {
    const int64_t *given = q.strides[i];
    if (given[0] < 0 || given[1] < 0 || given[2] < 0) return fail("negative stride", op);
    const bool packed = !(given[0] | given[1] | given[2]);
    s->strides[i][2] = packed ? width[i] : given[2];
    s->strides[i][1] = packed ? heads[i] * width[i] : given[1];
    s->strides[i][0] = packed ? rows[i] * heads[i] * width[i] : given[0];
  }
  // Every result element has a place of its own: sorted by their strides, each axis steps over the ones below.
  {
    const int64_t *y = s->strides[3];
    struct Axis { int64_t stride, count; } axis[3] = {{y[0], s->batch}, {y[1], p.m}, {y[2], s->heads}};
    std::sort(axis, axis + 3, [](const Axis &a, const Axis &b) { return a.stride < b.stride; });
    int64_t reach = s->v_width;
    for (const Axis &x : axis) {
      if (x.count == 1) continue;
      if (x.stride < reach) return fail("result rows overlap", op);
      reach += x.stride * (x.count - 1);
    }
  }
  const int widest = std::max(q.width, (int32_t)s->v_width);
  s->dp = widest <= 64 ? 64 : widest <= 128 ? 128 : 256;
  const double first = p.flags & OPARA_FLAG_CAUSAL ? (double)q.first : (double)p.n - p.m;
  s->keys = p.n;
  if (p.flags & (OPARA_FLAG_CAUSAL | OPARA_FLAG_CAUSAL_END)) s->keys = std::min<double>(p.n, std::max(1.0, first + 0.5 * p.m));
  return OPARA_OK;
}

// What the forms of attention cost: nanoseconds per key for a workgroup with a compute unit to itself whose keys are in
// a cache (`alone`) or, all of them more than kAttendCached, come from memory (`far`), and in a full launch (`busy`);
// microseconds of the launch and everything else outside the keys (`fixed`), of every further 256 workgroups
// (`each`), of a join (`join`), of every workgroup that a tile is joined from (`part`) and of every 256 that leave a
// record (`records`).  Fitted to 600 to 1000 launches per type and width (1..2048 rows of 1..32 key heads,
// 60..65536 keys, 1..256 splits) within 5 to 21 %, fp16 of width 256 apart, whose row is an estimate; the fp16 rows forms
// before they had a second product, which costs up to 7 %.  What they pick
// for keys that are loaded directly is 1 to 3 % slower than the best in the mean and 32 % at worst (one row of 12 heads of
// 256, 65536 keys), for unaligned keys, which go through registers, 1 to 5 % and 45 %; these priced as the others
// (5 to 22 times too fast) were 6 to 42 % slower than the best, up to 3.7 times (one row of 32 heads over 8 of 101,
// 16384 keys: 258 us, now 69).
// The deep forms (eight wavefronts) against four: 12 heads of 64, 1500 keys, one row 8.0 -> 7.6 us, one key head of 64,
// 2048 rows, 4096 keys 17.8 -> 14.2; where many workgroups run at once the small ones are the faster, 12 heads of 64,
// 1024 rows, 512 keys 11.9 and 9.3.
struct AttendForm {
  int kernel, rows, key_tile, threads;
  double alone, far, busy, fixed, each, join, part, records;
};
constexpr double kAttendCached = 85e6;
const AttendForm kAttendF16[3][3] = {
    {{K_attend_f16_rows64, 16, 128, 256, 3.7, 6.7, 3.1, 3.7, 0.39, 2.4, 0.080, 1.7},
     {K_attend_f16_deep64, 16, 256, 512, 2.4, 6.6, 3.1, 4.0, 0.79, 3.7, 0.027, 2.9},
     {K_attend_f16_wide64, 128, 64, 256, 13.7, 14.0, 10.4, 4.5, 0.79, 2.9, 0.440, 1.9}},
    {{K_attend_f16_rows128, 16, 128, 256, 4.9, 10.9, 6.5, 4.7, 0.95, 2.3, 0.095, 1.9},
     {K_attend_f16_deep128, 16, 256, 512, 4.9, 10.6, 7.0, 4.4, 1.80, 3.6, 0.038, 4.5},
     {K_attend_f16_wide128, 128, 64, 256, 21.2, 21.2, 16.6, 5.8, 1.78, 3.1, 0.804, 3.7}},
    {{K_attend_f16_rows256, 16, 128, 256, 16.0, 16.0, 22.0, 6.0, 2.50, 2.5, 0.150, 3.0}}};
const AttendForm kAttendF32[3][3] = {
    {{K_attend_f32_rows64, 16, 64, 256, 12.3, 13.4, 10.6, 4.1, 0.48, 2.4, 0.082, 1.2},
     {K_attend_f32_deep64, 16, 128, 512, 9.4, 11.0, 10.5, 4.6, 1.22, 3.7, 0.031, 1.7}},
    {{K_attend_f32_rows128, 16, 64, 256, 20.9, 21.1, 21.8, 5.0, 1.17, 2.7, 0.093, 1.2},
     {K_attend_f32_deep128, 16, 128, 512, 16.9, 19.5, 21.5, 5.5, 3.27, 3.7, 0.052, 2.8}},
    {{K_attend_f32_rows256, 16, 64, 256, 43.3, 43.3, 50.6, 7.6, 4.97, 1.9, 0.146, 1.0}}};
const AttendForm kAttendAny[2][3] = {                       // unaligned keys; f32, f16
    {{K_attend_f32_any64, 16, 64, 256, 60.2, 95.8, 26.9, 2.4, 0.0, 2.0, 0.093, 2.0},
     {K_attend_f32_any128, 16, 64, 256, 119.0, 181.0, 89.8, 1.9, 0.0, 3.1, 0.138, 1.1},
     {K_attend_f32_any256, 16, 64, 256, 251.0, 341.0, 299.0, 2.0, 0.0, 4.2, 0.190, 0.0}},
    {{K_attend_f16_any64, 16, 128, 256, 51.4, 71.3, 17.8, 2.0, 0.0, 1.0, 0.106, 2.8},
     {K_attend_f16_any128, 16, 128, 256, 106.0, 159.0, 71.6, 2.0, 0.0, 3.2, 0.141, 0.4},
     {K_attend_f16_any256, 16, 128, 256, 168.0, 217.0, 196.0, 3.1, 0.0, 3.9, 0.203, 0.0}}};

struct AttendPick { const AttendForm *form; int64_t tiles, splits, counter_bytes, scratch; };

// vec: keys and values can be loaded straight into workgroup memory; room: scratch memory there is.
AttendPick attend_pick(const opara_op_desc &op, const AttendShape &s, bool vec, uint64_t room) {
  const bool f16 = op.dtype == OPARA_F16;
  const int size = s.dp == 64 ? 0 : s.dp == 128 ? 1 : 2;
  const AttendForm *forms = !vec ? &kAttendAny[f16][size] : f16 ? kAttendF16[size] : kAttendF32[size];
  const double bytes = s.batch * s.kv_heads * s.keys * (s.width + s.v_width) * (f16 ? 2 : 4);
  AttendPick best{};
  double least = 0.0;
  for (int i = 0; i < (vec ? 3 : 1) && forms[i].rows; ++i) {
    const AttendForm &f = forms[i];
    const int64_t tiles = cdiv((int64_t)op.params.m * s.share, f.rows), work = tiles * s.kv_heads * s.batch;
    for (int64_t n = 1; n <= kAttendMaxSplits; n = n < 4 ? n + 1 : n + n / 2) {
      if (n > 1 && n * f.key_tile > s.keys) break;           // two tiles for every wavefront
      if (n > (f.rows == kAttendRows ? kAttendMaxSplits : kAttendMaxWideSplits)) break;
      AttendPick p{&f, tiles, n, cdiv(4 * work, 256) * 256, 0};
      const int64_t records = work * n * (f.rows * s.dp + 2 * f.rows) * 4;
      if (n > 1) p.scratch = p.counter_bytes + records;
      if ((uint64_t)p.scratch > room || p.scratch > kAttendMaxScratch) break;
      const double keys = std::ceil(s.keys / (f.key_tile * n)) * f.key_tile, groups = work * n;
      // Between one and four workgroups per compute unit the fuller ones decide, half of the time.
      const double per_cu = groups > 256 && groups < 1024 ? 0.5 * (std::ceil(groups / 256) + groups / 256) : groups / 256;
      double cost = f.fixed + std::max({keys * (bytes > kAttendCached ? f.far : f.alone) * 1e-3, per_cu * (keys * f.busy * 1e-3 + f.each), bytes / 6e6});
      if (n > 1) cost += f.join + f.part * n + f.records * groups / 256;
      if (!best.form || cost < least) { best = p; least = cost; }
    }
  }
  return best;
}

int plan_attention(const opara_op_desc &op, const opara_op_more &q, const void *const *in, KernelPlan *out) {
  const opara_op_params &p = op.params;
  const int ve = op.dtype == OPARA_F16 ? 8 : 4;
  AttendShape s;
  const int rc = attend_shape(op, q, &s);
  if (rc != OPARA_OK) return rc;
  if (op.n_inputs < 3 || op.n_inputs > 4) return fail("attention takes queries, keys, values and optionally lengths", op);
  if ((uintptr_t)q.scratch & 255u) return fail("scratch is not 256-byte aligned", op);
  AttendArgs a;
  std::memset(&a, 0, sizeof a);
  a.q = in[0]; a.k = in[1]; a.v = in[2]; a.y = op.out;
  a.lengths = op.n_inputs > 3 ? (const int32_t *)in[3] : nullptr;
  std::memcpy(a.q_s, s.strides[0], sizeof a.q_s);
  std::memcpy(a.k_s, s.strides[1], sizeof a.k_s);
  std::memcpy(a.v_s, s.strides[2], sizeof a.v_s);
  std::memcpy(a.y_s, s.strides[3], sizeof a.y_s);
  // Loads straight into workgroup memory need aligned 16-byte pieces, rows that do not overlap (a tile of keys
  // ends with its last row) and 32-bit offsets inside a tile.
  auto vectors = [&](const void *base, const int64_t *st, int64_t width) {
    return aligned16(base) && width % ve == 0 && st[0] % ve == 0 && st[1] % ve == 0 && st[2] % ve == 0 &&
           st[1] >= width && st[1] < (int64_t)kOperandMaxBytes / (64 * 4);
  };
  const bool vec = vectors(a.k, a.k_s, q.width) && vectors(a.v, a.v_s, s.v_width);
  const AttendPick pick = attend_pick(op, s, vec, q.scratch ? q.scratch_bytes : 0);
  a.m = p.m; a.n = p.n; a.share = (int32_t)s.share; a.width = q.width; a.v_width = (int32_t)s.v_width;
  a.batch = (int32_t)s.batch;
  a.causal = (p.flags & OPARA_FLAG_CAUSAL) ? 1 : (p.flags & OPARA_FLAG_CAUSAL_END) ? 2 : 0;
  a.first = q.first;
  // Above zero, so that a masked score stays -inf: with alpha 0 the queries are zeros and all visible keys count the same.
  a.scale = std::max(std::fabs(p.alpha) * 1.44269504088896341f, FLT_MIN);
  a.sign = p.alpha < 0.f ? -1.f : p.alpha > 0.f ? 1.f : 0.f;
  a.tiles = (int32_t)pick.tiles;
  a.splits = (int32_t)pick.splits;
  if (a.splits > 1) {
    a.counters = (uint32_t *)q.scratch;
    a.partials = (float *)((unsigned char *)q.scratch + pick.counter_bytes);
  }
  a.div_share = div_magic(s.share);
  a.div_splits = div_magic(a.splits);
  out->kernel = pick.form->kernel;
  const int64_t gx = pick.tiles * pick.splits;
  if (gx * s.kv_heads * s.batch > kInt) return too_large("more rows than one launch holds", op);
  out->gx = (uint32_t)gx; out->gy = (uint32_t)s.kv_heads; out->gz = (uint32_t)s.batch; out->block = (uint32_t)pick.form->threads;
  out->args.attend = a;
  return OPARA_OK;
}

}  // namespace

int plan_decoder(const opara_op_desc &op, const opara_op_more &more, const void *const *in, KernelPlan *out) {
  int rc;
  switch (op.op_type) {
    case OPARA_ROTARY: rc = plan_rotary(op, more, in, out); break;
    case OPARA_RESIDUAL_NORM: rc = plan_norm(op, more, in, out); break;
    case OPARA_GATED: rc = plan_gated(op, more, in, out); break;
    default: rc = plan_attention(op, more, in, out);
  }
  // A launch counts the threads along an axis in 32 bits.
  if (rc == OPARA_OK && (uint64_t)out->gx * out->block > UINT32_MAX) return too_large("more rows or columns than one launch holds", op);
  return rc;
}

}  // namespace opara

using namespace opara;

extern "C" int opara_rotary_table(int32_t rotated, double base, double factor, double original_length, double low, double high,
                                  uint64_t *turns) {
  if (!turns || rotated < 2 || rotated > 4096 || rotated % 2 || !(base > 0.0) || !std::isfinite(base) || !(factor > 0.0) ||
      !std::isfinite(factor) || !(original_length >= 0.0) || !std::isfinite(original_length) ||
      (original_length > 0.0 && !(low < high && std::isfinite(low) && std::isfinite(high)))) {
    set_error("opara_rotary_table: bad argument");
    return OPARA_EINVAL;
  }
  const long double two_pi = 6.283185307179586476925286766559L, turn = 18446744073709551616.0L;
  for (int32_t i = 0; i < rotated / 2; ++i) {
    long double f = powl((long double)base, -2.0L * i / rotated) / two_pi;
    if (original_length > 0.0) {
      const long double mix = std::min(1.0L, std::max(0.0L, (original_length * f - low) / ((long double)high - low)));
      f = f * (mix + (1.0L - mix) / factor);
    } else {
      f = f / factor;
    }
    f -= floorl(f);                                          // whole turns change nothing
    const long double v = f * turn + 0.5L;
    turns[i] = v >= turn ? 0 : (uint64_t)v;
  }
  return OPARA_OK;
}

extern "C" int opara_scratch_bytes(const opara_op_desc *op, const opara_op_more *more, uint64_t *bytes) {
  if (!op || !bytes) { set_error("opara_scratch_bytes: null pointer"); return OPARA_EINVAL; }
  *bytes = 0;
  if (op->op_type < 0 || op->op_type >= OPARA_N_OP_TYPES || (op->dtype != OPARA_F32 && op->dtype != OPARA_F16)) {
    set_error("opara_scratch_bytes: unknown op_type or dtype");
    return OPARA_EINVAL;
  }
  if (op->op_type != OPARA_ATTENTION) return OPARA_OK;
  AttendShape s;
  const int rc = attend_shape(*op, more ? *more : opara_op_more{}, &s);
  if (rc != OPARA_OK) return rc;
  // Whether keys and values are aligned shows later: enough for either case.
  for (bool vec : {false, true}) *bytes = std::max<uint64_t>(*bytes, (uint64_t)attend_pick(*op, s, vec, UINT64_MAX).scratch);
  return OPARA_OK;
}
