// C ABI of the operators of a cache in 8 bits (see include/lagkv.h): host-side validation, launch shapes and launches.
#include <cstring>

#include "compress_ws.h"
#include "lagkv.h"
#include "lagkv_internal.hpp"
#include "quant_internal.hpp"

using namespace lagkv;

namespace {

constexpr int64_t kMostRows = 0x7fffffffLL - (1 << 16);  // (the kernels count in steps, the last of which may reach beyond)

int esize_of(const lagkv_quant_params* p) { return p->dtype == LAGKV_F32 ? 4 : 2; }
bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

int check_codes(const lagkv_quant_params* p) {
  if (!p) return LAGKV_EINVAL;
  if (p->dtype != LAGKV_F32 && p->dtype != LAGKV_BF16 && p->dtype != LAGKV_F16) return LAGKV_EDTYPE;
  if (p->code != LAGKV_CODE_INT8 && p->code != LAGKV_CODE_E4M3) return LAGKV_EDTYPE;
  if (p->B < 1 || p->H < 1 || p->D < kMinCodes || p->D > kMaxHead) return LAGKV_ESHAPE;
  if ((int64_t)p->B * p->H > (1 << 24) || p->T < 0 || p->T > kMostRows) return LAGKV_ESHAPE;
  if (p->block < 16 || p->block > 1024 || (p->block & (p->block - 1)) != 0) return LAGKV_EINVAL;
  if (p->code_stride_b < 0 || p->code_stride_h < 0 || p->code_stride_t < 0 || p->scale_stride_b < 0 || p->scale_stride_h < 0 ||
      p->row_stride_b < 0 || p->row_stride_h < 0 || p->row_stride_t < 0)
    return LAGKV_ESHAPE;
  return LAGKV_OK;
}

int go_over_codes(const lagkv_quant_params* p, const void* K, const void* V, const void* Kq, const void* Vq, const float* ks,
                  const float* vs, const int32_t* lengths, int64_t start, bool back, void* hip_stream) {
  const int rc = check_codes(p);
  if (rc != LAGKV_OK) return rc;
  if (start < 0) return LAGKV_EINVAL;
  if (p->T == 0 || start >= p->T) return LAGKV_OK;
  if (!K || !V || !Kq || !Vq || !ks || !vs) return LAGKV_EINVAL;
  const int es = esize_of(p);
  if (!aligned(K, es) || !aligned(V, es) || !aligned(ks, 4) || !aligned(vs, 4) || !aligned(lengths, 4)) return LAGKV_EINVAL;
  const int64_t nb = (p->T + p->block - 1) / p->block, n[3] = {p->B, p->H, p->T};
  if (back) {
    const int64_t st[3] = {p->row_stride_b, p->row_stride_h, p->row_stride_t};
    if (!rows_apart(p->D, n, st)) return LAGKV_ESHAPE;
  } else {
    const int64_t st[3] = {p->code_stride_b, p->code_stride_h, p->code_stride_t};
    const int64_t m[3] = {p->B, p->H, 1}, ss[3] = {p->scale_stride_b, p->scale_stride_h, 0};
    if (!rows_apart(p->D, n, st) || !rows_apart(nb, m, ss)) return LAGKV_ESHAPE;
  }
  CodeArgs a;
  std::memset(&a, 0, sizeof(a));
  a.first = (int32_t)(start / p->block);
  a.count = (int32_t)(nb - a.first);
  a.units = 2 * (int64_t)p->B * p->H * a.count;
  if (a.units > kMostRows) return LAGKV_ESHAPE;
  a.K = (const char*)K;
  a.V = (const char*)V;
  a.Kq = (const char*)Kq;
  a.Vq = (const char*)Vq;
  a.ks = const_cast<float*>(ks);
  a.vs = const_cast<float*>(vs);
  a.lengths = lengths;
  a.rsb = p->row_stride_b * es;
  a.rsh = p->row_stride_h * es;
  a.rst = p->row_stride_t * es;
  a.csb = p->code_stride_b;
  a.csh = p->code_stride_h;
  a.cst = p->code_stride_t;
  a.ssb = p->scale_stride_b;
  a.ssh = p->scale_stride_h;
  a.T = p->T;
  a.start = start;
  a.B = p->B;
  a.H = p->H;
  a.D = p->D;
  a.block = p->block;
  a.slices = (p->D + 7) / 8;
  a.by_count = Divide::by(a.count);
  a.by_h = Divide::by(p->H);
  a.by_slices = Divide::by(a.slices);
  hipStream_t s = (hipStream_t)hip_stream;
  const hipError_t e = back ? launch_dequantize(a, p->dtype, p->code, s) : launch_quantize(a, p->dtype, p->code, s);
  return e == hipSuccess ? LAGKV_OK : LAGKV_EHIP;
}

// The tail and the new tokens, or a call without rows in 8 bits, as a call of lagkv_attend.
lagkv_attend_params rows_of(const lagkv_quant_params* p) {
  lagkv_attend_params r;
  std::memset(&r, 0, sizeof(r));
  r.B = p->B;
  r.H = p->H;
  r.G = p->G;
  r.N = p->N;
  r.D = p->D;
  r.dtype = p->dtype;
  r.T = p->R;
  r.scale = p->scale;
  r.q_stride_b = p->q_stride_b;
  r.q_stride_h = p->q_stride_h;
  r.q_stride_n = p->q_stride_n;
  r.kv_stride_b = p->row_stride_b;
  r.kv_stride_h = p->row_stride_h;
  r.kv_stride_t = p->row_stride_t;
  r.new_stride_b = p->new_stride_b;
  r.new_stride_h = p->new_stride_h;
  r.new_stride_n = p->new_stride_n;
  r.out_stride_b = p->out_stride_b;
  r.out_stride_h = p->out_stride_h;
  r.out_stride_n = p->out_stride_n;
  r.parents_stride_b = p->parents_stride_b;
  return r;
}

int check_quant(const lagkv_quant_params* p) {
  const int rc = check_codes(p);
  if (rc != LAGKV_OK) return rc;
  const lagkv_attend_params r = rows_of(p);
  return attend_check(&r, false);
}

// The kernel of few rows: tiles of 16, or of 32 where the registers hold them, the cache rows of a step in 8 bits and in the type, and the
// microseconds of a step with one workgroup on a compute unit, of one with others beside it, of a workgroup's beginning and end, and of the kernel that
// joins the pieces; a step of the tail and the new tokens takes `of_rows` of one in 8 bits.
struct QuantForm {
  int row_tile, step, step_of_rows;
  double alone, beside, ends, join, of_rows;
};
QuantForm quant_form(const lagkv_quant_params* p, int64_t rows) {
  if (p->dtype == LAGKV_F32) {
    if (p->D > 128) return {16, 32, 16, 0.55, 0.62, 9.8, 4.4, 1.4};
    if (p->D > 64) return rows <= 16 ? QuantForm{16, 64, 16, 0.61, 1.05, 5, 5, 0.71} : QuantForm{32, 32, 16, 0.4, 0.59, 5, 8.3, 1.6};
    return rows <= 16 ? QuantForm{16, 64, 16, 0.44, 0.64, 3.8, 4.6, 0.64} : QuantForm{32, 64, 16, 0.41, 0.69, 5.2, 5.5, 0.92};
  }
  if (p->D > 128) return {16, 32, 32, 0.52, 0.52, 10.3, 2.4, 1.7};
  if (p->D > 64) return rows <= 16 ? QuantForm{16, 64, 32, 0.58, 1.06, 6.8, 2.2, 0.74} : QuantForm{32, 32, 32, 0.3, 0.47, 5.9, 6.5, 1.5};
  return rows <= 16 ? QuantForm{16, 64, 32, 0.43, 0.66, 5, 3.2, 0.75} : QuantForm{32, 64, 32, 0.38, 0.6, 5.4, 4.9, 0.75};
}
int64_t next_of(int64_t pieces) { return pieces + (pieces < 4 ? 1 : pieces % 3 == 0 ? pieces / 3 : pieces / 2); }  // 1 2 3 4 6 8 12 16 24 ...

// Its pieces of the rows in 8 bits and of the others by the microseconds that they take: rounds of workgroups on the fullest of the eight
// XCDs (two a compute unit; one beyond 128 channels), or all rows past memory at 5.5 TB/s; and the kernel that joins the pieces.
double quant_narrow_shape(const lagkv_quant_params* p, const QuantForm& f, int64_t units, int64_t rows, int* pieces, int* pieces_of_rows) {
  const int64_t steps = (p->T + f.step - 1) / f.step, others = (p->R + f.step_of_rows - 1) / f.step_of_rows + (p->N + f.step_of_rows - 1) / f.step_of_rows;
  const int64_t tiles = (rows + f.row_tile - 1) / f.row_tile, places = p->D > 128 ? 32 : 64;
  const double memory = (double)units * (double)p->D * ((double)p->T * 2 + (double)(p->R + p->N) * 2 * esize_of(p)) / 5.5e6;
  double least = 1e30;
  for (int64_t sq = 1; sq <= 512 && (sq == 1 || sq * 4 <= steps); sq = next_of(sq)) {
    // (their share of the pieces, some less and some more; with one piece of the rows in 8 bits any number)
    const int64_t share = others * sq / steps, choices[] = {1, 2, 3, share / 2, share, 2 * share};
    int64_t st = 0;
    for (int i = 0; sq == 1 || i < 6; ++i) {
      const int64_t now = sq == 1 ? next_of(st) : choices[i];
      if (sq == 1 && (now > 128 || (now > 1 && now * 4 > others))) break;
      if (now <= st || (now > 1 && now * 4 > others)) continue;
      st = now;
      const double nq = (double)((units * sq + 7) / 8 * tiles), nt = (double)((units * st + 7) / 8 * tiles);
      const double step = nq + nt > 32 ? f.beside : f.alone;
      const double tq = (double)((steps + sq - 1) / sq) * step + f.ends, tt = (double)((others + st - 1) / st) * step * f.of_rows + f.ends;
      const int64_t rounds = ((int64_t)nq + places - 1) / places;
      // (pieces of a kind end together: what does not fit beside them comes behind, where it is not dealt out to those that end sooner)
      double us = (double)rounds * tq + (nq + nt > (double)(rounds * places) ? 0.4 * (tt < tq ? tt : tq) : 0);
      us = us > tt ? us : tt;
      const double all = (nq * tq + nt * tt) / (double)places;
      us = us > all ? us : all;
      us = us > memory + f.ends ? us : memory + f.ends;
      us += f.join + (double)(units * rows * (sq + st)) * (double)p->D * 2.5e-6;
      if (us < least) {
        least = us;
        *pieces = (int)sq;
        *pieces_of_rows = (int)st;
      }
    }
  }
  return least;
}

// The kernel of many rows: tiles of 128, and the pieces of all rows.
// Of both: over 4417 shapes (1 to 4000 query rows of 1 to 256 streams, 64 to 256 channels, 64 to 65536 rows in 8 bits and up to 2048 behind them, some
// with lengths that differ; all types) the choice takes 2.4 % longer in the mean than the best form and pieces of up to 128 that were measured: half of them
// at most 0.1 %, nine in ten 9 %.
double quant_wide_shape(const lagkv_quant_params* p, int64_t units, int64_t rows, int* pieces) {
  const int64_t kt = p->D > 128 ? 32 : 64, steps = (p->T + kt - 1) / kt + (p->R + kt - 1) / kt + (p->N + kt - 1) / kt;
  const int64_t tiles = (rows + 127) / 128, places = p->D > 128 ? 32 : 64;
  const double alone = p->D <= 64 ? 1.35 : 1.6, beside = p->D <= 64 ? 1.6 : p->D <= 128 ? 2.15 : 1.6;
  const double ends = p->D <= 64 ? 9 : p->D <= 128 ? 12.5 : 24, traffic = p->D <= 128 ? 2.2e-6 : 1.2e-6;
  double least = 1e30;
  for (int64_t s = 1; s <= 512 && s <= steps; s = next_of(s)) {
    const int64_t groups = (units * s + 7) / 8 * tiles;
    const double us = (double)((groups + places - 1) / places) * ((double)((steps + s - 1) / s) * (groups > 32 ? beside : alone) + ends) +
                      (s > 1 ? 2.2 + (double)(units * rows * s) * (double)p->D * traffic : 0);
    if (us < least) {
      least = us;
      *pieces = (int)s;
    }
  }
  return least;
}

struct QuantPlan {
  AttendPlan rows;  // of the tail and the new tokens; units, rows and tiles are those of both
  int splits;       // pieces of the rows in 8 bits; of many query rows, all pieces
  int64_t groups, groups_of_rows;
  size_t off_ml, ws_bytes;
};
bool quant_plan_of(const lagkv_quant_params* p, QuantPlan* pl) {
  AttendPlan& t = pl->rows;
  std::memset(&t, 0, sizeof(t));
  t.units = (int64_t)p->B * p->H;
  t.rows = p->G * p->N;
  const int64_t all = t.units * t.rows;
  if (all > kMostRows || !grid_fits((all + 3) / 4, 256)) return false;
  const QuantForm f = quant_form(p, t.rows);
  t.row_tile = f.row_tile;
  t.waves = 4;
  const double us = quant_narrow_shape(p, f, t.units, t.rows, &pl->splits, &t.splits);
  if (p->dtype != LAGKV_F32 && t.rows > 32 && p->D % 16 <= 8) {  // (a row's last channels: see attend_quant_wide_body)
    int pieces = 1;
    t.wide = quant_wide_shape(p, t.units, t.rows, &pieces) < us;
    if (t.wide) {
      t.row_tile = 128;
      pl->splits = t.splits = pieces;
    }
  }
  t.row_tiles = (int)((t.rows + t.row_tile - 1) / t.row_tile);
  for (;;) {
    pl->groups = (t.units * pl->splits + 7) / 8 * 8 * t.row_tiles;
    pl->groups_of_rows = t.wide ? 0 : (t.units * t.splits + 7) / 8 * 8 * t.row_tiles;
    if (grid_fits(pl->groups + pl->groups_of_rows, 256)) break;
    if (pl->splits == 1 && t.splits == 1) return false;
    pl->splits = t.splits = 1;  // (one piece where the grids do not hold more)
  }
  const int pieces = t.wide ? pl->splits : pl->splits + t.splits;
  const int64_t parts = pieces > 1 ? all * pieces : 0, ld = (p->D + 3) & ~3;
  pl->off_ml = ws_align_up((size_t)parts * ld * 4);
  pl->ws_bytes = pl->off_ml + ws_align_up((size_t)parts * 8);
  return true;
}

}  // namespace

extern "C" {

int lagkv_quantize(const lagkv_quant_params* p, const void* K, const void* V, const int32_t* lengths, int64_t start, void* Kq,
                   void* Vq, float* K_scale, float* V_scale, void* hip_stream) {
  return go_over_codes(p, K, V, Kq, Vq, K_scale, V_scale, lengths, start, false, hip_stream);
}

int lagkv_dequantize(const lagkv_quant_params* p, const void* Kq, const void* Vq, const float* K_scale, const float* V_scale,
                     const int32_t* lengths, int64_t start, void* K, void* V, void* hip_stream) {
  return go_over_codes(p, K, V, Kq, Vq, K_scale, V_scale, lengths, start, true, hip_stream);
}

size_t lagkv_attend_quantized_workspace_bytes(const lagkv_quant_params* p) {
  if (check_quant(p) != LAGKV_OK || p->N == 0) return 0;
  if (p->T == 0) {
    const lagkv_attend_params r = rows_of(p);
    return lagkv_attend_workspace_bytes(&r);
  }
  QuantPlan pl;
  return quant_plan_of(p, &pl) ? pl.ws_bytes : 0;
}

int lagkv_attend_quantized_plan(const lagkv_quant_params* p, lagkv_attend_plan_t* codes, lagkv_attend_plan_t* rows) {
  if (!codes || !rows) return LAGKV_EINVAL;
  const int rc = check_quant(p);
  if (rc != LAGKV_OK) return rc;
  std::memset(codes, 0, sizeof(*codes));
  std::memset(rows, 0, sizeof(*rows));
  if (p->N == 0) return LAGKV_OK;
  const lagkv_attend_params r = rows_of(p);
  if (p->T == 0) return lagkv_attend_plan(&r, rows);
  QuantPlan pl;
  if (!quant_plan_of(p, &pl)) return LAGKV_ESHAPE;
  rows->many_rows = pl.rows.wide;
  rows->row_tile = pl.rows.row_tile;
  rows->wavefronts = pl.rows.waves;
  rows->pieces = pl.rows.splits;
  *codes = *rows;
  codes->pieces = pl.splits;
  return LAGKV_OK;
}

int lagkv_attend_quantized(const lagkv_quant_params* p, const void* Q, const void* Kq, const void* Vq, const float* K_scale,
                           const float* V_scale, const int32_t* lengths, const void* K_tail, const void* V_tail,
                           const int32_t* tail_lengths, const void* K_new, const void* V_new, const int32_t* parents, void* out,
                           float* lse, void* ws, size_t ws_bytes, void* hip_stream) {
  const int rc = check_quant(p);
  if (rc != LAGKV_OK) return rc;
  if (p->N == 0) return LAGKV_OK;
  const lagkv_attend_params r = rows_of(p);
  if (p->T == 0) return lagkv_attend(&r, Q, K_tail, V_tail, tail_lengths, K_new, V_new, parents, out, lse, ws, ws_bytes, hip_stream);
  if (!Q || !out || !Kq || !Vq || !K_scale || !V_scale || (p->R > 0 && (!K_tail || !V_tail)) || !K_new != !V_new || (parents && !K_new))
    return LAGKV_EINVAL;
  if (parents && p->N > kMaxTree) return LAGKV_ESHAPE;
  const int64_t n[3] = {p->B, (int64_t)p->H * p->G, p->N};
  const int64_t st[3] = {p->out_stride_b, p->out_stride_h, p->out_stride_n};
  if (!rows_apart(p->D, n, st)) return LAGKV_ESHAPE;
  const int es = esize_of(p);
  if (!aligned(Q, es) || !aligned(K_tail, es) || !aligned(V_tail, es) || !aligned(K_new, es) || !aligned(V_new, es) || !aligned(out, es) ||
      !aligned(lengths, 4) || !aligned(tail_lengths, 4) || !aligned(parents, 4) || !aligned(lse, 4) || !aligned(K_scale, 4) ||
      !aligned(V_scale, 4))
    return LAGKV_EINVAL;
  QuantPlan pl;
  if (!quant_plan_of(p, &pl)) return LAGKV_ESHAPE;
  if (pl.ws_bytes > 0 && (!ws || ws_bytes < pl.ws_bytes || !aligned(ws, 16))) return LAGKV_EWORKSPACE;
  const bool rows = p->R > 0 || K_new;
  QuantBoth both;
  std::memset(&both, 0, sizeof(both));
  AttendArgs& t = both.rows;
  t = attend_args(&r, pl.rows, false, Q, K_tail, V_tail, tail_lengths, nullptr, K_new, V_new, parents, out, lse, ws);
  t.part_ml = (float*)((char*)ws + pl.off_ml);
  t.part_splits = pl.splits + (rows && !pl.rows.wide ? pl.rows.splits : 0);
  t.part_first = pl.rows.wide ? 0 : pl.splits;
  QuantArgs& a = both.codes;
  a.Q = (const char*)Q;
  a.Kq = (const char*)Kq;
  a.Vq = (const char*)Vq;
  a.ks = K_scale;
  a.vs = V_scale;
  a.lengths = lengths;
  a.part_o = t.part_o;
  a.part_ml = t.part_ml;
  a.qsb = t.qsb;
  a.qsh = t.qsh;
  a.qsn = t.qsn;
  a.csb = p->code_stride_b;
  a.csh = p->code_stride_h;
  a.cst = p->code_stride_t;
  a.ssb = p->scale_stride_b;
  a.ssh = p->scale_stride_h;
  a.T = p->T;
  a.units = t.units;
  a.B = p->B;
  a.H = p->H;
  a.G = p->G;
  a.N = p->N;
  a.D = p->D;
  a.block_shift = __builtin_ctz((unsigned)p->block);
  a.part_ld = t.part_ld;
  a.rows = t.rows;
  a.row_tiles = t.row_tiles;
  a.splits = pl.splits;
  a.part_splits = t.part_splits;
  a.by_tiles = t.by_tiles;
  a.by_splits = Divide::by(pl.splits);
  a.by_h = t.by_h;
  a.by_g = t.by_g;
  a.scale = t.scale;
  both.groups = (uint32_t)pl.groups;
  const int64_t groups = pl.groups + (rows ? pl.groups_of_rows : 0);
  const int tile = pl.rows.row_tile;
  hipStream_t s = (hipStream_t)hip_stream;
  hipError_t e = pl.rows.wide ? (p->dtype == LAGKV_BF16 ? launch_quant_wide_bf16(both, groups, p->code, s)
                                                        : launch_quant_wide_f16(both, groups, p->code, s))
                 : p->dtype == LAGKV_F32  ? launch_quant_f32(both, groups, p->code, tile, s)
                 : p->dtype == LAGKV_BF16 ? launch_quant_bf16(both, groups, p->code, tile, s)
                                          : launch_quant_f16(both, groups, p->code, tile, s);
  t.splits = t.part_splits;  // (all of the pieces are joined; of few query rows there are always some)
  if (e == hipSuccess && (t.splits > 1 || !pl.rows.wide)) e = launch_attend_join(t, p->dtype, s);
  return e == hipSuccess ? LAGKV_OK : LAGKV_EHIP;
}

}  // extern "C"
