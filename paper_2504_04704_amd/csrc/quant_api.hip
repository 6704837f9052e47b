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

// Rows in 8 bits: tiles of 16 or 32 query rows and the pieces that attend_narrow_shape gives for as many bytes; then the tail and the
// new tokens, as they would be alone.
struct QuantPlan {
  AttendPlan rows;  // (its units and rows are of both)
  int row_tile, row_tiles, splits;
  int total;  // pieces of both
  size_t off_ml, ws_bytes;
};
bool quant_plan_of(const lagkv_quant_params* p, QuantPlan* pl) {
  const lagkv_attend_params r = rows_of(p);
  if (!attend_plan_of(&r, false, &pl->rows)) return false;
  const int64_t units = pl->rows.units, rows = pl->rows.rows, all = units * rows;
  pl->row_tile = rows <= 16 || p->D > 128 ? 16 : 32;
  pl->row_tiles = (int)((rows + pl->row_tile - 1) / pl->row_tile);
  int64_t splits = 1;
  attend_narrow_shape(units, rows, pl->row_tile, p->D, p->dtype == LAGKV_F32, (p->T + 63) / 64, &splits);
  auto fits = [&](int64_t s) { return grid_fits((units * s + 7) / 8 * 8 * pl->row_tiles, 256); };
  if (!fits(splits)) splits = 1;
  if (!fits(splits) || !grid_fits((all + 3) / 4, 256)) return false;
  pl->splits = (int)splits;
  pl->total = pl->splits + pl->rows.splits;
  const int64_t parts = all * pl->total, ld = (p->D + 3) & ~3;
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
  lagkv_attend_plan(&r, rows);
  codes->row_tile = pl.row_tile;
  codes->wavefronts = 4;
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
  if (!ws || ws_bytes < pl.ws_bytes || !aligned(ws, 16)) return LAGKV_EWORKSPACE;
  AttendArgs t = attend_args(&r, pl.rows, false, Q, K_tail, V_tail, tail_lengths, nullptr, K_new, V_new, parents, out, lse, ws);
  const bool tail = p->R > 0 || K_new;
  t.part_ml = (float*)((char*)ws + pl.off_ml);
  t.part_splits = tail ? pl.total : pl.splits;
  t.part_first = pl.splits;
  QuantArgs a;
  std::memset(&a, 0, sizeof(a));
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
  a.row_tiles = pl.row_tiles;
  a.splits = pl.splits;
  a.part_splits = t.part_splits;
  a.by_tiles = Divide::by(pl.row_tiles);
  a.by_splits = Divide::by(pl.splits);
  a.by_h = t.by_h;
  a.by_g = t.by_g;
  a.scale = t.scale;
  hipStream_t s = (hipStream_t)hip_stream;
  hipError_t e = p->dtype == LAGKV_F32  ? launch_quant_f32(a, p->code, pl.row_tile, s)
                 : p->dtype == LAGKV_BF16 ? launch_quant_bf16(a, p->code, pl.row_tile, s)
                                          : launch_quant_f16(a, p->code, pl.row_tile, s);
  if (e == hipSuccess && tail) e = launch_attend(t, pl.rows, p->dtype, s);
  t.splits = t.part_splits;  // (all of the pieces are joined)
  if (e == hipSuccess) e = launch_attend_join(t, p->dtype, s);
  return e == hipSuccess ? LAGKV_OK : LAGKV_EHIP;
}

}  // extern "C"
