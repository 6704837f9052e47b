// C ABI of the operators that read a cache (see include/lagkv.h): host-side validation, launch shapes and launches.
#include <cmath>
#include <cstring>

#include "attend_internal.hpp"
#include "compress_ws.h"
#include "lagkv.h"
#include "lagkv_internal.hpp"

using namespace lagkv;

namespace {

constexpr int64_t kMost = 0x7fffffffLL;           // tokens times query heads
constexpr int64_t kMostRows = kMost - (1 << 16);  // (the kernels count in steps, the last of which may reach beyond)

int esize_of(const lagkv_attend_params* p) { return p->dtype == LAGKV_F32 ? 4 : 2; }
bool known(int32_t dtype) { return dtype == LAGKV_F32 || dtype == LAGKV_BF16 || dtype == LAGKV_F16; }
bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
int shift_of(int32_t block) { return __builtin_ctz((unsigned)block); }
bool block_ok(int32_t block) { return block >= 16 && block <= 1024 && (block & (block - 1)) == 0; }

int check_heads(const lagkv_attend_params* p) {
  if (!p) return LAGKV_EINVAL;
  if (!known(p->dtype)) return LAGKV_EDTYPE;
  if (p->B < 1 || p->H < 1 || p->D < kMinHead || p->D > kMaxHead) return LAGKV_ESHAPE;
  if ((int64_t)p->B * p->H > (1 << 24) || p->T < 0 || p->T > kMostRows) return LAGKV_ESHAPE;
  return LAGKV_OK;
}

int check_tokens(const lagkv_attend_params* p) {
  if (p->G < 1 || p->N < 0) return LAGKV_ESHAPE;
  if ((int64_t)p->G * p->N > kMost || (int64_t)p->B * p->H * p->G > kMost) return LAGKV_ESHAPE;
  if (p->q_stride_b < 0 || p->q_stride_h < 0 || p->q_stride_n < 0) return LAGKV_ESHAPE;
  return LAGKV_OK;
}

// Rows [B, heads, N] of D channels that lie apart: with the axes of more than one entry from the smallest stride up, each
// steps over all of what the ones before it span.
bool apart(int64_t D, const int64_t (&n)[3], const int64_t (&stride)[3]) {
  int order[3] = {0, 1, 2};
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (stride[order[j]] < stride[order[i]]) {
        const int t = order[i];
        order[i] = order[j];
        order[j] = t;
      }
  int64_t span = D;
  for (int i : order) {
    if (n[i] <= 1) continue;
    if (stride[i] < span) return false;
    span += stride[i] * (n[i] - 1);
  }
  return true;
}

int check_attend(const lagkv_attend_params* p, bool pick) {
  int rc = check_heads(p);
  if (rc != LAGKV_OK) return rc;
  rc = check_tokens(p);
  if (rc != LAGKV_OK) return rc;
  if (!std::isfinite((float)(p->scale * 1.4426950408889634))) return LAGKV_EINVAL;
  if (pick && (!block_ok(p->block) || p->n_blocks < 1 || (int64_t)p->n_blocks * p->block > kMostRows)) return LAGKV_EINVAL;
  if (p->kv_stride_b < 0 || p->kv_stride_h < 0 || p->kv_stride_t < 0 || p->new_stride_b < 0 || p->new_stride_h < 0 ||
      p->new_stride_n < 0 || p->out_stride_b < 0 || p->out_stride_h < 0 || p->out_stride_n < 0 || p->parents_stride_b < 0)
    return LAGKV_ESHAPE;
  return LAGKV_OK;
}

// Workgroups of the fullest of the eight XCDs (work_item deals units and pieces to them in turn, with all their tiles).
int64_t fullest_xcd(int64_t units, int64_t pieces, int64_t row_tiles) { return (units * pieces + 7) / 8 * row_tiles; }

// 1 2 3 4 6 8 12 16 24 ...
int64_t next_pieces(int64_t s) { return s + (s < 4 ? 1 : s % 3 == 0 ? s / 3 : s / 2); }

// Tiles of many rows: 128 query rows (four wavefronts, two workgroups a compute unit) or, for 65 to 128 channels, 256 (eight, one;
// for fewer channels they were the faster ones of none of 164 shapes), and the pieces that
// the cache is cut into, by the microseconds that they take: a step of 64 cache rows, the beginning and end of a workgroup,
// and, with pieces, a second kernel and every piece of a row written and read.  A step takes longer the more compute
// units are at work, and less where wavefronts of the eight have no rows.  Measured, 128 channels, model beside it (us; it
// falls short by a seventh in the mean, as narrow_shape's does, and what counts is which is the least):
//    8 streams,  256 query rows, 1000 rows   128 in 4 19 (18)   128 in 8 18 (16)   256 in 8 23 (20)   few rows 16 (15)
//   32 streams,  256 query rows, 2000 rows   128 in 4 33 (27)   128 in 8 35 (28)   256 in 4 36 (32)   256 in 8 34 (30)
//   32 streams,  256 query rows, 8000 rows   128 in 4 77 (62)   128 in 8 70 (57)   256 in 4 77 (74)   256 in 8 63 (54)
//   64 streams,  160 query rows, 8000 rows   128 in 4 100 (91)   128 in 8 105 (105)   256 in 2 124 (106)   256 in 4 82 (69)
// Over 914 shapes (64, 128 and 256 channels, 48 to 2048 query rows of 2 to 400 streams, 200 to 16000 rows) its choice takes 1.1 %
// longer than the best tile and number of pieces in the mean.
double wide_shape(int64_t units, int64_t rows, int64_t D, int64_t steps, int* row_tile, int64_t* pieces) {
  const double channels = D <= 64 ? 0.57 : D <= 128 ? 1 : 2.2;
  double least = 1e30;
  for (int tile = 128; tile <= (D > 64 && D <= 128 && rows > 128 ? 256 : 128); tile += 128) {
    const int64_t groups = units * ((rows + tile - 1) / tile), places = tile == 256 || D > 128 ? 256 : 512;
    const double full = (double)(units * rows) / (double)(groups * tile);
    for (int64_t s = 1; s <= 256 && s <= steps; s = next_pieces(s)) {
      const int64_t all = 8 * fullest_xcd(units, s, (rows + tile - 1) / tile);
      const double busy = all < 256 ? (double)all / 256 : 1;
      const double step = tile == 256 ? 0.85 + (0.65 + 0.5 * busy) * full : channels * (all > 256 && D <= 128 ? 2.35 : 1.25 + 0.2 * busy);
      const double ends = tile == 256 ? 12 : D <= 64 ? 7.3 : D <= 128 ? 9 : 8.5;
      const double us = (double)((all + places - 1) / places) * ((double)((steps + s - 1) / s) * step + ends) +
                        (s > 1 ? 2.5 + (double)(units * rows * s) * (double)D * 8 / 9e6 : 0);
      if (us < least) {
        least = us;
        *row_tile = tile;
        *pieces = s;
      }
    }
  }
  return least;
}

// Tiles of 16 or 32 query rows: the pieces of the cache by the microseconds that they take, none below a step a wavefront.
// A workgroup's steps take 0.45 us for 128 channels and it has beginning and end (5.5 us); a compute unit holds two of them, at
// no cost to each other but memory's with 16 query rows (32: 0.75 us beside another, in fp32 0.75 alone and 1.4), and one where
// the outputs fill its registers.  All rows together pass memory at 6 TB/s, less where some compute
// units have a workgroup more than others.  With pieces, a second kernel and every piece of a row written and read.
// Over 205 shapes (16-bit and fp32, 64 to 256 channels, 4 to 600 query rows, 1 to 1000 workgroups, 200 to 50000 rows) the
// time is 1 % above that of the best number of pieces in the mean; with as many pieces as make 512 workgroups, 11.9 %.  Where
// lengths differ within a batch (a quarter of T to T; 57 shapes) 3.9 % and 7.1 %.  (us: 40 streams of 4000 rows in 1 136, in 4
// 115; 192 streams in 1 70, in 2 79.)
double narrow_shape(int64_t units, int64_t rows, int64_t row_tile, int64_t D, bool f32, int64_t steps, int64_t* pieces) {
  const bool heavy = f32 && row_tile == 32;  // (bound by the products)
  const int64_t tiles = (rows + row_tile - 1) / row_tile, places = D > 128 ? 32 : 64;  // of an XCD
  const double channels = D <= 64 ? 0.5 : D <= 128 ? 1 : 2, alone = (heavy ? 0.75 : 0.45) * channels;
  const double both = (heavy ? 1.4 : row_tile == 32 ? 0.75 : 0.45) * channels;  // (beside another workgroup)
  const double ends = 5.5;
  const double memory = (double)units * (double)steps * (double)D * 128 / 6e6;
  double least = 1e30;
  for (int64_t s = 1; s <= 256 && (s == 1 || s <= steps / 4); s = next_pieces(s)) {
    const int64_t load = fullest_xcd(units, s, tiles);
    const double uneven = load > 32 ? (double)((load + 31) / 32 * 32) / (double)load - 1 : 0;
    const int64_t full = load / places, rest = load - full * places;
    const double each = (double)((steps + s - 1) / s);
    const double go = (double)full * (each * both + ends) + (rest > 32 ? each * both + ends : rest > 0 ? each * alone + ends : 0);
    const double pass = memory * (1 + 0.35 * uneven) + ends;
    const double us = (go > pass ? go : pass) + (s > 1 ? 3.5 + (double)(units * rows * s) * (double)D * 8 / 3e6 : 0);
    if (us < least) {
      least = us;
      *pieces = s;
    }
  }
  return least;
}

// Tiles of few query rows: as many as there are, up to what the registers hold.  Of many (16-bit types): tiles of 128 or 256
// where they take less time, by the two models.  (Over the 914 shapes of wide_shape, without new tokens, the time is 1.6 % above
// that of the better kernel at its best, with tiles of many rows for all of them 5.3 %, of few 39 %; over 299 with trees, 40 to
// 600 query rows, it is 0.4 % above the less of itself and of few rows, which take 19 % more in the mean.  us, few and many: 8
// streams, 256 query rows, 500 rows 15 and 16, 1000 rows 16 and 18; 32 streams, 256, 2000 rows 47 and 33; 8 streams of 256
// channels, 500 query rows, 4000 rows 140 and 53.)
bool plan_of(const lagkv_attend_params* p, bool pick, AttendPlan* pl) {
  pl->units = (int64_t)p->B * p->H * (pick ? p->N : 1);
  pl->rows = pick ? p->G : p->G * p->N;
  const int64_t all_rows = pl->units * pl->rows;
  if (pl->units > kMost || all_rows > kMostRows) return false;  // (they are numbered in 31 bits)
  const bool f32 = p->dtype == LAGKV_F32;
  const int64_t seen = pick ? (int64_t)p->n_blocks * p->block : p->T;
  auto steps_of = [&](int64_t kt) { return (seen + kt - 1) / kt + (p->N + kt - 1) / kt; };
  const int64_t steps = steps_of(f32 ? 16 : 32);
  int64_t splits = 1;
  pl->row_tile = pl->rows <= 16 || p->D > 128 ? 16 : 32;
  const double us = narrow_shape(pl->units, pl->rows, pl->row_tile, p->D, f32, steps, &splits);
  pl->wide = false;
  if (!pick && !f32 && pl->rows > 32) {
    int row_tile;
    int64_t pieces;
    pl->wide = wide_shape(pl->units, pl->rows, p->D, steps_of(64), &row_tile, &pieces) < us;
    if (pl->wide) {
      pl->row_tile = row_tile;
      splits = pieces;
    }
  }
  pl->row_tiles = (int)(((int64_t)pl->rows + pl->row_tile - 1) / pl->row_tile);
  const int64_t groups = pl->units * pl->row_tiles;
  // Short caches whole, by twice the wavefronts in one kernel: up to two steps a wavefront.  (One token over 300 rows of 128
  // 16-bit channels 7.1 us, in pieces about 8; over 640 rows, three steps, 9.5 us, over 1000 12.9 us and in pieces 8.4 us.
  // Rows of 64 fp32 channels: 300 rows 7.6 us, 640 rows 11.2 us and in pieces 7.6 us.)
  pl->waves = 4;
  if (!pl->wide && steps <= 16 && groups <= 256 && pl->row_tile == 16 && p->D <= 128) {
    splits = 1;
    pl->waves = 8;
  }
  // one piece where the grids do not hold more
  auto fits = [&](int64_t s) {
    const int64_t join = all_rows >= kJoinByWave ? (all_rows + 3) / 4 : all_rows;
    return grid_fits((pl->units * s + 7) / 8 * 8 * pl->row_tiles, pl->wide ? pl->row_tile * 2 : pl->waves * 64) && (s == 1 || grid_fits(join, 256));
  };
  if (!fits(splits)) splits = 1;
  pl->splits = (int)splits;
  const int64_t parts = all_rows * splits, ld = (p->D + 3) & ~3;
  pl->off_ml = splits > 1 ? ws_align_up((size_t)parts * ld * 4) : 0;
  pl->ws_bytes = splits > 1 ? pl->off_ml + ws_align_up((size_t)parts * 8) : 0;
  return fits(splits);
}

int attend(const lagkv_attend_params* p, const void* Q, const void* K, const void* V, const int32_t* lengths,
           const int32_t* blocks, const void* K_new, const void* V_new, const int32_t* parents, void* out, float* lse,
           void* ws, size_t ws_bytes, void* hip_stream, bool pick) {
  int rc = check_attend(p, pick);
  if (rc != LAGKV_OK) return rc;
  if (p->N == 0) return LAGKV_OK;
  if (!Q || !out || (p->T > 0 && (!K || !V)) || (pick && !blocks) || !K_new != !V_new || (parents && !K_new)) return LAGKV_EINVAL;
  if (parents && p->N > kMaxTree) return LAGKV_ESHAPE;
  const int64_t n[3] = {p->B, (int64_t)p->H * p->G, p->N};
  const int64_t st[3] = {p->out_stride_b, p->out_stride_h, p->out_stride_n};
  if (!apart(p->D, n, st)) return LAGKV_ESHAPE;
  const int es = esize_of(p);
  if (!aligned(Q, es) || !aligned(K, es) || !aligned(V, es) || !aligned(K_new, es) || !aligned(V_new, es) || !aligned(out, es) ||
      !aligned(lengths, 4) || !aligned(parents, 4) || !aligned(blocks, 4) || !aligned(lse, 4))
    return LAGKV_EINVAL;
  AttendPlan pl;
  if (!plan_of(p, pick, &pl)) return LAGKV_ESHAPE;
  if (pl.ws_bytes > 0 && (!ws || ws_bytes < pl.ws_bytes || !aligned(ws, 16))) return LAGKV_EWORKSPACE;
  AttendArgs a;
  std::memset(&a, 0, sizeof(a));
  a.Q = (const char*)Q;
  a.K = (const char*)K;
  a.V = (const char*)V;
  a.K_new = (const char*)K_new;
  a.V_new = (const char*)V_new;
  a.lengths = lengths;
  a.parents = parents;
  a.blocks = pick ? blocks : nullptr;
  a.out = (char*)out;
  a.lse = lse;
  a.part_o = (float*)ws;
  a.part_ml = (float*)((char*)ws + pl.off_ml);
  a.qsb = p->q_stride_b * es;
  a.qsh = p->q_stride_h * es;
  a.qsn = p->q_stride_n * es;
  a.ksb = p->kv_stride_b * es;
  a.ksh = p->kv_stride_h * es;
  a.kst = p->kv_stride_t * es;
  a.nsb = p->new_stride_b * es;
  a.nsh = p->new_stride_h * es;
  a.nst = p->new_stride_n * es;
  a.osb = p->out_stride_b * es;
  a.osh = p->out_stride_h * es;
  a.osn = p->out_stride_n * es;
  a.psb = p->parents_stride_b;
  a.T = p->T;
  a.units = pl.units;
  a.B = p->B;
  a.H = p->H;
  a.G = p->G;
  a.N = p->N;
  a.D = p->D;
  a.n_new = K_new ? p->N : 0;
  a.block = pick ? p->block : 0;
  a.block_shift = pick ? shift_of(p->block) : 0;
  a.n_blocks = pick ? p->n_blocks : 0;
  a.part_ld = (p->D + 3) & ~3;
  a.rows = pl.rows;
  a.row_tiles = pl.row_tiles;
  a.splits = pl.splits;
  a.by_tiles = Divide::by(pl.row_tiles);
  a.by_splits = Divide::by(pl.splits);
  a.by_n = Divide::by(p->N);
  a.by_h = Divide::by(p->H);
  a.by_g = Divide::by(p->G);
  a.by_rows = Divide::by(pl.rows);
  a.scale = (float)(p->dtype == LAGKV_F32 ? p->scale : p->scale * 1.4426950408889634);
  hipStream_t s = (hipStream_t)hip_stream;
  hipError_t e = pl.wide ? (p->dtype == LAGKV_BF16 ? launch_wide_bf16(a, pl.row_tile, s) : launch_wide_f16(a, pl.row_tile, s))
                 : p->dtype == LAGKV_F32  ? launch_attend_f32(a, pl.row_tile, pl.waves, s)
                 : p->dtype == LAGKV_BF16 ? launch_attend_bf16(a, pl.row_tile, pl.waves, s)
                                          : launch_attend_f16(a, pl.row_tile, pl.waves, s);
  if (e == hipSuccess && pl.splits > 1) e = launch_attend_join(a, p->dtype, s);
  return e == hipSuccess ? LAGKV_OK : LAGKV_EHIP;
}

}  // namespace

extern "C" {

size_t lagkv_attend_workspace_bytes(const lagkv_attend_params* p) {
  if (!p) return 0;
  const bool pick = p->n_blocks > 0;
  AttendPlan pl;
  if (check_attend(p, pick) != LAGKV_OK || p->N == 0 || !plan_of(p, pick, &pl)) return 0;
  return pl.ws_bytes;
}

int lagkv_attend_plan(const lagkv_attend_params* p, lagkv_attend_plan_t* out) {
  if (!p || !out) return LAGKV_EINVAL;
  const bool pick = p->n_blocks > 0;
  const int rc = check_attend(p, pick);
  if (rc != LAGKV_OK) return rc;
  std::memset(out, 0, sizeof(*out));
  if (p->N == 0) return LAGKV_OK;
  AttendPlan pl;
  if (!plan_of(p, pick, &pl)) return LAGKV_ESHAPE;
  out->many_rows = pl.wide;
  out->row_tile = pl.row_tile;
  out->wavefronts = pl.wide ? pl.row_tile / 32 : pl.waves;
  out->pieces = pl.splits;
  return LAGKV_OK;
}

int lagkv_attend(const lagkv_attend_params* p, const void* Q, const void* K, const void* V, const int32_t* lengths,
                 const void* K_new, const void* V_new, const int32_t* parents, void* out, float* lse, void* ws, size_t ws_bytes,
                 void* hip_stream) {
  return attend(p, Q, K, V, lengths, nullptr, K_new, V_new, parents, out, lse, ws, ws_bytes, hip_stream, false);
}

int lagkv_attend_blocks(const lagkv_attend_params* p, const void* Q, const void* K, const void* V, const int32_t* lengths,
                        const int32_t* blocks, const void* K_new, const void* V_new, const int32_t* parents, void* out,
                        float* lse, void* ws, size_t ws_bytes, void* hip_stream) {
  return attend(p, Q, K, V, lengths, blocks, K_new, V_new, parents, out, lse, ws, ws_bytes, hip_stream, true);
}

int lagkv_block_bounds(const lagkv_attend_params* p, const void* K, const int32_t* lengths, int64_t start, void* lo, void* hi,
                       void* hip_stream) {
  int rc = check_heads(p);
  if (rc != LAGKV_OK) return rc;
  if (!block_ok(p->block) || start < 0) return LAGKV_EINVAL;
  if (p->kv_stride_b < 0 || p->kv_stride_h < 0 || p->kv_stride_t < 0 || p->out_stride_b < 0 || p->out_stride_h < 0 ||
      p->out_stride_n < 0)
    return LAGKV_ESHAPE;
  if (p->T == 0 || start >= p->T) return LAGKV_OK;
  if (!K || !lo || !hi) return LAGKV_EINVAL;
  const int es = esize_of(p);
  if (!aligned(K, es) || !aligned(lo, es) || !aligned(hi, es) || !aligned(lengths, 4)) return LAGKV_EINVAL;
  const int64_t nb = (p->T + p->block - 1) / p->block;
  const int64_t n[3] = {p->B, p->H, nb}, st[3] = {p->out_stride_b, p->out_stride_h, p->out_stride_n};
  if (!apart(p->D, n, st)) return LAGKV_ESHAPE;
  BoundsArgs a;
  a.osb = p->out_stride_b * es;
  a.osh = p->out_stride_h * es;
  a.ost = p->out_stride_n * es;
  a.K = (const char*)K;
  a.lengths = lengths;
  a.lo = (char*)lo;
  a.hi = (char*)hi;
  a.ksb = p->kv_stride_b * es;
  a.ksh = p->kv_stride_h * es;
  a.kst = p->kv_stride_t * es;
  a.T = p->T;
  a.nb = nb;
  a.first = start / p->block;
  a.B = p->B;
  a.H = p->H;
  a.D = p->D;
  a.block = p->block;
  a.dtype = p->dtype;
  if (!grid_fits(((int64_t)p->B * p->H * (a.nb - a.first) + 3) / 4, 256)) return LAGKV_ESHAPE;
  return launch_block_bounds(a, (hipStream_t)hip_stream) == hipSuccess ? LAGKV_OK : LAGKV_EHIP;
}

int lagkv_select_blocks(const lagkv_attend_params* p, const void* Q, const void* lo, const void* hi, const int32_t* lengths,
                        int32_t n_first, int32_t n_last, int32_t* blocks, void* ws, size_t ws_bytes, void* hip_stream) {
  int rc = check_heads(p);
  if (rc != LAGKV_OK) return rc;
  rc = check_tokens(p);
  if (rc != LAGKV_OK) return rc;
  if (!block_ok(p->block) || p->n_blocks < 1 || n_first < 0 || n_last < 0 || (int64_t)n_first + n_last > p->n_blocks)
    return LAGKV_EINVAL;
  if (p->kv_stride_b < 0 || p->kv_stride_h < 0 || p->kv_stride_t < 0) return LAGKV_ESHAPE;
  if (p->N == 0) return LAGKV_OK;
  if (!Q || !blocks || (p->T > 0 && (!lo || !hi))) return LAGKV_EINVAL;
  const int es = esize_of(p);
  if (!aligned(Q, es) || !aligned(lo, es) || !aligned(hi, es) || !aligned(lengths, 4) || !aligned(blocks, 4)) return LAGKV_EINVAL;
  SelectArgs a;
  a.Q = (const char*)Q;
  a.lo = (const char*)lo;
  a.hi = (const char*)hi;
  a.lengths = lengths;
  a.score = (double*)ws;
  a.blocks = blocks;
  a.qsb = p->q_stride_b * es;
  a.qsh = p->q_stride_h * es;
  a.qsn = p->q_stride_n * es;
  a.bsb = p->kv_stride_b * es;
  a.bsh = p->kv_stride_h * es;
  a.bst = p->kv_stride_t * es;
  a.T = p->T;
  a.nb = (p->T + p->block - 1) / p->block;
  a.B = p->B;
  a.H = p->H;
  a.G = p->G;
  a.N = p->N;
  a.D = p->D;
  a.block = p->block;
  a.k = p->n_blocks;
  a.first = n_first;
  a.last = n_last;
  a.dtype = p->dtype;
  const int64_t units = (int64_t)p->B * p->H * p->N;
  if (!grid_fits(units, 512) || !grid_fits(((int64_t)p->B * p->H * ((a.nb + 63) / 64) + 7) * (((int64_t)p->N + 15) / 16), 256))
    return LAGKV_ESHAPE;
  if (a.nb > 0 && (!ws || ws_bytes < 8 * (size_t)(units * a.nb) || !aligned(ws, 16))) return LAGKV_EWORKSPACE;
  hipStream_t s = (hipStream_t)hip_stream;
  hipError_t e = a.nb > 0 ? launch_block_scores(a, s) : hipSuccess;
  if (e == hipSuccess) e = launch_block_select(a, s);
  return e == hipSuccess ? LAGKV_OK : LAGKV_EHIP;
}

}  // extern "C"
