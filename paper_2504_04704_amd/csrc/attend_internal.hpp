// Internal interface between the host layer of the cache-reading operators (attend_api.hip) and their kernels
// (attend_pass.hpp, block_pass.hip).  Not part of the public ABI.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lagkv.h"

namespace lagkv {

// n / d for n below 2^31 by a product (a division takes some twenty instructions, one behind the other, and the kernels
// begin with several).  With l the smallest for which d <= 2^l, and m = floor(2^32 (2^l - d) / d) + 1, the quotient is
// (floor(m n / 2^32) + n) / 2^l: m + 2^32 is 2^(32+l) / d rounded up by less than 2^l.
struct Divide {
  uint32_t m, l;
  __host__ static Divide by(uint32_t d) {
    Divide x = {0, 0};
    while ((uint64_t(1) << x.l) < d) ++x.l;
    x.m = (uint32_t)((((uint64_t(1) << x.l) - d) << 32) / d + 1);
    return x;
  }
  __host__ __device__ uint32_t of(uint32_t n) const { return ((uint32_t)((uint64_t)m * n >> 32) + n) >> l; }
};

// A unit is what one list of cache rows is for: a stream (b, h) with its G*N query rows, token-major (row n*G + g), or
// with blocks listed for each token, (b, h, n) with its G query rows.  Strides are in BYTES here.
struct AttendArgs {
  const char *Q, *K, *V, *K_new, *V_new;
  const int32_t* lengths;  // [B] or nullptr
  const int32_t* parents;  // [B,N] (or [N]) or nullptr
  const int32_t* blocks;   // [B,H,N,n_blocks] or nullptr
  char* out;
  float* lse;      // [B,H*G,N] or nullptr
  float* part_o;   // [units, splits, rows, part_ld], where splits > 1
  float* part_ml;  // [units, splits, rows, 2]: maximum (base 2), sum
  int64_t qsb, qsh, qsn, ksb, ksh, kst, nsb, nsh, nst, osb, osh, osn, psb;
  int64_t T, units;
  int32_t B, H, G, N, D;
  int32_t n_new;  // N with K_new, else 0
  int32_t block, block_shift, n_blocks;
  int32_t part_ld;  // D, rounded up to 4
  int32_t rows;    // of a unit
  int32_t row_tiles, splits;
  Divide by_tiles, by_splits, by_n, by_h, by_g, by_rows;  // row_tiles, splits, N, H, G, rows
  float scale;  // times log2 e for the 16-bit types
};

// Launch shape, a pure function of the parameters: rows of a tile, tiles of a unit, pieces the cache is cut into.
struct AttendPlan {
  bool wide;
  int row_tile, row_tiles, waves, splits;
  int64_t units;
  int32_t rows;
  size_t off_ml, ws_bytes;
};

hipError_t launch_attend_f32(const AttendArgs& a, int row_tile, int waves, hipStream_t s);
hipError_t launch_attend_bf16(const AttendArgs& a, int row_tile, int waves, hipStream_t s);
hipError_t launch_attend_f16(const AttendArgs& a, int row_tile, int waves, hipStream_t s);
hipError_t launch_wide_bf16(const AttendArgs& a, int row_tile, hipStream_t s);
hipError_t launch_wide_f16(const AttendArgs& a, int row_tile, hipStream_t s);
hipError_t launch_attend_join(const AttendArgs& a, int dtype, hipStream_t s);

struct BoundsArgs {
  const char* K;
  const int32_t* lengths;
  char *lo, *hi;  // [B,H,nb,D]
  int64_t ksb, ksh, kst, osb, osh, ost;
  int64_t T, nb, first;  // first block that is written
  int32_t B, H, D, block, dtype;
};
hipError_t launch_block_bounds(const BoundsArgs& a, hipStream_t s);

struct SelectArgs {
  const char *Q, *lo, *hi;
  const int32_t* lengths;
  double* score;     // [B,H,N,nb]
  int32_t* blocks;   // [B,H,N,k]
  int64_t qsb, qsh, qsn, bsb, bsh, bst;
  int64_t T, nb;
  int32_t B, H, G, N, D, block, k, first, last, dtype;
};
hipError_t launch_block_scores(const SelectArgs& a, hipStream_t s);
hipError_t launch_block_select(const SelectArgs& a, hipStream_t s);

constexpr int kJoinByWave = 2048;  // rows from which a wavefront joins the pieces of one, else a workgroup
constexpr int kMaxTree = 256;  // tokens of a drafted tree
constexpr int kMinHead = 8, kMaxHead = 256;

}  // namespace lagkv
