// Internal interface between the host layer of the operators of a cache in 8 bits (quant_api.hip) and their kernels
// (quant_rows.hip, quant_attend.hpp).  Not part of the public ABI.
#pragma once
#include "attend_internal.hpp"

namespace lagkv {

// Rows into codes or back.  Strides of rows and codes in BYTES, of scales in elements.
struct CodeArgs {
  const char *K, *V;  // rows (written by the way back)
  const char *Kq, *Vq;
  float *ks, *vs;
  const int32_t* lengths;
  int64_t rsb, rsh, rst, csb, csh, cst, ssb, ssh;
  int64_t T, start, units;  // units: blocks of K and V, of all streams
  int32_t B, H, D, block, first, count;  // first block, and how many from it on
  int32_t slices;                        // of a row, eight channels each
  int32_t walk_rows, walk_slices;        // whole rows that the slices of all threads are, and what is left
  Divide by_count, by_h, by_slices;
};
hipError_t launch_quantize(const CodeArgs& a, int dtype, int code, hipStream_t s);
hipError_t launch_dequantize(const CodeArgs& a, int dtype, int code, hipStream_t s);

// Attention over rows in 8 bits: states of pieces of them, for launch_attend_join.  Strides of Q and codes in BYTES, of scales in
// elements.
struct QuantArgs {
  const char *Q, *Kq, *Vq;
  const float *ks, *vs;
  const int32_t* lengths;
  float *part_o, *part_ml;  // [units, part_splits, rows, ..]: this kernel's are the first `splits` of a unit's pieces
  int64_t qsb, qsh, qsn, csb, csh, cst, ssb, ssh;
  int64_t T, units;
  int32_t B, H, G, N, D;
  int32_t block_shift, part_ld, rows, row_tiles, splits, part_splits;
  Divide by_tiles, by_splits, by_h, by_g;
  float scale;  // times log2 e for the 16-bit types
};
// Both parts of a call; the tail and the new tokens are the pieces behind those of the rows in 8 bits.
struct QuantBoth {
  QuantArgs codes;
  AttendArgs rows;
  uint32_t groups;  // workgroups of the first
};
hipError_t launch_quant_f32(const QuantBoth& a, int64_t groups, int code, int row_tile, hipStream_t s);
hipError_t launch_quant_bf16(const QuantBoth& a, int64_t groups, int code, int row_tile, hipStream_t s);
hipError_t launch_quant_f16(const QuantBoth& a, int64_t groups, int code, int row_tile, hipStream_t s);
hipError_t launch_quant_wide_bf16(const QuantBoth& a, int64_t groups, int code, hipStream_t s);
hipError_t launch_quant_wide_f16(const QuantBoth& a, int64_t groups, int code, hipStream_t s);

constexpr int kMinCodes = 16;  // channels: a slice of codes has sixteen

}  // namespace lagkv
