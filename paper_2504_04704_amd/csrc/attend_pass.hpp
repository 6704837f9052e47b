// Attention of new tokens over a cache and over themselves (lagkv_attend, lagkv_attend_blocks).
//
// For a query row q and the rows (k_t, v_t) that it sees, with x_t = scale * q.k_t:
//     m = max x_t,  l = sum exp(x_t - m),  out = sum exp(x_t - m) v_t / l,  lse = m + log l
// in one pass over the rows: a wavefront that has gone over some of them holds m, l and o = sum exp(x_t - m) v_t, and
// two such states (m1, l1, o1), (m2, l2, o2) join to m = max(m1, m2), l = l1 e^(m1-m) + l2 e^(m2-m), o likewise.  All of
// it is held in fp32, in base 2 (exp2 is the hardware's).
//
// A workgroup of four wavefronts takes a tile of 16, 32 or 64 query rows of a unit and a piece of its cache rows; each
// wavefront takes every fourth step of 32 rows (16 in fp32) for all query rows, so nothing is shared until the four
// states join at the end.  Both products go to the matrix cores, transposed:
//     S^T = K Q^T     (rows of K, as they lie in memory, are the operand whose k index runs along a lane's registers)
//     O^T += V^T P^T  (S^T leaves the matrix core with one query row a lane and four cache rows in its registers, which
//                      is how P^T has to be put in: nothing moves between lanes)
// V^T needs four cache rows of one channel in a lane: V goes through LDS, into memory private to the wavefront, and
// comes back through the transposing read (16-bit types) or element by element (fp32).
//
// P is put in as the sum of two 16-bit numbers (the value rounded, and what the rounding left): one alone would add as
// much error to the output as its own rounding, and the pass is bound by memory where tiles are small.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attend_internal.hpp"
#include "wave_ops.hpp"

namespace lagkv {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32v4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32v4_any __attribute__((ext_vector_type(4), aligned(2)));  // (wide loads take any address)
typedef uint32_t u32v2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;

__device__ __forceinline__ void wave_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

template <int DT>
struct AElem;
template <>
struct AElem<LAGKV_F32> {
  static constexpr int SIZE = 4, SUBS = 1, PAD = 16;
  static constexpr float UNIT = 1.44269504088896f;  // logits in natural units: the difference is scaled, not each of them
  static constexpr float LIFT = 0.f;
};
template <>
struct AElem<LAGKV_BF16> {
  static constexpr int SIZE = 2, SUBS = 2, PAD = 32;
  static constexpr float UNIT = 1.f;  // logits in base 2 (the scale holds the factor)
  static constexpr float LIFT = 0.f;
  static __device__ __forceinline__ f32x4 mma(u32v4 a, u32v4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float x, float y) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, bf16x2));
  }
  static __device__ __forceinline__ f32x2 unpack(uint32_t v) { return f32x2{__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)}; }
  static __device__ __forceinline__ float one(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
};
template <>
struct AElem<LAGKV_F16> {
  static constexpr int SIZE = 2, SUBS = 2, PAD = 32;
  static constexpr float UNIT = 1.f;  // logits in base 2 (the scale holds the factor)
  // exp(x - m) is held times 2^14: binary16 has no numbers between 0 and 2^-24, and a million rows of 2^-25 are no
  // trifle beside one of 1.  (l carries the same factor.)
  static constexpr float LIFT = 14.f;
  static __device__ __forceinline__ f32x4 mma(u32v4 a, u32v4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float x, float y) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, f16x2));
  }
  static __device__ __forceinline__ f32x2 unpack(uint32_t v) { return __builtin_convertvector(__builtin_bit_cast(f16x2, v), f32x2); }
  static __device__ __forceinline__ float one(uint16_t v) { return (float)__builtin_bit_cast(_Float16, v); }
};

// lse of a state, natural
template <int DT>
__device__ __forceinline__ float lse_of(float m, float l) {
  using E = AElem<DT>;
  if constexpr (DT == LAGKV_F32) return m + __builtin_amdgcn_logf(l) * 0.693147180559945f;
  return (m + __builtin_amdgcn_logf(l) - E::LIFT) * 0.693147180559945f;
}

// Channel at which the c-th 16-byte slice of a row of D begins: the last one of a row that is no whole number of slices
// is taken from the row's end, so that nothing behind the row is read.  The channels it shares with the slice before it
// are zeroed in q (they count once) and not stored (they come out twice).
__device__ __forceinline__ int slice_at(int c, int D, int per) {
  const int at = c * per;
  return at + per <= D ? at : D - per;
}

// The workgroup's unit, row tile and piece.  Tiles of one unit and piece read the same cache rows: they are dealt to
// workgroups whose numbers differ by multiples of eight, which share an L2.
struct WorkItem {
  int64_t unit;
  int tile, split;
  bool any;
};
__device__ __forceinline__ WorkItem work_item(const AttendArgs& a) {
  const int64_t id = blockIdx.x, slot = id % 8, rest = id / 8;
  const int64_t us = rest / a.row_tiles * 8 + slot;
  WorkItem w;
  w.tile = (int)(rest % a.row_tiles);
  w.any = us < a.units * a.splits;
  w.unit = us / a.splits;
  w.split = (int)(us % a.splits);
  return w;
}

template <int DT, int DP, int RT, bool PICK>
struct AttendShape {
  using E = AElem<DT>;
  static constexpr int WAVES = 4;
  static constexpr int PER = 16 / E::SIZE;         // elements of a slice
  static constexpr int NC = DP * E::SIZE / 64;     // slices of a row a lane holds
  static constexpr int KT = 16 * E::SUBS;          // cache rows of a step
  static constexpr int ROWS = 16 * RT;
  static constexpr int LDV = DP * E::SIZE + E::PAD;  // bytes between rows of V in LDS
  static constexpr int LDO = DP + 4;                 // floats between rows of the joined output
  static constexpr int V_BYTES = WAVES * KT * LDV;
  static constexpr int O_BYTES = ROWS * LDO * 4;
  static constexpr int MASK_WORDS = ROWS * (kMaxTree / 32);
  static constexpr int MAIN = V_BYTES > O_BYTES ? V_BYTES : O_BYTES;
};

template <int DT, int DP, int RT, bool PICK>
__global__ __launch_bounds__(256) void attend_kernel(const AttendArgs a) {
  using E = AElem<DT>;
  using Sh = AttendShape<DT, DP, RT, PICK>;
  constexpr int PER = Sh::PER, NC = Sh::NC, SUBS = E::SUBS, KT = Sh::KT, ROWS = Sh::ROWS, WAVES = Sh::WAVES;
  constexpr int LDV = Sh::LDV, LDO = Sh::LDO, DT16 = DP / 16;
  __shared__ __attribute__((aligned(16))) char lds[Sh::MAIN];
  __shared__ float sh_ml[WAVES][ROWS][2];
  __shared__ int32_t sh_parent[kMaxTree];
  __shared__ uint32_t sh_mask[Sh::MASK_WORDS];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 15, grp = lane >> 4;

  const WorkItem w = work_item(a);
  if (!w.any) return;
  const int n_fixed = PICK ? (int)(w.unit % a.N) : 0;
  const int64_t stream = PICK ? w.unit / a.N : w.unit;
  const int64_t b = stream / a.H, h = stream % a.H;
  const int row0 = w.tile * ROWS, row1 = min(row0 + ROWS, a.rows);  // query rows of this tile
  auto token_of = [&](int r) { return PICK ? n_fixed : r / a.G; };
  auto group_of = [&](int r) { return PICK ? r : r % a.G; };

  // rows this tile may see, in steps: of the cache, then of the new tokens (up to the tile's last one, where each sees
  // those before it)
  int64_t len = a.lengths ? a.lengths[b] : a.T;
  len = len < 0 ? 0 : len > a.T ? a.T : len;
  const int64_t listed = PICK ? (int64_t)a.n_blocks * a.block : len;
  const int64_t cache_steps = len > 0 ? (listed + KT - 1) / KT : 0;
  const int last_token = token_of(row1 - 1);
  const int seen_new = a.n_new > 0 ? (a.parents ? a.n_new : last_token + 1) : 0;
  const int64_t steps = cache_steps + (seen_new + KT - 1) / KT;
  const int64_t share = ((steps + a.splits - 1) / a.splits + WAVES - 1) / WAVES * WAVES;
  const int64_t step0 = w.split * share, step1 = step0 + share < steps ? step0 + share : steps;

  // which new tokens each of the tile's tokens sees, as bits
  const int words = (seen_new + 31) / 32, token0 = token_of(row0), tokens = last_token - token0 + 1;
  if (a.parents && step1 > cache_steps) {  // (uniform in the workgroup)
    const int32_t* parents = a.parents + b * a.psb;
    for (int i = tid; i < a.N; i += 256) sh_parent[i] = parents[i];
    for (int i = tid; i < tokens * words; i += 256) sh_mask[i] = 0;
    __syncthreads();
    if (tid < tokens) {
      // a parent comes before its child: the walk ends
      for (int at = token0 + tid; at >= 0;) {
        const int up = sh_parent[at];
        if (up < -1 || up >= at) break;  // not a token
        sh_mask[tid * words + (at >> 5)] |= 1u << (at & 31);
        at = up;
      }
    }
    __syncthreads();
  }

  // q: one row a lane
  u32v4 q[RT][NC];
  for (int rt = 0; rt < RT; ++rt) {
    const int r = row0 + rt * 16 + col;
    const bool ok = r < row1;
    const int rr = ok ? r : row0;
    const char* p = a.Q + b * a.qsb + (h * a.G + group_of(rr)) * a.qsh + (int64_t)token_of(rr) * a.qsn;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int slice = c * 4 + grp, begin = slice * PER;
      u32v4 v = {0, 0, 0, 0};
      if (ok && begin < a.D) {
        const int at = slice_at(slice, a.D, PER);
        v = *(const u32v4_any*)(p + at * E::SIZE);
        const int dup = begin - at;  // leading channels that the slice before has
        if (dup > 0) {
#pragma unroll
          for (int i = 0; i < PER; ++i)
            if (i < dup) {
              if constexpr (E::SIZE == 4) v[i] = 0;
              else v[i / 2] &= i % 2 ? 0x0000ffffu : 0xffff0000u;
            }
        }
      }
      q[rt][c] = v;
    }
  }

  float m[RT], l[RT];
  f32x4 o[RT][DT16];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m[rt] = -INFINITY;
    l[rt] = 0.f;
#pragma unroll
    for (int d = 0; d < DT16; ++d) o[rt][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const char* kb = a.K + b * a.ksb + h * a.ksh;
  const char* vb = a.V + b * a.ksb + h * a.ksh;
  const char* knb = a.K_new + b * a.nsb + h * a.nsh;
  const char* vnb = a.V_new + b * a.nsb + h * a.nsh;
  const int32_t* list = PICK ? a.blocks + w.unit * a.n_blocks : nullptr;
  const int64_t n_full = PICK ? (len + a.block - 1) >> a.block_shift : 0;
  char* vl = lds + wave * (KT * LDV);

  for (int64_t step = step0 + wave; step < step1; step += WAVES) {
    const bool fresh = step >= cache_steps;  // rows of the new tokens
    // first row of each 16 and how many rows there are
    int64_t first[SUBS], limit[SUBS];
#pragma unroll
    for (int s = 0; s < SUBS; ++s) {
      if (fresh) {
        first[s] = (step - cache_steps) * KT + s * 16;
        limit[s] = seen_new;
      } else if (!PICK) {
        first[s] = step * KT + s * 16;
        limit[s] = len;
      } else {
        const int64_t at = step * KT + s * 16;
        const int64_t e = at >> a.block_shift;
        const int id = e < a.n_blocks ? list[e] : -1;
        const bool ok = id >= 0 && id < n_full;
        first[s] = ok ? ((int64_t)id << a.block_shift) + (at & (a.block - 1)) : 0;
        limit[s] = ok ? len : 0;
      }
    }
    bool whole = true;
#pragma unroll
    for (int s = 0; s < SUBS; ++s) whole = whole && first[s] + 16 <= limit[s];
    const char* kp = fresh ? knb : kb;
    const char* vp = fresh ? vnb : vb;
    const int64_t st = fresh ? a.nst : a.kst;
    u32v4 kf[SUBS][NC], vf[SUBS][NC];
    bool odd = false;  // a value that is no number, or infinite
#pragma unroll
    for (int s = 0; s < SUBS; ++s) {
      int64_t row = first[s] + col;
      const bool in = row < limit[s];
      row = in ? row : 0;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int slice = c * 4 + grp;
        const bool have = slice * PER < a.D;
        const int64_t off = row * st + (have ? slice_at(slice, a.D, PER) : 0) * E::SIZE;
        kf[s][c] = *(const u32v4_any*)(kp + off);
        u32v4 v = *(const u32v4_any*)(vp + off);
        if (!in) v = u32v4{0, 0, 0, 0};
        vf[s][c] = v;
        if (fresh) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if constexpr (DT == LAGKV_F32) odd = odd || (v[i] & 0x7f800000u) == 0x7f800000u;
            if constexpr (DT == LAGKV_BF16) odd = odd || (v[i] & 0x7f80u) == 0x7f80u || (v[i] & 0x7f800000u) == 0x7f800000u;
            if constexpr (DT == LAGKV_F16) odd = odd || (v[i] & 0x7c00u) == 0x7c00u || (v[i] & 0x7c000000u) == 0x7c000000u;
          }
        }
      }
    }
    wave_order();
#pragma unroll
    for (int s = 0; s < SUBS; ++s)
#pragma unroll
      for (int c = 0; c < NC; ++c) *(u32v4*)(vl + (s * 16 + col) * LDV + (c * 4 + grp) * 16) = vf[s][c];
    wave_order();
    odd = __any(odd);

    f32x4 p[RT][SUBS];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int s = 0; s < SUBS; ++s) {
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        if constexpr (DT == LAGKV_F32) {
          // four sums of a quarter of the channels each: shorter chains, of steps and of roundings
          f32x4 y[4] = {x, x, x, x};
#pragma unroll
          for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              y[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[s][c][i]), __uint_as_float(q[rt][c][i]), y[i], 0, 0, 0);
          x = (y[0] + y[1]) + (y[2] + y[3]);
        } else {
#pragma unroll
          for (int c = 0; c < NC; ++c) x = E::mma(kf[s][c], q[rt][c], x);
        }
        p[rt][s] = x;
      }

    uint32_t seen[RT][SUBS];  // bits of the four cache rows a lane holds, for its query row
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float top = -INFINITY;
#pragma unroll
      for (int s = 0; s < SUBS; ++s) {
        uint32_t bits = 15u;
        if (!whole) {
          const int64_t left = limit[s] - (first[s] + grp * 4);
          bits = left >= 4 ? 15u : left <= 0 ? 0u : (1u << left) - 1u;
        }
        if (fresh) {
          const int r = min(row0 + rt * 16 + col, row1 - 1), n = token_of(r), j = (int)first[s] + grp * 4;
          if (a.parents) {
            bits &= sh_mask[(n - token0) * words + (j >> 5 < words ? j >> 5 : 0)] >> (j & 31);
          } else {
            const int upto = n - j + 1;
            bits &= upto >= 4 ? 15u : upto <= 0 ? 0u : (1u << upto) - 1u;
          }
        }
        seen[rt][s] = bits;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = p[rt][s][i] * a.scale;
          p[rt][s][i] = (bits >> i) & 1 ? x : -INFINITY;
          top = fmaxf(top, p[rt][s][i]);
        }
      }
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float before = m[rt], now = fmaxf(before, top);
      m[rt] = now;
      const float at = now == -INFINITY ? 0.f : now;
      const float keep = __builtin_amdgcn_exp2f((before - at) * E::UNIT);
      float sum = 0.f;
#pragma unroll
      for (int s = 0; s < SUBS; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          // (the difference first: its rounding is that of a number near zero)
          const float e = __builtin_amdgcn_exp2f((p[rt][s][i] - at) * E::UNIT + E::LIFT);
          p[rt][s][i] = e;
          sum += e;
        }
      l[rt] = l[rt] * keep + sum;
      if (__any(keep != 1.f)) {
#pragma unroll
        for (int d = 0; d < DT16; ++d) o[rt][d] *= keep;
      }
    }

    if (odd) {
      // an infinite or undefined value in a new token's row must not reach those that do not see it, as 0 * inf would
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          float w4[SUBS];
#pragma unroll
          for (int s = 0; s < SUBS; ++s) {
            const int i = t & 3;
            w4[s] = i == 0 ? p[rt][s][0] : i == 1 ? p[rt][s][1] : i == 2 ? p[rt][s][2] : p[rt][s][3];
          }
          const int from = ((t & 15) >> 2) * 16 + col;
          const float e = __shfl(SUBS == 2 && t >= 16 ? w4[SUBS - 1] : w4[0], from);
          const uint32_t bits = __shfl(SUBS == 2 && t >= 16 ? seen[rt][SUBS - 1] : seen[rt][0], from);
          const bool see = (bits >> (t & 3)) & 1;
#pragma unroll
          for (int d = 0; d < DT16; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const char* at = vl + t * LDV + (d * 16 + grp * 4 + i) * E::SIZE;
              float v;
              if constexpr (DT == LAGKV_F32) v = *(const float*)at;
              else v = E::one(*(const uint16_t*)at);
              if (see) o[rt][d][i] += e * v;
            }
        }
    } else if constexpr (DT == LAGKV_F32) {
#pragma unroll
      for (int d = 0; d < DT16; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float v = *(const float*)(vl + (grp * 4 + i) * LDV + (d * 16 + col) * 4);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) o[rt][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, p[rt][0][i], o[rt][d], 0, 0, 0);
        }
    } else {
      u32v4 ph[RT], pl[RT];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int s = 0; s < SUBS; ++s)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float x = p[rt][s][2 * i], y = p[rt][s][2 * i + 1];
            const uint32_t hi = E::pack(x, y);
            const f32x2 back = E::unpack(hi);
            ph[rt][s * 2 + i] = hi;
            pl[rt][s * 2 + i] = E::pack(x - back.x, y - back.y);
          }
#pragma unroll
      for (int d = 0; d < DT16; ++d) {
        u32v4 v;
#pragma unroll
        for (int s = 0; s < SUBS; ++s) {
          const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (lds_s16x4)(vl + (s * 16 + grp * 4 + (col >> 2)) * LDV + (d * 16 + (col & 3) * 4) * 2));
          const u32v2 y = __builtin_bit_cast(u32v2, x);
          v[s * 2] = y.x;
          v[s * 2 + 1] = y.y;
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          o[rt][d] = E::mma(v, ph[rt], o[rt][d]);
          o[rt][d] = E::mma(v, pl[rt], o[rt][d]);
        }
      }
    }
  }

  // the four states join: maxima and sums first, then the outputs one wavefront after another
  __syncthreads();
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float sum = l[rt];
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (grp == 0) {
      sh_ml[wave][rt * 16 + col][0] = m[rt];
      sh_ml[wave][rt * 16 + col][1] = sum;
    }
  }
  __syncthreads();
  float* ol = (float*)lds;
  for (int turn = 0; turn < WAVES; ++turn) {
    if (wave == turn) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float top = -INFINITY;
#pragma unroll
        for (int x = 0; x < WAVES; ++x) top = fmaxf(top, sh_ml[x][rt * 16 + col][0]);
        const float f = m[rt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m[rt] - top) * E::UNIT);
        const bool none = m[rt] == -INFINITY;
#pragma unroll
        for (int d = 0; d < DT16; ++d) {
          f32x4* at = (f32x4*)(ol + (rt * 16 + col) * LDO + d * 16 + grp * 4);
          f32x4 v = none ? f32x4{0.f, 0.f, 0.f, 0.f} : o[rt][d] * f;
          if (turn > 0) v += *at;
          *at = v;
        }
      }
    }
    __syncthreads();
  }

  // out: a row's slices, four slots of them a thread
  constexpr int QUADS = DP / 4;
  for (int i = tid; i < ROWS * QUADS; i += 256) {
    const int rl = i / QUADS, quad = i % QUADS, r = row0 + rl;
    if (r >= row1) continue;
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int x = 0; x < WAVES; ++x) top = fmaxf(top, sh_ml[x][rl][0]);
#pragma unroll
    for (int x = 0; x < WAVES; ++x) {
      const float mx = sh_ml[x][rl][0];
      if (mx != -INFINITY) sum += sh_ml[x][rl][1] * __builtin_amdgcn_exp2f((mx - top) * E::UNIT);
    }
    const f32x4 v = *(const f32x4*)(ol + rl * LDO + quad * 4);
    const int slot = quad * 4, slice = slot / PER, own_at = slice * PER;
    if (a.splits > 1) {
      const int64_t at = (w.unit * a.splits + w.split) * a.rows + r;
      if (own_at < a.D) {
        const int shift = own_at - slice_at(slice, a.D, PER);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int ch = slot + e - shift;
          if (slot + e - own_at >= shift && ch < a.D) a.part_o[at * a.part_ld + ch] = v[e];
        }
      }
      if (quad == 0) {
        a.part_ml[at * 2] = top;
        a.part_ml[at * 2 + 1] = sum;
      }
      continue;
    }
    const int n = token_of(r);
    const int64_t head = h * a.G + group_of(r);
    bool blind = sum == 0.f;
    if (a.parents) {
      const int up = a.parents[b * a.psb + n];
      blind = blind || up < -1 || up >= n;
    }
    const float inv = blind ? 0.f : 1.f / sum;
    if (own_at < a.D) {
      const int shift = own_at - slice_at(slice, a.D, PER);
      char* op = a.out + b * a.osb + head * a.osh + (int64_t)n * a.osn;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int ch = slot + e - shift;
        if (slot + e - own_at >= shift && ch < a.D) {
          const float y = blind ? 0.f : v[e] * inv;
          if constexpr (DT == LAGKV_F32) *(float*)(op + ch * 4) = y;
          else *(uint16_t*)(op + ch * 2) = (uint16_t)E::pack(y, 0.f);
        }
      }
    }
    if (quad == 0 && a.lse)
      a.lse[(b * a.H * a.G + head) * a.N + n] = blind ? -INFINITY : lse_of<DT>(top, sum);
  }
}

// Row tiles by the registers they take: 16 query rows of 256 channels or 32 of 128 are what a lane holds without spilling.
template <int DT, int DP, int RT>
hipError_t launch_attend_as(const AttendArgs& a, hipStream_t s) {
  const int64_t groups = (a.units * a.splits + 7) / 8 * 8 * a.row_tiles;
  if (a.blocks) attend_kernel<DT, DP, RT, true><<<dim3((uint32_t)groups), dim3(256), 0, s>>>(a);
  else attend_kernel<DT, DP, RT, false><<<dim3((uint32_t)groups), dim3(256), 0, s>>>(a);
  return hipGetLastError();
}

template <int DT>
hipError_t launch_attend_of(const AttendArgs& a, int row_tile, hipStream_t s) {
  const int rt = row_tile / 16;
  if (a.D <= 64) return rt == 1 ? launch_attend_as<DT, 64, 1>(a, s) : launch_attend_as<DT, 64, 2>(a, s);
  if (a.D <= 128) return rt == 1 ? launch_attend_as<DT, 128, 1>(a, s) : launch_attend_as<DT, 128, 2>(a, s);
  return launch_attend_as<DT, 256, 1>(a, s);
}

}  // namespace lagkv
