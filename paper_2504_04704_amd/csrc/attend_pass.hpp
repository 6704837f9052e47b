// Attention of new tokens over a cache and over themselves (lagkv_attend, lagkv_attend_blocks).
//
// For a query row q and the rows (k_t, v_t) that it sees, with x_t = scale * q.k_t:
//     m = max x_t,  l = sum exp(x_t - m),  out = sum exp(x_t - m) v_t / l,  lse = m + log l
// in one pass over the rows: a wavefront that has gone over some of them holds m, l and o = sum exp(x_t - m) v_t, and
// two such states (m1, l1, o1), (m2, l2, o2) join to m = max(m1, m2), l = l1 e^(m1-m) + l2 e^(m2-m), o likewise.  All of
// it is held in fp32, in base 2 (exp2 is the hardware's).
//
// A workgroup of four wavefronts (eight for short caches) takes a tile of 16 or 32 query rows of a unit and a piece of its
// cache rows; each wavefront takes every fourth (eighth) step of 32 rows (16 in fp32) for all query rows, so nothing is
// shared until their states join at the end.  Both products go to the matrix cores, transposed:
//     S^T = K Q^T     (rows of K, as they lie in memory, are the operand whose k index runs along a lane's registers)
//     O^T += V^T P^T  (S^T leaves the matrix core with one query row a lane and four cache rows in its registers, which
//                      is how P^T has to be put in: nothing moves between lanes)
// V^T needs four cache rows of one channel in a lane: V goes through LDS, into memory private to the wavefront, and
// comes back through the transposing read (16-bit types) or element by element (fp32).
//
// P is put in as the sum of two 16-bit numbers (the value's leading bits, and the rest): one alone would add as
// much error to the output as its own rounding, and the pass is bound by memory where tiles are small.
//
// Bound by memory where the rows of K and V are many (four query rows of 256 streams of up to 8384 rows, bf16: 155 us,
// 5.4 TB/s, where a copy reaches 5.07; 32 streams x 8192 rows 28 us; fp32 55 us), by latency where they are few (one token,
// 8 streams x 4288 rows: 9.4 us and 2.5 for joining the pieces, at the copy's rate 3.5), by the products for 32 fp32 rows and more
// (256 rows of 32 streams x 8192, 326 us: 105 Tflop/s of the 151 of a large product).  The next step's K and V
// are on their way, in registers, while one is worked on.
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

// x of this lane and of the lane 32 (16) away, joined
__device__ __forceinline__ float max_across_32(float x) {
  const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}
__device__ __forceinline__ float max_across_16(float x) {
  const auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}
__device__ __forceinline__ float sum_across_32(float x) {
  const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(y[0]) + __uint_as_float(y[1]);
}

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
  // Weights x and y >= 0 as pairs of numbers of the type: their leading bits, and the rest rounded.  The rest is above 0 if the
  // weight is: both parts' products with an infinity then add up to it, and are NaN with a rest of 0 or below.  It has
  // 2^-22 of the weight too much for that (the rounding of the rest leaves 2^-15).
  static __device__ __forceinline__ void split(float x, float y, uint32_t& hi, uint32_t& lo) {
    const uint32_t a = __float_as_uint(x), b = __float_as_uint(y);
    hi = __builtin_amdgcn_perm(b, a, 0x07060302);
    lo = pack(__builtin_fmaf(x, 1 + 0x1p-22f, -__uint_as_float(a & 0xffff0000u)), __builtin_fmaf(y, 1 + 0x1p-22f, -__uint_as_float(b & 0xffff0000u)));
  }
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
  // (here the rest has to be of the smallest number at least; x - lead <= x, so that the middle one of the three is that)
  static __device__ __forceinline__ void split(float x, float y, uint32_t& hi, uint32_t& lo) {
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(x, y));
    const f32x2 back = __builtin_convertvector(__builtin_bit_cast(f16x2, hi), f32x2);
    lo = pack(__builtin_amdgcn_fmed3f(x - back.x, 0x1p-24f, x), __builtin_amdgcn_fmed3f(y - back.y, 0x1p-24f, y));
  }
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
// are zeroed in q and in k (they count once, and 0 alone in one of them would make an infinity there NaN) and not stored (they
// come out twice).
__device__ __forceinline__ int slice_at(int c, int D, int per) {
  const int at = c * per;
  return at + per <= D ? at : D - per;
}
// The slice v that begins at channel `begin` of a row of D, in place of which slice_at's was loaded: 0 where it has no channels of
// its own.  (Worked out where it is used: kept, the conditions take more scalar registers than there are.)
template <int PER>
__device__ __forceinline__ u32v4 own_channels(u32v4 v, int begin, int D) {
  asm volatile("" : "+v"(begin));
  if (begin >= D) v = u32v4{0, 0, 0, 0};
  if (D % PER != 0) {
    const bool part = begin < D && begin + PER > D;
    const int dup = PER - D % PER;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t own = PER == 4 ? (i < dup ? 0u : ~0u) : (2 * i < dup ? 0u : 0x0000ffffu) | (2 * i + 1 < dup ? 0u : 0xffff0000u);
      v[i] &= part ? own : ~0u;
    }
  }
  return v;
}

// Asks for every line of the kernel's arguments at once.  They lie in host memory, and the compiler loads them where they
// are used: one line after another, each a trip of its own for the first workgroups of a compute unit.
template <typename T>
__device__ __forceinline__ void fetch_arguments() {
  typedef const __attribute__((address_space(4))) uint32_t* args_t;
  const args_t p = (args_t)__builtin_amdgcn_kernarg_segment_ptr();
  constexpr int LINES = (int)(sizeof(T) + 63) / 64;
  uint32_t x[LINES];
#pragma unroll
  for (int i = 0; i < LINES; ++i) x[i] = p[16 * i];
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < LINES; ++i) any |= x[i];
  asm volatile("" ::"s"(any));
}

// The kernel's arguments, loaded where they are used next: for a part that hardly ever runs, so that the others' registers do not hold
// what it needs.
template <typename T>
__device__ __forceinline__ const T& arguments_again() {
  typedef const __attribute__((address_space(4))) T* args_t;
  args_t p = (args_t)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const T*)p;
}

// The workgroup's unit, row tile and piece.  Tiles of one unit and piece read the same cache rows: they are dealt to
// workgroups whose numbers differ by multiples of eight, which share an L2.
struct WorkItem {
  int64_t unit;
  int tile, split;
  bool any;
};
template <typename Args>
__device__ __forceinline__ WorkItem work_item(const Args& a, uint32_t group = blockIdx.x) {
  const uint32_t slot = group % 8, rest = group / 8, many = a.by_tiles.of(rest), us = many * 8 + slot;
  const uint32_t unit = a.by_splits.of(us);
  WorkItem w;
  w.tile = (int)(rest - many * a.row_tiles);
  w.any = unit < (uint32_t)a.units;
  w.unit = unit;
  w.split = (int)(us - unit * a.splits);
  return w;
}

// Which new tokens each of a tile's tokens sees, as bits: `words` words a token.  A parent comes before its child: the walk ends.
__device__ __forceinline__ void ancestors(const int32_t* parents, int N, int token0, int tokens, int words, int32_t* sh_parent,
                                          uint32_t* sh_mask, int tid, int threads) {
  for (int i = tid; i < N; i += threads) sh_parent[i] = parents[i];
  for (int i = tid; i < tokens * words; i += threads) sh_mask[i] = 0;
  __syncthreads();
  if (tid < tokens)
    for (int at = token0 + tid; at >= 0;) {
      const int up = sh_parent[at];
      if (up < -1 || up >= at) break;  // not a token
      sh_mask[tid * words + (at >> 5)] |= 1u << (at & 31);
      at = up;
    }
}

// All ones in each number of a pair (fp32: in the number) that is infinite or none
template <int DT>
__device__ __forceinline__ uint32_t odd_bits(uint32_t v) {
  constexpr uint32_t EXP = DT == LAGKV_F32 ? 0x7f800000u : DT == LAGKV_BF16 ? 0x7f80u : 0x7c00u;
  if constexpr (DT == LAGKV_F32) return (v & EXP) == EXP ? ~0u : 0u;
  return ((v & EXP) == EXP ? 0x0000ffffu : 0u) | ((v >> 16 & EXP) == EXP ? 0xffff0000u : 0u);
}
// What four channels of a row have of such numbers, added to o
template <int DT>
__device__ __forceinline__ void add_odd(const char* at, float* o) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (DT == LAGKV_F32) {
      const float v = ((const float*)at)[i];
      if (odd_bits<DT>(__float_as_uint(v))) o[i] += v;
    } else {
      const uint16_t v = ((const uint16_t*)at)[i];
      if (odd_bits<DT>(v)) o[i] += AElem<DT>::one(v);
    }
  }
}

template <int DT, int DP, int RT, int WAVES>
struct AttendShape {
  using E = AElem<DT>;
  static constexpr int PER = 16 / E::SIZE;           // elements of a slice
  static constexpr int CPR = DP / PER;               // slices of a row
  static constexpr int NC = CPR / 4;                 // of those, a lane holds of K
  static constexpr int KT = 16 * E::SUBS;            // cache rows of a step
  static constexpr int ROWS = 16 * RT;
  static constexpr int LDV = DP * E::SIZE + E::PAD;  // bytes between rows of V in LDS
  static constexpr int LDO = DP + 4;                 // floats between rows of the outputs in LDS
  static constexpr int V_BYTES = WAVES * KT * LDV, O_BYTES = WAVES * ROWS * LDO * 4;
  static constexpr int MAIN = V_BYTES > O_BYTES ? V_BYTES : O_BYTES;
};

// Two wavefronts a SIMD where 256 registers do for each (the compiler then keeps all in vector registers; with 512 it
// moves the outputs in and out of the accumulators' in every step).
template <int DT, int DP, int RT>
constexpr int kAttendWaves = DP > 128 ? 1 : 2;
// 32 fp32 rows of 128 channels: q in LDS, one copy for the workgroup, where V's rows leave room beside them, for 256 to do.
template <int DT, int DP, int RT>
constexpr bool kQueryInLds = DT == LAGKV_F32 && DP == 128 && RT == 2;

// The kernels are also those of lagkv_attend_quantized's tail and new tokens: `Part` says what else a workgroup does.  (What follows is a kernel's own text, and not a
// function of two kernels': as one it had twice the scalars spilled, read back lane by lane in the loops, and took up to 3 % longer.)
struct RowsAlone {
  using Args = AttendArgs;
  static constexpr bool ALONE = true;
  static __device__ __forceinline__ const AttendArgs& rows(const Args& a) { return a; }
};

template <int DT, int DP, int RT, int WAVES, bool PICK, typename Part>
__global__ __launch_bounds__(WAVES * 64, (kAttendWaves<DT, DP, RT>)) void attend_kernel(const typename Part::Args args) {
  using E = AElem<DT>;
  using Sh = AttendShape<DT, DP, RT, WAVES>;
  constexpr int PER = Sh::PER, NC = Sh::NC, CPR = Sh::CPR, SUBS = E::SUBS, KT = Sh::KT, ROWS = Sh::ROWS, THREADS = WAVES * 64;
  constexpr int LDV = Sh::LDV, LDO = Sh::LDO, DT16 = DP / 16, NV = SUBS * NC, VROWS = 64 / CPR;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ float sh_ml[WAVES][ROWS][2];
  __shared__ int32_t sh_parent[kMaxTree];
  __shared__ uint32_t sh_mask[ROWS * (kMaxTree / 32)];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 15, grp = lane >> 4;

  fetch_arguments<typename Part::Args>();
  const AttendArgs& a = Part::rows(args);
  uint32_t group = blockIdx.x;
  if constexpr (!Part::ALONE) {
    if (group < args.groups) return Part::go(args, lds);
    group -= args.groups;
  }
  const WorkItem w = work_item(a, group);
  if (!w.any) return;
  const uint32_t stream = PICK ? a.by_n.of((uint32_t)w.unit) : (uint32_t)w.unit, bu = a.by_h.of(stream);
  const int n_fixed = PICK ? (int)((uint32_t)w.unit - stream * a.N) : 0;
  const int64_t b = bu, h = stream - bu * a.H;
  const int row0 = w.tile * ROWS, row1 = min(row0 + ROWS, a.rows);  // query rows of this tile
  auto token_of = [&](int r) { return PICK ? n_fixed : (int)a.by_g.of(r); };
  auto group_of = [&](int r) { return PICK ? r : r - (int)a.by_g.of(r) * a.G; };

  // rows this tile may see, in steps: of the cache, then of the new tokens (up to the tile's last one, where each sees
  // those before it)
  int64_t held = a.lengths ? a.lengths[b] : a.T;
  const int len = (int)(held < 0 ? 0 : held > a.T ? a.T : held);
  const int listed = PICK ? a.n_blocks << a.block_shift : len;
  const int cache_steps = len > 0 ? (int)(((int64_t)listed + KT - 1) / KT) : 0;
  const int last_token = token_of(row1 - 1), token0 = token_of(row0), tokens = last_token - token0 + 1;
  const int seen_new = a.n_new > 0 ? (a.parents ? a.n_new : last_token + 1) : 0, words = (seen_new + 31) / 32;
  const int steps = cache_steps + (seen_new + KT - 1) / KT;
  const int step0 = (int)((int64_t)steps * w.split / a.splits), step1 = (int)((int64_t)steps * (w.split + 1) / a.splits);
  const char* kb = a.K + b * a.ksb + h * a.ksh;
  const char* vb = a.V + b * a.ksb + h * a.ksh;
  const char* knb = a.K_new + b * a.nsb + h * a.nsh;
  const char* vnb = a.V_new + b * a.nsb + h * a.nsh;
  const int32_t* list = PICK ? a.blocks + w.unit * a.n_blocks : nullptr;
  const int n_full = PICK ? (int)(((int64_t)len + a.block - 1) >> a.block_shift) : 0;
  char* vl = lds + wave * (KT * LDV);

  // A step: the first row of each sixteen, and how many rows there are.
  struct Step {
    int first[SUBS], limit[SUBS];
    int fresh;  // (of the new tokens)
    int whole;  // rows of the cache, all there
  };
  // (lane i has the entries of this wavefront's step i, or 64 + i, ...: one wait for all of them)
  int ids[SUBS];
  auto entries = [&](int step) {
    if constexpr (PICK) {
#pragma unroll
      for (int s = 0; s < SUBS; ++s) {
        const int at = step + lane * WAVES, e = (int)(((int64_t)at * KT + s * 16) >> a.block_shift);
        ids[s] = at < cache_steps && e < a.n_blocks ? list[e] : -1;
      }
    }
  };
  auto step_of = [&](int step, int turn) {  // the turn-th of this wavefront
    Step x;
    x.fresh = step >= cache_steps;
#pragma unroll
    for (int s = 0; s < SUBS; ++s) {
      if (x.fresh) {
        x.first[s] = (step - cache_steps) * KT + s * 16;
        x.limit[s] = seen_new;
      } else if (!PICK) {
        x.first[s] = step * KT + s * 16;
        x.limit[s] = len;
      } else {
        const int id = __builtin_amdgcn_readlane(ids[s], turn & 63);
        const bool ok = id >= 0 && id < n_full;
        x.first[s] = ok ? (id << a.block_shift) + ((step * KT + s * 16) & (a.block - 1)) : 0;
        x.limit[s] = ok ? len : 0;
      }
    }
    x.whole = !x.fresh;
#pragma unroll
    for (int s = 0; s < SUBS; ++s) x.whole = x.whole && x.first[s] + 16 <= x.limit[s];
    return x;
  };
  // K: lane (col, grp) has row col of each sixteen, slices grp, 4 + grp, ...: what its operand takes.  V: whole rows, a slice
  // a lane.  Slices behind a row's last repeat another: q and K are made 0 there, and what V gives for them is not stored.
  u32v4 kf[SUBS][NC], vf[NV];
  const int vslice = lane % CPR, vrow = lane / CPR;
  auto offset = [&](int slice) { return (slice * PER < a.D ? slice_at(slice, a.D, PER) : 0) * E::SIZE; };
  int koff[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) koff[c] = offset(c * 4 + grp);
  auto own = [&](int c, u32v4 v) { return own_channels<PER>(v, (c * 4 + grp) * PER, a.D); };
  const int64_t klane = (int64_t)col * a.kst, vlane = (int64_t)vrow * a.kst + offset(vslice), vpass = a.kst * VROWS;
  auto load_k = [&](const Step& x) {
    if (x.whole) {
#pragma unroll
      for (int s = 0; s < SUBS; ++s) {
        const char* at = kb + (int64_t)x.first[s] * a.kst + klane;
#pragma unroll
        for (int c = 0; c < NC; ++c)
          kf[s][c] = *(const u32v4_any*)(at + (DP > 64 && c < NC / 2 ? koff[0] + c * 64 : koff[c]));  // (D is more than DP / 2 there)
      }
      return;
    }
    const char* p = x.fresh ? knb : kb;
    const int64_t st = x.fresh ? a.nst : a.kst;
#pragma unroll
    for (int s = 0; s < SUBS; ++s) {
      const int row = x.first[s] + col;
      const char* at = p + (int64_t)(row < x.limit[s] ? row : 0) * st;
#pragma unroll
      for (int c = 0; c < NC; ++c) kf[s][c] = *(const u32v4_any*)(at + koff[c]);
    }
  };
  auto load_v = [&](const Step& x) {
    if (x.whole) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int s = i * VROWS / 16;
        vf[i] = *(const u32v4_any*)(vb + (int64_t)x.first[s] * a.kst + (i - s * 16 / VROWS) * vpass + vlane);
      }
      return;
    }
    const char* p = (x.fresh ? vnb : vb) + offset(vslice);
    const int64_t st = x.fresh ? a.nst : a.kst;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int s = i * VROWS / 16, row = x.first[s] + i * VROWS % 16 + vrow;
      vf[i] = *(const u32v4_any*)(p + (int64_t)(row < x.limit[s] ? row : 0) * st);
    }
  };

  entries(step0 + wave);
  // q: one row a lane
  u32v4 q[RT][NC];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = row0 + rt * 16 + col;
    const int rr = r < row1 ? r : row0;
    const char* p = a.Q + b * a.qsb + (h * a.G + group_of(rr)) * a.qsh + (int64_t)token_of(rr) * a.qsn;
#pragma unroll
    for (int c = 0; c < NC; ++c) q[rt][c] = *(const u32v4_any*)(p + koff[c]);
  }

  int step = step0 + wave, turn = 0;
  Step now;
  if (step < step1) {
    now = step_of(step, 0);
    load_k(now);
    load_v(now);
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

  if (a.parents && step1 > cache_steps && step0 < step1) {  // (uniform in the workgroup)
    ancestors(a.parents + b * a.psb, a.N, token0, tokens, words, sh_parent, sh_mask, tid, THREADS);
    __syncthreads();
  }
  // q's channels that the slice before has, and those behind its row's end, are 0.  (It is waited for here, behind the
  // first rows' loads, and not in every step.)
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      u32v4 v = own(c, q[rt][c]);
      if (row0 + rt * 16 + col >= row1) v = u32v4{0, 0, 0, 0};
      asm volatile("" : "+v"(v));
      q[rt][c] = v;
    }
  constexpr bool QLDS = kQueryInLds<DT, DP, RT>;
  char* ql = lds + Sh::V_BYTES + lane * 16;
  if constexpr (QLDS) {
    static_assert(Sh::V_BYTES + RT * NC * 1024 <= Sh::MAIN, "");
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (c % WAVES == wave) *(u32v4*)(ql + (rt * NC + c) * 1024) = q[rt][c];
    __syncthreads();
  }
  auto query = [&](int rt, int c) {
    if constexpr (QLDS) return *(const u32v4*)(ql + (rt * NC + c) * 1024);
    else return q[rt][c];
  };

  for (; step < step1; step += WAVES) {
    const bool more = step + WAVES < step1;
    Step next = now;
    ++turn;
    if (more) {
      if (PICK && (turn & 63) == 0) entries(step + WAVES);
      next = step_of(step + WAVES, turn);
    }
    // V into LDS, rows that are not there as zeros, and the next step's on its way
    bool odd = false;
    wave_order();
    if (!now.whole) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int s = i * VROWS / 16;
        if (now.first[s] + i * VROWS % 16 + vrow >= now.limit[s]) vf[i] = u32v4{0, 0, 0, 0};
        if (now.fresh) {
          // what is no finite number goes in as 0 (0 * inf is not) and is added to the query rows that see it afterwards
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t bits = odd_bits<DT>(vf[i][e]);
            odd = odd || bits;
            vf[i][e] &= ~bits;
          }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) *(u32v4*)(vl + (i * VROWS + vrow) * LDV + vslice * 16) = vf[i];
    wave_order();
    if (more) load_v(next);
    __builtin_amdgcn_sched_barrier(0);

    if (a.D != DP) {
#pragma unroll
      for (int s = 0; s < SUBS; ++s)
#pragma unroll
        for (int c = DP > 64 ? NC / 2 : 0; c < NC; ++c) kf[s][c] = own(c, kf[s][c]);
    }
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
          for (int c = 0; c < NC; ++c) {
            const u32v4 qv = query(rt, c);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              y[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[s][c][i]), __uint_as_float(qv[i]), y[i], 0, 0, 0);
          }
          x = (y[0] + y[1]) + (y[2] + y[3]);
        } else {
#pragma unroll
          for (int c = 0; c < NC; ++c) x = E::mma(kf[s][c], query(rt, c), x);
        }
        p[rt][s] = x;
      }
    __builtin_amdgcn_sched_barrier(0);
    if (more) load_k(next);
    __builtin_amdgcn_sched_barrier(0);

#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
      for (int s = 0; s < SUBS; ++s) p[rt][s] *= a.scale;
      if (!now.whole) {
#pragma unroll
        for (int s = 0; s < SUBS; ++s) {
          const int j = now.first[s] + grp * 4, left = now.limit[s] - j;
          uint32_t bits = left >= 4 ? 15u : left <= 0 ? 0u : (1u << left) - 1u;
          if (now.fresh) {
            const int n = token_of(min(row0 + rt * 16 + col, row1 - 1));
            if (a.parents) {
              bits &= sh_mask[(n - token0) * words + min(j >> 5, words - 1)] >> (j & 31);
            } else {
              const int upto = n - j + 1;
              bits &= upto >= 4 ? 15u : upto <= 0 ? 0u : (1u << upto) - 1u;
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!(bits >> i & 1)) p[rt][s][i] = -INFINITY;
        }
      }
      float top = p[rt][0][0];
#pragma unroll
      for (int s = 0; s < SUBS; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, p[rt][s][i]);
      top = max_across_32(max_across_16(top));
      const float before = m[rt];
      m[rt] = fmaxf(before, top);
      const float at = m[rt] == -INFINITY ? 0.f : m[rt];
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

    if constexpr (DT == LAGKV_F32) {
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
            uint32_t hi, lo;
            E::split(p[rt][s][2 * i], p[rt][s][2 * i + 1], hi, lo);
            ph[rt][s * 2 + i] = hi;
            pl[rt][s * 2 + i] = lo;
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
    if (now.fresh && __any(odd)) {
      for (int j = now.first[0]; j < now.first[0] + KT && j < seen_new; ++j) {
        const char* row = vnb + (int64_t)j * a.nst;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          const int n = token_of(min(row0 + rt * 16 + col, row1 - 1));
          if (!(a.parents ? sh_mask[(n - token0) * words + (j >> 5)] >> (j & 31) & 1 : j <= n)) continue;
#pragma unroll
          for (int d = 0; d < DT16; ++d) {
            const int slot = d * 16 + grp * 4;
            if (slot / PER * PER >= a.D) continue;
            float v[4] = {o[rt][d][0], o[rt][d][1], o[rt][d][2], o[rt][d][3]};
            add_odd<DT>(row + (slice_at(slot / PER, a.D, PER) + slot % PER) * E::SIZE, v);
            o[rt][d] = f32x4{v[0], v[1], v[2], v[3]};
          }
        }
      }
    }
    now = next;
  }

  // the wavefronts' states join: maxima and sums, then each writes its outputs, scaled to the common maximum
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
  __syncthreads();  // (V of all wavefronts is done with as well)
  float* ol = (float*)lds;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float top = -INFINITY;
#pragma unroll
    for (int x = 0; x < WAVES; ++x) top = fmaxf(top, sh_ml[x][rt * 16 + col][0]);
    const bool none = sh_ml[wave][rt * 16 + col][1] == 0.f;  // (what is no number has a maximum of -inf too, and is not dropped)
    const float f = none ? 0.f : __builtin_amdgcn_exp2f((m[rt] - top) * E::UNIT);
#pragma unroll
    for (int d = 0; d < DT16; ++d)
      *(f32x4*)(ol + (wave * ROWS + rt * 16 + col) * LDO + d * 16 + grp * 4) = none ? f32x4{0.f, 0.f, 0.f, 0.f} : o[rt][d] * f;
  }
  __syncthreads();

  // out: four slots of a row a thread
  constexpr int QUADS = DP / 4;
  const bool slices = a.D % PER == 0;
  const bool wide_out = slices && !(((uintptr_t)a.out | a.osb | a.osh | a.osn) & (4 * E::SIZE - 1));
  for (int i = tid; i < ROWS * QUADS; i += THREADS) {
    const int rl = i / QUADS, quad = i % QUADS, r = row0 + rl;
    if (r >= row1) continue;
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int x = 0; x < WAVES; ++x) top = fmaxf(top, sh_ml[x][rl][0]);
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < WAVES; ++x) {
      const float lx = sh_ml[x][rl][1];
      if (lx != 0.f) sum += lx * __builtin_amdgcn_exp2f((sh_ml[x][rl][0] - top) * E::UNIT);
      v += *(const f32x4*)(ol + (x * ROWS + rl) * LDO + quad * 4);
    }
    // the slots' channels: `dup` leading ones of a slice are the slice before's
    const int slot = quad * 4, begin = slot / PER * PER;
    const int base = begin < a.D ? slice_at(slot / PER, a.D, PER) : 0, dup = begin - base, within = slot - begin;
    const int pieces = Part::ALONE ? a.splits : a.part_splits;
    if (pieces > 1) {
      const int64_t at = (w.unit * pieces + (Part::ALONE ? 0 : a.part_first) + w.split) * a.rows + r;
      if (slices && begin < a.D) {
        *(f32x4*)(a.part_o + at * a.part_ld + slot) = v;
      } else if (begin < a.D) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (within + e >= dup) a.part_o[at * a.part_ld + base + within + e] = v[e];
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
    if (begin < a.D) {
      char* op = a.out + b * a.osb + head * a.osh + (int64_t)n * a.osn;
      const f32x4 y = blind ? f32x4{0.f, 0.f, 0.f, 0.f} : v * inv;
      if (wide_out) {
        if constexpr (DT == LAGKV_F32) *(f32x4*)(op + slot * 4) = y;
        else *(u32v2*)(op + slot * 2) = u32v2{E::pack(y[0], y[1]), E::pack(y[2], y[3])};
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (within + e >= dup) {
            const int ch = base + within + e;
            if constexpr (DT == LAGKV_F32) *(float*)(op + ch * 4) = y[e];
            else *(uint16_t*)(op + ch * 2) = (uint16_t)E::pack(y[e], 0.f);
          }
      }
    }
    if (quad == 0 && a.lse) a.lse[(b * a.H * a.G + head) * a.N + n] = blind ? -INFINITY : lse_of<DT>(top, sum);
  }
}

template <int DT, int DP, int RT, int WAVES, bool PICK>
hipError_t launch_attend_one(const AttendArgs& a, hipStream_t s) {
  const int64_t groups = (a.units * a.splits + 7) / 8 * 8 * a.row_tiles;
  constexpr size_t lds = AttendShape<DT, DP, RT, WAVES>::MAIN;
  auto kernel = attend_kernel<DT, DP, RT, WAVES, PICK, RowsAlone>;
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  kernel<<<dim3((uint32_t)groups), dim3(WAVES * 64), lds, s>>>(a);
  return hipGetLastError();
}
template <int DT, int DP, int RT, int WAVES>
hipError_t launch_attend_as(const AttendArgs& a, hipStream_t s) {
  return a.blocks ? launch_attend_one<DT, DP, RT, WAVES, true>(a, s) : launch_attend_one<DT, DP, RT, WAVES, false>(a, s);
}

// Row tiles by the registers they take: 16 query rows of 256 channels or 32 of 128 are what a lane holds without spilling.
template <int DT>
hipError_t launch_attend_of(const AttendArgs& a, int row_tile, int waves, hipStream_t s) {
  const bool one = row_tile == 16;
  if (one && waves == 8) return a.D <= 64 ? launch_attend_as<DT, 64, 1, 8>(a, s) : launch_attend_as<DT, 128, 1, 8>(a, s);
  if (a.D <= 64) return one ? launch_attend_as<DT, 64, 1, 4>(a, s) : launch_attend_as<DT, 64, 2, 4>(a, s);
  if (a.D <= 128) return one ? launch_attend_as<DT, 128, 1, 4>(a, s) : launch_attend_as<DT, 128, 2, 4>(a, s);
  return launch_attend_as<DT, 256, 1, 4>(a, s);
}

}  // namespace lagkv
