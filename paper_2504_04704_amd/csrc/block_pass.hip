// Bounds of blocks of keys (lagkv_block_bounds) and the blocks that a token reads (lagkv_select_blocks).
//
//   lo[j,d] = min, hi[j,d] = max of K[t,d] over the rows of block j        (Eq. 7-8 for every block)
//   s[j]    = sum over the G query heads and the channels of max(q_d lo[j,d], q_d hi[j,d])
//
// s[j] is at least the sum over the query heads of q.k_t for every row t of the block.  max(q lo, q hi) is q hi for q >= 0
// and q lo for q < 0, so the heads' sum is P.hi + M.lo with P = sum_g max(q_g, 0) and M = sum_g min(q_g, 0): one pass over
// the bounds, whatever G.  Scores are summed in 64 bits: products of two 16-bit numbers are exact there and their sums
// nearly always, so that which of two blocks is taken does not hang on the order in which a kernel adds.
//
// With an infinite bound P.hi + M.lo is infinite or no number, while max(q lo, q hi) may be finite (q < 0, hi = inf), and where a
// P or M is 0 only because a lane has no channel there it says nothing at all.  Finite numbers never add up to such a score: a
// score that is not finite is worked out again, without the infinite bounds, and stays if none of them counts: if P is 0 where hi
// is infinite and M where lo is, and no query head has a 0 there.  What is infinite or none even so comes behind all
// others: a bound of infinity is that of a logit which leaves attention without a number.  (us, 2048 blocks of 32 streams: one
// token 13.7, with one block of each stream so 15.5, with all 24; sixteen 28, 37 and 62.)
#include "attend_pass.hpp"
#include "row_ops.hpp"

namespace lagkv {

namespace {

template <int DT>
struct Of;
template <>
struct Of<LAGKV_F32> {
  using T = F32;
};
template <>
struct Of<LAGKV_BF16> {
  using T = BF16;
};
template <>
struct Of<LAGKV_F16> {
  using T = F16;
};

template <typename ET>
__device__ __forceinline__ uint4 repack(const float (&x)[ET::VEC]) {  // of values that came from the type
  uint4 v;
  if constexpr (ET::KIND == 0) {
    v = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  } else {
    using E = AElem<ET::KIND>;
    v = make_uint4(E::pack(x[0], x[1]), E::pack(x[2], x[3]), E::pack(x[4], x[5]), E::pack(x[6], x[7]));
  }
  return v;
}

__device__ __forceinline__ uint4 ld16_any(const char* p) {
  const u32v4 v = *(const u32v4_any*)p;
  return make_uint4(v.x, v.y, v.z, v.w);
}

__device__ __forceinline__ int64_t rows_held(const int32_t* lengths, int64_t b, int64_t T) {
  const int64_t n = lengths ? lengths[b] : T;
  return n < 0 ? 0 : n > T ? T : n;
}

// A wavefront takes a block: LPR lanes a row (a power of two), one slice each, 64 / LPR rows at a time.  A value is
// unpacked, compared twice and never summed, so that this is exact.  Bound by memory: 1.07 GB of keys (32 streams x
// 131072 rows, bf16) in 201 us, 5.5 TB/s; the last 200 rows of 32 streams in 4 us, the launch.
template <int DT>
__global__ __launch_bounds__(256) void block_bounds_kernel(const BoundsArgs a, int lpr) {
  using ET = typename Of<DT>::T;
  constexpr int VEC = ET::VEC, SIZE = 16 / VEC;
  fetch_arguments<BoundsArgs>();
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t per = a.nb - a.first, id = (int64_t)blockIdx.x * 4 + wave;
  const int64_t stream = id / per, j = a.first + id % per;
  if (stream >= (int64_t)a.B * a.H) return;
  const int64_t b = stream / a.H, h = stream % a.H;
  const int64_t len = rows_held(a.lengths, b, a.T);
  const int slice = lane % lpr, sub = lane / lpr, step = 64 / lpr;
  const bool have = slice * VEC < a.D;
  const int at = have ? slice_at(slice, a.D, VEC) : 0;
  const char* base = a.K + b * a.ksb + h * a.ksh + at * SIZE;
  float lo[VEC], hi[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    lo[i] = INFINITY;
    hi[i] = -INFINITY;
  }
  const int64_t end = (j + 1) * a.block < len ? (j + 1) * a.block : len;
#pragma unroll 4
  for (int64_t t = j * a.block + sub; t < end; t += step) {
    float x[VEC];
    unpack<ET>(ld16_any(base + t * a.kst), x);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      lo[i] = fminf(lo[i], x[i]);
      hi[i] = fmaxf(hi[i], x[i]);
    }
  }
  for (int far = lpr; far < 64; far <<= 1)
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      lo[i] = fminf(lo[i], __shfl_xor(lo[i], far));
      hi[i] = fmaxf(hi[i], __shfl_xor(hi[i], far));
    }
  if (sub == 0 && have) {
    const int64_t to = b * a.osb + h * a.osh + j * a.ost + at * SIZE;
    const uint4 l4 = repack<ET>(lo), h4 = repack<ET>(hi);
    *(u32v4_any*)(a.lo + to) = u32v4{l4.x, l4.y, l4.z, l4.w};
    *(u32v4_any*)(a.hi + to) = u32v4{h4.x, h4.y, h4.z, h4.w};
  }
}

// x of the lane that FAR (1, 2, 4 or 8) lanes or the mirror image away is, within a row of sixteen lanes
template <int CTRL>
__device__ __forceinline__ double dpp_mov_d(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  return __builtin_bit_cast(double, (uint64_t)(uint32_t)dpp_mov_i<CTRL>((int)(u >> 32)) << 32 | (uint32_t)dpp_mov_i<CTRL>((int)u));
}
__device__ __forceinline__ double far_d(double x, int far) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  return __builtin_bit_cast(double, (uint64_t)(uint32_t)__shfl_xor((int)(u >> 32), far) << 32 | (uint32_t)__shfl_xor((int)u, far));
}
// Sum over groups of lpr lanes, in every lane of the group.
__device__ __forceinline__ double lanes_sum(double x, int lpr) {
  if (lpr >= 2) x += dpp_mov_d<0xB1>(x);
  if (lpr >= 4) x += dpp_mov_d<0x4E>(x);
  if (lpr >= 8) x += dpp_mov_d<0x141>(x);
  if (lpr >= 16) x += dpp_mov_d<0x140>(x);
  if (lpr >= 32) x += far_d(x, 16);
  if (lpr >= 64) x += far_d(x, 32);
  return x;
}

// P and M (above) of `count` slots of tokens 0, 1, ...  A slot is a channel of a slice; those that repeat channels of the slice
// before, and those behind the last, are 0.
template <int DT, typename Put>
__device__ __forceinline__ void query_parts(const SelectArgs& a, int64_t b, int64_t h, int width, int from, int count, Put put) {
  constexpr int SIZE = AElem<DT>::SIZE, VEC = 16 / SIZE;
  const char* base = a.Q + b * a.qsb + h * a.G * a.qsh;
  for (int i = from; i < count; i += 256) {
    const int slot = i % width, begin = slot / VEC * VEC;
    const int ch = begin < a.D ? slice_at(slot / VEC, a.D, VEC) + slot - begin : 0;
    const bool real = begin < a.D && ch >= begin;
    const char* at = base + (int64_t)(i / width) * a.qsn + (real ? ch * SIZE : 0);
    double p = 0, m = 0;
#pragma unroll 4
    for (int g = 0; g < a.G; ++g) {
      const char* q = at + g * a.qsh;
      float x;
      if constexpr (DT == LAGKV_F32) x = *(const float*)q;
      else x = AElem<DT>::one(*(const uint16_t*)q);
      p += x > 0.f ? (double)x : 0.0;
      m += x > 0.f ? 0.0 : (double)x;
    }
    put(i / width, slot, real ? p : 0.0, real ? m : 0.0);
  }
}
// The same of sixteen tokens from n0 on, by slices: a thread asks for what four query heads have of its slices in one go.
// (Channel by channel the loads, four or eight times as many, were a third of the kernel.)  Tokens behind the last are 0.
template <int DT, int DP, typename Put>
__device__ __forceinline__ void query_slices(const SelectArgs& a, int64_t b, int64_t h, int n0, int tid, Put put) {
  using ET = typename Of<DT>::T;
  constexpr int VEC = ET::VEC, SIZE = 16 / VEC, CPR = DP / VEC, U = 16 * CPR > 256 ? 16 * CPR / 256 : 1;
  if (tid >= 16 * CPR) return;
  const char* at[U];
  double p[U][VEC], m[U][VEC];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = tid + 256 * u, n = i / CPR, slice = i % CPR;
    at[u] = a.Q + b * a.qsb + h * a.G * a.qsh + (int64_t)(n0 + n < a.N ? n0 + n : 0) * a.qsn + (slice * VEC < a.D ? slice_at(slice, a.D, VEC) : 0) * SIZE;
#pragma unroll
    for (int e = 0; e < VEC; ++e) p[u][e] = m[u][e] = 0;
  }
  for (int g0 = 0; g0 < a.G; g0 += 4) {
    uint4 v[4][U];
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
      for (int u = 0; u < U; ++u) v[g][u] = ld16_any(at[u] + (g0 + g < a.G ? g0 + g : g0) * a.qsh);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      if (g0 + g >= a.G) break;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float x[VEC];
        unpack<ET>(v[g][u], x);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          p[u][e] += x[e] > 0.f ? (double)x[e] : 0.0;
          m[u][e] += x[e] > 0.f ? 0.0 : (double)x[e];
        }
      }
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = tid + 256 * u, n = i / CPR, begin = i % CPR * VEC, dup = begin < a.D ? begin - slice_at(i % CPR, a.D, VEC) : 0;
    const bool real = n0 + n < a.N && begin < a.D;
#pragma unroll
    for (int e = 0; e < VEC; ++e) put(n, begin + e, real && e >= dup ? p[u][e] : 0.0, real && e >= dup ? m[u][e] : 0.0);
  }
}

__device__ __forceinline__ bool is_finite(double s) { return __builtin_fabs(s) < (double)INFINITY; }

// A channel's bounds for a score that is not finite: in their order, and what of them is infinite put aside as 0.  NaN stays.
struct Edge {
  double lo, hi;
  bool far_lo, far_hi;
};
__device__ __forceinline__ Edge edge_of(float lo, float hi) {
  const bool none = lo != lo || hi != hi;
  const float low = none ? NAN : fminf(lo, hi), top = none ? NAN : fmaxf(lo, hi);
  Edge e;
  e.far_lo = __builtin_fabsf(low) == INFINITY;
  e.far_hi = __builtin_fabsf(top) == INFINITY;
  e.lo = e.far_lo ? 0.0 : (double)low;
  e.hi = e.far_hi ? 0.0 : (double)top;
  return e;
}
// Channels of a token's slice, as bits, in which a query head has 0: an infinite bound counts there (0 * inf is no number), as it
// does where its P or M is not 0.
template <int DT>
__device__ __forceinline__ uint32_t zeros_of(const SelectArgs& a, int64_t b, int64_t h, int n, int slice) {
  using ET = typename Of<DT>::T;
  constexpr int VEC = ET::VEC, SIZE = 16 / VEC;
  if (n >= a.N || slice * VEC >= a.D) return 0;
  const int at = slice_at(slice, a.D, VEC);
  const char* q = a.Q + b * a.qsb + h * a.G * a.qsh + (int64_t)n * a.qsn + at * SIZE;
  uint32_t bits = 0;
#pragma unroll 1
  for (int g = 0; g < a.G; ++g) {
    float x[VEC];
    unpack<ET>(ld16_any(q + g * a.qsh), x);
#pragma unroll
    for (int i = 0; i < VEC; ++i) bits |= (x[i] == 0.f ? 1u : 0u) << i;
  }
  return bits >> (slice * VEC - at) << (slice * VEC - at);  // (without those of the slice before)
}

// Scores of one, two or three tokens: a wavefront takes 16 blocks, LPR lanes a block; the bounds are on their way while P
// and M are made.  Bound by reading the bounds (34 MB, 32 streams x 2048 blocks: 9 us traced, 6.6 at a copy's rate) and the
// latency of q, of the sums and of the launch; 64-bit products of two tokens take as long as that (beyond three tokens the
// matrix cores are faster or as fast: four 26.8 us and 24.8, fp32 29.9 and 30.8, five 26.8 and 27.8, fp32 29.9 and 34.1).
constexpr int kScoreBlocks = 64;  // of a workgroup
constexpr int kFewTokens = 3;
constexpr int kManyGroups = 512;  // (two a compute unit)
template <int DT>
__global__ __launch_bounds__(256, 4) void block_scores_kernel(const SelectArgs a, int lpr) {
  using ET = typename Of<DT>::T;
  constexpr int VEC = ET::VEC, SIZE = 16 / VEC, AHEAD = 4;
  __shared__ double sh_p[kFewTokens][kMaxHead], sh_m[kFewTokens][kMaxHead];  // of a token: [channel of a slice][slice]
  fetch_arguments<SelectArgs>();
  const uint32_t tiles = (uint32_t)((a.nb + kScoreBlocks - 1) / kScoreBlocks), st = blockIdx.x / tiles;
  const int64_t stream = st, j0 = (int64_t)(blockIdx.x % tiles) * kScoreBlocks, b = st / (uint32_t)a.H, h = st % (uint32_t)a.H;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int slice = lane % lpr, sub = lane / lpr, step = 64 / lpr;
  const int at = slice * VEC < a.D ? slice_at(slice, a.D, VEC) : 0;
  const int64_t jw = j0 + wave * 16;
  const int passes = (16 + step - 1) / step;  // of `step` blocks
  uint64_t again = 0;  // scores that are not finite: bit 16 n + block
  for (int p0 = 0; p0 < passes; p0 += AHEAD) {
    uint4 lo4[AHEAD], hi4[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int64_t j = jw + (p0 + i) * step + sub, jj = j < a.nb ? j : a.nb - 1;
      const int64_t from = b * a.bsb + h * a.bsh + jj * a.bst + at * SIZE;
      lo4[i] = ld16_any(a.lo + from);
      hi4[i] = ld16_any(a.hi + from);
    }
    if (p0 == 0) {
      query_parts<DT>(a, b, h, lpr * VEC, threadIdx.x, a.N * lpr * VEC, [&](int n, int slot, double p, double m) {
        sh_p[n][slot % VEC * lpr + slot / VEC] = p;
        sh_m[n][slot % VEC * lpr + slot / VEC] = m;
      });
      __syncthreads();
    }
    for (int n = 0; n < a.N; ++n) {
      double p[VEC], m[VEC];
#pragma unroll
      for (int c = 0; c < VEC; ++c) {
        p[c] = sh_p[n][c * lpr + slice];
        m[c] = sh_m[n][c * lpr + slice];
      }
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int of = (p0 + i) * step + sub;
        const int64_t j = jw + of;
        // (unpacked in every turn: all of them at once, as 64-bit numbers ahead of the turns, would not fit the registers)
        asm volatile("" : "+v"(lo4[i].x), "+v"(lo4[i].y), "+v"(lo4[i].z), "+v"(lo4[i].w));
        asm volatile("" : "+v"(hi4[i].x), "+v"(hi4[i].y), "+v"(hi4[i].z), "+v"(hi4[i].w));
        float lo[VEC], hi[VEC];
        unpack<ET>(lo4[i], lo);
        unpack<ET>(hi4[i], hi);
        double s0 = 0, s1 = 0;
#pragma unroll
        for (int c = 0; c < VEC; ++c) {
          s0 = __builtin_fma(p[c], (double)hi[c], s0);
          s1 = __builtin_fma(m[c], (double)lo[c], s1);
        }
        const double s = lanes_sum(s0 + s1, lpr);
        if (slice == 0 && of < 16 && j < a.nb) {
          a.score[(stream * a.N + n) * a.nb + j] = s;
          again |= is_finite(s) ? 0 : 1ull << (n * 16 + of);
        }
      }
    }
  }
  if (!__any(again != 0)) return;
  const SelectArgs& r = arguments_again<SelectArgs>();
  const int64_t held = (rows_held(r.lengths, b, r.T) + r.block - 1) / r.block;  // (blocks without rows are nobody's choice)
#pragma unroll 1
  for (int n = 0; n < r.N; ++n) {
    if (!__any((again >> (16 * n) & 0xffff) != 0)) continue;
    const uint32_t zeros = zeros_of<DT>(r, b, h, n, slice);
#pragma unroll 1
    for (int pass = 0; pass < passes; ++pass) {
      const int of = pass * step + sub;
      const int64_t j = jw + of, jj = j < r.nb ? j : r.nb - 1;
      const bool mine = of < 16 && j < held && (again >> (16 * n + of) & 1);
      if (!__any(mine)) continue;
      const int64_t from = b * r.bsb + h * r.bsh + jj * r.bst + at * SIZE;
      float lo[VEC], hi[VEC];
      unpack<ET>(ld16_any(r.lo + from), lo);
      unpack<ET>(ld16_any(r.hi + from), hi);
      double s = 0;
#pragma unroll
      for (int c = 0; c < VEC; ++c) {
        const double p = sh_p[n][c * lpr + slice], m = sh_m[n][c * lpr + slice];
        const Edge e = edge_of(lo[c], hi[c]);
        const bool zero = zeros >> c & 1;
        s += (e.far_hi && (p != 0 || zero)) || (e.far_lo && (m != 0 || zero)) ? (double)NAN : p * e.hi + m * e.lo;
      }
      s = lanes_sum(s, lpr);
      if (mine) r.score[(stream * r.N + n) * r.nb + j] = is_finite(s) ? s : (double)NAN;
    }
  }
}

// Scores of more tokens: sixteen blocks times sixteen tokens at a time on the matrix cores (64-bit), whose operand of
// the blocks is the bounds as they lie in memory (lane l: block l % 16, a slice of its channels), and that of the tokens is
// P and M, in LDS for the workgroup's sixteen tokens and `sets` of 64 blocks (the next set comes while other wavefronts
// multiply).  Workgroups of other tokens and the same blocks follow on the same XCD, whose L2 has the bounds.  A product
// takes what 64-bit vector arithmetic takes, but nothing has to be summed across lanes.  Bound by the products: 16 tokens of
// 32 streams x 2048 blocks 20 us, 9 at the rate of a large 64-bit product (the rest are P and M, 64-bit conversions and
// the launch).
typedef double f64x4 __attribute__((ext_vector_type(4)));
template <int DT, int DP>
__global__ __launch_bounds__(256) void block_scores_many_kernel(const SelectArgs a, int sets) {
  using ET = typename Of<DT>::T;
  constexpr int VEC = ET::VEC, SIZE = 16 / VEC, NC = DP / VEC / 4;
  constexpr int LD = DP + 1;  // doubles between tokens: sixteen lanes' reads on different banks
  extern __shared__ __attribute__((aligned(16))) double sh_pm[];  // [16][LD] of P, then of M
  fetch_arguments<SelectArgs>();
  const uint32_t tiles = (uint32_t)((a.nb + kScoreBlocks * sets - 1) / (kScoreBlocks * sets)), token_groups = (uint32_t)(a.N + 15) / 16;
  const uint32_t slot = blockIdx.x % 8, rest = blockIdx.x / 8, of = rest / token_groups, id = of * 8 + slot, st = id / tiles;
  if (st >= (uint32_t)a.B * (uint32_t)a.H) return;
  const int n0 = (int)(rest - of * token_groups) * 16;
  const int64_t stream = st, b = st / (uint32_t)a.H, h = st % (uint32_t)a.H;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const int64_t j0 = (int64_t)(id - st * tiles) * kScoreBlocks * sets + wave * 16;
  uint32_t again = 0;  // scores that are not finite: bit 4 set + i (eight sets at most)
  int here = 0;  // sets that are there
  while (here < sets && j0 - wave * 16 + here * kScoreBlocks < a.nb) ++here;
  uint4 lo4[NC], hi4[NC];
  auto load = [&](int set) {
    const int64_t j = j0 + set * kScoreBlocks + col, jj = j < a.nb ? j : a.nb - 1;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int slice = c * 4 + grp;
      const int64_t from = b * a.bsb + h * a.bsh + jj * a.bst + (slice * VEC < a.D ? slice_at(slice, a.D, VEC) : 0) * SIZE;
      lo4[c] = ld16_any(a.lo + from);
      hi4[c] = ld16_any(a.hi + from);
    }
  };
  load(0);
  query_slices<DT, DP>(a, b, h, n0, threadIdx.x, [&](int n, int slot, double p, double m) {
    sh_pm[n * LD + slot] = p;
    sh_pm[(16 + n) * LD + slot] = m;
  });
  __syncthreads();
  for (int set = 0; set < here; ++set) {
    f64x4 s = {0, 0, 0, 0};
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      __builtin_amdgcn_sched_barrier(0);  // (not all bounds as 64-bit numbers at once: half the wavefronts a SIMD)
      float lo[VEC], hi[VEC];
      unpack<ET>(lo4[c], lo);
      unpack<ET>(hi4[c], hi);
      const bool have = (c * 4 + grp) * VEC < a.D;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const int slot = (c * 4 + grp) * VEC + i;
        s = __builtin_amdgcn_mfma_f64_16x16x4f64(have ? (double)hi[i] : 0.0, sh_pm[col * LD + slot], s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f64_16x16x4f64(have ? (double)lo[i] : 0.0, sh_pm[(16 + col) * LD + slot], s, 0, 0, 0);
      }
    }
    if (set + 1 < here) load(set + 1);
    // s[i]: block grp + 4 i of the sixteen, token col
    const int n = n0 + col;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t to = j0 + set * kScoreBlocks + grp + 4 * i;
      if (n < a.N && to < a.nb) {
        a.score[(stream * a.N + n) * a.nb + to] = s[i];
        again |= is_finite(s[i]) ? 0 : 1u << (4 * set + i);
      }
    }
  }
  if (!__any(again != 0)) return;
  const SelectArgs& r = arguments_again<SelectArgs>();
  const int64_t held = (rows_held(r.lengths, b, r.T) + r.block - 1) / r.block;  // (blocks without rows are nobody's choice)
#pragma unroll 1
  for (int set = 0; set < here; ++set) {
    uint32_t mine = again >> (4 * set) & 15;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (j0 + set * kScoreBlocks + grp + 4 * i >= held) mine &= ~(1u << i);
    if (!__any(mine != 0)) continue;
    const int64_t j = j0 + set * kScoreBlocks + col, row = b * r.bsb + h * r.bsh + (j < r.nb ? j : r.nb - 1) * r.bst;
    f64x4 s = {0, 0, 0, 0};  // (with 1e300 for each infinite bound that counts; finite ones add up to less than 1e90)
#pragma unroll 1
    for (int c = 0; c < NC; ++c) {
      const int slice = c * 4 + grp;
      const bool have = slice * VEC < r.D;
      const uint32_t zeros = zeros_of<DT>(r, b, h, n0 + col, slice);
      const int64_t from = row + (have ? slice_at(slice, r.D, VEC) : 0) * SIZE;
      float lo[VEC], hi[VEC];
      unpack<ET>(ld16_any(r.lo + from), lo);
      unpack<ET>(ld16_any(r.hi + from), hi);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const double p = sh_pm[col * LD + slice * VEC + i], m = sh_pm[(16 + col) * LD + slice * VEC + i];
        const Edge e = edge_of(have ? lo[i] : 0.f, have ? hi[i] : 0.f);
        s = __builtin_amdgcn_mfma_f64_16x16x4f64(e.hi, p, s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f64_16x16x4f64(e.lo, m, s, 0, 0, 0);
        const bool zero = zeros >> i & 1;
        s = __builtin_amdgcn_mfma_f64_16x16x4f64(e.far_hi ? 1e300 : 0.0, p != 0 || zero ? 1.0 : 0.0, s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f64_16x16x4f64(e.far_lo ? 1e300 : 0.0, m != 0 || zero ? 1.0 : 0.0, s, 0, 0, 0);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (mine >> i & 1)
        r.score[(stream * r.N + n0 + col) * r.nb + j0 + set * kScoreBlocks + grp + 4 * i] = __builtin_fabs(s[i]) < 1e200 ? s[i] : (double)NAN;
  }
}

// 64-bit key in the order of the scores (-0 like 0, what is no number below all; none is infinite); 0 is no key.
__device__ __forceinline__ uint64_t score_key(double s) {
  if (s != s) return 1;
  const uint64_t u = __builtin_bit_cast(uint64_t, s + 0.0);
  return u >> 63 ? ~u : u | 1ull << 63;
}

__device__ __forceinline__ double key_score(uint64_t u) { return __builtin_bit_cast(double, u >> 63 ? u ^ 1ull << 63 : ~u); }

// Largest of all lanes.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
  const uint32_t far = (uint32_t)dpp_mov_i<CTRL>((int)v);
  return far > v ? far : v;
}
__device__ __forceinline__ uint32_t wave_largest(uint32_t v) {
  const int x = (int)dpp_max<0x140>(dpp_max<0x141>(dpp_max<0x4E>(dpp_max<0xB1>(v))));
  const uint32_t a = __builtin_amdgcn_readlane(x, 0), b = __builtin_amdgcn_readlane(x, 16), c = __builtin_amdgcn_readlane(x, 32),
                 d = __builtin_amdgcn_readlane(x, 48), ab = a > b ? a : b, cd = c > d ? c : d;
  return ab > cd ? ab : cd;
}

// Bits that any lane has.
__device__ __forceinline__ uint32_t wave_or(uint32_t v) {
  v |= (uint32_t)dpp_mov_i<0xB1>((int)v);
  v |= (uint32_t)dpp_mov_i<0x4E>((int)v);
  v |= (uint32_t)dpp_mov_i<0x141>((int)v);
  v |= (uint32_t)dpp_mov_i<0x140>((int)v);
  const int x = (int)v;
  return (uint32_t)(__builtin_amdgcn_readlane(x, 0) | __builtin_amdgcn_readlane(x, 16) | __builtin_amdgcn_readlane(x, 32) |
                    __builtin_amdgcn_readlane(x, 48));
}
__device__ __forceinline__ uint64_t wave_or(uint64_t v) { return (uint64_t)wave_or((uint32_t)(v >> 32)) << 32 | wave_or((uint32_t)v); }
// Sum over the lanes up to this one (row_shr: 0 where a row begins).
__device__ __forceinline__ uint32_t sum_upto(uint32_t v, int lane) {
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, false);
  const uint32_t a = __builtin_amdgcn_readlane((int)v, 15), b = __builtin_amdgcn_readlane((int)v, 31), c = __builtin_amdgcn_readlane((int)v, 47);
  return v + (lane >= 16 ? a : 0) + (lane >= 32 ? b : 0) + (lane >= 48 ? c : 0);
}

// A workgroup takes a token's list.  The k-th largest score is found eight bits at a time (a histogram in LDS of the keys that
// share the digits found), down to where the keys that share all digits found are as many as are still wanted: two
// passes as a rule.  The digits are those of where a score lies between the least and the largest, as a 32-bit fraction: its own
// leading bits are its exponent, which nearly all scores share.  Where more scores than wanted share a fraction, or the
// range is not finite, those scores' keys are gone through in the same way, from the highest bit in which two differ.
// Then the blocks above, and the first of those that are equal, are written in order.  Bound by latency: a chain of
// barriers for short lists (32 lists of 2048 blocks 6 us, 2048 lists of 512 10 us), one compute unit's instructions for
// long ones (8192 blocks 16 us; in digits of the keys alone 18).  E keys a thread in registers; E = 0: read again in every pass.
constexpr int kSelectThreads = 512, kSelectWaves = kSelectThreads / 64;
template <int E>
__global__ __launch_bounds__(kSelectThreads) void block_select_kernel(const SelectArgs a) {
  __shared__ uint32_t sh_hist[2][256];
  __shared__ uint64_t sh_wave[2][kSelectWaves];
  __shared__ uint32_t sh_ends[2][kSelectWaves];
  __shared__ uint32_t sh_digit, sh_need, sh_in;
  __shared__ uint32_t sh_count[2][kSelectWaves];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  fetch_arguments<SelectArgs>();
  const int64_t unit = blockIdx.x, b = (uint32_t)blockIdx.x / (uint32_t)a.N / (uint32_t)a.H;
  const int64_t len = rows_held(a.lengths, b, a.T), nb = (len + a.block - 1) / a.block;
  const double* score = a.score + unit * a.nb;
  int32_t* to = a.blocks + unit * a.k;
  if (nb <= a.k) {
    for (int64_t i = tid; i < a.k; i += kSelectThreads) to[i] = i < nb ? (int32_t)i : -1;
    return;
  }
  const int free0 = a.first, free1 = (int)nb - a.last;  // the others are taken anyway
  uint64_t mine[E ? E : 1];
  uint32_t lies[E ? E : 1];  // (fractions)
  // a wavefront takes `slabs` times 64 blocks, one behind the other: what it writes lies together
  const int slabs = (int)((nb + kSelectThreads - 1) / kSelectThreads);
  auto block_of = [&](int e) { return e < slabs ? (wave * slabs + e) * 64 + lane : (int)nb; };
  auto read = [&](int e) {
    const int j = block_of(e);
    return j >= free0 && j < free1 ? score_key(score[j]) : 0;
  };
  bool linear = false;
  uint64_t first_key = 0;
  double least = 0, scale = 0;
  auto fraction = [&](uint64_t u) { return linear ? (uint32_t)((key_score(u ? u : first_key) - least) * scale) : 0u; };
  auto each = [&](auto f) {  // key and fraction
    if constexpr (E > 0) {
#pragma unroll
      for (int e = 0; e < E; ++e) f(e, mine[e], lies[e]);
    } else {
      for (int e0 = 0; e0 < slabs; e0 += 8) {  // (eight on their way together; behind the last: no keys)
        uint64_t u[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = read(e0 + i);
#pragma unroll
        for (int i = 0; i < 8; ++i) f(e0 + i, u[i], fraction(u[i]));
      }
    }
  };
  if constexpr (E > 0) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      mine[e] = read(e);
      lies[e] = 0;
    }
  }
  // the two ends of the keys' leading halves (the least as its complement)
  uint32_t top = 0, bottom = 0;
  each([&](int, uint64_t u, uint32_t) {
    const uint32_t half = (uint32_t)(u >> 32), c = u ? ~half : 0;
    top = half > top ? half : top;
    bottom = c > bottom ? c : bottom;
  });
  top = wave_largest(top);
  bottom = wave_largest(bottom);
  if (lane == 0) {
    sh_ends[0][wave] = top;
    sh_ends[1][wave] = bottom;
  }
  (&sh_hist[0][0])[tid] = 0;  // (kSelectThreads bins)
  __syncthreads();
#pragma unroll
  for (int x = 0; x < kSelectWaves; ++x) {
    top = sh_ends[0][x] > top ? sh_ends[0][x] : top;
    bottom = sh_ends[1][x] > bottom ? sh_ends[1][x] : bottom;
  }
  uint32_t need = (uint32_t)(a.k - a.first - a.last);
  int turn = 0;
  // One digit of the keys that f counts: the one at which `need` keys are reached from the top.  The keys above it are taken
  // off `need`; true where all that have it are wanted.
  auto digit_of = [&](auto count, uint32_t* digit) {
    count(&sh_hist[turn][0]);
    __syncthreads();
    if (wave == 0) {
      // digits from the top: lane l has 255 - 4 l down to 252 - 4 l
      uint32_t c[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        c[i] = sh_hist[turn][255 - 4 * lane - i];
        sum += c[i];
      }
      const uint32_t upto = sum_upto(sum, lane);
      uint32_t before = upto - sum;
      if (before < need && upto >= need) {
        int i = 0;
        while (i < 3 && before + c[i] < need) before += c[i++];
        sh_digit = 255 - 4 * lane - i;
        sh_need = need - before;
        sh_in = i == 0 ? c[0] : i == 1 ? c[1] : i == 2 ? c[2] : c[3];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) sh_hist[turn][255 - 4 * lane - i] = 0;  // (for the pass after the next)
    }
    __syncthreads();
    *digit = sh_digit;
    need = sh_need;
    turn ^= 1;
    return sh_in == need;
  };
  // Taken: scores whose fraction is above `at`; of those at it, keys above `edge` or (if set) at or above `above_edge`, and the
  // first `need` of the keys at `edge`.
  first_key = (uint64_t)~bottom << 32;
  least = key_score(first_key);
  const double range = key_score((uint64_t)top << 32 | 0xffffffffu) - least;
  linear = range >= 1e-290 && range <= 1.7e308;  // (and a number)
  scale = linear ? 4294967295.0 / range : 0;
  if constexpr (E > 0) {
#pragma unroll
    for (int e = 0; e < E; ++e) lies[e] = fraction(mine[e]);
  }
  uint32_t at = 0;
  uint64_t edge = ~0ull, above_edge = 0;
  if (need == 0) {
    at = ~0u;
  } else {
    bool done = false;
    for (int shift = 24; linear && shift >= 0 && !done; shift -= 8) {
      uint32_t digit;
      done = digit_of([&](uint32_t* hist) {
        each([&](int, uint64_t u, uint32_t f) {
          if (u && (shift == 24 || f >> (shift + 8) == at >> (shift + 8))) atomicAdd(&hist[f >> shift & 255], 1u);
        });
      }, &digit);
      at |= digit << shift;
      if (done) --at;  // (not all keys are taken: it was not 0)
    }
    if (!done) {
      // bits in which the keys at this fraction differ: those that some have and not all
      uint64_t some = 0, all = ~0ull;
      each([&](int, uint64_t u, uint32_t f) {
        if (u && f == at) {
          some |= u;
          all &= u;
        }
      });
      some = wave_or(some);
      all = ~wave_or(~all);
      if (lane == 0) {
        sh_wave[0][wave] = some;
        sh_wave[1][wave] = all;
      }
      __syncthreads();
#pragma unroll
      for (int x = 0; x < kSelectWaves; ++x) {
        some |= sh_wave[0][x];
        all &= sh_wave[1][x];
      }
      const uint64_t differ = some & ~all;
      edge = some & all;
      if (differ != 0) {
        int low = 63 - __builtin_clzll(differ);  // the highest differing bit, then the lowest one found
        edge = low == 63 ? 0 : edge >> (low + 1) << (low + 1);
        for (int high = low;; high = low - 1) {
          const int width = high + 1 < 8 ? high + 1 : 8;
          low = high + 1 - width;
          uint32_t digit;
          done = digit_of([&](uint32_t* hist) {
            each([&](int, uint64_t u, uint32_t f) {
              if (u && f == at && (high == 63 || (u >> (high + 1)) == (edge >> (high + 1)))) atomicAdd(&hist[(u >> low) & ((1u << width) - 1)], 1u);
            });
          }, &digit);
          edge |= (uint64_t)digit << low;
          if (done) above_edge = edge;
          if (done || low == 0) break;
        }
      }
    }
  }
  // (keys from `from` on at the fraction `at`; no key is all ones)
  const uint64_t from = above_edge ? above_edge : edge == ~0ull ? edge : edge + 1, tied = above_edge ? ~0ull : edge;
  auto over_of = [&](int j, uint64_t u, uint32_t f) {
    return (j < free0) | ((j >= free1) & (j < (int)nb)) | ((u != 0) & ((f > at) | ((f == at) & (u >= from))));
  };
  auto tie_of = [&](uint64_t u, uint32_t f) { return (u == tied) & (f == at); };
  uint32_t n_over = 0, n_tie = 0;  // of the wavefront
  each([&](int e, uint64_t u, uint32_t f) {
    n_over += __popcll(__ballot(over_of(block_of(e), u, f)));
    n_tie += __popcll(__ballot(tie_of(u, f)));
  });
  if (lane == 0) {
    sh_count[0][wave] = n_over;
    sh_count[1][wave] = n_tie;
  }
  __syncthreads();
  uint32_t before_o = 0, before_t = 0;
#pragma unroll
  for (int x = 0; x < kSelectWaves; ++x) {
    before_o += x < wave ? sh_count[0][x] : 0;
    before_t += x < wave ? sh_count[1][x] : 0;
  }
  each([&](int e, uint64_t u, uint32_t f) {
    const int j = block_of(e);
    const bool over = over_of(j, u, f), tie = tie_of(u, f);
    const uint64_t overs = __ballot(over), ties = __ballot(tie);
    const uint32_t o = before_o + prefix_popc(overs), t = before_t + prefix_popc(ties);
    if (over || (tie && t < need)) to[o + (t < need ? t : need)] = j;
    before_o += __popcll(overs);
    before_t += __popcll(ties);
  });
}

int lanes_a_row(int D, int dtype) {
  const int slices = (D * (dtype == LAGKV_F32 ? 4 : 2) + 15) / 16;
  int lpr = 1;
  while (lpr < slices) lpr <<= 1;
  return lpr;
}

}  // namespace

hipError_t launch_block_bounds(const BoundsArgs& a, hipStream_t s) {
  const int64_t groups = ((int64_t)a.B * a.H * (a.nb - a.first) + 3) / 4;
  const int lpr = lanes_a_row(a.D, a.dtype);
  const dim3 grid((uint32_t)groups), group(256);
  if (a.dtype == LAGKV_F32) block_bounds_kernel<LAGKV_F32><<<grid, group, 0, s>>>(a, lpr);
  else if (a.dtype == LAGKV_BF16) block_bounds_kernel<LAGKV_BF16><<<grid, group, 0, s>>>(a, lpr);
  else block_bounds_kernel<LAGKV_F16><<<grid, group, 0, s>>>(a, lpr);
  return hipGetLastError();
}

namespace {
template <int DT>
hipError_t launch_scores(const SelectArgs& a, hipStream_t s) {
  const int64_t streams = (int64_t)a.B * a.H, token_groups = (a.N + 15) / 16;
  auto tiles = [&](int sets) { return streams * ((a.nb + kScoreBlocks * sets - 1) / (kScoreBlocks * sets)); };
  // (several sets of blocks a workgroup where there are workgroups enough, as each makes P and M for itself: 16 tokens of 32
  // streams over 2048 blocks 29.9 us with two sets and 31.3 with one, fp32 34 and 38, 64 tokens over 512 blocks 35.3 and 37.3)
  int sets = 1;
  while (sets < 8 && tiles(2 * sets) * token_groups >= kManyGroups) sets *= 2;
  const dim3 grid((uint32_t)(a.N <= kFewTokens ? tiles(1) : (tiles(sets) + 7) / 8 * 8 * token_groups)), group(256);
  auto lds = [](int dp) { return (size_t)32 * (dp + 1) * 8; };
  if (a.N <= kFewTokens) block_scores_kernel<DT><<<grid, group, 0, s>>>(a, lanes_a_row(a.D, DT));
  else if (a.D <= 64) block_scores_many_kernel<DT, 64><<<grid, group, lds(64), s>>>(a, sets);
  else if (a.D <= 128) block_scores_many_kernel<DT, 128><<<grid, group, lds(128), s>>>(a, sets);
  else {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(block_scores_many_kernel<DT, 256>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds(256));
    if (e != hipSuccess) return e;
    block_scores_many_kernel<DT, 256><<<grid, group, lds(256), s>>>(a, sets);
  }
  return hipGetLastError();
}
}  // namespace

hipError_t launch_block_scores(const SelectArgs& a, hipStream_t s) {
  return a.dtype == LAGKV_F32 ? launch_scores<LAGKV_F32>(a, s) : a.dtype == LAGKV_BF16 ? launch_scores<LAGKV_BF16>(a, s) : launch_scores<LAGKV_F16>(a, s);
}

hipError_t launch_block_select(const SelectArgs& a, hipStream_t s) {
  const dim3 grid((uint32_t)((int64_t)a.B * a.H * a.N)), group(kSelectThreads);
  if (a.nb <= kSelectThreads) block_select_kernel<1><<<grid, group, 0, s>>>(a);
  else if (a.nb <= 4 * kSelectThreads) block_select_kernel<4><<<grid, group, 0, s>>>(a);
  else if (a.nb <= 16 * kSelectThreads) block_select_kernel<16><<<grid, group, 0, s>>>(a);
  else block_select_kernel<0><<<grid, group, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace lagkv
