// Bounds of blocks of keys (lagkv_block_bounds) and the blocks that a token reads (lagkv_select_blocks).
//
//   lo[j,d] = min, hi[j,d] = max of K[t,d] over the rows of block j        (Eq. 7-8 for every block)
//   s[j]    = sum over the G query heads and the channels of max(q_d lo[j,d], q_d hi[j,d])
//
// s[j] is at least the sum over the query heads of q.k_t for every row t of the block.  max(q lo, q hi) is q hi for q >= 0
// and q lo for q < 0, so the heads' sum is P.hi + M.lo with P = sum_g max(q_g, 0) and M = sum_g min(q_g, 0): one pass over
// the bounds, whatever G.  Scores are summed in 64 bits: products of two 16-bit numbers are exact there and their sums
// nearly always, so that which of two blocks is taken does not hang on the order in which a kernel adds.
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

// A wavefront takes a block: LPR lanes a row (a power of two), one slice each, 64 / LPR rows at a time.
template <int DT>
__global__ __launch_bounds__(256) void block_bounds_kernel(const BoundsArgs a, int lpr) {
  using ET = typename Of<DT>::T;
  constexpr int VEC = ET::VEC, SIZE = 16 / VEC;
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
    const int64_t to = ((stream * a.nb + j) * a.D + at) * SIZE;
    const uint4 l4 = repack<ET>(lo), h4 = repack<ET>(hi);
    *(u32v4_any*)(a.lo + to) = u32v4{l4.x, l4.y, l4.z, l4.w};
    *(u32v4_any*)(a.hi + to) = u32v4{h4.x, h4.y, h4.z, h4.w};
  }
}

__device__ __forceinline__ double add_from(double x, int far) {
  const long long u = __builtin_bit_cast(long long, x);
  return x + __builtin_bit_cast(double, ((long long)__shfl_xor((int)(u >> 32), far) << 32) | (uint32_t)__shfl_xor((int)u, far));
}

// A workgroup takes up to 64 blocks of a stream and all its tokens: P and M of a token in LDS, LPR lanes a block.
constexpr int kScoreBlocks = 64;
template <int DT>
__global__ __launch_bounds__(256) void block_scores_kernel(const SelectArgs a, int lpr) {
  using ET = typename Of<DT>::T;
  constexpr int VEC = ET::VEC, SIZE = 16 / VEC;
  __shared__ double sh_p[kMaxHead], sh_m[kMaxHead];
  const int64_t tiles = (a.nb + kScoreBlocks - 1) / kScoreBlocks;
  const int64_t stream = blockIdx.x / tiles, j0 = blockIdx.x % tiles * kScoreBlocks;
  const int64_t b = stream / a.H, h = stream % a.H;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int slice = lane % lpr, sub = lane / lpr, step = 64 / lpr;
  const bool have = slice * VEC < a.D;
  const int at = have ? slice_at(slice, a.D, VEC) : 0, dup = have ? slice * VEC - at : 0;
  for (int n = 0; n < a.N; ++n) {
    __syncthreads();
    for (int d = threadIdx.x; d < a.D; d += 256) {
      double p = 0, m = 0;
      for (int g = 0; g < a.G; ++g) {
        const char* q = a.Q + b * a.qsb + (h * a.G + g) * a.qsh + (int64_t)n * a.qsn + (int64_t)d * SIZE;
        float x;
        if constexpr (DT == LAGKV_F32) x = *(const float*)q;
        else x = AElem<DT>::one(*(const uint16_t*)q);
        p += x > 0.f ? (double)x : 0.0;
        m += x > 0.f ? 0.0 : (double)x;
      }
      sh_p[d] = p;
      sh_m[d] = m;
    }
    __syncthreads();
    for (int i = wave * step + sub; i < kScoreBlocks; i += 4 * step) {
      const int64_t j = j0 + i;
      double s = 0;
      if (j < a.nb && have) {
        const int64_t from = ((stream * a.nb + j) * a.D + at) * SIZE;
        float lo[VEC], hi[VEC];
        unpack<ET>(ld16_any(a.lo + from), lo);
        unpack<ET>(ld16_any(a.hi + from), hi);
#pragma unroll
        for (int c = 0; c < VEC; ++c)
          if (c >= dup) {
            s = __builtin_fma(sh_p[at + c], (double)hi[c], s);
            s = __builtin_fma(sh_m[at + c], (double)lo[c], s);
          }
      }
      for (int far = 1; far < lpr; far <<= 1) s = add_from(s, far);
      if (slice == 0 && j < a.nb) a.score[((stream * a.N) + n) * a.nb + j] = s;
    }
  }
}

// 64-bit key in the order of the scores: blocks that are always taken first, equal scores equal (-0 like 0).
__device__ __forceinline__ uint64_t score_key(double s, bool always) {
  if (always) return ~0ull;
  const uint64_t u = __builtin_bit_cast(uint64_t, s + 0.0);
  return u >> 63 ? ~u : u | 1ull << 63;
}

// A workgroup takes a token's list: the k-th largest key digit by digit (eight bits a pass, a histogram in LDS), then
// the blocks above it and the first of those equal to it, in order.
__global__ __launch_bounds__(256) void block_select_kernel(const SelectArgs a) {
  __shared__ uint32_t sh_hist[256];
  __shared__ uint64_t sh_prefix;
  __shared__ int32_t sh_need;
  __shared__ int32_t sh_count[2][4];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int64_t unit = blockIdx.x, b = unit / a.N / a.H;
  const int64_t len = rows_held(a.lengths, b, a.T), nb = (len + a.block - 1) / a.block;
  const double* score = a.score + unit * a.nb;
  int32_t* to = a.blocks + unit * a.k;
  if (nb <= a.k) {
    for (int64_t i = tid; i < a.k; i += 256) to[i] = i < nb ? (int32_t)i : -1;
    return;
  }
  auto key = [&](int64_t j) { return score_key(score[j], j < a.first || j >= nb - a.last); };
  if (tid == 0) {
    sh_prefix = 0;
    sh_need = a.k;
  }
  for (int shift = 56; shift >= 0; shift -= 8) {
    sh_hist[tid] = 0;
    __syncthreads();
    const uint64_t prefix = sh_prefix;
    for (int64_t j = tid; j < nb; j += 256) {
      const uint64_t u = key(j);
      if (shift == 56 || (u >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&sh_hist[(u >> shift) & 255], 1u);
    }
    __syncthreads();
    if (tid == 0) {
      int need = sh_need, digit = 255;
      while (digit > 0 && (int)sh_hist[digit] < need) need -= (int)sh_hist[digit--];
      sh_need = need;
      sh_prefix = prefix | (uint64_t)digit << shift;
    }
    __syncthreads();
  }
  const uint64_t edge = sh_prefix;
  const int ties = sh_need;  // of the keys equal to the edge, this many are taken
  int taken = 0, equal = 0;
  for (int64_t j0 = 0; j0 < nb; j0 += 256) {
    const int64_t j = j0 + tid;
    const uint64_t u = j < nb ? key(j) : 0;
    const uint64_t above = __ballot(j < nb && u > edge), same = __ballot(j < nb && u == edge);
    if (lane == 0) {
      sh_count[0][wave] = __popcll(above);
      sh_count[1][wave] = __popcll(same);
    }
    __syncthreads();
    int before_a = taken, before_s = equal;
    for (int x = 0; x < 4; ++x) {
      if (x < wave) {
        before_a += sh_count[0][x];
        before_s += sh_count[1][x];
      }
      taken += sh_count[0][x];
      equal += sh_count[1][x];
    }
    before_a += prefix_popc(above);
    before_s += prefix_popc(same);
    if (j < nb && (u > edge || (u == edge && before_s < ties))) to[before_a + (before_s < ties ? before_s : ties)] = (int32_t)j;
    __syncthreads();
  }
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

hipError_t launch_block_scores(const SelectArgs& a, hipStream_t s) {
  const int64_t groups = (int64_t)a.B * a.H * ((a.nb + kScoreBlocks - 1) / kScoreBlocks);
  const int lpr = lanes_a_row(a.D, a.dtype);
  const dim3 grid((uint32_t)groups), group(256);
  if (a.dtype == LAGKV_F32) block_scores_kernel<LAGKV_F32><<<grid, group, 0, s>>>(a, lpr);
  else if (a.dtype == LAGKV_BF16) block_scores_kernel<LAGKV_BF16><<<grid, group, 0, s>>>(a, lpr);
  else block_scores_kernel<LAGKV_F16><<<grid, group, 0, s>>>(a, lpr);
  return hipGetLastError();
}

hipError_t launch_block_select(const SelectArgs& a, hipStream_t s) {
  block_select_kernel<<<dim3((uint32_t)((int64_t)a.B * a.H * a.N)), dim3(256), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace lagkv
