// Attention of many query rows over all rows of a cache (lagkv_attend, 16-bit types; the mathematics is attend_pass.hpp's; when
// it is taken, plan_of says).
//
// Where a stream has tens of query rows (a drafted tree under grouped heads, a chunk of a prompt) the matrix cores are the
// bound, not memory: 256 rows make 256 flop of a cache byte.  A workgroup of four or eight wavefronts goes over 64 cache
// rows (32 beyond 128 channels) at a time, which lie in LDS for all of them (the next ones are on their way through
// registers meanwhile); each wavefront keeps 32 query rows to itself, so that nothing is exchanged between wavefronts.  32x32
// products: a lane holds one query row (of S^T, P^T and O^T), so that maxima and sums need one exchange between the lane's
// halves only.  Measured: 256 rows of 32 streams x 33536 (bf16, 128 channels) 191 to 196 us, 0.73 Pflop/s, and 8.7 for joining the
// pieces; 2048 rows of 8 streams x 8640 111 us, 0.66 Pflop/s, and 9.5 (a large product of the library: 1.09).  The matrix cores are
// busy in 65 % of the cycles, at a clock of 1.6 GHz; there are no conflicts of LDS banks to speak of.
//
// P is put in as two numbers, as in the narrow kernel: which of the two runs goes by time, and so by what else is in the batch, and
// the precision of a request's result must not.  One number, rounded, takes a third of the products less, 147 us in place of
// 191, and puts an error of the size of the output's own rounding into the outputs.
//
// Products and exponentials take about the same time (48 products of 32 cycles, 32 elements a lane of some 50), on
// different units.  So eight wavefronts go in two halves, one of each on every SIMD, between barriers: while one half
// multiplies (the scores of its step, the outputs of the step before), the other makes weights and moves rows.  With
// h counting the phases, the first half multiplies for step i in h = 2i and makes weights in 2i + 1, the other one phase later.
// K of step i and V of step i - 1 are read in 2i and 2i + 1; K(i+1) and V(i) are written into the other buffers in
// 2i + 1 by the first half and in 2i by the second, when nobody reads these any more.  (Halves in phase took 15 % longer.)  Four
// wavefronts, for fewer rows or 64 channels, leave that to the two workgroups of a compute unit (for 256 it holds one): one barrier
// a step.
//
// The reference m of the exponentials is only moved when a row's maximum leaves it by more than SLACK (base 2): exp(x - m) is then
// up to 2^SLACK, which costs nothing in a floating-point number, and the outputs are rescaled in a few steps, not most.
#pragma once
#include "attend_pass.hpp"

namespace lagkv {

typedef float f32x16 __attribute__((ext_vector_type(16)));

template <int DT>
struct Wide;
template <>
struct Wide<LAGKV_BF16> {
  static constexpr float LIFT = 0.f, SLACK = 8.f;
  static __device__ __forceinline__ f32x16 mma(u32v4 a, u32v4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <>
struct Wide<LAGKV_F16> {
  // 2^(LIFT + SLACK) is in binary16's range; weights down to 2^-34 of the largest are not lost
  static constexpr float LIFT = 10.f, SLACK = 4.f;
  static __device__ __forceinline__ f32x16 mma(u32v4 a, u32v4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};

// N products, of what the reads of LDS give that are made AHEAD products before.  (Left to itself the compiler reads, waits
// and multiplies in turn, in one set of registers.)
template <int N, int AHEAD, typename Read, typename Mul>
__device__ __forceinline__ void products(Read read, Mul mul) {
  u32v4 f[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) f[i] = read(i);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    __builtin_amdgcn_sched_barrier(0);
    mul(i, f[i % AHEAD]);
    if (i + AHEAD < N) f[i % AHEAD] = read(i + AHEAD);
  }
  __builtin_amdgcn_sched_barrier(0);
}

template <int DP>
struct WideShape {
  static constexpr int KT = DP > 128 ? 32 : 64, CPR = DP / 8;  // (the registers hold no more of long rows)
  static constexpr int LDK = DP * 2 + 16, LDV = DP * 2 + 64;  // bytes between rows: sixteen lanes' reads on different banks
  static constexpr int BUF = KT * (LDK + LDV);
};

template <int DT, int DP, int WAVES>
__global__ __launch_bounds__(WAVES * 64, DP <= 128 ? 2 : 1) void attend_wide_kernel(const AttendArgs a) {
  using E = AElem<DT>;
  using W = Wide<DT>;
  using Sh = WideShape<DP>;
  constexpr int KT = Sh::KT, CPR = Sh::CPR, LDK = Sh::LDK, LDV = Sh::LDV, THREADS = WAVES * 64, ROWS = WAVES * 32;
  constexpr int HALVES = KT / 32, KS = DP / 16, DT32 = DP / 32, PASSES = KT * CPR / THREADS;
  static_assert(KT * CPR % THREADS == 0, "");
  extern __shared__ __attribute__((aligned(16))) char wide_lds[];  // two buffers of [K rows][V rows]
  __shared__ int32_t sh_parent[kMaxTree];
  __shared__ uint32_t sh_mask[ROWS * (kMaxTree / 32)];
  __shared__ int sh_odd[2];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, half = lane >> 5;
  const int late = wave >> 2;  // (of the half of eight wavefronts that is a phase behind)

  fetch_arguments<AttendArgs>();
  const WorkItem w = work_item(a);
  if (!w.any) return;
  const uint32_t bu = a.by_h.of((uint32_t)w.unit);
  const int64_t b = bu, h = (uint32_t)w.unit - bu * a.H;
  const int row0 = w.tile * ROWS, row1 = min(row0 + ROWS, a.rows);
  int64_t len = a.lengths ? a.lengths[b] : a.T;
  len = len < 0 ? 0 : len > a.T ? a.T : len;
  const int cache_steps = (int)((len + KT - 1) / KT);
  const int token0 = (int)a.by_g.of(row0), last_token = (int)a.by_g.of(row1 - 1), tokens = last_token - token0 + 1;
  const int seen_new = a.n_new > 0 ? (a.parents ? a.n_new : last_token + 1) : 0;
  const int steps = cache_steps + (seen_new + KT - 1) / KT;
  const int step0 = (int)((int64_t)steps * w.split / a.splits), step1 = (int)((int64_t)steps * (w.split + 1) / a.splits);
  const int n = step1 - step0;

  const int words = (seen_new + 31) / 32;
  if (tid < 2) sh_odd[tid] = 0;

  // q, with the scale's sign: what is left of it is not negative, and the largest logit that of the largest product
  const int r = row0 + wave * 32 + col;
  const bool mine = r < row1, idle = row0 + wave * 32 >= row1;  // (a wavefront without rows loads for the others)
  const int rr = mine ? r : row0, token = (int)a.by_g.of(rr), head = (int)h * a.G + rr - token * a.G;
  const float c = fmaxf(fabsf(a.scale), 1e-30f);
  const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
  u32v4 q[KS];
  {
    const char* p = a.Q + b * a.qsb + head * a.qsh + (int64_t)token * a.qsn;
#pragma unroll
    for (int k = 0; k < KS; ++k) q[k] = *(const u32v4_any*)(p + ((2 * k + half) * 8 < a.D ? slice_at(2 * k + half, a.D, 8) : 0) * 2);
  }

  const char* kb = a.K + b * a.ksb + h * a.ksh;
  const char* vb = a.V + b * a.ksb + h * a.ksh;
  const char* knb = a.K_new + b * a.nsb + h * a.nsh;
  const char* vnb = a.V_new + b * a.nsb + h * a.nsh;
  // This thread's slice of each row it loads, and where it is in the next step's first row.  (Slices behind a row's last
  // repeat its first: q and K are made 0 there, and what V gives for them is not stored.)
  const int lslice = tid % CPR, lrow = tid / CPR;
  const int loff = (lslice * 8 < a.D ? slice_at(lslice, a.D, 8) : 0) * 2;
  constexpr int LROWS = THREADS / CPR;
  struct Tile {
    int64_t first;
    int limit;
    bool fresh;  // of the new tokens
  };
  auto tile_of = [&](int i) {  // i-th step of this piece
    const int step = step0 + i;
    const bool fresh = step >= cache_steps;
    return Tile{(int64_t)(fresh ? step - cache_steps : step) * KT, fresh ? seen_new : (int)len, fresh};
  };
  // (rows of new tokens that every query row of the tile sees, in a chunk of a prompt, need no masks either)
  auto seen_by_all = [&](const Tile& x) { return x.fresh && !a.parents && x.first + KT <= token0 + 1; };
  const int n_whole = min(n, (int)(len / KT) - step0);  // steps of rows of the cache that are all there
  const char* kp = kb + loff + ((int64_t)step0 * KT + lrow) * a.kst;
  const char* vp = vb + loff + ((int64_t)step0 * KT + lrow) * a.kst;
  const int64_t pass = a.kst * LROWS, stride = a.kst * KT;
  u32v4 kr[PASSES], vr[PASSES];
  auto load_edge = [&](int i, const char* cache, const char* tokens_at, u32v4 (&to)[PASSES]) {
    const Tile x = tile_of(i);
    const char* p = (x.fresh ? tokens_at : cache) + loff;
    const int64_t st = x.fresh ? a.nst : a.kst;
#pragma unroll
    for (int k = 0; k < PASSES; ++k) {
      const int64_t row = x.first + lrow + k * LROWS;
      to[k] = *(const u32v4_any*)(p + (row < x.limit ? row : x.limit - 1) * st);
    }
  };
  auto load_next = [&](const char*& p, u32v4 (&to)[PASSES]) {
#pragma unroll
    for (int k = 0; k < PASSES; ++k) to[k] = *(const u32v4_any*)(p + k * pass);
    p += stride;
  };
  // (called for one step after another)
  auto load_k = [&](int i) {
    if (i < n_whole) load_next(kp, kr);
    else if (i < n) load_edge(i, kb, knb, kr);
  };
  auto load_v = [&](int i) {
    if (i < n_whole) load_next(vp, vr);
    else if (i < n) load_edge(i, vb, vnb, vr);
  };
  auto k_at = [&](int i) { return wide_lds + (i & 1) * (KT * LDK); };
  auto v_at = [&](int i) { return wide_lds + 2 * KT * LDK + (i & 1) * (KT * LDV); };
  auto store = [&](const u32v4 (&from)[PASSES], char* to, int ld) {
    to += lrow * ld + lslice * 16;
#pragma unroll
    for (int k = 0; k < PASSES; ++k) *(u32v4*)(to + k * LROWS * ld) = from[k];
  };
  auto store_k = [&](int i) {
    if (a.D != DP) {
#pragma unroll
      for (int k = 0; k < PASSES; ++k) kr[k] = own_channels<8>(kr[k], lslice * 8, a.D);
    }
    store(kr, k_at(i), LDK);
  };
  auto store_v = [&](int i) {
    if (i >= n_whole && i < n) {
      const Tile x = tile_of(i);
      const bool all = seen_by_all(x);
      bool odd = false;
#pragma unroll
      for (int k = 0; k < PASSES; ++k) {
        if (all) break;
        if (x.first + lrow + k * LROWS >= x.limit) vr[k] = u32v4{0, 0, 0, 0};
        if (x.fresh) {
          // what is no finite number is put in as 0 (0 * inf is not) and added to the rows that see it afterwards
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t bits = odd_bits<DT>(vr[k][e]);
            odd = odd || bits;
            vr[k][e] &= ~bits;
          }
        }
      }
      if (x.fresh && odd) sh_odd[i & 1] = 1;
    }
    store(vr, v_at(i), LDV);
  };
  // which of 32 rows from first + 32 t on this lane's query row sees
  auto sees = [&](const Tile& x, int t) {
    const int64_t left = x.limit - (x.first + t * 32);
    uint32_t bits = left >= 32 ? ~0u : left <= 0 ? 0u : (1u << left) - 1u;
    if (x.fresh) {
      const int j = (int)x.first + t * 32;
      if (a.parents) {
        bits &= (j >> 5) < words ? sh_mask[(token - token0) * words + (j >> 5)] : 0u;
      } else {
        const int upto = token - j + 1;
        bits &= upto >= 32 ? ~0u : upto <= 0 ? 0u : (1u << upto) - 1u;
      }
    }
    return bits;
  };

  float m = -INFINITY, l = 0.f;  // m in units of base 2
  f32x16 o[DT32], s[HALVES];
  u32v4 p[2 * HALVES], pl[2 * HALVES];  // P, in steps of 16 rows: its leading bits, and the rest
#pragma unroll
  for (int d = 0; d < DT32; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;

  // Scores of step i and outputs of step i - 1, in one stream of products.  (Before the first step P and V are 0; behind the
  // last the scores are not used.)
  constexpr int NS = KS * HALVES, NO = 2 * HALVES * DT32;
  auto multiply = [&](int i) {
    const char* kl = k_at(i) + col * LDK + half * 16;
    const char* vl = v_at(i - 1) + (half * 4 + (lane & 15) / 4) * LDV + (lane >> 4 & 1) * 32 + (lane & 3) * 8;
#pragma unroll
    for (int t = 0; t < HALVES; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[t][e] = 0.f;
    products<NS + NO, 4>(
        [&](int j) {
          if (j < NS) return *(const u32v4*)(kl + j % HALVES * 32 * LDK + j / HALVES * 32);
          const char* at = vl + (j - NS) / DT32 * 16 * LDV + (j - NS) % DT32 * 64;
          const u32v2 y = __builtin_bit_cast(u32v2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)at));
          const u32v2 z = __builtin_bit_cast(u32v2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(at + 8 * LDV)));
          return u32v4{y.x, y.y, z.x, z.y};
        },
        [&](int j, u32v4 f) {
          if (j < NS) s[j % HALVES] = W::mma(f, q[j < NS ? j / HALVES : 0], s[j % HALVES]);
          else o[(j - NS) % DT32] = W::mma(f, pl[(j - NS) / DT32], W::mma(f, p[(j - NS) / DT32], o[(j - NS) % DT32]));
        });
  };
  // infinities of the rows of step i
  auto strays = [&](int i) {
    const Tile x = tile_of(i);
    if (x.fresh && sh_odd[i & 1] && !seen_by_all(x)) {
      for (int t = 0; t < KT && x.first + t < x.limit; ++t) {
        if (!(sees(x, t >> 5) >> (t & 31) & 1)) continue;
        const char* row = vnb + (x.first + t) * a.nst + half * 8;
#pragma unroll
        for (int d = 0; d < DT32; ++d)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int slice = d * 4 + e;
            if (slice * 8 >= a.D) continue;
            float v[4] = {o[d][4 * e], o[d][4 * e + 1], o[d][4 * e + 2], o[d][4 * e + 3]};
            add_odd<DT>(row + slice_at(slice, a.D, 8) * 2, v);
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) o[d][4 * e + i4] = v[i4];
          }
      }
    }
  };
  auto weights = [&](int i) {
    if (i >= n_whole && !seen_by_all(tile_of(i))) {
      const Tile x = tile_of(i);
#pragma unroll
      for (int t = 0; t < HALVES; ++t) {
        const uint32_t bits = sees(x, t) >> (4 * half);
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (!(bits >> (8 * (e / 4) + e % 4) & 1)) s[t][e] = -INFINITY;
      }
    }
    float top = s[0][0];
#pragma unroll
    for (int t = 0; t < HALVES; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, s[t][e]);
    top = max_across_32(top) * c;
    if (__any(top > m + W::SLACK)) {
      const float now = fmaxf(m, top);
      const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - now);
      m = now;
      l *= keep;
#pragma unroll
      for (int d = 0; d < DT32; ++d) o[d] *= keep;
    }
    const float at = m == -INFINITY ? 0.f : m - W::LIFT;
    float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
    for (int t = 0; t < HALVES; ++t)
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][e], c, -at));
        const float z = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][e + 1], c, -at));
        sum0 += y;
        sum1 += z;
        uint32_t hi, lo;
        E::split(y, z, hi, lo);
        p[t * 2 + e / 8][e % 8 / 2] = hi;
        pl[t * 2 + e / 8][e % 8 / 2] = lo;
      }
    l += sum0 + sum1;
  };

  if (n > 0) {
#pragma unroll
    for (int k = 0; k < 2 * HALVES; ++k) p[k] = pl[k] = u32v4{0, 0, 0, 0};
    for (int k = tid; k < KT * LDV / 16; k += THREADS) *(u32v4*)(v_at(1) + k * 16) = u32v4{0, 0, 0, 0};
    load_k(0);
    load_v(0);
    if (a.parents && step1 > cache_steps)
      ancestors(a.parents + b * a.psb, a.N, token0, tokens, words, sh_parent, sh_mask, tid, THREADS);
    // q's channels that the slice before has, and those behind its row's end, are 0.  (It is waited for here, behind the
    // first rows' loads, and not with what else is on its way in every step.)
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      u32v4 v = mine ? own_channels<8>(q[k] ^ flip, (2 * k + half) * 8, a.D) : u32v4{0, 0, 0, 0};
      asm volatile("" : "+v"(v));
      q[k] = v;
    }
    store_k(0);
    load_k(1);
    __syncthreads();
    if (late) {
      store_k(1);
      store_v(0);
      load_k(2);
      load_v(1);
      __syncthreads();
    }
    for (int i = 0; i <= n; ++i) {
      if (!idle) {
        multiply(i);
        if (i > n_whole) strays(i - 1);
      }
      if (WAVES == 8) __syncthreads();  // (four wavefronts write buffers that nobody reads in this step)
      if (i < n) {
        if (!idle) weights(i);
        store_k(i + late + 1);  // (behind the last step: what was there)
        store_v(i + late);
        load_k(i + late + 2);
        load_v(i + late + 1);
      }
      __syncthreads();
    }
    if (!late) __syncthreads();
  }

  if (!mine) return;
  l = sum_across_32(l);
  const bool whole = a.D % 8 == 0;
  if (a.splits > 1) {
    const int64_t at = (w.unit * a.splits + w.split) * a.rows + r;
    float* po = a.part_o + at * a.part_ld;
#pragma unroll
    for (int d = 0; d < DT32; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int slot = d * 32 + 8 * e + 4 * half, begin = slot & ~7;
        if (begin >= a.D) continue;
        const f32x4 v = {o[d][4 * e], o[d][4 * e + 1], o[d][4 * e + 2], o[d][4 * e + 3]};
        if (whole) {
          *(f32x4*)(po + slot) = v;
        } else {
          const int base = slice_at(begin / 8, a.D, 8), dup = begin - base;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if ((slot & 7) + i >= dup) po[base + (slot & 7) + i] = v[i];
        }
      }
    if (half == 0) {
      a.part_ml[at * 2] = m - W::LIFT + E::LIFT;  // (the same state, with the factor that the join counts on)
      a.part_ml[at * 2 + 1] = l;
    }
    return;
  }
  bool blind = l == 0.f;
  if (a.parents) {
    const int up = a.parents[b * a.psb + token];
    blind = blind || up < -1 || up >= token;
  }
  const float inv = blind ? 0.f : 1.f / l;
  char* op = a.out + b * a.osb + head * a.osh + (int64_t)token * a.osn;
  const bool wide_out = whole && !(((uintptr_t)a.out | a.osb | a.osh | a.osn) & 7);
#pragma unroll
  for (int d = 0; d < DT32; ++d)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int slot = d * 32 + 8 * e + 4 * half, begin = slot & ~7;
      if (begin >= a.D) continue;
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = blind ? 0.f : o[d][4 * e + i] * inv;
      const u32v2 y = {E::pack(v[0], v[1]), E::pack(v[2], v[3])};
      if (wide_out) {
        *(u32v2*)(op + slot * 2) = y;
      } else {
        const int base = slice_at(begin / 8, a.D, 8), dup = begin - base;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if ((slot & 7) + i >= dup) *(uint16_t*)(op + (base + (slot & 7) + i) * 2) = (uint16_t)(y[i / 2] >> (16 * (i % 2)));
      }
    }
  if (half == 0 && a.lse)
    a.lse[(b * a.H * a.G + head) * a.N + token] = blind ? -INFINITY : (m + __builtin_amdgcn_logf(l) - W::LIFT) * 0.693147180559945f;
}

template <int DT, int DP, int WAVES>
hipError_t launch_wide_as(const AttendArgs& a, hipStream_t s) {
  const int64_t groups = (a.units * a.splits + 7) / 8 * 8 * a.row_tiles;
  constexpr size_t lds = 2 * WideShape<DP>::BUF;
  auto kernel = attend_wide_kernel<DT, DP, WAVES>;
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  kernel<<<dim3((uint32_t)groups), dim3(WAVES * 64), lds, s>>>(a);
  return hipGetLastError();
}

template <int DT>
hipError_t launch_wide_of(const AttendArgs& a, int row_tile, hipStream_t s) {
  if (a.D <= 64) return launch_wide_as<DT, 64, 4>(a, s);
  if (a.D <= 128) return row_tile == 128 ? launch_wide_as<DT, 128, 4>(a, s) : launch_wide_as<DT, 128, 8>(a, s);
  return launch_wide_as<DT, 256, 4>(a, s);
}

}  // namespace lagkv
