// Attention of many query rows over rows in 8 bits (lagkv_attend_quantized of 16-bit types; when it is taken, quant_plan_of says).
// attend_wide.hpp's way, by workgroups of four wavefronts with 32 query rows each, with quant_attend.hpp's numbers: the rows in LDS are of 16 bits,
// made of codes on the way from the registers that they are loaded into, and the scales of a step lie beside them.  (Eight wavefronts, 256 query rows, in
// two phases as there were the better ones of 14 in 100 of 528 shapes, by 4 % in the mean.)
//
// A lane has one query row and, of 32 cache rows, eight of the first sixteen and eight of the others in its registers, and scales are those of
// sixteen rows: a logit's goes into the factor that it is multiplied by anyway, and a weight's into what is taken from the logit, as its logarithm.
//
// Codes become numbers behind the products, one word at a time, and a wavefront that multiplies goes before the other workgroup's on its SIMD,
// whose weights then fill the cycles between products: without either 212 us in place of 183, with one of them alone 209 and 205 (256
// query rows of 32 streams x 33536 rows, 128 channels, bf16, int8; weights as one number, as in the next comparisons).  Given to the wavefront that
// makes weights, priority gains 2 us.
//
// Bound by the vector instructions (some 335 a step and wavefront, 64 % of the cycles) and the matrix cores (48 products of 32 cycles, 59 %) together, of which two
// wavefronts on a SIMD overlap a part: 217 to 221 us for those rows in e4m3, 0.65 Pflop/s (a product with V counted once).
#pragma once
#include "attend_wide.hpp"
#include "quant_attend.hpp"

namespace lagkv {

constexpr float kLargeLogit = 0x1p16f;  // in base 2

template <int DP>
struct QuantWideShape {
  static constexpr int KT = DP > 128 ? 32 : 64, SUBS = KT / 16, CPR = DP / 16;
  static constexpr int LDK = DP * 2 + 16, LDV = DP * 2 + 64;  // bytes between rows, as in WideShape
  static constexpr int BUF = KT * (LDK + LDV);
};

// The part of a piece that is in 8 bits; returns the state that it leaves, as attend_wide_body goes on from it, and the steps that the unit's
// rows in 8 bits are.  `others`: steps of the rows behind them.
template <int DT, int CODE, int DP>
__device__ __forceinline__ WideState<DP> attend_quant_wide_body(const QuantArgs& a, const WorkItem& w, char* wide_lds, int others, int& steps) {
  constexpr int KEY = kKeyType<DT>;
  using W = Wide<LAGKV_F16>;
  using Sh = QuantWideShape<DP>;
  constexpr int KT = Sh::KT, SUBS = Sh::SUBS, CPR = Sh::CPR, LDK = Sh::LDK, LDV = Sh::LDV, THREADS = 256, ROWS = 128;
  constexpr int HALVES = KT / 32, KS = DP / 16, DT32 = DP / 32, PASSES = KT * CPR / THREADS;
  static_assert(KT * CPR % THREADS == 0, "");
  __shared__ __attribute__((aligned(16))) float sh_scale[2][2][4];  // of a step's sixteens of K, of V
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, half = lane >> 5;

  const uint32_t bu = a.by_h.of((uint32_t)w.unit);
  const int64_t b = bu, h = (uint32_t)w.unit - bu * (uint32_t)a.H;
  const int row0 = w.tile * ROWS, row1 = min(row0 + ROWS, a.rows);
  int64_t held = a.lengths ? a.lengths[b] : a.T;
  const int len = (int)(held < 0 ? 0 : held > a.T ? a.T : held);
  steps = (int)(((int64_t)len + KT - 1) / KT);
  const int all = steps + others, step0 = min((int)((int64_t)all * w.split / a.splits), steps);
  const int step1 = min((int)((int64_t)all * (w.split + 1) / a.splits), steps);
  const int n = step1 - step0, n_whole = min(n, len / KT - step0);  // steps, and those whose rows are all there

  const int r = row0 + wave * 32 + col;
  const bool mine = r < row1, idle = row0 + wave * 32 >= row1;  // (a wavefront without rows loads for the others)
  const int rr = mine ? r : row0, token = (int)a.by_g.of(rr), head = (int)h * a.G + rr - token * a.G;
  // In LDS a row has the first halves of its slices and then the second ones: what a lane writes at a time lies beside what its neighbours
  // write.  `eight` gives the eight channels that the i-th eight there are.
  auto eight = [](int i) { return i < CPR ? 2 * i : 2 * (i - CPR) + 1; };
  QuerySlots<DT> raw[KS];
  {
    const char* p = a.Q + b * a.qsb + head * a.qsh + (int64_t)token * a.qsn;
#pragma unroll
    for (int k = 0; k < KS; ++k) raw[k].load(p, eight(2 * k + half), a.D);
  }

  // This thread's slice of each row it loads, and where it is in the next step's first row.
  const int lslice = tid % CPR, lrow = tid / CPR;
  const int loff = lslice * 16 < a.D ? slice_at(lslice, a.D, 16) : 0;
  constexpr int LROWS = THREADS / CPR;
  const char* kb = a.Kq + b * a.csb + h * a.csh + loff;
  const char* vb = a.Vq + b * a.csb + h * a.csh + loff;
  const float* sb = ((tid & 4) ? a.vs : a.ks) + b * a.ssb + h * a.ssh;
  const char* kp = kb + ((int64_t)step0 * KT + lrow) * a.cst;
  const char* vp = vb + ((int64_t)step0 * KT + lrow) * a.cst;
  const int64_t pass = a.cst * LROWS, stride = a.cst * KT;
  u32v4 kr[PASSES], vr[PASSES];
  float scale_in = 0.f;  // of threads 0 to 7: a step's scales of K, of V
  auto load_rows = [&](int i, const char*& p, const char* base, u32v4 (&to)[PASSES]) {
    if (i < n_whole) {
#pragma unroll
      for (int k = 0; k < PASSES; ++k) to[k] = *(const u32v4_bytes*)(p + k * pass);
      p += stride;
    } else if (i < n) {
#pragma unroll
      for (int k = 0; k < PASSES; ++k) {
        const int row = (step0 + i) * KT + lrow + k * LROWS;
        to[k] = *(const u32v4_bytes*)(base + (int64_t)(row < len ? row : len - 1) * a.cst);
      }
    }
  };
  // (called for one step after another)
  auto load_k = [&](int i) {
    load_rows(i, kp, kb, kr);
    if (i < n) scale_in = sb[min((step0 + i) * KT + (tid & 3) * 16, len - 1) >> a.block_shift];
  };
  auto load_v = [&](int i) { load_rows(i, vp, vb, vr); };
  auto k_at = [&](int i) { return wide_lds + (i & 1) * (KT * LDK); };
  auto v_at = [&](int i) { return wide_lds + 2 * KT * LDK + (i & 1) * (KT * LDV); };
  auto store = [&](const u32v4 (&from)[PASSES], char* to, int ld, auto type) {
    to += lrow * ld + lslice * 16;
#pragma unroll
    for (int k = 0; k < PASSES; ++k) {
      u32v4 lo, hi;
      numbers_of<CODE, decltype(type)::value>(from[k], lo, hi);
      *(u32v4*)(to + k * LROWS * ld) = lo;
      *(u32v4*)(to + k * LROWS * ld + CPR * 16) = hi;
    }
  };
  auto store_scales = [&](int i) {
    if (tid < 8) sh_scale[i & 1][tid >> 2][tid & 3] = scale_in;
  };
  auto clear_v = [&](int i) {
    // (a row that is not there: its codes may be no numbers)
#pragma unroll
    for (int k = 0; k < PASSES; ++k)
      if ((step0 + i) * KT + lrow + k * LROWS >= len) vr[k] = u32v4{0, 0, 0, 0};
  };

  float c = 0.f;                   // what a query row's products are multiplied by, without the cache rows' scales
  Sums sum;                        // (l of this half's cache rows)
  float k_most = 0.f;              // a scale of K with which logits may be large
  int base = kNoBase;
  f32x16 o[DT32];
  constexpr int PP = kWeightParts;
  u32v4 q[KS], p[2 * HALVES][PP];  // P, in steps of 16 rows
#pragma unroll
  for (int d = 0; d < DT32; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;

  // Scores of step i and outputs of step i - 1, in one stream of products; behind every second one four codes of V of step i, then of K of step
  // i + 1, become numbers, and go to LDS when they are eight.  (Before the first step P and V are 0; behind the last the scores are not used, nor what
  // is written.)
  constexpr int NS = KS * HALVES, NO = 2 * HALVES * DT32;
  static_assert(NS + NO == 2 * (2 * PASSES * 4), "");
  auto multiply = [&](int i, f32x16 (&s)[HALVES]) {
    const char* kl = k_at(i) + col * LDK + half * 16;
    const char* vl = v_at(i - 1) + (half * 4 + (lane & 15) / 4) * LDV + (lane >> 4 & 1) * 32 + (lane & 3) * 8;
#pragma unroll
    for (int t = 0; t < HALVES; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[t][e] = 0.f;
    u32v4 eight_now;
    products<NS + NO, 4>(
        [&](int j) {
          if (j < NS) return *(const u32v4*)(kl + j % HALVES * 32 * LDK + j / HALVES * 32);
          const char* at = vl + (j - NS) / DT32 * 16 * LDV + (j - NS) % DT32 * 64;
          const u32v2 y = __builtin_bit_cast(u32v2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)at));
          const u32v2 z = __builtin_bit_cast(u32v2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(at + 8 * LDV)));
          return u32v4{y.x, y.y, z.x, z.y};
        },
        [&](int j, u32v4 f) {
          if (j < NS) s[j % HALVES] = Wide<KEY>::mma(f, q[j < NS ? j / HALVES : 0], s[j % HALVES]);
          else {
#pragma unroll
            for (int k = 0; k < PP; ++k) o[(j - NS) % DT32] = W::mma(f, p[(j - NS) / DT32][k], o[(j - NS) % DT32]);
          }
        },
        [&](int j) {
          if (j % 2 != 0) return;
          const int word = j / 2 % 4, pass_now = j / 8 % PASSES;
          const bool of_k = j / 8 >= PASSES;
          uint32_t x, y;
          if (of_k) codes_as<CODE, KEY>(kr[pass_now][word], x, y);
          else codes_as<CODE, LAGKV_F16>(vr[pass_now][word], x, y);
          eight_now[word % 2 * 2] = x;
          eight_now[word % 2 * 2 + 1] = y;
          if (word % 2 == 1) {
            char* to = (of_k ? k_at(i + 1) : v_at(i)) + (lrow + pass_now * LROWS) * (of_k ? LDK : LDV) + lslice * 16;
            *(u32v4*)(to + word / 2 * CPR * 16) = eight_now;
          }
        });
  };
  // (Rounded by itself, as R was, which is one of them: of logits so large that fp32 does not hold their fractions the difference is to be that of two rounded ones.)
  auto logit = [](float product, float by) {
    float x = product * by;
    asm("" : "+v"(x));
    return x;
  };
  auto weights = [&](int i, f32x16 (&s)[HALVES], auto part) {
    const f32x4 ks = *(const f32x4*)sh_scale[i & 1][0], vs = *(const f32x4*)sh_scale[i & 1][1];
    const int left = decltype(part)::value ? len - (step0 + i) * KT : KT;
    float by[SUBS], of[SUBS];
#pragma unroll
    for (int u = 0; u < SUBS; ++u) by[u] = ks[u] * c;
    float most_of, least_of;
    auto logs = [&] {
#pragma unroll
      for (int u = 0; u < SUBS; ++u) {
        of[u] = u * 16 < left ? log_scale(vs[u], base) : 0.f;  // (rows that are not there have logits of -inf, whatever their scale)
        most_of = u == 0 ? of[0] : fmaxf(most_of, of[u]);
        least_of = u == 0 ? of[0] : fminf(least_of, of[u]);
      }
    };
    logs();
    if constexpr (decltype(part)::value) {
      // Rows that are not there get -inf, by a product of a column that has it for them with ones.  (-inf times a factor of 0 would be none; what is no
      // number stays that.)
#pragma unroll
      for (int t = 0; t < HALVES; ++t)
        s[t] = W::mma(u32v4{half == 0 && t * 32 + col >= left ? 0xfc00u : 0u, 0, 0, 0}, u32v4{0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u}, s[t]);
#pragma unroll
      for (int u = 0; u < SUBS; ++u) by[u] = by[u] < 1e-30f ? 1e-30f : by[u];
    }
    float xs[SUBS];  // the largest logit of each scale's rows (by is not negative)
#pragma unroll
    for (int u = 0; u < SUBS; ++u) {
      float x = s[u / 2][u % 2 * 8];
#pragma unroll
      for (int e = 1; e < 8; ++e) x = fmaxf(x, s[u / 2][u % 2 * 8 + e]);
      xs[u] = logit(x, by[u]);
    }
    bool far_scales = false, large = false;
    float most_k = ks[0];
#pragma unroll
    for (int u = 1; u < SUBS; ++u) most_k = fmaxf(most_k, ks[u]);
    if (__builtin_expect(__any(!(most_of <= kNearBase && least_of >= -kFarBelow && most_k < k_most)), 0)) {
      large = __any(!(most_k < k_most));
      if (__any(most_of > kNearBase)) {
        float most = 0.f;
#pragma unroll
        for (int u = 0; u < SUBS; ++u) most = fmaxf(most, u * 16 < left ? vs[u] : 0.f);
        const int now = __builtin_amdgcn_readfirstlane(__builtin_amdgcn_frexp_expf(most));
        sum.a = fmaxf(sum.a - (float)(now - base), kNoWeight);
        base = now;
        logs();
      }
      far_scales = __any(least_of < -kFarBelow);
    }
    auto largest = [&] {
      float x = -INFINITY;
#pragma unroll
      for (int u = 0; u < SUBS; ++u) x = fmaxf(x, xs[u] - sum.R + of[u]);
      return max_across_32(x);
    };
    float top = largest();
    if (__any(top > sum.a + W::SLACK)) {
      float x = xs[0];
#pragma unroll
      for (int u = 1; u < SUBS; ++u) x = fmaxf(x, xs[u]);
      x = max_across_32(x);
      if (top > sum.a) sum.raise(x, 1.f);
      top = largest();
      if (top > sum.a) {
        const float keep = __builtin_amdgcn_exp2f(sum.a - top);
#pragma unroll
        for (int d = 0; d < DT32; ++d) o[d] *= keep;
        sum.a = top;
      }
    }
    uint32_t apart = 0;  // sixteens whose weights are summed by themselves
    if (__builtin_expect(far_scales, 0)) {
      float x = -INFINITY, none = 0.f;
#pragma unroll
      for (int u = 0; u < SUBS; ++u) {
        none += u * 16 < left ? vs[u] : 0.f;
        if (sum.a - of[u] > kFar) {
          apart |= 1u << u;
          x = fmaxf(x, xs[u]);
        }
      }
      sum.raise(max_across_32(x), 1.f);
#pragma unroll
      for (int u = 0; u < SUBS; ++u)
        if (apart >> u & 1) {
#pragma unroll
          for (int e = 0; e < 8; ++e) sum.l += __builtin_amdgcn_exp2f(logit(s[u / 2][u % 2 * 8 + e], by[u]) - sum.R + W::LIFT);
        }
      // (a scale that is no number: neither are the outputs)
      if (none != none) {
#pragma unroll
        for (int d = 0; d < DT32; ++d) o[d] *= none;
      }
    }
    float total[SUBS];
    auto exponentials = [&](auto weight_of) {
#pragma unroll
      for (int u = 0; u < SUBS; ++u) {
        float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const float y = weight_of(u, s[u / 2][u % 2 * 8 + e]), z = weight_of(u, s[u / 2][u % 2 * 8 + e + 1]);
          sum0 += y;
          sum1 += z;
          uint32_t part[PP];
          split_weights(y, z, part);
#pragma unroll
          for (int k = 0; k < PP; ++k) p[u][k][e / 2] = part[k];
        }
        total[u] = sum0 + sum1;
      }
    };
    float more[SUBS];
#pragma unroll
    for (int u = 0; u < SUBS; ++u) more[u] = of[u] - (sum.a - W::LIFT) - (large ? 0.f : sum.R);
    if (__builtin_expect(large, 0)) exponentials([&](int u, float x) { return __builtin_amdgcn_exp2f(logit(x, by[u]) - sum.R + more[u]); });
    else exponentials([&](int u, float x) { return __builtin_amdgcn_exp2f(__builtin_fmaf(x, by[u], more[u])); });
    if (__builtin_expect(far_scales, 0)) {
#pragma unroll
      for (int u = 0; u < SUBS; ++u)
        if (!(apart >> u & 1)) sum.l = __builtin_fmaf(total[u], __builtin_amdgcn_exp2f(sum.a - of[u]), sum.l);
    } else {
#pragma unroll
      for (int u = 0; u < SUBS; ++u) sum.l = __builtin_fmaf(total[u], __builtin_amdgcn_exp2f(sum.a - of[u]), sum.l);
    }
  };

  if (n > 0) {
#pragma unroll
    for (int k = 0; k < 2 * HALVES; ++k)
#pragma unroll
      for (int i = 0; i < PP; ++i) p[k][i] = u32v4{0, 0, 0, 0};
    for (int k = tid; k < KT * LDV / 16; k += THREADS) *(u32v4*)(v_at(1) + k * 16) = u32v4{0, 0, 0, 0};
    load_k(0);
    load_v(0);
    // q, with the scale's sign: what is left of it is not negative, and the largest logit that of the largest product.  (It is waited for
    // here, behind the first rows' loads.)
    {
      const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
      float most = 0.f, size = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        raw[k].own(eight(2 * k + half), a.D, mine);
        if constexpr (DT != LAGKV_F16) most = raw[k].most(most);
#pragma unroll
        for (int e = 0; e < 8; ++e) size += fabsf(raw[k].at(e));
      }
      k_most = kLargeLogit / (sum_across_32(size) * fabsf(a.scale) * (CODE == LAGKV_CODE_INT8 ? 128.f : 448.f));
      const QueryUnit u(max_across_32(most));
      c = fabsf(a.scale) * (DT == LAGKV_F16 ? 1.f : u.unit);
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        u32v4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          v[i] = (DT == LAGKV_F16 ? raw[k].w[i] : __builtin_amdgcn_perm(__float_as_uint(raw[k].at(2 * i + 1) * u.by), __float_as_uint(raw[k].at(2 * i) * u.by), 0x07060302u)) ^ flip;
        asm volatile("" : "+v"(v));
        q[k] = v;
      }
    }
    store(kr, k_at(0), LDK, std::integral_constant<int, KEY>());
    store_scales(0);
    load_k(1);
    __syncthreads();
    // (one barrier a step: what is written in one are the buffers that nobody reads in it)
    auto load_next = [&](int i) {
      store_scales(i + 1);  // (behind the last step: what was there)
      load_k(i + 2);
      load_v(i + 1);
    };
    // (A wavefront without rows has a loop of its own, and so have the steps whose rows are all there: where the scores of two ways come together they
    // are copied in every step.  256 channels 164 us without, 145 with; 64 channels 94 and 90.)
    if (idle) {
      for (int i = 0; i <= n; ++i) {
        if (i < n) {
          if (i >= n_whole) clear_v(i);
          store(vr, v_at(i), LDV, std::integral_constant<int, LAGKV_F16>());
          store(kr, k_at(i + 1), LDK, std::integral_constant<int, KEY>());
          load_next(i);
        }
        __syncthreads();
      }
    } else {
      auto step = [&](int i, auto part) {
        f32x16 s[HALVES];
        if (decltype(part)::value && i < n) clear_v(i);
        __builtin_amdgcn_s_setprio(1);
        multiply(i, s);
        __builtin_amdgcn_s_setprio(0);
        if (i < n) {
          load_next(i);
          weights(i, s, part);
        }
        __syncthreads();
      };
      int i = 0;
      for (; i < n_whole; ++i) step(i, std::false_type());
      for (; i <= n; ++i) step(i, std::true_type());
    }
  }

  // Relative to the sum's reference, with the type's factor in place of this kernel's, and channels where attend_wide_body has them.  (A last slice of sixteen that
  // is no whole one has the row's last eight channels, of which there are at most eight of its own, as its second half.)
  constexpr int LIFT = (int)(Wide<DT>::LIFT - W::LIFT);
  const Power of(sum.a, base + LIFT);
  WideState<DP> x;
#pragma unroll
  for (int i = 0; i < DP / 8; ++i) {
    const int to = eight(i);
#pragma unroll
    for (int e = 0; e < 4; ++e) x.o[to / 4][to % 4 * 4 + e] = of.times(o[i / 4][i % 4 * 4 + e]);
  }
#pragma unroll
  for (int slice = 0; slice < CPR; ++slice)
    if (slice * 16 < a.D && a.D < slice * 16 + 16) {
#pragma unroll
      for (int e = 0; e < 4; ++e) x.o[slice / 2][slice % 2 * 8 + e] = x.o[slice / 2][slice % 2 * 8 + 4 + e];
    }
  x.m = sum.reference();
  x.l = __builtin_ldexpf(sum.l, LIFT);
  return x;
}

// A piece goes over the rows in 8 bits, the tail and the new tokens as one line of steps: its workgroup does what of it is in 8 bits, and goes
// on with the rest.  (With workgroups apart, as in BesideCodes, 290 query rows of 128 streams x 508 rows and 8 took 62 us in place of
// 48: every piece of a query row is 4 bytes a channel, written and read.)
template <int DT, int CODE, int DP>
struct AfterCodes {
  using Args = QuantBoth;
  static constexpr bool ALONE = false;
  static __device__ __forceinline__ const AttendArgs& rows(const Args& a) { return a.rows; }
  static __device__ __forceinline__ WideState<DP> go(const Args& a, const WorkItem& w, char* lds, int others, int& steps) {
    return attend_quant_wide_body<DT, CODE, DP>(a.codes, w, lds, others, steps);
  }
};

template <int DT, int CODE, int DP>
hipError_t launch_quant_wide_as(const QuantBoth& a, int64_t groups, hipStream_t s) {
  static_assert(QuantWideShape<DP>::BUF == WideShape<DP>::BUF, "");
  constexpr int lds = 2 * QuantWideShape<DP>::BUF;
  auto kernel = attend_wide_kernel<DT, DP, 4, AfterCodes<DT, CODE, DP>>;
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  kernel<<<dim3((uint32_t)groups), dim3(256), lds, s>>>(a);
  return hipGetLastError();
}
template <int DT, int CODE>
hipError_t launch_quant_wide_code(const QuantBoth& a, int64_t groups, hipStream_t s) {
  if (a.codes.D <= 64) return launch_quant_wide_as<DT, CODE, 64>(a, groups, s);
  return a.codes.D <= 128 ? launch_quant_wide_as<DT, CODE, 128>(a, groups, s) : launch_quant_wide_as<DT, CODE, 256>(a, groups, s);
}
template <int DT>
hipError_t launch_quant_wide_of(const QuantBoth& a, int64_t groups, int code, hipStream_t s) {
  return code == LAGKV_CODE_INT8 ? launch_quant_wide_code<DT, LAGKV_CODE_INT8>(a, groups, s) : launch_quant_wide_code<DT, LAGKV_CODE_E4M3>(a, groups, s);
}

}  // namespace lagkv
