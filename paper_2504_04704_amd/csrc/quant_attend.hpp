// Attention of few query rows over rows in 8 bits (lagkv_attend_quantized; the mathematics is attend_pass.hpp's).
//
// With codes k_t, v_t and their blocks' scales s_t, r_t the logits are x_t = scale s_t q.k_t and the outputs sum (p_t r_t) v_t: a
// scale is a factor of a logit and of a weight, and the products take the codes as they are.  Binary16 holds them (whole numbers up to 128,
// and numbers of 4 mantissa bits from 2^-9 to 448), and so does bf16: the products with V go to the matrix cores in the first, with q in its own type (fp32: as three
// numbers of bf16).
//
// A wavefront takes every fourth step of 64 cache rows (32 where 64 do not fit the registers) for all query rows of its workgroup; K's codes become
// numbers in the registers that they are loaded into, V's on their way into LDS.  Scales are those of sixteen rows that
// lie in one block.  Weights times scales go in as two numbers of binary16 (split_weights).  They are exponentials of logits with their scale's
// logarithm, relative to the largest of these, so that it does not matter how far apart scales are, nor which of them comes first; the weights' sum is without the
// scales (see Sums).
//
// Each piece of a cache leaves its maximum, sum and outputs; launch_attend_join joins them with those of the tail and the new tokens, which
// other workgroups of the same launch have gone over.
//
// Bound by memory where there are rows enough: one token each of 32 requests, 8 heads of 128 channels (bf16, up to 8128 rows in int8 and 256 behind them)
// 85 to 90 us, 5.0 TB/s, and 4 for the join; where there are few, by latency: one request's 4032 rows 10.7 us and 2.5 to 3.
#pragma once
#include "code_ops.hpp"
#include "quant_internal.hpp"

namespace lagkv {

constexpr float kQuantLift = 14.f;  // weights are held times 2^14, as in AElem<LAGKV_F16>

// Logarithms of scales of V are those of base 2 less `base`, an exponent near the largest of those met so far: they are small numbers then, and so are their roundings.
// (-inf of 0, of what is below 2^-126 of 2^base, and of what is no number, with which the outputs are none anyway.)
constexpr int kNoBase = -1000;  // (any scale is inf beside it)
constexpr float kNearBase = 16.f;
__device__ __forceinline__ float log_scale(float s, int base) { return fmaxf(__builtin_amdgcn_logf(__builtin_ldexpf(s, -base)), -INFINITY); }

// What a query row's sums are relative to.  R is a logit near the largest: l = sum exp(x - R) over its rows.  The weights in the products have their row's scale exp(s) in them, and
// are relative to exp(R + a), a the largest x - R + s: o = sum exp(x - R + s - a) v.  (R and a by themselves: their sum would lose a where R is large.)  l is made of the same exponentials,
// of sixteen rows of a scale times exp(a - s).  That is done up to 2^kFar; beyond, those may have left the range of fp32 while they are a large part of the sum,
// and are worked out by themselves.  (a is of a row whose logit R is not below and whose s is kNearBase + 1 at most: from s = -kFarBelow on the factor is no larger.)
constexpr float kFar = 64.f, kFarBelow = kFar - kNearBase - 1.f;
constexpr float kNoLogit = -3.40282347e38f, kNoWeight = -1e30f;  // R and a where there are none yet: less than any, but numbers
struct Sums {
  float R = kNoLogit, l = 0.f, a = kNoWeight;  // a in base 2
  __device__ __forceinline__ void raise(float to, float unit) {
    if (to > R) {
      const float down = (R - to) * unit;
      l *= __builtin_amdgcn_exp2f(down);
      a = fmaxf(a + down, kNoWeight);
      R = to;
    }
  }
  // R as it is joined with others': what is no number, or saw nothing, has -inf
  __device__ __forceinline__ float reference() const { return R == kNoLogit ? -INFINITY : R; }
};

// 2^(x + more), as a factor of what may be as far from 1 as it is.
struct Power {
  float f;
  int e;
  __device__ __forceinline__ Power(float x, int more) {
    const float whole = fmaxf(floorf(x), -2000.f);
    f = __builtin_amdgcn_exp2f(x - whole);
    e = (int)whole + more;
  }
  __device__ __forceinline__ float times(float y) const { return __builtin_ldexpf(y * f, e); }
};

template <int DP, int RT>
struct QuantShape {
  static constexpr int SUBS = DP * RT > 128 ? 2 : 4, KT = 16 * SUBS;  // sixteens of a step
  static constexpr int CPR = DP / 16, NC = CPR / 4;              // slices of 16 codes in a row; a lane's of K
  static constexpr int VROWS = 64 / CPR, NV = KT / VROWS;        // rows that a wavefront loads at a time
  static constexpr int ROWS = 16 * RT;
  static constexpr int LDV = DP * 2 + 32;  // bytes between rows of V in LDS
  static constexpr int LDO = DP + 4;       // floats between rows of the outputs in LDS
  static constexpr int V_BYTES = 4 * KT * LDV, O_BYTES = 4 * ROWS * LDO * 4;
  static constexpr int MAIN = V_BYTES > O_BYTES ? V_BYTES : O_BYTES;
};

// Eight slots of a query row: those of codes come in slices of sixteen, of which slice_at gives the channels.  What a slice behind the
// row's end repeats is 0.
template <int DT>
struct QuerySlots {
  static constexpr int ES = AElem<DT>::SIZE;
  uint32_t w[2 * ES];
  __device__ __forceinline__ void load(const char* p, int eight, int D) {
    const int slice = eight >> 1, base = (slice * 16 < D ? slice_at(slice, D, 16) : 0) + (eight & 1) * 8;
#pragma unroll
    for (int i = 0; i < 2 * ES; i += 4) {
      const u32v4 v = *(const u32v4_any*)(p + base * ES + i * 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[i + e] = v[e];
    }
  }
  __device__ __forceinline__ void own(int eight, int D, bool there) {
    const int begin = (eight >> 1) * 16, dup = begin + 16 <= D ? 0 : begin < D ? begin + 16 - D : 16;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool mine = there && (eight & 1) * 8 + e >= dup;
      if constexpr (DT == LAGKV_F32) w[e] = mine ? w[e] : 0u;
      else w[e / 2] &= mine ? ~0u : e % 2 ? 0x0000ffffu : 0xffff0000u;
    }
  }
  __device__ __forceinline__ float at(int e) const {
    if constexpr (DT == LAGKV_F32) return __uint_as_float(w[e]);
    else return AElem<DT>::one((uint16_t)(w[e / 2] >> (16 * (e % 2))));
  }
  // the largest finite magnitude
  __device__ __forceinline__ float most(float m) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = fabsf(at(e));
      m = fmaxf(m, x < INFINITY ? x : 0.f);
    }
    return m;
  }
};
// The power of two, near a row's largest magnitude, that is taken out of the row before the products (which might leave fp32's range otherwise); and its inverse.
// What is 2^-126 of the largest and more goes in as it is.
struct QueryUnit {
  float unit, by;
  __device__ __forceinline__ explicit QueryUnit(float most) {
    const uint32_t exponent = min(max(__float_as_uint(most) >> 23, 1u), 253u);
    unit = __uint_as_float(exponent << 23);
    by = __uint_as_float((254u - exponent) << 23);
  }
};

// A lane's part of a query row: eight slots of each of 2 * NC, of bf16 and fp32 times a power of two.  fp32 is three numbers of bf16, each the leading bits of what
// the ones before it leave.
template <int DT, int NC>
struct Query {
  static constexpr int PARTS = DT == LAGKV_F32 ? 3 : 1;
  u32v4 part[PARTS][2 * NC];
  float unit;  // that power's inverse
  __device__ __forceinline__ void load(const char* p, int grp, int D, bool there) {
    QuerySlots<DT> raw[2 * NC];
    auto eight = [&](int j) { return (j / 2 * 4 + grp) * 2 + j % 2; };
#pragma unroll
    for (int j = 0; j < 2 * NC; ++j) raw[j].load(p, eight(j), D);
#pragma unroll
    for (int j = 0; j < 2 * NC; ++j) raw[j].own(eight(j), D, there);
    if constexpr (DT == LAGKV_F16) {
      unit = 1.f;
#pragma unroll
      for (int j = 0; j < 2 * NC; ++j) part[0][j] = u32v4{raw[j].w[0], raw[j].w[1], raw[j].w[2], raw[j].w[3]};
    } else {
      float most = 0.f;
#pragma unroll
      for (int j = 0; j < 2 * NC; ++j) most = raw[j].most(most);
      const QueryUnit u(max_across_32(max_across_16(most)));
      unit = u.unit;
#pragma unroll
      for (int j = 0; j < 2 * NC; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t x = __float_as_uint(raw[j].at(2 * i) * u.by), y = __float_as_uint(raw[j].at(2 * i + 1) * u.by);
#pragma unroll
          for (int k = 0; k < PARTS; ++k) {
            part[k][j][i] = __builtin_amdgcn_perm(y, x, 0x07060302u);
            if (k + 1 == PARTS) break;
            // (nothing is left of an infinity or of what is no number, which the first part is)
            auto rest = [](uint32_t v) {
              const float all = __uint_as_float(v), lead = __uint_as_float(v & 0xffff0000u);
              return __float_as_uint(fabsf(all) < INFINITY ? all - lead : 0.f);
            };
            x = rest(x);
            y = rest(y);
          }
        }
    }
  }
};

// Sixteen codes as eight numbers twice, of binary16 or bf16.
template <int CODE, int DT>
__device__ __forceinline__ void numbers_of(u32v4 w, u32v4& lo, u32v4& hi) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t a, b;
    codes_as<CODE, DT>(w[i], a, b);
    lo[2 * i] = a;
    lo[2 * i + 1] = b;
    codes_as<CODE, DT>(w[2 + i], a, b);
    hi[2 * i] = a;
    hi[2 * i + 1] = b;
  }
}

// What a workgroup does with a piece of the rows in 8 bits.
template <int DT, int CODE, int DP, int RT>
__device__ __forceinline__ void attend_quant_body(const QuantArgs& a, const WorkItem& w, char* quant_lds) {
#pragma clang fp contract(off)  // (a logit is rounded before R, one of them, is taken from it: where logits are large, the rounding is more than a weight's exponent holds)
  using E = AElem<DT>;
  using F = AElem<LAGKV_F16>;
  using Sh = QuantShape<DP, RT>;
  constexpr int SUBS = Sh::SUBS, KT = Sh::KT, CPR = Sh::CPR, NC = Sh::NC, VROWS = Sh::VROWS, NV = Sh::NV, ROWS = Sh::ROWS;
  constexpr int LDV = Sh::LDV, LDO = Sh::LDO, DT16 = DP / 16, WAVES = 4, THREADS = 256;
  __shared__ float sh_ml[WAVES][ROWS][2];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 15, grp = lane >> 4;

  const uint32_t bu = a.by_h.of((uint32_t)w.unit);
  const int64_t b = bu, h = (uint32_t)w.unit - bu * (uint32_t)a.H;
  const int row0 = w.tile * ROWS, row1 = min(row0 + ROWS, a.rows);
  const int64_t held = a.lengths ? a.lengths[b] : a.T;
  const int len = (int)(held < 0 ? 0 : held > a.T ? a.T : held);
  const int steps = (int)(((int64_t)len + KT - 1) / KT);
  const int step0 = (int)((int64_t)steps * w.split / a.splits), step1 = (int)((int64_t)steps * (w.split + 1) / a.splits);
  const char* kb = a.Kq + b * a.csb + h * a.csh;
  const char* vb = a.Vq + b * a.csb + h * a.csh;
  const float* ksb = a.ks + b * a.ssb + h * a.ssh;
  const float* vsb = a.vs + b * a.ssb + h * a.ssh;
  char* vl = quant_lds + wave * (KT * LDV);

  auto offset = [&](int slice) { return slice * 16 < a.D ? slice_at(slice, a.D, 16) : 0; };
  const int vslice = lane % CPR, vrow = lane / CPR, voff = offset(vslice);
  int koff[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) koff[c] = offset(c * 4 + grp);
  u32v4 kf[SUBS][NC], vf[NV];
  float ks[SUBS], vs[SUBS];  // of the rows in kf and vf, as the step's scales are loaded with them
  auto load_k = [&](int step) {
    const int first = step * KT;
#pragma unroll
    for (int s = 0; s < SUBS; ++s) {
      const int row = first + s * 16 + col;
      const char* at = kb + (int64_t)(row < len ? row : len - 1) * a.cst;
#pragma unroll
      for (int c = 0; c < NC; ++c) kf[s][c] = *(const u32v4_bytes*)(at + koff[c]);
      ks[s] = ksb[min(first + s * 16, len - 1) >> a.block_shift];
    }
  };
  auto load_v = [&](int step) {
    const int first = step * KT;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int row = first + i * VROWS + vrow;
      vf[i] = *(const u32v4_bytes*)(vb + (int64_t)(row < len ? row : len - 1) * a.cst + voff);
    }
#pragma unroll
    for (int s = 0; s < SUBS; ++s) vs[s] = vsb[min(first + s * 16, len - 1) >> a.block_shift];
  };

  // sixteen channels of 32 rows, as the product with weights takes them
  auto values_at = [&](int d, int t) {
    u32v4 v;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_s16x4)(vl + ((t * 2 + s) * 16 + grp * 4 + (col >> 2)) * LDV + (d * 16 + (col & 3) * 4) * 2));
      const u32v2 y = __builtin_bit_cast(u32v2, x);
      v[s * 2] = y.x;
      v[s * 2 + 1] = y.y;
    }
    return v;
  };

  int step = step0 + wave;
  if (step < step1) {
    load_k(step);
    load_v(step);
  }
  Query<DT, NC> q[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = row0 + rt * 16 + col, rr = r < row1 ? r : row0, n = (int)a.by_g.of(rr);
    q[rt].load(a.Q + b * a.qsb + (h * a.G + rr - n * a.G) * a.qsh + (int64_t)n * a.qsn, grp, a.D, r < row1);
  }
  Sums sum[RT];  // (l of this lane's cache rows)
  f32x4 o[RT][DT16];
  int base = kNoBase;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int d = 0; d < DT16; ++d) o[rt][d] = f32x4{0.f, 0.f, 0.f, 0.f};

  for (; step < step1; step += WAVES) {
    const bool more = step + WAVES < step1, whole = (step + 1) * KT <= len;
    const int first = step * KT;
    wave_order();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      // (a row that is not there: its codes may be no numbers)
      if (!whole && first + i * VROWS + vrow >= len) vf[i] = u32v4{0, 0, 0, 0};
      u32v4 lo, hi;
      numbers_of<CODE, LAGKV_F16>(vf[i], lo, hi);
      char* at = vl + (i * VROWS + vrow) * LDV + vslice * 32;
      *(u32v4*)at = lo;
      *(u32v4*)(at + 16) = hi;
    }
    wave_order();
    float scale[SUBS], of[SUBS];  // of V, and their logarithms
#pragma unroll
    for (int s = 0; s < SUBS; ++s) scale[s] = whole || first + s * 16 < len ? vs[s] : 0.f;
    if (more) load_v(step + WAVES);
    __builtin_amdgcn_sched_barrier(0);

    f32x4 p[RT][SUBS];
    float x_scale[SUBS];
#pragma unroll
    for (int s = 0; s < SUBS; ++s) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) p[rt][s] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        u32v4 k[2];
        numbers_of<CODE, kKeyType<DT>>(kf[s][c], k[0], k[1]);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int part = 0; part < Query<DT, NC>::PARTS; ++part) p[rt][s] = AElem<kKeyType<DT>>::mma(k[i], q[rt].part[part][c * 2 + i], p[rt][s]);
      }
      x_scale[s] = ks[s] * a.scale;
    }
    __builtin_amdgcn_sched_barrier(0);
    if (more) load_k(step + WAVES);
    __builtin_amdgcn_sched_barrier(0);

    float most_of, least_of;
    auto logs = [&] {
#pragma unroll
      for (int s = 0; s < SUBS; ++s) {
        // (rows that are not there have logits of -inf, whatever their scale)
        of[s] = whole || first + s * 16 < len ? log_scale(scale[s], base) : 0.f;
        most_of = s == 0 ? of[0] : fmaxf(most_of, of[s]);
        least_of = s == 0 ? of[0] : fminf(least_of, of[s]);
      }
    };
    logs();
    if (__any(most_of > kNearBase)) {
      float most = 0.f;
#pragma unroll
      for (int s = 0; s < SUBS; ++s) most = fmaxf(most, scale[s]);
      const int now = __builtin_amdgcn_readfirstlane(__builtin_amdgcn_frexp_expf(most));
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) sum[rt].a = fmaxf(sum[rt].a - (float)(now - base), kNoWeight);
      base = now;
      logs();
    }
    const bool far_scales = __any(least_of < -kFarBelow);
    constexpr int PP = kWeightParts;
    u32v4 weight[RT][SUBS / 2][PP];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
      for (int s = 0; s < SUBS; ++s) p[rt][s] *= x_scale[s] * q[rt].unit;
      if (!whole) {
#pragma unroll
        for (int s = 0; s < SUBS; ++s)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (first + s * 16 + grp * 4 + i >= len) p[rt][s][i] = -INFINITY;
      }
      float most[SUBS];
#pragma unroll
      for (int s = 0; s < SUBS; ++s) most[s] = fmaxf(fmaxf(p[rt][s][0], p[rt][s][1]), fmaxf(p[rt][s][2], p[rt][s][3]));
      auto largest = [&] {
        float x = -INFINITY;
#pragma unroll
        for (int s = 0; s < SUBS; ++s) x = fmaxf(x, __builtin_fmaf(most[s] - sum[rt].R, E::UNIT, of[s]));
        return max_across_32(max_across_16(x));
      };
      float top = largest();
      if (__any(top > sum[rt].a)) {
        float x = most[0];
#pragma unroll
        for (int s = 1; s < SUBS; ++s) x = fmaxf(x, most[s]);
        x = max_across_32(max_across_16(x));
        if (top > sum[rt].a) sum[rt].raise(x, E::UNIT);
        top = largest();
        if (top > sum[rt].a) {
          const float keep = __builtin_amdgcn_exp2f(sum[rt].a - top);
#pragma unroll
          for (int d = 0; d < DT16; ++d) o[rt][d] *= keep;
          sum[rt].a = top;
        }
      }
      uint32_t apart = 0;  // sixteens whose weights are summed by themselves
      if (__builtin_expect(far_scales, 0)) {
        float x = -INFINITY, none = 0.f;
#pragma unroll
        for (int s = 0; s < SUBS; ++s) {
          none += scale[s];
          if (sum[rt].a - of[s] > kFar) {
            apart |= 1u << s;
            x = fmaxf(x, most[s]);
          }
        }
        sum[rt].raise(max_across_32(max_across_16(x)), E::UNIT);
#pragma unroll
        for (int s = 0; s < SUBS; ++s)
          if (apart >> s & 1) {
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[rt].l += __builtin_amdgcn_exp2f(__builtin_fmaf(p[rt][s][i] - sum[rt].R, E::UNIT, kQuantLift));
          }
        // (a scale that is no number: neither are the outputs)
        if (none != none) {
#pragma unroll
          for (int d = 0; d < DT16; ++d) o[rt][d] *= none;
        }
      }
      float y[SUBS];
#pragma unroll
      for (int s = 0; s < SUBS; ++s) {
        y[s] = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          // (the difference first: its rounding is that of a number near zero)
          p[rt][s][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[rt][s][i] - sum[rt].R, E::UNIT, of[s] - sum[rt].a + kQuantLift));
          y[s] += p[rt][s][i];
        }
      }
      if (__builtin_expect(far_scales, 0)) {
#pragma unroll
        for (int s = 0; s < SUBS; ++s)
          if (!(apart >> s & 1)) sum[rt].l = __builtin_fmaf(y[s], __builtin_amdgcn_exp2f(sum[rt].a - of[s]), sum[rt].l);
      } else {
#pragma unroll
        for (int s = 0; s < SUBS; ++s) sum[rt].l = __builtin_fmaf(y[s], __builtin_amdgcn_exp2f(sum[rt].a - of[s]), sum[rt].l);
      }
#pragma unroll
      for (int s = 0; s < SUBS; ++s)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint32_t part[PP];
          split_weights(p[rt][s][2 * i], p[rt][s][2 * i + 1], part);
#pragma unroll
          for (int k = 0; k < PP; ++k) weight[rt][s / 2][k][s % 2 * 2 + i] = part[k];
        }
    }
#pragma unroll
    for (int d = 0; d < DT16; ++d)
#pragma unroll
      for (int t = 0; t < SUBS / 2; ++t) {
        const u32v4 v = values_at(d, t);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int k = 0; k < PP; ++k) o[rt][d] = F::mma(v, weight[rt][t][k], o[rt][d]);
      }
  }

  // the wavefronts' states join, relative to the sums' reference
  constexpr int LIFT = (int)(E::LIFT - kQuantLift);  // what launch_attend_join counts on, over what there is
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float l = sum[rt].l;
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (grp == 0) {
      sh_ml[wave][rt * 16 + col][0] = sum[rt].reference();
      sh_ml[wave][rt * 16 + col][1] = l;
    }
  }
  __syncthreads();  // (V of all wavefronts is done with as well)
  float* ol = (float*)quant_lds;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float top = -INFINITY;
#pragma unroll
    for (int x = 0; x < WAVES; ++x) top = fmaxf(top, sh_ml[x][rt * 16 + col][0]);
    const bool none = sh_ml[wave][rt * 16 + col][1] == 0.f;  // (what is no number has a reference of -inf too, and is not dropped)
    const Power of(fmaxf(sum[rt].a + (sum[rt].R - top) * E::UNIT, kNoWeight), base + LIFT);
#pragma unroll
    for (int d = 0; d < DT16; ++d) {
      f32x4 y;
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = none ? 0.f : of.times(o[rt][d][i]);
      *(f32x4*)(ol + (wave * ROWS + rt * 16 + col) * LDO + d * 16 + grp * 4) = y;
    }
  }
  __syncthreads();
  constexpr int QUADS = DP / 4;
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
    const int slot = quad * 4, begin = slot / 16 * 16;
    const int base = begin < a.D ? slice_at(slot / 16, a.D, 16) : 0, dup = begin - base, within = slot - begin;
    const int64_t at = (w.unit * a.part_splits + w.split) * a.rows + r;
    if (begin < a.D && dup == 0) {
      *(f32x4*)(a.part_o + at * a.part_ld + slot) = v;
    } else if (begin < a.D) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (within + e >= dup) a.part_o[at * a.part_ld + base + within + e] = v[e];
    }
    if (quad == 0) {
      a.part_ml[at * 2] = top;
      a.part_ml[at * 2 + 1] = __builtin_ldexpf(sum, LIFT);
    }
  }
}

// The pieces of rows in 8 bits and, by attend_pass.hpp's way, those of the tail and the new tokens: workgroups of one launch.
template <int DT, int CODE, int DP, int RT>
struct BesideCodes {
  using Args = QuantBoth;
  static constexpr bool ALONE = false;
  static __device__ __forceinline__ const AttendArgs& rows(const Args& a) { return a.rows; }
  static __device__ __forceinline__ void go(const Args& a, char* lds) {
    const WorkItem w = work_item(a.codes);
    if (w.any) attend_quant_body<DT, CODE, DP, RT>(a.codes, w, lds);
  }
};

template <int DT, int CODE, int DP, int RT>
hipError_t launch_quant_as(const QuantBoth& a, int64_t groups, hipStream_t s) {
  constexpr int of_codes = QuantShape<DP, RT>::MAIN, of_rows = AttendShape<DT, DP, RT, 4>::MAIN, lds = of_codes > of_rows ? of_codes : of_rows;
  auto kernel = attend_kernel<DT, DP, RT, 4, false, BesideCodes<DT, CODE, DP, RT>>;
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  kernel<<<dim3((uint32_t)groups), dim3(256), lds, s>>>(a);
  return hipGetLastError();
}
template <int DT, int CODE>
hipError_t launch_quant_code(const QuantBoth& a, int64_t groups, int row_tile, hipStream_t s) {
  const bool one = row_tile == 16;
  if (a.codes.D <= 64) return one ? launch_quant_as<DT, CODE, 64, 1>(a, groups, s) : launch_quant_as<DT, CODE, 64, 2>(a, groups, s);
  if (a.codes.D <= 128) return one ? launch_quant_as<DT, CODE, 128, 1>(a, groups, s) : launch_quant_as<DT, CODE, 128, 2>(a, groups, s);
  return launch_quant_as<DT, CODE, 256, 1>(a, groups, s);
}
template <int DT>
hipError_t launch_quant_of(const QuantBoth& a, int64_t groups, int code, int row_tile, hipStream_t s) {
  return code == LAGKV_CODE_INT8 ? launch_quant_code<DT, LAGKV_CODE_INT8>(a, groups, row_tile, s)
                                 : launch_quant_code<DT, LAGKV_CODE_E4M3>(a, groups, row_tile, s);
}

}  // namespace lagkv
