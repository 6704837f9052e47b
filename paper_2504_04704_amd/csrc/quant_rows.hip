// Rows of a cache into 8-bit codes with a scale for each block of rows, and back (lagkv_quantize, lagkv_dequantize).
//
// With a = max |x| over a block, code = 127 x / a rounded (int8) or x / 2^e rounded to 4 mantissa bits (e4m3).  The block is
// read once and waits in registers for its maximum: a wavefront or a workgroup of four takes a block, eight channels of a row a
// lane at a time.  Bound by memory, at three bytes an element of 16 bits: 32 x 8 streams of 33536 rows with 128 channels, bf16 to int8,
// blocks of 64, 1057 us (6.2 TB/s; a large copy reaches 5.1).  The vector units are then busy too, with the exact quotients of int8, but e4m3, which has half as
// many instructions, takes no less.  4 x 8 streams back to bf16 138 to 142 us (6.0 to 5.8 TB/s), to fp32 314 (4.4).  A block of more than 16384 numbers is read
// twice: 256 streams x 16384 rows of 256 channels in blocks of 128 rows 1433 us (4.5 TB/s), of 64 1066 (6.0).
#include "code_ops.hpp"
#include "lagkv_internal.hpp"
#include "quant_internal.hpp"

namespace lagkv {

// A block of K or V: which, and its rows that there are.
struct BlockOf {
  int64_t b, h, row0;
  uint32_t block;
  bool values;
  int rows;
};
__device__ __forceinline__ BlockOf block_of(const CodeArgs& a, uint32_t unit) {
  const uint32_t of = a.by_count.of(unit), streams = (uint32_t)(a.B * a.H);
  BlockOf x;
  x.block = a.first + (unit - of * (uint32_t)a.count);
  x.values = of >= streams;
  const uint32_t stream = x.values ? of - streams : of, b = a.by_h.of(stream);
  x.b = b;
  x.h = stream - b * (uint32_t)a.H;
  x.row0 = (int64_t)x.block * a.block;
  int64_t len = a.lengths ? a.lengths[b] : a.T;
  len = len > a.T ? a.T : len;
  const int64_t rows = len - x.row0;
  x.rows = (int)(rows < 0 ? 0 : rows > a.block ? a.block : rows);
  return x;
}

// Eight channels of a row
template <int DT>
struct Eight {
  static constexpr int WORDS = DT == LAGKV_F32 ? 8 : 4;
  uint32_t w[WORDS];
  // (FAR: past the caches, of rows that these do not hold)
  template <bool FAR>
  __device__ __forceinline__ void load(const char* p) {
#pragma unroll
    for (int i = 0; i < WORDS; i += 4) {
      const u32v4 v = FAR ? __builtin_nontemporal_load((const u32v4_any*)(p + i * 4)) : *(const u32v4_any*)(p + i * 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[i + e] = v[e];
    }
  }
  __device__ __forceinline__ void store(char* p) const {
#pragma unroll
    for (int i = 0; i < WORDS; i += 4) *(u32v4_any*)(p + i * 4) = u32v4{w[i], w[i + 1], w[i + 2], w[i + 3]};
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (DT == LAGKV_F32) return __uint_as_float(w[i]);
    else return AElem<DT>::one((uint16_t)(w[i / 2] >> (16 * (i % 2))));
  }
  // The largest magnitude's bits, of a number of the type (fp32) or of each of a pair of them: those of positive numbers are in order, and
  // infinities and what is no number come last.
  __device__ __forceinline__ uint32_t most(uint32_t m) const {
    if constexpr (DT == LAGKV_F32) {
#pragma unroll
      for (int i = 0; i < WORDS; ++i) m = max(m, w[i] & 0x7fffffffu);
      return m;
    } else {
      typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
      u16x2 x = __builtin_bit_cast(u16x2, m);
#pragma unroll
      for (int i = 0; i < WORDS; ++i) x = __builtin_elementwise_max(x, __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu));
      return __builtin_bit_cast(uint32_t, x);
    }
  }
};
template <int DT>
__device__ __forceinline__ uint32_t one_of(uint32_t m) {
  if constexpr (DT == LAGKV_F32) return m;
  return max(m & 0xffffu, m >> 16);
}

// What a block's maximum makes of its rows.
template <int DT, int CODE>
struct Coder {
  float a, scale, by, inv;
  bool bad;
  __device__ __forceinline__ explicit Coder(uint32_t bits) {
    constexpr uint32_t EXP = DT == LAGKV_F32 ? 0x7f800000u : DT == LAGKV_BF16 ? 0x7f80u : 0x7c00u;
    bad = bits >= EXP;
    if constexpr (DT == LAGKV_F32) a = __uint_as_float(bits);
    else a = AElem<DT>::one((uint16_t)bits);
    if constexpr (CODE == LAGKV_CODE_INT8) {
      // (the quotient is worked out with a near 1: 127 x is then in range, and 1 / a)
      const float near = a >= 0x1p64f ? 0x1p-64f : a < 0x1p-64f ? 0x1p80f : 1.f;
      scale = a / 127.f;
      by = 127.f * near;
      a *= near;
      inv = a > 0.f ? 1.f / a : 0.f;
    } else {
      // a <= 448 * 2^e with 448 = 1.75 * 2^8
      const uint32_t f = __float_as_uint(a);
      int e = (int)(f >> 23) - 127 - 8 + ((f & 0x7fffffu) > 0x600000u ? 1 : 0);
      e = e < -126 ? -126 : e;
      scale = a > 0.f ? __uint_as_float((uint32_t)(e + 127) << 23) : 0.f;
      by = __uint_as_float((uint32_t)(127 - e) << 23);
      inv = 0.f;
    }
    if (bad) scale = __uint_as_float(0x7fc00000u);
  }
  // 127 x / a rounded to nearest, as the low byte of the result.  127 x is exact in 16-bit types, and so is the remainder: the
  // corrected quotient of a tie is that tie, and no other quotient comes as near to one as its error (two such numbers'
  // fraction is 2^-19 from any other).  In fp32 the quotients next to a tie are settled by 254 |x| against (2k + 1) a, exact in 64 bits.
  __device__ __forceinline__ uint32_t whole(float x) const {
    constexpr float SHIFT = 12582912.f;  // 1.5 * 2^23
    const float t = x * by, q0 = t * inv, q = __builtin_fmaf(__builtin_fmaf(-q0, a, t), inv, q0);
    float y = q + SHIFT;
    if constexpr (DT == LAGKV_F32) {
      const float off = q - (y - SHIFT);
      if (__any(fabsf(off) > 0.4999f)) {
        const float k = floorf(fabsf(q));
        const double s = 254.0 * fabs((double)x) - (2.0 * k + 1.0) * ((double)a * (127.0 / (double)by));
        const bool up = s > 0.0 || (s == 0.0 && ((int)k & 1));
        const float r = copysignf(k + (up ? 1.f : 0.f), q);
        if (fabsf(off) > 0.4999f) y = r + SHIFT;
      }
    }
    return __float_as_uint(y);
  }
  __device__ __forceinline__ u32v2 codes(const Eight<DT>& x) const {
    u32v2 w;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if constexpr (CODE == LAGKV_CODE_INT8) {
        uint32_t y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = whole(x.at(i * 4 + e));
        w[i] = __builtin_amdgcn_perm(y[1], y[0], 0x0c0c0400u) | __builtin_amdgcn_perm(y[3], y[2], 0x04000c0cu);
      } else {
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = x.at(i * 4 + e) * by;
        int v = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], v, true);
      }
      if (bad) w[i] = 0;
    }
    return w;
  }
};

__device__ __forceinline__ uint32_t wave_most(uint32_t m) {
#pragma unroll
  for (int far = 1; far < 64; far <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, far));
  return m;
}

// NV slices of eight channels a lane; AGAIN: of a block that has more, and is read a second time (from the L2 as a rule) for its codes.
template <int DT, int CODE, int WAVES, int NV, bool AGAIN, bool FAR>
__global__ __launch_bounds__(256) void quantize_kernel(const CodeArgs a) {
  constexpr int ES = AElem<DT>::SIZE, THREADS = WAVES * 64, PER_GROUP = 4 / WAVES;
  __shared__ uint32_t sh_most[2][4];
  fetch_arguments<CodeArgs>();
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), t = WAVES == 1 ? (int)threadIdx.x & 63 : (int)threadIdx.x;
  const uint32_t units = (uint32_t)a.units, step = gridDim.x * PER_GROUP;
  int turn = 0;
  for (uint32_t unit = blockIdx.x * PER_GROUP + (WAVES == 1 ? wave : 0); unit < units; unit += step) {
    const BlockOf x = block_of(a, unit);
    if (x.rows == 0) continue;  // (of all of the workgroup, or this wavefront)
    const char* from = (x.values ? a.V : a.K) + x.b * a.rsb + x.h * a.rsh + x.row0 * a.rst;
    char* to = (char*)(x.values ? a.Vq : a.Kq) + x.b * a.csb + x.h * a.csh + x.row0 * a.cst;
    const int n = x.rows * a.slices;
    Eight<DT> v[NV];
    // (a lane with none takes the first slice: the maximum does not change)
    auto place = [&](int i, int64_t& row, int& ch) {
      const int at = i < n ? i : 0, r = (int)a.by_slices.of(at);
      row = r;
      ch = slice_at(at - r * a.slices, a.D, 8);
    };
    auto load = [&](int i0) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        int64_t row;
        int ch;
        place(i0 + k * THREADS + t, row, ch);
        v[k].template load<FAR>(from + row * a.rst + ch * ES);
      }
    };
    uint32_t m = 0;
    for (int i0 = 0; i0 < (AGAIN ? n : 1); i0 += NV * THREADS) {
      load(i0);
#pragma unroll
      for (int k = 0; k < NV; ++k) m = v[k].most(m);
    }
    m = wave_most(one_of<DT>(m));
    if constexpr (WAVES > 1) {
      // (two sets in turn: the next block's maxima are not written over ones that are still read)
      if ((threadIdx.x & 63) == 0) sh_most[turn][wave] = m;
      __syncthreads();
      m = max(max(sh_most[turn][0], sh_most[turn][1]), max(sh_most[turn][2], sh_most[turn][3]));
      turn ^= 1;
    }
    const Coder<DT, CODE> coder(m);
    if (t == 0) ((x.values ? a.vs : a.ks) + x.b * a.ssb + x.h * a.ssh)[x.block] = coder.scale;
    for (int i0 = 0; i0 < (AGAIN ? n : 1); i0 += NV * THREADS) {
      if (AGAIN) load(i0);
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int i = i0 + k * THREADS + t;
        const u32v2 w = coder.codes(v[k]);
        int64_t row;
        int ch;
        place(i, row, ch);
        if (i < n) __builtin_nontemporal_store(w, (u32v2_any*)(to + row * a.cst + ch));
      }
    }
  }
}

// A lane's slices of a block's rows, THREADS apart: where the next one is by additions.  (With a quotient for each, as in quantize_kernel, 141 us
// in place of 138 on the way back of 4 x 8 streams x 33536 rows; that kernel, whose slices wait in registers, gains nothing: 1161 and 1172.)
template <int THREADS>
struct Walk {
  const CodeArgs& a;
  int64_t stride, skip;  // of a row, of the rows that THREADS slices are
  char* p;               // the row's
  int i, slice;
  __device__ __forceinline__ Walk(const CodeArgs& a, char* base, int64_t stride, int t)
      : a(a), stride(stride), skip(stride * a.walk_rows), i(t) {
    const int row = (int)a.by_slices.of(t);
    slice = t - row * a.slices;
    p = base + row * stride;
  }
  __device__ __forceinline__ int channel() const { return slice_at(slice, a.D, 8); }
  __device__ __forceinline__ void next() {
    i += THREADS;
    p += skip;
    slice += a.walk_slices;
    if (slice >= a.slices) {
      slice -= a.slices;
      p += stride;
    }
  }
};

template <int DT, int CODE, int WAVES, int NV>
__global__ __launch_bounds__(256) void dequantize_kernel(const CodeArgs a) {
  constexpr int ES = AElem<DT>::SIZE, THREADS = WAVES * 64, PER_GROUP = 4 / WAVES;
  fetch_arguments<CodeArgs>();
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), t = WAVES == 1 ? (int)threadIdx.x & 63 : (int)threadIdx.x;
  const uint32_t units = (uint32_t)a.units, step = gridDim.x * PER_GROUP;
  for (uint32_t unit = blockIdx.x * PER_GROUP + (WAVES == 1 ? wave : 0); unit < units; unit += step) {
    const BlockOf x = block_of(a, unit);
    const int skip = a.start > x.row0 ? (int)(a.start - x.row0) : 0, n = (x.rows - skip) * a.slices;
    if (n <= 0) continue;
    const int64_t row0 = x.row0 + skip;
    char* from = (char*)(x.values ? a.Vq : a.Kq) + x.b * a.csb + x.h * a.csh + row0 * a.cst;
    char* to = (char*)(x.values ? a.V : a.K) + x.b * a.rsb + x.h * a.rsh + row0 * a.rst;
    const float scale = ((x.values ? a.vs : a.ks) + x.b * a.ssb + x.h * a.ssh)[x.block];
    Walk<THREADS> in(a, from, a.cst, t), at(a, to, a.rst, t);
    do {
      u32v2 w[NV];
#pragma unroll
      for (int k = 0; k < NV; ++k, in.next()) w[k] = *(const u32v2_any*)(in.i < n ? in.p + in.channel() : from);
#pragma unroll
      for (int k = 0; k < NV; ++k, at.next()) {
        float y[8];
        Code<CODE>::to_float(w[k].x, y);
        Code<CODE>::to_float(w[k].y, y + 4);
        Eight<DT> v;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          if constexpr (DT == LAGKV_F32) {
            v.w[e] = __float_as_uint(y[e] * scale);
            v.w[e + 1] = __float_as_uint(y[e + 1] * scale);
          } else {
            v.w[e / 2] = AElem<DT>::pack(y[e] * scale, y[e + 1] * scale);
          }
        }
        if (at.i < n) v.store(at.p + at.channel() * ES);
      }
    } while (at.i - t < n);
  }
}

constexpr int64_t kMostGroups = 1 << 22;  // (a larger call's go over several blocks)

template <int PER_GROUP>
dim3 groups_of(const CodeArgs& a) {
  const int64_t g = (a.units + PER_GROUP - 1) / PER_GROUP;
  return dim3((uint32_t)(g < kMostGroups ? g : kMostGroups));
}

// (the steps of a Walk)
inline CodeArgs walked(CodeArgs a, int threads) {
  a.walk_rows = threads / a.slices;
  a.walk_slices = threads % a.slices;
  return a;
}

template <int DT, int CODE, bool FAR>
void launch_quantize_as(const CodeArgs& a, hipStream_t s) {
  const int n = a.block * a.slices;
  if (n <= 64 * 8) quantize_kernel<DT, CODE, 1, 8, false, FAR><<<groups_of<4>(a), dim3(256), 0, s>>>(a);
  else if (n <= 256 * 4) quantize_kernel<DT, CODE, 4, 4, false, FAR><<<groups_of<1>(a), dim3(256), 0, s>>>(a);
  else if (n <= 256 * 8) quantize_kernel<DT, CODE, 4, 8, false, FAR><<<groups_of<1>(a), dim3(256), 0, s>>>(a);
  else quantize_kernel<DT, CODE, 4, 4, true, false><<<groups_of<1>(a), dim3(256), 0, s>>>(a);
}
// Codes are stored past the caches, and rows that fill these (256 MiB) are read past them: 8 x 32 streams x 33536 rows, 128 channels of bf16
// to int8, 1057 us in place of 1161 (the stores alone: 1131).  At 256 MiB, 64 streams x 8192 rows of 128 channels in bf16 take 65 us in place of 71 (e4m3 68
// and 72), 32 of them in fp32 59 in place of 61; rows of 65 MB in
// fp32, which the caches may still hold, would take 30 us in place of 24, and ones that are read again 117 in place of 107.  Rows on
// their way back are stored as usual: past the caches the call itself takes 114 us in place of 135 at 512 MB, but with the one that
// reads them 318 in place of 311.
template <int DT, int CODE>
hipError_t launch_quantize_of(const CodeArgs& a, hipStream_t s) {
  const bool far = (double)a.units * a.block * a.D * AElem<DT>::SIZE >= 268435456.0;
  if (far) launch_quantize_as<DT, CODE, true>(a, s);
  else launch_quantize_as<DT, CODE, false>(a, s);
  return hipGetLastError();
}
template <int DT, int CODE>
hipError_t launch_dequantize_of(const CodeArgs& args, hipStream_t s) {
  const CodeArgs a = walked(args, args.block * args.slices <= 64 * 8 ? 64 : 256);
  if (a.block * a.slices <= 64 * 8) dequantize_kernel<DT, CODE, 1, 4><<<groups_of<4>(a), dim3(256), 0, s>>>(a);
  else dequantize_kernel<DT, CODE, 4, 4><<<groups_of<1>(a), dim3(256), 0, s>>>(a);
  return hipGetLastError();
}
template <int DT>
hipError_t launch_codes_of(const CodeArgs& a, int code, bool back, hipStream_t s) {
  if (code == LAGKV_CODE_INT8) return back ? launch_dequantize_of<DT, LAGKV_CODE_INT8>(a, s) : launch_quantize_of<DT, LAGKV_CODE_INT8>(a, s);
  return back ? launch_dequantize_of<DT, LAGKV_CODE_E4M3>(a, s) : launch_quantize_of<DT, LAGKV_CODE_E4M3>(a, s);
}
static hipError_t launch_codes(const CodeArgs& a, int dtype, int code, bool back, hipStream_t s) {
  return dtype == LAGKV_F32 ? launch_codes_of<LAGKV_F32>(a, code, back, s)
         : dtype == LAGKV_BF16 ? launch_codes_of<LAGKV_BF16>(a, code, back, s) : launch_codes_of<LAGKV_F16>(a, code, back, s);
}
hipError_t launch_quantize(const CodeArgs& a, int dtype, int code, hipStream_t s) { return launch_codes(a, dtype, code, false, s); }
hipError_t launch_dequantize(const CodeArgs& a, int dtype, int code, hipStream_t s) { return launch_codes(a, dtype, code, true, s); }

}  // namespace lagkv
