// Joins the pieces that a unit's cache rows were cut into (see attend_pass.hpp for how two states join): a workgroup
// or a wavefront takes one query row, a lane four channels of every so many pieces.  Few rows: bound by the launch
// and the latency of two dependent reads (2.5 to 3 us, at most 256 pieces of a row).  Many: by memory (8192 rows in 8 pieces,
// 33 MB, 8.6 us).  The workgroups of the first kernel cannot do it, the last one to end say: a count of those that have ended
// would have to be cleared before, which is a launch as well.
#include "attend_pass.hpp"

namespace lagkv {

template <int DT, int WAVES>
__global__ __launch_bounds__(256) void attend_join_kernel(const AttendArgs a) {
  using E = AElem<DT>;
  __shared__ float sh_o[4][kMaxHead];
  __shared__ float sh_l[4];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  fetch_arguments<AttendArgs>();
  const uint32_t id = WAVES == 1 ? blockIdx.x * 4 + wave : blockIdx.x, at_unit = a.by_rows.of(id);
  const int64_t unit = at_unit;
  if (unit >= a.units) return;
  const int r = (int)(id - at_unit * a.rows);
  const bool pick = a.blocks != nullptr;
  const uint32_t stream = pick ? a.by_n.of(at_unit) : at_unit, bu = a.by_h.of(stream);
  const int n = pick ? (int)(at_unit - stream * a.N) : (int)a.by_g.of(r), g = pick ? r : r - n * a.G;
  const int64_t b = bu, h = stream - bu * a.H, head = h * a.G + g;
  const int64_t first = unit * a.splits * a.rows + r;  // of the pieces' rows, `rows` apart
  // lanes: four channels each, of one piece or of two or four
  const int per = a.D <= 64 ? 16 : a.D <= 128 ? 32 : 64, quad = lane % per, sub = lane / per, pieces = 64 / per;
  const bool have = quad * 4 < a.D;
  // the first of a lane's pieces are asked for before the largest maximum is known
  constexpr int AHEAD = 4;
  const int turn = (WAVES == 1 ? 0 : wave * pieces) + sub, stride = WAVES * pieces;
  f32x4 x[AHEAD];
  float mx[AHEAD], lx[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) {
    const int s = turn + i * stride;
    const int64_t at = first + (int64_t)(s < a.splits ? s : 0) * a.rows;
    x[i] = *(const f32x4*)(a.part_o + at * a.part_ld + (have ? quad * 4 : 0));
    mx[i] = a.part_ml[at * 2];
    lx[i] = s < a.splits ? a.part_ml[at * 2 + 1] : 0.f;
  }
  float top = -INFINITY;
  for (int s = lane; s < a.splits; s += kWave) top = fmaxf(top, a.part_ml[(first + (int64_t)s * a.rows) * 2]);
  top = wave_max(top);
  float sum = 0.f;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  auto add = [&](f32x4 x, float mx, float lx) {
    // (a piece that saw nothing has zeros)
    const float f = lx == 0.f ? 0.f : __builtin_amdgcn_exp2f((mx - top) * E::UNIT);
    sum += f * lx;
    v += lx == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : f * x;
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) add(x[i], mx[i], lx[i]);
#pragma unroll 4
  for (int s = turn + AHEAD * stride; s < a.splits; s += stride) {
    const int64_t at = first + (int64_t)s * a.rows;
    add(*(const f32x4*)(a.part_o + at * a.part_ld + (have ? quad * 4 : 0)), a.part_ml[at * 2], a.part_ml[at * 2 + 1]);
  }
  for (int far = per; far < 64; far <<= 1) {
    sum += __shfl_xor(sum, far);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += __shfl_xor(v[e], far);
  }
  if constexpr (WAVES > 1) {
    if (sub == 0) {
      if (have) *(f32x4*)(&sh_o[wave][quad * 4]) = v;
      if (lane == 0) sh_l[wave] = sum;
    }
    __syncthreads();
    if (wave > 0) return;
    sum = (sh_l[0] + sh_l[1]) + (sh_l[2] + sh_l[3]);
    if (have) v = (*(const f32x4*)&sh_o[0][quad * 4] + *(const f32x4*)&sh_o[1][quad * 4]) +
                  (*(const f32x4*)&sh_o[2][quad * 4] + *(const f32x4*)&sh_o[3][quad * 4]);
  }
  bool blind = sum == 0.f;
  if (a.parents) {
    const int up = a.parents[b * a.psb + n];
    blind = blind || up < -1 || up >= n;
  }
  const float inv = blind ? 0.f : 1.f / sum;
  if (sub == 0 && have) {
    char* op = a.out + b * a.osb + head * a.osh + (int64_t)n * a.osn;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (quad * 4 + e < a.D) {
        const float y = blind ? 0.f : v[e] * inv;
        if constexpr (DT == LAGKV_F32) *(float*)(op + (quad * 4 + e) * 4) = y;
        else *(uint16_t*)(op + (quad * 4 + e) * 2) = (uint16_t)E::pack(y, 0.f);
      }
  }
  if (lane == 0 && a.lse) a.lse[(b * a.H * a.G + head) * a.N + n] = blind ? -INFINITY : lse_of<DT>(top, sum);
}

// A wavefront a row where there are rows for all compute units, else a workgroup.
template <int DT>
static hipError_t launch_join_of(const AttendArgs& a, hipStream_t s) {
  const int64_t rows = a.units * a.rows;
  if (rows >= kJoinByWave) attend_join_kernel<DT, 1><<<dim3((uint32_t)((rows + 3) / 4)), dim3(256), 0, s>>>(a);
  else attend_join_kernel<DT, 4><<<dim3((uint32_t)rows), dim3(256), 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_attend_join(const AttendArgs& a, int dtype, hipStream_t s) {
  return dtype == LAGKV_F32 ? launch_join_of<LAGKV_F32>(a, s) : dtype == LAGKV_BF16 ? launch_join_of<LAGKV_BF16>(a, s) : launch_join_of<LAGKV_F16>(a, s);
}

}  // namespace lagkv
