// Joins the pieces that a unit's cache rows were cut into (see attend_pass.hpp for how two states join): a workgroup
// takes one query row, its four wavefronts every fourth piece, its lanes four channels each.  Bound by the launch
// and the latency of two dependent reads: there are at most some hundred pieces of a row.
#include "attend_pass.hpp"

namespace lagkv {

template <int DT>
__global__ __launch_bounds__(256) void attend_join_kernel(const AttendArgs a) {
  using E = AElem<DT>;
  __shared__ float sh_o[4][kMaxHead];
  __shared__ float sh_l[4];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t unit = blockIdx.x / a.rows;
  const int r = (int)(blockIdx.x % a.rows);
  const bool pick = a.blocks != nullptr;
  const int64_t stream = pick ? unit / a.N : unit;
  const int n = pick ? (int)(unit % a.N) : r / a.G, g = pick ? r : r % a.G;
  const int64_t b = stream / a.H, h = stream % a.H, head = h * a.G + g;
  const int64_t first = unit * a.splits * a.rows + r;  // of the pieces' rows, `rows` apart
  float top = -INFINITY;
  for (int s = lane; s < a.splits; s += kWave) top = fmaxf(top, a.part_ml[(first + (int64_t)s * a.rows) * 2]);
  top = wave_max(top);
  float sum = 0.f;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  for (int s = wave; s < a.splits; s += 4) {
    const int64_t at = first + (int64_t)s * a.rows;
    const float mx = a.part_ml[at * 2];
    if (mx == -INFINITY) continue;  // (nothing seen: its outputs were written as zeros)
    const float f = __builtin_amdgcn_exp2f((mx - top) * E::UNIT);
    sum += f * a.part_ml[at * 2 + 1];
    if (lane * 4 < a.D) v += f * *(const f32x4*)(a.part_o + at * a.part_ld + lane * 4);
  }
  if (lane * 4 < a.D) *(f32x4*)(&sh_o[wave][lane * 4]) = v;
  if (lane == 0) sh_l[wave] = sum;
  __syncthreads();
  sum = sh_l[0] + sh_l[1] + sh_l[2] + sh_l[3];
  bool blind = sum == 0.f;
  if (a.parents) {
    const int up = a.parents[b * a.psb + n];
    blind = blind || up < -1 || up >= n;
  }
  const float inv = blind ? 0.f : 1.f / sum;
  char* op = a.out + b * a.osb + head * a.osh + (int64_t)n * a.osn;
  for (int c = threadIdx.x; c < a.D; c += 256) {
    const float y = blind ? 0.f : (sh_o[0][c] + sh_o[1][c] + sh_o[2][c] + sh_o[3][c]) * inv;
    if constexpr (DT == LAGKV_F32) *(float*)(op + c * 4) = y;
    else *(uint16_t*)(op + c * 2) = (uint16_t)E::pack(y, 0.f);
  }
  if (threadIdx.x == 0 && a.lse)
    a.lse[(b * a.H * a.G + head) * a.N + n] = blind ? -INFINITY : lse_of<DT>(top, sum);
}

hipError_t launch_attend_join(const AttendArgs& a, int dtype, hipStream_t s) {
  const dim3 grid((uint32_t)(a.units * a.rows)), group(256);
  if (dtype == LAGKV_F32) attend_join_kernel<LAGKV_F32><<<grid, group, 0, s>>>(a);
  else if (dtype == LAGKV_BF16) attend_join_kernel<LAGKV_BF16><<<grid, group, 0, s>>>(a);
  else attend_join_kernel<LAGKV_F16><<<grid, group, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace lagkv
