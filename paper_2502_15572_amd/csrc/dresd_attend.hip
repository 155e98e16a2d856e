// gfx950 attention of chunks of new tokens over a paged cache of keys and values
// (batch verification, DReSD Section 3.6: the drafts' forward beside the cached
// context).
//
//   out_t = sum_p e^(s_p - lse) v_p,  s_p = scale q_t . k_p,  lse = log sum_p e^(s_p)
//
// over the positions p that row t sees, in one pass over the keys with the running
// maximum and sum of the softmax (in powers of two: s_p log2 e).  Here: how a call is
// cut into workgroups, and the kernel that joins the parts of rows whose keys
// were split.
//
// The query rows that share a cache head (tokens times heads of the group) are one
// matrix operand, so grouped heads read the cache once.  Up to 64 rows: the wave
// kernel (dresd_attend_wave.hip), whose waves stream the keys each for itself;
// more: the tile kernel (dresd_attend_tile.hip), whose waves share them.
#include "dresd_attend.h"

namespace dresd {

AttendKernel attend_wave_kernel_64(int qt, bool f8, int ct);
AttendKernel attend_wave_kernel_128(int qt, bool f8, int ct);
AttendKernel attend_wave_kernel_256(int qt, bool f8, int ct);
AttendKernel attend_wave_kernel(int qt, bool f8, int dp, int ct) {
  return dp == 64    ? attend_wave_kernel_64(qt, f8, ct)
         : dp == 128 ? attend_wave_kernel_128(qt, f8, ct)
                     : attend_wave_kernel_256(qt, f8, ct);
}

namespace {

constexpr int kSplitsMax = 64;
constexpr int kJoinThreads = 256;

// Joins the parts of every row: one wave per row and head, four dims a lane.
template <int QT>
__global__ void __launch_bounds__(kJoinThreads) dresd_attend_join(AttendPlan pl) {
  const AttendParams &p = pl.p;
  const int lane = threadIdx.x & 63;
  const int64_t rows = p.T * p.q_heads;
  const int64_t r = (int64_t)blockIdx.x * (kJoinThreads / kWaveSize) + threadIdx.x / kWaveSize;
  if (r >= rows) return;
  if (p.ragged) {            // rows outside the chunks have no parts
    const int64_t t = r / p.q_heads;
    if (t < p.starts[0] || t >= p.starts[p.B]) return;
  }
  const float2 *ml = reinterpret_cast<const float2 *>(pl.part_ml);
  float2 own = {-3e38f, 0.f};                    // lane s: part s
  if (lane < pl.splits) own = ml[(int64_t)lane * rows + r];
  float top = own.x;
#pragma unroll
  for (int o = 1; o < kWaveSize; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, kWaveSize));
  const float a = own.y != 0.f ? exp2_hw(own.x - top) : 0.f;
  float l = own.y * a;
#pragma unroll
  for (int o = 1; o < kWaveSize; o <<= 1) l += __shfl_xor(l, o, kWaveSize);
  const int d = lane * 4;
  f4 x = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < pl.splits; ++s) {
    const float w = __shfl(a, s, kWaveSize);
    if (w == 0.f || d >= p.c.dim) continue;      // (w: the wave's; NaN parts have weight)
    const f4 y = *reinterpret_cast<const f4 *>(pl.part_o + ((int64_t)s * rows + r) * p.c.dim + d);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] += y[i] * w;
  }
  if (d < p.c.dim) finish_row<QT>(p, r, d, x, top, l);
}

AttendPlan plan_of(const AttendParams &p, int cus) {
  AttendPlan pl = {};
  pl.p = p;
  pl.group = p.q_heads / p.c.heads;
  // rows of the longest chunk (of ragged chunks: were they all alike)
  const int64_t tokens = p.ragged ? (p.T + (p.B > 0 ? p.B : 1) - 1) / (p.B > 0 ? p.B : 1) : p.n;
  const int64_t rows = tokens * pl.group;
  const bool wide = p.c.dim > 128;
  if (rows <= 16) pl.ct = 1;
  else if (rows <= 32 || wide) pl.ct = 2;
  else pl.ct = 4;
  pl.rows = 16 * pl.ct;
  pl.blocks = (int)(p.ragged ? p.T * pl.group / pl.rows + p.B
                             : (int64_t)p.B * ((rows + pl.rows - 1) / pl.rows));
  const int64_t units = (int64_t)pl.blocks * p.c.heads;
  // Enough workgroups for every compute unit to hold several, but none without a
  // round of tiles.
  const int64_t room = (int64_t)p.width << p.c.page_log;
  int64_t s = units > 0 ? (4 * (int64_t)cus + units - 1) / units : 1;
  const int64_t most = (room + 127) / 128;
  s = s < most ? s : most;
  pl.splits = (int)(s < 1 ? 1 : s < kSplitsMax ? s : kSplitsMax);
  pl.total = units * pl.splits;
  return pl;
}

int64_t part_floats(const AttendPlan &pl) {
  return pl.splits > 1 ? (int64_t)pl.splits * pl.p.T * pl.p.q_heads : 0;
}

}  // namespace

int64_t attend_workspace(const AttendParams &p, int cus) {
  const AttendPlan pl = plan_of(p, cus);
  return part_floats(pl) * (p.c.dim + 2) * 4;
}

hipError_t launch_attend(const AttendParams &p, int cus, hipStream_t st) {
  if (p.T == 0) return hipSuccess;
  AttendPlan pl = plan_of(p, cus);
  pl.part_o = static_cast<float *>(p.work);
  pl.part_ml = pl.part_o + part_floats(pl) * p.c.dim;
  const bool f8 = p.c.dtype == kF8;
  const int dp = p.c.dim <= 64 ? 64 : p.c.dim <= 128 ? 128 : 256;
  const AttendKernel k = attend_wave_kernel(p.dtype, f8, dp, pl.ct);
  const size_t lds = attend_wave_lds(f8, dp, pl.ct);
  if (!k) return hipErrorInvalidConfiguration;
  void *args[] = {&pl};
  hipError_t e = hipLaunchKernel((const void *)k, dim3((unsigned)((pl.total + 7) / 8 * 8)),
                                 dim3(256), args, lds, st);
  if (e != hipSuccess || pl.splits == 1) return e;
  const int64_t rows = p.T * p.q_heads, per = kJoinThreads / kWaveSize;
  const void *j = p.dtype == kF16 ? (const void *)dresd_attend_join<kF16>
                                  : (const void *)dresd_attend_join<kBF16>;
  return hipLaunchKernel(j, dim3((unsigned)((rows + per - 1) / per)), dim3(kJoinThreads), args, 0,
                         st);
}

}  // namespace dresd
