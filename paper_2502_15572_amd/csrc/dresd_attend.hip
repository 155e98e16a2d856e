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
// matrix operand, so grouped heads read the cache once.  Few rows: the wave
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

size_t attend_wave_lds_64(bool f8, int ct);
size_t attend_wave_lds_128(bool f8, int ct);
size_t attend_wave_lds_256(bool f8, int ct);
size_t attend_wave_lds(bool f8, int dp, int ct) {
  return dp == 64    ? attend_wave_lds_64(f8, ct)
         : dp == 128 ? attend_wave_lds_128(f8, ct)
                     : attend_wave_lds_256(f8, ct);
}

namespace {

constexpr int kSplitsMax = 64;
constexpr int kJoinThreads = 256;
constexpr int64_t kGroupsMax = (1 << 24) - 8;  // workgroups of 256 threads: a launch has fewer than 2^32

// Joins the parts of every row and head: `GS` 32-lane groups of a workgroup a row, of
// which each takes every GS-th part, `NP` of them at most and all on their way at once, four dims
// a lane (the dims past 128 in a second turn), and whose sums meet in LDS.
template <int QT, int GS, int NP>
__global__ void __launch_bounds__(kJoinThreads) dresd_attend_join(AttendPlan pl) {
  constexpr int G = kJoinThreads / 32;
  __shared__ f4 part[G][32];
  const AttendParams &p = pl.p;
  const int g = threadIdx.x / 32, j = threadIdx.x % 32, gs = g % GS;
  const int64_t rows = p.T * p.q_heads, r = (int64_t)blockIdx.x * (G / GS) + g / GS;
  bool real = r < rows;
  if (real && p.ragged) {    // rows outside the chunks have no parts
    const int64_t t = r / p.q_heads;
    real = t >= p.starts[0] && t < p.starts[p.B];
  }
  const float2 *ml = reinterpret_cast<const float2 *>(pl.part_ml);
  float2 own[2];                                 // parts j and j + 32
  float top = -3e38f, l = 0.f;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    own[i] = real && j + 32 * i < pl.splits ? ml[(int64_t)(j + 32 * i) * rows + r]
                                            : float2{-3e38f, 0.f};
    top = fmaxf(top, own[i].x);
  }
  // the sums are on their way before the weights are known (a part without weight has none: what
  // is read in their place is not used)
  f4 y[NP];
  auto fetch = [&](int d) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int s = GS * i + gs;
      y[i] = f4{};
      if (real && s < pl.splits && d < p.c.dim)
        y[i] = *reinterpret_cast<const f4 *>(pl.part_o + ((int64_t)s * rows + r) * p.c.dim + d);
    }
  };
  fetch(4 * j);
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, 32));
  float a[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    a[i] = own[i].y != 0.f ? exp2_hw(own[i].x - top) : 0.f;
    l += own[i].y * a[i];
  }
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) l += __shfl_xor(l, o, 32);
  for (int d0 = 0; d0 < p.c.dim; d0 += 128) {
    const int d = d0 + 4 * j;
    if (d0 > 0) fetch(d);
    f4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int s = GS * i + gs;
      const float w = __shfl(GS * NP <= 32 || i < 32 / GS ? a[0] : a[1], s & 31, 32);
      if (w != 0.f)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] += y[i][e] * w;
    }
    if constexpr (GS > 1) {
      part[g][j] = x;
      __syncthreads();
    }
    if (real && gs == 0 && d < p.c.dim) {
#pragma unroll
      for (int i = 1; i < GS; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] += part[g + i][j][e];
      finish_row<QT>(p, r, d, x, top, l);
    }
    if constexpr (GS > 1) __syncthreads();
  }
}

template <int QT>
const void *join_kernel(int groups) {
  return groups == 1   ? (const void *)dresd_attend_join<QT, 1, 2>
         : groups == 2 ? (const void *)dresd_attend_join<QT, 2, 2>
         : groups == 4 ? (const void *)dresd_attend_join<QT, 4, 4>
                       : (const void *)dresd_attend_join<QT, 8, 8>;
}

AttendPlan plan_of(const AttendParams &p, int cus) {
  AttendPlan pl = {};
  pl.p = p;
  pl.group = p.q_heads / p.c.heads;
  // rows of the longest chunk (of ragged chunks: were they all alike)
  const int64_t tokens = p.ragged ? (p.T + (p.B > 0 ? p.B : 1) - 1) / (p.B > 0 ? p.B : 1) : p.n;
  const int64_t rows = tokens * pl.group;
  // Up to 32 rows the wave kernel; in 8 bits up to 64, in two blocks, since the tile kernel
  // converts what it reads before it shares it (8 sequences of 1,000 to 4,000 tokens, 32 heads; 64
  // rows in 8 bits 70 to 75 us against 85 to 90, with heads of 256 167 against 215; 91 rows 106
  // against 96; 64 rows in 16 bits 104 against 90).  The wave kernel copies 16 bytes at a time.
  const bool f8 = p.c.dtype == kF8;
  const bool wave = rows <= (f8 ? 64 : 32) && !(f8 && p.c.dim % 16);
  pl.ct = !wave ? 0 : rows <= 16 ? 1 : 2;
  pl.rows = pl.ct ? 16 * pl.ct : 128;
  pl.blocks = (int)(p.ragged ? p.T * pl.group / pl.rows + p.B
                             : (int64_t)p.B * ((rows + pl.rows - 1) / pl.rows));
  const int64_t units = (int64_t)pl.blocks * p.c.heads;
  // As many workgroups as the compute units hold at once (two each, heads past 128: one), none
  // without a round of tiles.  Rounded down, since a part of a second round costs what it has fewer
  // (464 units of up to 282 tokens on 512 places: two splits 20.9 us, one 15.1; drawn shapes 4 to 5%
  // on average).  Where one split leaves more than a quarter of the places empty, two, if the keys are
  // many (280 units of up to 12,000 tokens 190 us with one, 154 with two; 264 of 1,900 58
  // with one, 64 with two).  By the table's room: the lengths are on the device.
  const int64_t room = (int64_t)p.width << p.c.page_log;
  const int64_t slots = p.c.dim > 128 ? cus : 2 * (int64_t)cus;
  int64_t s = units > 0 ? slots / units : 1;
  if (s <= 1 && 4 * units < 3 * slots && room >= 4096) s = 2;
  // Few rows over few keys: reading them alone takes what a second launch takes (8 x 4 heads of 128:
  // 300 tokens 10.8 us with one split, 10.6 with three; 200 10.2 against 10.9, 450 12.4 against
  // 11.1), and the caller's thread is done after one.
  if (pl.ct == 1 && room <= 320) s = 1;
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
  if (pl.total > kGroupsMax) return -1;
  return part_floats(pl) * (p.c.dim + 2) * 4;
}

hipError_t launch_attend(const AttendParams &p, int cus, hipStream_t st) {
  if (p.T == 0) return hipSuccess;
  AttendPlan pl = plan_of(p, cus);
  pl.part_o = static_cast<float *>(p.work);
  pl.part_ml = pl.part_o + part_floats(pl) * p.c.dim;
  const bool f8 = p.c.dtype == kF8;
  const int dp = p.c.dim <= 64 ? 64 : p.c.dim <= 128 ? 128 : 256;
  const AttendKernel k = pl.ct ? attend_wave_kernel(p.dtype, f8, dp, pl.ct)
                               : attend_tile_kernel(p.dtype, f8, dp);
  const size_t lds = pl.ct ? attend_wave_lds(f8, dp, pl.ct) : attend_tile_lds(dp);
  void *args[] = {&pl};
  hipError_t e = hipLaunchKernel((const void *)k, dim3((unsigned)((pl.total + 7) / 8 * 8)),
                                 dim3(256), args, lds, st);
  if (e != hipSuccess || pl.splits == 1) return e;
  // few parts: more rows a workgroup (10 parts by four groups 39.4 us of a call, by eight 42.7; two by
  // one group 102.5, by two 105.5)
  const int groups = pl.splits <= 2 ? 1 : pl.splits <= 4 ? 2 : pl.splits <= 16 ? 4 : 8;
  const void *j = p.dtype == kF16 ? join_kernel<kF16>(groups) : join_kernel<kBF16>(groups);
  const int64_t rows = p.T * p.q_heads, per = kJoinThreads / 32 / groups;
  return hipLaunchKernel(j, dim3((unsigned)((rows + per - 1) / per)), dim3(kJoinThreads), args, 0,
                         st);
}

}  // namespace dresd
