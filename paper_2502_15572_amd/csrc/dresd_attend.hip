// gfx950 attention of chunks of new tokens over a paged cache of keys and values
// (batch verification, DReSD Section 3.6: the drafts' forward beside the cached
// context).
//
//   out_t = sum_p e^(s_p - lse) v_p,  s_p = scale q_t . k_p,  lse = log sum_p e^(s_p)
//
// over the positions p that row t sees.  One pass over the keys with the running
// maximum and sum of the softmax.  One wave per row and head, a key per lane for
// the scores, four dims per lane for the output.
#include "dresd_device.h"
#include "dresd_verify.h"

namespace dresd {

namespace {

constexpr int kAttendThreads = 256;

template <int DT>
__device__ __forceinline__ float elem(const void *x, int64_t at) {
  if constexpr (DT == kF16) return (float)static_cast<const _Float16 *>(x)[at];
  else if constexpr (DT == kBF16)
    return __uint_as_float((uint32_t)static_cast<const uint16_t *>(x)[at] << 16);
  else return __builtin_amdgcn_cvt_pk_f32_fp8((int)static_cast<const uint8_t *>(x)[at], false)[0];
}

template <int QT, int CT>
__global__ void __launch_bounds__(kAttendThreads) dresd_attend_rows(AttendParams p) {
  __shared__ float qs[kAttendThreads / kWaveSize][kHeadDimMax];
  const int wid = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * (kAttendThreads / kWaveSize) + wid;
  const int64_t row = unit / p.q_heads;
  const int h = (int)(unit - row * p.q_heads);
  if (row >= p.T) return;
  int b, t, n;
  if (p.starts) {
    b = -1;
    for (int i = 0; i < p.B; ++i)
      if (row >= p.starts[i] && row < p.starts[i + 1]) b = i;
    if (b < 0) return;
    t = (int)row - p.starts[b];
    n = p.starts[b + 1] - p.starts[b];
  } else {
    n = p.n;
    b = (int)(row / n);
    t = (int)(row - (int64_t)b * n);
  }
  const int D = p.c.dim, hk = h / (p.q_heads / p.c.heads);
  for (int d = lane; d < D; d += kWaveSize)
    qs[wid][d] = elem<QT>(p.q, row * p.q_row + h * p.q_head + d);
  wave_sync_lds();
  const int len = p.lengths[b], before = len - n;
  const int64_t room = (int64_t)p.width << p.c.page_log;
  const int L = len < room ? len : (int)room;
  float m = -__builtin_huge_valf(), l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int base = 0; base < L; base += kWaveSize) {
    const int pos = base + lane;
    bool see = pos < L;
    if (see) {
      const int j = pos - before;
      if (p.mask) {
        if (j >= 0)
          see = j / 64 < p.words && ((p.mask[row * p.words + j / 64] >> (j & 63)) & 1);
      } else {
        see = j <= t;
      }
    }
    int64_t slot = 0;
    if (see) {
      const int page = p.table[(int64_t)b * p.width + (pos >> p.c.page_log)];
      see = page >= 0 && page < p.c.pages;
      slot = (((int64_t)page * p.c.heads + hk) << p.c.page_log) +
             (pos & ((1 << p.c.page_log) - 1));
    }
    float s = -__builtin_huge_valf(), vs = 1.f;
    if (see) {
      s = 0.f;
      for (int d = 0; d < D; ++d) s += qs[wid][d] * elem<CT>(p.c.k, slot * D + d);
      s *= p.scale;
      if constexpr (CT == kF8) {
        s = ldexpf(s, (int)p.c.k_exp[slot] - 127);
        vs = ldexpf(1.f, (int)p.c.v_exp[slot] - 127);
      }
    }
    float top = s;
    for (int o = 1; o < kWaveSize; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, kWaveSize));
    const float mn = fmaxf(m, top);
    if (mn == -__builtin_huge_valf()) continue;  // nothing seen so far
    const float w = see ? expf(s - mn) : 0.f, a = expf(m - mn);
    float sum = w;
    for (int o = 1; o < kWaveSize; o <<= 1) sum += __shfl_xor(sum, o, kWaveSize);
    l = l * a + sum;
    m = mn;
    for (int i = 0; i < 4; ++i) acc[i] *= a;
    for (int j = 0; j < kWaveSize; ++j) {
      if (!__shfl(see, j, kWaveSize)) continue;
      const float wj = __shfl(w * vs, j, kWaveSize);
      const int64_t sj = __shfl(slot, j, kWaveSize);
      for (int i = 0; i < 4; ++i)
        if (lane + i * kWaveSize < D) acc[i] += wj * elem<CT>(p.c.v, sj * D + lane + i * kWaveSize);
    }
  }
  const int64_t at = row * p.q_heads + h;
  for (int i = 0; i < 4; ++i) {
    const int d = lane + i * kWaveSize;
    if (d >= D) continue;
    const float o = l > 0.f || l != l ? acc[i] / l : 0.f;
    if constexpr (QT == kF16) static_cast<_Float16 *>(p.out)[at * D + d] = (_Float16)o;
    else static_cast<__bf16 *>(p.out)[at * D + d] = (__bf16)o;
  }
  if (lane == 0 && p.lse) p.lse[at] = l > 0.f || l != l ? m + logf(l) : -__builtin_huge_valf();
}

}  // namespace

int64_t attend_workspace(const AttendParams &, int) { return 0; }

hipError_t launch_attend(const AttendParams &p, int, hipStream_t st) {
  if (p.T == 0) return hipSuccess;
  AttendParams q = p;
  void *args[] = {&q};
  const void *k =
      p.c.dtype == kF8 ? (p.dtype == kF16 ? (const void *)dresd_attend_rows<kF16, kF8>
                                          : (const void *)dresd_attend_rows<kBF16, kF8>)
      : p.dtype == kF16 ? (const void *)dresd_attend_rows<kF16, kF16>
                        : (const void *)dresd_attend_rows<kBF16, kBF16>;
  const int64_t units = p.T * p.q_heads, per = kAttendThreads / kWaveSize;
  return hipLaunchKernel(k, dim3((unsigned)((units + per - 1) / per)), dim3(kAttendThreads), args,
                         0, st);
}

}  // namespace dresd
