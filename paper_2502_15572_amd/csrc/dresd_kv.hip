// gfx950 writes into and reads from a paged cache of keys and values
// ([pages, heads, page_size, dim]), 16-bit or 8-bit (e4m3 with one power of two
// a row, a row being one token of one head).
//
// Quantisation of a row x: amax = m 2^E with 1 <= m < 2 has its exponent
//   e = E - 8 + (m > 1.75)   (amax 2^-e in (224, 448]; 448 = 1.75 2^8 is the
//                             largest e4m3 value), at least -126,
// and stores e4m3(x 2^-e), rounded to nearest even, and e + 127.  e4m3 is a
// floating type: its relative step is the same at every power of two, so a power
// of two costs no precision against amax / 448 and scales without rounding.
// A row read back is exact in fp32, and from e = -124 on in bf16 (its smallest code times 2^e is
// 2^(e - 9), bf16's smallest number 2^-133); writing it again stores the same values.
//
// What bounds both is memory: every element is read once and written once.  A
// lane carries 8 elements (16 bytes of a 16-bit row); the 8, 16 or 32 lanes of a row
// find its largest magnitude by exchanges among them.  A write takes the key and
// the value row of a token and head together: one look at the slot, two loads on their way
// (16,384 tokens of 32 heads of 128, bf16 to 8 bits: 88 us a call, 4.6 TB/s of the 4.8 that a large
// copy reaches; a row at a time 115).
#include "dresd_device.h"
#include "dresd_verify.h"

namespace dresd {

namespace {

constexpr int kKvThreads = 256;

typedef float f8v __attribute__((ext_vector_type(8)));
typedef uint16_t w8 __attribute__((ext_vector_type(8)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));

// Eight elements as fp32.
template <int DT>
__device__ __forceinline__ f8v load8(const void *base, int64_t at) {
  f8v x;
  if constexpr (DT == kF32) {
    const f4 *p = reinterpret_cast<const f4 *>(static_cast<const float *>(base) + at);
    const f4 a = p[0], b = p[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = a[i];
      x[4 + i] = b[i];
    }
  } else if constexpr (DT == kF16) {
    const h8 a = *reinterpret_cast<const h8 *>(static_cast<const _Float16 *>(base) + at);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)a[i];
  } else if constexpr (DT == kBF16) {
    const w8 a = *reinterpret_cast<const w8 *>(static_cast<const uint16_t *>(base) + at);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float((uint32_t)a[i] << 16);
  } else {
    const u2 a = *reinterpret_cast<const u2 *>(static_cast<const uint8_t *>(base) + at);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)a[i], false);
      const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)a[i], true);
      x[4 * i] = lo[0];
      x[4 * i + 1] = lo[1];
      x[4 * i + 2] = hi[0];
      x[4 * i + 3] = hi[1];
    }
  }
  return x;
}

// Eight fp32 elements, rounded to nearest even.
template <int DT>
__device__ __forceinline__ void store8(void *base, int64_t at, f8v x) {
  if constexpr (DT == kF32) {
    f4 *p = reinterpret_cast<f4 *>(static_cast<float *>(base) + at);
    p[0] = f4{x[0], x[1], x[2], x[3]};
    p[1] = f4{x[4], x[5], x[6], x[7]};
  } else if constexpr (DT == kF16) {
    h8 a;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = (_Float16)x[i];
    *reinterpret_cast<h8 *>(static_cast<_Float16 *>(base) + at) = a;
  } else if constexpr (DT == kBF16) {
    b8 a;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = (__bf16)x[i];
    *reinterpret_cast<b8 *>(static_cast<__bf16 *>(base) + at) = a;
  } else {
    u2 a;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      int w = 0;
      w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i], x[4 * i + 1], w, false);
      w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2], x[4 * i + 3], w, true);
      a[i] = (uint32_t)w;
    }
    *reinterpret_cast<u2 *>(static_cast<uint8_t *>(base) + at) = a;
  }
}

// Exponent of a row whose largest finite magnitude is amax.
__device__ __forceinline__ int row_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  if (u == 0) return -9;
  const int E = (int)(u >> 23) - 127;  // below the normal numbers: -127
  const int e = E - 8 + (int)((u & 0x7fffffu) > 0x600000u);
  return e < -126 ? -126 : e;
}

// Row pair i of n heads: the key and the value row of one token and head, heads innermost.
struct Row {
  bool inside;
  uint32_t head, token;
  int64_t exp;               // exponent in the cache (its first element: times dim)
};
__device__ __forceinline__ Row row_of(const KvParams &p, uint32_t i) {
  Row w;
  w.token = i / (uint32_t)p.c.heads;
  w.head = i - w.token * (uint32_t)p.c.heads;
  const int64_t slot = p.slots[w.token];
  const int64_t page = slot >> p.c.page_log;
  w.inside = slot >= 0 && page < p.c.pages;
  w.exp = ((page * p.c.heads + w.head) << p.c.page_log) + (slot & ((1ll << p.c.page_log) - 1));
  return w;
}

// LG: lanes of a row (a power of two, 8 LG >= dim).
template <int IN, int CACHE, int LG>
__global__ void __launch_bounds__(kKvThreads) dresd_kv_put(KvParams p) {
  const uint32_t i = blockIdx.x * (uint32_t)(kKvThreads / LG) + threadIdx.x / LG;
  const int j = (threadIdx.x % LG) * 8;
  if (i >= (uint32_t)(p.n * p.c.heads)) return;
  const Row w = row_of(p, i);
  if (!w.inside) return;
  const bool mine = j < p.c.dim;
  f8v x[2] = {};
  if (mine) {
    x[0] = load8<IN>(p.k_in, w.token * p.k_row + w.head * p.k_head + j);
    x[1] = load8<IN>(p.v_in, w.token * p.v_row + w.head * p.v_head + j);
  }
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    if constexpr (CACHE == kF8) {
      float amax = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float a = fabsf(x[v][k]);
        // an infinite element has no magnitude the row could be scaled to: NaN
        if (!(a < __builtin_huge_valf())) x[v][k] = __uint_as_float(0x7fc00000u);
        else amax = fmaxf(amax, a);
      }
#pragma unroll
      for (int o = 1; o < LG; o <<= 1) amax = fmaxf(amax, __shfl_xor(amax, o, kWaveSize));
      const int e = row_exponent(amax);
      const float s = __uint_as_float((uint32_t)(127 - e) << 23);  // 2^-e, -e in [-120, 126]
      // at the top of fp32 (e = 120) the codes past 240 would stand for 2^128
      const float most = e == 120 ? 240.f : 448.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float y = x[v][k];
        x[v][k] = y != y ? y : fminf(fmaxf(y * s, -most), most);
      }
      if (j == 0) (v ? p.c.v_exp : p.c.k_exp)[w.exp] = (uint8_t)(e + 127);
    }
    if (mine) store8<CACHE>(v ? p.c.v : p.c.k, w.exp * p.c.dim + j, x[v]);
  }
}

// Keys (blockIdx.y 0) or values (1): one stream to read and one to write at a time measured 5%
// faster here than both.
template <int OUT, int CACHE, int LG>
__global__ void __launch_bounds__(kKvThreads) dresd_kv_get(KvParams p) {
  const uint32_t i = blockIdx.x * (uint32_t)(kKvThreads / LG) + threadIdx.x / LG;
  const int j = (threadIdx.x % LG) * 8;
  if (i >= (uint32_t)(p.n * p.c.heads) || j >= p.c.dim) return;
  const bool value = blockIdx.y != 0;
  const Row w = row_of(p, i);
  f8v x = {};
  if (w.inside) {
    x = load8<CACHE>(value ? p.c.v : p.c.k, w.exp * p.c.dim + j);
    if constexpr (CACHE == kF8) {
      const int e = (int)(value ? p.c.v_exp : p.c.k_exp)[w.exp] - 127;
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = ldexpf(x[k], e);
    }
  }
  store8<OUT>(value ? p.v_out : p.k_out, (int64_t)i * p.c.dim + j, x);
}

typedef void (*KvKernel)(KvParams);

template <int IO, int CACHE>
KvKernel pick_lanes(bool put, int dim) {
  const int lanes = dim / 8;
  if (lanes <= 8) return put ? dresd_kv_put<IO, CACHE, 8> : dresd_kv_get<IO, CACHE, 8>;
  if (lanes <= 16) return put ? dresd_kv_put<IO, CACHE, 16> : dresd_kv_get<IO, CACHE, 16>;
  return put ? dresd_kv_put<IO, CACHE, 32> : dresd_kv_get<IO, CACHE, 32>;
}

template <int IO>
KvKernel pick_cache(bool put, int cache, int dim) {
  if (cache == kF16) return pick_lanes<IO, kF16>(put, dim);
  if (cache == kBF16) return pick_lanes<IO, kBF16>(put, dim);
  return pick_lanes<IO, kF8>(put, dim);
}

hipError_t launch(bool put, const KvParams &p, hipStream_t st) {
  if (p.n == 0) return hipSuccess;
  KvKernel k = p.dtype == kF32 ? pick_cache<kF32>(put, p.c.dtype, p.c.dim)
             : p.dtype == kF16 ? pick_cache<kF16>(put, p.c.dtype, p.c.dim)
                               : pick_cache<kBF16>(put, p.c.dtype, p.c.dim);
  const int lg = p.c.dim <= 64 ? 8 : p.c.dim <= 128 ? 16 : 32;
  const int64_t rows = p.n * p.c.heads, per = kKvThreads / lg;
  KvParams q = p;
  void *args[] = {&q};
  return hipLaunchKernel((const void *)k, dim3((unsigned)((rows + per - 1) / per), put ? 1 : 2),
                         dim3(kKvThreads), args, 0, st);
}

}  // namespace

hipError_t launch_kv_write(const KvParams &p, hipStream_t st) { return launch(true, p, st); }
hipError_t launch_kv_read(const KvParams &p, hipStream_t st) { return launch(false, p, st); }

}  // namespace dresd
