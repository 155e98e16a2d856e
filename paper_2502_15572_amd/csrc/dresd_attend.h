// What the attention kernels share (dresd_attend_wave.hip, dresd_attend_tile.hip,
// dresd_attend.hip).
#pragma once
#include "dresd_device.h"
#include "dresd_verify.h"

namespace dresd {

typedef float f16v __attribute__((ext_vector_type(16)));
typedef short s4v __attribute__((ext_vector_type(4)));
typedef uint16_t w8 __attribute__((ext_vector_type(8)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));

// How a call is launched.  Query rows of one sequence and cache head (token
// t, head g of the group: row t group + g) are cut into blocks of `rows`; a unit
// is a block of one cache head, and its keys are cut into `splits`.
struct AttendPlan {
  AttendParams p;
  int group;                 // query heads per cache head
  int rows;                  // rows of a block
  int ct;                    // 0: tile kernel, else column tiles of the wave kernel
  int blocks;                // blocks of all sequences (an upper bound if ragged)
  int splits;
  int64_t total;             // workgroups before padding to 8
  float *part_o;             // [splits][T q_heads][dim] unnormalised sums (splits > 1)
  float *part_ml;            // [splits][T q_heads][2] their reference and weight
};

typedef void (*AttendKernel)(AttendPlan);
// By query type, 8-bit cache, padded width (64, 128, 256); null if not built.
AttendKernel attend_wave_kernel(int qt, bool f8, int dp, int ct);
AttendKernel attend_tile_kernel(int qt, bool f8, int dp);
size_t attend_wave_lds(bool f8, int dp, int ct);
size_t attend_tile_lds(int dp);

// 16-bit operands of one matrix instruction.
template <int QT>
struct Half;
template <>
struct Half<kF16> {
  typedef h8 v8;
  static __device__ __forceinline__ f4 mfma16(v8 a, v8 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f16v mfma32(v8 a, v8 b, f16v c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
  // the 16 x 16 x 16 instruction, four elements a lane
  static __device__ __forceinline__ f4 mfma16_half(u2 a, u2 b, f4 c) {
    typedef _Float16 h4 __attribute__((ext_vector_type(4)));
    return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(h4, a),
                                                 __builtin_bit_cast(h4, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ _Float16 round(float x) { return (_Float16)x; }
  static constexpr uint32_t kInf = 0x7c00u;
  // Weights are kept at 2^10 times their value against the reference, so that small ones
  // stay normal numbers, and may pass the reference by 2^4.
  static constexpr float kBias = 10.f, kSlack = 4.f;
};
template <>
struct Half<kBF16> {
  typedef b8 v8;
  static __device__ __forceinline__ f4 mfma16(v8 a, v8 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f16v mfma32(v8 a, v8 b, f16v c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f4 mfma16_half(u2 a, u2 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s4v, a),
                                                     __builtin_bit_cast(s4v, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ __bf16 round(float x) { return (__bf16)x; }
  static constexpr uint32_t kInf = 0x7f80u;
  static constexpr float kBias = 0.f, kSlack = 8.f;
};

// Eight e4m3 values (exact in either 16-bit type).
template <int QT>
__device__ __forceinline__ typename Half<QT>::v8 from_f8(u2 x) {
  typename Half<QT>::v8 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (QT == kF16) {
      const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x[i], 1.f, false);
      const auto hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x[i], 1.f, true);
      r[4 * i] = lo[0];
      r[4 * i + 1] = lo[1];
      r[4 * i + 2] = hi[0];
      r[4 * i + 3] = hi[1];
    } else {
      const auto lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], 1.f, false);
      const auto hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], 1.f, true);
      r[4 * i] = lo[0];
      r[4 * i + 1] = lo[1];
      r[4 * i + 2] = hi[0];
      r[4 * i + 3] = hi[1];
    }
  }
  return r;
}

// Reads a 4 x 16 block of 16-bit values transposed, per 16 lanes: lane i names row
// i / 4 and columns 4 (i % 4) .. + 3, and receives column i of the four rows.
__device__ __forceinline__ s4v read_transposed(const uint8_t *lds) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s4v *)(lds));
}

// The same for an 8 x 16 block of bytes: lane i names row i / 2 and columns 8 (i % 2) .. + 7,
// and receives column i of the eight rows.
__device__ __forceinline__ u2 read_transposed8(const uint8_t *lds) {
  typedef int i2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                                    (__attribute__((address_space(3))) i2 *)(lds)));
}

typedef __attribute__((address_space(3))) uint8_t lds_byte;
__device__ __forceinline__ uint32_t lds_address(const uint8_t *p) {
  return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_byte *)(p));
}
// Copies from each lane's own address to LDS: 16 bytes to lds + 16 lane; one byte,
// widened to a dword, to lds + 4 lane.  copy16_past does not keep what it reads in the caches.
// Callers wait with wait_vmcnt.
__device__ __forceinline__ void copy16_from(const uint8_t *src, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %1\n\ts_nop 0\n\t"
      "global_load_lds_dwordx4 %0, off"
      :
      : "v"(src), "s"(lds)
      : "memory");
}
__device__ __forceinline__ void copy16_past(const uint8_t *src, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %1\n\ts_nop 0\n\t"
      "global_load_lds_dwordx4 %0, off nt"
      :
      : "v"(src), "s"(lds)
      : "memory");
}
__device__ __forceinline__ void copy_byte_from(const uint8_t *src, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %1\n\ts_nop 0\n\t"
      "global_load_lds_ubyte %0, off"
      :
      : "v"(src), "s"(lds)
      : "memory");
}

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// Zeros in place of infinities and NaN among 16 bytes of a cache row; whether there
// were any.
template <int QT, bool F8>
__device__ __forceinline__ bool drop_nonfinite(u4 &x) {
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (F8) {      // bytes of 7 ones: those that a carry into their sign shows
      const uint32_t m = ((x[i] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
      any |= m;
      x[i] &= ~((m >> 7) * 255u);
    } else {
      const uint32_t lo = (x[i] & Half<QT>::kInf) == Half<QT>::kInf ? 0xffffu : 0u;
      const uint32_t hi = ((x[i] >> 16) & Half<QT>::kInf) == Half<QT>::kInf ? 0xffff0000u : 0u;
      any |= lo | hi;
      x[i] &= ~(lo | hi);
    }
  }
  return any != 0;
}

// From a product q . k (or (-q) . k, for a negative scale) to powers of two.  Never 0,
// so that a masked score stays -inf.
__device__ __forceinline__ float score_factor(float scale) {
  return fmaxf(fabsf(scale) * 1.44269504088896341f, 1e-30f);
}

// Factor of a value row of an 8-bit cache.  Byte 255 is none: NaN for every row,
// or, where some rows do not see it, 0 (and the rows that do get NaN scores).
__device__ __forceinline__ float value_factor(uint32_t byte, bool masked) {
  return byte != 255u ? __uint_as_float(byte << 23) : masked ? 0.f : __builtin_nanf("");
}

// What a value row's exponent adds to its score where weights are f16, in powers of two: the
// reference goes by the weight of the value as it is stored, which then stays below 2^15.  Between
// -60 (values that small are zero in f16) and 80 (values of 2^88): there the row's own weight in
// the sum is 2^-70 at least, and 2^31 weights that exponentials flush, each below 2^-126,
// are still 2^-25 of it.
__device__ __forceinline__ float value_exponent(uint32_t byte) {
  const int e = (int)byte - 127;
  return (float)(e < -60 ? -60 : e > 80 ? 80 : e);
}

// Positions past this are not seen (a tile's stay inside 31 bits).
constexpr int kPositions = 0x7fffff00;

// The block of a workgroup.
struct Unit {
  int b, head, split;        // sequence, cache head, split of its keys
  int row0, rows;            // first row of the block, rows of the sequence and head
  int64_t token0;            // q row of the sequence's first token
  int n, len, before, L;     // chunk, tokens, tokens before the chunk, positions there are
};

// Workgroups go round the 8 XCDs in turn; each XCD takes a contiguous eighth of
// the units, in an order in which neighbours read the same keys, so that they meet in its L2.
// False: no such block.
__device__ __forceinline__ bool unit_of(const AttendPlan &pl, Unit &u) {
  const int64_t eighth = (pl.total + 7) / 8;
  const int64_t at = (int64_t)(blockIdx.x % 8) * eighth + blockIdx.x / 8;
  if (at >= pl.total) return false;
  const int col = (int)(at / pl.blocks);
  int blk = (int)(at - (int64_t)col * pl.blocks);
  u.head = col / pl.splits;
  u.split = col - u.head * pl.splits;
  const AttendParams &p = pl.p;
  if (!p.ragged) {
    const int per = (p.n * pl.group + pl.rows - 1) / pl.rows;
    u.b = blk / per;
    blk -= u.b * per;
    u.n = p.n;
    u.token0 = (int64_t)u.b * p.n;
  } else {
    // the sequence that holds this block: 64 sequences at a time
    const int lane = threadIdx.x & 63;
    int seen = 0;            // blocks of the sequences before
    u.b = -1;
    for (int i0 = 0; i0 < p.B; i0 += kWaveSize) {
      const int i = i0 + lane;
      int64_t a = 0, e = 0;
      if (i < p.B) {
        a = p.starts[i];
        e = p.starts[i + 1];
      }
      const int64_t n = a >= 0 && e <= p.T && e > a ? e - a : 0;
      int x = (int)((n * pl.group + pl.rows - 1) / pl.rows);
      const int own = x;
#pragma unroll
      for (int o = 1; o < kWaveSize; o <<= 1) {
        const int y = __shfl_up(x, o, kWaveSize);
        if (lane >= o) x += y;
      }
      const uint64_t past = __ballot(seen + x > blk);
      if (past) {
        const int w = __ffsll((long long)past) - 1;
        u.b = i0 + w;
        blk -= seen + __shfl(x - own, w, kWaveSize);
        u.n = __shfl((int)n, w, kWaveSize);
        u.token0 = __shfl((int)a, w, kWaveSize);
        break;
      }
      seen += __shfl(x, kWaveSize - 1, kWaveSize);
    }
    if (u.b < 0) return false;
    u.b = __builtin_amdgcn_readfirstlane(u.b);
    blk = __builtin_amdgcn_readfirstlane(blk);
    u.n = __builtin_amdgcn_readfirstlane(u.n);
    u.token0 = __builtin_amdgcn_readfirstlane((int)u.token0);
  }
  u.rows = u.n * pl.group;
  if (blk < 0 || blk > (u.rows - 1) / pl.rows) return false;  // (chunks that overlap)
  u.row0 = blk * pl.rows;
  const int len = p.lengths[u.b];
  u.len = len > 0 ? len : 0;                 // (so that the difference stays inside 32 bits)
  u.before = u.len - u.n;
  const int64_t room = (int64_t)p.width << p.c.page_log;
  u.L = u.len < room ? u.len : (int)room;
  u.L = u.L < kPositions ? u.L : kPositions;
  return true;
}

// First position past those that a block's rows may see.
__device__ __forceinline__ int reach(const AttendPlan &pl, const Unit &u, int rows) {
  if (pl.p.mask) return u.L;
  const int last = u.row0 + rows < u.rows ? u.row0 + rows : u.rows;  // rows past the last are not
  const int64_t end = (int64_t)u.before + (last - 1) / pl.group + 1;
  return end < u.L ? (int)end : u.L;
}

// Positions that every row of the block sees, as far as there are pages.
__device__ __forceinline__ int seen_by_all(const AttendPlan &pl, const Unit &u) {
  const int64_t c = (int64_t)u.before + (pl.p.mask ? 0 : u.row0 / pl.group + 1);
  return c < u.L ? (int)c : u.L;
}

// Which of the 64 positions from pos on the row of chunk token t sees, by the
// length, the chunk and the mask.
__device__ __forceinline__ uint64_t window(const AttendPlan &pl, const Unit &u, int64_t row, int t,
                                           int pos) {
  auto below = [](int64_t c) -> uint64_t {   // the lowest c bits
    return c <= 0 ? 0ull : c >= 64 ? ~0ull : (1ull << c) - 1;
  };
  uint64_t w = below((int64_t)u.L - pos);
  const int64_t j = (int64_t)pos - u.before;  // chunk token of the first position
  if (!pl.p.mask) return w & below((int64_t)t + 1 - j);
  const uint64_t *m = pl.p.mask + row * pl.p.words;
  auto word = [&](int64_t i) -> uint64_t { return i >= 0 && i < pl.p.words ? m[i] : 0ull; };
  if (j >= 0) {
    const int s = (int)(j & 63);
    const uint64_t lo = word(j >> 6) >> s;
    return w & (s ? lo | word((j >> 6) + 1) << (64 - s) : lo);
  }
  if (j <= -64) return w;
  return w & (below(-j) | word(0) << (int)-j);
}

// out = x / l, lse = (ref + log2 l) ln 2, where l's power of two and the reference, which may cancel
// (f16 weights are kept at 2^10, those of 8-bit values at their values' power too), are joined
// first, without a rounding larger than the result's.
template <int QT>
__device__ __forceinline__ void finish_row(const AttendParams &p, int64_t out, int d, f4 x,
                                           float ref, float l) {
  typedef uint16_t us4 __attribute__((ext_vector_type(4)));
  const float inv = l != 0.f ? 1.f / l : 0.f;
  us4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = __builtin_bit_cast(uint16_t, Half<QT>::round(x[i] * inv));
  *reinterpret_cast<us4 *>(static_cast<uint16_t *>(p.out) + out * p.c.dim + d) = y;
  if (d == 0 && p.lse) {
    const float whole = ref + (float)__builtin_amdgcn_frexp_expf(l);
    p.lse[out] = l != 0.f ? (whole + log2f(__builtin_amdgcn_frexp_mantf(l))) * 0.693147180559945309f
                          : -__builtin_huge_valf();
  }
}

// Four dims of a row of the output (head and row at `out` of [T, q_heads]): sums x
// of weights 2^(s - ref), l the sum of the weights.
template <int QT>
__device__ __forceinline__ void store_row(const AttendPlan &pl, int split, int64_t out, int d, f4 x,
                                          float ref, float l) {
  const AttendParams &p = pl.p;
  if (pl.splits > 1) {
    const int64_t at = (int64_t)split * p.T * p.q_heads + out;
    // (a part without weight is not read)
    if (l != 0.f) *reinterpret_cast<f4 *>(pl.part_o + at * p.c.dim + d) = x;
    if (d == 0) *reinterpret_cast<float2 *>(pl.part_ml + 2 * at) = float2{ref, l};
    return;
  }
  finish_row<QT>(p, out, d, x, ref, l);
}

}  // namespace dresd
