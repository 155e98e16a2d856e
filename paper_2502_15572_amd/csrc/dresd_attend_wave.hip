// gfx950 attention of few rows over a paged cache: up to 16, 32 or 64 rows (tokens
// times query heads of one cache head) a workgroup.
//
// What bounds it is reading the cache: a workgroup does 16 to 64 multiply-adds per
// 16-bit value read, the matrix cores' and the memory's rates being some 350
// apart.  So nothing is shared: each of the 4 waves streams tiles of its own (wave
// w the tiles w, w + 4, ... of the split), keys from memory to registers as the
// operand that the matrix instruction takes, values through a swizzled LDS tile of
// the wave's own that is read transposed, and no barrier holds a wave up before the
// end.  While a tile is computed, the next one is on its way.
//
// Scores are formed transposed, S^T = K Q^T: a lane then holds one row (lane % 16)
// and 4 keys of every 16, which is, keys in another order, the operand that the
// second product O^T = V^T P^T takes.  The weights never leave their registers,
// and a row's statistics and the rescaling of its sums are one lane's.
//
// Running softmax: the reference m of a row is moved only when a score passes it by
// kSlack (in powers of two); until then weights and sums grow past 1.  With m moved
// at most once for most rows, the exchange between a row's 4 lanes is rare.
#include <type_traits>

#include "dresd_attend.h"

#ifndef DRESD_ATTEND_DP
#error "DRESD_ATTEND_DP: the padded width that this unit builds"
#endif

namespace dresd {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = 4;

// Keys of a tile: 16 KiB of keys and values at a width of 128.
constexpr int tile_keys(bool f8) { return f8 ? 64 : 32; }

// LDS of a wave: values [keys][DP] 16 bit, row offsets [keys] i64, factors of
// keys and values [keys] f32 each (8-bit caches).
constexpr size_t wave_bytes(bool f8, int dp) {
  return (size_t)tile_keys(f8) * (dp * 2 + 8 + 8);
}
// At the end: sums [waves][rows][DP + 4] and statistics [waves][rows][2].
constexpr size_t end_bytes(int dp, int ct) {
  return (size_t)kWaves * 16 * ct * (dp + 4 + 2) * 4;
}

template <int QT, bool F8, int DP, int CT>
__global__ void __launch_bounds__(kThreads, CT == 1 && DP <= 128 ? 2 : 1)
    dresd_attend_wave(AttendPlan pl) {
  typedef Half<QT> H;
  typedef typename H::v8 v8;
  constexpr int KT = tile_keys(F8), U = KT / 32;  // 32-key groups of a tile
  constexpr int KS = DP / 32;                     // 32-dim steps
  constexpr int VR = F8 ? DP / 32 : DP / 16;      // value loads per 32 keys
  constexpr int VL = F8 ? DP / 16 : DP / 8;       // lanes of a value row
  extern __shared__ __align__(16) uint8_t lds[];
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  const int col = lane & 15, kq = lane >> 4;
  Unit u;
  if (!unit_of(pl, u)) return;
  const AttendParams &p = pl.p;
  const int D = p.c.dim;

  uint8_t *vt = lds + (size_t)wid * wave_bytes(F8, DP);
  int64_t *offs = reinterpret_cast<int64_t *>(vt + (size_t)KT * DP * 2);
  float *kf = reinterpret_cast<float *>(offs + KT), *vf = kf + KT;

  // queries: operand of row 16 c + col, dims in the order in which keys are read
  v8 q[CT][KS];
  int tok[CT];
  int64_t row[CT];
  const uint32_t flip = p.scale < 0.f ? 0x80008000u : 0u;  // (-q) . k |scale|
  const float c2 = score_factor(p.scale);
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    int r = u.row0 + 16 * c + col;
    r = r < u.rows ? r : u.rows - 1;
    tok[c] = r / pl.group;
    row[c] = u.token0 + tok[c];
    const int h = u.head * pl.group + (r - tok[c] * pl.group);
    const uint16_t *src = static_cast<const uint16_t *>(p.q) + row[c] * p.q_row + h * p.q_head;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int d = F8 ? 64 * (s / 2) + 16 * kq + 8 * (s & 1) : 32 * s + 8 * kq;
      u4 x = {};
      if (d < D) x = *reinterpret_cast<const u4 *>(src + d);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] ^= flip;
      q[c][s] = __builtin_bit_cast(v8, x);
    }
  }

  f4 acc[CT][DP / 16];
  float m[CT], l[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    m[c] = -3e38f;
    l[c] = 0.f;
#pragma unroll
    for (int d = 0; d < DP / 16; ++d) acc[c][d] = f4{0.f, 0.f, 0.f, 0.f};
  }

  // this split's tiles
  const int end = reach(pl, u, pl.rows);
  const int tiles = end > 0 ? (end + KT - 1) / KT : 0;
  // (whole rounds of the four waves)
  const int per = ((tiles + kWaves - 1) / kWaves + pl.splits - 1) / pl.splits * kWaves;
  const int64_t lo = (int64_t)u.split * per;
  const int first = lo < tiles ? (int)lo : tiles;
  const int last = first + per < tiles ? first + per : tiles;

  const uint8_t *kbase = static_cast<const uint8_t *>(p.c.k);
  const uint8_t *vbase = static_cast<const uint8_t *>(p.c.v);
  const int row_bytes = F8 ? D : 2 * D;
  const int32_t *table = p.table + (int64_t)u.b * p.width;
  const int in_page = (1 << p.c.page_log) - 1;

  // page of this lane's key of a tile (lanes past the tile: unused)
  auto page_of = [&](int t) -> int {
    if (t >= last || lane >= KT) return -1;
    const int pos = t * KT + lane;
    return pos < u.L ? table[pos >> p.c.page_log] : -1;
  };
  // offsets of a tile's rows into LDS; which of its keys there are
  uint32_t ke = 0, ve = 0;                        // their exponents
  auto place = [&](int t, int page) -> uint64_t {
    const bool ok = (uint32_t)page < (uint32_t)p.c.pages;
    const int64_t r = ok ? ((((int64_t)page * p.c.heads + u.head) << p.c.page_log) +
                            ((t * KT + lane) & in_page))
                         : 0;
    if (lane < KT) offs[lane] = r * row_bytes;
    if constexpr (F8) {
      ke = ok ? p.c.k_exp[r] : 127u;
      ve = ok ? p.c.v_exp[r] : 127u;
    }
    return __ballot(ok);
  };

  u4 kr[U][2][F8 ? KS / 2 : KS], vr[U][VR];
  const int vl = lane % VL, vk = lane / VL;       // 16 bytes of a row, row within a load
  // Where the head is narrower than DP, the dims past it are read from the row's
  // start: against queries of zero, and for outputs that are not stored.
  int kd[F8 ? KS / 2 : KS];
#pragma unroll
  for (int i = 0; i < (F8 ? KS / 2 : KS); ++i) {
    const int d = F8 ? 64 * i + 16 * kq : 32 * i + 8 * kq;
    kd[i] = d < D ? (F8 ? d : 2 * d) : 0;
  }
  const int vd = 16 * vl < row_bytes ? 16 * vl : 0;
  // (rows of 8-bit caches are 8-byte aligned, and may end inside 16 bytes, at odd multiples of 8)
  auto load16 = [&](auto halves, const uint8_t *src, int at) -> u4 {
    if constexpr (decltype(halves)::value) {
      const u2 a = *reinterpret_cast<const u2 *>(src + at);
      const u2 b = *reinterpret_cast<const u2 *>(src + (at + 8 < row_bytes ? at + 8 : at));
      return u4{a[0], a[1], b[0], b[1]};
    } else {
      return *reinterpret_cast<const u4 *>(src + at);
    }
  };
  auto load_tile = [&](auto halves) {
#pragma unroll
    for (int g = 0; g < U; ++g)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const uint8_t *src = kbase + offs[32 * g + 16 * s + col];
#pragma unroll
        for (int i = 0; i < (F8 ? KS / 2 : KS); ++i) kr[g][s][i] = load16(halves, src, kd[i]);
      }
#pragma unroll
    for (int g = 0; g < U; ++g)
#pragma unroll
      for (int i = 0; i < VR; ++i)
        vr[g][i] = load16(halves, vbase + offs[32 * g + (64 / VL) * i + vk], vd);
  };
  auto load = [&]() {
    if (F8 && (D & 8)) load_tile(std::true_type{});
    else load_tile(std::false_type{});
  };
  // LDS address of 16-byte chunk c of key k: the 32-byte pairs of 8 keys that are
  // read together lie in different banks
  auto chunk = [&](int k, int c) -> uint8_t * {
    return vt + ((size_t)k * (DP / 8) + (c ^ ((DP == 64 ? (k >> 1) & 3 : k & 7) << 1))) * 16;
  };

  // one tile: its keys and values are in registers, ok its keys that there are
  auto compute = [&](int t, bool masked, uint64_t ok, int next, int next_page,
                     uint64_t &next_ok) {
    // scores, rows of keys x columns of query rows
    f4 s[CT][U][2];
#pragma unroll
    for (int g = 0; g < U; ++g)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int c = 0; c < CT; ++c) s[c][g][h] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KS; ++i) {
          v8 k;
          if constexpr (F8) {
            const u4 x = kr[g][h][i / 2];
            k = from_f8<QT>(i & 1 ? u2{x[2], x[3]} : u2{x[0], x[1]});
          } else {
            k = __builtin_bit_cast(v8, kr[g][h][i]);
          }
#pragma unroll
          for (int c = 0; c < CT; ++c) s[c][g][h] = H::mfma16(k, q[c][i], s[c][g][h]);
        }
      }
    // values into LDS; where not every row sees all keys, keys that are not there as zeros,
    // and keys with a value that is not finite apart
    uint64_t bad = 0;
    if (masked) {
      if constexpr (F8) bad = __ballot(lane < KT && ve == 255u);
#pragma unroll
      for (int g = 0; g < U; ++g)
#pragma unroll
        for (int i = 0; i < VR; ++i) {
          constexpr int RL = 64 / VL;             // rows of a load
          if (!(((ok >> vk) >> (32 * g + RL * i)) & 1)) vr[g][i] = u4{};
          uint64_t w = __ballot(drop_nonfinite<QT, F8>(vr[g][i]));
          while (w) {                             // rare
            const int j = __ffsll((long long)w) - 1;
            bad |= 1ull << (32 * g + RL * i + j / VL);
            w &= w - 1;
          }
        }
    }
    if constexpr (F8) {
      if (lane < KT) {
        kf[lane] = __uint_as_float(ke << 23);
        vf[lane] = value_factor(ve, masked);
      }
    }
#pragma unroll
    for (int g = 0; g < U; ++g)
#pragma unroll
      for (int i = 0; i < VR; ++i) {
        const int k = 32 * g + (64 / VL) * i + vk;
        if constexpr (F8) {
          *reinterpret_cast<v8 *>(chunk(k, 2 * vl)) = from_f8<QT>(u2{vr[g][i][0], vr[g][i][1]});
          *reinterpret_cast<v8 *>(chunk(k, 2 * vl + 1)) = from_f8<QT>(u2{vr[g][i][2], vr[g][i][3]});
        } else {
          *reinterpret_cast<u4 *>(chunk(k, vl)) = vr[g][i];
        }
      }
    wave_sync_lds();
    f4 kfac[U][2], vfac[U][2];
    if constexpr (F8) {
#pragma unroll
      for (int g = 0; g < U; ++g)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          kfac[g][h] = *reinterpret_cast<const f4 *>(kf + 32 * g + 16 * h + 4 * kq);
          vfac[g][h] = *reinterpret_cast<const f4 *>(vf + 32 * g + 16 * h + 4 * kq);
        }
    }
    // the next tile is on its way while this one's weights are formed
    wave_sync_lds();
    if (next < last) {
      next_ok = place(next, next_page);
      wave_sync_lds();
      load();
    }
    // weights
    v8 w[CT][U];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      if constexpr (F8)
#pragma unroll
        for (int g = 0; g < U; ++g)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[c][g][h][i] *= kfac[g][h][i];
      if (masked) {
        const uint64_t see = (window(pl, u, row[c], tok[c], t * KT) & ok) >> (4 * kq);
        const uint64_t inf = bad >> (4 * kq);
#pragma unroll
        for (int g = 0; g < U; ++g) {
          const uint32_t is = (uint32_t)(see >> (32 * g)), no = (uint32_t)(inf >> (32 * g));
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float x = s[c][g][h][i];
              x = (no >> (16 * h + i)) & 1 ? __builtin_nanf("") : x;
              s[c][g][h][i] = (is >> (16 * h + i)) & 1 ? x : -__builtin_huge_valf();
            }
        }
      }
      float top = -3e38f;
#pragma unroll
      for (int g = 0; g < U; ++g)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float x = s[c][g][h][i];
            if constexpr (F8 && QT == kF16) {
              // the largest weight is that of the value as it is stored
              const int e = (int)((__float_as_uint(vfac[g][h][i]) >> 23) & 255u) - 127;
              x = x * c2 + (float)(e < -60 ? -60 : e > 20 ? 20 : e);
            }
            top = fmaxf(top, x);
          }
      if constexpr (!(F8 && QT == kF16)) top *= c2;  // (in powers of two)
      if (__any(top > m[c] + H::kSlack)) {
        top = fmaxf(top, __shfl_xor(top, 16, kWaveSize));
        top = fmaxf(top, __shfl_xor(top, 32, kWaveSize));
        const float mn = fmaxf(m[c], top);
        const float a = exp2_hw(m[c] - mn);
        m[c] = mn;
        l[c] *= a;
#pragma unroll
        for (int d = 0; d < DP / 16; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[c][d][i] *= a;
      }
      const float ref = m[c] - H::kBias;
      float sum = 0.f;
#pragma unroll
      for (int g = 0; g < U; ++g)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float x = exp2_hw(fmaf(s[c][g][h][i], c2, -ref));
            sum += x;
            if constexpr (F8) x *= vfac[g][h][i];
            w[c][g][4 * h + i] = H::round(x);
          }
      l[c] += sum;
    }
    // O^T += V^T P^T
#pragma unroll
    for (int g = 0; g < U; ++g)
#pragma unroll
      for (int d = 0; d < DP / 16; ++d) {
        const int k = 32 * g + 4 * kq + (col >> 2);
        const int at = 2 * d + ((col & 3) >> 1), in = (col & 1) * 8;
        const s4v a = read_transposed(chunk(k, at) + in);
        const s4v b = read_transposed(chunk(k + 16, at) + in);
        typedef short s8v __attribute__((ext_vector_type(8)));
        const v8 x = __builtin_bit_cast(
            v8, s8v{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
#pragma unroll
        for (int c = 0; c < CT; ++c) acc[c][d] = H::mfma16(x, w[c][g], acc[c][d]);
      }
    wave_sync_lds();
  };

  int t = first + wid;
  if (t < last) {
    uint64_t ok = place(t, page_of(t));
    wave_sync_lds();
    load();
    int page = page_of(t + kWaves);
    const uint64_t whole = KT == 64 ? ~0ull : (1ull << KT) - 1;
    const int plain = seen_by_all(pl, u);
    for (; t < last; t += kWaves) {
      const int ahead = page_of(t + 2 * kWaves);
      uint64_t next_ok = 0;
      // keys that are all there and that every row sees
      const bool masked = (t + 1) * KT > plain || (ok & whole) != whole;
      compute(t, masked, ok, t + kWaves, page, next_ok);
      ok = next_ok;
      page = ahead;
    }
  }

  // the four waves' sums: rows of a wave [16 CT][DP + 4], statistics
  constexpr int R = 16 * CT, OS = DP + 4;
  float *o = reinterpret_cast<float *>(lds), *ml = o + (size_t)kWaves * R * OS;
  __syncthreads();
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    l[c] += __shfl_xor(l[c], 16, kWaveSize);
    l[c] += __shfl_xor(l[c], 32, kWaveSize);
    if (kq == 0) {
      ml[(wid * R + 16 * c + col) * 2] = m[c];
      ml[(wid * R + 16 * c + col) * 2 + 1] = l[c];
    }
#pragma unroll
    for (int d = 0; d < DP / 16; ++d)
      *reinterpret_cast<f4 *>(o + (size_t)(wid * R + 16 * c + col) * OS + 16 * d + 4 * kq) =
          acc[c][d];
  }
  __syncthreads();
  for (int e = tid; e < R * (DP / 4); e += kThreads) {
    const int r = e / (DP / 4), d = (e - r * (DP / 4)) * 4;
    if (u.row0 + r >= u.rows || d >= D) continue;
    float top = -3e38f, sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, ml[(w * R + r) * 2]);
    f4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float a = exp2_hw(ml[(w * R + r) * 2] - top);
      sum += ml[(w * R + r) * 2 + 1] * a;
      const f4 y = *reinterpret_cast<const f4 *>(o + (size_t)(w * R + r) * OS + d);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] += y[i] * a;
    }
    const int tk = (u.row0 + r) / pl.group;
    const int64_t out =
        (u.token0 + tk) * p.q_heads + u.head * pl.group + (u.row0 + r - tk * pl.group);
    store_row<QT>(pl, u.split, out, d, x, top - H::kBias, sum);
  }
}

template <int QT, bool F8>
AttendKernel pick(int ct) {
  constexpr int DP = DRESD_ATTEND_DP;
  if (ct == 1) return dresd_attend_wave<QT, F8, DP, 1>;
  if (ct == 2) return dresd_attend_wave<QT, F8, DP, 2>;
  if constexpr (DP <= 128)
    if (ct == 4) return dresd_attend_wave<QT, F8, DP, 4>;
  return nullptr;
}

}  // namespace

#define DRESD_CAT2(a, b) a##b
#define DRESD_CAT(a, b) DRESD_CAT2(a, b)
AttendKernel DRESD_CAT(attend_wave_kernel_, DRESD_ATTEND_DP)(int qt, bool f8, int ct) {
  if (qt == kF16) return f8 ? pick<kF16, true>(ct) : pick<kF16, false>(ct);
  return f8 ? pick<kBF16, true>(ct) : pick<kBF16, false>(ct);
}

#if DRESD_ATTEND_DP == 128
size_t attend_wave_lds(bool f8, int dp, int ct) {
  const size_t a = kWaves * wave_bytes(f8, dp), b = end_bytes(dp, ct);
  return a > b ? a : b;
}
#endif

}  // namespace dresd
