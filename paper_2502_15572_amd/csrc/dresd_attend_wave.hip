// gfx950 attention of few rows over a paged cache: 16 or 32 rows (tokens times query
// heads of one cache head) a workgroup.
//
// What bounds it is reading the cache: a workgroup does 16 or 32 multiply-adds per
// value read, the matrix cores' and the memory's rates being some 350 apart.  So
// the reading is all that is arranged for.  The four waves share nothing before
// the end: each streams tiles of its own (wave w the tiles w, w + 4, ... of the
// split) through a ring of LDS slots, by copies that go from memory to LDS without
// registers, past the caches and without a barrier; all slots but the one at hand are
// on their way.  Page ids run one ring further ahead, as copies too, so that nothing
// waits for memory but the wait for a whole tile.
// 16-bit caches are read at 5.7 TB/s, 8-bit ones at 5.4 (64 sequences of 2,000 to 8,000 tokens,
// 8 heads of 128, 8 query heads each); the copies alone, without the products,
// reach 6.4 and 6.0, loads through the caches a tenth less.
//
// Copies land lane after lane, so what a lane fetches decides the layout: 16-byte
// chunks of a row are exchanged so that the keys that 16 lanes read at once, and the
// values that are read transposed, lie in different banks.
//
// Scores are formed transposed, S^T = K Q^T: a lane then holds one row (lane % 16)
// and 4 keys of every 16, which is the operand that the second product
// O^T = V^T P^T takes.  The weights never leave their registers, and a row's
// statistics and the rescaling of its sums are one lane's.
//
// Running softmax: the reference m of a row is moved only when a score passes it by
// kSlack (in powers of two); until then weights and sums grow past 1.  With m moved
// at most once for most rows, the exchange between a row's 4 lanes is rare.
#include "dresd_attend.h"

#ifndef DRESD_ATTEND_DP
#error "DRESD_ATTEND_DP: the padded width that this unit builds"
#endif

namespace dresd {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = 4;

// Shape of the ring: a tile is one 16-key group (16 bit) or two (8 bit), a slot its
// keys and its values, each row of DP elements.
template <bool F8, int DP>
struct Ring {
  // Up to a width of 128 registers are left for two waves a SIMD, which share the LDS (one
  // wave with a ring of four slots had the memory wait for its products: 64 sequences of
  // up to 8,000 tokens, 8 heads of 128 in 8 bits, 145 us against 120).
  static constexpr bool kPair = DP <= 128;
  static constexpr int kKeys = F8 ? 32 : 16;
  static constexpr int kPitch = DP * (F8 ? 1 : 2);      // bytes of a row
  static constexpr int kHalf = kKeys * kPitch;          // of a tile's keys, or values
  static constexpr int kSlots = (kPair ? 16384 : 32768) / (2 * kHalf);
  static constexpr int kCopies = kHalf / 1024;          // of keys, and of values
  static constexpr int kRows = 1024 / kPitch;           // rows of a copy
  // of a wave: slots, row offsets of a tile, page ids of two rings of tiles, exponents of
  // keys and values
  static constexpr int kOffs = kKeys * 8;
  static constexpr int kIds = 2 * kSlots * kKeys * 4;
  static constexpr int kExps = F8 ? kSlots * kKeys * 8 : 0;
  static constexpr int kBytes = kSlots * 2 * kHalf + kOffs + kIds + kExps;
  // operations of a tile's copies
  static constexpr int kOps = 2 * kCopies + (F8 ? 2 : 0);
};

// At the end: sums [waves][rows][DP + 4] and statistics [waves][rows][2].
constexpr size_t end_bytes(int dp, int ct) {
  return (size_t)kWaves * 16 * ct * (dp + 4 + 2) * 4;
}

template <int QT, bool F8, int DP, int CT>
__global__ void __launch_bounds__(kThreads, (Ring<F8, DP>::kPair ? 2 : 1)) dresd_attend_wave(AttendPlan pl) {
  typedef Half<QT> H;
  typedef typename H::v8 v8;
  typedef Ring<F8, DP> R;
  constexpr int KT = R::kKeys, U = KT / 16;       // 16-key groups of a tile
  constexpr int KS = DP / 32;                     // 32-dim steps
  constexpr int NS = R::kSlots;
  extern __shared__ __align__(16) uint8_t lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, kq = lane >> 4;
  Unit u;
  if (!unit_of(pl, u)) return;
  const AttendParams &p = pl.p;
  const int D = p.c.dim;

  uint8_t *ring = lds + (size_t)wid * R::kBytes;
  int64_t *offs = reinterpret_cast<int64_t *>(ring + NS * 2 * R::kHalf);
  const int32_t *ids = reinterpret_cast<const int32_t *>(offs + KT);
  const uint32_t *exps = reinterpret_cast<const uint32_t *>(ids + 2 * NS * KT);
  const uint32_t ring_at = lds_address(ring);
  const uint32_t ids_at = ring_at + NS * 2 * R::kHalf + R::kOffs, exps_at = ids_at + R::kIds;

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

  // this split's tiles; tile i of this wave is t0 + kWaves i, i < count
  const int end = reach(pl, u, pl.rows);
  const int tiles = end > 0 ? (end + KT - 1) / KT : 0;
  // (whole rounds of the four waves)
  const int per = ((tiles + kWaves - 1) / kWaves + pl.splits - 1) / pl.splits * kWaves;
  const int64_t lo = (int64_t)u.split * per;
  const int first = lo < tiles ? (int)lo : tiles;
  const int last = first + per < tiles ? first + per : tiles;
  const int t0 = first + wid;
  const int count = t0 < last ? (last - t0 + kWaves - 1) / kWaves : 0;

  const int row_bytes = F8 ? D : 2 * D;
  const int in_page = (1 << p.c.page_log) - 1;
  const int32_t *table = p.table + (int64_t)u.b * p.width;
  // rows of this cache head: page * page_rows + position in the page
  const int64_t page_rows = (int64_t)p.c.heads << p.c.page_log;
  const int64_t head_row = (int64_t)u.head << p.c.page_log;
  const uint8_t *kbase = static_cast<const uint8_t *>(p.c.k);
  const uint8_t *vbase = static_cast<const uint8_t *>(p.c.v);

  // chunk exchange of a row of keys and of values (16-byte chunks: exclusive or)
  auto kswap = [](int k) -> int {
    if constexpr (F8) return DP == 64 ? (k >> 2) & 3 : DP == 128 ? (k >> 1) & 7 : k & 15;
    else return DP == 64 ? (k >> 1) & 7 : k & 15;
  };
  auto vswap = [&](int k) -> int {
    if constexpr (F8) return kswap(k);
    else return (DP == 64 ? (k >> 1) & 3 : k & 7) << 1;
  };
  // what this lane copies of a row: keys' and values' bytes.  Where the head is narrower
  // than DP, the dims past it are its first ones again: against queries of zero, and
  // for outputs that are not stored.
  constexpr int kPer = R::kPitch / 16;            // lanes of a row
  const int crow = lane / kPer;
  int kat[R::kCopies], vat[R::kCopies];
#pragma unroll
  for (int j = 0; j < R::kCopies; ++j) {
    const int k = R::kRows * j + crow, c = lane % kPer;
    kat[j] = 16 * (c ^ kswap(k));
    vat[j] = 16 * (c ^ vswap(k));
    kat[j] = kat[j] < row_bytes ? kat[j] : 0;
    vat[j] = vat[j] < row_bytes ? vat[j] : 0;
  }

  // page ids of tile i (one operation; nothing for positions past the last)
  auto fetch_ids = [&](int i) {
    const int pos = (t0 + kWaves * i) * KT + lane;
    if (lane < KT && pos < u.L)
      copy1_to_lds(table + (pos >> p.c.page_log), ids_at + (i % (2 * NS)) * KT * 4);
  };
  // page id of this lane's key of tile i, -1 where there is none
  const int klane = lane & (KT - 1);
  auto page_of = [&](int i) -> int {
    const int pos = (t0 + kWaves * i) * KT + klane, id = ids[(i % (2 * NS)) * KT + klane];
    return pos < u.L && (uint32_t)id < (uint32_t)p.c.pages ? id : -1;
  };
  // row of this lane's key of tile i (of the first page, where there is none); the offsets of
  // the tile's rows go to LDS
  auto place = [&](int i, int page) -> int64_t {
    const int64_t r = (int64_t)(page < 0 ? 0 : page) * page_rows + head_row +
                      (((t0 + kWaves * i) * KT + klane) & in_page);
    offs[klane] = r * row_bytes;
    return r;
  };
  // keys and values of tile i, of row r for this lane's key (kOps operations)
  auto fetch = [&](int i, int64_t r) {
    const uint32_t at = ring_at + (i % NS) * 2 * R::kHalf;
    int64_t o[R::kCopies];
#pragma unroll
    for (int j = 0; j < R::kCopies; ++j) o[j] = offs[R::kRows * j + crow];
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the slot has been read
    if constexpr (F8) {
      const uint32_t e = exps_at + (i % NS) * KT * 8;
      if (lane < KT) {
        copy_byte_from(p.c.k_exp + r, e);
        copy_byte_from(p.c.v_exp + r, e + KT * 4);
      }
    }
#pragma unroll
    for (int j = 0; j < R::kCopies; ++j) {
      copy16_past(kbase + o[j] + kat[j], at + 1024 * j);
      copy16_past(vbase + o[j] + vat[j], at + R::kHalf + 1024 * j);
    }
  };

  const int plain = seen_by_all(pl, u);
  if (count > 0) {
    const int ahead = count < 2 * NS ? count : 2 * NS;
    for (int i = 0; i < ahead; ++i) fetch_ids(i);
    wait_vmcnt<0>();
    const int begin = count < NS ? count : NS;
    for (int i = 0; i < begin; ++i) {
      const int64_t r = place(i, page_of(i));
      wave_sync_lds();
      fetch(i, r);
    }
  }
  for (int i = 0; i < count; ++i) {
    // Tile i is here when no more operations are under way than the tiles after it
    // have (page ids among them only make the wait longer).
    if (i + NS - 1 < count) wait_vmcnt<(NS - 1) * R::kOps>();
    else wait_vmcnt<0>();
    const int t = t0 + kWaves * i;
    uint8_t *kt = ring + (i % NS) * 2 * R::kHalf, *vt = kt + R::kHalf;

    // Everything of the tile that is read from LDS is on its way before the first product:
    // keys, values (transposed), exponents, page ids of this tile and of the next in its slot.
    u4 kx[U][F8 ? KS / 2 : KS];
#pragma unroll
    for (int g = 0; g < U; ++g) {
      const int k = 16 * g + col;
#pragma unroll
      for (int n = 0; n < (F8 ? KS / 2 : KS); ++n)
        kx[g][n] = *reinterpret_cast<const u4 *>(kt + k * R::kPitch +
                                                 16 * ((4 * n + kq) ^ kswap(k)));
    }
    const int page = page_of(i), next = i + NS < count ? i + NS : i;
    const int next_page = page_of(next);
    const uint32_t *ke = exps + (i % NS) * KT * 2, *ve = ke + KT;
    u4 kb[U], vb[U];
    if constexpr (F8)
#pragma unroll
      for (int g = 0; g < U; ++g) {
        kb[g] = *reinterpret_cast<const u4 *>(ke + 16 * g + 4 * kq);
        vb[g] = *reinterpret_cast<const u4 *>(ve + 16 * g + 4 * kq);
      }
    u2 vx[DP / 16];
    auto read_values = [&]() {
      // 16 bit: rows 4 kq .. + 3; 8 bit: of either group, the 8 keys of this lane's weights
      const int r = F8 ? col >> 1 : col >> 2, k = F8 ? 4 * kq + (r & 3) + 16 * (r >> 2) : 4 * kq + r;
      const uint8_t *vr = vt + k * R::kPitch + 8 * (col & 1);
#pragma unroll
      for (int d = 0; d < DP / 16; ++d) {
        if constexpr (F8) vx[d] = read_transposed8(vr + 16 * (d ^ vswap(k)));
        else
          vx[d] = __builtin_bit_cast(
              u2, read_transposed(vr + 16 * ((2 * d + ((col & 3) >> 1)) ^ vswap(k))));
      }
    };
    read_values();

    // scores, rows of keys x columns of query rows
    f4 s[CT][U];
#pragma unroll
    for (int g = 0; g < U; ++g)
#pragma unroll
      for (int c = 0; c < CT; ++c) s[c][g] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int n = 0; n < (F8 ? KS / 2 : KS); ++n)
#pragma unroll
      for (int g = 0; g < U; ++g) {
        const u4 x = kx[g][n];
        if constexpr (F8) {
          const v8 a = from_f8<QT>(u2{x[0], x[1]}), b = from_f8<QT>(u2{x[2], x[3]});
#pragma unroll
          for (int c = 0; c < CT; ++c) s[c][g] = H::mfma16(a, q[c][2 * n], s[c][g]);
#pragma unroll
          for (int c = 0; c < CT; ++c) s[c][g] = H::mfma16(b, q[c][2 * n + 1], s[c][g]);
        } else {
          const v8 a = __builtin_bit_cast(v8, x);
#pragma unroll
          for (int c = 0; c < CT; ++c) s[c][g] = H::mfma16(a, q[c][n], s[c][g]);
        }
      }
    const int64_t next_row = place(next, next_page);
    const uint64_t there = __ballot(page >= 0 && lane < KT), whole = (1ull << KT) - 1;
    const bool masked = (t + 1) * KT > plain || there != whole;

    // Where not every row sees all keys, keys that are not there become zeros, and
    // keys with a value that is not finite are kept apart, for the rows that do not see them.
    uint64_t bad = 0;
    if (masked) {
      if constexpr (F8) bad = __ballot(lane < KT && ve[klane] == 255u);
      for (int j = 0; j < R::kCopies; ++j) {
        u4 *at = reinterpret_cast<u4 *>(vt + 1024 * j + 16 * lane);
        u4 x = *at;
        if (!((there >> (R::kRows * j + crow)) & 1)) x = u4{};
        uint64_t w = __ballot(drop_nonfinite<QT, F8>(x));
        *at = x;
        while (w) {                               // rare
          const int n = __ffsll((long long)w) - 1;
          bad |= 1ull << (R::kRows * j + n / kPer);
          w &= w - 1;
        }
      }
      wave_sync_lds();
      read_values();
      // (byte 255 is no factor: rows that do not see the key are to have nothing of it)
      if constexpr (F8)
#pragma unroll
        for (int g = 0; g < U; ++g)
#pragma unroll
          for (int e = 0; e < 4; ++e) vb[g][e] = vb[g][e] == 255u ? 0u : vb[g][e];
    }

    // weights
    f4 vfac[U], vexp[U];
    if constexpr (F8) {
#pragma unroll
      for (int g = 0; g < U; ++g) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma unroll
          for (int c = 0; c < CT; ++c) s[c][g][e] *= __uint_as_float(kb[g][e] << 23);
          vfac[g][e] = __uint_as_float(vb[g][e] << 23);
          if constexpr (QT == kF16) vexp[g][e] = value_exponent(vb[g][e]);
        }
      }
    }
    u2 w[CT][U];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      if (masked) {
        const uint64_t see = (window(pl, u, row[c], tok[c], t * KT) & there) >> (4 * kq);
        const uint32_t is = (uint32_t)see, no = (uint32_t)(bad >> (4 * kq));
#pragma unroll
        for (int g = 0; g < U; ++g)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float x = s[c][g][e];
            x = (no >> (16 * g + e)) & 1 ? __builtin_nanf("") : x;
            s[c][g][e] = (is >> (16 * g + e)) & 1 ? x : -__builtin_huge_valf();
          }
      }
      float top = -3e38f;
#pragma unroll
      for (int g = 0; g < U; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float x = s[c][g][e];
          if constexpr (F8 && QT == kF16) x = fmaf(x, c2, vexp[g][e]);
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
          for (int e = 0; e < 4; ++e) acc[c][d][e] *= a;
      }
      const float ref = m[c] - H::kBias;
      float sum = 0.f;
#pragma unroll
      for (int g = 0; g < U; ++g) {
        uint16_t r[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float x = exp2_hw(fmaf(s[c][g][e], c2, -ref));
          sum += x;
          if constexpr (F8) x *= vfac[g][e];
          r[e] = __builtin_bit_cast(uint16_t, H::round(x));
        }
        w[c][g] = u2{r[0] | (uint32_t)r[1] << 16, r[2] | (uint32_t)r[3] << 16};
      }
      l[c] += sum;
    }

    // O^T += V^T P^T
#pragma unroll
    for (int d = 0; d < DP / 16; ++d) {
      if constexpr (F8) {
        const v8 x = from_f8<QT>(vx[d]);
#pragma unroll
        for (int c = 0; c < CT; ++c)
          acc[c][d] = H::mfma16(
              x, __builtin_bit_cast(v8, u4{w[c][0][0], w[c][0][1], w[c][1][0], w[c][1][1]}),
              acc[c][d]);
      } else {
#pragma unroll
        for (int c = 0; c < CT; ++c) acc[c][d] = H::mfma16_half(vx[d], w[c][0], acc[c][d]);
      }
    }
    // the slot is free
    if (i + 2 * NS < count) fetch_ids(i + 2 * NS);
    if (i + NS < count) fetch(i + NS, next_row);
  }

  // the four waves' sums: rows of a wave [16 CT][DP + 4], statistics
  constexpr int RW = 16 * CT, OS = DP + 4;
  float *o = reinterpret_cast<float *>(lds), *ml = o + (size_t)kWaves * RW * OS;
  __syncthreads();
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    l[c] += __shfl_xor(l[c], 16, kWaveSize);
    l[c] += __shfl_xor(l[c], 32, kWaveSize);
    if (kq == 0) {
      ml[(wid * RW + 16 * c + col) * 2] = m[c];
      ml[(wid * RW + 16 * c + col) * 2 + 1] = l[c];
    }
#pragma unroll
    for (int d = 0; d < DP / 16; ++d)
      *reinterpret_cast<f4 *>(o + (size_t)(wid * RW + 16 * c + col) * OS + 16 * d + 4 * kq) =
          acc[c][d];
  }
  __syncthreads();
  for (int e = tid; e < RW * (DP / 4); e += kThreads) {
    const int r = e / (DP / 4), d = (e - r * (DP / 4)) * 4;
    if (u.row0 + r >= u.rows || d >= D) continue;
    float top = -3e38f, sum = 0.f;
#pragma unroll
    for (int n = 0; n < kWaves; ++n) top = fmaxf(top, ml[(n * RW + r) * 2]);
    f4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int n = 0; n < kWaves; ++n) {
      const float a = exp2_hw(ml[(n * RW + r) * 2] - top);
      sum += ml[(n * RW + r) * 2 + 1] * a;
      const f4 y = *reinterpret_cast<const f4 *>(o + (size_t)(n * RW + r) * OS + d);
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] += y[k] * a;
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
  return ct == 1 ? dresd_attend_wave<QT, F8, DP, 1> : dresd_attend_wave<QT, F8, DP, 2>;
}

}  // namespace

#define DRESD_CAT2(a, b) a##b
#define DRESD_CAT(a, b) DRESD_CAT2(a, b)
AttendKernel DRESD_CAT(attend_wave_kernel_, DRESD_ATTEND_DP)(int qt, bool f8, int ct) {
  if (qt == kF16) return f8 ? pick<kF16, true>(ct) : pick<kF16, false>(ct);
  return f8 ? pick<kBF16, true>(ct) : pick<kBF16, false>(ct);
}

size_t DRESD_CAT(attend_wave_lds_, DRESD_ATTEND_DP)(bool f8, int ct) {
  const size_t a = (size_t)kWaves * (f8 ? Ring<true, DRESD_ATTEND_DP>::kBytes
                                        : Ring<false, DRESD_ATTEND_DP>::kBytes);
  const size_t b = end_bytes(DRESD_ATTEND_DP, ct);
  return a > b ? a : b;
}

}  // namespace dresd
