// gfx950 attention of many rows over a paged cache: 128 rows (tokens times query
// heads of one cache head) a workgroup, 32 a wave.
//
// What bounds it is the matrix cores, and beside them the exponentials: 128 rows do 128
// multiply-adds per 16-bit value read (busy 46% and 45% of the time, LDS 27%: a wave's products
// and exponentials follow one another, and two waves a SIMD overlap theirs).  The four waves
// share each tile of 64 keys and values through LDS, two tiles deep: while one is computed the
// next is copied to the other buffer (8-bit rows through registers, where they are converted,
// once for all four waves), and a tile has one barrier.  A chunk of 2,048 tokens over 16,000 and
// two shorter ones (8 x 4 heads of 128, bf16): 1.16 to 1.22 ms by card, 910 to 960 TFLOP/s,
// where a 16,384^3 product of the library reaches 1,374; rows through registers took 0.13 ms
// more.
//
// Scores are formed transposed, S^T = K Q^T, with 32 x 32 x 16 instructions: a lane
// holds one row (lane % 32) and half the keys, which is, keys in another order, the
// operand of O^T = V^T P^T.  The weights never leave their registers, and a row's
// statistics and rescaling are those of two lanes.  Keys are stored so that the 16
// bytes that 16 lanes read at once lie in different banks, values so that the
// transposed reads of 4 keys by 32 dims do.
//
// Running softmax: as in the wave kernel, a row's reference moves only when a score
// passes it by kSlack.
#include <type_traits>

#include "dresd_attend.h"

namespace dresd {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = 4;
constexpr int kKeys = 64;

// Of each wave: row offsets [keys] i64, factors of keys and values, and the values' exponents as
// a row's maximum takes them, [keys] f32 each.
constexpr size_t kWaveBytes = kKeys * 20;
// Whether a key of the tile has a value that is not finite, two tiles.
constexpr size_t kFlagBytes = 2 * kKeys;
constexpr size_t tile_bytes(int dp) { return (size_t)kKeys * dp * 2; }

template <int QT, bool F8, int DP>
__global__ void __launch_bounds__(kThreads, DP <= 128 ? 2 : 1) dresd_attend_tile(AttendPlan pl) {
  typedef Half<QT> H;
  typedef typename H::v8 v8;
  typedef short s8v __attribute__((ext_vector_type(8)));
  constexpr int KS = DP / 16;                     // 16-dim steps
  constexpr int LR = F8 ? DP / 16 : DP / 8;       // lanes of a row in a load
  constexpr int RP = kThreads / LR;               // rows of a load
  constexpr int NP = kKeys / RP;                  // loads of a tile
  // Addresses of values in LDS are formed anew for each tile where the compiler, which would
  // keep them all, runs out of registers (3 sequences of 16,000 tokens and 2,048 new ones, 8 x 4
  // heads of 256: 8 bits 4.2 ms against 5.7, 16 bits 3.3 against 3.2 to 4.2).
  constexpr bool kAnew = DP == 256;
  extern __shared__ __align__(16) uint8_t lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  Unit u;
  if (!unit_of(pl, u)) return;
  const AttendParams &p = pl.p;
  const int D = p.c.dim;

  uint8_t *kt = lds, *vt = lds + 2 * tile_bytes(DP);
  uint8_t *mine = lds + 4 * tile_bytes(DP) + (size_t)wid * kWaveBytes;
  int64_t *offs = reinterpret_cast<int64_t *>(mine);
  float *kf = reinterpret_cast<float *>(offs + kKeys), *vf = kf + kKeys, *va = vf + kKeys;
  uint8_t *flags = lds + 4 * tile_bytes(DP) + kWaves * kWaveBytes;

  // queries: operand of row 32 wid + col
  v8 q[KS];
  const float c2 = score_factor(p.scale);
  int r = u.row0 + 32 * wid + col;
  const bool real = r < u.rows;
  r = real ? r : u.rows - 1;
  const int tok = r / pl.group;
  const int64_t row = u.token0 + tok;
  const int head = u.head * pl.group + (r - tok * pl.group);
  {
    const uint32_t flip = p.scale < 0.f ? 0x80008000u : 0u;  // (-q) . k |scale|
    const uint16_t *src = static_cast<const uint16_t *>(p.q) + row * p.q_row + head * p.q_head;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int d = 16 * s + 8 * half;
      u4 x = {};
      if (d < D) x = *reinterpret_cast<const u4 *>(src + d);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] ^= flip;
      q[s] = __builtin_bit_cast(v8, x);
    }
  }
  f16v acc[DP / 32];
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;
  float m = -3e38f, l = 0.f;

  // A wave without rows of its own takes part in the copies alone, and leaves the LDS to the others
  // (trees of 91 nodes, 32 heads: 109 -> 104 us).
  const bool works = u.row0 + 32 * wid < u.rows;

  // this split's tiles
  const int end = reach(pl, u, pl.rows);
  const int tiles = end > 0 ? (end + kKeys - 1) / kKeys : 0;
  const int per = (tiles + pl.splits - 1) / pl.splits;
  const int64_t lo = (int64_t)u.split * per;
  const int first = lo < tiles ? (int)lo : tiles;
  const int last = first + per < tiles ? first + per : tiles;
  const int plain = seen_by_all(pl, u);

  const uint8_t *kbase = static_cast<const uint8_t *>(p.c.k);
  const uint8_t *vbase = static_cast<const uint8_t *>(p.c.v);
  const int row_bytes = F8 ? D : 2 * D;
  const int32_t *table = p.table + (int64_t)u.b * p.width;
  const int in_page = (1 << p.c.page_log) - 1;

  // page of key `lane` of a tile
  auto page_of = [&](int t) -> int {
    if (t >= last) return -1;
    const int pos = t * kKeys + lane;
    return pos < u.L ? table[pos >> p.c.page_log] : -1;
  };
  // offsets of a tile's rows into the wave's LDS; which of its keys there are
  uint32_t ke = 0, ve = 0;                        // their exponents
  auto place = [&](int t, int page) -> uint64_t {
    const bool ok = (uint32_t)page < (uint32_t)p.c.pages;
    const int64_t at = ok ? ((((int64_t)page * p.c.heads + u.head) << p.c.page_log) +
                             ((t * kKeys + lane) & in_page))
                          : 0;
    offs[lane] = at * row_bytes;
    if constexpr (F8) {
      ke = ok ? p.c.k_exp[at] : 127u;
      ve = ok ? p.c.v_exp[at] : 127u;
    }
    wave_sync_lds();
    return __ballot(ok);
  };

  // 8-bit rows come through registers, where they are converted, 16-bit rows straight to LDS.
  u4 kr[F8 ? NP : 1], vr[F8 ? NP : 1];
  const int sl = tid % LR, sr = tid / LR;         // 16 bytes of a row, row within a load
  const int sd = 16 * sl < row_bytes ? 16 * sl : 0;  // (dims past the head: as in the wave kernel)
  [[maybe_unused]] auto load16 = [&](const uint8_t *src) -> u4 {
    if (F8 && (D & 8)) {                          // rows are 8-byte aligned
      const u2 a = *reinterpret_cast<const u2 *>(src + sd);
      const u2 b = *reinterpret_cast<const u2 *>(src + (sd + 8 < row_bytes ? sd + 8 : sd));
      return u4{a[0], a[1], b[0], b[1]};
    }
    return *reinterpret_cast<const u4 *>(src + sd);
  };
  auto kswap = [](int k) -> int { return k & (DP == 64 ? 7 : 15); };
  auto vswap = [](int k) -> int { return (DP == 64 ? (k >> 1) & 1 : k & 3) << 2; };
  auto kchunk = [&](auto buf, int k, int c) -> uint8_t * {
    return kt + buf * tile_bytes(DP) + ((size_t)k * (DP / 8) + (c ^ kswap(k))) * 16;
  };
  auto vchunk = [&](auto buf, int k, int c) -> uint8_t * {
    return vt + buf * tile_bytes(DP) + ((size_t)k * (DP / 8) + (c ^ vswap(k))) * 16;
  };
  // what this lane copies of a row of keys and of values, in its place after the exchange of
  // chunks (dims past the head: as in the wave kernel)
  int kat[F8 ? 1 : NP], vat[F8 ? 1 : NP];
  const uint32_t kt_at = lds_address(kt), vt_at = lds_address(vt);
  if constexpr (!F8) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int k = RP * i + sr;
      kat[i] = 16 * (sl ^ kswap(k)) < row_bytes ? 16 * (sl ^ kswap(k)) : 0;
      vat[i] = 16 * (sl ^ vswap(k)) < row_bytes ? 16 * (sl ^ vswap(k)) : 0;
    }
  }
  // a tile on its way: to registers, or to LDS
  auto load = [&](auto buf) {
    int64_t o[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) o[i] = offs[RP * i + sr];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      if constexpr (F8) {
        kr[i] = load16(kbase + o[i]);
        vr[i] = load16(vbase + o[i]);
      } else {
        // rows RP i + 64 / LR wid .. of the tile
        const uint32_t at = buf * (uint32_t)tile_bytes(DP) + (4 * i + wid) * 1024;
        copy16_from(kbase + o[i] + kat[i], kt_at + at);
        copy16_from(vbase + o[i] + vat[i], vt_at + at);
      }
    }
  };
  // a tile that has arrived into its buffer; where not every row sees all of its keys, keys that
  // are not there as zeros, and values that are not finite apart
  auto store = [&](auto buf, bool masked, uint64_t ok) {
    if constexpr (!F8) wait_vmcnt<0>();
    if (masked) {
      const uint64_t there = ok >> sr, none = F8 ? __ballot(ve == 255u) >> sr : 0ull;
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        // (16 bit: what this lane has copied; 8 bit: in its registers)
        u4 *at = reinterpret_cast<u4 *>(vt + buf * tile_bytes(DP) + (4 * i + wid) * 1024 + lane * 16);
        u4 x;
        if constexpr (F8) x = vr[i];
        else x = *at;
        if (!((there >> (RP * i)) & 1)) x = u4{};
        const uint64_t w = __ballot(drop_nonfinite<QT, F8>(x)) >> (lane & ~(LR - 1));
        if constexpr (F8) vr[i] = x;
        else *at = x;
        if (sl == 0)
          flags[buf * kKeys + RP * i + sr] =
              (w & ((1ull << LR) - 1)) != 0 || ((none >> (RP * i)) & 1);
      }
    }
    if constexpr (F8) {
      int sl = tid % LR, sr = tid / LR;
      if constexpr (kAnew) asm volatile("" : "+v"(sl), "+v"(sr));
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int k = RP * i + sr;
        *reinterpret_cast<v8 *>(kchunk(buf, k, 2 * sl)) = from_f8<QT>(u2{kr[i][0], kr[i][1]});
        *reinterpret_cast<v8 *>(kchunk(buf, k, 2 * sl + 1)) = from_f8<QT>(u2{kr[i][2], kr[i][3]});
        *reinterpret_cast<v8 *>(vchunk(buf, k, 2 * sl)) = from_f8<QT>(u2{vr[i][0], vr[i][1]});
        *reinterpret_cast<v8 *>(vchunk(buf, k, 2 * sl + 1)) = from_f8<QT>(u2{vr[i][2], vr[i][3]});
      }
      kf[lane] = __uint_as_float(ke << 23);
      vf[lane] = value_factor(ve, masked);
      if constexpr (QT == kF16) va[lane] = value_exponent(ve);
    }
  };

  auto compute = [&](auto buf, int t, bool masked, uint64_t ok) {
    f16v s[2];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
    // (keys are read kAhead steps before their product, no further: registers)
    __builtin_amdgcn_s_setprio(1);
    constexpr int kAhead = 2;
    v8 kx[kAhead + 1][2];
#pragma unroll
    for (int i = 0; i < KS + kAhead; ++i) {
      if (i < KS)
#pragma unroll
        for (int b = 0; b < 2; ++b)
          kx[i % (kAhead + 1)][b] =
              *reinterpret_cast<const v8 *>(kchunk(buf, 32 * b + col, 2 * i + half));
      if (i >= kAhead)
#pragma unroll
        for (int b = 0; b < 2; ++b)
          s[b] = H::mfma32(kx[(i - kAhead) % (kAhead + 1)][b], q[i - kAhead], s[b]);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
    // key of element 4 j + i of block b: 32 b + 8 j + 4 half + i
    if constexpr (F8)
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f4 kfac = *reinterpret_cast<const f4 *>(kf + 32 * b + 8 * j + 4 * half);
#pragma unroll
          for (int i = 0; i < 4; ++i) s[b][4 * j + i] *= kfac[i];
        }
    if (masked) {
      const uint64_t see = (window(pl, u, row, tok, t * kKeys) & ok) >> (4 * half);
      const uint64_t bad = __ballot(flags[buf * kKeys + lane] != 0) >> (4 * half);
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const uint32_t is = (uint32_t)(see >> (32 * b)), no = (uint32_t)(bad >> (32 * b));
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int bit = 8 * (e / 4) + e % 4;
          float x = s[b][e];
          x = (no >> bit) & 1 ? __builtin_nanf("") : x;
          s[b][e] = (is >> bit) & 1 ? x : -__builtin_huge_valf();
        }
      }
    }
    float top = -3e38f;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        f4 vexp;
        if constexpr (F8 && QT == kF16)
          vexp = *reinterpret_cast<const f4 *>(va + 32 * b + 8 * j + 4 * half);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x = s[b][4 * j + i];
          if constexpr (F8 && QT == kF16) x = fmaf(x, c2, vexp[i]);
          top = fmaxf(top, x);
        }
      }
    if constexpr (!(F8 && QT == kF16)) top *= c2;  // (in powers of two)
    if (__any(top > m + H::kSlack)) {
      top = fmaxf(top, __shfl_xor(top, 32, kWaveSize));
      const float mn = fmaxf(m, top);
      const float a = exp2_hw(m - mn);
      m = mn;
      l *= a;
#pragma unroll
      for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] *= a;
    }
    const float ref = m - H::kBias;
    float sum = 0.f;
    v8 w[4];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k0 = 32 * b + 8 * j + 4 * half;
        f4 vfac;
        if constexpr (F8) vfac = *reinterpret_cast<const f4 *>(vf + k0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x = exp2_hw(fmaf(s[b][4 * j + i], c2, -ref));
          sum += x;
          if constexpr (F8) x *= vfac[i];
          w[2 * b + j / 2][4 * (j & 1) + i] = H::round(x);
        }
      }
    l += sum;
    int ln = lane;
    if constexpr (kAnew) asm volatile("" : "+v"(ln));
    const int g = (ln >> 4) & 1, i16 = ln & 15, in = (i16 & 1) * 8;
    __builtin_amdgcn_s_setprio(1);
    constexpr int kV = 4 * (DP / 32), kVAhead = 4;
    v8 vx[kVAhead + 1];
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < kV + kVAhead; ++i) {
      if (i < kV) {
        const int kk = i / (DP / 32), d = i % (DP / 32);
        const int k = 16 * kk + 4 * half + (i16 >> 2), c = 4 * d + 2 * g + ((i16 & 3) >> 1);
        const s4v a = read_transposed(vchunk(buf, k, c) + in);
        const s4v b = read_transposed(vchunk(buf, k + 8, c) + in);
        vx[i % (kVAhead + 1)] = __builtin_bit_cast(
            v8, s8v{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
      }
      if (i >= kVAhead) {
        const int j = i - kVAhead;
        acc[j % (DP / 32)] =
            H::mfma32(vx[j % (kVAhead + 1)], w[j / (DP / 32)], acc[j % (DP / 32)]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
  };

  if (first < last) {
    typedef std::integral_constant<int, 0> B0;
    typedef std::integral_constant<int, 1> B1;
    uint64_t ok = place(first, page_of(first));
    load(B0{});
    int page = page_of(first + 1);
    bool masked = (first + 1) * kKeys > plain || ok != ~0ull;
    store(B0{}, masked, ok);
    __syncthreads();
    auto step = [&](auto buf, int t) {
      typedef std::integral_constant<int, 1 - decltype(buf)::value> Other;
      const bool more = t + 1 < last;
      uint64_t next_ok = 0;
      bool next_masked = false;
      if (more) {
        next_ok = place(t + 1, page);
        load(Other{});
        page = page_of(t + 2);
        next_masked = (t + 2) * kKeys > plain || next_ok != ~0ull;
      }
      __builtin_amdgcn_sched_barrier(0);
      if (works) compute(buf, t, masked, ok);
      __builtin_amdgcn_sched_barrier(0);
      if (more) store(Other{}, next_masked, next_ok);
      __syncthreads();
      ok = next_ok;
      masked = next_masked;
    };
    for (int t = first; t < last; t += 2) {
      step(B0{}, t);
      if (t + 1 < last) step(B1{}, t + 1);
    }
  }

  l += __shfl_xor(l, 32, kWaveSize);
  if (!real) return;
  const int64_t out = row * p.q_heads + head;
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int dim = 32 * d + 8 * j + 4 * half;
      if (dim < D)
        store_row<QT>(pl, u.split, out, dim,
                      f4{acc[d][4 * j], acc[d][4 * j + 1], acc[d][4 * j + 2], acc[d][4 * j + 3]},
                      m - H::kBias, l);
    }
}

template <int QT, bool F8>
AttendKernel pick(int dp) {
  if (dp == 64) return dresd_attend_tile<QT, F8, 64>;
  if (dp == 128) return dresd_attend_tile<QT, F8, 128>;
  return dresd_attend_tile<QT, F8, 256>;
}

}  // namespace

AttendKernel attend_tile_kernel(int qt, bool f8, int dp) {
  if (qt == kF16) return f8 ? pick<kF16, true>(dp) : pick<kF16, false>(dp);
  return f8 ? pick<kBF16, true>(dp) : pick<kBF16, false>(dp);
}

size_t attend_tile_lds(int dp) { return 4 * tile_bytes(dp) + kWaves * kWaveBytes + kFlagBytes; }

}  // namespace dresd
