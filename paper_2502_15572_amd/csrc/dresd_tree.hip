// gfx950 prefix tree of drafts, and acceptance of its path by the model's own
// tokens (batch verification, DReSD Section 3.6).
//
// Tree.  Draft i has len_i tokens before its first EOS (none if it does not
// start with the next token).  With lcp(i, j) the common prefix of two drafts,
//   seen_i = max(1, max_{j < i} lcp(i, j))   prefix that earlier drafts have
//   base_i = 1 + sum_{j < i} max(0, len_j - seen_j)
// draft i's new nodes are its positions p = seen_i .. len_i - 1, numbered base_i +
// p - seen_i: a run, whose first node hangs on the node of position seen_i - 1
// in the first draft j that has that prefix (it is one of j's own: were it
// shared with an earlier draft, that one would have it first).  So a node's
// ancestors are runs of consecutive numbers, and its bits are written a run at a
// time.  What bounds it is latency, and for wide trees the bits: B N W words.  One
// workgroup per query; the drafts in LDS; the pairs of drafts spread evenly over
// the threads, four tokens compared at once; a lane per word of the bits, so that
// rows are written whole (a thread per node wrote 8 bytes a row apart).
//
// Acceptance.  From node 0, the arg max of the node's logits names the child
// to go on to.  Only the path's rows are read, and with each row's last bytes the first of
// the row of its lowest child (the best draft's): its path needs no wait for them, another one
// has them read in vain.  One workgroup per query: what bounds it is what one compute unit
// reads (some 60 GB/s) and 1.8 us a node between rows (8 nodes with rows of 10 KB 15 us, of 250 KB
// 32, for 64 queries 42; without the rows ahead, with 1,024 threads, which were in each
// other's way, and fmaxf 28, 48 and 54).  More units a query would have to wait for one another
// at every node.  A lane keeps the largest of its 16 bytes and which they were; the element
// among them is looked up at the end.
#include <algorithm>

#include "dresd_device.h"
#include "dresd_verify.h"

namespace dresd {

namespace {

constexpr int kTreeThreads = 1024;
constexpr int kTreeStage = 12288;    // tokens staged in LDS (rows of a multiple of four)
constexpr int kDraftsMax = DRESD_K_MAX_INTERNAL;

typedef int32_t i4 __attribute__((ext_vector_type(4)));

template <bool STAGED>
__global__ void __launch_bounds__(kTreeThreads) dresd_tree(TreeParams p) {
  extern __shared__ __align__(16) int32_t stage[];
  __shared__ uint32_t len[kDraftsMax];       // tokens of each draft
  __shared__ uint32_t best[kDraftsMax];      // longest earlier prefix | ~first draft that has it
  __shared__ uint32_t base[kDraftsMax];      // first new node
  __shared__ uint32_t run[kNodesMax];        // a node's run: its first node | what that hangs on
  __shared__ uint16_t owner[kNodesMax];      // and the draft that it is new in
  __shared__ uint32_t wsum[kTreeThreads / kWaveSize];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  const int r = p.r, N = p.N;
  // a node of depth p has a number of at least p: later tokens cannot get one
  const int length = p.length < N ? p.length : N, pitch = (length + 3) & ~3;
  const int32_t *src = p.drafts + (size_t)b * r * p.length;
  const int32_t first = p.next_tok[b];
  int cnt = p.count[b];
  cnt = cnt < 0 ? 0 : cnt > r ? r : cnt;
  if (tid < r) {
    len[tid] = tid < cnt ? (uint32_t)length : 0u;
    best[tid] = 0;
  }
  if (tid == 0) run[0] = 0;
  __syncthreads();

  // 1. lengths; the drafts into LDS
  const int di = kTreeThreads / length, dc = kTreeThreads - di * length;
  for (int i = tid / length, c = tid - i * length; i < cnt; i += di, c += dc) {
    if (c >= length) {
      c -= length;
      ++i;
      if (i >= cnt) break;
    }
    const int32_t x = src[(size_t)i * p.length + c];
    if constexpr (STAGED) stage[i * pitch + c] = x;
    if (c == 0 && x != first) atomicMin(&len[i], 0u);
    else if (x == p.eos) atomicMin(&len[i], (uint32_t)c);
  }
  __syncthreads();
  auto token = [&](int i, int j) -> int32_t {
    if constexpr (STAGED) return stage[i * pitch + j];
    else return src[(size_t)i * p.length + j];
  };

  // 2. longest prefix that an earlier draft has, and the first draft that has it
  for (int e = tid; e < cnt * (cnt - 1) / 2; e += kTreeThreads) {
    // pair e: draft i after the i (i - 1) / 2 pairs of those before
    int i = (int)((1.f + sqrtf(1.f + 8.f * (float)e)) * 0.5f);
    while (i * (i - 1) / 2 > e) --i;
    while (i * (i + 1) / 2 <= e) ++i;
    const int j = e - i * (i - 1) / 2;
    const int m = (int)(len[i] < len[j] ? len[i] : len[j]);
    int c = 0;
    bool same = true;
    while (same && c < m) {
      if constexpr (STAGED) {                // (what a row's pitch adds ends past m)
        const i4 x = *reinterpret_cast<const i4 *>(stage + i * pitch + c);
        const i4 y = *reinterpret_cast<const i4 *>(stage + j * pitch + c);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          same = same && x[k] == y[k];
          c += same;
        }
      } else {
        same = token(i, c) == token(j, c);
        c += same;
      }
    }
    c = c < m ? c : m;
    if (c > 0) atomicMax(&best[i], ((uint32_t)c << 16) | (0xffffu - (uint32_t)j));
  }
  __syncthreads();

  // 3. number of each draft's first new node: workgroup prefix sum
  const int shared = tid < r && best[tid] ? (int)(best[tid] >> 16) : 1;
  const int own = tid < r ? (int)len[tid] : 0;
  const uint32_t fresh = own > shared ? (uint32_t)(own - shared) : 0u;
  uint32_t x = fresh;
#pragma unroll
  for (int o = 1; o < kWaveSize; o <<= 1) {
    const uint32_t y = __shfl_up(x, o, kWaveSize);
    if (lane >= o) x += y;
  }
  if (lane == kWaveSize - 1) wsum[wid] = x;
  __syncthreads();
  uint32_t before = 1, total = 1;
#pragma unroll
  for (int w = 0; w < kTreeThreads / kWaveSize; ++w) {
    const uint32_t c = wsum[w];
    if (w < wid) before += c;
    total += c;
  }
  if (tid < r) base[tid] = before + x - fresh;
  __syncthreads();
  const int nodes = total < (uint32_t)N ? (int)total : N;

  // 4. the new nodes' tokens, parents and depths; threads T i .. T i + T - 1 share draft i
  int T = 1;
  while (T < kWaveSize && r * 2 * T <= kTreeThreads) T <<= 1;
  int32_t *tok = p.token + (size_t)b * N, *par = p.parent + (size_t)b * N,
          *dep = p.depth + (size_t)b * N;
  const int i = tid / T, sub = tid & (T - 1);
  if (i < cnt) {
    const uint32_t k = best[i], at = base[i];
    const int s = k ? (int)(k >> 16) : 1, n = (int)len[i] - s;
    int hang = 0;
    if (s > 1) {
      const int j = (int)(0xffffu - (k & 0xffffu));
      hang = (int)base[j] + s - 1 - (best[j] ? (int)(best[j] >> 16) : 1);
    }
    for (int e = sub; e < n && at + e < (uint32_t)N; e += T) {
      run[at + e] = (at << 16) | (uint32_t)hang;
      owner[at + e] = (uint16_t)i;
      tok[at + e] = token(i, s + e);
      par[at + e] = e == 0 ? hang : (int)at + e - 1;
      dep[at + e] = s + e;
    }
  }
  if (tid == 0) {
    tok[0] = first;
    par[0] = -1;
    dep[0] = 0;
    p.nodes[b] = nodes;
  }
  for (int u = nodes + tid; u < N; u += kTreeThreads) {
    tok[u] = p.eos;
    par[u] = -1;
    dep[u] = 0;
  }
  __syncthreads();

  // 5. ancestors, a lane per word: of each draft's first new node into LDS, by its runs, highest
  //    first; its new nodes add their own run to them
  const int W = (N + 63) / 64;
  uint64_t *rows = p.mask + (size_t)b * N * W;
  auto bits_of = [](int lo, int hi, int w0) -> uint64_t {  // lo .. hi, in the word from w0
    const int from = lo > w0 ? lo - w0 : 0, to = hi < w0 + 63 ? hi - w0 : 63;
    return from <= to ? (~0ull >> (63 - (to - from))) << from : 0ull;
  };
  const int du = kTreeThreads / W, dw = kTreeThreads - du * W;
  uint64_t *above = reinterpret_cast<uint64_t *>(stage);   // (the drafts are read no more)
  for (int i = tid / W, w = tid - i * W; i <= cnt; i += du, w += dw) {
    if (w >= W) {
      w -= W;
      ++i;
      if (i > cnt) break;
    }
    // (past the last draft: node 0)
    const int u = i < cnt ? (int)base[i] : 0;
    if (u >= nodes) continue;
    uint64_t bits = 0;
    int hi = u;                              // top of the run at hand
    while (hi >= 64 * w) {
      const uint32_t k = run[hi];
      bits |= bits_of((int)(k >> 16), hi, 64 * w);
      hi = hi > 0 ? (int)(k & 0xffffu) : -1;
    }
    // (a draft without new nodes writes what the next one that has some does)
    if (i < cnt) above[(size_t)i * W + w] = bits;
    else rows[w] = bits;
  }
  __syncthreads();
  for (int u = tid / W, w = tid - u * W; u < N; u += du, w += dw) {
    if (w >= W) {
      w -= W;
      ++u;
      if (u >= N) break;
    }
    if (u == 0) continue;
    rows[(size_t)u * W + w] =
        u < nodes ? above[(size_t)owner[u] * W + w] | bits_of((int)(run[u] >> 16), u, 64 * w) : 0ull;
  }
}

constexpr int kAcceptThreads = 512;
constexpr int kAcceptWaves = kAcceptThreads / kWaveSize;

// The largest of three, one instruction.  fmaxf adds one for each operand that may be a signalling
// NaN, which IEEE mode would let through; without that mode it counts as a quiet one does.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm volatile("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
__device__ __forceinline__ void leave_ieee_mode() {
  __builtin_amdgcn_s_setreg(1 | 9 << 6, 0);  // register MODE, bit 9, one bit
}

template <int DT>
struct Logits;
template <>
struct Logits<kF32> {
  static constexpr int kPer = 4;             // elements of 16 bytes
  typedef float Raw;
  static __device__ __forceinline__ float value(Raw x) { return x; }
  static __device__ __forceinline__ float get(u4 x, int e) { return __uint_as_float(x[e]); }
};
template <>
struct Logits<kF16> {
  static constexpr int kPer = 8;
  typedef _Float16 Raw;
  static __device__ __forceinline__ float value(Raw x) { return (float)x; }
  static __device__ __forceinline__ float get(u4 x, int e) {
    return (float)__builtin_bit_cast(h8, x)[e];
  }
};
template <>
struct Logits<kBF16> {
  static constexpr int kPer = 8;
  typedef uint16_t Raw;
  static __device__ __forceinline__ float value(Raw x) {
    return __uint_as_float((uint32_t)x << 16);
  }
  static __device__ __forceinline__ float get(u4 x, int e) {
    return __uint_as_float(e & 1 ? x[e / 2] & 0xffff0000u : x[e / 2] << 16);
  }
};

// The largest of 16 bytes, NaNs left out (NaN if there is nothing else; outside IEEE mode).
template <int DT>
__device__ __forceinline__ float largest(u4 x) {
  typedef Logits<DT> X;
  float m;
  if constexpr (DT == kF32) {
    m = max3(X::get(x, 0), X::get(x, 1), X::get(x, 2));
    m = max3(m, X::get(x, 3), m);
  } else {
    m = max3(X::get(x, 0), X::get(x, 1), X::get(x, 2));
    m = max3(m, X::get(x, 3), X::get(x, 4));
    m = max3(m, X::get(x, 5), X::get(x, 6));
    m = max3(m, X::get(x, 7), m);
  }
  return m;
}

// The largest of a wave's numbers, for every lane.
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  auto with = [&](uint32_t y) { x = x > y ? x : y; };
  with(__builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));  // 1, 2, 4, 8 lanes on in the row
  with(__builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
  with(__builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
  with(__builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
  with(__builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));  // row 0 to 1, 2 to 3
  with(__builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));  // rows 0 and 1 to 2 and 3
  return __builtin_amdgcn_readlane(x, 63);
}

// The largest of a wave's logits (as order bits) and the lowest place that has it.
__device__ __forceinline__ void wave_best(uint32_t &x, uint32_t &at) {
  const uint32_t top = wave_max(x);
  at = ~wave_max(x == top ? ~at : 0u);
  x = top;
}

template <int DT>
__global__ void __launch_bounds__(kAcceptThreads) dresd_accept(AcceptParams p) {
  typedef Logits<DT> X;
  constexpr int E = X::kPer, kElem = 16 / E, kRing = 8;
  __shared__ uint32_t wtop[kAcceptWaves], wat[kAcceptWaves];
  __shared__ int32_t tok[kNodesMax], par[kNodesMax];
  __shared__ uint32_t heir[kNodesMax];       // lowest child
  __shared__ uint32_t lowest;
  __shared__ int32_t now[2];                 // the next node, the present one's token (-1: not known)
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  int nodes = p.nodes[b];
  nodes = nodes < 0 ? 0 : nodes > p.N ? p.N : nodes;
  leave_ieee_mode();

  // A row: up to the first whole 16 bytes, 16 bytes at a time, the rest.
  struct Row {
    const uint8_t *src, *vec;
    int head, body, tail;
  };
  auto row_of = [&](int node) -> Row {
    Row w;
    w.src = static_cast<const uint8_t *>(p.logits) + ((int64_t)b * p.N + node) * p.row * kElem;
    w.head = (int)((16 - ((uintptr_t)w.src & 15)) & 15) / kElem;
    w.head = w.head < p.V ? w.head : p.V;
    w.vec = w.src + w.head * kElem;
    w.body = (p.V - w.head) / E;
    w.tail = p.V - w.head - w.body * E;
    return w;
  };
  // this thread's element before or past the row's whole 16 bytes (if any, else the first), ...
  auto edge_at = [&](const Row &w) -> int {
    return tid < w.head ? tid : tid >= 64 && tid < 64 + w.tail ? p.V - w.tail + tid - 64 : -1;
  };
  typename X::Raw edge = 0;
  auto load_edge = [&](const Row &w) -> typename X::Raw {
    const int e = edge_at(w);
    return reinterpret_cast<const typename X::Raw *>(w.src)[e < 0 ? 0 : e];
  };
  // ... and its 16 bytes of those from `at` on (past the last those again)
  u4 v[kRing];
  auto load = [&](const uint8_t *vec, uint32_t at, uint32_t last) -> u4 {
    at += (uint32_t)tid * 16;
    return *reinterpret_cast<const u4 *>(vec + (at < last ? at : last));
  };

  Row w = row_of(0);
  bool ready = false;                        // whether the row's first 16 bytes are on their way
  if (nodes > 0 && w.body > 0) {
    edge = load_edge(w);
#pragma unroll
    for (int k = 0; k < kRing; ++k)
      v[k] = load(w.vec, k * kAcceptThreads * 16, (uint32_t)(w.body - 1) * 16);
    ready = true;
  }
  for (int c = tid; c < nodes; c += kAcceptThreads) {
    tok[c] = p.token[(size_t)b * p.N + c];
    par[c] = p.parent[(size_t)b * p.N + c];
    heir[c] = ~0u;
  }
  __syncthreads();
  for (int c = tid; c < nodes; c += kAcceptThreads)
    if (par[c] >= 0 && par[c] < c) atomicMin(&heir[par[c]], (uint32_t)c);
  __syncthreads();
  int u = nodes > 0 ? 0 : -1, done = 0;
  int32_t g = -1;
  while (u >= 0) {
    if (!ready) {
      edge = load_edge(w);
      if (w.body > 0)
#pragma unroll
        for (int k = 0; k < kRing; ++k)
          v[k] = load(w.vec, k * kAcceptThreads * 16, (uint32_t)(w.body - 1) * 16);
    }
    if (tid == 0) p.path[(size_t)b * p.most + done] = u;
    ++done;
    // the row that is read next, if its path is that of the lowest children
    const int guess = __builtin_amdgcn_readfirstlane(done < p.most ? (int)heir[u] : -1);
    const Row next = row_of(guess < 0 ? u : guess);
    const typename X::Raw mine = edge;
    float best = -__builtin_huge_valf();
    int which = -1;                          // of this thread's 16 bytes
    for (int r = 0; r < w.body; r += kRing * kAcceptThreads) {
      const bool end = r + kRing * kAcceptThreads >= w.body;
      // (nothing to guess, or a row without whole 16 bytes: this row's first bytes again)
      const bool ahead = end && guess >= 0 && next.body > 0;
      const uint8_t *from = ahead ? next.vec : w.vec;
      const uint32_t at = end ? 0u : (uint32_t)(r + kRing * kAcceptThreads) * 16;
      const uint32_t last = ahead  ? (uint32_t)(next.body - 1) * 16
                            : !end ? (uint32_t)(w.body - 1) * 16
                                   : 0u;
      if (end) edge = load_edge(next);
#pragma unroll
      for (int k = 0; k < kRing; ++k) {
        if (r + k * kAcceptThreads < w.body) {
          const float m = largest<DT>(v[k]);
          const bool up = m > best;
          best = up ? m : best;
          which = up ? r / kAcceptThreads + k : which;
        }
        v[k] = load(from, at + k * kAcceptThreads * 16, last);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    int where = p.V;                         // element at which the best 16 bytes begin
    if (which >= 0) {
      const int c = which * kAcceptThreads + tid;
      where = w.head + (c < w.body ? c : w.body - 1) * E;
    }
    const int e = edge_at(w);
    const float own = X::value(mine);
    if (e >= 0 && (own > best || (own == best && e < where && where < p.V))) {
      best = own;
      where = e;
    }
    uint32_t top = order_bits(best), first = (uint32_t)where;
    wave_best(top, first);
    if (lane == 0) {
      wtop[tid >> 6] = top;
      wat[tid >> 6] = first;
    }
    // the lowest child with a token; children have higher numbers
    auto child = [&](int32_t token) -> int {
      if (done < p.most)
        for (int c0 = u + 1; c0 < nodes; c0 += kWaveSize) {
          const int c = c0 + lane;
          const uint64_t hit = __ballot(c < nodes && par[c] == u && tok[c] == token);
          if (hit) return c0 + __ffsll((long long)hit) - 1;
        }
      return -1;
    };
    __syncthreads();
    if (tid < kWaveSize) {                   // (one wave: they would only be in each other's way)
      top = wtop[lane % kAcceptWaves];
      first = wat[lane % kAcceptWaves];
      wave_best(top, first);
      int32_t is = __builtin_amdgcn_readfirstlane((int)first);
      if (is >= w.head && is < p.V - w.tail) {
        // the first of the 16 bytes' elements that has the value (a scalar load, which does not
        // wait for those under way)
        typedef const __attribute__((address_space(4))) u4 cu4;
        const u4 x = *(cu4 *)(uintptr_t)(w.src + (int64_t)is * kElem);
        const float most = order_value(top);
        int e0 = 0;
#pragma unroll
        for (int e = E - 1; e >= 0; --e) e0 = X::get(x, e) == most ? e : e0;
        is += __builtin_amdgcn_readfirstlane(e0);
      }
      const int to = is < p.V ? child(is) : -1;
      if (lane == 0) {
        now[0] = to;
        now[1] = is < p.V ? is : -1;
        lowest = p.V;
      }
    }
    __syncthreads();
    int to = __builtin_amdgcn_readfirstlane(now[0]);
    g = __builtin_amdgcn_readfirstlane(now[1]);
    if (g < 0) {                             // nothing above -inf: the first -inf, else (NaN alone) 0
      uint32_t low = p.V;
      for (int e = tid; e < p.V && low == (uint32_t)p.V; e += kAcceptThreads)
        if (X::value(reinterpret_cast<const typename X::Raw *>(w.src)[e]) == -__builtin_huge_valf())
          low = e;
      if (low < (uint32_t)p.V) atomicMin(&lowest, low);
      __syncthreads();
      g = lowest < (uint32_t)p.V ? (int)lowest : 0;
      to = child(g);
      __syncthreads();
    }
    u = to;
    ready = u >= 0 && u == guess && w.body > 0 && next.body > 0;
    if (u >= 0) w = u == guess ? next : row_of(u);
  }
  for (int e = done + tid; e < p.most; e += kAcceptThreads) p.path[(size_t)b * p.most + e] = -1;
  if (tid == 0) {
    p.accepted[b] = done;
    p.next_tok[b] = g;
  }
}

}  // namespace

hipError_t launch_draft_tree(const TreeParams &p, hipStream_t st) {
  if (p.B == 0) return hipSuccess;
  TreeParams q = p;
  void *args[] = {&q};
  const int64_t tokens = (int64_t)p.r * (((p.length < p.N ? p.length : p.N) + 3) & ~3);
  const bool staged = tokens <= kTreeStage;
  // LDS: the drafts, then the bits above each one's new nodes (at most 128 KiB)
  const size_t lds = std::max(staged ? (size_t)tokens * 4 : 0, (size_t)p.r * ((p.N + 63) / 64) * 8);
  return hipLaunchKernel(staged ? (const void *)dresd_tree<true> : (const void *)dresd_tree<false>,
                         dim3((unsigned)p.B), dim3(kTreeThreads), args, lds, st);
}

hipError_t launch_accept(const AcceptParams &p, hipStream_t st) {
  if (p.B == 0) return hipSuccess;
  AcceptParams q = p;
  void *args[] = {&q};
  const void *k = p.dtype == kF32   ? (const void *)dresd_accept<kF32>
                  : p.dtype == kF16 ? (const void *)dresd_accept<kF16>
                                    : (const void *)dresd_accept<kBF16>;
  return hipLaunchKernel(k, dim3((unsigned)p.B), dim3(kAcceptThreads), args, 0, st);
}

}  // namespace dresd
