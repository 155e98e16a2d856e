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
// to go on to.  Only the path's rows are read.  One workgroup per query: what
// bounds it is one compute unit's reading (about 100 GB/s) and some 2 us of latency
// a node.  A lane keeps the largest of every 16 bytes and where the first of them
// began; which of the 16 bytes' elements it was is looked up at the end.
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

constexpr int kAcceptThreads = 1024;

template <int DT>
struct Logits;
template <>
struct Logits<kF32> {
  static constexpr int kPer = 4;             // elements of 16 bytes
  static __device__ __forceinline__ float one(const void *x, int64_t at) {
    return static_cast<const float *>(x)[at];
  }
  static __device__ __forceinline__ float largest(u4 x) {
    return fmaxf(fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1])),
                 fmaxf(__uint_as_float(x[2]), __uint_as_float(x[3])));
  }
};
template <>
struct Logits<kF16> {
  static constexpr int kPer = 8;
  static __device__ __forceinline__ float one(const void *x, int64_t at) {
    return (float)static_cast<const _Float16 *>(x)[at];
  }
  static __device__ __forceinline__ float largest(u4 x) {
    const h8 h = __builtin_bit_cast(h8, x);
    float m = fmaxf((float)h[0], (float)h[1]);
#pragma unroll
    for (int i = 2; i < 8; ++i) m = fmaxf(m, (float)h[i]);
    return m;
  }
};
template <>
struct Logits<kBF16> {
  static constexpr int kPer = 8;
  static __device__ __forceinline__ float one(const void *x, int64_t at) {
    return __uint_as_float((uint32_t)static_cast<const uint16_t *>(x)[at] << 16);
  }
  static __device__ __forceinline__ float largest(u4 x) {
    float m = -__builtin_huge_valf();
#pragma unroll
    for (int i = 0; i < 4; ++i)
      m = fmaxf(m, fmaxf(__uint_as_float(x[i] << 16), __uint_as_float(x[i] & 0xffff0000u)));
    return m;
  }
};

// Ranking key of a place in a row: the larger logit, then the lower place.  Places
// where no logit was above -inf (NaN among them) rank by the place alone.
__device__ __forceinline__ uint64_t place_key(float x, int at) {
  return ((uint64_t)order_bits(x) << 32) | (uint64_t)(~(uint32_t)at);
}

template <int DT>
__global__ void __launch_bounds__(kAcceptThreads) dresd_accept(AcceptParams p) {
  typedef Logits<DT> X;
  constexpr int E = X::kPer, kUnroll = 8;
  __shared__ uint64_t wbest[kAcceptThreads / kWaveSize];
  __shared__ int32_t tok[kNodesMax], par[kNodesMax];
  __shared__ int32_t child;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  int nodes = p.nodes[b];
  nodes = nodes < 0 ? 0 : nodes > p.N ? p.N : nodes;
  if (tid < nodes) {
    tok[tid] = p.token[(size_t)b * p.N + tid];
    par[tid] = p.parent[(size_t)b * p.N + tid];
  }
  int u = nodes > 0 ? 0 : -1, done = 0;
  int32_t g = -1;
  while (u >= 0) {
    if (tid == 0) {
      p.path[(size_t)b * p.most + done] = u;
      child = p.N;
    }
    ++done;
    // the row: up to the first whole 16 bytes, 16 bytes at a time, the rest
    const int64_t row = ((int64_t)b * p.N + u) * p.row;
    const uint8_t *at = static_cast<const uint8_t *>(p.logits) + row * (16 / E);
    int head = (int)((16 - ((uintptr_t)at & 15)) & 15) / (16 / E);
    head = head < p.V ? head : p.V;
    const int body = (p.V - head) / E, tail = p.V - head - body * E;
    const u4 *vec = reinterpret_cast<const u4 *>(at + head * (16 / E));
    float best = -__builtin_huge_valf();
    int where = p.V;                         // element at which the best 16 bytes begin
    for (int c0 = tid; c0 < body; c0 += kUnroll * kAcceptThreads) {
      u4 v[kUnroll];
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {    // (past the end the first again, which changes nothing)
        const int c = c0 + k * kAcceptThreads;
        v[k] = vec[c < body ? c : c0];
      }
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        const float m = X::largest(v[k]);
        if (m > best) {
          best = m;
          where = head + (c0 + k * kAcceptThreads) * E;
        }
      }
    }
    if (tid < head || (tid >= 64 && tid < 64 + tail)) {
      const int e = tid < head ? tid : head + body * E + tid - 64;
      const float m = X::one(at, e);
      if (m > best || (m == best && e < where && where < p.V)) {
        best = m;
        where = e;
      }
    }
    uint64_t key = place_key(best, where);
#pragma unroll
    for (int o = 1; o < kWaveSize; o <<= 1) {
      const uint64_t other = __shfl_xor(key, o, kWaveSize);
      key = other > key ? other : key;
    }
    if (lane == 0) wbest[tid >> 6] = key;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kAcceptThreads / kWaveSize; ++w) key = wbest[w] > key ? wbest[w] : key;
    best = order_value((uint32_t)(key >> 32));
    where = (int)~(uint32_t)key;
    if (where < p.V) {
      // the first of its elements that has the value
      const bool is = lane < E && where + lane < p.V && X::one(at, where + lane) == best;
      g = where + __ffsll((long long)__ballot(is)) - 1;
    } else {
      // nothing above -inf: the first -inf, else (NaN alone) token 0
      int low = p.V;
      for (int e = tid; e < p.V && low == p.V; e += kAcceptThreads)
        if (X::one(at, e) == -__builtin_huge_valf()) low = e;
      __syncthreads();
      if (tid == 0) wbest[0] = (uint64_t)p.V;
      __syncthreads();
      if (low < p.V) atomicMin(reinterpret_cast<unsigned long long *>(wbest), (unsigned long long)low);
      __syncthreads();
      g = (int)wbest[0] < p.V ? (int)wbest[0] : 0;
    }
    // the lowest child with that token; children have higher numbers
    const int c = u + 1 + tid;               // at most kNodesMax - 1 of them
    if (done < p.most && c < nodes && par[c] == u && tok[c] == g) atomicMin(&child, c);
    __syncthreads();
    u = child < p.N ? child : -1;
    __syncthreads();
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
