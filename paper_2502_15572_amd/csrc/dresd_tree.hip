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
// time.  What bounds it is latency: one read of the drafts, then LDS, and the
// writes of the bits.  One workgroup per query, T threads per draft.
//
// Acceptance.  From node 0, the arg max of the node's logits names the child
// to go on to.  Only the path's rows are read.  One workgroup per query.
#include "dresd_device.h"
#include "dresd_verify.h"

namespace dresd {

namespace {

constexpr int kTreeThreads = 1024;
constexpr int kTreeStage = 12288;    // tokens staged in LDS
constexpr int kDraftsMax = DRESD_K_MAX_INTERNAL;

template <bool STAGED>
__global__ void __launch_bounds__(kTreeThreads) dresd_tree(TreeParams p) {
  extern __shared__ int32_t stage[];
  __shared__ uint16_t len[kDraftsMax], seen[kDraftsMax], from[kDraftsMax];
  __shared__ uint16_t owner[kNodesMax];      // draft that a node is new in
  __shared__ uint32_t base[kDraftsMax];
  __shared__ uint32_t wsum[kTreeThreads / kWaveSize];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  const int r = p.r, N = p.N;
  // a node of depth p has a number of at least p: later tokens cannot get one
  const int length = p.length < N ? p.length : N;
  const int32_t *src = p.drafts + (size_t)b * r * p.length;
  const int32_t first = p.next_tok[b];
  int cnt = p.count[b];
  cnt = cnt < 0 ? 0 : cnt > r ? r : cnt;
  if constexpr (STAGED) {
    for (int e = tid; e < cnt * length; e += kTreeThreads)
      stage[e] = src[(size_t)(e / length) * p.length + e % length];
    __syncthreads();
  }
  auto token = [&](int i, int j) -> int32_t {
    if constexpr (STAGED) return stage[i * length + j];
    else return src[(size_t)i * p.length + j];
  };

  // 1. lengths
  if (tid < r) {
    int n = 0;
    if (tid < cnt && token(tid, 0) == first)
      while (n < length && token(tid, n) != p.eos) ++n;
    len[tid] = (uint16_t)n;
  }
  __syncthreads();

  // 2. longest prefix that an earlier draft has, and the first draft that has it;
  //    threads T i .. T i + T - 1 share draft i
  int T = 1;
  while (T < kWaveSize && r * 2 * T <= kTreeThreads) T <<= 1;
  const int i = tid / T, sub = tid & (T - 1);
  const int n = i < cnt ? len[i] : 0;
  uint32_t best = 0;                         // common prefix, then the lower draft
  if (n > 0) {
    for (int j = sub; j < i; j += T) {
      const int m = len[j] < n ? len[j] : n;
      int c = 0;
      while (c < m && token(i, c) == token(j, c)) ++c;
      const uint32_t key = c > 0 ? ((uint32_t)c << 16) | (0xffffu - (uint32_t)j) : 0u;
      best = key > best ? key : best;
    }
  }
  for (int o = 1; o < T; o <<= 1) {
    const uint32_t other = __shfl_xor(best, o, kWaveSize);
    best = other > best ? other : best;
  }
  const int shared = best ? (int)(best >> 16) : 1;
  const uint32_t fresh = n > shared ? (uint32_t)(n - shared) : 0u;
  if (i < r && sub == 0) {
    seen[i] = (uint16_t)shared;
    from[i] = (uint16_t)(0xffffu - (best & 0xffffu));
  }

  // 3. number of each draft's first new node: workgroup prefix sum
  uint32_t x = sub == 0 ? fresh : 0u;
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
  if (i < r && sub == 0) base[i] = before + x - fresh;
  __syncthreads();
  const int nodes = total < (uint32_t)N ? (int)total : N;

  // 4. the new nodes' tokens, parents and depths
  int32_t *tok = p.token + (size_t)b * N, *par = p.parent + (size_t)b * N,
          *dep = p.depth + (size_t)b * N;
  auto hangs_on = [&](int d) -> int {        // node that a draft's first new one hangs on
    const int s = seen[d];
    if (s <= 1) return 0;
    const int j = from[d];
    return (int)base[j] + s - 1 - (int)seen[j];
  };
  if (fresh > 0) {
    const uint32_t at = base[i];
    for (uint32_t e = sub; e < fresh && at + e < (uint32_t)N; e += T) {
      owner[at + e] = (uint16_t)i;
      tok[at + e] = token(i, shared + (int)e);
      par[at + e] = e == 0 ? hangs_on(i) : (int)(at + e) - 1;
      dep[at + e] = shared + (int)e;
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

  // 5. ancestors: runs of consecutive nodes, highest first
  const int W = (N + 63) / 64;
  for (int u = tid; u < N; u += kTreeThreads) {
    uint64_t *row = p.mask + ((size_t)b * N + u) * W;
    int hi = u < nodes ? u : -1;             // top of the run at hand
    int lo = hi > 0 ? (int)base[owner[hi]] : 0;
    for (int w = W - 1; w >= 0; --w) {
      uint64_t bits = 0;
      while (hi >= 64 * w) {
        const int a = lo > 64 * w ? lo : 64 * w;             // the run's part in this word
        bits |= (~0ull >> (63 - (hi - a))) << (a - 64 * w);
        if (lo < 64 * w) {
          hi = 64 * w - 1;                                   // its rest is in lower words
        } else if (lo == 0) {
          hi = -1;
        } else {
          hi = hangs_on(owner[hi]);
          lo = hi > 0 ? (int)base[owner[hi]] : 0;
        }
      }
      row[w] = bits;
    }
  }
}

constexpr int kAcceptThreads = 1024;

template <int DT>
__device__ __forceinline__ float logit(const void *x, int64_t at) {
  if constexpr (DT == kF32) return static_cast<const float *>(x)[at];
  else if constexpr (DT == kF16) return (float)static_cast<const _Float16 *>(x)[at];
  else return __uint_as_float((uint32_t)static_cast<const uint16_t *>(x)[at] << 16);
}

// A token's ranking key: the larger logit, then the lower token; NaN lowest.
__device__ __forceinline__ uint64_t token_key(float x, uint32_t v) {
  const uint32_t h = x != x ? 0u : order_bits(x);
  return ((uint64_t)h << 32) | (uint64_t)(~v);
}

template <int DT>
__global__ void __launch_bounds__(kAcceptThreads) dresd_accept(AcceptParams p) {
  __shared__ uint64_t wbest[kAcceptThreads / kWaveSize];
  __shared__ int32_t child;
  const int b = blockIdx.x, tid = threadIdx.x;
  const int32_t *tok = p.token + (size_t)b * p.N, *par = p.parent + (size_t)b * p.N;
  int nodes = p.nodes[b];
  nodes = nodes < 0 ? 0 : nodes > p.N ? p.N : nodes;
  int u = nodes > 0 ? 0 : -1, done = 0;
  int32_t g = -1;
  while (u >= 0) {
    if (tid == 0) {
      p.path[(size_t)b * p.most + done] = u;
      child = p.N;
    }
    ++done;
    const int64_t at = ((int64_t)b * p.N + u) * p.row;
    uint64_t best = 0;
    for (int v = tid; v < p.V; v += kAcceptThreads) {
      const uint64_t key = token_key(logit<DT>(p.logits, at + v), (uint32_t)v);
      best = key > best ? key : best;
    }
#pragma unroll
    for (int o = 1; o < kWaveSize; o <<= 1) {
      const uint64_t other = __shfl_xor(best, o, kWaveSize);
      best = other > best ? other : best;
    }
    if ((tid & 63) == 0) wbest[tid >> 6] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kAcceptThreads / kWaveSize; ++w) best = wbest[w] > best ? wbest[w] : best;
    g = (int32_t)~(uint32_t)best;
    // the lowest child with that token; children have higher numbers
    const int v = u + 1 + tid;               // at most kNodesMax - 1 of them
    if (done < p.most && v < nodes && par[v] == u && tok[v] == g) atomicMin(&child, v);
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
  const int64_t tokens = (int64_t)p.r * (p.length < p.N ? p.length : p.N);
  const bool staged = tokens <= kTreeStage;
  return hipLaunchKernel(staged ? (const void *)dresd_tree<true> : (const void *)dresd_tree<false>,
                         dim3((unsigned)p.B), dim3(kTreeThreads), args,
                         staged ? (size_t)tokens * 4 : 0, st);
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
