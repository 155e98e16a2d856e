// Declarations of the kernels of batch verification (dresd_tree.hip,
// dresd_kv.hip, dresd_attend.hip), shared with the host runtime.
#pragma once
#include "dresd_internal.h"

namespace dresd {

constexpr int kF8 = 3;               // DRESD_F8: e4m3, caches alone
constexpr int kNodesMax = 1024;      // DRESD_NODES_MAX
constexpr int kHeadDimMax = 256;     // widest head of a cache
// A launch has fewer than 2^32 threads: queries of a call whose workgroups have 1,024, ...
constexpr int kQueriesMax = (1 << 22) - 1;
// ... and rows (tokens times heads) of a cache write or read, dim / 8 lanes each, rounded up to
// 8, 16 or 32.
constexpr int64_t kv_rows_max(int dim) {
  return (dim <= 64 ? 1ll << 29 : dim <= 128 ? 1ll << 28 : 1ll << 27) - 32;
}

// Prefix tree of drafts (dresd_tree.hip).
struct TreeParams {
  const int32_t *drafts, *count, *next_tok;
  int32_t *token, *parent, *depth, *nodes;
  uint64_t *mask;
  int B, r, length, eos, N;
};
hipError_t launch_draft_tree(const TreeParams &p, hipStream_t st);

// Acceptance of a tree's path (dresd_tree.hip).
struct AcceptParams {
  const void *logits;
  int64_t row;               // elements from one node's logits to the next
  const int32_t *token, *parent, *nodes;
  int32_t *path, *accepted, *next_tok;
  int B, N, V, most, dtype;
};
hipError_t launch_accept(const AcceptParams &p, hipStream_t st);

// Paged cache of keys and values (dresd_kv_cache of the public header).
struct CacheRef {
  void *k, *v;
  uint8_t *k_exp, *v_exp;
  int64_t pages;
  int page_log, heads, dim, dtype;
};

// Cache writes and reads (dresd_kv.hip).
struct KvParams {
  CacheRef c;
  const void *k_in, *v_in;   // write: element strides of rows and heads
  int64_t k_row, k_head, v_row, v_head;
  void *k_out, *v_out;       // read: [n, heads, dim]
  const int64_t *slots;
  int64_t n;
  int dtype;
};
hipError_t launch_kv_write(const KvParams &p, hipStream_t st);
hipError_t launch_kv_read(const KvParams &p, hipStream_t st);

// Attention of chunks over a paged cache (dresd_attend.hip).
struct AttendParams {
  CacheRef c;
  const void *q;
  int64_t q_row, q_head;
  const int32_t *starts;     // ragged: [B + 1]; else n rows each
  const int32_t *table, *lengths;
  const uint64_t *mask;      // may be null
  void *out;
  float *lse;                // may be null
  void *work;
  int64_t T;
  float scale;
  int dtype, q_heads, n, B, width, words;
  bool ragged;
};
// Bytes; -1: more blocks than one launch takes.
int64_t attend_workspace(const AttendParams &p, int cus);
hipError_t launch_attend(const AttendParams &p, int cus, hipStream_t st);

}  // namespace dresd
