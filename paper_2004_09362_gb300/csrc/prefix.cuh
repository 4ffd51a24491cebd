// Attention over shared prefixes: its parts' results and their join.
#pragma once

#include <cuda.h>

#include "gar_device.cuh"

namespace gar {

// Normalised outputs and logarithms of the sums of weights, of one part of the rows.
struct PrefixParts {
  float *out, *lse;
  int64_t row;  // floats of a row of out
};

// What many queries of shared prefixes need: those of one cached head and one prefix are `rows` rows, in blocks of 128 or
// (pair) 256; an item is such a block.
struct PrefixArgs {
  gar_kv_cache c;
  const void *q;
  int64_t qb, qh, table_stride;
  const int32_t *table, *lengths;
  Divide page, by_heads;   // by a page's rows; by heads_each
  int most_rows;           // of the cache that the table's width can hold
  int groups, share, heads_each, rows, blocks;
  float scale_log2;        // of the scores, positive: q is negated where it was not
  uint32_t negate;         // bits of q that are turned over
  int ctas, device, give_up;
  int box;                 // rows of the boxes that a tile can be copied in, or 0
  bool pair;
  // Partial results of CTA i and item j at place i + j: [2][128] (m, l) and [2][channels / 4][128][4] o.
  float2 *ml;
  float *o;
};

struct JoinArgs {
  PrefixParts parts[2];  // own rows: [batch][heads]; prefixes: [group of sequences][cached head][its sequences][group]
  void *out;
  float *lse;
  int64_t ob, oh, rows;
  int dim, heads, group, share, out_dtype;
  bool wide;             // four neighbouring outputs can be stored at once
};

constexpr int kKeys = 128;  // cached rows of a tile

// A prefix's rows.  report: one that the table cannot hold.
__device__ __forceinline__ int prefix_rows(const PrefixArgs &a, int g, bool report) {
  int n = a.lengths[g];
  if (n < 0 || n > a.most_rows) {
    if (report && a.c.status) atomicOr(a.c.status, GAR_KV_BAD_LENGTH);
    n = n < 0 ? 0 : a.most_rows;
  }
  return n;
}
// The tiles of each of its items.
__device__ __forceinline__ int prefix_tiles(int rows) { return (int)(((unsigned)rows + kKeys - 1) / kKeys); }

// The items' tiles stand one behind the other, [prefix][cached head][block]; CTA i takes the i-th of equal shares.  By a
// warp: all of the tiles, and those of the prefixes before `g`.
__device__ __forceinline__ int2 prefix_line(const PrefixArgs &a, int g, bool report) {
  const int lane = threadIdx.x & 31;
  int all = 0, before = 0;
  for (int i = lane; i < a.groups; i += 32) {
    const int t = prefix_tiles(prefix_rows(a, i, report));
    all += t;
    if (i < g) before += t;
  }
  const int items = a.c.heads * a.blocks;
  return make_int2(__reduce_add_sync(~0u, all) * items, __reduce_add_sync(~0u, before) * items);
}
__device__ __forceinline__ int share_of(int all, int ctas) { return (all + ctas - 1) / ctas; }

// Bytes of a call's workspace, and where its parts are.
size_t prefix_workspace(int batch, int heads, int dim, char *base, PrefixParts *parts);
int join_prefix(const JoinArgs &a, gar_stream_t stream);

// Places for partial results: of every CTA, and one for each item beyond an item that a CTA begins with.
size_t prefix_partials(int items, int dim, char *base, PrefixArgs *a);
int prefix_mma(const PrefixArgs &a, const CUtensorMap (&maps)[2], gar_stream_t stream);
int join_partials(const PrefixArgs &a, const JoinArgs &j, gar_stream_t stream);

}  // namespace gar
