// Attention over shared prefixes: its parts' results and their join.
#pragma once

#include "gar_device.cuh"

namespace gar {

// Normalised outputs and logarithms of the sums of weights, of one part of the rows.
struct PrefixParts {
  float *out, *lse;
  int64_t row;  // floats of a row of out
};

struct JoinArgs {
  PrefixParts parts[2];  // own rows: [batch][heads]; prefixes: [group of sequences][cached head][its sequences][group]
  void *out;
  float *lse;
  int64_t ob, oh, rows;
  int dim, heads, group, share, out_dtype;
};

// Bytes of a call's workspace, and where its parts are.
size_t prefix_workspace(int batch, int heads, int dim, char *base, PrefixParts *parts);
int join_prefix(const JoinArgs &a, gar_stream_t stream);

}  // namespace gar
