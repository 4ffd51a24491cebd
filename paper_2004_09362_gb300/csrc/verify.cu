// Which drafted tokens stand, and the token that comes after them.
//
// A draft token t stands with probability min(1, p(t) / q(t)); where one does not, the next token is drawn from
// max(p - q, 0), by inversion: the first v at which the running sum passes u times the whole.  Both steps together give
// tokens distributed as p.
//
// Bound by memory: of all the probabilities only one row of the target and one of the draft are needed
// whole, those at the first draft that does not stand (the drafts' own probabilities are a few words).  A cluster of CTAs
// takes a sequence, each warp a run of neighbouring tokens; the warps' sums are exchanged through the cluster's shared memory, every
// warp finds the run in which the running sum passes, and the warp of that run reads it again (from the L2).
//
// The token is a choice at a border between running sums, so these have to be better than 32 bits: after 131072 terms a sum in 32 bits
// is off by more than a whole token's share.  A lane adds in twice 32 bits (the error of each addition is computed
// exactly and added up beside it: Knuth's TwoSum), lanes and warps in 64 bits, which this GPU does at 1/64 the rate.
#include <climits>

#include "cluster.cuh"

namespace gar {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMostCtas = 8;  // of a cluster

struct VerifyArgs {
  const void *target, *draft;
  int64_t tb, tr, db, dr;
  const void *tokens;
  void *out;
  int32_t *accepted;
  const float *uniform;
  int vocab, drafts, ctas;
  int run;                   // tokens of a warp
  bool wide;                 // 64-bit tokens
};

// A sum in twice 32 bits.
struct Sum {
  float high = 0.f, low = 0.f;
  __device__ __forceinline__ void add(float x, float rest) {
    const float t = high + x, b = t - high;
    low += ((high - (t - b)) + (x - b)) + rest;
    high = t;
  }
};

template <typename T> __device__ __forceinline__ float probability(const T *p) {
  return fminf(fmaxf(to_f32(*p), 0.f), 1.f);  // (of a NaN and a number the number)
}

__device__ __forceinline__ int64_t token_at(const VerifyArgs &a, int64_t i) {
  return a.wide ? static_cast<const int64_t *>(a.tokens)[i] : (int64_t) static_cast<const int32_t *>(a.tokens)[i];
}
__device__ __forceinline__ void put_token(const VerifyArgs &a, int64_t i, int64_t token) {
  if (a.wide)
    static_cast<int64_t *>(a.out)[i] = token;
  else
    static_cast<int32_t *>(a.out)[i] = (int32_t)token;
}

// What may be drawn at the row: of the target, less the draft's where there is one.
template <typename T> struct Row {
  const T *p, *q;
  bool less;
  __device__ __forceinline__ double operator()(int v) const {
    const double x = (double)probability(p + v) - (less ? (double)probability(q + v) : 0.);
    return x > 0. ? x : 0.;
  }
};

template <typename T> __device__ __forceinline__ double run_sum(const Row<T> &row, int from, int to) {
  constexpr int N = 8;  // loads of each row in flight
  Sum s;
  for (int v0 = from + (int)(threadIdx.x & 31); v0 < to; v0 += 32 * N) {
    float p[N], q[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int v = v0 + 32 * i;
      p[i] = v < to ? probability(row.p + v) : 0.f;
      q[i] = row.less && v < to ? probability(row.q + v) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float d = p[i] - q[i];
      if (d > 0.f) {
        const float b = d - p[i];
        s.add(d, (p[i] - (d - b)) - (q[i] + b));
      }
    }
  }
  double x = (double)s.high + (double)s.low;
#pragma unroll
  for (int d = 16; d > 0; d /= 2) x += __shfl_xor_sync(~0u, x, d);
  return x;
}

template <typename T> __device__ __forceinline__ int last_of(const Row<T> &row, int from, int to) {
  int last = -1;
  for (int v = from + (int)(threadIdx.x & 31); v < to; v += 32)
    if (row(v) > 0.) last = v;
  return __reduce_max_sync(~0u, last);
}

// The first token of the run at which `before` and the running sum pass `goal`; all of the run does.
template <typename T> __device__ __forceinline__ int find(const Row<T> &row, int from, int to, double before, double goal) {
  const int lane = threadIdx.x & 31, each = (to - from + 31) / 32;
  const int v0 = min(to, from + lane * each), v1 = min(to, v0 + each);
  double sum = 0.;
#pragma unroll 8
  for (int v = v0; v < v1; ++v) sum += row(v);
  double upto = sum;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const double x = __shfl_up_sync(~0u, upto, d);
    if (lane >= d) upto += x;
  }
  // (Where rounding hides the border, the last that counts.)
  const uint32_t past = __ballot_sync(~0u, before + upto > goal && sum > 0.), some = __ballot_sync(~0u, sum > 0.);
  const int from_lane = past ? __ffs(past) - 1 : 31 - __clz(some | 1u);
  int found = -1;
  if (lane == from_lane) {
    double x = before + (upto - sum);
#pragma unroll 8
    for (int v = v0; v < v1; ++v) {
      const double w = row(v);
      if (w > 0. && !(x > goal)) x += w, found = v;
    }
  }
  return __shfl_sync(~0u, found, from_lane);
}

template <typename T> __global__ void __launch_bounds__(kThreads) verify_kernel(const VerifyArgs a) {
  __shared__ double totals[2][kMostCtas * kWarps];
  __shared__ int lasts[kMostCtas * kWarps];
  __shared__ int stop, refused;
  const int rank = cluster_rank(), warp = threadIdx.x / 32, lane = threadIdx.x & 31, me = rank * kWarps + warp;
  const int64_t b = blockIdx.x / a.ctas;
  cluster_arrive();
  after_earlier_kernels();

  const T *const target = static_cast<const T *>(a.target) + b * a.tb, *const draft = static_cast<const T *>(a.draft) + b * a.db;
  if (warp == 0) {
    // A lane for each draft.
    int at = 0, why = 0;
    for (;; at += 32) {
      const int i = at + lane;
      int64_t token = -1;
      bool stands = false;
      if (i < a.drafts) {
        token = token_at(a, b * a.drafts + i);
        if (token >= 0 && token < a.vocab) {
          const double p = probability(target + i * a.tr + token), q = probability(draft + i * a.dr + token);
          stands = (double)fmaxf(a.uniform[b * (a.drafts + 1) + i], 0.f) * q < p;
        }
      }
      const uint32_t not_one = __ballot_sync(~0u, !stands);
      if (not_one == 0) continue;
      const int first = __ffs(not_one) - 1;
      why = __shfl_sync(~0u, (int)(token >= 0), first);
      at += first;
      break;
    }
    if (lane == 0) stop = at, refused = why;
  }
  __syncthreads();
  Row<T> row{target + stop * a.tr, refused ? draft + stop * a.dr : nullptr, refused != 0};
  const int from = min((int64_t)a.vocab, (int64_t)me * a.run), to = min((int64_t)a.vocab, (int64_t)from + a.run);
  cluster_wait();

  // The running sums before and after each run; this lane knows those of 4 runs.
  constexpr int EACH = kMostCtas * kWarps / 32;
  double before = 0., goal = 0., all = 0.;
  int chosen = -1;
  const float u = fmaxf(a.uniform[b * (a.drafts + 1) + a.drafts], 0.f);
  for (int pass = 0; pass < 2; ++pass) {
    const double mine = run_sum(row, from, to);
    if (lane < a.ctas) store_in_cta(&totals[pass][me], lane, mine);
    cluster_sync();
    double upto[EACH], sum = 0.;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int k = lane * EACH + i;
      upto[i] = sum += k < a.ctas * kWarps ? totals[pass][k] : 0.;
    }
    double x = sum;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const double y = __shfl_up_sync(~0u, x, d);
      if (lane >= d) x += y;
    }
    const double base = __shfl_up_sync(~0u, x, 1);
    const double start = lane == 0 ? 0. : base;
    all = __shfl_sync(~0u, start + upto[EACH - 1], 31);
    if (!(all > 0.) && row.less) {
      row.less = false;  // nothing is left of the target: all of it
      continue;
    }
    goal = (double)u * all;
    int k = -1;
    double low = 0.;
#pragma unroll
    for (int i = EACH - 1; i >= 0; --i) {
      const double lower = i == 0 ? start : start + upto[i - 1];
      if (start + upto[i] > goal) k = lane * EACH + i, low = lower;
    }
    const uint32_t past = __ballot_sync(~0u, k >= 0);
    if (past) {
      chosen = __shfl_sync(~0u, k, __ffs(past) - 1);
      before = __shfl_sync(~0u, low, __ffs(past) - 1);
    }
    break;
  }

  const int64_t out = b * (a.drafts + 1);
  if (chosen == me) {
    const int token = find(row, from, to, before, goal);
    if (lane == 0) put_token(a, out + stop, token);
  } else if (chosen < 0) {
    const int last = last_of(row, from, to);
    if (lane == 0) store_in_cta(&lasts[me], 0, last);
    cluster_sync();
    if (me == 0) {
      int token = -1;
      for (int k = lane; k < a.ctas * kWarps; k += 32) token = max(token, lasts[k]);
      token = __reduce_max_sync(~0u, token);
      if (lane == 0) put_token(a, out + stop, token);
    }
  }
  if (rank == 0) {
    for (int i = threadIdx.x; i <= a.drafts; i += kThreads)
      if (i != stop) put_token(a, out + i, i < stop ? token_at(a, b * a.drafts + i) : -1);
    if (threadIdx.x == 0) a.accepted[b] = stop;
  }
}

}  // namespace
}  // namespace gar

using namespace gar;

extern "C" int gar_verify_drafts(const void *target, int64_t target_batch_stride, int64_t target_row_stride, const void *draft,
                                 int64_t draft_batch_stride, int64_t draft_row_stride, int dtype, int64_t vocab,
                                 const void *tokens, int token_bytes, const float *uniform, int batch, int drafts,
                                 void *out_tokens, int32_t *accepted, gar_stream_t stream) {
  if (!float_type(dtype)) return refuse("probabilities are GAR_F32, GAR_BF16 or GAR_F16");
  if (token_bytes != 4 && token_bytes != 8) return refuse("tokens are 4 or 8 bytes wide");
  if (vocab < 1 || vocab > INT_MAX / 2) return refuse("vocab must be 1..2^30 - 1");
  if (batch < 0 || drafts < 0 || drafts > (1 << 20)) return refuse("bad batch or drafts");
  if (batch > INT_MAX / kMostCtas) return refuse("too many sequences");
  if (batch == 0) return GAR_OK;
  if (target == nullptr || uniform == nullptr || out_tokens == nullptr || accepted == nullptr ||
      (drafts > 0 && (draft == nullptr || tokens == nullptr)))
    return refuse("null pointer");
  const int size = element_size(dtype);
  if ((uintptr_t)target % size || (uintptr_t)draft % size || (uintptr_t)uniform % 4 || (uintptr_t)accepted % 4 ||
      (uintptr_t)tokens % token_bytes || (uintptr_t)out_tokens % token_bytes) {
    set_error("a buffer is not aligned to its elements");
    return GAR_EALIGN;
  }
  VerifyArgs a{};
  a.target = target, a.draft = draft;
  a.tb = target_batch_stride, a.tr = target_row_stride, a.db = draft_batch_stride, a.dr = draft_row_stride;
  a.tokens = tokens, a.out = out_tokens, a.accepted = accepted, a.uniform = uniform;
  a.vocab = (int)vocab, a.drafts = drafts, a.wide = token_bytes == 8;
  // CTAs of a sequence: enough to fill the GPU, with 2048 tokens each at least.
  a.ctas = 1;
  while (a.ctas < kMostCtas && (int64_t)batch * a.ctas < 152 * 4 && vocab > 2048 * a.ctas) a.ctas *= 2;
  const int warps = a.ctas * kWarps;
  a.run = (int)((vocab + warps - 1) / warps + 31) / 32 * 32;
  return with_float(dtype, [&](auto t) {
    using T = typename decltype(t)::type;
    return launch_clusters("gar_verify_drafts", verify_kernel<T>, (int64_t)batch * a.ctas, a.ctas, kThreads, stream, a);
  });
}
