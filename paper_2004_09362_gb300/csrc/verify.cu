// Which drafted tokens stand, and the token that comes after them.
//
// A draft token t stands with probability min(1, p(t) / q(t)); where one does not, the next token is drawn from
// max(p - q, 0), by inversion: the first v at which the running sum passes u times the whole.  Both steps together give
// tokens distributed as p.
//
// Bound by memory: of all the probabilities only one row of the target and one of the draft are needed
// whole, those at the first draft that does not stand (the drafts' own probabilities are a few words).  A cluster of CTAs
// takes a sequence, each warp a run of neighbouring tokens, whose pieces a lane sums side by side; the warps' sums are exchanged through
// the cluster's shared memory, every warp finds the run in which the running sum passes, and the warp of that run reads one of its
// pieces again (from the L2).
//
// The token is a choice at a border between running sums, so these have to be better than 32 bits: after 131072 terms a sum in 32 bits
// is off by more than a whole token's share.  All sums are held in twice 32 bits: the error of each addition is computed
// exactly and added up beside it (Knuth's TwoSum).  64 bits are out of the question, this GPU does two such additions a clock and SM:
// the warps' sums and scans alone took most of the time in 64 bits.  But the errors that are added up beside are rounded themselves, and
// with very many they lose what they are there for (400 million numbers, half of them equal: 2^-24 of the sum).  So a lane of a longer run
// adds up kRounds groups at a time, and those sums in 64 bits.
//
// 256 sequences, 131072 f32: 67 us, 4.0 TB/s; 57, 50021 bf16: 12 us; one, 32768 f32: 7 us, which is the chain of drafts, their
// probabilities, rows, sums and the token, each a round trip.
#include <climits>

#include "cluster.cuh"

namespace gar {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMostCtas = 8;  // of a cluster
constexpr int kSubs = 4;      // pieces of a warp's run
constexpr int kGroup = 4;     // neighbouring tokens of a lane
constexpr float kUnit = 0x1p64f;  // sums are compared in multiples of 1 / kUnit, see up_to_unit()
constexpr int kRounds = 64;   // sums are held in twice 32 bits over so many groups of a lane and piece

struct VerifyArgs {
  const void *target, *draft;
  int64_t tb, tr, db, dr;
  const void *tokens;
  void *out;
  int32_t *accepted;
  const float *uniform;
  int vocab, drafts, ctas;
  int piece;                 // tokens of a piece of a warp's run
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
// A sum of probabilities times kUnit, exactly.  The product with u rounds to 2^-149 at best, which is a whole probability of the smallest;
// of 2^-149 times kUnit it is 2^-64, and no sum comes to 2^95 (2^30 tokens).
__device__ __forceinline__ Sum up_to_unit(Sum a) {
  a.high *= kUnit, a.low *= kUnit;
  return a;
}
// The low part no more than a rounding error of the high one.
__device__ __forceinline__ Sum neat(Sum a) {
  Sum s;
  s.high = a.high + a.low, s.low = a.low - (s.high - a.high);
  return s;
}
__device__ __forceinline__ Sum operator+(Sum a, Sum b) {
  a.add(b.high, b.low);
  return neat(a);
}
__device__ __forceinline__ Sum operator*(Sum a, float x) {
  Sum s;
  s.high = a.high * x, s.low = fmaf(a.high, x, -s.high) + a.low * x;
  return neat(s);
}
__device__ __forceinline__ bool operator>(Sum a, Sum b) { return a.high > b.high || (a.high == b.high && a.low > b.low); }
__device__ __forceinline__ Sum up(Sum a, int d) {
  Sum s;
  s.high = __shfl_up_sync(~0u, a.high, d), s.low = __shfl_up_sync(~0u, a.low, d);
  return s;
}
__device__ __forceinline__ Sum from_lane(Sum a, int lane) {
  Sum s;
  s.high = __shfl_sync(~0u, a.high, lane), s.low = __shfl_sync(~0u, a.low, lane);
  return s;
}
// The sums over the lanes up to each.
__device__ __forceinline__ Sum running(Sum a) {
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const Sum x = up(a, d);
    if ((int)(threadIdx.x & 31) >= d) a = x + a;
  }
  return a;
}

// Within [0, 1]; of a NaN 0.
__device__ __forceinline__ float probable(float x) { return __saturatef(x); }
template <typename T> __device__ __forceinline__ float probability(const T *p) { return probable(to_f32(*p)); }

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
};

// max(p - q, 0), exactly.
__device__ __forceinline__ Sum remaining(float p, float q) {
  const float x = probable(p), y = probable(q), d = x - y, b = d - x;
  Sum s;
  if (d > 0.f) s.high = d, s.low = (x - (d - b)) - (y + b);
  return s;
}

// kGroup neighbouring tokens as they lie in memory: loaded at once where they are aligned, else one by one.  (What is loaded is
// taken apart later, when all loads are on their way.)
template <typename T, bool WIDE> struct Group;
template <typename T> struct Group<T, true> {
  static_assert(kGroup == 4, "four or eight bytes a pair");
  uint32_t w[kGroup * sizeof(T) / 4];
  __device__ __forceinline__ void load(const T *p, bool there) {
    if constexpr (sizeof(T) == 4) {
      const uint4 x = there ? *reinterpret_cast<const uint4 *>(p) : make_uint4(0, 0, 0, 0);
      w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
    } else {
      const uint2 x = there ? *reinterpret_cast<const uint2 *>(p) : make_uint2(0, 0);
      w[0] = x.x, w[1] = x.y;
    }
  }
  __device__ __forceinline__ float2 pair(int i) const {
    if constexpr (sizeof(T) == 4)
      return make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
    else
      return unpack2(w[i], T());
  }
};
template <typename T> struct Group<T, false> {
  T x[kGroup];
  __device__ __forceinline__ void load(const T *p, bool there) {
#pragma unroll
    for (int i = 0; i < kGroup; ++i) x[i] = there ? p[i] : T(0.f);
  }
  __device__ __forceinline__ float2 pair(int i) const { return make_float2(to_f32(x[2 * i]), to_f32(x[2 * i + 1])); }
};
// A group at the row's ends, token by token.
template <typename T> __device__ __forceinline__ void load_ends(const T *p, int v, int vocab, float (&x)[kGroup]) {
#pragma unroll
  for (int i = 0; i < kGroup; ++i) x[i] = (unsigned)(v + i) < (unsigned)vocab ? to_f32(p[v + i]) : 0.f;
}
enum { DRAFT_NONE, DRAFT_WIDE, DRAFT_NARROW };  // how the draft's row is read

// Two sums side by side.
struct Sums {
  float2 high = {0.f, 0.f}, low = {0.f, 0.f};
};
__device__ __forceinline__ float2 sub2(float2 a, float2 b) { return fma2(b, make_float2(-1.f, -1.f), a); }

// d + rest = max(p - q, 0), exactly; then the same of high + d, whose rest goes to the low part.
__device__ __forceinline__ void add_pair(Sums &s, float2 p, float2 q) {
  const float2 x = make_float2(probable(p.x), probable(p.y));
  const float2 y = make_float2(fminf(probable(q.x), x.x), fminf(probable(q.y), x.y));
  const float2 d = sub2(x, y), b = sub2(d, x), rest = sub2(sub2(x, sub2(d, b)), add2(y, b));
  const float2 t = add2(s.high, d), c = sub2(t, s.high);
  s.low = add2(s.low, add2(add2(sub2(s.high, sub2(t, c)), sub2(d, c)), rest));
  s.high = t;
}

// A lane's part of the sums of tokens [at, end) of a run's kSubs pieces.  Groups of tokens begin `shift` tokens early, where the
// target's row is aligned.
template <typename T, int DRAFT>
__device__ __forceinline__ void add_run(const Row<T> &row, int64_t from, int piece, int vocab, int shift, int at, int end, Sums (&s)[kSubs]) {
  const int lane = threadIdx.x & 31;
#pragma unroll 1
  for (int k = at + lane * kGroup; k < end; k += 32 * kGroup) {
    Group<T, true> p[kSubs];
    Group<T, DRAFT == DRAFT_WIDE> q[kSubs];
    int v[kSubs];
#pragma unroll
    for (int i = 0; i < kSubs; ++i) {
      v[i] = (int)min(from + i * piece + k - shift, (int64_t)vocab);
      const bool there = v[i] >= 0 && v[i] + kGroup <= vocab;
      p[i].load(row.p + v[i], there);
      if (DRAFT != DRAFT_NONE) q[i].load(row.q + v[i], there);
    }
#pragma unroll
    for (int i = 0; i < kSubs; ++i) {
#pragma unroll
      for (int j = 0; j < kGroup / 2; ++j) add_pair(s[i], p[i].pair(j), DRAFT != DRAFT_NONE ? q[i].pair(j) : make_float2(0.f, 0.f));
      if (v[i] < vocab && (v[i] < 0 || v[i] + kGroup > vocab)) {
        float x[kGroup], y[kGroup] = {};
        load_ends(row.p, v[i], vocab, x);
        if (DRAFT != DRAFT_NONE) load_ends(row.q, v[i], vocab, y);
#pragma unroll
        for (int j = 0; j < kGroup; j += 2) add_pair(s[i], make_float2(x[j], x[j + 1]), make_float2(y[j], y[j + 1]));
      }
    }
  }
}

__device__ __forceinline__ Sum both(const Sums &s) {
  Sum a, b;
  a.high = s.high.x, a.low = s.low.x, b.high = s.high.y, b.low = s.low.y;
  return neat(a) + neat(b);
}
__device__ __forceinline__ double in_64(Sum a) { return (double)a.high + a.low; }
__device__ __forceinline__ Sum in_twice_32(double x) {
  Sum a;
  a.high = (float)x, a.low = (float)(x - a.high);
  return a;
}

// The sum over the lanes, in the same order in each.
__device__ __forceinline__ Sum over_lanes(Sum a) {
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    Sum x;
    x.high = __shfl_xor_sync(~0u, a.high, d), x.low = __shfl_xor_sync(~0u, a.low, d);
    a = a + x;
  }
  return a;
}

template <typename T> __device__ __forceinline__ int last_of(const Row<T> &row, int from, int to) {
  int last = -1;
  for (int v = from + (int)(threadIdx.x & 31); v < to; v += 32)
    if (remaining(to_f32(row.p[v]), row.less ? to_f32(row.q[v]) : 0.f).high > 0.f) last = v;
  return __reduce_max_sync(~0u, last);
}

// The first token that counts, of the groups from `from` on, up to `to`, at which `before` and the running sum pass `goal`, as they do; where
// rounding hides that, the last that counts.  (A token that does not count passes where the one before it did.  But a lane's running sum
// begins with one that was added up in another order than the lane's before it, so rounding may show that passing at the next token first.)
template <typename T, bool LONG>
__device__ __forceinline__ int find(const Row<T> &row, int64_t from, int64_t to, int vocab, Sum before, Sum goal) {
  const int lane = threadIdx.x & 31;
  int last = -1;
  double whole = LONG ? in_64(before) : 0.;
  Sum part;  // (LONG) what has come to `before` since it was `whole`
  int rounds = 0;
#pragma unroll 1
  for (int64_t v0 = from; v0 < to; v0 += 32 * kGroup) {
    const int v = (int)min(v0 + lane * kGroup, (int64_t)vocab);
    float p[kGroup], q[kGroup] = {};
    load_ends(row.p, v, vocab, p);
    if (row.less) load_ends(row.q, v, vocab, q);
    Sum upto[kGroup], sum;
    uint32_t counts = 0;  // which of the lane's tokens count
#pragma unroll
    for (int i = 0; i < kGroup; ++i) {
      const Sum w = up_to_unit(remaining(p[i], q[i]));
      if (w.high > 0.f) counts |= 1u << i;
      upto[i] = sum = sum + w;
    }
    const Sum with = running(sum);
    Sum start = up(with, 1);
    start = lane == 0 ? before : before + start;
    int passed = kGroup;
#pragma unroll
    for (int i = kGroup - 1; i >= 0; --i)
      if (start + upto[i] > goal) passed = i;
    const uint32_t later = counts & ~0u << passed;
    const uint32_t past = __ballot_sync(~0u, later != 0), some = __ballot_sync(~0u, counts != 0);
    if (past) return __shfl_sync(~0u, v + __ffs(later) - 1, __ffs(past) - 1);
    if (some) last = __shfl_sync(~0u, v + 31 - __clz(counts), 31 - __clz(some));
    before = before + from_lane(with, 31);
    if constexpr (LONG) {
      part = part + from_lane(with, 31);
      if (++rounds % kRounds == 0) whole += in_64(part), before = in_twice_32(whole), part = Sum();
    }
  }
  return last;
}

// LONG: pieces of more than kRounds groups a lane.
template <typename T, bool LONG> __global__ void __launch_bounds__(kThreads, 4) verify_kernel(const VerifyArgs a) {
  __shared__ float2 totals[2][kMostCtas * kWarps];
  __shared__ int lasts[kMostCtas * kWarps];
  __shared__ int stop, refused, picked, empty;
  __shared__ float2 bounds[2];
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
  // Runs begin where the target's row is aligned: a few tokens early.
  constexpr uintptr_t kWide = kGroup * sizeof(T);
  const int shift = (int)((uintptr_t)row.p % kWide / sizeof(T)), run = kSubs * a.piece;
  const int64_t begin = (int64_t)me * run;
  const int from = (int)min((int64_t)a.vocab, max((int64_t)0, begin - shift)), to = (int)min((int64_t)a.vocab, begin + run - shift);
  cluster_wait();

  const float u = fmaxf(a.uniform[b * (a.drafts + 1) + a.drafts], 0.f);
  Sum pieces[kSubs];  // this lane's part
  for (int pass = 0; pass < 2; ++pass) {
    double whole[LONG ? kSubs : 1] = {};
    for (int at = 0;;) {
      const int end = LONG ? min(a.piece, at + kRounds * 32 * kGroup) : a.piece;
      Sums sums[kSubs];
      if (!row.less)
        add_run<T, DRAFT_NONE>(row, begin, a.piece, a.vocab, shift, at, end, sums);
      else if ((uintptr_t)(row.q - shift) % kWide == 0)
        add_run<T, DRAFT_WIDE>(row, begin, a.piece, a.vocab, shift, at, end, sums);
      else
        add_run<T, DRAFT_NARROW>(row, begin, a.piece, a.vocab, shift, at, end, sums);
#pragma unroll
      for (int i = 0; i < kSubs; ++i) {
        pieces[i] = up_to_unit(both(sums[i]));
        if constexpr (LONG) whole[i] += in_64(pieces[i]), pieces[i] = in_twice_32(whole[i]);
      }
      if (!LONG || (at = end) >= a.piece) break;
    }
    Sum mine = pieces[0];
#pragma unroll
    for (int i = 1; i < kSubs; ++i) mine = mine + pieces[i];
    mine = over_lanes(mine);
    if (lane < a.ctas) store_in_cta(&totals[pass][me], lane, make_float2(mine.high, mine.low));
    cluster_sync();
    // One warp finds the run; this lane knows the running sums before and after EACH of them.
    constexpr int EACH = kMostCtas * kWarps / 32;
    if (warp == 0) {
      Sum upto[EACH], sum;
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        const int k = lane * EACH + i;
        if (k < a.ctas * kWarps) {
          Sum x;
          x.high = totals[pass][k].x, x.low = totals[pass][k].y;
          sum = sum + x;
        }
        upto[i] = sum;
      }
      const Sum with = running(sum);
      Sum start = up(with, 1);
      if (lane == 0) start = Sum();
#pragma unroll
      for (int i = 0; i < EACH; ++i) upto[i] = start + upto[i];
      const Sum all = from_lane(upto[EACH - 1], 31), goal = all * u;
      int k = -1;
      Sum low;
#pragma unroll
      for (int i = EACH - 1; i >= 0; --i) {  // (a run that counts, as in find())
        const int at = lane * EACH + i;
        if (upto[i] > goal && at < a.ctas * kWarps && totals[pass][at].x > 0.f) k = at, low = i == 0 ? start : upto[i - 1];
      }
      const uint32_t past = __ballot_sync(~0u, k >= 0);
      if (lane == (past ? __ffs(past) - 1 : 0)) {
        picked = past ? k : -1, empty = !(all.high > 0.f);
        bounds[0] = make_float2(low.high, low.low), bounds[1] = make_float2(goal.high, goal.low);
      }
    }
    __syncthreads();
    if (!empty || !row.less) break;
    row.less = false;  // nothing is left of the target: all of it
    __syncthreads();
  }

  const int64_t out = b * (a.drafts + 1);
  if (picked == me) {
    Sum sum, goal;
    sum.high = bounds[0].x, sum.low = bounds[0].y, goal.high = bounds[1].x, goal.low = bounds[1].y;
    // The piece in which that is; the last that has any where rounding hides it.
    int piece = 0;
    Sum start = sum;
    bool found = false;
#pragma unroll
    for (int i = 0; i < kSubs; ++i) {
      const Sum x = over_lanes(pieces[i]), next = sum + x;
      if (!found && x.high > 0.f) piece = i, start = sum, found = next > goal;
      sum = next;
    }
    const int64_t first = begin + piece * a.piece - shift;
    const int token = find<T, LONG>(row, first, first + a.piece, a.vocab, start, goal);
    if (lane == 0) put_token(a, out + stop, token);
  } else if (picked < 0) {
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
  // CTAs of a sequence: enough to fill the GPU, with 2048 tokens each at least.  (Two, four and eight: 256 x 131072 f32 75, 71 and 78 us;
  // 57 x 50021 bf16 27, 20 and 15.)
  a.ctas = 1;
  while (a.ctas < kMostCtas && (int64_t)batch * a.ctas < 152 * 4 && vocab > 2048 * a.ctas) a.ctas *= 2;
  const int warps = a.ctas * kWarps;
// (the last tokens of a row that begins shifted are a group more)
  const int64_t round = (int64_t)warps * kSubs * 32 * kGroup;
  a.piece = (int)((vocab + kGroup - 1 + round - 1) / round) * 32 * kGroup;
  return with_float(dtype, [&](auto t) {
    using T = typename decltype(t)::type;
    const auto kernel = a.piece > kRounds * 32 * kGroup ? verify_kernel<T, true> : verify_kernel<T, false>;
    return launch_clusters("gar_verify_drafts", kernel, (int64_t)batch * a.ctas, a.ctas, kThreads, stream, a);
  });
}
