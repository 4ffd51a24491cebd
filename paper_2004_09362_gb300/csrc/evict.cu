// Cuts the sequences of a cache down to the rows of most weight.
//
// A cluster of CTAs takes a sequence's rows of one head.  A row's key is its weight as an unsigned integer of the same
// order (the largest there is for rows that are kept whatever they weigh, 0 for a NaN), and the keep-th largest key is found by four
// counts of 8 bits each, from the top; among rows of just that key the lowest stay.  Only the rows that have to move
// are copied: a kept row from `keep` on takes the place of one below that goes.  Sources and targets are
// therefore disjoint, and their order does not matter.  The i-th target and the i-th source are listed where
// the outputs' entries from `keep` on will be, which the kernel clears at the end: no more of either than there are rows from
// `keep` on.
//
// Bound by the chain of steps, each with a barrier of the CTA or cluster: 48 sequences of 1025 rows of 8 heads x 128 bf16, one row too many,
// 13 us; 8 sequences of up to 16001 rows of 4 heads x 96 i8, cut to 4000, 39 us, 24 of them the moves.  The keys stay in registers between the
// counts where they fit.
#include <algorithm>
#include <climits>

#include "cluster.cuh"

namespace gar {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMostCtas = 8;  // of a cluster

struct EvictArgs {
  gar_kv_cache c;
  const float *weights;
  const int32_t *positions, *table, *lengths;
  float *out_weights;
  int32_t *out_positions, *out_lengths;
  int64_t rows, table_stride;
  Divide page;
  int most_rows, keep, first, recent, ctas;
  int each;        // rows of a lane
  int units;       // of a key row: what is copied at once
  int lanes;       // power of two: lanes that copy one row's keys and values
  bool apart;      // rows are moved by a kernel of their own
};

// The order of floats as that of integers; 0: a NaN.
__device__ __forceinline__ uint32_t order_of(float x) {
  if (x != x) return 0;
  const uint32_t u = __float_as_uint(x + 0.f);  // (-0 is 0)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The sum of the counts of the warps before this one, and of all.
struct Before {
  int before, all;
};
__device__ __forceinline__ Before count_before(const int *counts, int me, int warps) {
  int x = 0, y = 0;
  for (int k = threadIdx.x & 31; k < warps; k += 32) {
    const int n = counts[k];
    y += n;
    if (k < me) x += n;
  }
  return {__reduce_add_sync(~0u, x), __reduce_add_sync(~0u, y)};
}

// Where a row of the sequence is: its page, and the row in it.
struct Place {
  int page, in;
};
__device__ __forceinline__ Place look_up(const EvictArgs &a, int b, int row) {
  if (row < 0) return {0, -1};
  const int p = (int)a.page((uint32_t)row);
  return {a.table[b * a.table_stride + p], row - p * a.c.page_size};
}
// The place in the cache; false where there is none.
__device__ __forceinline__ bool locate(const EvictArgs &a, int head, Place p, int64_t *at, int64_t *scale) {
  *at = *scale = 0;
  if (p.in < 0) return false;
  if ((unsigned)p.page >= (uint64_t)a.c.pages) {
    if (a.c.status) atomicOr(a.c.status, GAR_KV_BAD_PAGE);
    return false;
  }
  *at = p.page * a.c.page_stride + head * a.c.head_stride + p.in * a.c.token_stride;
  *scale = p.page * a.c.scale_page_stride + head * a.c.scale_head_stride + p.in * a.c.scale_token_stride;
  return true;
}

// Moves some of the `count` rows of the lists behind `keep`: a warp the neighbouring ones from `first` on, then those `step` rows
// further; a.lanes lanes to each, kRows of them on their way at a time.  OWN: the lists may end earlier, and what has been read of them is cleared.
template <typename U, bool OWN>
__device__ __forceinline__ void move_rows(const EvictArgs &a, int b, int head, const float *w, const int32_t *pos, float *out_w,
                                          int32_t *out_p, int keep, int count, int first, int step) {
  constexpr int kRows = 4;
  const int sub = threadIdx.x & (a.lanes - 1), group = (threadIdx.x & 31) / a.lanes;
  const bool scaled = a.c.k_scale != nullptr;
  const int el = a.c.dtype == GAR_F32 ? 4 : a.c.dtype == GAR_I8 || a.c.dtype == GAR_E4M3 ? 1 : 2;
  for (int base = first; base < count; base += step * kRows) {
    const int i0 = base + group;
    int to[kRows], from[kRows];
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      const int i = i0 + k * step;
      to[k] = i < count ? __ldcg(out_p + keep + i) : -1, from[k] = i < count ? __float_as_int(__ldcg(out_w + keep + i)) : -1;
      if (OWN && to[k] < 0) from[k] = -1;
    }
    if (OWN && __all_sync(~0u, to[0] < 0)) break;  // past the lists' ends
    int64_t at_to[kRows], at_from[kRows], scale_to[kRows], scale_from[kRows];
    bool good[kRows];
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      const Place x = look_up(a, b, to[k]), y = look_up(a, b, from[k]);
      good[k] = locate(a, head, x, &at_to[k], &scale_to[k]);
      good[k] = locate(a, head, y, &at_from[k], &scale_from[k]) && good[k];
    }
    for (int u = sub; u < 2 * a.units; u += a.lanes) {
      char *const at = static_cast<char *>(u < a.units ? a.c.k : a.c.v) + (int64_t)(u < a.units ? u : u - a.units) * (int)sizeof(U);
      U x[kRows];
#pragma unroll
      for (int k = 0; k < kRows; ++k)
        if (good[k]) x[k] = *reinterpret_cast<const U *>(at + at_from[k] * el);
#pragma unroll
      for (int k = 0; k < kRows; ++k)
        if (good[k]) *reinterpret_cast<U *>(at + at_to[k] * el) = x[k];
    }
    // A lane for each row's scales, weight and position.
    if (OWN) __syncwarp();
#pragma unroll
    for (int k = 0; k < kRows; ++k)
      if (k % a.lanes == sub) {
        if (to[k] >= 0) {
          if (scaled && good[k]) a.c.k_scale[scale_to[k]] = a.c.k_scale[scale_from[k]], a.c.v_scale[scale_to[k]] = a.c.v_scale[scale_from[k]];
          out_w[to[k]] = w[from[k]], out_p[to[k]] = pos[from[k]];
        }
        if (OWN && to[k] >= 0) out_w[keep + i0 + k * step] = 0.f, out_p[keep + i0 + k * step] = -1;
      }
  }
}

// NK: keys that a lane holds in registers; 0: they are made anew each time.  U: what rows are copied in.
template <int NK, typename U> __global__ void __launch_bounds__(kThreads, 4) evict_kernel(const EvictArgs a) {
  constexpr int WARPS = kMostCtas * kWarps;
  __shared__ int histogram[4][256], total[256], largest[WARPS], counts[3][WARPS];
  __shared__ uint32_t found[4];
  __shared__ int left[4], alike[4];
  const int rank = cluster_rank(), warp = threadIdx.x / 32, lane = threadIdx.x & 31, me = rank * kWarps + warp;
  const int item = blockIdx.x / a.ctas, b = item / a.c.heads, head = item - b * a.c.heads, warps = a.ctas * kWarps;
  const int each = NK ? NK : a.each;
  for (int i = threadIdx.x; i < 4 * 256; i += kThreads) histogram[0][i] = 0;
  const bool alone = a.ctas == 1;
  const auto sync = [&] {
    if (alone)
      __syncthreads();
    else
      cluster_sync();
  };
  sync();
  after_earlier_kernels();

  const float *const w = a.weights + (int64_t)item * a.rows;
  const int32_t *const pos = a.positions + (int64_t)item * a.rows;
  float *const out_w = a.out_weights + (int64_t)item * a.rows;
  int32_t *const out_p = a.out_positions + (int64_t)item * a.rows;
  int n = a.lengths[b];
  if (n < 0 || n > a.most_rows) {
    if (a.c.status) atomicOr(a.c.status, GAR_KV_BAD_LENGTH);
    n = n < 0 ? 0 : a.most_rows;
  }
  const int keep = min(a.keep, n);
  if (head == 0 && rank == 0 && threadIdx.x == 0) a.out_lengths[b] = keep;
  const int row0 = me * each * 32 + lane;  // this lane's rows: 32 apart

  int moved = 0, clear = keep;
  uint32_t stay[NK ? NK : 1] = {};         // (NK > 0) the rows' keys
  if (n > a.keep) {
    int newest = INT_MIN;
    int32_t p[NK ? NK : 1];
    if constexpr (NK > 0) {
#pragma unroll
      for (int j = 0; j < NK; ++j) {
        const int row = row0 + 32 * j;
        stay[j] = row < n ? __float_as_uint(w[row]) : 0, p[j] = row < n ? pos[row] : INT_MIN;
        newest = max(newest, p[j]);
      }
    } else {
      for (int j = 0; j < each; ++j)
        if (row0 + 32 * j < n) newest = max(newest, pos[row0 + 32 * j]);
    }
    if (a.recent > 0) {
      newest = __reduce_max_sync(~0u, newest);
      if (lane < a.ctas) store_in_cta(&largest[me], lane, newest);
      sync();
      newest = INT_MIN;
      for (int k = lane; k < warps; k += 32) newest = max(newest, largest[k]);
      newest = __reduce_max_sync(~0u, newest);
    } else {
      newest = INT_MAX;  // (no position is above it)
    }
    const int64_t old = (int64_t)newest - a.recent;  // positions up to this one are not kept for being recent
    const auto make_key = [&](int row, float weight, int32_t position) {
      return row < a.first || position > old ? 0xffffffffu : order_of(weight);
    };
    if constexpr (NK > 0) {
#pragma unroll
      for (int j = 0; j < NK; ++j) stay[j] = make_key(row0 + 32 * j, __uint_as_float(stay[j]), p[j]);
    }
    const auto key_of = [&](int j) { return NK ? stay[NK ? j : 0] : make_key(row0 + 32 * j, w[row0 + 32 * j], pos[row0 + 32 * j]); };
    const auto each_row = [&](auto f) {
      if constexpr (NK > 0) {
#pragma unroll
        for (int j = 0; j < NK; ++j) f(j, row0 + 32 * j, row0 + 32 * j < n);
      } else {
        for (int j = 0; j < each; ++j) f(j, row0 + 32 * j, row0 + 32 * j < n);
      }
    };

    // The keep-th largest key, 8 bits at a time; `need` rows of it are kept, `same` have it.
    uint32_t threshold = 0;
    int need = a.keep, same = INT_MAX;
#pragma unroll 1
    for (int digit = 0; digit < 4 && need < same; ++digit) {
      const int shift = 24 - 8 * digit;
      const uint32_t above = digit == 0 ? 0 : ~0u << (shift + 8);
      each_row([&](int j, int, bool there) {
        if (!there) return;
        const uint32_t key = key_of(j);
        if (((key ^ threshold) & above) == 0) atomicAdd(&histogram[digit][key >> shift & 255], 1);
      });
      sync();
      if (!alone) {
        // The CTAs' counts, a value to a thread.  (By one warp, 64 reads of other CTAs' memory a lane, this took most of the time.)
        static_assert(kThreads == 256, "a thread for each value");
        int its[kMostCtas], sum = 0;
#pragma unroll
        for (int r = 0; r < kMostCtas; ++r) its[r] = r < a.ctas ? load_from_cta(&histogram[digit][threadIdx.x], r) : 0;
#pragma unroll
        for (int r = 0; r < kMostCtas; ++r) sum += its[r];
        total[threadIdx.x] = sum;
        __syncthreads();
      }
      if (warp == 0) {
        // A lane for 8 values, the largest first.
        int count[8], sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          count[i] = (alone ? histogram[digit] : total)[255 - 8 * lane - i];
          sum += count[i];
        }
        int upto = sum;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
          const int x = __shfl_up_sync(~0u, upto, d);
          if (lane >= d) upto += x;
        }
        if (upto >= need && upto - sum < need) {
          int rest = need - (upto - sum), value = 0, many = 0;
          bool done = false;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (!done && count[i] >= rest) done = true, value = 255 - 8 * lane - i, many = count[i];
            if (!done) rest -= count[i];
          }
          found[digit] = (uint32_t)value << shift, left[digit] = rest, alike[digit] = many;
        }
      }
      __syncthreads();
      threshold |= found[digit], need = left[digit], same = alike[digit];
    }
    // Rows of that key: the lowest `need` stay.  (After fewer than four counts all that begin with its bits do: no key of theirs is
    // below it.)
    Before equal{0, same};
    const bool all = need == same;
    if (!all) {
      int mine = 0;
      each_row([&](int j, int, bool there) { mine += __popc(__ballot_sync(~0u, there && key_of(j) == threshold)); });
      if (lane < a.ctas) store_in_cta(&counts[0][me], lane, mine);
      sync();
      equal = count_before(counts[0], me, warps);
    }
    // Which rows stay; the targets below `keep`, the sources from there on.
    int targets = 0, sources = 0, seen = equal.before;
    const auto stays = [&](int j, bool there) {
      const uint32_t key = there ? key_of(j) : 0;
      const uint32_t its = __ballot_sync(~0u, there && key == threshold);
      const bool yes = there && (key > threshold || (all && key == threshold) || (key == threshold && seen + __popc(its & ((1u << lane) - 1)) < need));
      seen += __popc(its);
      return yes;
    };
    each_row([&](int j, int row, bool there) {
      const bool yes = stays(j, there);
      targets += __popc(__ballot_sync(~0u, there && row < keep && !yes));
      sources += __popc(__ballot_sync(~0u, row >= keep && yes));
    });
    if (lane < a.ctas) store_in_cta(&counts[1][me], lane, targets), store_in_cta(&counts[2][me], lane, sources);
    sync();
    const Before t = count_before(counts[1], me, warps), s = count_before(counts[2], me, warps);
    moved = t.all;
    targets = t.before, sources = s.before, seen = equal.before;
    each_row([&](int j, int row, bool there) {
      const bool yes = stays(j, there), is_target = there && row < keep && !yes, is_source = row >= keep && yes;
      const uint32_t to = __ballot_sync(~0u, is_target), from = __ballot_sync(~0u, is_source), low = (1u << lane) - 1;
      if (is_target) out_p[keep + targets + __popc(to & low)] = row;
      if (is_source) out_w[keep + sources + __popc(from & low)] = __int_as_float(row);
      if (there && row < keep && yes) out_w[row] = w[row], out_p[row] = pos[row];
      targets += __popc(to), sources += __popc(from);
    });
    sync();

    if (a.apart) {
      clear = keep + moved;  // (the lists are cleared as they are read, by the kernel that moves the rows; they end at a -1)
    } else {
      const int per = 32 / a.lanes;
      move_rows<U, false>(a, b, head, w, pos, out_w, out_p, keep, moved, me * per, warps * per);
      sync();
    }
  } else {
    for (int j = 0; j < each; ++j) {
      const int row = row0 + 32 * j;
      if (row < n) out_w[row] = w[row], out_p[row] = pos[row];
    }
  }
  for (int64_t row = clear + (int64_t)rank * kThreads + threadIdx.x; row < a.rows; row += (int64_t)a.ctas * kThreads)
    out_w[row] = 0.f, out_p[row] = -1;
}

// The lists' rows, by `parts` CTAs for each item.
template <typename U> __global__ void __launch_bounds__(kThreads, 4) move_kernel(const EvictArgs a, int parts) {
  after_earlier_kernels();
  const int item = blockIdx.x / parts, part = blockIdx.x - item * parts, b = item / a.c.heads, head = item - b * a.c.heads;
  const int n = min(a.lengths[b], a.most_rows), per = 32 / a.lanes;
  if (n <= a.keep) return;
  const int64_t at = (int64_t)item * a.rows;
  move_rows<U, true>(a, b, head, a.weights + at, a.positions + at, a.out_weights + at, a.out_positions + at, a.keep, n - a.keep,
                     (part * kWarps + (int)threadIdx.x / 32) * per, parts * kWarps * per);
}

}  // namespace
}  // namespace gar

using namespace gar;

extern "C" int gar_kv_evict(const gar_kv_cache *cache, const float *weights, const int32_t *positions, int64_t rows,
                            const int32_t *page_table, int64_t table_stride, int table_width, const int32_t *lengths, int batch,
                            int keep, int first, int recent, float *out_weights, int32_t *out_positions, int32_t *out_lengths,
                            gar_stream_t stream) {
  if (int rc = check_cache(cache)) return rc;
  if (batch < 0 || table_width < 0) return refuse("negative batch or table_width");
  if (rows < 0 || rows > 1 << 24) return refuse("rows must be 0..2^24");
  if (keep < 1 || first < 0 || recent < 0 || (int64_t)first + recent > keep)
    return refuse("keep must be positive, first and recent together no more than it");
  if (batch == 0) return GAR_OK;
  if (lengths == nullptr || out_lengths == nullptr || (page_table == nullptr && table_width > 0) ||
      (rows > 0 && (weights == nullptr || positions == nullptr || out_weights == nullptr || out_positions == nullptr)))
    return refuse("null pointer");
  if ((uintptr_t)weights % 4 || (uintptr_t)positions % 4 || (uintptr_t)page_table % 4 || (uintptr_t)lengths % 4 ||
      (uintptr_t)out_weights % 4 || (uintptr_t)out_positions % 4 || (uintptr_t)out_lengths % 4) {
    set_error("a buffer is not aligned to its elements");
    return GAR_EALIGN;
  }
  if (weights == out_weights || positions == out_positions || lengths == out_lengths) return refuse("an output is an input");
  const int64_t items = (int64_t)batch * cache->heads;
  if (items > INT_MAX / kMostCtas) return refuse("too many sequences and heads");
  EvictArgs a{};
  a.c = *cache;
  a.weights = weights, a.positions = positions, a.table = page_table, a.lengths = lengths;
  a.out_weights = out_weights, a.out_positions = out_positions, a.out_lengths = out_lengths;
  a.rows = rows, a.table_stride = table_stride, a.page = divide_by((uint32_t)cache->page_size);
  a.most_rows = (int)std::min<int64_t>(rows, (int64_t)table_width * cache->page_size);
  a.keep = keep, a.first = first, a.recent = recent;
  // CTAs of an item: enough to fill the GPU with 2048 rows each at least, and so many that the keys fit the registers.  (With 1024 and 4096 rows each:
  // 48 x 1025 of 8 heads 33 and 13.5 us for 13.5, 8 x up to 16001 of 4 heads 37 and 40 for 37, 64 x 4096 of 8 heads 38 and 24 for 38.)
  a.ctas = 1;
  while (a.ctas < kMostCtas && ((items * a.ctas < 152 * 4 && a.most_rows > 2048 * a.ctas) || a.most_rows > 16 * kThreads * a.ctas))
    a.ctas *= 2;
  const int lanes = a.ctas * kThreads;
  a.each = std::max(1, (a.most_rows + lanes - 1) / lanes);
  // Rows are copied in the largest units that all of them are made of.
  const int size = element_size(cache->dtype);
  const uintptr_t all = (uintptr_t)cache->k | (uintptr_t)cache->v | (uintptr_t)(cache->dim * size) |
                        (uintptr_t)(cache->page_stride * size) | (uintptr_t)(cache->head_stride * size) |
                        (uintptr_t)(cache->token_stride * size);
  const auto run = [&](auto unit) {
    using U = typename decltype(unit)::type;
    a.units = cache->dim * size / (int)sizeof(U);
    a.lanes = 1;
    while (a.lanes < 32 && a.lanes < 2 * a.units) a.lanes *= 2;
    // (Keys made anew each time: 48 x 1025 18 us for 13.5, 8 x 16001 55 for 37, 64 x 4096 77 for 38; 8 x 20000 of 8 heads, which need 16 a lane, 50 for 29.)
    const auto kernel = a.each <= 8 ? evict_kernel<8, U> : a.each <= 16 ? evict_kernel<16, U> : evict_kernel<0, U>;
    // Many rows are moved by a kernel of its own, all over the GPU.  (8 x up to 16001 rows cut to 4000, 4 heads x 96 i8: 55 us when this
    // was built, by the clusters that chose them 70; a kernel more costs 2 us where there is one row to move.)
    const int64_t most = std::min(a.most_rows - keep, keep - first), per = kWarps * (32 / a.lanes) * 4;
    a.apart = most > 256;
    if (int rc = launch_clusters("gar_kv_evict", kernel, items * a.ctas, a.ctas, kThreads, stream, a)) return rc;
    if (!a.apart) return (int)GAR_OK;
    const int parts = (int)std::max<int64_t>(1, std::min<int64_t>((most + per - 1) / per, 152 * 4 / items));
    return launch("gar_kv_evict", move_kernel<U>, dim3((unsigned)(items * parts)), kThreads, 0, stream, a, parts);
  };
  if (all % 16 == 0) return run(type_tag<uint4>{});
  if (all % 4 == 0) return run(type_tag<uint32_t>{});
  if (all % 2 == 0) return run(type_tag<uint16_t>{});
  return run(type_tag<uint8_t>{});
}
