// Attention of many queries over a shared prefix, on the tensor cores' own memory.
//
// S = Q K^T of 128 queries (of all the sequences and query heads that read a cached head) by 128 cached rows, then
// P = 2^(S - m) and O += P V: with fewer than some 300 queries for a cached row the rows' way from memory is what it takes, with more
// the products.  A CTA keeps two streams of such tiles going, so that one's products run while the other's weights are computed: two
// blocks of queries over the same rows (pair), or the even and the odd tiles of rows for one block.
//
//  * 2 warps copy the rows, by cp.async since pages may be of any size, to a ring of tiles in shared memory.
//  * A thread for each stream issues its products.  S and O are in tensor memory, 128 columns each.
//  * 4 warps for each stream turn S to P, a query to a thread: no exchange between lanes.  P goes where S was, as two 16-bit parts
//    (its sum is 17 bits or more), 16 columns each for 32 rows.
//  * m is not the running maximum but a number within kLazy of it: O is rescaled only where the maximum passes m + kLazy.
//
// The tiles of all items are shared out among the CTAs as one line.  Each CTA leaves (m, l, O) for its part of
// an item; the parts are joined in their order by the kernel after this.
#include <algorithm>
#include <climits>

#include "decode_mma.cuh"
#include "prefix.cuh"
#include "tcgen05.cuh"

namespace gar {
namespace {

constexpr int kThreads = 32 * 12;  // (more than 12 warps get no more than 128 registers a thread)
enum { kWeights = 0, kCopies = 8, kIssue = 10 };  // first warps of a part of the work
constexpr int kCopyRows = 64;      // of a tile, copied by one warp

template <typename T> struct Parts;
template <> struct Parts<__nv_bfloat16> {
  static constexpr float kLazy = 8.f, kUnit = 0.f;
};
// f16's smallest step, 2^-24, is 2^-34 of m's weight; weights are below 2^15.
template <> struct Parts<__half> {
  static constexpr float kLazy = 5.f, kUnit = 10.f;
};

template <int DP, bool PAIR> struct PrefixShape {
  static constexpr int kTile = kKeys * DP * 2;     // bytes of a tile's keys, or values
  static constexpr int kQueries = (PAIR ? 2 : 1) * kTile;
  static constexpr int kStages = (227 * 1024 - 2048 - kQueries) / kTile < 12 ? (227 * 1024 - 2048 - kQueries) / kTile : 12;
  static constexpr int kShared = kQueries + kStages * kTile + 1024;
  static constexpr int kFlying = kStages - 1;      // tiles on their way
};

// One part of an item: tiles [from, from + tiles) of its rows.
struct PrefixPart {
  int g, kv, block, item, from, tiles, rows;
};
struct PrefixWalk {
  int pos, end, item_at, g, in_group, item, tiles, rows;
  __device__ __forceinline__ void start(const PrefixArgs &a) {
    const int lane = threadIdx.x & 31, items = a.c.heads * a.blocks;
    const int all = prefix_line(a, 0, true).x, per = share_of(all, a.ctas);
    pos = min(all, (int)blockIdx.x * per), end = min(all, pos + per);
    int before = 0;
    g = 0, in_group = 0, rows = tiles = 0;
    if (pos < end)
      for (int g0 = 0;; g0 += 32) {
        // A prefix for each lane; the one that pos is in.
        const int n = g0 + lane < a.groups ? prefix_rows(a, g0 + lane, false) : 0, mine = prefix_tiles(n) * items;
        int upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
          const int x = __shfl_up_sync(~0u, upto, d);
          if (lane >= d) upto += x;
        }
        const uint32_t past = __ballot_sync(~0u, before + upto > pos);
        if (past) {
          const int from = __ffs(past) - 1;
          g = g0 + from, rows = __shfl_sync(~0u, n, from);
          before += __shfl_sync(~0u, upto - mine, from);
          break;
        }
        before += __shfl_sync(~0u, upto, 31);
      }
    tiles = max(1, prefix_tiles(rows));
    in_group = (pos - before) / tiles, item_at = before + in_group * tiles;
    item = g * items + in_group;
  }
  __device__ __forceinline__ bool next(const PrefixArgs &a, PrefixPart *p) {
    if (pos >= end) return false;
    const int items = a.c.heads * a.blocks;
    while (pos >= item_at + tiles) {
      item_at += tiles, ++item;
      if (++in_group < items) continue;
      in_group = 0;
      do {  // (the next prefix that has rows)
        rows = prefix_rows(a, ++g, false), tiles = prefix_tiles(rows);
        if (tiles == 0) item += items;
      } while (tiles == 0);
    }
    p->g = g, p->kv = in_group / a.blocks, p->block = in_group - p->kv * a.blocks, p->item = item;
    p->from = pos - item_at, p->tiles = min(tiles - p->from, end - pos), p->rows = rows;
    pos += p->tiles;
    return true;
  }
};

template <typename T, int DP, bool PAIR> __global__ void __launch_bounds__(kThreads, 1) prefix_kernel(const PrefixArgs a) {
  using S = PrefixShape<DP, PAIR>;
  constexpr int N = S::kStages, ROW = DP * 2, CHUNKS = ROW / 16;
  constexpr bool BF16 = std::is_same<T, __nv_bfloat16>::value;
  extern __shared__ char shared_from[];
  __shared__ __align__(8) uint64_t full[N], empty[N], scores[2], weights[2], values[2], drained[2];
  __shared__ uint32_t tensor_at;
  __shared__ int late_flag;
  const uint32_t shared = (uint32_t)__cvta_generic_to_shared(shared_from) + 1023 & ~1023u;
  char *const shared_p = shared_from + (shared - (uint32_t)__cvta_generic_to_shared(shared_from));
  const uint32_t ring = shared + S::kQueries;
  volatile int *const late = &late_flag;
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const auto at = [](const uint64_t &b) { return (uint32_t)__cvta_generic_to_shared(&b); };
  if (warp == kIssue) tensor_alloc((uint32_t)__cvta_generic_to_shared(&tensor_at));
  if (threadIdx.x == 0) {
    late_flag = 0;
    for (int i = 0; i < N; ++i) init_barrier(at(full[i]), 64), init_barrier(at(empty[i]), PAIR ? 2 : 1);
    for (int s = 0; s < 2; ++s) {
      init_barrier(at(scores[s]), 1), init_barrier(at(weights[s]), 128), init_barrier(at(values[s]), 1);
      init_barrier(at(drained[s]), 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  tensor_before_sync();
  __syncthreads();
  tensor_after_sync();
  const uint32_t tensor = tensor_at;
  after_earlier_kernels();

  PrefixWalk walk;
  walk.start(a);
  PrefixPart part;
  if (warp >= kIssue) {
    // Issues the products of one stream.
    const int s = warp - kIssue;
    const uint32_t s_at = tensor + 256 * s, o_at = s_at + 128;
    constexpr uint32_t scores_kind = product_of(BF16, kKeys, false), values_kind = product_of(BF16, DP, true);
    const uint32_t q_at = shared + (PAIR ? s * S::kTile : 0);
    int done = 0, pos = 0;
    bool good = true;
    while (walk.next(a, &part)) {
      asm volatile("bar.sync 2, 320;" ::: "memory");  // (the queries are there)
      if (lane == 0) {
        for (int j = PAIR ? 0 : s; good && j < part.tiles; j += PAIR ? 1 : 2) {
          const int k = pos + 2 * j, v = k + 1;
          good = j < a.give_up && wait_phase(at(full[k % N]), k / N & 1, late) && (done == 0 || wait_phase(at(values[s]), done - 1 & 1, late));
          if (!good) break;
          tensor_after_sync();
          const uint32_t k_at = ring + k % N * S::kTile, v_at = ring + v % N * S::kTile;
#pragma unroll
          for (int i = 0; i < DP / 16; ++i) {
            const uint32_t off = i / 4 * (kKeys * 128) + i % 4 * 32;
            product(s_at, operand_k_major(q_at + off), operand_k_major(k_at + off), scores_kind, i > 0);
          }
          commit(at(scores[s]));
          commit(at(empty[k % N]));
          good = wait_phase(at(weights[s]), done & 1, late) && wait_phase(at(full[v % N]), v / N & 1, late);
          if (!good) break;
          tensor_after_sync();
#pragma unroll
          for (int i = 0; i < kKeys / 16; ++i) {
            const uint32_t p_at = s_at + i / 2 * 32 + i % 2 * 8;
            const uint64_t b = operand_mn_major(v_at + i * 2048, kKeys * 128);
            product_tensor(o_at, p_at, b, values_kind, j > (PAIR ? 0 : s) || i > 0);
            product_tensor(o_at, p_at + 16, b, values_kind, true);
          }
          commit(at(values[s]));
          commit(at(empty[v % N]));
          ++done;
        }
        if (!good) *late = 1;
      }
      __syncwarp();
      pos += 2 * part.tiles;
    }
    if (lane == 0) {
      // Nothing is on its way any more when the tensor memory is given back.
      int never = 0;
      commit(at(drained[s]));
      wait_phase(at(drained[s]), 0, &never);
    }
    __syncwarp();
  } else if (warp >= kCopies) {
    // Copies tiles: a warp half of the rows of each.
    const int w = warp - kCopies;
    const gar_kv_cache &c = a.c;
    const char *const kp = static_cast<const char *>(c.k), *const vp = static_cast<const char *>(c.v);
    int pos = 0;       // the next tile's place in the ring
    const auto signal = [&](int left) {
      // Of the last kFlying + 1 tiles the oldest but `left` are there.
      if (left == S::kFlying)
        asm volatile("cp.async.wait_group %0;" ::"n"(S::kFlying) : "memory");
      else
        asm volatile("cp.async.wait_group 0;" ::: "memory");
      shared_for_mma();
    };
    int signalled = 0;
    bool good = true;
    constexpr int PER = 32 / CHUNKS;  // rows that the warp copies at a time
    const int chunk = lane % CHUNKS, sub = lane / CHUNKS;
    while (good && walk.next(a, &part)) {
      const auto find = [&](int tile, int half) {
        const int n = (part.from + tile) * kKeys + w * kCopyRows + half * 32 + lane;
        if (tile >= part.tiles || n >= part.rows) return (int64_t)-1;
        const int p = (int)a.page((uint32_t)n), page = a.table[part.g * a.table_stride + p];
        if ((unsigned)page >= (uint64_t)c.pages) {
          if (c.status) atomicOr(c.status, GAR_KV_BAD_PAGE);
          return (int64_t)-1;
        }
        return page * c.page_stride + part.kv * c.head_stride + (n - p * c.page_size) * c.token_stride;
      };
      int64_t row[2] = {find(0, 0), find(0, 1)};
      for (int j = 0; good && j < part.tiles; ++j) {
        const int64_t later[2] = {find(j + 1, 0), find(j + 1, 1)};
#pragma unroll
        for (int half = 0; half < 2; ++half) {  // keys, values
          const int stage = pos % N;
          good = good && (pos < N || wait_phase(at(empty[stage]), (pos / N - 1) & 1, late));
          good = __all_sync(~0u, good);
          if (!good) break;
          const char *const base = half ? vp : kp;
          const uint32_t tile = ring + stage * S::kTile;
#pragma unroll
          for (int r = 0; r < kCopyRows; r += PER) {
            const int to = r + sub, line_row = w * kCopyRows + to;
            const int64_t x = __shfl_sync(~0u, row[r / 32], to & 31);
            const bool in = x >= 0 && chunk * 8 < c.dim;
            copy_async<16>(tile + chunk / 8 * (kKeys * 128) + line_row * 128 + ((chunk ^ line_row) & 7) * 16,
                           in ? base + x * 2 + chunk * 16 : base, in);
          }
          asm volatile("cp.async.commit_group;" ::: "memory");
          ++pos;
          if (pos - signalled > S::kFlying) {
            signal(S::kFlying);
            arrive(at(full[signalled % N]));
            ++signalled;
          }
        }
        row[0] = later[0], row[1] = later[1];
      }
    }
    signal(0);
    if (good)
      for (; signalled < pos; ++signalled) arrive(at(full[signalled % N]));
  } else {
    // Turns scores to weights.
    const int s = warp / 4, quarter = warp & 3, row = quarter * 32 + lane;
    const uint32_t s_at = tensor + 256 * s + ((uint32_t)(quarter * 32) << 16), o_at = s_at + 128;
    int done = 0;
    bool good = true;
    // (After a wait that ran out the barriers of the parts that are left are still met.)
    while (walk.next(a, &part)) {
      asm volatile("bar.sync 1, 256;" ::: "memory");  // (both streams are done with the last part's queries)
      // Queries: row m is that of the prefix's sequence m / heads_each.
      const int row0 = part.block * (PAIR ? 256 : 128), many = min(a.rows - row0, PAIR ? 256 : 128);
      for (int i = threadIdx.x; i < (PAIR ? 256 : 128) * CHUNKS; i += 256) {
        const int r = i / CHUNKS, chunk = i % CHUNKS, m = row0 + r;
        uint4 x = make_uint4(0, 0, 0, 0);
        if (r < many && chunk * 8 < a.c.dim) {
          const int b = (int)a.by_heads((uint32_t)m), h = part.kv * a.heads_each + (m - b * a.heads_each);
          x = *reinterpret_cast<const uint4 *>(static_cast<const char *>(a.q) +
                                               2 * (((int64_t)part.g * a.share + b) * a.qb + h * a.qh) + chunk * 16);
          x.x ^= a.negate, x.y ^= a.negate, x.z ^= a.negate, x.w ^= a.negate;
        }
        *reinterpret_cast<uint4 *>(shared_p + r / 128 * S::kTile + chunk / 8 * (kKeys * 128) + r % 128 * 128 + ((chunk ^ r) & 7) * 16) = x;
      }
      shared_for_mma();
      asm volatile("bar.sync 2, 320;" ::: "memory");

      const bool idle = (PAIR ? s * 128 : 0) + quarter * 32 >= many;  // no query in this warp
      float m = -INFINITY, l = 0.f;
      bool first = true;
      for (int j = PAIR ? 0 : s; good && j < part.tiles; j += PAIR ? 1 : 2) {
        good = __all_sync(~0u, wait_phase(at(scores[s]), done & 1, late));
        if (!good) break;
        ++done;
        tensor_after_sync();
        if (!idle) {
          const int n = part.rows - (part.from + j) * kKeys;  // rows of the tile that exist: n or all
          float top = -INFINITY;
#pragma unroll
          for (int c = 0; c < kKeys; c += 32) {
            uint32_t x[32];
            tensor_load32(x, s_at + c);
            wait_tensor_loads(x);
            float part_top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            if (n - c >= 32) {
#pragma unroll
              for (int i = 0; i < 32; ++i) part_top[i % 4] = fmaxf(part_top[i % 4], __uint_as_float(x[i]));
            } else {
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (c + i < n) part_top[i % 4] = fmaxf(part_top[i % 4], __uint_as_float(x[i]));
            }
            top = fmaxf(top, fmaxf(fmaxf(part_top[0], part_top[1]), fmaxf(part_top[2], part_top[3])));
          }
          top *= a.scale_log2;
          const bool grown = top > m + Parts<T>::kLazy;
          if (__any_sync(~0u, grown)) {
            const float shrink = grown ? exp2_fast(m - top) : 1.f;  // (0 at first)
            if (grown) m = top;
            l *= shrink;
            if (!first) {
#pragma unroll 1
              for (int c = 0; c < DP; c += 32) {
                uint32_t x[32];
                tensor_load32(x, o_at + c);
                wait_tensor_loads(x);
#pragma unroll
                for (int i = 0; i < 32; ++i) x[i] = __float_as_uint(__uint_as_float(x[i]) * shrink);
                tensor_store32(o_at + c, x);
              }
            }
          }
          const float off = Parts<T>::kUnit - offset_of(m);
          float sum[4] = {};
#pragma unroll
          for (int c = 0; c < kKeys; c += 32) {
            uint32_t x[32], y[32];
            tensor_load32(x, s_at + c);
            wait_tensor_loads(x);
            const bool whole = n - c >= 32;
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              float p = exp2_fast(fmaf(__uint_as_float(x[i]), a.scale_log2, off)), q = exp2_fast(fmaf(__uint_as_float(x[i + 1]), a.scale_log2, off));
              if (!whole) p = c + i < n ? p : 0.f, q = c + i + 1 < n ? q : 0.f;
              sum[i % 4] += p, sum[i % 4 + 1] += q;
              split<T>(p, q, &y[i / 2], &y[16 + i / 2]);
            }
            tensor_store32(s_at + c, y);
          }
          l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
          wait_tensor_stores();
        }
        first = false;
        tensor_before_sync();
        arrive(at(weights[s]));
      }
      if (!good) continue;
      // This part's result, in units of one.
      constexpr float unit = Parts<T>::kUnit == 0.f ? 1.f : 1.f / 1024.f;
      const int64_t place = ((int64_t)blockIdx.x + part.item) * 2 + s;
      if (!first) {
        good = __all_sync(~0u, wait_phase(at(values[s]), (done - 1) & 1, late));
        if (!good) continue;
        tensor_after_sync();
      }
      if (!idle) {
        a.ml[place * 128 + row] = make_float2(first ? -INFINITY : m, l * unit);
        if (!first) {
          float4 *const o = reinterpret_cast<float4 *>(a.o) + place * (DP / 4 * 128) + row;
#pragma unroll 1
          for (int c = 0; c < DP; c += 32) {
            uint32_t x[32];
            tensor_load32(x, o_at + c);
            wait_tensor_loads(x);
#pragma unroll
            for (int i = 0; i < 32; i += 4)
              o[(c + i) / 4 * 128] = make_float4(__uint_as_float(x[i]) * unit, __uint_as_float(x[i + 1]) * unit,
                                                 __uint_as_float(x[i + 2]) * unit, __uint_as_float(x[i + 3]) * unit);
          }
        }
      }
      tensor_before_sync();
    }
  }
  tensor_before_sync();
  __syncthreads();
  tensor_after_sync();
  if (warp == kIssue) tensor_free(tensor);
  if (threadIdx.x == 0 && late_flag && a.c.status) atomicOr(a.c.status, GAR_KV_TIMEOUT);
}

constexpr int kJoinThreads = 256, kJoinRows = 32;

// Joins the parts of 32 queries of an item, and their sequences' own rows': a query to a lane, four channels at a time to a warp.
template <int DP> __global__ void __launch_bounds__(kJoinThreads) join_kernel(const PrefixArgs a, const JoinArgs j) {
  after_earlier_kernels();
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, per_item = (a.pair ? 256 : 128) / kJoinRows;
  const int item = blockIdx.x / per_item, items = a.c.heads * a.blocks, g = item / items, in_group = item - g * items;
  const int kv = in_group / a.blocks, block = in_group - kv * a.blocks;
  const int in_block = (blockIdx.x - item * per_item) * kJoinRows, row = block * (a.pair ? 256 : 128) + in_block + lane;
  if (row - lane >= a.rows) return;
  const int2 line = prefix_line(a, g, false);
  const int per = share_of(line.x, a.ctas), tiles = prefix_tiles(prefix_rows(a, g, false)), begin = line.y + in_group * tiles;
  const int first = tiles ? begin / per : 0, parts = tiles ? (begin + tiles - 1) / per - first + 1 : 0;
  const int subs = a.pair ? 1 : 2, sub0 = a.pair ? in_block / 128 : 0, in_sub = in_block % 128 + lane;
  const bool there = row < a.rows;
  const int i = (int)a.by_heads((uint32_t)min(row, a.rows - 1)), h = kv * a.heads_each + (min(row, a.rows - 1) - i * a.heads_each);
  const int64_t b = (int64_t)g * a.share + i, own_at = b * j.heads + h;
  const float own = __ldcg(j.parts[0].lse + own_at) * 1.44269504088896341f;
  const float2 *const ml = a.ml + ((int64_t)first + item) * 256 + sub0 * 128 + in_sub;
  float top = own;
  for (int p = 0; p < parts; ++p)
    for (int s = 0; s < subs; ++s) top = fmaxf(top, __ldcg(ml + p * 256 + s * 128).x);
  const float off = offset_of(top), own_weight = exp2_fast(own - off);
  float l = own_weight;
  for (int p = 0; p < parts; ++p)
    for (int s = 0; s < subs; ++s) {
      const float2 x = __ldcg(ml + p * 256 + s * 128);
      l += exp2_fast(x.x - off) * x.y;
    }
  const float inverse = l == 0.f ? 0.f : 1.f / l;
  if (warp == 0 && there && j.lse) j.lse[own_at] = l == 0.f ? -INFINITY : (off + log2f(l)) * 0.693147180559945f;
  for (int d = warp * 4; d < j.dim; d += kJoinThreads / 32 * 4) {
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    const float *const q = j.parts[0].out + own_at * j.parts[0].row + d;
    if (own_weight > 0.f || own_weight != own_weight) {
      const float4 y = __ldcg(reinterpret_cast<const float4 *>(q));
      x.x = own_weight * y.x, x.y = own_weight * y.y, x.z = own_weight * y.z, x.w = own_weight * y.w;
    }
    const float4 *const o = reinterpret_cast<const float4 *>(a.o) + (((int64_t)first + item) * 2 + sub0) * (DP / 4 * 128) + d / 4 * 128 + in_sub;
#pragma unroll 4
    for (int p = 0; p < parts * subs; ++p) {
      const int at = subs == 2 ? p : 2 * p;
      const float2 v = __ldcg(ml + at * 128);
      const float f = exp2_fast(v.x - off);
      const float4 y = __ldcg(o + (int64_t)at * (DP / 4 * 128));
      if (!(f == 0.f)) x.x += f * y.x, x.y += f * y.y, x.z += f * y.z, x.w += f * y.w;
    }
    x.x *= inverse, x.y *= inverse, x.z *= inverse, x.w *= inverse;
    if (!there) continue;
    const int64_t at = b * j.ob + h * j.oh + d;
    const float z[4] = {x.x, x.y, x.z, x.w};
    if (j.out_dtype == GAR_F32) {
      float *const out = static_cast<float *>(j.out) + at;
      if (j.wide)
        *reinterpret_cast<float4 *>(out) = x;
      else
        for (int k = 0; k < 4 && d + k < j.dim; ++k) out[k] = z[k];
    } else if (j.wide) {
      const uint2 y = j.out_dtype == GAR_BF16 ? make_uint2(pack2(make_float2(x.x, x.y), __nv_bfloat16()), pack2(make_float2(x.z, x.w), __nv_bfloat16()))
                                              : make_uint2(pack2(make_float2(x.x, x.y), __half()), pack2(make_float2(x.z, x.w), __half()));
      *reinterpret_cast<uint2 *>(static_cast<char *>(j.out) + 2 * at) = y;
    } else {
      for (int k = 0; k < 4 && d + k < j.dim; ++k) {
        if (j.out_dtype == GAR_BF16)
          static_cast<__nv_bfloat16 *>(j.out)[at + k] = from_f32<__nv_bfloat16>(z[k]);
        else
          static_cast<__half *>(j.out)[at + k] = from_f32<__half>(z[k]);
      }
    }
  }
}

template <typename T, int DP, bool PAIR> int launch_prefix(const PrefixArgs &a, gar_stream_t stream) {
  constexpr auto kernel = prefix_kernel<T, DP, PAIR>;
  static DeviceSet allowed;
  const int e = once_for_device(allowed, a.device, [&] {
    return (int)cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, PrefixShape<DP, PAIR>::kShared);
  });
  if (e != 0) return cuda_fail((cudaError_t)e, "cudaFuncSetAttribute");
  return launch("gar_prefix_attention", kernel, a.ctas, kThreads, PrefixShape<DP, PAIR>::kShared, stream, a);
}

}  // namespace

size_t prefix_partials(int items, int dim, char *base, PrefixArgs *a) {
  const int dp = dim <= 64 ? 64 : 128;
  const size_t places = (size_t)items + 152, sums = places * 256 * sizeof(float2);
  if (a) a->ml = reinterpret_cast<float2 *>(base), a->o = reinterpret_cast<float *>(base + sums);
  return sums + places * 256 * dp * sizeof(float);
}

int prefix_mma(const PrefixArgs &a, gar_stream_t stream) {
  const auto run = [&](auto t) {
    using T = typename decltype(t)::type;
    if (a.c.dim <= 64) return a.pair ? launch_prefix<T, 64, true>(a, stream) : launch_prefix<T, 64, false>(a, stream);
    return a.pair ? launch_prefix<T, 128, true>(a, stream) : launch_prefix<T, 128, false>(a, stream);
  };
  return a.c.dtype == GAR_BF16 ? run(type_tag<__nv_bfloat16>{}) : run(type_tag<__half>{});
}

int join_partials(const PrefixArgs &a, const JoinArgs &j, gar_stream_t stream) {
  const int64_t blocks = (int64_t)a.groups * a.c.heads * a.blocks * ((a.pair ? 256 : 128) / kJoinRows);
  return launch("gar_prefix_attention", a.c.dim <= 64 ? join_kernel<64> : join_kernel<128>, blocks, kJoinThreads, 0, stream, a, j);
}

}  // namespace gar
