// Attention of many queries over a shared prefix, on the tensor cores' own memory.
//
// S = Q K^T of 128 queries (of all the sequences and query heads that read a cached head) by 128 cached rows, then
// P = 2^(S - m) and O += P V.  A CTA keeps two streams of such tiles going, so that one's products run while the other's weights are
// computed: two blocks of queries over the same rows (pair), or the even and the odd tiles of rows for one block.
//
//  * 4 warps copy the rows to a ring of tiles in shared memory: boxes of pages by tensor copies where tiles are whole pages or pages
//    whole tiles, cp.async for pages of any other size and for last tiles, whose rows past the end have to be zeros.
//    (131072 rows, one block, when this was built: 117 us with boxes of 64 rows, 131 with cp.async.  A lane's tensor copy takes some 190 clocks to issue.)
//  * A thread for each stream issues its products.  S and O are in tensor memory, 128 columns each.  S is computed by halves of 64 rows, the
//    next half's while the weights of one are computed (16384 rows x 1000 queries: 171 us a call, with whole tiles 180).
//  * 4 warps for each stream turn S to P, a query to a thread: no exchange between lanes.  P goes where S was, as two 16-bit parts
//    (2^-17 of the weight in bf16; one part alone would be 2^-9, as much as the output's rounding, and saved a tenth), 16 columns each for
//    32 rows.  These warps have 192 registers, the others 64: a half's scores fit them.
//  * The tensor cores cut their sums off rather than round them: 2^-24 and more of the sum for each of 16 products a tile, all one way (parts
//    of 1024 tiles came out 1.6e-3 short, of 54 tiles 3e-5).  So O holds 16 tiles at most, and is then added to the part's result in
//    memory, rounded: less than 2^-15 is missing (2e-5 measured).  (8 tiles, by reductions in the L2: 1e-5, and 40 us more of 150.)
//  * m is not the running maximum but a number within kLazy of it: O is rescaled only where the maximum passes m + kLazy.
//
// The tiles of all items are shared out among the CTAs as one line.  Each CTA leaves (m, l, O) for its part of
// an item; the parts are joined in their order by the kernel after this.
//
// Bound, with few queries, by the rows' way from memory: 32 sequences of 32/8 heads x 128 bf16 over 131072 rows 112 us, 4.8 TB/s.  With many, 250
// sequences over 16384 rows f16, 105 us: 0.64 PFLOP/s of S and P V, 0.97 counting both parts of P.  There a pair of tiles takes
// 6200 clocks, of which its products take 4700 alone (3100 at the peak rate) and its weights 4400; leaving the exponentials, the
// parts or the stores out changed little, so what remains is that products and weights hardly overlap.  The first 12 us of a
// launch are the pages, the queries and the first copies, one after the other, and the instructions.
#include <algorithm>
#include <climits>

#include "decode_mma.cuh"
#include "prefix.cuh"
#include "tcgen05.cuh"

namespace gar {
namespace {

constexpr int kThreads = 32 * 16;  // at 128 registers; the weights' 8 warps take 64 of them from each thread of the others
enum { kWeights = 0, kCopies = 8, kIssue = 12 };  // first warps of a part of the work
constexpr int kSpan = 32;           // halves of tiles that the tensor cores add up
constexpr int kCopyRows = 32;      // of a tile, copied by one warp

template <typename T> struct Parts;
template <> struct Parts<__nv_bfloat16> {
  static constexpr float kLazy = 8.f, kUnit = 0.f;
};
// f16's smallest step, 2^-24, is 2^-34 of m's weight; weights are below 2^15.
template <> struct Parts<__half> {
  static constexpr float kLazy = 5.f, kUnit = 10.f;
};

// Two weights as a high and a low part each, both rounded: the high one is off by 2^-9 of the weight (bf16), the low one by 2^-8 of that.
__device__ __forceinline__ void split_weights(float2 p, uint32_t *hi, uint32_t *lo, __nv_bfloat16) {
  *hi = pack2(p, __nv_bfloat16());
  *lo = pack2(fma2(unpack2(*hi, __nv_bfloat16()), make_float2(-1.f, -1.f), p), __nv_bfloat16());
}
__device__ __forceinline__ void split_weights(float2 p, uint32_t *hi, uint32_t *lo, __half) {
  *hi = pack2(p, __half());
  *lo = pack2(fma2(unpack2(*hi, __half()), make_float2(-1.f, -1.f), p), __half());
}

// One line of a box of rows of the cache.
__device__ __forceinline__ void copy_line(uint32_t to, const CUtensorMap *map, int row, int line, int head, int page, uint32_t barrier) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], "
      "[%7];" ::"r"(to), "l"(map), "r"(0), "r"(row), "r"(line), "r"(head), "r"(page), "r"(barrier)
      : "memory");
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

template <int DP, bool PAIR> struct PrefixShape {
  static constexpr int kTile = kKeys * DP * 2;     // bytes of a tile's keys, or values
  static constexpr int kQueries = (PAIR ? 2 : 1) * kTile;
  static constexpr int kStages = (227 * 1024 - 2048 - kQueries) / kTile < 12 ? (227 * 1024 - 2048 - kQueries) / kTile : 12;
  static_assert(PAIR || kStages % 2 == 0, "two rings");
  static constexpr int kShared = kQueries + kStages * kTile + 1024;
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

template <typename T, int DP, bool PAIR> __global__ void __launch_bounds__(kThreads, 1)
    prefix_kernel(const PrefixArgs a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
  using S = PrefixShape<DP, PAIR>;
  // The ring's stages: both streams read each tile of it, or each stream has half of the stages for its own.  (With one ring
  // for both, a stream that is a lap ahead of the other would take that one's tile, not there yet, for its own: a barrier tells a phase
  // from the next, but not from the one after that.)
  constexpr int N = S::kStages, RING = PAIR ? N : N / 2, ROW = DP * 2, CHUNKS = ROW / 16;
  constexpr bool BF16 = std::is_same<T, __nv_bfloat16>::value;
  extern __shared__ char shared_from[];
  __shared__ __align__(8) uint64_t full[N], empty[N], scores[2][2], weights[2][2], values[2], drained[2];
  __shared__ uint32_t tensor_at;
  __shared__ int late_flag, copied[2];
  const uint32_t shared = (uint32_t)__cvta_generic_to_shared(shared_from) + 1023 & ~1023u;
  char *const shared_p = shared_from + (shared - (uint32_t)__cvta_generic_to_shared(shared_from));
  const uint32_t ring = shared + S::kQueries;
  volatile int *const late = &late_flag;
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const auto at = [](const uint64_t &b) { return (uint32_t)__cvta_generic_to_shared(&b); };
  if (warp == kIssue) tensor_alloc((uint32_t)__cvta_generic_to_shared(&tensor_at));
  if (threadIdx.x == 0) {
    late_flag = 0;
    for (int i = 0; i < N; ++i) init_barrier(at(full[i]), a.box > 0 ? 4 : 128), init_barrier(at(empty[i]), PAIR ? 2 : 1);
    for (int s = 0; s < 2; ++s) {
      init_barrier(at(scores[s][0]), 1), init_barrier(at(scores[s][1]), 1), init_barrier(at(values[s]), 1);
      init_barrier(at(weights[s][0]), 4), init_barrier(at(weights[s][1]), 4);
      init_barrier(at(drained[s]), 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  tensor_before_sync();
  __syncthreads();
  tensor_after_sync();
  const uint32_t tensor = tensor_at;
  after_earlier_kernels();

  // Each warp's walk, kept out of the registers between parts.
  __shared__ PrefixWalk walks[kThreads / 32];
  {
    PrefixWalk walk;
    walk.start(a);
    if (lane == 0) walks[warp] = walk;
    __syncwarp();
  }
  PrefixPart part;
  const auto next_part = [&] {
    PrefixWalk walk = walks[warp];
    const bool is = walk.next(a, &part);
    __syncwarp();
    if (lane == 0) walks[warp] = walk;
    __syncwarp();
    return is;
  };
  if (warp >= kCopies)
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
  else
    asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
  if (warp >= kIssue + 2) {
    // (two warps fill up the fourth warpgroup)
  } else if (warp >= kIssue) {
    // Issues the products of one stream.
    const int s = warp - kIssue;
    const uint32_t s_at = tensor + 256 * s, o_at = s_at + 128;
    constexpr uint32_t scores_kind = product_of(BF16, kKeys / 2, false), values_kind = product_of(BF16, DP, true);
    const uint32_t q_at = shared + (PAIR ? s * S::kTile : 0);
    const int stage0 = PAIR ? 0 : s * RING;
    // done: halves of tiles whose values are added; pos: the stream's first tile of keys or values that is not done with.
    int done = 0, pos = 0;
    bool good = true;
    while (next_part()) {
      asm volatile("bar.sync 2, 320;" ::: "memory");  // (the queries are there)
      if (lane == 0) {
        constexpr int STEP = PAIR ? 1 : 2;
        const int first = PAIR ? 0 : s, halves = part.tiles > first ? 2 * ((part.tiles - first + STEP - 1) / STEP) : 0;
        // The scores of the part's i-th half of a tile: keys of tile i / 2, of which every second in the ring is one.
        const auto scores_of = [&](int i) {
          const int at_pos = pos + i / 2 * 2, k = stage0 + at_pos % RING;
          if (i % 2 == 0) {
            if (first + i / 2 * STEP >= a.give_up || !wait_phase(at(full[k]), at_pos / RING & 1, late)) return false;
            shared_for_mma();
          }
          tensor_after_sync();
          const uint32_t k_at = ring + k * S::kTile + i % 2 * (kKeys / 2 * 128);
#pragma unroll
          for (int x = 0; x < DP / 16; ++x) {
            const uint32_t off = x / 4 * (kKeys * 128) + x % 4 * 32;
            product(s_at + i % 2 * (kKeys / 2), operand_k_major(q_at + off), operand_k_major(k_at + off), scores_kind, x > 0);
          }
          commit(at(scores[s][i % 2]));
          if (i % 2) commit(at(empty[k]));
          return true;
        };
        if (good && halves > 0) good = scores_of(0) && scores_of(1);
        for (int i = 0; good && i < halves; ++i) {
          const int at_pos = pos + i / 2 * 2 + 1, v = stage0 + at_pos % RING;
          const uint32_t v_at = ring + v * S::kTile;
          if (i % 2 == 0) {
            good = wait_phase(at(full[v]), at_pos / RING & 1, late);
            shared_for_mma();
          }
          good = good && wait_phase(at(weights[s][i % 2]), done / 2 & 1, late);
          if (!good) break;
          tensor_after_sync();
#pragma unroll
          for (int x = 0; x < kKeys / 32; ++x) {
            const int y = i % 2 * (kKeys / 32) + x;
            const uint32_t p_at = s_at + y / 2 * 32 + y % 2 * 8;
            const uint64_t b = operand_mn_major(v_at + y * 2048, kKeys * 128);
            product_tensor(o_at, p_at, b, values_kind, i % kSpan > 0 || x > 0);
            product_tensor(o_at, p_at + 16, b, values_kind, true);
          }
          commit(at(values[s]));
          if (i % 2) commit(at(empty[v]));
          ++done;
          // The next scores but one go where these weights are: a thread's products run in the order that they are issued in.
          if (i + 2 < halves) good = scores_of(i + 2);
        }
        pos += halves;
        if (!good) *late = 1;
      }
      __syncwarp();
    }
    if (lane == 0) {
      // Nothing is on its way any more when the tensor memory is given back.
      int never = 0;
      commit(at(drained[s]));
      wait_phase(at(drained[s]), 0, &never);
    }
    __syncwarp();
  } else if (warp >= kCopies) {
    // Copies tiles: a warp a quarter of the rows of each.
    const int w = warp - kCopies;
    const gar_kv_cache &c = a.c;
    const char *const kp = static_cast<const char *>(c.k), *const vp = static_cast<const char *>(c.v);
    int pos[2] = {0, 0};  // the next tile of keys or values, of each ring
    bool good = true;
    constexpr int PER = 32 / CHUNKS;  // rows that the warp copies at a time
    const int chunk = lane % CHUNKS, sub = lane / CHUNKS;
    while (good && next_part()) {
      // Pages are looked up a tile before they are used, and checked only then.
      struct Found {
        int page, in;  // in: the row of the page, or -1
      };
      const auto place = [&](Found f) {
        if (f.in < 0) return (int64_t)-1;
        if ((unsigned)f.page >= (uint64_t)c.pages) {
          if (c.status) atomicOr(c.status, GAR_KV_BAD_PAGE);
          return (int64_t)-1;
        }
        return f.page * c.page_stride + part.kv * c.head_stride + f.in * c.token_stride;
      };
      // Whole tiles go in boxes where pages allow it: the page of this lane's box and the row in it.
      const int boxes = a.box > 0 ? kKeys / a.box : 1, box = lane % boxes, line = lane / boxes;
      const auto in_boxes = [&](int tile) { return a.box > 0 && (part.from + tile + 1) * kKeys <= part.rows; };
      const auto look_any = [&](int tile) {
        const int n = (part.from + tile) * kKeys + (in_boxes(tile) ? box * a.box : w * kCopyRows + lane);
        Found f{0, -1};
        if (tile < part.tiles && n < part.rows) {
          const int p = (int)a.page((uint32_t)n);
          f.page = a.table[part.g * a.table_stride + p], f.in = n - p * c.page_size;
        }
        return f;
      };
      Found found = look_any(0);
      for (int j = 0; good && j < part.tiles; ++j) {
        const Found now = found;
        found = look_any(j + 1);
        if (in_boxes(j)) {
          // One line (128 bytes) of a box's rows to a lane.  What is on no page becomes zeros.
          if (w == 0 && (unsigned)now.page >= (uint64_t)c.pages && c.status) atomicOr(c.status, GAR_KV_BAD_PAGE);
#pragma unroll 1
          for (int half = 0; half < 2; ++half) {
            int &its = PAIR || j % 2 == 0 ? pos[0] : pos[1];
            const int stage = (PAIR ? 0 : j % 2 * RING) + its % RING;
            good = good && (its < RING || wait_phase(at(empty[stage]), (its / RING - 1) & 1, late));
            good = __all_sync(~0u, good);
            if (!good) break;
            if (w == 0) {
              if (lane == 0)
                asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(at(full[stage])), "r"(S::kTile) : "memory");
              __syncwarp();
              if (line < DP / 64)
                copy_line(ring + stage * S::kTile + line * (kKeys * 128) + box * (a.box * 128), half ? &v_map : &k_map, now.in, line,
                          part.kv, now.page, at(full[stage]));
            } else if (lane == 0) {
              arrive(at(full[stage]));
            }
            ++its;
          }
          continue;
        }
        const int64_t row = place(now);
#pragma unroll
        for (int half = 0; half < 2; ++half) {  // keys, values
          int &its = PAIR || j % 2 == 0 ? pos[0] : pos[1];
          const int stage = (PAIR ? 0 : j % 2 * RING) + its % RING;
          good = good && (its < RING || wait_phase(at(empty[stage]), (its / RING - 1) & 1, late));
          good = __all_sync(~0u, good);
          if (!good) break;
          const char *const base = half ? vp : kp;
          const uint32_t tile = ring + stage * S::kTile;
#pragma unroll
          for (int r = 0; r < kCopyRows; r += PER) {
            const int to = r + sub, line_row = w * kCopyRows + to;
            const int64_t x = __shfl_sync(~0u, row, to);
            const bool in = x >= 0 && chunk * 8 < c.dim;
            copy_async<16>(tile + chunk / 8 * (kKeys * 128) + line_row * 128 + ((chunk ^ line_row) & 7) * 16,
                           in ? base + x * 2 + chunk * 16 : base, in);
          }
          if (a.box > 0) {  // (a last tile after boxes)
            asm volatile("cp.async.wait_all;" ::: "memory");
            shared_for_mma();
            __syncwarp();
            if (lane == 0) arrive(at(full[stage]));
          } else {
            arrive_after_copies(at(full[stage]));
          }
          ++its;
        }
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (threadIdx.x == 32 * kCopies) copied[0] = pos[0], copied[1] = pos[1];
  } else {
    // Turns scores to weights.
    const int s = warp / 4, quarter = warp & 3, row = quarter * 32 + lane;
    const uint32_t s_at = tensor + 256 * s + ((uint32_t)(quarter * 32) << 16), o_at = s_at + 128;
    int done = 0;
    bool good = true;
    // (After a wait that ran out the barriers of the parts that are left are still met.)
    while (next_part()) {
      asm volatile("bar.sync 1, 256;" ::: "memory");  // (both streams are done with the last part's queries)
      // Queries: row m is that of the prefix's sequence m / heads_each.
      const int row0 = part.block * (PAIR ? 256 : 128), many = min(a.rows - row0, PAIR ? 256 : 128);
      constexpr int ALL = (PAIR ? 256 : 128) * CHUNKS / 256, AT_ONCE = 8;
      static_assert(ALL % 4 == 0, "whole rounds");
#pragma unroll 1
      for (int i0 = 0; i0 < ALL; i0 += ALL < AT_ONCE ? ALL : AT_ONCE) {
        uint4 x[ALL < AT_ONCE ? ALL : AT_ONCE];
#pragma unroll
        for (int i = 0; i < (ALL < AT_ONCE ? ALL : AT_ONCE); ++i) {
          const int at_chunk = (i0 + i) * 256 + threadIdx.x, r = at_chunk / CHUNKS, chunk = at_chunk % CHUNKS, m = row0 + r;
          x[i] = make_uint4(0, 0, 0, 0);
          if (r < many && chunk * 8 < a.c.dim) {
            const int b = (int)a.by_heads((uint32_t)m), h = part.kv * a.heads_each + (m - b * a.heads_each);
            x[i] = *reinterpret_cast<const uint4 *>(static_cast<const char *>(a.q) +
                                                    2 * (((int64_t)part.g * a.share + b) * a.qb + h * a.qh) + chunk * 16);
          }
        }
#pragma unroll
        for (int i = 0; i < (ALL < AT_ONCE ? ALL : AT_ONCE); ++i) {
          const int at_chunk = (i0 + i) * 256 + threadIdx.x, r = at_chunk / CHUNKS, chunk = at_chunk % CHUNKS;
          x[i].x ^= a.negate, x[i].y ^= a.negate, x[i].z ^= a.negate, x[i].w ^= a.negate;
          *reinterpret_cast<uint4 *>(shared_p + r / 128 * S::kTile + chunk / 8 * (kKeys * 128) + r % 128 * 128 + ((chunk ^ r) & 7) * 16) = x[i];
        }
      }
      shared_for_mma();
      asm volatile("bar.sync 2, 320;" ::: "memory");

      const bool idle = (PAIR ? s * 128 : 0) + quarter * 32 >= many;  // no query in this warp
      float m = -INFINITY, l = 0.f;
      // The part's result, in units of one: what O holds comes to what it held before, which was relative to m_before.
      constexpr float unit = Parts<T>::kUnit == 0.f ? 1.f : 1.f / 1024.f;
      const int64_t place = ((int64_t)blockIdx.x + part.item) * 2 + s;
      float4 *const result = reinterpret_cast<float4 *>(a.o) + place * (DP / 4 * 128) + row;
      float m_before = -INFINITY;
      bool fresh = true;
      const auto add_up = [&] {
        const float f = fresh ? 0.f : exp2_fast(m_before - offset_of(m));
#pragma unroll 1
        for (int c = 0; c < DP; c += 32) {
          float4 *const to = result + c / 4 * 128;
          float4 z[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) z[i] = fresh ? make_float4(0.f, 0.f, 0.f, 0.f) : __ldcg(to + i * 128);
          uint32_t x[32];
          tensor_load32(x, o_at + c);
          wait_tensor_loads(x);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            __stcg(to + i * 128, make_float4(fmaf(z[i].x, f, __uint_as_float(x[4 * i]) * unit), fmaf(z[i].y, f, __uint_as_float(x[4 * i + 1]) * unit),
                                             fmaf(z[i].z, f, __uint_as_float(x[4 * i + 2]) * unit), fmaf(z[i].w, f, __uint_as_float(x[4 * i + 3]) * unit)));
        }
        fresh = false, m_before = m;
      };
      const int first_tile = PAIR ? 0 : s, step = PAIR ? 1 : 2;
      const int halves = part.tiles > first_tile ? 2 * ((part.tiles - first_tile + step - 1) / step) : 0;
#pragma unroll 1
      for (int i = 0; good && i < halves; ++i) {
        const uint32_t half_at = s_at + i % 2 * (kKeys / 2);
        good = __all_sync(~0u, wait_phase(at(scores[s][i % 2]), done / 2 & 1, late));
        if (!good) break;
        tensor_after_sync();
        if (!idle && i > 0 && i % kSpan == 0) {
          // (the values before these have been added; those before them had been when the scores were there)
          good = __all_sync(~0u, wait_phase(at(values[s]), (done - 1) & 1, late));
          if (!good) break;
          tensor_after_sync();
          add_up();
        }
        if (!idle) {
          const int n = part.rows - (part.from + first_tile + i / 2 * step) * kKeys - i % 2 * (kKeys / 2);  // rows that exist: n or all
          uint32_t x[2][32];
          tensor_load32(x[0], half_at);
          tensor_load32(x[1], half_at + 32);
          wait_tensor_loads(x[0]);
          loaded(x[1]);
          if (n < kKeys / 2) {
#pragma unroll
            for (int k = 0; k < kKeys / 2; ++k)
              if (k >= n) x[k / 32][k % 32] = 0xff800000u;  // -infinity: its weight is 0
          }
          float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int k = 0; k < 32; k += 4)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const uint32_t *const y = &x[c / 2][k + c % 2 * 2];
              tops[c] = max3(tops[c], __uint_as_float(y[0]), __uint_as_float(y[1]));
            }
          const float top = fmaxf(max3(tops[0], tops[1], tops[2]), tops[3]) * a.scale_log2;
          const bool grown = top > m + Parts<T>::kLazy;
          if (__any_sync(~0u, grown)) {
            const float shrink = grown ? exp2_fast(m - top) : 1.f;  // (0 at first)
            if (grown) m = top;
            l *= shrink;
            if (i % kSpan > 0) {
              good = __all_sync(~0u, wait_phase(at(values[s]), (done - 1) & 1, late));
              if (!good) break;
              tensor_after_sync();
#pragma unroll 1
              for (int c = 0; c < DP; c += 8) {
                uint32_t y[8];
                tensor_load8(y, o_at + c);
#pragma unroll
                for (int k = 0; k < 8; ++k) y[k] = __float_as_uint(__uint_as_float(y[k]) * shrink);
                tensor_store8(o_at + c, y);
              }
            }
          }
          const float off = Parts<T>::kUnit - offset_of(m);
          const float2 scale2 = make_float2(a.scale_log2, a.scale_log2), off2 = make_float2(off, off);
          float2 sum[2] = {};
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t y[32];
#pragma unroll
            for (int k = 0; k < 32; k += 2) {
              float2 p = fma2(make_float2(__uint_as_float(x[c][k]), __uint_as_float(x[c][k + 1])), scale2, off2);
              p.x = exp2_fast(p.x), p.y = exp2_fast(p.y);
              sum[k / 2 % 2] = add2(sum[k / 2 % 2], p);
              split_weights(p, &y[k / 2], &y[16 + k / 2], T());
            }
            tensor_store32(half_at + 32 * c, y);
          }
          l += (sum[0].x + sum[1].x) + (sum[0].y + sum[1].y);
          wait_tensor_stores();
        }
        if (i == halves - 1) {
          // The last products but one.  They are waited for before this warp arrives, as the last cannot end until it does: a barrier tells whether
          // the latest of its phases is the one asked for, and once the last has ended, a wait for the one before does not end.
          good = __all_sync(~0u, wait_phase(at(values[s]), (done - 1) & 1, late));
          if (!good) break;
        }
        ++done;
        tensor_before_sync();
        __syncwarp();
        if (lane == 0) arrive(at(weights[s][i % 2]));
        __syncwarp();
      }
      const bool first = halves == 0;
      if (!good) continue;
      if (!first) {
        good = __all_sync(~0u, wait_phase(at(values[s]), (done - 1) & 1, late));
        if (!good) continue;
        tensor_after_sync();
      }
      if (!idle) {
        a.ml[place * 128 + row] = make_float2(first ? -INFINITY : m, l * unit);
        if (!first) add_up();
      }
      tensor_before_sync();
    }
  }
  tensor_before_sync();
  __syncthreads();
  tensor_after_sync();
  if (warp == kIssue) tensor_free(tensor);
  if (late_flag && threadIdx.x == 32 * kCopies) {
    if (a.c.status) atomicOr(a.c.status, GAR_KV_TIMEOUT);
    // What is on its way lands before the CTA's memory is another's.
    int never = 0;
    for (int s = 0; s < (PAIR ? 1 : 2); ++s)
      for (int i = max(0, copied[s] - RING); i < copied[s]; ++i) wait_phase(at(full[s * RING + i % RING]), i / RING & 1, &never);
  }
}

constexpr int kJoinThreads = 256, kJoinRows = 32, kJoinChannels = 16;

// Joins the parts of 32 queries of an item and their sequences' own rows' results, for 16 channels: a query to a lane, four
// channels of half the parts to a warp.
template <int DP> __global__ void __launch_bounds__(kJoinThreads) join_kernel(const PrefixArgs a, const JoinArgs j) {
  extern __shared__ float factors[];  // [part][query]: what the part counts for
  __shared__ float tops[kJoinThreads / 32][32], sums[kJoinThreads / 32][32];
  __shared__ float4 others[4][32];
  after_earlier_kernels();
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, per_item = (a.pair ? 256 : 128) / kJoinRows;
  const int item = blockIdx.x / per_item, items = a.c.heads * a.blocks, g = item / items, in_group = item - g * items;
  const int kv = in_group / a.blocks, block = in_group - kv * a.blocks;
  const int in_block = (blockIdx.x - item * per_item) * kJoinRows, row = block * (a.pair ? 256 : 128) + in_block + lane;
  if (row - lane >= a.rows) return;
  const int2 line = prefix_line(a, g, false);
  const int per = share_of(line.x, a.ctas), tiles = prefix_tiles(prefix_rows(a, g, false)), begin = line.y + in_group * tiles;
  const int first = tiles ? begin / per : 0, subs = a.pair ? 1 : 2;
  const int parts = tiles ? ((begin + tiles - 1) / per - first + 1) * subs : 0;
  const int sub0 = a.pair ? in_block / 128 : 0, in_sub = in_block % 128 + lane, step = a.pair ? 2 : 1;  // places of 128 rows
  const bool there = row < a.rows;
  const int i = (int)a.by_heads((uint32_t)min(row, a.rows - 1)), h = kv * a.heads_each + (min(row, a.rows - 1) - i * a.heads_each);
  const int64_t b = (int64_t)g * a.share + i, own_at = b * j.heads + h;
  const float own = __ldcg(j.parts[0].lse + own_at) * 1.44269504088896341f;
  const float2 *const ml = a.ml + (((int64_t)first + item) * 2 + sub0) * 128 + in_sub;
  float top = own;
#pragma unroll 4
  for (int p = warp; p < parts; p += kJoinThreads / 32) top = fmaxf(top, __ldcg(ml + p * step * 128).x);
  tops[warp][lane] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kJoinThreads / 32; ++w) top = fmaxf(top, tops[w][lane]);
  const float off = offset_of(top), own_weight = exp2_fast(own - off);
  float l = 0.f;
#pragma unroll 4
  for (int p = warp; p < parts; p += kJoinThreads / 32) {
    const float2 x = __ldcg(ml + p * step * 128);
    const float f = exp2_fast(x.x - off);
    factors[p * 32 + lane] = f;
    l += f * x.y;
  }
  sums[warp][lane] = l;
  __syncthreads();
  l = own_weight;
#pragma unroll
  for (int w = 0; w < kJoinThreads / 32; ++w) l += sums[w][lane];
  const float inverse = l == 0.f ? 0.f : 1.f / l;
  if (warp == 0 && blockIdx.y == 0 && there && j.lse) j.lse[own_at] = l == 0.f ? -INFINITY : (off + log2f(l)) * 0.693147180559945f;
  const int quad = warp & 3, upper = warp / 4, d = blockIdx.y * kJoinChannels + quad * 4, half = (parts + 1) / 2;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  if (d < j.dim) {
    if (!upper && !(own_weight == 0.f)) {
      const float4 y = __ldcg(reinterpret_cast<const float4 *>(j.parts[0].out + own_at * j.parts[0].row + d));
      x.x = own_weight * y.x, x.y = own_weight * y.y, x.z = own_weight * y.z, x.w = own_weight * y.w;
    }
    const float4 *const o = reinterpret_cast<const float4 *>(a.o) + ((((int64_t)first + item) * 2 + sub0) * (DP / 4) + d / 4) * 128 + in_sub;
    const int end = upper ? parts : half;
#pragma unroll 8
    for (int p = upper ? half : 0; p < end; ++p) {
      const float f = factors[p * 32 + lane];
      const float4 y = __ldcg(o + (int64_t)p * step * (DP / 4 * 128));
      // (a part without rows has left no o)
      if (!(f == 0.f)) x.x += f * y.x, x.y += f * y.y, x.z += f * y.z, x.w += f * y.w;
    }
  }
  if (upper) others[quad][lane] = x;
  __syncthreads();
  if (upper || d >= j.dim || !there) return;
  const float4 y = others[quad][lane];
  x.x += y.x, x.y += y.y, x.z += y.z, x.w += y.w;
  const float z[4] = {x.x * inverse, x.y * inverse, x.z * inverse, x.w * inverse};
  const int64_t at = b * j.ob + h * j.oh + d;
  if (j.out_dtype == GAR_F32) {
    float *const out = static_cast<float *>(j.out) + at;
    if (j.wide)
      *reinterpret_cast<float4 *>(out) = make_float4(z[0], z[1], z[2], z[3]);
    else
      for (int k = 0; k < 4 && d + k < j.dim; ++k) out[k] = z[k];
  } else if (j.wide) {
    const float2 u = make_float2(z[0], z[1]), v = make_float2(z[2], z[3]);
    *reinterpret_cast<uint2 *>(static_cast<char *>(j.out) + 2 * at) =
        j.out_dtype == GAR_BF16 ? make_uint2(pack2(u, __nv_bfloat16()), pack2(v, __nv_bfloat16())) : make_uint2(pack2(u, __half()), pack2(v, __half()));
  } else {
    for (int k = 0; k < 4 && d + k < j.dim; ++k) {
      if (j.out_dtype == GAR_BF16)
        static_cast<__nv_bfloat16 *>(j.out)[at + k] = from_f32<__nv_bfloat16>(z[k]);
      else
        static_cast<__half *>(j.out)[at + k] = from_f32<__half>(z[k]);
    }
  }
}

template <typename T, int DP, bool PAIR> int launch_prefix(const PrefixArgs &a, const CUtensorMap (&maps)[2], gar_stream_t stream) {
  constexpr auto kernel = prefix_kernel<T, DP, PAIR>;
  static DeviceSet allowed;
  const int e = once_for_device(allowed, a.device, [&] {
    return (int)cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, PrefixShape<DP, PAIR>::kShared);
  });
  if (e != 0) return cuda_fail((cudaError_t)e, "cudaFuncSetAttribute");
  return launch("gar_prefix_attention", kernel, a.ctas, kThreads, PrefixShape<DP, PAIR>::kShared, stream, a, maps[0], maps[1]);
}

}  // namespace

size_t prefix_partials(int items, int dim, char *base, PrefixArgs *a) {
  const int dp = dim <= 64 ? 64 : 128;
  const size_t places = (size_t)items + 152, sums = places * 256 * sizeof(float2);
  if (a) a->ml = reinterpret_cast<float2 *>(base), a->o = reinterpret_cast<float *>(base + sums);
  return sums + places * 256 * dp * sizeof(float);
}

int prefix_mma(const PrefixArgs &a, const CUtensorMap (&maps)[2], gar_stream_t stream) {
  const auto run = [&](auto t) {
    using T = typename decltype(t)::type;
    if (a.c.dim <= 64) return a.pair ? launch_prefix<T, 64, true>(a, maps, stream) : launch_prefix<T, 64, false>(a, maps, stream);
    return a.pair ? launch_prefix<T, 128, true>(a, maps, stream) : launch_prefix<T, 128, false>(a, maps, stream);
  };
  return a.c.dtype == GAR_BF16 ? run(type_tag<__nv_bfloat16>{}) : run(type_tag<__half>{});
}

int join_partials(const PrefixArgs &a, const JoinArgs &j, gar_stream_t stream) {
  const int64_t blocks = (int64_t)a.groups * a.c.heads * a.blocks * ((a.pair ? 256 : 128) / kJoinRows);
  return launch("gar_prefix_attention", a.c.dim <= 64 ? join_kernel<64> : join_kernel<128>,
                dim3((unsigned)blocks, (unsigned)((a.c.dim + kJoinChannels - 1) / kJoinChannels)), kJoinThreads,
                (size_t)(a.pair ? 1 : 2) * a.ctas * 32 * sizeof(float), stream, a, j);
}

}  // namespace gar
