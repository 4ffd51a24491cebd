// Decode attention on tensor cores, over a cache whose rows are 16-byte aligned.
//
// Bound by memory: each cached row is read once for up to 8 NG query heads.  Per 16 rows of 128
// channels the products take 40 (NG = 1) warp-wide m16n8k16 instructions, a small part of
// the time those rows' 8 KB need from memory, so the plain warp-level instruction does and the
// layouts are chosen to keep the rows out of everything but registers:
//
//  * Scores are computed transposed, S^T = K Q^T, rows of the cache as the 16-row operand and
//    the (at most 8, else zero) query heads as the 8 columns.  Which channel sits at which place of the
//    summed dimension is free as long as K and Q agree, so a lane's part of a K row is whole 16-byte chunks.
//  * O^T = V^T P^T, channels as the 16 rows.  Which channel is which row is free too, so a lane's part of a
//    V row is whole chunks as well; the pairs of neighbouring rows that the instruction wants are
//    made with byte permutes.  P^T comes out of the scores' layout by one 8x8 transpose.
//  * Which row of the cache is which row of S^T is free as well, within 8 rows.  Tiles lie in shared
//    memory as the bulk copies' swizzle leaves them (16-byte chunk c of row r at c ^ (r % 8), for 64-byte
//    rows at c ^ (r / 2 % 4)), and the order of the rows (key_row) is one for which
//    both the keys' and the values' reads meet every bank once.
//  * A warp copies its tiles to its own part of shared memory and is the only one to read them:
//    it waits for its own copies, never for another warp.  It keeps kStages - 1 tiles in flight, and
//    goes on to the next segment's while the CTA still joins the last one's results.
//  * Rows are copied by cp.async, a line (at most 128 bytes) at a time.  Rows of 256 channels of 2 or 4 bytes go
//    in tensor copies, a tile's keys or values by one lane in one copy, where pages are whole tiles.  The times of
//    tensor copies and of cp.async (sequences x most rows, query/cached heads x channels): 4 x 20000, 32/2 x 256 bf16
//    35.7 and 38.3 us; 8 x 8192, 16/4 x 256 f32 87 and 97.  Shorter rows came no faster in tensor copies, or slower:
//    64 x 16384, 64/4 x 128 f32 685 and 567; 127 x 8192, 32/8 x 128 e4m3 203 and 204; 24 x 1000 rows, 20/4 x 64 i8
//    15.2 and 13.5; 1 x 262143, 64/8 x 128 bf16 156 both.
//  * The warps of a CTA take a segment's tiles in turn and join at its end; an item of few
//    tiles (DecodeArgs::solo) goes to one warp whole, so that short sequences need no barrier.
//
// Measured: 1 x 262143 rows, 64/8 x 128 bf16 156 us (6.9 TB/s, what a copy reaches); 64 x 8192, 32/8 x 128 bf16 165 us
// (6.5 TB/s); 127 x 8192, 32/8 x 128 e4m3 206 us (5.3 TB/s: its
// warps wait for their own instructions, the expansion of the codes among them, as long as for copies), i8 229, with 32-bit queries
// 233 and 250; 16 x 8192, 8/8 x 128 f32 99 us (5.0 TB/s).  1 x 425, 32/8 x 128 bf16 9 us, which is the launch, the lengths, the
// pages, the rows, the join of a CTA and that of the item one after the other, each a round trip to memory or more.
//
// 8-bit codes become f16, exactly; a row's key scale multiplies its scores, its value scale
// its weight.  That product has to stay in f16's range, so a head's running maximum m is that of score + log2 of the value
// scale, and o and l are relative to it: the products are at most 1, and 2^14 once split.  A row of little
// weight takes no bits from the others, however large its scale.  Weights are split into a high and a low 16-bit part, one product each; so are 32-bit queries of
// an 8-bit cache.  Weights over an f16 cache are multiplied by 2^14 too.
//
// The tensor cores cut their sums off rather than round them: in long sums that is a bias (4e-5 relative after
// 100000 rows).  So they sum no more than the products of one tile; those sums are added up, and rescaled
// where the maximum has grown, by fused multiply-adds in 32 bits.
//
// In a 32-bit cache everything is split in two, x = high + low with 11 significant bits each (TF32), and a
// product is high high + high low + low high: off by 2^-21 relative at most.  Where that gives a score
// that is no number (an infinite key: infinity times a low part of zero), the score is summed again without.
#pragma once

#include <cuda.h>

#include "decode.cuh"
#include "device_once.hpp"

namespace gar {

template <typename C> struct operand {  // the tensor cores' type
  using type = __half;
};
template <> struct operand<__nv_bfloat16> {
  using type = __nv_bfloat16;
};

template <typename T>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1);
template <>
__device__ __forceinline__ void mma<__half>(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                            uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma<__nv_bfloat16>(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                                   uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Channels by 8 rows of the cache, in TF32.
__device__ __forceinline__ void mma_tf32(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
struct Split {
  uint32_t high, low;
};
__device__ __forceinline__ Split split32(uint32_t x) {
  Split s;
  asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(s.high) : "f"(__uint_as_float(x)));
  s.low = __float_as_uint(__uint_as_float(x) - __uint_as_float(s.high));
  return s;
}
// d += the high parts' product, e += the others'.
__device__ __forceinline__ void mma_split(float (&d)[4], float (&e)[4], const Split (&a)[4], Split b0, Split b1) {
  mma_tf32(e, a[0].low, a[1].low, a[2].low, a[3].low, b0.high, b1.high);
  mma_tf32(e, a[0].high, a[1].high, a[2].high, a[3].high, b0.low, b1.low);
  mma_tf32(d, a[0].high, a[1].high, a[2].high, a[3].high, b0.high, b1.high);
}

__device__ __forceinline__ uint32_t bits(__half2 x) { return *reinterpret_cast<uint32_t *>(&x); }
__device__ __forceinline__ uint32_t bits(__nv_bfloat162 x) { return *reinterpret_cast<uint32_t *>(&x); }

// Two weights as a high and a low part.
template <typename T> __device__ __forceinline__ void split(float x, float y, uint32_t *hi, uint32_t *lo);
template <> __device__ __forceinline__ void split<__half>(float x, float y, uint32_t *hi, uint32_t *lo) {
  const __half2 h = __floats2half2_rn(x, y);
  const float2 b = __half22float2(h);
  *hi = bits(h), *lo = bits(__floats2half2_rn(x - b.x, y - b.y));
}
template <> __device__ __forceinline__ void split<__nv_bfloat16>(float x, float y, uint32_t *hi, uint32_t *lo) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
  const float2 b = __bfloat1622float2(h);
  *hi = bits(h), *lo = bits(__floats2bfloat162_rn(x - b.x, y - b.y));
}

// Four 8-bit codes to two pairs of f16.
template <typename C> __device__ __forceinline__ void expand(uint32_t x, uint32_t *a, uint32_t *b);
template <> __device__ __forceinline__ void expand<e4m3>(uint32_t x, uint32_t *a, uint32_t *b) {
  asm("{.reg .b16 l, h; mov.b32 {l, h}, %2; cvt.rn.f16x2.e4m3x2 %0, l; cvt.rn.f16x2.e4m3x2 %1, h;}"
      : "=r"(*a), "=r"(*b)
      : "r"(x));
}
template <> __device__ __forceinline__ void expand<i8>(uint32_t x, uint32_t *a, uint32_t *b) {
  // 0x6400 + u is 1024 + u in f16: with u = x + 128, taking away 1152 leaves x exactly.
  const uint32_t u = x ^ 0x80808080u;
  const __half2 off = __floats2half2_rn(1152.f, 1152.f);
  uint32_t p = __byte_perm(u, 0x64646464u, 0x4140), q = __byte_perm(u, 0x64646464u, 0x4342);
  *a = bits(__hsub2(*reinterpret_cast<__half2 *>(&p), off));
  *b = bits(__hsub2(*reinterpret_cast<__half2 *>(&q), off));
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

template <int BYTES> __device__ __forceinline__ void copy_async(uint32_t to, const void *from, bool there) {
  if (BYTES == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(from), "r"(there ? 4 : 0) : "memory");
}

// The rows of the cache from (row, head, page) on that a tile holds, zeros outside.
__device__ __forceinline__ void copy_box(uint32_t to, const CUtensorMap *map, int row, int head, int page,
                                         uint32_t barrier) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], "
      "[%7];" ::"r"(to), "l"(map), "r"(0), "r"(row), "r"(0), "r"(head), "r"(page), "r"(barrier)
      : "memory");
}

// Waits for the barrier's phase; false when that takes longer than anything could (some 0.1 s or more).
__device__ __forceinline__ bool wait_barrier(uint32_t barrier, uint32_t parity) {
  for (int i = 0; i < 1 << 18; ++i) {
    uint32_t done;
    asm volatile(
        "{.reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p;}"
        : "=r"(done)
        : "r"(barrier), "r"(parity)
        : "memory");
    if (done) return true;
  }
  return false;
}

template <int N> struct words;
template <> struct words<16> {
  using type = uint4;
};
template <> struct words<8> {
  using type = uint2;
};

// What the largest weight is in f16 parts: their smallest step, 2^-24, is 2^-38 of it.  (With 1 the weights under 2^-25 of the
// largest vanish: 16384 rows of 2^-22 beside one whose value is zero came out 8 % short.)
constexpr float kWeightUnit = 16384.f;

// DP: the head's channels rounded up to 64, 96 (no 8-bit), 128, 192 or 256; NG: groups of 8 query heads.  (The queries' type has no part
// in it.)
template <typename C, int DP, int NG> struct MmaShape {
  static constexpr int EL = sizeof(C);
  static constexpr bool Q8 = quantised<C>::value;
  static constexpr int KC = DP * EL / 64;                          // 16-byte chunks of a key row in a lane
  static constexpr int LINE = DP * EL % 128 ? 64 : 128;            // bytes of a row that lie together
  static constexpr int VB = LINE / 8;                              // bytes of a value chunk
  static constexpr int PARTS = DP * EL / LINE;
  static_assert(PARTS * LINE == DP * EL, "whole lines");
  static constexpr int kLogTile = DP * EL <= 128 ? 5 : 4, KT = 1 << kLogTile;  // rows of a tile
  static constexpr int kTile = 2 * KT * DP * EL;                   // bytes, keys and values
  // One CTA per SM; its 192 KB of tiles are divided among as many warps as the registers allow, two tiles each at least.
  // (12 warps and 8: 1 x 262143, 64/8 x 128 bf16 156 and 162 us; 127 x 8192, 32/8 x 128 e4m3 203 and 218.)
  static constexpr int kMost = 196608 / kTile / 2, kLike = NG == 1 && DP <= 128 ? 12 : 8;
  static constexpr int kWarps = kMost < kLike ? kMost : kLike;
  static constexpr int kStages = 196608 / kWarps / kTile;
  // Rows that can be copied as boxes.
  static constexpr bool kBoxes = DP == 256 && !Q8;
  static constexpr int kScales = Q8 ? 2 * KT * 4 : 0;
  // Floats of an o row; a row of o for each head fits a stage.  A few floats more than DP spread
  // the rows over the banks.
  static constexpr int kRow = 8 * NG * (DP + 4) * 4 <= kTile ? DP + 4 : DP;
  static_assert(8 * NG * kRow * 4 <= kTile, "o must fit a stage");
  static constexpr int kShared = kWarps * kStages * (kTile + kScales) + 1024;  // from a multiple of 1024 on
};

// log2 of a value scale, near enough for a reference.  Within [-96, 120], whatever the scale (zero, an infinity, NaN), so that the
// sum l of 2^(score - m) stays finite and does not vanish.  (Next to a scale of 2^s weights under 2^(s - 126) of the largest count
// nothing.)
__device__ __forceinline__ float scale_log2(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(fabsf(x)));
  return fminf(fmaxf(y, -96.f), 120.f);
}

// The row of the cache, of 8, that is row i of the scores.
template <int LINE> __device__ __forceinline__ int key_row(int i) {
  if (LINE == 128) return i & 1 ? (i + 4) & 7 : i;      // 0 5 2 7 4 1 6 3
  const int e = i / 2 + (i / 2 & 2);
  return i & 1 ? e ^ 3 : e;                             // 0 3 1 2 4 7 5 6
}

// Where 16-byte chunk c of row r of a tile lies.
template <int LINE> __device__ __forceinline__ int place(int r, int c) {
  return r * LINE + (LINE == 128 ? c ^ (r & 7) : c ^ (r / 2 & 3)) * 16;
}

template <typename C, int DP, int NG, bool BOXES, bool Q32, typename A>
__global__ void __launch_bounds__(32 * MmaShape<C, DP, NG>::kWarps, 1)
    mma_kernel(const A a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
  using S = MmaShape<C, DP, NG>;
  using T = typename operand<C>::type;
  constexpr int EL = S::EL, KC = S::KC, VB = S::VB, LINE = S::LINE, PARTS = S::PARTS, KT = S::KT, SUBS = KT / 16;
  constexpr int W = S::kWarps;
  constexpr bool Q8 = S::Q8, F32 = std::is_same<C, float>::value, F16 = std::is_same<C, __half>::value;
  constexpr int MT = DP / 16;          // tiles of 16 channels of the output
  constexpr int QW = Q32 ? DP / 4 : DP / 8;  // words of a head's queries in a lane
  extern __shared__ char shared_from[];
  __shared__ JoinShared<W> join;
  __shared__ __align__(8) uint64_t barriers[W][S::kStages];
  const gar_kv_cache &c = a.c;
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31, g = lane / 4, t = lane & 3;
  char *const shared = shared_from + (-(uint32_t)__cvta_generic_to_shared(shared_from) & 1023);
  char *const mine = shared + warp * (S::kStages * S::kTile);
  float *const scales = reinterpret_cast<float *>(shared + W * S::kStages * S::kTile + warp * (S::kStages * S::kScales));
  const uint32_t mine_at = (uint32_t)__cvta_generic_to_shared(mine);
  const uint32_t scales_at = (uint32_t)__cvta_generic_to_shared(scales);
  const uint32_t barrier = (uint32_t)__cvta_generic_to_shared(barriers[warp]);
  if (BOXES && lane < S::kStages)
    asm volatile("mbarrier.init.shared::cta.b64 [%0], 1; fence.mbarrier_init.release.cluster;" ::"r"(barrier + 8 * lane) : "memory");
  if (BOXES && threadIdx.x == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&v_map) : "memory");
  }
  __syncwarp();
  after_earlier_kernels();

  // The warp's notes of the CTA's segments, two halves of kNotes that are filled in turn; a bit for each
  // that the warp has to do with.  The copies are ahead of the products by a half at most.
  __shared__ Notes course[W];
  __shared__ Note notes[W][2 * kNotes];
  Note *const note = notes[warp];
  {
    Notes n;
    n.start(a);
    if (lane == 0) course[warp] = n;
    __syncwarp();
  }
  uint32_t mine_mask = 0;                // of the notes that are not done
  uint32_t copied_mask = 0;              // of those, the ones whose copies have been started
  int filled = 0;                        // halves
  bool more = course[warp].more();
  const auto tiles_of = [&](const Note &n) { return (max(0, n.to - n.from) + KT - 1) / KT; };
  // Few tiles of a whole item, or hardly any: one warp's, in turn.  Else tile by tile the warps'.
  const auto group_of = [&](int i, const Note &n) {
    const int tiles = tiles_of(n);
    return tiles <= (n.whole ? a.solo : 1) ? Group{i % W, 1} : Group{0, min(W, tiles)};
  };
  const auto fill = [&] {
    Notes c = course[warp];
    __syncwarp();
    Note n;
    const bool there = c.next(a, &n);
    const Group group = group_of(filled * kNotes + lane, n);
    if (there) note[(filled & 1) * kNotes + lane] = n;
    if (lane == 0) course[warp] = c;
    const uint32_t mine = __ballot_sync(~0u, there && warp >= group.first && warp < group.first + group.count);
    mine_mask |= mine << (filled & 1) * kNotes;
    ++filled;
    more = c.more();
    __syncwarp();
  };
  // The notes in order: the older half's bits first.  (With an odd number of halves filled the first is the newer.)
  const auto first_of = [&](uint32_t mask) {
    const uint32_t older = filled & 1 ? mask & 0xffff0000u : mask & 0xffffu;
    return __ffs(older ? older : mask) - 1;
  };
  struct {
    int from, lo, to, b, kv_head, tile, step, tiles;
  } get{};                               // what is being copied
  bool ready = false;                    // get's tile exists and its pages are known
  // The cache rows of get's tile.  Copied row by row: this lane's row of the tile, its page and the row in it.  In
  // boxes: the first row of the lane-th of the warp's next tiles, and of the 32 tiles after those.
  struct Rows {
    int page, row;
  } rows{-1, 0}, later{-1, 0};
  int held = 0;                          // boxes: tiles of `rows` that have been copied
  const auto find_rows = [&](int tile) {
    int n;
    Rows x{-1, 0};
    bool there;
    if (BOXES) {
      tile += lane * get.step;
      n = get.from + tile * KT;
      there = tile < get.tiles && n < get.to && n + KT > get.lo;
    } else {
      n = get.from + tile * KT + (lane & (KT - 1));
      there = n >= get.lo && n < get.to;
    }
    if (there) {
      const int32_t *const table = table_of(a, get.b, n);
      const int p = (int)a.page(n);
      x.page = table[p], x.row = n - p * c.page_size;
      if ((unsigned)x.page >= (uint64_t)c.pages) {
        x.page = -1;
        if (c.status) atomicOr(c.status, GAR_KV_BAD_PAGE);
      }
    }
    return x;
  };
  bool late = false;                     // boxes: a wait ran out; nothing is copied any more, and the rest left out
  const auto advance = [&] {
    while (get.tile >= get.tiles || (BOXES && late)) {
      uint32_t left = mine_mask & ~copied_mask;
      if (left == 0) {
        // The half to be filled next must be done with.
        if (!more || (mine_mask & (filled & 1 ? 0xffff0000u : 0xffffu))) break;
        fill();
        continue;
      }
      const int i = first_of(left);
      copied_mask |= 1u << i;
      const Note n = note[i];
      const int half = i / kNotes, age = (filled & 1) == half ? 2 : 1;  // halves filled since this one began
      const Group group = group_of((filled - age) * kNotes + i % kNotes, n);
      get = {n.from, n.lo, n.to, n.b, a.item_groups == 1 ? n.hh : n.hh / a.item_groups,
             group.count == 1 ? 0 : warp, group.count == 1 ? 1 : W, tiles_of(n)};
    }
    ready = get.tile < get.tiles;
    if (ready) {
      rows = find_rows(get.tile);
      held = 0;
      if (BOXES) later = find_rows(get.tile + 32 * get.step);
    }
  };
  // Starts the copies of get's tile and goes to the next.
  const auto issue = [&](int stage) {
    const uint32_t tile_at = mine_at + stage * S::kTile;
    if constexpr (BOXES) {
      // The lane that holds the tile copies it: rows of one page, those outside the segment too; zeros where there
      // is no page.
      const uint32_t bar = barrier + 8 * stage;
      if (lane == held) {
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(S::kTile) : "memory");
        copy_box(tile_at, &k_map, rows.row, get.kv_head, rows.page, bar);
        copy_box(tile_at + KT * DP * EL, &v_map, rows.row, get.kv_head, rows.page, bar);
      }
    } else {
      const int n = get.from + get.tile * KT + (lane & (KT - 1)), page = rows.page, row = rows.row;
      const bool there = page >= 0 && n >= get.lo && n < get.to;
      if (Q8 && lane < KT) {
        const int64_t scale_at =
            there ? page * c.scale_page_stride + row * c.scale_token_stride + get.kv_head * c.scale_head_stride : 0;
        const uint32_t to = scales_at + stage * S::kScales + lane * 4;
        copy_async<4>(to, c.k_scale + scale_at, there);
        copy_async<4>(to + KT * 4, c.v_scale + scale_at, there);
      }
      const int64_t at = there ? (page * c.page_stride + get.kv_head * c.head_stride + row * c.token_stride) * EL : -1;
      constexpr int LANES = LINE / 16, ROWS = 32 / LANES;
      const char *const kp = static_cast<const char *>(c.k), *const vp = static_cast<const char *>(c.v);
      const int chunk = lane & (LANES - 1);
#pragma unroll
      for (int r = 0; r < KT; r += ROWS) {
        const int to_row = r + lane / LANES;
        const int64_t x = __shfl_sync(~0u, at, to_row);
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
          const int off = p * LINE + chunk * 16;
          const bool in = x >= 0 && off < c.dim * EL;
          const uint32_t to = tile_at + p * KT * LINE + place<LINE>(to_row, chunk);
          copy_async<16>(to, in ? kp + x + off : kp, in);
          copy_async<16>(to + KT * DP * EL, in ? vp + x + off : vp, in);
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
    get.tile += get.step;
    if (get.tile >= get.tiles) {
      advance();
    } else if (!BOXES) {
      rows = find_rows(get.tile);
    } else if (++held == 32) {
      rows = later, held = 0;
      later = find_rows(get.tile + 32 * get.step);
    }
  };
  int in = 0, out = 0, flying = 0;  // stages copied into and used next; tiles on their way or here
  uint32_t parity = 0;
  const auto pump = [&](int most) {
    while (flying < most && !(BOXES && late)) {
      if (!ready) advance();
      if (!ready) break;
      issue(in);
      if (++in == S::kStages) in = 0;
      ++flying;
    }
  };

  // This lane's places in a tile: rows g and g + 8 of the scores, rows 2t and 2t + 1 of the values (32 bits: t, t + 4).
  const int k_at = place<LINE>(key_row<LINE>(g), t);
  int v_at[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    v_at[i] = KT * DP * EL + place<LINE>(key_row<LINE>(F32 ? t + 4 * i : 2 * t + i), VB == 16 ? g : g / 2) +
              (VB == 16 ? 0 : (g & 1) * 8);

  // Queries: head g (+ 8 ng), the channels of this lane's chunks.
  uint32_t qf[NG][QW];
  const auto load_queries = [&](const Segment &seg) {
    constexpr int QB = Q32 ? 4 : 2, V = 16 / QB, PER = 16 / EL / V;  // 16 bytes have V channels, a chunk PER times as many
#pragma unroll
    for (int ng = 0; ng < NG; ++ng) {
      const bool there = g + 8 * ng < seg.heads;
      const uint4 *q = reinterpret_cast<const uint4 *>(static_cast<const char *>(a.q) + QB * query_at(a, seg, g + 8 * ng));
#pragma unroll
      for (int k = 0; k < QW / 4; ++k) {
        const int at = (t + 4 * (k / PER)) * PER + k % PER;
        const uint4 x = there && at * V < c.dim ? q[at] : make_uint4(0, 0, 0, 0);
        qf[ng][4 * k] = x.x, qf[ng][4 * k + 1] = x.y, qf[ng][4 * k + 2] = x.z, qf[ng][4 * k + 3] = x.w;
      }
    }
  };

  // The next segment that the warp has to do with: its rows and which tiles are the warp's.
  int using_note = 0, from = 0, lo = 0, to = 0, tile = 0, step = 1, tiles = 0;
  const auto group_in_use = [&] {
    const int half = using_note / kNotes, age = (filled & 1) == half ? 2 : 1;
    return group_of((filled - age) * kNotes + using_note % kNotes, note[using_note]);
  };
  const auto segment_in_use = [&] {
    Segment seg;
    course[warp].segment(a, note[using_note], &seg);
    return seg;
  };
  const auto take = [&] {
    if (mine_mask == 0) advance();  // (fills)
    if (mine_mask == 0) return false;
    using_note = first_of(mine_mask);
    const Segment seg = segment_in_use();
    load_queries(seg);
    const Group group = group_in_use();
    from = seg.from, lo = seg.lo, to = seg.to;
    tile = group.count == 1 ? 0 : warp, step = group.count == 1 ? 1 : W, tiles = tiles_of(note[using_note]);
    return true;
  };

  advance();
  bool have = take();
  pump(S::kStages - 1);
  while (have) {
    float q_scale[NG][2];
#pragma unroll
    for (int ng = 0; ng < NG; ++ng) {
      // Over an 8-bit cache bf16 and 32-bit queries become f16, the head's largest brought to [2^14, 2^15): the smallest
      // step of f16 is then 2^-38 of it.  (Brought to [1, 2) that was 2^-24: a channel of 2^-20 beside one that the keys have as
      // zero kept 4 bits.)
      float up = 1.f;
      if (Q8 && (Q32 || a.q_dtype == GAR_BF16)) {
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < QW; ++i)
          most = Q32 ? max(most, qf[ng][i] & 0x7fffffffu)
                     : max(most, max((qf[ng][i] & 0x7fffu) << 16, qf[ng][i] & 0x7fff0000u));
        most = max(most, __shfl_xor_sync(~0u, most, 1));
        most = max(most, __shfl_xor_sync(~0u, most, 2));
        const int e = min(max((int)(most >> 23), 15), 254);  // (of an infinity or a NaN as of the largest number)
        up = __int_as_float((e - 14) << 23);
        const float down = __int_as_float((268 - e) << 23);
        if constexpr (Q32) {
          uint32_t hi[QW / 2], low[QW / 2];
#pragma unroll
          for (int i = 0; i < QW / 2; ++i)
            split<__half>(__uint_as_float(qf[ng][2 * i]) * down, __uint_as_float(qf[ng][2 * i + 1]) * down, &hi[i], &low[i]);
#pragma unroll
          for (int i = 0; i < QW / 2; ++i) qf[ng][i] = hi[i], qf[ng][QW / 2 + i] = low[i];
        } else {
#pragma unroll
          for (int i = 0; i < QW; ++i)
            qf[ng][i] = bits(__floats2half2_rn(__uint_as_float(qf[ng][i] << 16) * down,
                                               __uint_as_float(qf[ng][i] & 0xffff0000u) * down));
        }
      }
      up *= a.scale_log2;
      q_scale[ng][0] = __shfl_sync(~0u, up, 8 * t);      // lane 4 (2t) holds head 2t's
      q_scale[ng][1] = __shfl_sync(~0u, up, 8 * t + 4);
    }

    float o[MT][NG][4] = {};
    float m[NG][2], l[NG][2] = {};
#pragma unroll
    for (int ng = 0; ng < NG; ++ng) m[ng][0] = m[ng][1] = -INFINITY;

    for (; tile < tiles; tile += step) {
      if (BOXES) {
        late = __any_sync(~0u, late || tile >= a.give_up || !wait_barrier(barrier + 8 * out, parity));
        if (late) {
          if (c.status) atomicOr(c.status, GAR_KV_TIMEOUT);
          break;
        }
      } else {
        if (flying == S::kStages - 1)
          asm volatile("cp.async.wait_group %0;" ::"n"(S::kStages - 2) : "memory");
        else
          asm volatile("cp.async.wait_group 0;" ::: "memory");
      }
      __syncwarp();
      pump(S::kStages);
      char *const at = mine + out * S::kTile;
      const float *k_scale = scales + out * (S::kScales / 4), *v_scale = k_scale + KT;
      const int n0 = from + tile * KT;
      const bool ragged = n0 < lo || n0 + KT > to;
      if (BOXES && ragged) {
        // What the copies brought of rows outside the segment must not meet the products: 0 * NaN is NaN.
        const int n = n0 + lane;
        if (lane < KT && (n < lo || n >= to))
          for (int i = 0; i < PARTS; ++i)
            for (int x = 0; x < LINE; x += 16)
              *reinterpret_cast<uint4 *>(at + KT * DP * EL + (i * KT + lane) * LINE + x) = make_uint4(0, 0, 0, 0);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
      }

      // Scores.
      constexpr int CHAINS = F32 ? 5 : 2;  // sums that are added up at the end (the last of 5: the low parts')
      float s[SUBS][NG][4];
#pragma unroll
      for (int sub = 0; sub < SUBS; ++sub) {
        float part[CHAINS][NG][4] = {};
#pragma unroll
        for (int k = 0; k < KC; ++k) {
          const char *const x_at = at + (k * 64 / LINE * KT + sub * 16) * LINE + (LINE == 128 && k % 2 ? k_at ^ 64 : k_at);
          const uint4 x = *reinterpret_cast<const uint4 *>(x_at), y = *reinterpret_cast<const uint4 *>(x_at + 8 * LINE);
          const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
          if constexpr (F32) {
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
              const Split x4[4] = {split32(xs[i]), split32(ys[i]), split32(xs[i + 1]), split32(ys[i + 1])};
#pragma unroll
              for (int ng = 0; ng < NG; ++ng)
                mma_split(part[k % 4][ng], part[CHAINS - 1][ng], x4, split32(qf[ng][k * 4 + i]), split32(qf[ng][k * 4 + i + 1]));
            }
          } else if constexpr (!Q8) {
#pragma unroll
            for (int i = 0; i < 4; i += 2)
#pragma unroll
              for (int ng = 0; ng < NG; ++ng)
                mma<T>(part[i / 2][ng], xs[i], ys[i], xs[i + 1], ys[i + 1], qf[ng][k * 4 + i], qf[ng][k * 4 + i + 1]);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t a0, a1, a2, a3;
              expand<C>(xs[i], &a0, &a2);
              expand<C>(ys[i], &a1, &a3);
#pragma unroll
              for (int ng = 0; ng < NG; ++ng) {
                if (Q32)
                  mma<T>(part[i % 2][ng], a0, a1, a2, a3, qf[ng][QW / 2 + k * 8 + 2 * i], qf[ng][QW / 2 + k * 8 + 2 * i + 1]);
                mma<T>(part[i % 2][ng], a0, a1, a2, a3, qf[ng][k * 8 + 2 * i], qf[ng][k * 8 + 2 * i + 1]);
              }
            }
          }
        }
#pragma unroll
        for (int ng = 0; ng < NG; ++ng)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float x = part[0][ng][i] + part[1][ng][i];
            if constexpr (F32) x = (x + (part[2][ng][i] + part[3][ng][i])) + part[4][ng][i];
            s[sub][ng][i] = x;
          }
      }
      if constexpr (F32) {
        bool odd = false;
#pragma unroll
        for (int ng = 0; ng < NG; ++ng)
#pragma unroll
          for (int i = 0; i < 4; ++i) odd |= s[0][ng][i] != s[0][ng][i];
        if (__any_sync(~0u, odd)) {
          const Segment seg = segment_in_use();
#pragma unroll
          for (int ng = 0; ng < NG; ++ng)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int head = 8 * ng + 2 * t + i % 2, row = key_row<LINE>(g) + i / 2 * 8;
              const float *q = static_cast<const float *>(a.q) + query_at(a, seg, head);
              float x = 0.f;
              if (head < seg.heads)
                for (int d = 0; d < c.dim; ++d)
                  x = fmaf(q[d], *reinterpret_cast<const float *>(at + d / 32 * KT * LINE + place<LINE>(row, d / 4 & 7) + d % 4 * 4), x);
              s[0][ng][i] = x;
            }
        }
      }
      float top[NG][2];
#pragma unroll
      for (int ng = 0; ng < NG; ++ng) top[ng][0] = m[ng][0], top[ng][1] = m[ng][1];
#pragma unroll
      for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int row = sub * 16 + key_row<LINE>(g) + 8 * r, n = n0 + row;
          const bool seen = !ragged || (n >= lo && n < to);
          const float f = Q8 ? k_scale[row] : 1.f, f_log2 = Q8 ? scale_log2(v_scale[row]) : 0.f;
#pragma unroll
          for (int ng = 0; ng < NG; ++ng)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float &x = s[sub][ng][2 * r + h];
              x = seen ? x * (Q8 ? f * q_scale[ng][h] : q_scale[ng][h]) : -INFINITY;
              top[ng][h] = fmaxf(top[ng][h], Q8 ? x + f_log2 : x);
            }
        }
      bool grown = false;
#pragma unroll
      for (int ng = 0; ng < NG; ++ng)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int d = 4; d < 32; d *= 2) top[ng][h] = fmaxf(top[ng][h], __shfl_xor_sync(~0u, top[ng][h], d));
          grown |= top[ng][h] > m[ng][h];
        }
      grown = __any_sync(~0u, grown);
      float shrink[NG][2];
#pragma unroll
      for (int ng = 0; ng < NG; ++ng)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          // (rows with values of zero, say, at 2^-96: l may be 2^96 and the next reference larger by 2^96 and more)
          const float d = m[ng][h] - offset_of(top[ng][h]);
          shrink[ng][h] = grown ? exp2_fast(d) : 1.f;
          l[ng][h] = !Q8 ? l[ng][h] * shrink[ng][h] : grown ? scaled<Q8>(l[ng][h], d) : l[ng][h];
          m[ng][h] = top[ng][h];
        }
      // Weights, in the layout of the second product's right operand.
      uint32_t hi[SUBS][NG][F32 ? 4 : 2], low[SUBS][NG][F32 ? 4 : 2];
#pragma unroll
      for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const float f = Q8 ? v_scale[sub * 16 + key_row<LINE>(g) + 8 * r] : 1.f;
#pragma unroll
          for (int ng = 0; ng < NG; ++ng) {
            float p[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              p[h] = exp2_fast(s[sub][ng][2 * r + h] - offset_of(m[ng][h]));
              l[ng][h] += p[h];
              if (Q8) p[h] *= f;
              if (Q8 || F16) p[h] *= kWeightUnit;
            }
            if constexpr (F32) {
              // Row t (i = 0) or t + 4 of these 8 rows and head g, for this lane: the lane that has them is known.
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const int from_lane = (t + 4 * i) * 4 + g / 2;
                const float x = __shfl_sync(~0u, p[0], from_lane), y = __shfl_sync(~0u, p[1], from_lane);
                const Split w = split32(__float_as_uint(g & 1 ? y : x));
                hi[sub][ng][2 * r + i] = w.high, low[sub][ng][2 * r + i] = w.low;
              }
            }
            if constexpr (!F32) {
              split<T>(p[0], p[1], &hi[sub][ng][r], &low[sub][ng][r]);
              hi[sub][ng][r] = transpose8x8(hi[sub][ng][r]);
              low[sub][ng][r] = transpose8x8(low[sub][ng][r]);
            }
          }
        }
      // Values.
      constexpr int TILES = VB / EL / 2;  // tiles of 16 channels that a chunk has part in
#pragma unroll
      for (int k = 0; k < PARTS; ++k)
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub) {
          using V = typename words<VB>::type;
          union {
            V v;
            uint32_t u[VB / 4];
          } y[4];
#pragma unroll
          for (int r = 0; r < 4; ++r)
            y[r].v = *reinterpret_cast<const V *>(at + (k * KT + sub * 16 + r / 2 * 8) * LINE + v_at[r & 1]);
#pragma unroll
          for (int i = 0; i < TILES; ++i) {
            float d[NG][4] = {}, e[NG][4] = {};
            if constexpr (F32) {
              // y[2r], y[2r + 1]: rows t and t + 4 of the r-th 8; words 2i and 2i + 1 are two channels.
#pragma unroll
              for (int r = 0; r < 2; ++r) {
                const Split v4[4] = {split32(y[2 * r].u[2 * i]), split32(y[2 * r].u[2 * i + 1]),
                                     split32(y[2 * r + 1].u[2 * i]), split32(y[2 * r + 1].u[2 * i + 1])};
#pragma unroll
                for (int ng = 0; ng < NG; ++ng)
                  mma_split(d[ng], e[ng], v4, Split{hi[sub][ng][2 * r], low[sub][ng][2 * r]},
                            Split{hi[sub][ng][2 * r + 1], low[sub][ng][2 * r + 1]});
              }
            } else {
              uint32_t a0, a1, a2, a3;
              if constexpr (Q8) {
                expand<C>(__byte_perm(y[0].u[i / 2], y[1].u[i / 2], i % 2 ? 0x7362 : 0x5140), &a0, &a1);
                expand<C>(__byte_perm(y[2].u[i / 2], y[3].u[i / 2], i % 2 ? 0x7362 : 0x5140), &a2, &a3);
              } else {
                a0 = __byte_perm(y[0].u[i], y[1].u[i], 0x5410), a1 = __byte_perm(y[0].u[i], y[1].u[i], 0x7632);
                a2 = __byte_perm(y[2].u[i], y[3].u[i], 0x5410), a3 = __byte_perm(y[2].u[i], y[3].u[i], 0x7632);
              }
#pragma unroll
              for (int ng = 0; ng < NG; ++ng) {
                mma<T>(d[ng], a0, a1, a2, a3, hi[sub][ng][0], hi[sub][ng][1]);
                mma<T>(d[ng], a0, a1, a2, a3, low[sub][ng][0], low[sub][ng][1]);
              }
            }
#pragma unroll
            for (int ng = 0; ng < NG; ++ng)
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                float &z = o[k * TILES + i][ng][j];
                z = fmaf(z, sub == 0 ? shrink[ng][j & 1] : 1.f, F32 ? d[ng][j] + e[ng][j] : d[ng][j]);
              }
          }
        }
      --flying;
      if (++out == S::kStages) out = 0, parity ^= 1;
    }
#pragma unroll
    for (int ng = 0; ng < NG; ++ng)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int d = 4; d < 32; d *= 2) l[ng][h] += __shfl_xor_sync(~0u, l[ng][h], d);
    constexpr int CE = VB / EL;  // channels of a chunk, two of them in a tile of 16
    constexpr float v_unit = Q8 || F16 ? 1.f / kWeightUnit : 1.f;
    const Segment ended = segment_in_use();
    const Group by = group_in_use();
    if (by.count == 1 && ended.whole && a.out_wide) {
      // One warp's alone: straight to the output, whole chunks at a time.
#pragma unroll
      for (int ng = 0; ng < NG; ++ng)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int head = 8 * ng + 2 * t + h;
          if (head >= ended.heads) continue;
          if (g == 0) store_lse(a, ended, head, m[ng][h], l[ng][h]);
          const float f = l[ng][h] == 0.f ? 0.f : v_unit / l[ng][h];
#pragma unroll
          for (int i = 0; i < MT; i += 2) {
            const int k = i / (CE / 2), d = (g + 8 * k) * CE + i % (CE / 2) * 2;
            float4 x = make_float4(o[i][ng][h], o[i][ng][2 + h], o[i + 1][ng][h], o[i + 1][ng][2 + h]);
            if (l[ng][h] == 0.f) x = make_float4(0.f, 0.f, 0.f, 0.f);
            if (d < c.dim) store_wide4(a, ended.b * a.ob + (ended.head + head) * a.oh + d, x.x * f, x.y * f, x.z * f, x.w * f);
          }
        }
      mine_mask &= ~(1u << using_note), copied_mask &= ~(1u << using_note);
      pump(S::kStages - 1);
      have = take();
      continue;
    }
    // The stage read last holds this warp's o until it is joined.
    float *const o_mine = reinterpret_cast<float *>(mine + (out == 0 ? S::kStages - 1 : out - 1) * S::kTile);
    __syncwarp();
#pragma unroll
    for (int ng = 0; ng < NG; ++ng)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int head = 8 * ng + 2 * t + h;
        if (g == 0) join.ml[warp][head] = make_float2(m[ng][h], l[ng][h]);
        float *const row = o_mine + head * S::kRow;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          // Two neighbouring channels, at a place that depends on the head so that the lanes meet all banks.
          const int k = i / (CE / 2), d = ((g + 8 * k) * CE + i % (CE / 2) * 2) ^ (head & 6);
          *reinterpret_cast<float2 *>(row + d) =
              Q8 || F16 ? make_float2(o[i][ng][h] * v_unit, o[i][ng][2 + h] * v_unit) : make_float2(o[i][ng][h], o[i][ng][2 + h]);
        }
      }
    // (copies into this stage come after the join's barrier)
    if (BOXES) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    const float *const o_all = reinterpret_cast<const float *>(shared);
    if (lane == 0) join.at[warp] = (int)(o_mine - o_all);
    // The next segment's first tiles and queries come while this one is joined.
    mine_mask &= ~(1u << using_note), copied_mask &= ~(1u << using_note);
    pump(S::kStages - 1);
    have = take();
    join_warps<W, true, Q8>(a, ended, by, join, o_all, S::kRow);
    if (!ended.whole) join_parts<W, Q8>(a, ended, by, join);
  }
  if (BOXES && late)                     // what is on its way lands before the CTA's memory is another's
    for (int i = out; i < out + flying; ++i)
      wait_barrier(barrier + 8 * (i < S::kStages ? i : i - S::kStages), i < S::kStages ? parity : parity ^ 1);
}

// A map of the cache's bytes as [pages][heads][lines of a row][page_size][128], boxes of the lines (or one line) of `rows`
// rows; false where it has none.
bool box_map(const gar_kv_cache &c, void *base, int rows, bool all_lines, CUtensorMap *map);

template <typename C, int DP, int NG, bool Q32, typename A> int launch_mma(A a, int sms, gar_stream_t stream) {
  using S = MmaShape<C, DP, NG>;
  a.item_heads = std::min(a.group, 8 * NG);
  a.item_groups = (a.group + 8 * NG - 1) / (8 * NG);
  a.items = divide_by((uint32_t)(a.c.heads * a.item_groups));
  // Tiles of an item that a warp takes whole: twice the items of a CTA, as the warps have the more time to even out.
  // (Twice and once as many: 256 sequences of up to 256 rows, 32/8 x 128 bf16 44 and 60 us; of up to 512, i8 65 and 95,
  // bf16 88 and 79.  64 of up to 512, 8/8 x 64 i8, 3 items a CTA: 24 with 6, 22 with 4, 30 with 12.)
  a.solo = std::min(64, std::max(4, (int)(2 * (int64_t)a.batch * a.c.heads * a.item_groups / sms)));
  CUtensorMap maps[2];
  const auto run = [&](auto boxes) {
    constexpr auto kernel = mma_kernel<C, DP, NG, decltype(boxes)::value, Q32, A>;
    static DeviceSet allowed;
    const int e = once_for_device(allowed, a.device, [&] {
      return (int)cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kShared);
    });
    if (e != 0) return cuda_fail((cudaError_t)e, "cudaFuncSetAttribute");
    return launch("gar_decode_attention", kernel, sms, 32 * S::kWarps, S::kShared, stream, a, maps[0], maps[1]);
  };
  if constexpr (S::kBoxes && std::is_same<A, DecodeArgs>::value)
    if (a.c.dim == DP && a.c.page_size % S::KT == 0 && box_map(a.c, a.c.k, S::KT, true, &maps[0]) &&
        box_map(a.c, a.c.v, S::KT, true, &maps[1]))
      return run(std::true_type{});
  return run(std::false_type{});
}

template <typename C, bool Q32, typename A> int decode_mma(const A &a, int sms, gar_stream_t stream) {
  // Sixteen heads at a time where there are more than eight (a row is read once for all; 256 channels' outputs do not fit the
  // registers).  64 x 16384, 64/4 x 128: bf16 202 us and 321 with eight at a time, i8 179 and 217, f32 573 and 761; 64 x 2000 bf16
  // 54 and 57, 8 x 60000, 16/1 x 128 39 and 38.  The slower of the two for one long sequence, 1 x 60000 36 and 22, 1 x 262143 55 and 42:
  // more to join in one CTA.
  const bool two = a.group > 8;
  // The channels that a tile is made for: a size more costs the copies' zeros, the products and the room of the tiles.  96
  // and 192 were worth (16 x 8192, 16/4 heads, in place of 128 and 256): 80 f32 42 us, 57; 96 bf16 25 and 26; 192 f32 92 and
  // 169, bf16 42 and 45, i8 37 and 42.  (96 channels of 8 bits are no whole lines of 64 bytes.)
  if (a.c.dim <= 64) return two ? launch_mma<C, 64, 2, Q32>(a, sms, stream) : launch_mma<C, 64, 1, Q32>(a, sms, stream);
  if constexpr (sizeof(C) > 1)
    if (a.c.dim <= 96)
      return two ? launch_mma<C, 96, 2, Q32>(a, sms, stream) : launch_mma<C, 96, 1, Q32>(a, sms, stream);
  if (a.c.dim <= 128)
    return two ? launch_mma<C, 128, 2, Q32>(a, sms, stream) : launch_mma<C, 128, 1, Q32>(a, sms, stream);
  return a.c.dim <= 192 ? launch_mma<C, 192, 1, Q32>(a, sms, stream) : launch_mma<C, 256, 1, Q32>(a, sms, stream);
}

}  // namespace gar
