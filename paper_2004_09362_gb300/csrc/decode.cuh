// What the decode-attention kernels share: their arguments, the division of the cache's rows
// among CTAs, and the join of partial results.
//
// Work.  An item is one sequence, one cached head and a group of up to kMaxGroup of the query heads
// that read it.  The CTAs share the items' rows in one of two ways.
//  * A segment each: every item is cut into parts of as many rows, the fewest (a multiple of 64) for which
//    there are no more parts than CTAs.  Taken for up to 32 sequences where a part is at most 5/4 of an equal
//    share, or 192 KB more: a second segment to start, and to join, takes a CTA as long as those.  (24 sequences, a
//    window of 1000 rows, 20/4 heads x 64 channels i8: 15 us so, 19.5 in a line.)
//  * A line: the items' rows, in units of 64 (more where the line would pass 2^30 units), stand one
//    behind the other, and CTA i of N takes the i-th of N equal shares.  So every CTA has the same number
//    of rows to read whatever the lengths are, and thousands of short sequences are not split at all.  Each item
//    counts 192 KB of rows more, for what a segment costs beside its rows, or the items' mean where that is
//    less.  (127 sequences of up to 8192 rows, 32/8 x 128 channels e4m3: 203 us; with 96 KB 208, with 64 rows 222.)
// The lengths are read on the device: nothing waits for the host, and a captured launch stays
// right when they change.
//
// Join.  A segment is the part of an item that one CTA takes.  Each keeps the running maximum m
// of the scores (in units of log 2; over 8-bit caches another number that o and l are relative to),
// l = sum 2^(score - m) and o = sum 2^(score - m) v.  Where an
// item has several segments, each CTA stores (m, l, o), and the one that arrives last at the
// item's counter adds them up in the order of the rows (so the bits do not depend on who
// was last):  m = max m_i,  l = sum l_i 2^(m_i - m),  o likewise.
#pragma once

#include "gar_device.cuh"

namespace gar {

constexpr int kMaxGroup = 16;         // query heads of an item
constexpr int kMaxCtas = 152 * 4;

struct DecodeArgs {
  gar_kv_cache c;
  const void *q;
  void *out;
  float *lse;
  int64_t qb, qh, ob, oh, table_stride;
  const int32_t *table, *lengths;
  Divide page;
  int most_rows;           // rows that the table's width can hold
  int unit;                // rows of a unit of the line
  int slack;               // units of 192 KB
  int solo;                // tiles of an item that a warp takes whole
  int batch, q_heads, group, item_groups, item_heads;  // group: q_heads / kv_heads
  Divide items;            // by a sequence's items
  int q_dtype, out_dtype, window;
  bool out_wide;           // four neighbouring outputs can be stored at once
  float scale_log2;        // scale * log2(e)
  // workspace: per CTA two segments' (m, l) and o, and a counter
  float2 *part_ml;
  float *part_o;
  unsigned int *count;
  int dim_pad;             // floats of a stored o row
  int device;              // the launch's
  int give_up;             // a segment's tiles from this one on count as copies that did not end
};

// Rows of a unit of the line: as many as it takes for the whole line, each item counted twice at most, to stay below 2^30
// units, or 0 where 2^15 do not.
inline int unit_of(int64_t items, int most_rows) {
  for (int unit = 64; unit <= 32768; unit *= 2)
    if (items * (most_rows / unit + 3) * 2 < 1 << 30) return unit;
  return 0;
}

// What calls of a batch that shares rows, and others than decode attention, need beside that.  (A type of its own: the same kernels
// with these questions in them took 206 us over the e4m3 batch above, then 220.)
struct ServingArgs : DecodeArgs {
  bool line;               // a line, whatever the batch (where parts need no join)
  // Sequences that share their rows count as one: its query m of a cached head is query m % heads_each, of that head, of
  // its sequence m / heads_each (share: its sequences; 0: there is nothing to share).
  int share, heads_each;
  Divide by_heads;         // by heads_each
  // Rows that come before each sequence's own (or null): before_share sequences have one row of this table.
  const int32_t *before_table, *before_lengths;
  int64_t before_stride;
  int before_share, before_most, own_most;
};

// x / d; a division in 32-bit floats, put right, where they hold x (the compiler's takes three times as long).
__device__ __forceinline__ int quotient(int x, int d) {
  if (x >= 1 << 23) return x / d;
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"((float)d));
  int q = (int)((float)x * r);
  const int rest = x - q * d;
  return rest >= d ? q + 1 : rest < 0 ? q - 1 : q;
}

// A length within what a table can hold.
__device__ __forceinline__ int held(const DecodeArgs &a, int n, int most) {
  if (n >= 0 && n <= most) return n;
  if (a.c.status) atomicOr(a.c.status, GAR_KV_BAD_LENGTH);
  return n < 0 ? 0 : most;
}
// The rows before a sequence's own, and all of its rows.
__device__ __forceinline__ int before_of(const ServingArgs &a, int b) { return held(a, a.before_lengths[b / a.before_share], a.before_most); }
__device__ __forceinline__ int length_of(const DecodeArgs &a, int b) { return a.lengths[b]; }
__device__ __forceinline__ int length_of(const ServingArgs &a, int b) {
  const int n = a.lengths[b];
  return a.before_lengths == nullptr ? n : held(a, n, a.own_most) + before_of(a, b);
}
// The pages that have row n of a sequence, which becomes the row of those pages.
__device__ __forceinline__ const int32_t *table_of(const DecodeArgs &a, int b, int &) { return a.table + b * a.table_stride; }
__device__ __forceinline__ const int32_t *table_of(const ServingArgs &a, int b, int &n) {
  if (a.before_lengths != nullptr) {
    const int before = before_of(a, b);
    if (n < before) return a.before_table + b / a.before_share * a.before_stride;
    n -= before;
  }
  return a.table + b * a.table_stride;
}
__device__ __forceinline__ bool in_a_line(const DecodeArgs &) { return false; }
__device__ __forceinline__ bool in_a_line(const ServingArgs &a) { return a.line; }

struct Span {
  int units;
  int lo, hi, base;        // rows [lo, hi); base: lo rounded down to a multiple of 32
};

// The span of a length, in units of `unit` rows.
__device__ __forceinline__ Span span_of(const DecodeArgs &a, int n, int unit) {
  Span s;
  if (n < 0 || n > a.most_rows) {
    if (a.c.status) atomicOr(a.c.status, GAR_KV_BAD_LENGTH);
    n = n < 0 ? 0 : a.most_rows;
  }
  s.hi = n;
  s.lo = a.window > 0 && n > a.window ? n - a.window : 0;
  s.base = s.lo & ~31;
  // (no more than 2^31: the sum of two ints)
  const unsigned up = (unsigned)(s.hi - s.base) + unit - 1;
  s.units = max(1, unit == 64 ? (int)(up >> 6) : up < 1u << 23 ? quotient((int)up, unit) : (int)(up / (unsigned)unit));
  return s;
}

// Rows [lo, to) of one item.
struct Segment {
  int b, kv_head, head, heads;  // head: the first of the item's query heads
  int lo, from, to;             // from: lo rounded down to a multiple of 32
  bool whole;
  int slot;                     // where the partial result goes
  int first, parts;             // the item's CTAs
  bool first_late;              // the first of them begins before the item does
};

// Walks one CTA's share.
struct Walk {
  int pos, end, per;
  int item;                     // where in the line the item at pos begins
  int b, hh, lead, unit;        // unit: rows
  bool first_segment;
  Span s;

  // By each warp on its own: a lane adds up a run of sequences, a scan over the lanes follows, and
  // the lane whose run holds the share's start looks it up.
  template <typename A> __device__ __forceinline__ void start(const A &a) {
    const int lane = threadIdx.x & 31, run = (a.batch + 31) / 32;
    const int b0 = min(a.batch, lane * run), b1 = min(a.batch, b0 + run);
    const int items = a.c.heads * a.item_groups, ctas = gridDim.x;
    unit = a.unit;
    int mine = 0, n = 0;
    for (int i = b0; i < b1; ++i) mine += span_of(a, n = length_of(a, i), unit).units;
    int total = __reduce_add_sync(~0u, mine);
    lead = min(a.slack, quotient(total, a.batch));
    if (!in_a_line(a) && run <= 1 && a.batch * items <= ctas) {
      // The smallest parts that are no more than the CTAs, from an equal share on.  Units that are no more than the
      // CTAs are such parts already.
      const int share = total * items <= ctas ? 1 : quotient(total * items + ctas - 1, ctas);
      if (share == 1) lead = 0;
      const auto parts_of = [&](int u, int *parts) {
        *parts = b0 < b1 ? span_of(a, n, u * a.unit).units : 0;
        return __reduce_add_sync(~0u, *parts);
      };
      int over = share + max(share / 4, a.slack), parts, all;
      if (share > 1 && over <= (1 << 30) / a.unit && (all = parts_of(over, &parts)) * items <= ctas) {
        int under = share - 1;  // does not fit, or is too small
        while (over - under > max(1, share / 16)) {
          const int u = under == share - 1 ? share : (over + under) / 2;
          int its_parts;
          const int its_all = parts_of(u, &its_parts);
          if (its_all * items <= ctas)
            over = u, parts = its_parts, all = its_all;
          else
            under = u;
        }
        unit = over * a.unit, lead = 0, mine = parts, total = all;
      }
    }
    total = (total + lead * a.batch) * items, mine = (mine + lead * (b1 - b0)) * items;
    int before = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int up = __shfl_up_sync(~0u, before, d);
      if (lane >= d) before += up;
    }
    before -= mine;
    per = total <= ctas ? 1 : quotient(total + ctas - 1, ctas);
    pos = min(total, (int)blockIdx.x * per);
    end = min(total, pos + per);
    if (pos >= end) return;
    int i = b0;
    const bool here = pos >= before && pos < before + mine;
    if (here && run > 1)
      for (; i < b1; ++i) {
        n = length_of(a, i);
        const int units = (span_of(a, n, unit).units + lead) * items;
        if (pos < before + units) break;
        before += units;
      }
    const int from = __ffs(__ballot_sync(~0u, here)) - 1;
    before = __shfl_sync(~0u, before, from);
    enter(a, __shfl_sync(~0u, i, from), __shfl_sync(~0u, n, from));
    hh = quotient(pos - before, s.units);
    item = before + hh * s.units;
    first_segment = true;
  }

  template <typename A> __device__ __forceinline__ void enter(const A &a, int sequence, int n) {
    b = sequence;
    s = span_of(a, n, unit);
    s.units += lead;
  }

  template <typename A> __device__ __forceinline__ bool next(const A &a, Segment *g) {
    if (pos >= end) return false;
    if (!first_segment) {
      if (++hh == a.c.heads * a.item_groups) hh = 0, enter(a, b + 1, length_of(a, b + 1));
      item = pos;
    }
    const int u = pos - item, n = min(s.units - u, end - pos);
    g->b = b;
    g->kv_head = a.item_groups == 1 ? hh : hh / a.item_groups;
    const int sub = (hh - g->kv_head * a.item_groups) * a.item_heads;
    g->head = g->kv_head * a.group + sub;
    g->heads = min(a.item_heads, a.group - sub);
    g->from = s.base + max(0, u - lead) * unit;
    g->to = (int)min((unsigned)s.hi, (unsigned)s.base + (unsigned)max(0, u + n - lead) * unit);
    g->lo = max(s.lo, g->from);
    g->whole = n == s.units;
    g->first = blockIdx.x, g->parts = 1, g->slot = 0, g->first_late = false;
    if (!g->whole) {
      g->slot = 2 * blockIdx.x + (first_segment ? 0 : 1);
      g->first = quotient(item, per);
      g->parts = quotient(item + s.units - 1, per) - g->first + 1;
      g->first_late = g->first * per < item;
    }
    pos += n;
    first_segment = false;
    return true;
  }
};

// A segment as it is noted for later: 32 bytes.
struct alignas(16) Note {
  int from, to, lo, b;
  int hh, item, units;  // the sequence's item; where it begins in the line, and its units
  short whole, first;   // all of the item; the first segment of its CTA
};
static_assert(sizeof(Note) == 32, "two 16-byte accesses");

// Notes a CTA's segments, kNotes at a time, a lane for each.
constexpr int kNotes = 16;
struct Notes {
  int begin, end, per, lead, unit;  // of the walk
  int next_item, at;                // the first item that is not noted yet, and where in the line it begins

  template <typename A> __device__ __forceinline__ void start(const A &a) {
    Walk w;
    w.start(a);
    begin = w.pos, end = w.end, per = w.per, lead = w.lead, unit = w.unit;
    next_item = at = 0;
    if (begin < end) next_item = w.b * (a.c.heads * a.item_groups) + w.hh, at = w.item;
  }
  __device__ __forceinline__ bool more() const { return at < end && begin < end; }

  // Lane i < kNotes: the i-th of the next segments, or none (from > to).
  template <typename A> __device__ __forceinline__ bool next(const A &a, Note *n) {
    const int lane = threadIdx.x & 31, items = a.c.heads * a.item_groups;
    const int item = next_item + min(lane, kNotes - 1);
    n->b = (int)a.items((uint32_t)item);
    n->hh = item - n->b * items;
    Span s{};
    if (n->b < a.batch) {
      s = span_of(a, length_of(a, n->b), unit);
      s.units += lead;
    }
    int upto = s.units;
#pragma unroll
    for (int d = 1; d < kNotes; d *= 2) {
      const int up = __shfl_up_sync(~0u, upto, d);
      if (lane >= d) upto += up;
    }
    n->item = at + upto - s.units, n->units = s.units;
    const int u0 = max(begin, n->item) - n->item, u1 = min(end, n->item + s.units) - n->item;
    n->from = s.base + max(0, u0 - lead) * unit;
    n->to = (int)min((unsigned)s.hi, (unsigned)s.base + (unsigned)max(0, u1 - lead) * unit);
    n->lo = max(s.lo, n->from);
    n->whole = u0 == 0 && u1 == s.units, n->first = n->item + u0 == begin;
    next_item += kNotes;
    at += __shfl_sync(~0u, upto, kNotes - 1);
    return lane < kNotes && n->b < a.batch && u0 < u1;
  }

  __device__ __forceinline__ void segment(const DecodeArgs &a, const Note &n, Segment *g) const {
    g->b = n.b;
    g->kv_head = a.item_groups == 1 ? n.hh : n.hh / a.item_groups;
    const int sub = (n.hh - g->kv_head * a.item_groups) * a.item_heads;
    g->head = g->kv_head * a.group + sub;
    g->heads = min(a.item_heads, a.group - sub);
    g->from = n.from, g->to = n.to, g->lo = n.lo;
    g->whole = n.whole;
    g->first = blockIdx.x, g->parts = 1, g->slot = 0, g->first_late = false;
    if (!n.whole) {
      g->slot = 2 * blockIdx.x + (n.first ? 0 : 1);
      g->first = quotient(n.item, per);
      g->parts = quotient(n.item + n.units - 1, per) - g->first + 1;
      g->first_late = g->first * per < n.item;
    }
  }
};

// The place of part i of an item: its CTA's second segment when that CTA's share begins before the item.
__device__ __forceinline__ int slot_of(const Segment &g, int i) {
  return 2 * (g.first + i) + (i == 0 && g.first_late ? 1 : 0);
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// x 2^d.  FAR: also where 2^d alone vanishes (d under -126) and x is as much larger than 1.
template <bool FAR> __device__ __forceinline__ float scaled(float x, float d) {
  if (!FAR) return x * exp2_fast(d);
  const float near = fmaxf(d, -100.f);
  return x * exp2_fast(near) * exp2_fast(d - near);
}

// m as an exponent's offset: nothing seen yet (-infinity) leaves 2^-infinity = 0 rather than NaN.
__device__ __forceinline__ float offset_of(float m) { return m == -INFINITY ? 0.f : m; }

__device__ __forceinline__ void store_out(const DecodeArgs &a, int64_t at, float x) {
  if (a.out_dtype == GAR_F32)
    static_cast<float *>(a.out)[at] = x;
  else if (a.out_dtype == GAR_BF16)
    static_cast<__nv_bfloat16 *>(a.out)[at] = from_f32<__nv_bfloat16>(x);
  else
    static_cast<__half *>(a.out)[at] = from_f32<__half>(x);
}

// Where the queries of head h of a segment are.
__device__ __forceinline__ int64_t query_at(const DecodeArgs &a, const Segment &g, int h) { return g.b * a.qb + (g.head + h) * a.qh; }
__device__ __forceinline__ int64_t query_at(const ServingArgs &a, const Segment &g, int h) {
  if (a.share == 0) return g.b * a.qb + (g.head + h) * a.qh;
  const int m = g.head + h - g.kv_head * a.group, i = (int)a.by_heads((uint32_t)m);
  return ((int64_t)g.b * a.share + i) * a.qb + (g.kv_head * a.heads_each + (m - i * a.heads_each)) * a.qh;
}

__device__ __forceinline__ float load_q(const DecodeArgs &a, int64_t at) {
  if (a.q_dtype == GAR_F32) return static_cast<const float *>(a.q)[at];
  if (a.q_dtype == GAR_BF16) return to_f32(static_cast<const __nv_bfloat16 *>(a.q)[at]);
  return to_f32(static_cast<const __half *>(a.q)[at]);
}

__device__ __forceinline__ void store_lse(const DecodeArgs &a, const Segment &g, int h, float m, float l) {
  if (a.lse) a.lse[(int64_t)g.b * a.q_heads + g.head + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.693147180559945f;
}

// Four neighbouring elements of the output, where a.out_wide says that they can be stored at once.
__device__ __forceinline__ void store_wide4(const DecodeArgs &a, int64_t at, float x, float y, float z, float w) {
  if (a.out_dtype == GAR_F32) {
    *reinterpret_cast<float4 *>(static_cast<float *>(a.out) + at) = make_float4(x, y, z, w);
    return;
  }
  uint2 v;
  if (a.out_dtype == GAR_BF16)
    v = make_uint2(pack2(make_float2(x, y), __nv_bfloat16()), pack2(make_float2(z, w), __nv_bfloat16()));
  else
    v = make_uint2(pack2(make_float2(x, y), __half()), pack2(make_float2(z, w), __half()));
  *reinterpret_cast<uint2 *>(static_cast<char *>(a.out) + 2 * at) = v;
}

// Four neighbouring channels [d, d + 4) of query head h's output, x / l.
__device__ __forceinline__ void store_out4(const DecodeArgs &a, const Segment &g, int h, int d, float4 x, float l) {
  const float f = 1.f / l;
  if (l == 0.f)
    x = make_float4(0.f, 0.f, 0.f, 0.f);
  else
    x.x *= f, x.y *= f, x.z *= f, x.w *= f;
  const int64_t at = g.b * a.ob + (g.head + h) * a.oh + d;
  if (a.out_wide) return store_wide4(a, at, x.x, x.y, x.z, x.w);
  for (int i = 0; i < 4 && d + i < a.c.dim; ++i) store_out(a, at + i, i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w);
}

template <int WARPS> struct JoinShared {
  float2 ml[WARPS][kMaxGroup];     // each warp's m and l, written by the kernel
  int at[WARPS];                   // where in shared memory its o begins, in floats
  float weight[WARPS][kMaxGroup];  // 2^(m_w - m)
  float l[WARPS][kMaxGroup];       // l of the join that begins with this warp
  bool last[WARPS];
};

// `count` warps from `first` on that work on one segment.  Groups of a size are of the same warps
// (one warp apart), so the size can name the barrier.
struct Group {
  int first, count;
  __device__ __forceinline__ void sync() const {
    if (count == 1)
      __syncwarp();
    else
      asm volatile("bar.sync %0, %1;" ::"r"(count), "r"(32 * count) : "memory");
  }
  __device__ __forceinline__ int thread() const { return threadIdx.x - 32 * first; }
};

// Joins the (m, l, o) of a group's warps and writes the item's output, or the segment's partial
// result.  Warp w holds head h's o at o[at[w] + h * row], 16-byte aligned.
// With TWIST its channel d is at d ^ (h & 6); with FAR l may be far from 1 (8-bit caches).
template <int WARPS, bool TWIST = false, bool FAR = false>
__device__ __forceinline__ void join_warps(const DecodeArgs &a, const Segment &g, Group group, JoinShared<WARPS> &sh,
                                           const float *o, int row) {
  static_assert(WARPS <= 16, "16 lanes hold a head's warps");
  const int thread = group.thread(), threads = 32 * group.count;
  group.sync();
  for (int i = thread; i - (int)(threadIdx.x & 31) < g.heads * 16; i += threads) {
    const int h = i / 16, w = i & 15;
    const float2 v = w < group.count && h < g.heads ? sh.ml[group.first + w][h] : make_float2(-INFINITY, 0.f);
    float m = v.x;
#pragma unroll
    for (int d = 8; d > 0; d /= 2) m = fmaxf(m, __shfl_xor_sync(~0u, m, d));
    const float f = exp2_fast(v.x - offset_of(m));
    float l = FAR ? scaled<FAR>(v.y, v.x - offset_of(m)) : f * v.y;
#pragma unroll
    for (int d = 8; d > 0; d /= 2) l += __shfl_xor_sync(~0u, l, d);
    if (h < g.heads) {
      if (w < group.count) sh.weight[group.first + w][h] = f;
      if (w == 0) {
        sh.l[group.first][h] = l;
        if (g.whole)
          store_lse(a, g, h, m, l);
        else
          a.part_ml[g.slot * kMaxGroup + h] = make_float2(m, l);
      }
    }
  }
  group.sync();
  const int columns = (a.c.dim + 3) / 4;
  for (int i = thread; i < g.heads * columns; i += threads) {
    const int h = i / columns, d = (i - h * columns) * 4;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int w = group.first; w < group.first + group.count; ++w) {
      const float f = sh.weight[w][h];
      const float4 y = *reinterpret_cast<const float4 *>(o + sh.at[w] + h * row + (TWIST ? d ^ (h & 4) : d));
      x.x += f * y.x, x.y += f * y.y, x.z += f * y.z, x.w += f * y.w;
    }
    if (TWIST && (h & 2)) x = make_float4(x.z, x.w, x.x, x.y);
    if (g.whole)
      store_out4(a, g, h, d, x, sh.l[group.first][h]);
    else
      *reinterpret_cast<float4 *>(a.part_o + (int64_t)(g.slot * kMaxGroup + h) * a.dim_pad + d) = x;
  }
  group.sync();
}

// After join_warps: where the item has several parts, the last group to get here joins them, 8 parts' loads in flight a
// thread (a long sequence alone has some 20 parts of 4 KB for each cached head; 16 at once cost the kernel registers:
// 1 x 425 rows, 32/8 heads x 128 bf16 10.1 us in place of 8.9, 127 x 8192 e4m3 213 in place of 205).
template <int WARPS, bool FAR = false>
__device__ __forceinline__ void join_parts(const DecodeArgs &a, const Segment &g, Group group, JoinShared<WARPS> &sh) {
  if (group.thread() == 0) {
    // After join_warps' barrier: what the group has stored is seen before the count, and what others have stored after it.
    // The counter returns to zero with the last arrival.
    unsigned int before;
    asm volatile("atom.acq_rel.gpu.global.inc.u32 %0, [%1], %2;" : "=r"(before) : "l"(a.count + g.first), "r"(g.parts - 1) : "memory");
    sh.last[group.first] = before == (unsigned)g.parts - 1;
  }
  group.sync();
  if (sh.last[group.first]) {
    constexpr int N = 8;
    const int columns = (a.c.dim + 3) / 4;
    for (int i = group.thread(); i < g.heads * columns; i += 32 * group.count) {
      const int h = i / columns, d = (i - h * columns) * 4;
      float m = -INFINITY, l = 0.f;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int p0 = 0; p0 < g.parts; p0 += N) {
        float2 v[N];
        float4 y[N];
        float top = m;
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const int at = slot_of(g, min(p0 + k, g.parts - 1)) * kMaxGroup + h;
          v[k] = __ldcg(a.part_ml + at);
          y[k] = __ldcg(reinterpret_cast<const float4 *>(a.part_o + (int64_t)at * a.dim_pad + d));
        }
#pragma unroll
        for (int k = 0; k < N; ++k) top = fmaxf(top, v[k].x);
        const float off = offset_of(top), shrink = exp2_fast(m - off);
        l = FAR ? scaled<FAR>(l, m - off) : l * shrink, m = top;
        x.x *= shrink, x.y *= shrink, x.z *= shrink, x.w *= shrink;
#pragma unroll
        for (int k = 0; k < N; ++k)
          if (p0 + k < g.parts) {
            const float f = exp2_fast(v[k].x - off);
            l += FAR ? scaled<FAR>(v[k].y, v[k].x - off) : f * v[k].y;
            x.x += f * y[k].x, x.y += f * y[k].y, x.z += f * y[k].z, x.w += f * y[k].w;
          }
      }
      store_out4(a, g, h, d, x, l);
      if (d == 0) store_lse(a, g, h, m, l);
    }
  }
  group.sync();
}

// decode_mma_<cache>[_f32]: the cache's type, and 32-bit queries over 8 bits.
int decode_general(const DecodeArgs &a, int sms, gar_stream_t stream);
int decode_mma_bf16(const DecodeArgs &a, int sms, gar_stream_t stream);
int decode_mma_f16(const DecodeArgs &a, int sms, gar_stream_t stream);
int decode_mma_i8(const DecodeArgs &a, int sms, gar_stream_t stream);
int decode_mma_e4m3(const DecodeArgs &a, int sms, gar_stream_t stream);
int decode_mma_f32(const DecodeArgs &a, int sms, gar_stream_t stream);
int decode_mma_i8_f32(const DecodeArgs &a, int sms, gar_stream_t stream);
int decode_mma_e4m3_f32(const DecodeArgs &a, int sms, gar_stream_t stream);
int decode_general(const ServingArgs &a, int sms, gar_stream_t stream);
int decode_mma_bf16(const ServingArgs &a, int sms, gar_stream_t stream);
int decode_mma_f16(const ServingArgs &a, int sms, gar_stream_t stream);
int decode_mma_i8(const ServingArgs &a, int sms, gar_stream_t stream);
int decode_mma_e4m3(const ServingArgs &a, int sms, gar_stream_t stream);
int decode_mma_f32(const ServingArgs &a, int sms, gar_stream_t stream);
int decode_mma_i8_f32(const ServingArgs &a, int sms, gar_stream_t stream);
int decode_mma_e4m3_f32(const ServingArgs &a, int sms, gar_stream_t stream);

}  // namespace gar
