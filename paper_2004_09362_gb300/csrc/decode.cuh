// What the decode-attention kernels share: their arguments, the division of the cache's rows
// among CTAs, and the join of partial results.
//
// Work.  An item is one sequence, one cached head and a group of up to kMaxGroup of the query heads
// that read it.  Its rows are cut into units of 64 (more where the line would pass 2^31 units);
// the items' units stand one behind the other in one line, and CTA i of N takes the i-th of
// N equal shares of the line.  So every CTA has the same number of rows to read whatever the
// lengths are, one long sequence is spread over the whole GPU, and thousands of short ones
// are not split at all.  Where the line is longer than the CTAs are many, each item counts one
// unit more, for what it costs beside its rows.  The lengths are read on the device: nothing waits for the
// host, and a captured launch stays right when they change.
//
// Join.  A segment is the part of an item that one CTA takes.  Each keeps the running maximum m
// of the scores (in units of log 2), l = sum 2^(score - m) and o = sum 2^(score - m) v.  Where an
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
  int unit_shift;          // rows of a unit: 1 << unit_shift
  int box_rows;            // rows of a tensor copy
  int batch, q_heads, group, item_groups, item_heads;  // group: q_heads / kv_heads
  int q_dtype, out_dtype, window;
  bool out_wide;           // four neighbouring outputs can be stored at once
  float scale_log2;        // scale * log2(e)
  // workspace: per CTA two segments' (m, l) and o, and a counter
  float2 *part_ml;
  float *part_o;
  unsigned int *count;
  int dim_pad;             // floats of a stored o row
};

struct Span {
  int units;
  int lo, hi, base;        // rows [lo, hi); base: lo rounded down to a multiple of 32
};

__device__ __forceinline__ Span span_of(const DecodeArgs &a, int n) {
  Span s;
  if (n < 0 || n > a.most_rows) {
    if (a.c.status) atomicOr(a.c.status, GAR_KV_BAD_LENGTH);
    n = n < 0 ? 0 : a.most_rows;
  }
  s.hi = n;
  s.lo = a.window > 0 && n > a.window ? n - a.window : 0;
  s.base = s.lo & ~31;
  s.units = max(1, (s.hi - s.base + (1 << a.unit_shift) - 1) >> a.unit_shift);
  return s;
}

// Rows [max(lo, from), to) of one item.
struct Segment {
  int b, kv_head, head, heads;  // head: the first of the item's query heads
  int lo, from, to;             // from is a multiple of 32
  bool whole;
  int slot;                     // where the partial result goes
  int first, parts;             // the item's CTAs
  bool first_late;              // the first of them begins before the item does
};

// Walks one CTA's share.  All threads hold the same state.
struct Walk {
  int pos, end, per;
  int item;                     // where in the line the item at pos begins
  int b, hh, lead;
  int ahead;                    // length of sequence b + 1
  bool first_segment;
  Span s;

  __device__ __forceinline__ int length(const DecodeArgs &a, int i) const { return i < a.batch ? a.lengths[i] : 0; }

  template <int THREADS> __device__ __forceinline__ void start(const DecodeArgs &a) {
    // Each thread adds up a run of sequences, a scan over the threads follows, and the thread
    // whose run holds the share's start looks it up.
    __shared__ int sums[THREADS / 32];
    __shared__ int found_item, found_b;
    const int per_thread = (a.batch + THREADS - 1) / THREADS;
    const int b0 = min(a.batch, (int)threadIdx.x * per_thread), b1 = min(a.batch, b0 + per_thread);
    const int items = a.c.heads * a.item_groups;
    int mine = 0;
    for (int i = b0; i < b1; ++i) mine += span_of(a, a.lengths[i]).units;
    int scan = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int up = __shfl_up_sync(~0u, scan, d);
      if ((threadIdx.x & 31) >= d) scan += up;
    }
    if ((threadIdx.x & 31) == 31) sums[threadIdx.x / 32] = scan;
    __syncthreads();
    int before = scan - mine, total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
      if (w < threadIdx.x / 32) before += sums[w];
      total += sums[w];
    }
    lead = total * items > (int)gridDim.x ? 1 : 0;
    total = (total + lead * a.batch) * items;
    before = (before + lead * b0) * items, mine = (mine + lead * (b1 - b0)) * items;
    per = (total + gridDim.x - 1) / gridDim.x;
    pos = min(total, (int)blockIdx.x * per);
    end = min(total, pos + per);
    if (pos >= before && pos < before + mine) {
      int i = b0;
      for (; i < b1; ++i) {
        const int n = (span_of(a, a.lengths[i]).units + lead) * items;
        if (pos < before + n) break;
        before += n;
      }
      found_b = i, found_item = before;
    }
    __syncthreads();
    if (pos >= end) return;
    enter(a, found_b, a.lengths[found_b]);
    hh = (pos - found_item) / s.units;
    item = found_item + hh * s.units;
    first_segment = true;
  }

  __device__ __forceinline__ void enter(const DecodeArgs &a, int sequence, int n) {
    b = sequence;
    s = span_of(a, n);
    s.units += lead;
    ahead = length(a, b + 1);
  }

  __device__ __forceinline__ bool next(const DecodeArgs &a, Segment *g) {
    if (pos >= end) return false;
    if (!first_segment) {
      if (++hh == a.c.heads * a.item_groups) hh = 0, enter(a, b + 1, ahead);
      item = pos;
    }
    const int u = pos - item, n = min(s.units - u, end - pos);
    g->b = b;
    g->kv_head = a.item_groups == 1 ? hh : hh / a.item_groups;
    const int sub = (hh - g->kv_head * a.item_groups) * a.item_heads;
    g->head = g->kv_head * a.group + sub;
    g->heads = min(a.item_heads, a.group - sub);
    g->from = s.base + (max(0, u - lead) << a.unit_shift);
    g->to = min(s.hi, s.base + (max(0, u + n - lead) << a.unit_shift));
    g->lo = max(s.lo, g->from);
    g->whole = n == s.units;
    g->first = blockIdx.x, g->parts = 1, g->slot = 0, g->first_late = false;
    if (!g->whole) {
      g->slot = 2 * blockIdx.x + (first_segment ? 0 : 1);
      g->first = item / per;
      g->parts = (item + s.units - 1) / per - g->first + 1;
      g->first_late = g->first * per < item;
    }
    pos += n;
    first_segment = false;
    return true;
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

__device__ __forceinline__ float load_q(const DecodeArgs &a, int64_t at) {
  if (a.q_dtype == GAR_F32) return static_cast<const float *>(a.q)[at];
  if (a.q_dtype == GAR_BF16) return to_f32(static_cast<const __nv_bfloat16 *>(a.q)[at]);
  return to_f32(static_cast<const __half *>(a.q)[at]);
}

__device__ __forceinline__ void store_lse(const DecodeArgs &a, const Segment &g, int h, float m, float l) {
  if (a.lse) a.lse[(int64_t)g.b * a.q_heads + g.head + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.693147180559945f;
}

// Four neighbouring channels [d, d + 4) of query head h's output, x / l.
__device__ __forceinline__ void store_out4(const DecodeArgs &a, const Segment &g, int h, int d, float4 x, float l) {
  const float f = 1.f / l;
  if (l == 0.f)
    x = make_float4(0.f, 0.f, 0.f, 0.f);
  else
    x.x *= f, x.y *= f, x.z *= f, x.w *= f;
  const int64_t at = g.b * a.ob + (g.head + h) * a.oh + d;
  if (a.out_wide) {
    if (a.out_dtype == GAR_F32) {
      *reinterpret_cast<float4 *>(static_cast<float *>(a.out) + at) = x;
    } else {
      uint2 y;
      if (a.out_dtype == GAR_BF16) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(x.x, x.y), q = __floats2bfloat162_rn(x.z, x.w);
        y = make_uint2(*reinterpret_cast<const uint32_t *>(&p), *reinterpret_cast<const uint32_t *>(&q));
      } else {
        const __half2 p = __floats2half2_rn(x.x, x.y), q = __floats2half2_rn(x.z, x.w);
        y = make_uint2(*reinterpret_cast<const uint32_t *>(&p), *reinterpret_cast<const uint32_t *>(&q));
      }
      *reinterpret_cast<uint2 *>(static_cast<char *>(a.out) + 2 * at) = y;
    }
    return;
  }
  for (int i = 0; i < 4 && d + i < a.c.dim; ++i) store_out(a, at + i, i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w);
}

template <int WARPS> struct JoinShared {
  float2 ml[WARPS][kMaxGroup];     // each warp's m and l, written by the kernel
  int at[WARPS];                   // where in shared memory its o begins, in floats
  float weight[WARPS][kMaxGroup];  // 2^(m_w - m)
  float l[WARPS][kMaxGroup];       // l of the join that begins with this warp
  float m[kMaxGroup];
  bool last;
};

// Joins the (m, l, o) of `count` warps from `first` on, by the `threads` threads that
// call it, and writes the item's output, or the segment's partial result.
// Warp w holds head h's o at o[at[w] + h * row], 16-byte aligned.
template <int WARPS, typename Barrier>
__device__ __forceinline__ void join_warps(const DecodeArgs &a, const Segment &g, JoinShared<WARPS> &sh, const float *o, int row,
                                           int first, int count, int thread, int threads, Barrier barrier) {
  barrier();
  if (thread < g.heads) {
    const int h = thread;
    float m = -INFINITY, l = 0.f;
    for (int w = first; w < first + count; ++w) m = fmaxf(m, sh.ml[w][h].x);
    for (int w = first; w < first + count; ++w) {
      const float f = exp2_fast(sh.ml[w][h].x - offset_of(m));
      sh.weight[w][h] = f;
      l += f * sh.ml[w][h].y;
    }
    sh.l[first][h] = l;
    if (g.whole)
      store_lse(a, g, h, m, l);
    else
      a.part_ml[g.slot * kMaxGroup + h] = make_float2(m, l);
  }
  barrier();
  const int columns = (a.c.dim + 3) / 4;
  for (int i = thread; i < g.heads * columns; i += threads) {
    const int h = i / columns, d = (i - h * columns) * 4;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int w = first; w < first + count; ++w) {
      const float f = sh.weight[w][h];
      const float4 y = *reinterpret_cast<const float4 *>(o + sh.at[w] + h * row + d);
      x.x += f * y.x, x.y += f * y.y, x.z += f * y.z, x.w += f * y.w;
    }
    if (g.whole)
      store_out4(a, g, h, d, x, sh.l[first][h]);
    else
      *reinterpret_cast<float4 *>(a.part_o + (int64_t)(g.slot * kMaxGroup + h) * a.dim_pad + d) = x;
  }
  barrier();
}

// After join_warps by the whole CTA: where the item has several parts, the last CTA to get here
// joins them.  A lane for each part finds the maximum; then every thread has the loads of 8 parts
// in flight (a long sequence alone has some 20 parts of 4 KB for each cached head).
template <int WARPS>
__device__ __forceinline__ void join_parts(const DecodeArgs &a, const Segment &g, JoinShared<WARPS> &sh) {
  __threadfence();
  __syncthreads();
  // The counter returns to zero with the last arrival.
  if (threadIdx.x == 0) sh.last = atomicInc(a.count + g.first, g.parts - 1) == (unsigned)g.parts - 1;
  __syncthreads();
  if (sh.last) {
    __threadfence();
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    for (int h = warp; h < g.heads; h += WARPS) {
      float m = -INFINITY;
      for (int p = lane; p < g.parts; p += 32) m = fmaxf(m, __ldcg(a.part_ml + slot_of(g, p) * kMaxGroup + h).x);
#pragma unroll
      for (int d = 16; d > 0; d /= 2) m = fmaxf(m, __shfl_xor_sync(~0u, m, d));
      if (lane == 0) sh.m[h] = m;
    }
    __syncthreads();
    const int columns = (a.c.dim + 3) / 4;
    for (int i = threadIdx.x; i < g.heads * columns; i += 32 * WARPS) {
      const int h = i / columns, d = (i - h * columns) * 4;
      const float m = sh.m[h], off = offset_of(m);
      float l = 0.f;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
      for (int p = 0; p < g.parts; ++p) {
        const int at = slot_of(g, p) * kMaxGroup + h;
        const float2 v = __ldcg(a.part_ml + at);
        const float4 y = __ldcg(reinterpret_cast<const float4 *>(a.part_o + (int64_t)at * a.dim_pad + d));
        const float f = exp2_fast(v.x - off);
        l += f * v.y;
        x.x += f * y.x, x.y += f * y.y, x.z += f * y.z, x.w += f * y.w;
      }
      store_out4(a, g, h, d, x, l);
      if (d == 0) store_lse(a, g, h, m, l);
    }
  }
  __syncthreads();
}

int decode_general(const DecodeArgs &a, int sms, cudaStream_t stream);
int decode_mma_bf16(const DecodeArgs &a, int sms, cudaStream_t stream);
int decode_mma_f16(const DecodeArgs &a, int sms, cudaStream_t stream);
int decode_mma_i8(const DecodeArgs &a, int sms, cudaStream_t stream);
int decode_mma_e4m3(const DecodeArgs &a, int sms, cudaStream_t stream);

}  // namespace gar
