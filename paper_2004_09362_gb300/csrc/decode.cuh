// What the decode-attention kernels share: their arguments, the division of the cache's rows
// among CTAs, and the join of partial results.
//
// Work.  An item is one sequence, one cached head and a group of up to G of the query heads that
// read it.  Its rows are cut into units of kUnit; the items' units stand one behind the other
// in one line, and CTA i of N takes the i-th of N equal shares of the line.  So every CTA has the same number of rows
// to read whatever the lengths are, one long sequence is spread over the whole GPU, and thousands
// of short ones are not split at all.  The lengths are read on the device: nothing waits for
// the host, and a captured launch stays right when they change.
//
// Join.  A segment is the part of an item that one CTA takes.  Each keeps the running maximum m
// of the scores (in units of log 2), l = sum 2^(score - m) and o = sum 2^(score - m) v.  Where an
// item has several segments, each CTA stores (m, l, o), and the one that arrives last at the
// item's counter adds them up in the order of the rows (so the bits do not depend on who
// was last):  m = max m_i,  l = sum l_i 2^(m_i - m),  o likewise.
#pragma once

#include "gar_device.cuh"

namespace gar {

constexpr int kDecodeThreads = 128;
constexpr int kDecodeWarps = kDecodeThreads / 32;
constexpr int kUnit = 64;             // rows
constexpr int kMaxGroup = 16;         // query heads of an item
constexpr int kMaxCtas = 152 * 8;

// n / d for n < 2^31.
struct Divide {
  uint32_t mul, shift;
  __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return (__umulhi(mul, n) + n) >> shift; }
};

struct DecodeArgs {
  gar_kv_cache c;
  const void *q;
  void *out;
  float *lse;
  int64_t qb, qh, ob, oh, table_stride;
  const int32_t *table, *lengths;
  Divide page;
  int64_t most_rows;       // rows that the table's width can hold
  int batch, q_heads, group, item_groups, item_heads;  // group: q_heads / kv_heads
  int q_dtype, out_dtype, window;
  float scale_log2;        // scale * log2(e)
  // workspace: per CTA two segments' (m, l) and o, and a counter
  float *part_ml, *part_o;
  unsigned int *count;
  int dim_pad;             // floats of a stored o row
};

struct Span {
  int64_t units;
  int lo, hi, base;        // rows [lo, hi); base: lo rounded down to a multiple of 32
};

__device__ __forceinline__ Span span_of(const DecodeArgs &a, int b) {
  Span s;
  int64_t n = a.lengths[b];
  if (n < 0 || n > a.most_rows) {
    if (a.c.status) atomicOr(a.c.status, GAR_KV_BAD_LENGTH);
    n = n < 0 ? 0 : a.most_rows;
  }
  s.hi = (int)n;
  s.lo = a.window > 0 && n > a.window ? (int)(n - a.window) : 0;
  s.base = s.lo & ~31;
  s.units = max(1, (s.hi - s.base + kUnit - 1) / kUnit);
  return s;
}

// A segment: rows [max(lo, from), min(hi, to)) of item (b, cached head, first query head).
struct Segment {
  int b, kv_head, head, heads;
  int from, to;            // from is a multiple of 32
  bool whole;
  int slot;                // where the partial result goes
  int first, parts;        // the item's CTAs
  int64_t first_from;      // units of the line before the item
};

// Walks one CTA's share.  All threads hold the same state.
struct Walk {
  int64_t pos, end, per;
  int64_t item;            // where in the line the item at pos begins
  int b, hh;
  bool first_segment;
  Span s;

  __device__ __forceinline__ void start(const DecodeArgs &a) {
    // Each thread adds up a run of sequences, a scan over the threads follows, and the thread
    // whose run holds the share's start looks it up.
    __shared__ int64_t sums[kDecodeWarps];
    __shared__ int64_t found_item;
    __shared__ int found_b;
    const int per_thread = (a.batch + kDecodeThreads - 1) / kDecodeThreads;
    const int b0 = min(a.batch, (int)threadIdx.x * per_thread), b1 = min(a.batch, b0 + per_thread);
    const int items = a.c.heads * a.item_groups;
    int64_t mine = 0;
    for (int i = b0; i < b1; ++i) mine += span_of(a, i).units;
    int64_t scan = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int64_t up = __shfl_up_sync(~0u, scan, d);
      if ((threadIdx.x & 31) >= d) scan += up;
    }
    if ((threadIdx.x & 31) == 31) sums[threadIdx.x / 32] = scan;
    __syncthreads();
    int64_t before = scan - mine, total = 0;
    for (int w = 0; w < kDecodeWarps; ++w) {
      if (w < threadIdx.x / 32) before += sums[w];
      total += sums[w];
    }
    total *= items, before *= items, mine *= items;
    per = (total + gridDim.x - 1) / gridDim.x;
    pos = blockIdx.x * per;
    end = min(total, pos + per);
    if (pos >= before && pos < before + mine) {
      int i = b0;
      for (; i < b1; ++i) {
        const int64_t n = span_of(a, i).units * items;
        if (pos < before + n) break;
        before += n;
      }
      found_b = i, found_item = before;
    }
    __syncthreads();
    if (pos >= end) return;
    b = found_b;
    s = span_of(a, b);
    hh = (int)((pos - found_item) / s.units);
    item = found_item + hh * s.units;
    first_segment = true;
  }

  __device__ __forceinline__ bool next(const DecodeArgs &a, Segment *g) {
    if (pos >= end) return false;
    if (!first_segment) {
      if (++hh == a.c.heads * a.item_groups) hh = 0, s = span_of(a, ++b);
      item = pos;
    }
    const int64_t u = pos - item, n = min(s.units - u, end - pos);
    g->b = b;
    g->kv_head = hh / a.item_groups;
    const int sub = (hh - g->kv_head * a.item_groups) * a.item_heads;
    g->head = g->kv_head * a.group + sub;
    g->heads = min(a.item_heads, a.group - sub);
    g->from = s.base + (int)u * kUnit;
    g->to = min(s.hi, s.base + (int)(u + n) * kUnit);
    g->whole = n == s.units;
    g->slot = 2 * blockIdx.x + (first_segment ? 0 : 1);
    g->first = (int)(item / per);
    g->parts = (int)((item + s.units - 1) / per) - g->first + 1;
    g->first_from = item;
    pos += n;
    first_segment = false;
    return true;
  }

  // The place of part i of the item's parts: a CTA's second segment when its share begins before the item.
  __device__ __forceinline__ int slot_of(const Segment &g, int i) const {
    const int cta = g.first + i;
    return 2 * cta + (i == 0 && cta * per < g.first_from ? 1 : 0);
  }
};

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

// Joins the warps' (m, l, o) in shared memory, then the CTAs' where the item has several.
// Warp w holds head h's m, l at ml[(w * kMaxGroup + h) * 2] and its o at o[(w * group_rows + h) * row].
__device__ __forceinline__ void finish(const DecodeArgs &a, const Walk &walk, const Segment &g, const float *ml,
                                       const float *o, int group_rows, int row) {
  const int dim = a.c.dim;
  __syncthreads();
  for (int i = threadIdx.x; i < g.heads * dim; i += kDecodeThreads) {
    const int h = i / dim, d = i - h * dim;
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < kDecodeWarps; ++w) m = fmaxf(m, ml[(w * kMaxGroup + h) * 2]);
    float l = 0.f, x = 0.f;
#pragma unroll
    for (int w = 0; w < kDecodeWarps; ++w) {
      const float f = exp2_fast(ml[(w * kMaxGroup + h) * 2] - offset_of(m));
      l += f * ml[(w * kMaxGroup + h) * 2 + 1];
      x += f * o[(w * group_rows + h) * row + d];
    }
    if (g.whole) {
      store_out(a, g.b * a.ob + (g.head + h) * a.oh + d, l == 0.f ? 0.f : x / l);
      if (d == 0) store_lse(a, g, h, m, l);
    } else {
      const int64_t at = (int64_t)g.slot * kMaxGroup + h;
      a.part_o[at * a.dim_pad + d] = x;
      if (d == 0) a.part_ml[at * 2] = m, a.part_ml[at * 2 + 1] = l;
    }
  }
  if (!g.whole) {
    __shared__ bool last;
    __threadfence();
    __syncthreads();
    // The counter returns to zero with the last arrival.
    if (threadIdx.x == 0) last = atomicInc(a.count + g.first, g.parts - 1) == (unsigned)g.parts - 1;
    __syncthreads();
    if (last) {
      __threadfence();
      for (int i = threadIdx.x; i < g.heads * dim; i += kDecodeThreads) {
        const int h = i / dim, d = i - h * dim;
        float m = -INFINITY;
        for (int p = 0; p < g.parts; ++p) m = fmaxf(m, __ldcg(a.part_ml + ((int64_t)walk.slot_of(g, p) * kMaxGroup + h) * 2));
        float l = 0.f, x = 0.f;
        for (int p = 0; p < g.parts; ++p) {
          const int64_t at = (int64_t)walk.slot_of(g, p) * kMaxGroup + h;
          const float2 v = __ldcg(reinterpret_cast<const float2 *>(a.part_ml) + at);
          const float f = exp2_fast(v.x - offset_of(m));
          l += f * v.y;
          x += f * __ldcg(a.part_o + at * a.dim_pad + d);
        }
        store_out(a, g.b * a.ob + (g.head + h) * a.oh + d, l == 0.f ? 0.f : x / l);
        if (d == 0) store_lse(a, g, h, m, l);
      }
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
