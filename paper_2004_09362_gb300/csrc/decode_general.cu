// Decode attention without tensor cores: head sizes and rows that are no multiple of 16 bytes.
#include <algorithm>

#include "decode.cuh"

namespace gar {
namespace {

constexpr int kHeads = 8;   // query heads of an item
constexpr int kRows = 4;    // rows a warp takes at once
constexpr int kWarps = 4, kThreads = 32 * kWarps;

// A warp takes kRows rows at a time; its lanes hold every 32nd channel (J each) of the rows, the
// queries and the outputs.  The 4 x 8 products of rows and heads are summed over the lanes by an
// exchange that halves the values with each step, so that 31 shuffles do them all and lane
// 8 r + h is left with the score of row r and head h.  Bound by arithmetic and by latency; the
// rows' loads (8 J of 128 bytes a warp) are in flight together.
//
// 16 sequences of up to 8192 rows, 32/8 heads x 100 channels bf16: 372 us (0.5 TB/s); the tensor cores'
// kernel needs 43 us for 96 channels, this one 378.  7 sequences of up to 2000 rows, 6/6 x 80 f32: 21 us, that one 18.
template <typename T, int J> __global__ void __launch_bounds__(kThreads) general_kernel(const DecodeArgs a) {
  __shared__ JoinShared<kWarps> join;
  extern __shared__ __align__(16) float o_shared[];
  const gar_kv_cache &c = a.c;
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const int row = lane / 8, head = lane & 7;
  const int o_row = J * 32;
  after_earlier_kernels();
  Walk walk;
  walk.start(a);
  const Group group{0, kWarps};
  if (lane == 0) join.at[warp] = warp * kHeads * o_row;
  Segment g;
  while (walk.next(a, &g)) {
    float q[kHeads][J], o[kHeads][J], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int h = 0; h < kHeads; ++h)
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int d = lane + 32 * j;
        q[h][j] = h < g.heads && d < c.dim ? load_q(a, g.b * a.qb + (g.head + h) * a.qh + d) : 0.f;
        o[h][j] = 0.f;
      }
    const int lo = g.lo;
    for (int n0 = g.from + warp * kRows; n0 < g.to; n0 += kWarps * kRows) {
      // Lane r < kRows finds row r.
      const int n = n0 + (lane & (kRows - 1));
      int64_t at = -1, at_scale = 0;
      if (n >= lo && n < g.to) {
        const int p = (int)a.page(n), r = n - p * c.page_size;
        const int page = a.table[g.b * a.table_stride + p];
        if ((unsigned)page < (uint64_t)c.pages) {
          at = page * c.page_stride + g.kv_head * c.head_stride + r * c.token_stride;
          at_scale = page * c.scale_page_stride + g.kv_head * c.scale_head_stride + r * c.scale_token_stride;
        } else if (c.status) {
          atomicOr(c.status, GAR_KV_BAD_PAGE);
        }
      }
      float k[kRows][J], v[kRows][J], ks[kRows], vs[kRows];
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        const int64_t x = __shfl_sync(~0u, at, r), y = __shfl_sync(~0u, at_scale, r);
        ks[r] = quantised<T>::value && x >= 0 ? c.k_scale[y] : 1.f;
        vs[r] = quantised<T>::value && x >= 0 ? c.v_scale[y] : 1.f;
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const int d = lane + 32 * j;
          const bool there = x >= 0 && d < c.dim;
          k[r][j] = there ? to_f32(static_cast<const T *>(c.k)[x + d]) : 0.f;
          v[r][j] = there ? to_f32(static_cast<const T *>(c.v)[x + d]) : 0.f;
        }
      }
      float s[32];
#pragma unroll
      for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int h = 0; h < kHeads; ++h) {
          float x = 0.f;
#pragma unroll
          for (int j = 0; j < J; ++j) x = fmaf(q[h][j], k[r][j], x);
          s[r * kHeads + h] = quantised<T>::value ? x * ks[r] : x;
        }
#pragma unroll
      for (int w = 16; w > 0; w /= 2)
#pragma unroll
        for (int i = 0; i < w; ++i) {
          const bool up = lane & w;
          const float keep = up ? s[i + w] : s[i], give = up ? s[i] : s[i + w];
          s[i] = keep + __shfl_xor_sync(~0u, give, w);
        }
      const int mine = n0 + row;
      const float y = mine >= lo && mine < g.to ? s[0] * a.scale_log2 : -INFINITY;
      float top = fmaxf(m, y);
      top = fmaxf(top, __shfl_xor_sync(~0u, top, 8));
      top = fmaxf(top, __shfl_xor_sync(~0u, top, 16));
      const float off = offset_of(top), shrink = exp2_fast(m - off), p = exp2_fast(y - off);
      l = l * shrink + p;
      if (__any_sync(~0u, top > m)) {
#pragma unroll
        for (int h = 0; h < kHeads; ++h) {
          const float f = __shfl_sync(~0u, shrink, h);
#pragma unroll
          for (int j = 0; j < J; ++j) o[h][j] *= f;
        }
      }
      m = top;
#pragma unroll
      for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int h = 0; h < kHeads; ++h) {
          const float f = __shfl_sync(~0u, p, r * 8 + h) * vs[r];
#pragma unroll
          for (int j = 0; j < J; ++j) o[h][j] = fmaf(f, v[r][j], o[h][j]);
        }
    }
    l += __shfl_xor_sync(~0u, l, 8);
    l += __shfl_xor_sync(~0u, l, 16);
    if (row == 0) join.ml[warp][head] = make_float2(m, l);
#pragma unroll
    for (int h = 0; h < kHeads; ++h)
#pragma unroll
      for (int j = 0; j < J; ++j) o_shared[(warp * kHeads + h) * o_row + lane + 32 * j] = o[h][j];
    join_warps(a, g, group, join, o_shared, o_row);
    if (!g.whole) join_parts(a, g, group, join);
  }
}

template <typename T, int J> int launch_general(DecodeArgs a, int sms, gar_stream_t stream) {
  const size_t shared = sizeof(float) * kWarps * kHeads * J * 32;
  a.item_heads = std::min(a.group, kHeads);
  a.item_groups = (a.group + kHeads - 1) / kHeads;
  return launch("gar_decode_attention", general_kernel<T, J>, sms * (J <= 4 ? 4 : 2), kThreads, shared, stream, a);
}

template <typename T> int by_dim(const DecodeArgs &a, int sms, gar_stream_t stream) {
  return a.c.dim <= 64 ? launch_general<T, 2>(a, sms, stream) : a.c.dim <= 128 ? launch_general<T, 4>(a, sms, stream) : launch_general<T, 8>(a, sms, stream);
}

}  // namespace

int decode_general(const DecodeArgs &a, int sms, gar_stream_t stream) {
  switch (a.c.dtype) {
    case GAR_F32: return by_dim<float>(a, sms, stream);
    case GAR_BF16: return by_dim<__nv_bfloat16>(a, sms, stream);
    case GAR_F16: return by_dim<__half>(a, sms, stream);
    case GAR_I8: return by_dim<i8>(a, sms, stream);
    default: return by_dim<e4m3>(a, sms, stream);
  }
}

}  // namespace gar
