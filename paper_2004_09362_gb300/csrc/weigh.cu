// The attention weights that cached rows gather: out[n] = weights[n] + sum_j exp(scale q_j.k_n - lse_j).
//
// Bound by memory: each key is read once for all the queries of its head, values not at all.  Scores are computed on tensor
// cores as in decode attention, S^T = K Q^T with 16 rows of the cache by 8 queries: which channel sits at which place of the summed
// dimension is free as long as keys and queries agree, so a lane's part of a row is whole 16-byte chunks (lane t of the
// four that share a row has chunks t, t + 4, ...).  A warp copies its rows to a ring of its own, two tiles and more ahead.  The rows of all
// sequences are shared out among the CTAs as in decode attention, by equal numbers; entries of other rows are copied by a
// warp of their own beside that.
//
// 24 x up to 8192 rows, 32/8 x 128 bf16: 49 us, 4.3 TB/s; 1 x 1021, 10/5 x 80 f16: 5 us.  What is missing to the copy rate are the ends of
// segments, where a CTA has nothing on its way.
//
// 8-bit codes become f16 exactly, as do the queries that go with them: the head's largest is brought to 2^14, 32-bit ones in two
// parts.  Keys of 32 bits are multiplied in 32 bits without tensor cores.
#include <algorithm>
#include <climits>
#include <cmath>

#include "decode_mma.cuh"

namespace gar {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kHeads = 32;  // queries whose parts lie in shared memory at a time

struct WeighArgs {
  ServingArgs d;
  const float *lse, *weights;
  float *out;
  int64_t wb, wh, ob, oh, rows;
  bool apart;                // out is not weights
};

// A query head's factor of the scores and log2 of the sum of its weights; infinite: it adds nothing.
__device__ __forceinline__ float2 factor_of(const WeighArgs &a, int b, int head, int q_head, float up) {
  const float x = a.lse[(int64_t)b * a.d.q_heads + q_head];
  return make_float2(up * a.d.scale_log2, x == -INFINITY ? INFINITY : x * 1.44269504088896341f);
}
__device__ __forceinline__ float weight_of(float score, float2 f) {
  return f.y == INFINITY ? 0.f : exp2_fast(fmaf(score, f.x, -f.y));
}

// The warps that weigh.
__device__ __forceinline__ void sync_weighing() { asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory"); }

// Entries of rows that the sequences do not have, or not in their window: by the CTA's last warp, beside the others.
__device__ __forceinline__ void copy_rest(const WeighArgs &a) {
  if (!a.apart) return;
  constexpr int N = 8;  // loads in flight
  const int lane = threadIdx.x & 31, items = a.d.batch * a.d.c.heads, parts = max(1, (int)gridDim.x / items);
  for (int64_t i = blockIdx.x; i < (int64_t)items * parts; i += gridDim.x) {
    const int item = (int)(i / parts), part = (int)(i - (int64_t)item * parts);
    const int b = (int)a.d.items((uint32_t)item), h = item - b * a.d.c.heads;
    const Span s = span_of(a.d, a.d.lengths[b], 64);
    const float *const from = a.weights + b * a.wb + h * a.wh;
    float *const to = a.out + b * a.ob + h * a.oh;
    const int64_t rest = a.rows - (s.hi - s.lo), each = (rest + parts - 1) / parts, end = min(rest, (part + 1) * each);
    for (int64_t k0 = part * each + lane; k0 < end; k0 += 32 * N) {
      float x[N];
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int64_t k = k0 + 32 * j;
        x[j] = k < end ? from[k < s.lo ? k : k + (s.hi - s.lo)] : 0.f;
      }
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int64_t k = k0 + 32 * j;
        if (k < end) to[k < s.lo ? k : k + (s.hi - s.lo)] = x[j];
      }
    }
  }
}

// A CTA's walk over its segments, kept in shared memory: in the registers it cost the keys their places.
struct Course {
  Walk walk;
  Segment segment;
  int more;
  __device__ __forceinline__ void start(const ServingArgs &d) {
    if (threadIdx.x < 32) {
      Walk w;
      w.start(d);
      if (threadIdx.x == 0) walk = w;
    }
  }
  // By all threads; the segment stays until the next call.
  __device__ __forceinline__ bool next(const ServingArgs &d) {
    sync_weighing();
    if (threadIdx.x == 0) {
      Walk w = walk;
      Segment s;
      more = w.next(d, &s);
      walk = w, segment = s;
    }
    sync_weighing();
    return more != 0;
  }
};

// Where a row's keys are and, over 8-bit caches, its scale; -1: on no page, or outside the segment.
__device__ __forceinline__ int64_t key_at(const DecodeArgs &d, const Segment &g, int n, int64_t *scale) {
  *scale = 0;
  if (n < g.lo || n >= g.to) return -1;
  const int p = (int)d.page((uint32_t)n), page = d.table[g.b * d.table_stride + p], row = n - p * d.c.page_size;
  if ((unsigned)page >= (uint64_t)d.c.pages) {
    if (d.c.status) atomicOr(d.c.status, GAR_KV_BAD_PAGE);
    return -1;
  }
  *scale = page * d.c.scale_page_stride + g.kv_head * d.c.scale_head_stride + row * d.c.scale_token_stride;
  return page * d.c.page_stride + g.kv_head * d.c.head_stride + row * d.c.token_stride;
}

// KC: 16-byte chunks of a row in a lane; Q32: 32-bit queries over 8-bit keys.
template <typename C, int KC, bool Q32> struct WeighShape {
  static constexpr int CH = 16 / sizeof(C);                    // channels of a chunk
  static constexpr int W4 = CH / 8;                            // 16-byte words of a chunk's queries
  static constexpr int PARTS = Q32 ? 2 : 1;
  static constexpr int CHUNKS = 4 * KC, ROW = 64 * KC;         // of a row: chunks, bytes
  static constexpr int kStage = 16 * ROW + 128;                // a tile's keys, 16 weights, 16 scales
  // CTAs of an SM, and tiles of a ring: two where their rings fit.  (24 x 8192, 32/8 heads x 128 bf16 49 us, by one CTA 59; i8 41 and 55; x 96 bf16 43 and 55.  Rings
  // of half as many tiles 48, 41 and 42; of half as many again, which leaves one CTA for up to 192 bytes, 49, 58 and 57.)
  static constexpr int kResident = KC <= 4 ? 2 : 1;
  static constexpr int kStages = KC == 1 ? 8 : KC == 2 ? 6 : KC == 3 ? 4 : 3;
  static constexpr int kRings = kWarps * kStages * kStage;
  // Where chunk c of row r lies: rows of a multiple of 128 bytes twisted, so that the 8 lanes of a read meet all banks.
  static __device__ __forceinline__ int place(int r, int c) { return KC % 2 == 0 ? c ^ (r & 1) * 4 : c; }
  // words: [group of 8 queries][part][chunk][W4][lane]
  static constexpr int kGroup = PARTS * KC * W4 * 32;
};

template <typename C, int KC, bool Q32> __global__ void __launch_bounds__(kThreads + 32, WeighShape<C, KC, Q32>::kResident) weigh_mma(const WeighArgs a) {
  using S = WeighShape<C, KC, Q32>;
  using T = typename operand<C>::type;
  constexpr bool Q8 = quantised<C>::value;
  extern __shared__ __align__(16) char shared[];
  constexpr int STEP = 16 * kWarps;
  __shared__ float2 factor[kHeads];
  __shared__ float down[kHeads];
  const ServingArgs &d = a.d;
  const gar_kv_cache &c = d.c;
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31, g = lane / 4, t = lane & 3;
  // The queries' parts are behind the warps' rings.
  char *const rings = shared + warp * (S::kStages * S::kStage);
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(rings);
  uint4 *const queries = reinterpret_cast<uint4 *>(shared + S::kRings);
  after_earlier_kernels();
  if (warp == kWarps) return copy_rest(a);
  __shared__ Course course;
  course.start(d);
  while (course.next(d)) {
    const Segment &seg = course.segment;
    if (seg.lo >= seg.to) continue;
    const float *const w = a.weights + seg.b * a.wb + seg.kv_head * a.wh;
    float *const out = a.out + seg.b * a.ob + seg.kv_head * a.oh;
    for (int head0 = 0; head0 < d.group; head0 += kHeads) {
      const int heads = min(kHeads, d.group - head0), groups = (heads + 7) / 8;
      const int64_t q0 = seg.b * d.qb + (seg.head + head0) * d.qh;
      const bool first = head0 == 0;
      if (!first) sync_weighing();  // (what the queries before these have left in `out` is read)

      // Rows are copied to the warp's ring, tiles ahead of the products.  Pages are looked up a tile before they are used, and
      // checked only then.
      const int lo = seg.lo, to = seg.to, kv_head = seg.kv_head;
      const int32_t *const table = d.table + seg.b * d.table_stride;
      const char *const keys = static_cast<const char *>(c.k) + kv_head * c.head_stride * (int)sizeof(C);
      const float *const from = first ? w : out;
      int page, in;  // of this lane's row (of 16) of the tile to be copied next
      const auto look = [&](int n0) {
        const int n = n0 + (lane & 15), p = (int)d.page((uint32_t)n);
        in = n >= lo && n < to ? n - p * c.page_size : -1;
        page = in >= 0 ? table[p] : 0;
      };
      const auto copy = [&](int n0, int stage) {
        const uint32_t at = ring + stage * S::kStage;
        bool there = in >= 0;
        if (lane < 16) copy_async<4>(at + 16 * S::ROW + lane * 4, there ? from + n0 + lane : from, there);
        if (there && (unsigned)page >= (uint64_t)c.pages) {
          if (c.status) atomicOr(c.status, GAR_KV_BAD_PAGE);
          there = false;
        }
        if (Q8 && lane < 16) {
          const int64_t scale_at = there ? page * c.scale_page_stride + kv_head * c.scale_head_stride + in * c.scale_token_stride : 0;
          copy_async<4>(at + 16 * S::ROW + 64 + lane * 4, c.k_scale + scale_at, there);
        }
        const int64_t row_at = there ? (page * c.page_stride + in * c.token_stride) * (int)sizeof(C) : -1;
        look(n0 + STEP);
#pragma unroll
        for (int i = 0; i < 16 * S::CHUNKS / 32; ++i) {
          const int x = i * 32 + lane, row = x / S::CHUNKS, chunk = x - row * S::CHUNKS;
          const int64_t y = __shfl_sync(~0u, row_at, row);
          const bool has = y >= 0 && chunk * S::CH < c.dim;
          copy_async<16>(at + row * S::ROW + S::place(row, chunk) * 16, has ? keys + y + chunk * 16 : keys, has);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
      };
      int n0 = seg.from + 16 * warp, ahead = n0, in_stage = 0, out_stage = 0;
      look(n0);
      const auto pump = [&] {
        if (ahead < to)
          copy(ahead, in_stage);
        else
          asm volatile("cp.async.commit_group;" ::: "memory");
        ahead += STEP;
        if (++in_stage == S::kStages) in_stage = 0;
      };
#pragma unroll 1
      for (int i = 0; i < S::kStages - 1; ++i) pump();
      sync_weighing();
      for (int h = warp; h < 8 * groups; h += kWarps) {
        float up = 1.f, shrink = 1.f;
        if (Q8 && d.q_dtype != GAR_F16 && h < heads) {
          uint32_t most = 0;
          for (int i = lane; i < c.dim; i += 32) most = max(most, __float_as_uint(fabsf(load_q(d, q0 + h * d.qh + i))));
          most = __reduce_max_sync(~0u, most);
          const int e = min(max((int)(most >> 23), 15), 254);
          up = __int_as_float((e - 14) << 23), shrink = __int_as_float((268 - e) << 23);
        }
        if (lane == 0) {
          factor[h] = h < heads ? factor_of(a, seg.b, h, seg.head + head0 + h, up) : make_float2(0.f, INFINITY);
          down[h] = shrink;
        }
      }
      sync_weighing();
      for (int i = threadIdx.x; i < groups * KC * S::W4 * 32; i += kThreads) {
        const int l = i & 31, rest = i / 32, x = rest % S::W4, k = rest / S::W4 % KC, ng = rest / S::W4 / KC;
        const int h = 8 * ng + l / 4, channel = ((l & 3) + 4 * k) * S::CH + 8 * x;
        uint32_t word[S::PARTS][4] = {};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float v[2] = {0.f, 0.f};
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (h < heads && channel + 2 * j + e < c.dim) v[e] = load_q(d, q0 + h * d.qh + channel + 2 * j + e) * (Q8 ? down[h] : 1.f);
          if constexpr (Q32)
            split<__half>(v[0], v[1], &word[0][j], &word[1][j]);
          else
            word[0][j] = pack2(make_float2(v[0], v[1]), T());
        }
#pragma unroll
        for (int p = 0; p < S::PARTS; ++p)
          queries[ng * S::kGroup + ((p * KC + k) * S::W4 + x) * 32 + l] = make_uint4(word[p][0], word[p][1], word[p][2], word[p][3]);
      }
      sync_weighing();
      for (; n0 < to; n0 += STEP) {
        pump();
        asm volatile("cp.async.wait_group %0;" ::"n"(S::kStages - 1) : "memory");
        __syncwarp();
        const char *const tile = rings + out_stage * S::kStage;
        if (++out_stage == S::kStages) out_stage = 0;
        uint4 now[2][KC];
        float scale[2], sum[2], p[2] = {0.f, 0.f};
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int row = g + 8 * r;
#pragma unroll
          for (int k = 0; k < KC; ++k) now[r][k] = *reinterpret_cast<const uint4 *>(tile + row * S::ROW + S::place(row, t + 4 * k) * 16);
          sum[r] = reinterpret_cast<const float *>(tile + 16 * S::ROW)[row];
          scale[r] = Q8 ? reinterpret_cast<const float *>(tile + 16 * S::ROW)[16 + row] : 1.f;
        }
        __syncwarp();  // (the stage may be copied to again)
        for (int ng = 0; ng < groups; ++ng) {
          float s[2][4] = {};
          const uint4 *const q = queries + ng * S::kGroup + lane;
#pragma unroll
          for (int k = 0; k < KC; ++k) {
            const uint32_t xs[4] = {now[0][k].x, now[0][k].y, now[0][k].z, now[0][k].w};
            const uint32_t ys[4] = {now[1][k].x, now[1][k].y, now[1][k].z, now[1][k].w};
            if constexpr (!Q8) {
              const uint4 b = q[k * 32];
              mma<T>(s[0], xs[0], ys[0], xs[1], ys[1], b.x, b.y);
              mma<T>(s[1], xs[2], ys[2], xs[3], ys[3], b.z, b.w);
            } else {
#pragma unroll
              for (int part = S::PARTS - 1; part >= 0; --part) {
                const uint4 b0 = q[(part * KC + k) * 64], b1 = q[(part * KC + k) * 64 + 32];
                const uint32_t bs[8] = {b0.x, b0.y, b0.z, b0.w, b1.x, b1.y, b1.z, b1.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  uint32_t a0, a1, a2, a3;
                  expand<C>(xs[i], &a0, &a2);
                  expand<C>(ys[i], &a1, &a3);
                  mma<T>(s[i % 2], a0, a1, a2, a3, bs[2 * i], bs[2 * i + 1]);
                }
              }
            }
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float2 f = factor[8 * ng + 2 * t + h];
            p[0] += weight_of((s[0][h] + s[1][h]) * scale[0], f);
            p[1] += weight_of((s[0][2 + h] + s[1][2 + h]) * scale[1], f);
          }
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          p[r] += __shfl_xor_sync(~0u, p[r], 1);
          p[r] += __shfl_xor_sync(~0u, p[r], 2);
          const int n = n0 + g + 8 * r;
          if (t == r && n >= lo && n < to) out[n] = sum[r] + p[r];
        }
      }
    }
  }
}

// Any types, strides and alignment; 32-bit keys.  A warp takes a row, a lane every 32nd of the groups of V channels.
template <typename C, int V> __global__ void __launch_bounds__(kThreads + 32) weigh_plain(const WeighArgs a) {
  extern __shared__ float query[];  // [heads][dim]
  __shared__ float2 factor[kHeads];
  const ServingArgs &d = a.d;
  const gar_kv_cache &c = d.c;
  constexpr bool Q8 = quantised<C>::value;
  constexpr int MOST = GAR_MAX_HEAD_DIM / 32 / V;  // groups of channels of a lane
  constexpr int ROWS = 4;                          // at a time
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  after_earlier_kernels();
  if (warp == kWarps) return copy_rest(a);
  __shared__ Course course;
  course.start(d);
  while (course.next(d)) {
    const Segment &seg = course.segment;
    if (seg.lo >= seg.to) continue;
    const float *const w = a.weights + seg.b * a.wb + seg.kv_head * a.wh;
    float *const out = a.out + seg.b * a.ob + seg.kv_head * a.oh;
    for (int head0 = 0; head0 < d.group; head0 += kHeads) {
      const int heads = min(kHeads, d.group - head0);
      const int64_t q0 = seg.b * d.qb + (seg.head + head0) * d.qh;
      sync_weighing();
      for (int i = threadIdx.x; i < heads * c.dim; i += kThreads) {
        const int h = i / c.dim;
        query[i] = load_q(d, q0 + h * d.qh + (i - h * c.dim));
      }
      for (int h = threadIdx.x; h < heads; h += kThreads) factor[h] = factor_of(a, seg.b, h, seg.head + head0 + h, 1.f);
      sync_weighing();
      const float *const base = head0 == 0 ? w : out;
      for (int n0 = seg.lo + ROWS * warp; n0 < seg.to; n0 += ROWS * kWarps) {
        float key[ROWS][MOST][V], scale[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
          int64_t scale_at;
          const int64_t at = key_at(d, seg, n0 + r, &scale_at);
          const C *const k = static_cast<const C *>(c.k) + at;
          scale[r] = at >= 0 ? (Q8 ? c.k_scale[scale_at] : 1.f) : 0.f;
#pragma unroll
          for (int m = 0; m < MOST; ++m) {
            const int channel = (lane + 32 * m) * V;
            const bool there = at >= 0 && channel < c.dim;
            if constexpr (V == 4) {
              const float4 x = there ? *reinterpret_cast<const float4 *>(k + channel) : make_float4(0.f, 0.f, 0.f, 0.f);
              key[r][m][0] = x.x, key[r][m][1] = x.y, key[r][m][2] = x.z, key[r][m][3] = x.w;
            } else {
              key[r][m][0] = there ? to_f32(k[channel]) : 0.f;
            }
          }
        }
        float sum[ROWS] = {};
        for (int h = 0; h < heads; ++h) {
          const float *const q = query + h * c.dim;
          float s[ROWS] = {};
#pragma unroll
          for (int m = 0; m < MOST; ++m)
#pragma unroll
            for (int v = 0; v < V; ++v) {
              const int channel = (lane + 32 * m) * V + v;
              const float x = channel < c.dim ? q[channel] : 0.f;
#pragma unroll
              for (int r = 0; r < ROWS; ++r) s[r] = channel < c.dim ? fmaf(x, key[r][m][v], s[r]) : s[r];
            }
#pragma unroll
          for (int r = 0; r < ROWS; ++r) {
#pragma unroll
            for (int k = 16; k > 0; k /= 2) s[r] += __shfl_xor_sync(~0u, s[r], k);
            sum[r] += weight_of(Q8 ? s[r] * scale[r] : s[r], factor[h]);
          }
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
          if (lane == r && n0 + r < seg.to) out[n0 + r] = base[n0 + r] + sum[r];
      }
    }
  }
}

template <typename C, int KC, bool Q32> int launch_mma_weigh(const WeighArgs &a, int sms, gar_stream_t stream) {
  using S = WeighShape<C, KC, Q32>;
  constexpr auto kernel = weigh_mma<C, KC, Q32>;
  const size_t shared = S::kRings + (size_t)((std::min(a.d.group, kHeads) + 7) / 8) * S::kGroup * 16;
  static DeviceSet allowed;
  const int e = once_for_device(allowed, a.d.device, [&] {
    return (int)cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kRings + kHeads / 8 * S::kGroup * 16);
  });
  if (e != 0) return cuda_fail((cudaError_t)e, "cudaFuncSetAttribute");
  return launch("gar_kv_weigh", kernel, sms * S::kResident, kThreads + 32, shared, stream, a);
}

template <typename C, bool Q32> int weigh(const WeighArgs &a, int sms, gar_stream_t stream) {
  const int chunks = (int)((a.d.c.dim * sizeof(C) + 63) / 64);
  if (chunks <= 1) return launch_mma_weigh<C, 1, Q32>(a, sms, stream);
  if (chunks <= 2) return launch_mma_weigh<C, 2, Q32>(a, sms, stream);
  if (chunks <= 3) return launch_mma_weigh<C, 3, Q32>(a, sms, stream);
  if constexpr (sizeof(C) == 2) {
    if (chunks <= 4) return launch_mma_weigh<C, 4, Q32>(a, sms, stream);
    if (chunks <= 6) return launch_mma_weigh<C, 6, Q32>(a, sms, stream);
    return launch_mma_weigh<C, 8, Q32>(a, sms, stream);
  } else {
    return launch_mma_weigh<C, 4, Q32>(a, sms, stream);
  }
}

template <typename C, int V> int weigh_any(const WeighArgs &a, int sms, gar_stream_t stream) {
  constexpr auto kernel = weigh_plain<C, V>;
  static DeviceSet allowed;
  const int e = once_for_device(allowed, a.d.device, [&] {
    return (int)cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kHeads * GAR_MAX_HEAD_DIM * 4);
  });
  if (e != 0) return cuda_fail((cudaError_t)e, "cudaFuncSetAttribute");
  return launch("gar_kv_weigh", kernel, sms * 2, kThreads + 32, (size_t)std::min(a.d.group, kHeads) * a.d.c.dim * 4, stream, a);
}

// Keys can be loaded 16 bytes at a time.
bool wide_keys(const gar_kv_cache &c) {
  const int64_t n = 16 / element_size(c.dtype);
  return (uintptr_t)c.k % 16 == 0 && c.dim % n == 0 && c.page_stride % n == 0 && c.head_stride % n == 0 && c.token_stride % n == 0;
}

}  // namespace
}  // namespace gar

using namespace gar;

extern "C" int gar_kv_weigh(const gar_kv_cache *cache, const void *q, int64_t q_batch_stride, int64_t q_head_stride, int q_dtype,
                            int q_heads, const float *lse, const float *weights, int64_t weights_batch_stride,
                            int64_t weights_head_stride, float *out, int64_t out_batch_stride, int64_t out_head_stride,
                            int64_t rows, const int32_t *page_table, int64_t table_stride, int table_width,
                            const int32_t *lengths, int batch, float scale, int window, gar_stream_t stream) {
  if (int rc = check_cache(cache)) return rc;
  if (!float_type(q_dtype)) return refuse("q is GAR_F32, GAR_BF16 or GAR_F16");
  if (float_type(cache->dtype) && cache->dtype != q_dtype) return refuse("a cache of float type goes with queries of its type");
  if (q_heads < 1 || q_heads % cache->heads) return refuse("q_heads must be a multiple of the cache's heads");
  if (batch < 0 || table_width < 0 || window < 0 || rows < 0) return refuse("negative batch, table_width, window or rows");
  if (!std::isfinite(scale)) return refuse("scale must be finite");
  if (batch == 0 || rows == 0) return GAR_OK;
  if (q == nullptr || lse == nullptr || weights == nullptr || out == nullptr || lengths == nullptr ||
      (page_table == nullptr && table_width > 0))
    return refuse("null pointer");
  if ((uintptr_t)q % element_size(q_dtype) || (uintptr_t)lse % 4 || (uintptr_t)weights % 4 || (uintptr_t)out % 4 ||
      (uintptr_t)page_table % 4 || (uintptr_t)lengths % 4) {
    set_error("a buffer is not aligned to its elements");
    return GAR_EALIGN;
  }
  if (weights == out && (weights_batch_stride != out_batch_stride || weights_head_stride != out_head_stride))
    return refuse("out is weights, with other strides");
  const int most_rows = (int)std::min<int64_t>(std::min<int64_t>(rows, (int64_t)table_width * cache->page_size), 0x7fffffff - 65536);
  const int unit = (int64_t)batch * cache->heads > INT_MAX / 2 ? 0 : unit_of((int64_t)batch * cache->heads, most_rows);
  if (unit == 0) return refuse("too many sequences and heads for tables this wide");
  int dev = -1, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return cuda_fail(e, "gar_kv_weigh");
  WeighArgs a{};
  ServingArgs &d = a.d;
  d.c = *cache, d.q = q, d.qb = q_batch_stride, d.qh = q_head_stride, d.q_dtype = q_dtype;
  d.table = page_table, d.table_stride = table_stride, d.lengths = lengths;
  d.page = divide_by((uint32_t)cache->page_size), d.items = divide_by((uint32_t)cache->heads);
  d.most_rows = most_rows, d.batch = batch, d.q_heads = q_heads, d.window = window, d.unit = unit, d.device = dev;
  d.group = d.item_heads = q_heads / cache->heads, d.item_groups = 1, d.line = true;
  // What a segment costs beside its rows: the units of 64 rows that 32 KB of keys are.  (That, a quarter and four times as much: 24 x 8192, 32/8 x 128 bf16 49, 51 and 49 us; i8 41, 44 and 42; f32
  // 239, 239 and 250; 128 x 500, 32/8 x 64 bf16 20, 28 and 20; 16 x 8192, 16/4 x 256 f16 35, 35 and 31.)
  d.slack = std::max(1, 32768 / (64 * cache->dim * element_size(cache->dtype)));
  d.scale_log2 = (float)((double)scale * 1.4426950408889634);
  a.lse = lse, a.weights = weights, a.out = out, a.rows = rows, a.apart = out != weights;
  a.wb = weights_batch_stride, a.wh = weights_head_stride, a.ob = out_batch_stride, a.oh = out_head_stride;
  const bool wide = wide_keys(*cache), q32 = q_dtype == GAR_F32;
  switch (cache->dtype) {
    case GAR_F32: return wide ? weigh_any<float, 4>(a, sms, stream) : weigh_any<float, 1>(a, sms, stream);
    case GAR_BF16: return wide ? weigh<__nv_bfloat16, false>(a, sms, stream) : weigh_any<__nv_bfloat16, 1>(a, sms, stream);
    case GAR_F16: return wide ? weigh<__half, false>(a, sms, stream) : weigh_any<__half, 1>(a, sms, stream);
    case GAR_I8:
      return !wide ? weigh_any<i8, 1>(a, sms, stream) : q32 ? weigh<i8, true>(a, sms, stream) : weigh<i8, false>(a, sms, stream);
    default:
      return !wide ? weigh_any<e4m3, 1>(a, sms, stream) : q32 ? weigh<e4m3, true>(a, sms, stream) : weigh<e4m3, false>(a, sms, stream);
  }
}
