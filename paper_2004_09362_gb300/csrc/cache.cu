// The paged key-value cache: rows quantised (keys rotated too) as they are written, and read back.
#include <algorithm>

#include "gar_device.cuh"

namespace gar {
namespace {

constexpr int kThreads = 256;
// Rows of a lane where there are many (read as below, i8/e4m3/bf16: two 41/36.5/42, four 43/34/42, eight 58/39/48 us).
constexpr int kReadRows = 4;

struct CacheArgs {
  gar_kv_cache cache;
  const void *in[2];
  void *out[2];
  int64_t ts[2], hs[2];        // strides of in[]
  const int64_t *slots;
  const void *positions;
  const float2 *table;
  int64_t table_rows;
  int rows;                    // tokens * heads; writing: tokens * runs
  int run, runs;               // writing: heads that the same lanes take, and such runs of a token
  int rot, interleaved, wide_positions;
  int lanes;                   // power of two: lanes that hold one row
  Divide heads, page;
};

// The place of a slot's row, or false where there is none.
struct Place {
  int64_t at, scale;
};
__device__ __forceinline__ bool find(const CacheArgs &a, int64_t slot, int head, Place *p) {
  const gar_kv_cache &c = a.cache;
  if (slot < 0) return false;
  const int64_t page = slot < 0x7fffffff ? a.page((uint32_t)slot) : slot / c.page_size;
  if (page >= c.pages) {
    if (c.status) atomicOr(c.status, GAR_KV_BAD_SLOT);
    return false;
  }
  const int row = (int)(slot - page * c.page_size);
  p->at = page * c.page_stride + head * c.head_stride + row * c.token_stride;
  p->scale = page * c.scale_page_stride + head * c.scale_head_stride + row * c.scale_token_stride;
  return true;
}

// N elements as they lie in memory, and their values.
template <typename T, int N> struct alignas(sizeof(T) * N < 16 ? sizeof(T) * N : 16) raw_chunk {
  uint32_t w[N * sizeof(T) / 4];
};
template <typename T, int N> __device__ __forceinline__ void values(const raw_chunk<T, N> &r, float2 (&v)[N / 2]) {
#pragma unroll
  for (int k = 0; k < N; k += 4) {
    if constexpr (sizeof(T) == 4) {
      v[k / 2] = make_float2(__uint_as_float(r.w[k]), __uint_as_float(r.w[k + 1]));
      v[k / 2 + 1] = make_float2(__uint_as_float(r.w[k + 2]), __uint_as_float(r.w[k + 3]));
    } else if constexpr (sizeof(T) == 2) {
      v[k / 2] = unpack2(r.w[k / 2], T()), v[k / 2 + 1] = unpack2(r.w[k / 2 + 1], T());
    } else {
      unpack4(r.w[k / 4], &v[k / 2], &v[k / 2 + 1], T());
    }
  }
}

// Channels [from, from + N) of a row, zeros past its end.  WIDE: all are there and aligned.
template <bool WIDE, typename T, int N> __device__ __forceinline__ void load(const T *p, int from, int dim, float2 (&v)[N / 2]) {
  if (WIDE) {
    values(*reinterpret_cast<const raw_chunk<T, N> *>(p + from), v);
  } else {
#pragma unroll
    for (int k = 0; k < N; k += 2)
      v[k / 2] = make_float2(from + k < dim ? to_f32(p[from + k]) : 0.f, from + k + 1 < dim ? to_f32(p[from + k + 1]) : 0.f);
  }
}

template <bool WIDE, typename T, int N>
__device__ __forceinline__ void store(T *p, int from, int dim, const float2 (&v)[N / 2]) {
  if constexpr (WIDE) {
    raw_chunk<T, N> r;
#pragma unroll
    for (int k = 0; k < N; k += 2) {
      if constexpr (sizeof(T) == 4)
        r.w[k] = __float_as_uint(v[k / 2].x), r.w[k + 1] = __float_as_uint(v[k / 2].y);
      else
        r.w[k / 2] = pack2(v[k / 2], T());
    }
    *reinterpret_cast<raw_chunk<T, N> *>(p + from) = r;
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (from + k < dim) p[from + k] = from_f32<T>(k % 2 ? v[k / 2].y : v[k / 2].x);
  }
}

template <bool WIDE, typename T, int N>
__device__ __forceinline__ void store_codes(T *p, int from, int dim, const raw_chunk<T, N> &r) {
  if (WIDE) {
    *reinterpret_cast<raw_chunk<T, N> *>(p + from) = r;
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (from + k < dim) reinterpret_cast<uint8_t *>(p)[from + k] = (uint8_t)(r.w[k / 4] >> 8 * (k % 4));
  }
}

// How keys are rotated: not at all; by the half layout, a lane's channels half of them from each side; by the
// interleaved layout; any way, channel by channel.
enum { TURN_NONE, TURN_HALF, TURN_PAIRS, TURN_ANY };

// A token's row of the table, null where the position is outside (and stands for NaN).
__device__ __forceinline__ const float2 *find_turn(const CacheArgs &a, int64_t token) {
  const int64_t pos = a.wide_positions ? static_cast<const int64_t *>(a.positions)[token]
                                       : (int64_t) static_cast<const int32_t *>(a.positions)[token];
  if ((uint64_t)pos < (uint64_t)a.table_rows) return a.table + pos * (a.rot / 2);
  if (a.cache.status) atomicOr(a.cache.status, GAR_KV_BAD_POSITION);
  return nullptr;
}

// A lane's channels rotated, by the entries c and s of their pairs.
template <int TURN, typename T, int N, int E>
__device__ __forceinline__ void rotate(const CacheArgs &a, const float2 *t, const float (&c)[E], const float (&s)[E],
                                       const T *row, int from, float2 (&v)[N / 2]) {
  if constexpr (TURN == TURN_PAIRS) {
#pragma unroll
    for (int k = 0; k < N / 2; ++k) {
      const float2 x = v[k];
      v[k].x = __fsub_rn(__fmul_rn(x.x, c[k]), __fmul_rn(x.y, s[k]));
      v[k].y = __fadd_rn(__fmul_rn(x.y, c[k]), __fmul_rn(x.x, s[k]));
    }
  } else if constexpr (TURN == TURN_HALF) {
#pragma unroll
    for (int k = 0; k < N / 4; ++k) {  // (one by one: paired, the compiler would fuse product and sum)
      const float2 x = v[k], y = v[k + N / 4];
      v[k].x = __fsub_rn(__fmul_rn(x.x, c[2 * k]), __fmul_rn(y.x, s[2 * k]));
      v[k].y = __fsub_rn(__fmul_rn(x.y, c[2 * k + 1]), __fmul_rn(y.y, s[2 * k + 1]));
      v[k + N / 4].x = __fadd_rn(__fmul_rn(y.x, c[2 * k]), __fmul_rn(x.x, s[2 * k]));
      v[k + N / 4].y = __fadd_rn(__fmul_rn(y.y, c[2 * k + 1]), __fmul_rn(x.y, s[2 * k + 1]));
    }
  } else {
    const int half = a.rot / 2;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int at = from + k;
      if (at >= a.rot) break;
      const int pair = a.interleaved ? at / 2 : at < half ? at : at - half;
      const bool second = a.interleaved ? at & 1 : at >= half;
      const int other = a.interleaved ? at ^ 1 : second ? at - half : at + half;
      const float2 cs = t ? t[pair] : make_float2(__int_as_float(0x7fc00000), 0.f);
      float &x = k % 2 ? v[k / 2].y : v[k / 2].x;
      const float p = __fmul_rn(x, cs.x), q = __fmul_rn(to_f32(row[other]), cs.y);
      x = second ? __fadd_rn(p, q) : __fsub_rn(p, q);
    }
  }
}

// The largest magnitude of N values as the bits of a float: magnitudes compare as integers, infinities
// and NaNs the largest.
template <int N> __device__ __forceinline__ uint32_t largest(const float2 (&v)[N]) {
  uint32_t most = 0;
#pragma unroll
  for (int k = 0; k < N; ++k)
    most = max(most, max(__float_as_uint(v[k].x) & 0x7fffffffu, __float_as_uint(v[k].y) & 0x7fffffffu));
  return most;
}
// The same of 16-bit floats as they lie in memory, two a word.
template <typename T, int N> __device__ __forceinline__ uint32_t largest(const raw_chunk<T, N> &r) {
  static_assert(sizeof(T) == 2, "16-bit floats");
  uint32_t m = r.w[0] & 0x7fff7fffu;
#pragma unroll
  for (int k = 1; k < N / 2; ++k) m = __vmaxu2(m, r.w[k] & 0x7fff7fffu);
  const float2 x = unpack2(m, T());
  return max(__float_as_uint(x.x), __float_as_uint(x.y));
}

// 1 / s rounded to nearest, for normal s whose reciprocal is normal.  One Newton step from a reciprocal that is off by at
// most one unit rounds correctly but for significands of all ones (Markstein, the same paper), whose
// reciprocal is one unit over a power of two.  (The rounded reciprocal as a call would cost the kernel its registers.)
__device__ __forceinline__ float reciprocal(float s) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
  r = __fmaf_rn(__fmaf_rn(-s, r, 1.f), r, r);
  const uint32_t b = __float_as_uint(s);
  return (b & 0x7fffffu) == 0x7fffffu ? __uint_as_float((253u << 23) - (b & 0x7f800000u) + 1) : r;
}

// Codes of the row of which this lane holds v, `most` the largest of them, and the row's scale.
//
// v / scale is rounded as the definition has it, without a division each: for r = 1 / scale rounded to
// nearest and q = v r, the remainder v - q scale is exact in a fused multiply-add, and
// q + r (v - q scale) is the correctly rounded quotient (P. Markstein, IBM J. Res. Dev. 34, 1990),
// as long as nothing underflows; rows of scales under 2^-90 are multiplied by 2^100 first.  Codes of a row with
// an infinity or a NaN mean nothing: its scale is a NaN.
template <typename C, int N>
__device__ __forceinline__ raw_chunk<C, N> quantise(float2 (&v)[N / 2], uint32_t most, int lanes, float *scale) {
  for (int d = lanes / 2; d > 0; d /= 2) most = max(most, __shfl_xor_sync(~0u, most, d));
  float s = __fmul_rn(__uint_as_float(most), 1.f / quantised<C>::largest);
  *scale = most >= 0x7f800000u ? __int_as_float(0x7fc00000) : s;
  const bool tiny = s < 0x1p-90f;
  if (tiny) {
    s *= 0x1p100f;
#pragma unroll
    for (int k = 0; k < N / 2; ++k) v[k] = mul2(v[k], make_float2(0x1p100f, 0x1p100f));
  }
  const float r = s > 0.f ? reciprocal(s) : 0.f;
  const float2 r2 = make_float2(r, r), minus = make_float2(-s, -s);
#pragma unroll
  for (int k = 0; k < N / 2; ++k) {
    const float2 q = mul2(v[k], r2);
    v[k] = fma2(fma2(q, minus, v[k]), r2, q);
  }
  if (tiny) {  // a subnormal scale may be rounded far down
    constexpr float top = quantised<C>::largest;
#pragma unroll
    for (int k = 0; k < N / 2; ++k)
      v[k] = make_float2(fminf(fmaxf(v[k].x, -top), top), fminf(fmaxf(v[k].y, -top), top));
  }
  raw_chunk<C, N> out;
#pragma unroll
  for (int k = 0; k < N; k += 4) out.w[k / 4] = codes4(v[k / 2].x, v[k / 2].y, v[k / 2 + 1].x, v[k / 2 + 1].y, C());
  return out;
}

// T -> C rows.  a.lanes neighbouring lanes hold a token's row of one head, N channels of the key
// and of the value each, so that the largest magnitudes are found by shuffles and the rows are
// read once.  With RUN they take a.run heads of the token one after the other, the next one's loads in flight while
// one is worked on: the slot is looked up and the table's entries are read (512 bytes for rows of 256) once for
// all of them.  Bound by memory, not far from the rate of issue; the registers are held down to
// keep 32 warps an SM: with 4, 3, 2 CTAs an SM rotated rows as below took 46, 52, 67 us.
//
// 32768 tokens x 8 heads x 128 channels from bf16: to codes 39.7 us (5.1 TB/s), keys rotated 47; to bf16 42 (6.4 TB/s),
// rotated 49.  24 tokens, e4m3, rotated: 2.5 us, the launch and three round trips to memory.
template <typename T, typename C, int N, bool RUN, bool WIDE, int TURN>
__global__ void __launch_bounds__(kThreads, RUN ? 4 : 1) write_kernel(const CacheArgs a) {
  static_assert(N == 8, "two words of codes, a half of a chunk each");
  after_earlier_kernels();
  const gar_kv_cache &c = a.cache;
  const int lane = threadIdx.x & (a.lanes - 1), from = lane * N;
  const int i = blockIdx.x * (kThreads / a.lanes) + threadIdx.x / a.lanes;
  const bool any = i < a.rows;
  const int64_t token = any ? a.heads(i) : 0;
  const int first = any ? (i - (int)token * a.runs) * a.run : 0, end = any ? min(first + a.run, c.heads) : 0;
  const int64_t slot = any ? a.slots[token] : -1;
  const T *const k_rows = static_cast<const T *>(a.in[0]) + token * a.ts[0];
  const T *const v_rows = static_cast<const T *>(a.in[1]) + token * a.ts[1];
  const bool in = any && from < c.dim, turned = TURN != TURN_NONE && in && from < a.rot;
  // The lane's channels: [from, from + N), but with TURN_HALF N / 2 each from two places.
  const int lower = TURN == TURN_HALF && from < a.rot ? from / 2 : from;
  const int upper = TURN == TURN_HALF && from < a.rot ? from / 2 + a.rot / 2 : from + N / 2;
  constexpr int E = TURN == TURN_HALF || TURN == TURN_PAIRS ? N / 2 : 1;
  float cosine[E], sine[E];
  const float2 *turn = nullptr;
  Place p{};
  struct Raw {
    raw_chunk<T, N> k, v;
  } now{}, next{};
  using Side = raw_chunk<T, N / 2>;
  using Codes = raw_chunk<C, N / 2>;
  const auto fetch = [&](Raw &r, int h) {
    if (WIDE && in && h < end) {
      const T *const k = k_rows + h * a.hs[0], *const v = v_rows + h * a.hs[1];
      if (TURN == TURN_HALF) {
        *reinterpret_cast<Side *>(r.k.w) = *reinterpret_cast<const Side *>(k + lower);
        *reinterpret_cast<Side *>(r.k.w + sizeof(Side) / 4) = *reinterpret_cast<const Side *>(k + upper);
      } else {
        r.k = *reinterpret_cast<const raw_chunk<T, N> *>(k + from);
      }
      r.v = *reinterpret_cast<const raw_chunk<T, N> *>(v + from);
    }
  };
  fetch(now, first);
  const bool there = find(a, slot, first, &p);
  if (turned && there) {
    turn = find_turn(a, token);
    if constexpr (TURN == TURN_HALF || TURN == TURN_PAIRS)
      load_rotation<E, true>(turn ? turn + from / 2 : nullptr, turn != nullptr, cosine, sine);
  }
  // All lanes of a warp go round as often: the shuffles are the warp's.
  for (int j = 0; j < (RUN ? a.run : 1); ++j) {
    const int h = first + j;
    if (RUN && h + 1 < first + a.run) fetch(next, h + 1);
    const bool mine = in && there && h < end;
    // (Lanes and heads with nothing to do go along with zeros or with what they had.)
    float2 k[N / 2], v[N / 2];
    if (WIDE) {
      values(now.k, k);
      values(now.v, v);
    } else {
      load<WIDE, T, N>(k_rows + h * a.hs[0], from, in && h < end ? c.dim : 0, k);
      load<WIDE, T, N>(v_rows + h * a.hs[1], from, in && h < end ? c.dim : 0, v);
    }
    if (TURN != TURN_NONE && turned && there && h < end)
      rotate<TURN, T, N, E>(a, turn, cosine, sine, k_rows + h * a.hs[0], from, k);
    if constexpr (quantised<C>::value) {
      uint32_t k_most, v_most;
      if constexpr (WIDE && sizeof(T) == 2) {
        k_most = TURN == TURN_NONE ? largest(now.k) : largest(k), v_most = largest(now.v);
      } else {
        k_most = largest(k), v_most = largest(v);
      }
      float k_scale, v_scale;
      const raw_chunk<C, N> k_codes = quantise<C, N>(k, k_most, a.lanes, &k_scale);
      const raw_chunk<C, N> v_codes = quantise<C, N>(v, v_most, a.lanes, &v_scale);
      if (mine && lane == 0) c.k_scale[p.scale] = k_scale, c.v_scale[p.scale] = v_scale;
      if (mine) {
        C *const row = static_cast<C *>(c.k) + p.at;
        if constexpr (TURN == TURN_HALF) {
          *reinterpret_cast<Codes *>(row + lower) = *reinterpret_cast<const Codes *>(k_codes.w);
          *reinterpret_cast<Codes *>(row + upper) = *reinterpret_cast<const Codes *>(k_codes.w + sizeof(Codes) / 4);
        } else {
          store_codes<WIDE>(row, from, c.dim, k_codes);
        }
        store_codes<WIDE>(static_cast<C *>(c.v) + p.at, from, c.dim, v_codes);
      }
      p.scale += c.scale_head_stride;
    } else if (mine) {
      C *const row = static_cast<C *>(c.k) + p.at;
      if constexpr (TURN == TURN_HALF) {
        const float2 x[N / 4] = {k[0], k[1]}, y[N / 4] = {k[2], k[3]};
        store<WIDE, C, N / 2>(row, lower, c.dim, x);
        store<WIDE, C, N / 2>(row, upper, c.dim, y);
      } else {
        store<WIDE, C, N>(row, from, c.dim, k);
      }
      store<WIDE, C, N>(static_cast<C *>(c.v) + p.at, from, c.dim, v);
    }
    p.at += c.head_stride;
    if (RUN) now = next;
  }
}

// C -> T rows, M of them to a lane: a row's place hangs on its slot, so that fewer bytes would be in flight.  Bound by
// memory: 32768 tokens x 8 heads x 128 channels to bf16 from e4m3 34 us (5.9 TB/s), from i8 43 (4.7), from bf16 42 (6.4).
template <typename T, typename C, int N, bool WIDE, int M>
__global__ void __launch_bounds__(kThreads) read_kernel(const CacheArgs a) {
  after_earlier_kernels();
  const gar_kv_cache &c = a.cache;
  const int lane = threadIdx.x & (a.lanes - 1), from = lane * N, step = kThreads / a.lanes;
  const int i0 = blockIdx.x * (step * M) + threadIdx.x / a.lanes;
  if (from >= c.dim) return;
  Place p[M];
  bool there[M];
#pragma unroll
  for (int m = 0; m < M; ++m) {
    const int i = i0 + m * step;
    const int token = i < a.rows ? a.heads(i) : 0;
    there[m] = i < a.rows && find(a, a.slots[token], i - token * c.heads, &p[m]);
  }
  raw_chunk<C, N> k[M], v[M];
  float k_scale[M], v_scale[M];
#pragma unroll
  for (int m = 0; m < M; ++m) {
    k_scale[m] = v_scale[m] = 0.f;
    if (there[m]) {
      if (WIDE) {
        k[m] = *reinterpret_cast<const raw_chunk<C, N> *>(static_cast<const C *>(c.k) + p[m].at + from);
        v[m] = *reinterpret_cast<const raw_chunk<C, N> *>(static_cast<const C *>(c.v) + p[m].at + from);
      }
      if (quantised<C>::value) k_scale[m] = c.k_scale[p[m].scale], v_scale[m] = c.v_scale[p[m].scale];
    }
  }
#pragma unroll
  for (int m = 0; m < M; ++m) {
    const int64_t i = i0 + m * step;
    if (i >= a.rows) break;
    float2 x[N / 2] = {}, y[N / 2] = {};
    if (there[m]) {
      if (WIDE) {
        values(k[m], x);
        values(v[m], y);
      } else {
        load<WIDE, C, N>(static_cast<const C *>(c.k) + p[m].at, from, c.dim, x);
        load<WIDE, C, N>(static_cast<const C *>(c.v) + p[m].at, from, c.dim, y);
      }
    }
    if (quantised<C>::value) {
#pragma unroll
      for (int e = 0; e < N / 2; ++e) {
        x[e] = mul2(x[e], make_float2(k_scale[m], k_scale[m]));
        y[e] = mul2(y[e], make_float2(v_scale[m], v_scale[m]));
      }
    }
    store<WIDE, T, N>(static_cast<T *>(a.out[0]) + i * c.dim, from, c.dim, x);
    store<WIDE, T, N>(static_cast<T *>(a.out[1]) + i * c.dim, from, c.dim, y);
  }
}

// Calls f with the tags of a float type and the cache's type.
template <typename F> int with_types(int dtype, int cache, F f) {
  return with_float(dtype, [&](auto t) {
    if (cache == GAR_I8) return f(t, type_tag<i8>{});
    if (cache == GAR_E4M3) return f(t, type_tag<e4m3>{});
    return f(t, t);
  });
}

int check_rows(const gar_kv_cache *cache, int dtype, int64_t tokens) {
  if (int rc = check_cache(cache)) return rc;
  if (!float_type(dtype)) return refuse("rows are GAR_F32, GAR_BF16 or GAR_F16");
  if (float_type(cache->dtype) && cache->dtype != dtype) return refuse("a cache of float type takes its own type");
  if (tokens < 0) return refuse("negative tokens");
  return GAR_OK;
}

// Sets the rows and the lanes of N channels each; false where the rows are too many.
bool shape(CacheArgs *a, int64_t tokens, int n) {
  const int need = (a->cache.dim + n - 1) / n;
  a->lanes = 1;
  while (a->lanes < need) a->lanes *= 2;
  if (tokens > 0x7fffffff / 2 / a->cache.heads) return false;
  a->rows = (int)tokens * a->cache.heads;
  a->heads = divide_by((uint32_t)a->cache.heads);
  a->page = divide_by((uint32_t)a->cache.page_size);
  return true;
}

int blocks(const CacheArgs &a, int rows_per_lane) {
  const int per = kThreads / a.lanes * rows_per_lane;
  return (a.rows + per - 1) / per;
}

// Whether every n channels of the cache (n: 8 or 16) can be accessed as raw_chunk.
bool wide_cache(const gar_kv_cache &c, int n) {
  const uintptr_t a = std::min(16, element_size(c.dtype) * n);
  return (uintptr_t)c.k % a == 0 && (uintptr_t)c.v % a == 0 && c.dim % n == 0 && c.page_stride % n == 0 &&
         c.head_stride % n == 0 && c.token_stride % n == 0;
}

}  // namespace

int check_cache(const gar_kv_cache *c) {
  if (c == nullptr) return refuse("null cache");
  if (!float_type(c->dtype) && c->dtype != GAR_I8 && c->dtype != GAR_E4M3) return refuse("unknown cache dtype");
  if (c->heads < 1 || c->dim < 1 || c->dim > GAR_MAX_HEAD_DIM || c->page_size < 1 || c->pages < 0)
    return refuse("bad heads, dim, page_size or pages of the cache");
  if (c->pages > 0 && (c->k == nullptr || c->v == nullptr)) return refuse("null cache buffers");
  const bool scaled = c->dtype == GAR_I8 || c->dtype == GAR_E4M3;
  if (scaled && c->pages > 0 && (c->k_scale == nullptr || c->v_scale == nullptr)) return refuse("an 8-bit cache needs scales");
  const int size = element_size(c->dtype);
  if ((uintptr_t)c->k % size || (uintptr_t)c->v % size || (uintptr_t)c->k_scale % 4 || (uintptr_t)c->v_scale % 4 ||
      (uintptr_t)c->status % 4) {
    set_error("a cache buffer is not aligned to its elements");
    return GAR_EALIGN;
  }
  return GAR_OK;
}

}  // namespace gar

using namespace gar;

extern "C" {

int gar_kv_write(const gar_kv_cache *cache, const void *k, int64_t k_token_stride, int64_t k_head_stride, const void *v,
                 int64_t v_token_stride, int64_t v_head_stride, int dtype, int64_t tokens, const int64_t *slots,
                 const void *positions, int position_bytes, const float *table, int64_t table_rows, int rot, int layout,
                 gar_stream_t stream) {
  if (int rc = check_rows(cache, dtype, tokens)) return rc;
  if (positions) {
    if (position_bytes != 4 && position_bytes != 8) return refuse("positions are 4 or 8 bytes wide");
    if (rot < 2 || rot % 2 || rot > cache->dim) return refuse("rot must be even, 2..dim");
    if (layout != GAR_ROPE_HALF && layout != GAR_ROPE_INTERLEAVED) return refuse("unknown layout");
    if (table_rows < 0 || (table == nullptr && table_rows > 0)) return refuse("bad table");
  }
  if (tokens == 0) return GAR_OK;
  if (k == nullptr || v == nullptr || slots == nullptr) return refuse("null pointer");
  const int size = element_size(dtype);
  if ((uintptr_t)k % size || (uintptr_t)v % size || (uintptr_t)slots % 8 || (uintptr_t)table % 8 ||
      (positions && (uintptr_t)positions % position_bytes)) {
    set_error("a buffer is not aligned to its elements (the table to 8 bytes)");
    return GAR_EALIGN;
  }
  CacheArgs a{};
  a.cache = *cache;
  a.in[0] = k, a.in[1] = v;
  a.ts[0] = k_token_stride, a.ts[1] = v_token_stride, a.hs[0] = k_head_stride, a.hs[1] = v_head_stride;
  a.slots = slots, a.positions = positions, a.table = reinterpret_cast<const float2 *>(table);
  a.table_rows = table_rows, a.rot = rot, a.interleaved = layout == GAR_ROPE_INTERLEAVED;
  a.wide_positions = position_bytes == 8;
  const int n = 16 / size;
  const bool rows_wide = (uintptr_t)k % 16 == 0 && (uintptr_t)v % 16 == 0 && k_token_stride % n == 0 &&
                         k_head_stride % n == 0 && v_token_stride % n == 0 && v_head_stride % n == 0;
  const int turn = positions ? (a.interleaved ? TURN_PAIRS : TURN_HALF) : TURN_NONE;
  const bool turn_wide = turn == TURN_NONE || ((uintptr_t)table % 16 == 0 && rot % 8 == 0);
  const bool wide = rows_wide && turn_wide && wide_cache(*cache, 8);
  if (!shape(&a, tokens, 8)) return refuse("too many rows");
  // One head at a time until the GPU is full, then up to 8 for the sake of what they share (32768 tokens x 8 heads x 128
  // channels, bf16 to i8: 40 us, rotated 47; one at a time 56 and 73.  To bf16 42 and 49; one at a time 42 and 56).
  a.run = wide && blocks(a, 1) >= 152 * 16 ? std::min(8, cache->heads) : 1;
  a.runs = (cache->heads + a.run - 1) / a.run;
  a.rows = (int)tokens * a.runs;
  a.heads = divide_by((uint32_t)a.runs);
  return with_types(dtype, cache->dtype, [&](auto t, auto c) {
    using T = typename decltype(t)::type;
    using C = typename decltype(c)::type;
    const auto pick = [&](auto kernel) {
      return launch("gar_kv_write", kernel, blocks(a, 1), kThreads, 0, stream, a);
    };
    if (!wide) return pick(positions ? write_kernel<T, C, 8, false, false, TURN_ANY> : write_kernel<T, C, 8, false, false, TURN_NONE>);
    if (a.run == 1)
      return pick(turn == TURN_NONE   ? write_kernel<T, C, 8, false, true, TURN_NONE>
                  : turn == TURN_HALF ? write_kernel<T, C, 8, false, true, TURN_HALF>
                                      : write_kernel<T, C, 8, false, true, TURN_PAIRS>);
    return pick(turn == TURN_NONE   ? write_kernel<T, C, 8, true, true, TURN_NONE>
                : turn == TURN_HALF ? write_kernel<T, C, 8, true, true, TURN_HALF>
                                    : write_kernel<T, C, 8, true, true, TURN_PAIRS>);
  });
}

int gar_kv_read(const gar_kv_cache *cache, const int64_t *slots, int64_t tokens, void *k, void *v, int dtype,
                gar_stream_t stream) {
  if (int rc = check_rows(cache, dtype, tokens)) return rc;
  if (tokens == 0) return GAR_OK;
  if (k == nullptr || v == nullptr || slots == nullptr) return refuse("null pointer");
  const int size = element_size(dtype);
  if ((uintptr_t)k % size || (uintptr_t)v % size || (uintptr_t)slots % 8) {
    set_error("a buffer is not aligned to its elements");
    return GAR_EALIGN;
  }
  CacheArgs a{};
  a.cache = *cache;
  a.out[0] = k, a.out[1] = v, a.slots = slots;
  const bool rows_wide = (uintptr_t)k % 16 == 0 && (uintptr_t)v % 16 == 0;
  const bool wide = rows_wide && wide_cache(*cache, 8) && (int64_t)cache->dim * size % 16 == 0;
  if (!shape(&a, tokens, 8)) return refuse("too many rows");
  return with_types(dtype, cache->dtype, [&](auto t, auto c) {
    using T = typename decltype(t)::type;
    using C = typename decltype(c)::type;
    auto kernel = wide ? read_kernel<T, C, 8, true, 1> : read_kernel<T, C, 8, false, 1>;
    int rows = 1;
    if (wide && blocks(a, kReadRows) >= 152 * 4)  // enough CTAs to fill the GPU
      kernel = read_kernel<T, C, 8, true, kReadRows>, rows = kReadRows;
    return launch("gar_kv_read", kernel, blocks(a, rows), kThreads, 0, stream, a);
  });
}

int gar_kv_status(const gar_kv_cache *cache, uint32_t *bits, gar_stream_t stream) {
  if (int rc = check_cache(cache)) return rc;
  uint32_t got = 0;
  if (cache->status) {
    cudaError_t e = cudaMemcpyAsync(&got, cache->status, 4, cudaMemcpyDeviceToHost, (cudaStream_t)stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize((cudaStream_t)stream);
    if (e == cudaSuccess && got) e = cudaMemsetAsync(cache->status, 0, 4, (cudaStream_t)stream);
    if (e == cudaSuccess && got) e = cudaStreamSynchronize((cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail(e, "gar_kv_status");
  }
  if (bits) *bits = got;
  if (got == 0) return GAR_OK;
  std::string why = "a kernel met";
  if (got & GAR_KV_BAD_SLOT) why += " a slot past the cache;";
  if (got & GAR_KV_BAD_PAGE) why += " a page number outside the cache;";
  if (got & GAR_KV_BAD_POSITION) why += " a position outside the table;";
  if (got & GAR_KV_BAD_LENGTH) why += " a length that its pages cannot hold;";
  if (got & GAR_KV_TIMEOUT) why += " a copy that did not end;";
  set_error(why);
  return got & GAR_KV_TIMEOUT ? GAR_ETIMEOUT : GAR_EINVAL;
}

}  // extern "C"
