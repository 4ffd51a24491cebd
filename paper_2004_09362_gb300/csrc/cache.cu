// The paged key-value cache: rows quantised (keys rotated too) as they are written, and read back.
#include <algorithm>

#include "gar_device.cuh"

namespace gar {
namespace {

constexpr int kChunk = 8;      // channels a lane holds
constexpr int kThreads = 256;

struct CacheArgs {
  gar_kv_cache cache;
  const void *in[2];
  void *out[2];
  int64_t ts[2], hs[2];        // strides of in[]
  const int64_t *slots;
  const void *positions;
  const float2 *table;
  int64_t table_rows;
  int rows;                    // tokens * heads
  int rot, interleaved, wide_positions;
  int lanes;                   // power of two: lanes that hold one row
  bool wide_table;             // a chunk's table entries lie at multiples of 16 bytes
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

// kChunk elements as they lie in memory, and their values.
template <typename T> struct alignas(sizeof(T) > 1 ? 16 : 8) raw_chunk {
  uint32_t w[kChunk * sizeof(T) / 4];
};
template <typename T> __device__ __forceinline__ void values(const raw_chunk<T> &r, float (&v)[kChunk]) {
#pragma unroll
  for (int k = 0; k < kChunk; k += 2) {
    float2 x;
    if constexpr (sizeof(T) == 4)
      x = make_float2(__uint_as_float(r.w[k]), __uint_as_float(r.w[k + 1]));
    else if constexpr (sizeof(T) == 2)
      x = unpack2(r.w[k / 2], T());
    else
      x = unpack2((uint16_t)(r.w[k / 4] >> (k & 2) * 8), T());
    v[k] = x.x, v[k + 1] = x.y;
  }
}

template <bool WIDE, typename T> __device__ __forceinline__ void load(const T *p, int from, int dim, float (&v)[kChunk]) {
  if (WIDE) {
    values(*reinterpret_cast<const raw_chunk<T> *>(p + from), v);
  } else {
#pragma unroll
    for (int k = 0; k < kChunk; ++k) v[k] = from + k < dim ? to_f32(p[from + k]) : 0.f;
  }
}

template <bool WIDE, typename T> __device__ __forceinline__ void store(T *p, int from, int dim, const float (&v)[kChunk]) {
  if (WIDE) {
    constexpr int N = sizeof(T) >= 2 ? 16 / sizeof(T) : kChunk;
#pragma unroll
    for (int k = 0; k < kChunk; k += N) {
      pack<T, N> u;
#pragma unroll
      for (int e = 0; e < N; ++e) u.e[e] = from_f32<T>(v[k + e]);
      *reinterpret_cast<pack<T, N> *>(p + from + k) = u;
    }
  } else {
#pragma unroll
    for (int k = 0; k < kChunk; ++k)
      if (from + k < dim) p[from + k] = from_f32<T>(v[k]);
  }
}

template <bool WIDE, typename T> __device__ __forceinline__ void store_codes(T *p, int from, int dim, const raw_chunk<T> &r) {
  if (WIDE) {
    *reinterpret_cast<raw_chunk<T> *>(p + from) = r;
  } else {
#pragma unroll
    for (int k = 0; k < kChunk; ++k)
      if (from + k < dim) reinterpret_cast<uint8_t *>(p)[from + k] = (uint8_t)(r.w[k / 4] >> 8 * (k % 4));
  }
}

// The channels [from, from + kChunk) of a row rotated.  With the half layout the channels they
// pair with are another lane's; they were read into w as well.
template <bool WIDE, typename T>
__device__ __forceinline__ void rotate(const CacheArgs &a, const T *row, int64_t token, int from, float (&v)[kChunk],
                                       const float (&w)[kChunk]) {
  const int64_t pos = a.wide_positions ? static_cast<const int64_t *>(a.positions)[token]
                                       : (int64_t) static_cast<const int32_t *>(a.positions)[token];
  const bool good = (uint64_t)pos < (uint64_t)a.table_rows;
  if (!good && a.cache.status) atomicOr(a.cache.status, GAR_KV_BAD_POSITION);
  const int half = a.rot / 2;
  const float2 *const t = a.table + (good ? pos * half : 0);
  if (WIDE && a.wide_table) {
    if (a.interleaved) {
      float c[kChunk / 2], s[kChunk / 2];
      load_rotation<kChunk / 2, true>(t + (good ? from / 2 : 0), good, c, s);
#pragma unroll
      for (int k = 0; k < kChunk; k += 2) {
        const float x = v[k], y = v[k + 1];
        v[k] = __fsub_rn(__fmul_rn(x, c[k / 2]), __fmul_rn(y, s[k / 2]));
        v[k + 1] = __fadd_rn(__fmul_rn(y, c[k / 2]), __fmul_rn(x, s[k / 2]));
      }
    } else {
      const bool second = from >= half;
      float c[kChunk], s[kChunk];
      load_rotation<kChunk, true>(t + (good ? from - (second ? half : 0) : 0), good, c, s);
#pragma unroll
      for (int k = 0; k < kChunk; ++k) {
        const float x = __fmul_rn(v[k], c[k]), y = __fmul_rn(w[k], s[k]);
        v[k] = second ? __fadd_rn(x, y) : __fsub_rn(x, y);
      }
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < kChunk; ++k) {
    const int c = from + k;
    if (c >= a.rot) break;
    const int pair = a.interleaved ? c / 2 : c < half ? c : c - half;
    const bool second = a.interleaved ? c & 1 : c >= half;
    const int other = a.interleaved ? c ^ 1 : second ? c - half : c + half;
    const float2 cs = good ? __ldg(t + pair) : make_float2(__int_as_float(0x7fc00000), 0.f);
    const float x = __fmul_rn(v[k], cs.x), y = __fmul_rn(to_f32(row[other]), cs.y);
    v[k] = second ? __fadd_rn(x, y) : __fsub_rn(x, y);
  }
}

// Codes of the row of which this lane holds v, and the row's scale.
//
// v / scale is rounded as the definition has it, without a division each: for r = 1 / scale rounded to
// nearest and q = v r, the remainder v - q scale is exact in a fused multiply-add, and
// q + r (v - q scale) is the correctly rounded quotient (P. Markstein, IBM J. Res. Dev. 34, 1990, theorem 8),
// as long as nothing underflows; rows of scales under 2^-90 divide.
template <typename C> __device__ __forceinline__ raw_chunk<C> quantise(const float (&v)[kChunk], int lanes, float *scale) {
  // Magnitudes compare as integers, NaNs and infinities the largest.
  uint32_t most = 0;
#pragma unroll
  for (int k = 0; k < kChunk; ++k) most = max(most, __float_as_uint(v[k]) & 0x7fffffffu);
  for (int d = lanes / 2; d > 0; d /= 2) most = max(most, __shfl_xor_sync(~0u, most, d));
  raw_chunk<C> out;
  float x[kChunk];
  const float s = __fmul_rn(__uint_as_float(most), 1.f / quantised<C>::largest);
  if (most >= 0x7f800000u) {  // an infinity or a NaN in the row: codes 0 under a NaN scale
    *scale = __int_as_float(0x7fc00000);
#pragma unroll
    for (int k = 0; k < kChunk; ++k) x[k] = 0.f;
  } else {
    *scale = s;
    const float r = __frcp_rn(s);
    if (s >= 0x1p-90f) {
#pragma unroll
      for (int k = 0; k < kChunk; ++k) {
        const float q = __fmul_rn(v[k], r);
        x[k] = __fmaf_rn(__fmaf_rn(-q, s, v[k]), r, q);
      }
    } else {
#pragma unroll
      for (int k = 0; k < kChunk; ++k)
        x[k] = s == 0.f ? 0.f : fminf(fmaxf(__fdiv_rn(v[k], s), -quantised<C>::largest), quantised<C>::largest);
    }
  }
#pragma unroll
  for (int k = 0; k < kChunk; k += 4) out.w[k / 4] = codes4(x[k], x[k + 1], x[k + 2], x[k + 3], C());
  return out;
}

// T -> C rows.  a.lanes neighbouring lanes hold a token's row of one head, kChunk channels of the key
// and of the value each, so that the largest magnitudes are found by shuffles and the rows are
// read once.  Bound by memory: all loads but the table's go out before any is waited for.
template <typename T, typename C, bool WIDE, bool ROTATE>
__global__ void __launch_bounds__(kThreads) write_kernel(const CacheArgs a) {
  const gar_kv_cache &c = a.cache;
  const int lane = threadIdx.x & (a.lanes - 1), from = lane * kChunk;
  const int i = blockIdx.x * (kThreads / a.lanes) + threadIdx.x / a.lanes;
  const bool any = i < a.rows;
  const int64_t token = any ? a.heads(i) : 0;
  const int head = any ? i - (int)token * c.heads : 0;
  const int64_t slot = any ? a.slots[token] : -1;
  const T *const k_row = static_cast<const T *>(a.in[0]) + token * a.ts[0] + head * a.hs[0];
  const T *const v_row = static_cast<const T *>(a.in[1]) + token * a.ts[1] + head * a.hs[1];
  float k[kChunk] = {}, v[kChunk] = {}, w[kChunk];
  const bool in = any && from < c.dim, turned = ROTATE && in && from < a.rot;
  if (in) {
    load<WIDE>(k_row, from, c.dim, k);
    load<WIDE>(v_row, from, c.dim, v);
    if (turned && WIDE && a.wide_table && !a.interleaved) {
      const int half = a.rot / 2;
      load<WIDE>(k_row, from >= half ? from - half : from + half, c.dim, w);
    }
  }
  Place p;
  const bool there = find(a, slot, head, &p);
  if (turned && there) rotate<WIDE>(a, k_row, token, from, k, w);
  if constexpr (quantised<C>::value) {
    float k_scale, v_scale;
    const raw_chunk<C> k_codes = quantise<C>(k, a.lanes, &k_scale), v_codes = quantise<C>(v, a.lanes, &v_scale);
    if (there && lane == 0) c.k_scale[p.scale] = k_scale, c.v_scale[p.scale] = v_scale;
    if (in && there) {
      store_codes<WIDE>(static_cast<C *>(c.k) + p.at, from, c.dim, k_codes);
      store_codes<WIDE>(static_cast<C *>(c.v) + p.at, from, c.dim, v_codes);
    }
  } else if (in && there) {
    store<WIDE>(static_cast<C *>(c.k) + p.at, from, c.dim, k);
    store<WIDE>(static_cast<C *>(c.v) + p.at, from, c.dim, v);
  }
}

// C -> T rows, N of them to a lane: a row's place hangs on its slot, so there are fewer bytes in flight.
template <typename T, typename C, bool WIDE, int N>
__global__ void __launch_bounds__(kThreads) read_kernel(const CacheArgs a) {
  const gar_kv_cache &c = a.cache;
  const int lane = threadIdx.x & (a.lanes - 1), from = lane * kChunk, step = kThreads / a.lanes;
  const int i0 = blockIdx.x * (step * N) + threadIdx.x / a.lanes;
  if (from >= c.dim) return;
  Place p[N];
  bool there[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int i = i0 + n * step;
    const int token = i < a.rows ? a.heads(i) : 0;
    there[n] = i < a.rows && find(a, a.slots[token], i - token * c.heads, &p[n]);
  }
  raw_chunk<C> k[N], v[N];
  float k_scale[N], v_scale[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    k_scale[n] = v_scale[n] = 0.f;
    if (there[n]) {
      if (WIDE) {
        k[n] = *reinterpret_cast<const raw_chunk<C> *>(static_cast<const C *>(c.k) + p[n].at + from);
        v[n] = *reinterpret_cast<const raw_chunk<C> *>(static_cast<const C *>(c.v) + p[n].at + from);
      }
      if (quantised<C>::value) k_scale[n] = c.k_scale[p[n].scale], v_scale[n] = c.v_scale[p[n].scale];
    }
  }
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int64_t i = i0 + n * step;
    if (i >= a.rows) break;
    float x[kChunk] = {}, y[kChunk] = {};
    if (there[n]) {
      if (WIDE) {
        values(k[n], x);
        values(v[n], y);
      } else {
        load<WIDE>(static_cast<const C *>(c.k) + p[n].at, from, c.dim, x);
        load<WIDE>(static_cast<const C *>(c.v) + p[n].at, from, c.dim, y);
      }
    }
    if (quantised<C>::value) {
#pragma unroll
      for (int e = 0; e < kChunk; ++e) x[e] = __fmul_rn(x[e], k_scale[n]), y[e] = __fmul_rn(y[e], v_scale[n]);
    }
    store<WIDE>(static_cast<T *>(a.out[0]) + i * c.dim, from, c.dim, x);
    store<WIDE>(static_cast<T *>(a.out[1]) + i * c.dim, from, c.dim, y);
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

// Sets the rows and lanes; false where the rows are too many.
bool shape(CacheArgs *a, int64_t tokens) {
  const int need = (a->cache.dim + kChunk - 1) / kChunk;
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

// 16 bytes of `size`-byte elements (8 of one byte) at every multiple of kChunk channels.
bool wide_cache(const gar_kv_cache &c) {
  const uintptr_t a = element_size(c.dtype) == 1 ? 8 : 16;
  return (uintptr_t)c.k % a == 0 && (uintptr_t)c.v % a == 0 && c.dim % kChunk == 0 && c.page_stride % kChunk == 0 &&
         c.head_stride % kChunk == 0 && c.token_stride % kChunk == 0;
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
  if (!shape(&a, tokens)) return refuse("too many rows");
  const int n = 16 / size;
  a.wide_table = (uintptr_t)table % 16 == 0 && rot % (a.interleaved ? kChunk : 2 * kChunk) == 0;
  const bool wide = wide_cache(*cache) && (uintptr_t)k % 16 == 0 && (uintptr_t)v % 16 == 0 && k_token_stride % n == 0 &&
                    k_head_stride % n == 0 && v_token_stride % n == 0 && v_head_stride % n == 0;
  return with_types(dtype, cache->dtype, [&](auto t, auto c) {
    using T = typename decltype(t)::type;
    using C = typename decltype(c)::type;
    const auto kernel = wide ? (positions ? write_kernel<T, C, true, true> : write_kernel<T, C, true, false>)
                             : (positions ? write_kernel<T, C, false, true> : write_kernel<T, C, false, false>);
    kernel<<<blocks(a, 1), kThreads, 0, (cudaStream_t)stream>>>(a);
    return launched("write_kernel");
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
  if (!shape(&a, tokens)) return refuse("too many rows");
  const bool wide = wide_cache(*cache) && (uintptr_t)k % 16 == 0 && (uintptr_t)v % 16 == 0;
  return with_types(dtype, cache->dtype, [&](auto t, auto c) {
    using T = typename decltype(t)::type;
    using C = typename decltype(c)::type;
    if (!wide)
      read_kernel<T, C, false, 1><<<blocks(a, 1), kThreads, 0, (cudaStream_t)stream>>>(a);
    else if (blocks(a, 4) < 152 * 4)   // too few CTAs to fill the GPU with four rows a lane
      read_kernel<T, C, true, 1><<<blocks(a, 1), kThreads, 0, (cudaStream_t)stream>>>(a);
    else
      read_kernel<T, C, true, 4><<<blocks(a, 4), kThreads, 0, (cudaStream_t)stream>>>(a);
    return launched("read_kernel");
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
