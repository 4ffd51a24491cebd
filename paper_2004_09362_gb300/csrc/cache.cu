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
  const void *positions;       // null: no rotation
  const float2 *table;
  int64_t table_rows;
  int64_t rows;                // tokens * heads
  int rot, interleaved, wide_positions;
  int lanes;                   // power of two: lanes that hold one row
};

// The place of a slot's row, or false where there is none.
struct Place {
  int64_t at, scale;
};
__device__ __forceinline__ bool find(const gar_kv_cache &c, int64_t slot, int head, Place *p) {
  if (slot < 0) return false;
  int64_t page;
  int row;
  if ((uint64_t)slot <= 0xffffffffu) {  // a 32-bit division where it does
    page = (uint32_t)slot / (uint32_t)c.page_size;
    row = (int)((uint32_t)slot - (uint32_t)page * (uint32_t)c.page_size);
  } else {
    page = slot / c.page_size;
    row = (int)(slot - page * c.page_size);
  }
  if (page >= c.pages) {
    if (c.status) atomicOr(c.status, GAR_KV_BAD_SLOT);
    return false;
  }
  p->at = page * c.page_stride + head * c.head_stride + row * c.token_stride;
  p->scale = page * c.scale_page_stride + head * c.scale_head_stride + row * c.scale_token_stride;
  return true;
}

template <bool WIDE, typename T> __device__ __forceinline__ void load(const T *p, int from, int dim, float (&v)[kChunk]) {
  if (WIDE) {
    constexpr int N = sizeof(T) >= 2 ? 16 / sizeof(T) : kChunk;
#pragma unroll
    for (int k = 0; k < kChunk; k += N) {
      const pack<T, N> u = *reinterpret_cast<const pack<T, N> *>(p + from + k);
#pragma unroll
      for (int e = 0; e < N; ++e) v[k + e] = to_f32(u.e[e]);
    }
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

// The channels [from, from + kChunk) of a row rotated; each needs its partner, which is read
// again (from the row that is in L1 by then) rather than exchanged.
template <typename T>
__device__ __forceinline__ void rotate(const CacheArgs &a, const T *row, int64_t token, int from, float (&v)[kChunk]) {
  if (from >= a.rot) return;
  const int64_t pos = a.wide_positions ? static_cast<const int64_t *>(a.positions)[token]
                                       : (int64_t) static_cast<const int32_t *>(a.positions)[token];
  const bool good = (uint64_t)pos < (uint64_t)a.table_rows;
  if (!good && a.cache.status) atomicOr(a.cache.status, GAR_KV_BAD_POSITION);
  const int half = a.rot / 2;
#pragma unroll
  for (int k = 0; k < kChunk; ++k) {
    const int c = from + k;
    if (c >= a.rot) break;
    const int pair = a.interleaved ? c / 2 : c < half ? c : c - half;
    const bool second = a.interleaved ? c & 1 : c >= half;
    const int other = a.interleaved ? c ^ 1 : second ? c - half : c + half;
    const float2 cs = good ? __ldg(a.table + pos * half + pair) : make_float2(__int_as_float(0x7fc00000), 0.f);
    const float w = to_f32(row[other]);
    v[k] = second ? __fadd_rn(__fmul_rn(v[k], cs.x), __fmul_rn(w, cs.y))
                  : __fsub_rn(__fmul_rn(v[k], cs.x), __fmul_rn(w, cs.y));
  }
}

// T -> C rows.  a.lanes neighbouring lanes hold a row, kChunk channels each, so that the largest
// magnitude is found by shuffles and the row is read once.  blockIdx.y: 0 keys, 1 values.
// Bound by memory.
template <typename T, typename C, bool WIDE> __global__ void __launch_bounds__(kThreads) write_kernel(const CacheArgs a) {
  const gar_kv_cache &c = a.cache;
  const int which = blockIdx.y;
  const int lane = threadIdx.x & (a.lanes - 1), from = lane * kChunk;
  const int64_t i = (int64_t)blockIdx.x * (kThreads / a.lanes) + threadIdx.x / a.lanes;
  Place p;
  const int64_t token = i / c.heads;
  const int head = (int)(i - token * c.heads);
  const bool there = i < a.rows && find(c, a.slots[token], head, &p);
  const bool mine = there && from < c.dim;
  float v[kChunk] = {};
  if (mine) {
    const T *row = static_cast<const T *>(a.in[which]) + token * a.ts[which] + head * a.hs[which];
    load<WIDE>(row, from, c.dim, v);
    if (which == 0 && a.positions) rotate(a, row, token, from, v);
  }
  if (quantised<C>::value) {
    float most = 0.f;
    bool sound = true;
#pragma unroll
    for (int k = 0; k < kChunk; ++k) {
      most = fmaxf(most, fabsf(v[k]));
      sound &= fabsf(v[k]) <= 3.402823466e38f;
    }
    if (!sound) most = __int_as_float(0x7f800000);
    for (int d = a.lanes / 2; d > 0; d /= 2) most = fmaxf(most, __shfl_xor_sync(~0u, most, d));
    // An infinity or a NaN in the row: codes 0 under a NaN scale.
    const bool bad = most > 3.402823466e38f;
    const float scale = bad ? __int_as_float(0x7fc00000) : __fmul_rn(most, 1.f / quantised<C>::largest);
#pragma unroll
    for (int k = 0; k < kChunk; ++k) v[k] = bad || scale == 0.f ? 0.f : __fdiv_rn(v[k], scale);
    if (there && lane == 0) (which ? c.v_scale : c.k_scale)[p.scale] = scale;
  }
  if (mine) store<WIDE>(static_cast<C *>(which ? c.v : c.k) + p.at, from, c.dim, v);
}

template <typename T, typename C, bool WIDE> __global__ void __launch_bounds__(kThreads) read_kernel(const CacheArgs a) {
  const gar_kv_cache &c = a.cache;
  const int which = blockIdx.y;
  const int lane = threadIdx.x & (a.lanes - 1), from = lane * kChunk;
  const int64_t i = (int64_t)blockIdx.x * (kThreads / a.lanes) + threadIdx.x / a.lanes;
  if (i >= a.rows || from >= c.dim) return;
  Place p;
  const int64_t token = i / c.heads;
  const int head = (int)(i - token * c.heads);
  float v[kChunk] = {};
  if (find(c, a.slots[token], head, &p)) {
    load<WIDE>(static_cast<const C *>(which ? c.v : c.k) + p.at, from, c.dim, v);
    if (quantised<C>::value) {
      const float scale = (which ? c.v_scale : c.k_scale)[p.scale];
#pragma unroll
      for (int k = 0; k < kChunk; ++k) v[k] = __fmul_rn(v[k], scale);
    }
  }
  store<WIDE>(static_cast<T *>(a.out[which]) + i * c.dim, from, c.dim, v);
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

// The launch's grid and lanes; false where the rows are too many.
bool shape(CacheArgs *a, int64_t tokens, dim3 *grid) {
  const int need = (a->cache.dim + kChunk - 1) / kChunk;
  a->lanes = 1;
  while (a->lanes < need) a->lanes *= 2;
  a->rows = tokens * a->cache.heads;
  const int64_t per = kThreads / a->lanes, blocks = (a->rows + per - 1) / per;
  *grid = dim3((unsigned)blocks, 2);
  return blocks <= 0x7fffffff;
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
  dim3 grid;
  if (!shape(&a, tokens, &grid)) return refuse("too many rows");
  const int n = 16 / size;
  const bool wide = wide_cache(*cache) && (uintptr_t)k % 16 == 0 && (uintptr_t)v % 16 == 0 && k_token_stride % n == 0 &&
                    k_head_stride % n == 0 && v_token_stride % n == 0 && v_head_stride % n == 0;
  return with_types(dtype, cache->dtype, [&](auto t, auto c) {
    using T = typename decltype(t)::type;
    using C = typename decltype(c)::type;
    if (wide)
      write_kernel<T, C, true><<<grid, kThreads, 0, (cudaStream_t)stream>>>(a);
    else
      write_kernel<T, C, false><<<grid, kThreads, 0, (cudaStream_t)stream>>>(a);
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
  dim3 grid;
  if (!shape(&a, tokens, &grid)) return refuse("too many rows");
  const bool wide = wide_cache(*cache) && (uintptr_t)k % 16 == 0 && (uintptr_t)v % 16 == 0;
  return with_types(dtype, cache->dtype, [&](auto t, auto c) {
    using T = typename decltype(t)::type;
    using C = typename decltype(c)::type;
    if (wide)
      read_kernel<T, C, true><<<grid, kThreads, 0, (cudaStream_t)stream>>>(a);
    else
      read_kernel<T, C, false><<<grid, kThreads, 0, (cudaStream_t)stream>>>(a);
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
