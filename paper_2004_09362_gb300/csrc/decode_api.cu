// Decode attention, and that over shared prefixes: plans, workspaces, checks of arguments, choice of the kernel.
#include <algorithm>
#include <climits>
#include <cmath>
#include <new>

#include "decode_mma.cuh"
#include "prefix.cuh"

struct gar_attn_plan {
  int q_heads, kv_heads, dim;
  int device = -1, sms = 0;
  int give_up = INT_MAX;
  void *ws = nullptr;
};

namespace gar {
namespace {

constexpr size_t kCounterBytes = (kMaxCtas * sizeof(unsigned) + 255) / 256 * 256;

int dim_pad(int dim) { return (dim + 31) / 32 * 32; }

size_t workspace_bytes(const gar_attn_plan &p) {
  const size_t rows = (size_t)kMaxCtas * 2 * kMaxGroup;
  return kCounterBytes + rows * (2 + dim_pad(p.dim)) * sizeof(float);
}

// The tensor-core kernels copy 16-byte chunks.
bool takes_mma(const gar_kv_cache &c, const void *q, int64_t q_batch_stride, int64_t q_head_stride, int q_dtype) {
  const int64_t n = 16 / element_size(c.dtype), m = 16 / element_size(q_dtype);
  return (uintptr_t)q % 16 == 0 && q_batch_stride % m == 0 && q_head_stride % m == 0 && (uintptr_t)c.k % 16 == 0 &&
         (uintptr_t)c.v % 16 == 0 && c.dim % n == 0 && c.page_stride % n == 0 && c.head_stride % n == 0 &&
         c.token_stride % n == 0;
}

}  // namespace

bool box_map(const gar_kv_cache &c, void *base, int rows, bool all_lines, CUtensorMap *map) {
  using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                              const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                              CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static const Encode encode = [] {
    void *f = nullptr;
    cudaDriverEntryPointQueryResult found;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found);
    return e == cudaSuccess && found == cudaDriverEntryPointSuccess ? (Encode)f : (Encode) nullptr;
  }();
  if (encode == nullptr || c.pages < 1) return false;
  const int size = element_size(c.dtype);
  const cuuint32_t line = 128, lines = (cuuint32_t)(c.dim * size) / line;
  const cuuint64_t extent[5] = {line, (cuuint64_t)c.page_size, lines, (cuuint64_t)c.heads, (cuuint64_t)c.pages};
  const cuuint64_t stride[4] = {(cuuint64_t)c.token_stride * size, line, (cuuint64_t)c.head_stride * size,
                                (cuuint64_t)c.page_stride * size};
  const cuuint32_t box[5] = {line, (cuuint32_t)rows, all_lines ? lines : 1, 1, 1}, step[5] = {1, 1, 1, 1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 5, base, extent, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace gar

namespace gar {
namespace {

int check_types(const gar_attn_plan *plan, const gar_kv_cache *cache, int q_dtype, int out_dtype) {
  if (plan == nullptr) return refuse("null plan");
  if (int rc = check_cache(cache)) return rc;
  if (cache->heads != plan->kv_heads || cache->dim != plan->dim) return refuse("the cache's heads or dim are not the plan's");
  if (!float_type(q_dtype)) return refuse("q is GAR_F32, GAR_BF16 or GAR_F16");
  if (float_type(cache->dtype) && cache->dtype != q_dtype) return refuse("a cache of float type goes with queries of its type");
  if (out_dtype != q_dtype && out_dtype != GAR_F32) return refuse("out is of q's type or GAR_F32");
  return GAR_OK;
}

int check_groups(const gar_attn_plan *plan, int batch, int groups) {
  if (batch < 0 || groups < 0 || (batch > 0 && (groups == 0 || batch % groups)))
    return refuse("the batch must be a multiple of the groups");
  if ((int64_t)batch * plan->q_heads > INT_MAX / 2) return refuse("too many sequences and heads");
  return GAR_OK;
}

// Queries of a cached head and a prefix from which on the prefix goes to the tensor cores' own memory, 128 at a time: more than the
// other kernel takes for one reading of the rows.  (The two, 8 cached heads x 128: 65536 rows bf16, 16 queries 96 us and 83, 24 95 and 118,
// 64 96 and 220; 20000 rows f16, 16 queries 56 and 49, 24 54 and 59.)
constexpr int kManyQueries = 17;
// Blocks of queries at most: each has 132 KB of partial results.  (With many prefixes there is not much to gain: 129 prefixes of up to 2000 rows, 20 queries,
// 1032 blocks, 271 us the other way and 302 this, of up to 500 rows 186 and 203; 128 x 2000 264 and 293; 64 x 2000, 32 queries, 512 blocks, 177 both.)
constexpr int kManyItems = 1024;
int blocks_of(int rows) { return rows > 128 ? (rows + 255) / 256 : 1; }

// Bytes of all sequences' rows, a shared one counted for each, up to which they are read for each sequence, mostly from the L2, in one
// launch.  (That and the three launches that read a prefix once, 32/8 heads x 128 bf16: 5 x 425 rows, 9 MB, 11 us and 30; 5 x 4000, 82
// MB, 20 and 32; 16 x 2000, 132 MB, 24 and 30; 64 x 500, 148 MB, 37 and 40; 120 x 1000 of 16/4 x 64 i8, 69 MB, 38 and 41.)
constexpr double kReread = 128 << 20;

bool reads_again(const gar_kv_cache &c, int batch, int prefix_width, int table_width) {
  return ((double)prefix_width + table_width) * c.page_size * batch * c.heads * c.dim * element_size(c.dtype) * 2 <= kReread;
}

bool many_queries(const gar_attn_plan &plan, int batch, int groups) {
  if (groups == 0 || plan.dim > 128) return false;
  const int rows = batch / groups * (plan.q_heads / plan.kv_heads);
  return rows >= kManyQueries && (int64_t)groups * plan.kv_heads * blocks_of(rows) <= kManyItems;
}

// Bytes of a call's workspace, whatever the cache and the tables: the own rows' results, and the prefixes' as they come from either way.
size_t prefix_bytes(const gar_attn_plan &plan, int batch, int groups) {
  const size_t both = prefix_workspace(batch, plan.q_heads, plan.dim, nullptr, nullptr);
  if (!many_queries(plan, batch, groups)) return both;
  const int items = groups * plan.kv_heads * blocks_of(batch / groups * (plan.q_heads / plan.kv_heads));
  return std::max(both, both / 2 + prefix_partials(items, plan.dim, nullptr, nullptr));
}

// What a call over this cache and tables of these widths needs of that: nothing in one launch, and partial results of the tensor cores' own
// memory (20 to 155 MB) with 16-bit rows only.
size_t call_bytes(const gar_attn_plan &plan, const gar_kv_cache &c, int batch, int groups, int prefix_width, int table_width) {
  if (batch == 0 || reads_again(c, batch, prefix_width, table_width)) return 0;
  return element_size(c.dtype) == 2 ? prefix_bytes(plan, batch, groups) : prefix_workspace(batch, plan.q_heads, plan.dim, nullptr, nullptr);
}

// The arguments that follow from the plan, the cache and what a call has set.
int complete(const gar_attn_plan *plan, const gar_kv_cache *cache, int64_t rows, float scale, DecodeArgs *a) {
  // Row numbers stay below 2^31 with room for a tile past the end.
  const int most_rows = (int)std::min<int64_t>(rows, 0x7fffffff - 65536);
  const int unit = unit_of((int64_t)a->batch * plan->kv_heads * ((a->group + 7) / 8), most_rows);
  if (unit == 0) return refuse("too many sequences and heads for tables this wide");
  if (plan->ws == nullptr) {
    set_error("gar_attn_plan_set_workspace has not been called");
    return GAR_ENOWS;
  }
  int dev = -1;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_fail(e, "cudaGetDevice");
  if (dev != plan->device) {
    set_error("the plan's workspace is on another device");
    return GAR_ESTATE;
  }
  a->c = *cache;
  a->page = divide_by((uint32_t)cache->page_size);
  a->most_rows = most_rows, a->q_heads = a->group * plan->kv_heads;
  a->scale_log2 = (float)((double)scale * 1.4426950408889634);
  char *ws = static_cast<char *>(plan->ws);
  a->count = reinterpret_cast<unsigned *>(ws);
  a->part_ml = reinterpret_cast<float2 *>(ws + kCounterBytes);
  a->part_o = reinterpret_cast<float *>(a->part_ml + (size_t)kMaxCtas * 2 * kMaxGroup);
  a->dim_pad = dim_pad(plan->dim), a->device = dev, a->give_up = plan->give_up;
  a->out_wide = (uintptr_t)a->out % (4 * element_size(a->out_dtype)) == 0 && plan->dim % 4 == 0 && a->ob % 4 == 0 && a->oh % 4 == 0;
  a->unit = unit;
  a->slack = std::max(1, 196608 / (128 * cache->dim * element_size(cache->dtype)));
  return GAR_OK;
}

template <typename A> int decode(const gar_attn_plan *plan, const A &a, gar_stream_t stream) {
  if (!takes_mma(a.c, a.q, a.qb, a.qh, a.q_dtype)) return decode_general(a, plan->sms, stream);
  const bool q32 = a.q_dtype == GAR_F32;
  switch (a.c.dtype) {
    case GAR_F32: return decode_mma_f32(a, plan->sms, stream);
    case GAR_BF16: return decode_mma_bf16(a, plan->sms, stream);
    case GAR_F16: return decode_mma_f16(a, plan->sms, stream);
    case GAR_I8: return q32 ? decode_mma_i8_f32(a, plan->sms, stream) : decode_mma_i8(a, plan->sms, stream);
    default: return q32 ? decode_mma_e4m3_f32(a, plan->sms, stream) : decode_mma_e4m3(a, plan->sms, stream);
  }
}

}  // namespace
}  // namespace gar

using namespace gar;

extern "C" {

int gar_attn_plan_create(gar_attn_plan **out, int q_heads, int kv_heads, int dim) {
  if (out == nullptr) return refuse("null output");
  if (kv_heads < 1 || q_heads < 1 || q_heads % kv_heads) return refuse("q_heads must be a multiple of kv_heads");
  if (dim < 1 || dim > GAR_MAX_HEAD_DIM) return refuse("dim must be 1..256");
  gar_attn_plan *p = new (std::nothrow) gar_attn_plan{q_heads, kv_heads, dim};
  if (p == nullptr) {
    set_error("no memory for a plan");
    return GAR_ENOMEM;
  }
  *out = p;
  return GAR_OK;
}

void gar_attn_plan_destroy(gar_attn_plan *plan) { delete plan; }

int gar_attn_plan_shape(const gar_attn_plan *plan, int *q_heads, int *kv_heads, int *dim) {
  if (plan == nullptr) return refuse("null plan");
  if (q_heads) *q_heads = plan->q_heads;
  if (kv_heads) *kv_heads = plan->kv_heads;
  if (dim) *dim = plan->dim;
  return GAR_OK;
}

int gar_attn_plan_bytes(const gar_attn_plan *plan, size_t *bytes) {
  if (plan == nullptr || bytes == nullptr) return refuse("null plan or output");
  *bytes = workspace_bytes(*plan);
  return GAR_OK;
}

int gar_attn_plan_set_workspace(gar_attn_plan *plan, void *dev_ptr, size_t bytes) {
  if (plan == nullptr) return refuse("null plan");
  if (dev_ptr == nullptr) {
    plan->ws = nullptr;
    return GAR_OK;
  }
  if ((uintptr_t)dev_ptr % 16) {
    set_error("the workspace must be 16-byte aligned");
    return GAR_EALIGN;
  }
  if (bytes < workspace_bytes(*plan)) {
    set_error("the workspace is smaller than gar_attn_plan_bytes");
    return GAR_ENOWS;
  }
  int dev = -1, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e == cudaSuccess) e = cudaMemset(dev_ptr, 0, kCounterBytes);
  if (e == cudaSuccess) e = cudaStreamSynchronize(nullptr);
  if (e != cudaSuccess) return cuda_fail(e, "gar_attn_plan_set_workspace");
  plan->ws = dev_ptr, plan->device = dev, plan->sms = std::min(sms, 152);
  return GAR_OK;
}

int gar_attn_plan_debug_wait(gar_attn_plan *plan, int tile) {
  if (plan == nullptr) return refuse("null plan");
  plan->give_up = tile < 0 ? INT_MAX : tile;
  return GAR_OK;
}

int gar_decode_attention(gar_attn_plan *plan, const gar_kv_cache *cache, const void *q, int64_t q_batch_stride,
                         int64_t q_head_stride, int q_dtype, void *out, int64_t out_batch_stride,
                         int64_t out_head_stride, int out_dtype, float *lse, const int32_t *page_table,
                         int64_t table_stride, int table_width, const int32_t *lengths, int batch, float scale,
                         int window, gar_stream_t stream) {
  if (int rc = check_types(plan, cache, q_dtype, out_dtype)) return rc;
  if (batch < 0 || table_width < 0 || window < 0) return refuse("negative batch, table_width or window");
  if (!std::isfinite(scale)) return refuse("scale must be finite");
  if (batch == 0) return GAR_OK;
  if (q == nullptr || out == nullptr || lengths == nullptr || (page_table == nullptr && table_width > 0))
    return refuse("null pointer");
  if ((uintptr_t)q % element_size(q_dtype) || (uintptr_t)out % element_size(out_dtype) || (uintptr_t)lse % 4 ||
      (uintptr_t)page_table % 4 || (uintptr_t)lengths % 4) {
    set_error("a buffer is not aligned to its elements");
    return GAR_EALIGN;
  }
  DecodeArgs a{};
  a.q = q, a.out = out, a.lse = lse;
  a.qb = q_batch_stride, a.qh = q_head_stride, a.ob = out_batch_stride, a.oh = out_head_stride;
  a.table = page_table, a.table_stride = table_stride, a.lengths = lengths;
  a.batch = batch, a.q_dtype = q_dtype, a.out_dtype = out_dtype, a.window = window;
  a.group = plan->q_heads / plan->kv_heads;
  if (int rc = complete(plan, cache, (int64_t)table_width * cache->page_size, scale, &a)) return rc;
  return decode(plan, a, stream);
}

int gar_prefix_attention_bytes(const gar_attn_plan *plan, int batch, int groups, size_t *bytes) {
  if (plan == nullptr || bytes == nullptr) return refuse("null plan or output");
  if (int rc = check_groups(plan, batch, groups)) return rc;
  *bytes = prefix_bytes(*plan, batch, groups);
  return GAR_OK;
}

int gar_prefix_attention_call_bytes(const gar_attn_plan *plan, const gar_kv_cache *cache, int batch, int groups, int prefix_width,
                                    int table_width, size_t *bytes) {
  if (plan == nullptr || bytes == nullptr) return refuse("null plan or output");
  if (int rc = check_cache(cache)) return rc;
  if (cache->heads != plan->kv_heads || cache->dim != plan->dim) return refuse("the cache's heads or dim are not the plan's");
  if (int rc = check_groups(plan, batch, groups)) return rc;
  if (table_width < 0 || prefix_width < 0) return refuse("negative table_width or prefix_width");
  *bytes = call_bytes(*plan, *cache, batch, groups, prefix_width, table_width);
  return GAR_OK;
}

int gar_prefix_attention(gar_attn_plan *plan, const gar_kv_cache *cache, const void *q, int64_t q_batch_stride,
                         int64_t q_head_stride, int q_dtype, void *out, int64_t out_batch_stride, int64_t out_head_stride,
                         int out_dtype, float *lse, const int32_t *prefix_table, int64_t prefix_stride, int prefix_width,
                         const int32_t *prefix_lengths, int groups, const int32_t *page_table, int64_t table_stride,
                         int table_width, const int32_t *lengths, int batch, float scale, void *workspace,
                         size_t workspace_bytes, gar_stream_t stream) {
  if (int rc = check_types(plan, cache, q_dtype, out_dtype)) return rc;
  if (int rc = check_groups(plan, batch, groups)) return rc;
  if (table_width < 0 || prefix_width < 0) return refuse("negative table_width or prefix_width");
  if (!std::isfinite(scale)) return refuse("scale must be finite");
  if (batch == 0) return GAR_OK;
  if (q == nullptr || out == nullptr || lengths == nullptr || prefix_lengths == nullptr ||
      (page_table == nullptr && table_width > 0) || (prefix_table == nullptr && prefix_width > 0))
    return refuse("null pointer");
  if ((uintptr_t)q % element_size(q_dtype) || (uintptr_t)out % element_size(out_dtype) || (uintptr_t)lse % 4 ||
      (uintptr_t)page_table % 4 || (uintptr_t)lengths % 4 || (uintptr_t)prefix_table % 4 || (uintptr_t)prefix_lengths % 4) {
    set_error("a buffer is not aligned to its elements");
    return GAR_EALIGN;
  }
  if ((uintptr_t)workspace % 16) {
    set_error("the workspace must be 16-byte aligned");
    return GAR_EALIGN;
  }
  const int dim = plan->dim, heads = plan->q_heads, group = heads / plan->kv_heads, share = batch / groups;
  PrefixParts parts[2];
  const size_t need = call_bytes(*plan, *cache, batch, groups, prefix_width, table_width);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need)) {
    set_error("the workspace is smaller than gar_prefix_attention_call_bytes");
    return GAR_ENOWS;
  }
  const size_t half = prefix_workspace(batch, heads, dim, static_cast<char *>(workspace), parts) / 2;
  // The parts' results: the sequences' own rows, and the prefixes with a group's queries as those of one sequence.
  ServingArgs own{}, prefix{};
  for (DecodeArgs *a : {static_cast<DecodeArgs *>(&own), static_cast<DecodeArgs *>(&prefix)})
    a->q = q, a->qb = q_batch_stride, a->qh = q_head_stride, a->q_dtype = q_dtype, a->out_dtype = GAR_F32;
  const int64_t row = parts[0].row;
  own.out = parts[0].out, own.lse = parts[0].lse, own.ob = heads * row, own.oh = row;
  own.table = page_table, own.table_stride = table_stride, own.lengths = lengths;
  own.batch = batch, own.group = group;
  prefix.out = parts[1].out, prefix.lse = parts[1].lse, prefix.ob = share * heads * row, prefix.oh = row;
  prefix.table = prefix_table, prefix.table_stride = prefix_stride, prefix.lengths = prefix_lengths;
  prefix.batch = groups, prefix.group = share * group;
  prefix.share = share, prefix.heads_each = group, prefix.by_heads = divide_by((uint32_t)group);
  const int64_t own_rows = (int64_t)table_width * cache->page_size, prefix_rows = (int64_t)prefix_width * cache->page_size;
  if (reads_again(*cache, batch, prefix_width, table_width)) {
    // As sequences of their own, the prefix's rows first.
    own.out = out, own.lse = lse, own.ob = out_batch_stride, own.oh = out_head_stride, own.out_dtype = out_dtype;
    own.before_table = prefix_table, own.before_stride = prefix_stride, own.before_lengths = prefix_lengths;
    own.before_share = share, own.before_most = (int)prefix_rows, own.own_most = (int)own_rows;
    if (int rc = complete(plan, cache, own_rows + prefix_rows, scale, &own)) return rc;
    return decode(plan, own, stream);
  }
  if (int rc = complete(plan, cache, own_rows, scale, &own)) return rc;
  if (int rc = complete(plan, cache, prefix_rows, scale, &prefix)) return rc;
  JoinArgs j{};
  j.parts[0] = parts[0], j.parts[1] = parts[1];
  j.out = out, j.ob = out_batch_stride, j.oh = out_head_stride, j.out_dtype = out_dtype, j.lse = lse;
  j.rows = (int64_t)batch * heads, j.dim = dim, j.heads = heads, j.group = group, j.share = share;
  const int64_t several = 4 * element_size(out_dtype);
  j.wide = (uintptr_t)out % several == 0 && dim % 4 == 0 && out_batch_stride % 4 == 0 && out_head_stride % 4 == 0;
  const int rows = share * group, blocks = blocks_of(rows);
  // (That way rows past the end have scores of -infinity, which a factor of zero would not leave so.)
  if (many_queries(*plan, batch, groups) && element_size(cache->dtype) == 2 && takes_mma(*cache, q, q_batch_stride, q_head_stride, q_dtype) &&
      prefix.scale_log2 != 0.f && (int64_t)groups * plan->kv_heads * blocks * (prefix.most_rows / kKeys + 2) < 1 << 30) {
    PrefixArgs p{};
    p.c = *cache, p.q = q, p.qb = q_batch_stride, p.qh = q_head_stride;
    p.table = prefix_table, p.table_stride = prefix_stride, p.lengths = prefix_lengths;
    p.page = prefix.page, p.by_heads = prefix.by_heads, p.most_rows = prefix.most_rows;
    p.groups = groups, p.share = share, p.heads_each = group, p.rows = rows, p.blocks = blocks;
    p.scale_log2 = std::fabs(prefix.scale_log2), p.negate = prefix.scale_log2 < 0.f ? 0x80008000u : 0u;
    p.ctas = plan->sms, p.device = plan->device, p.give_up = plan->give_up, p.pair = rows > 128;
    prefix_partials(groups * plan->kv_heads * blocks, dim, static_cast<char *>(workspace) + half, &p);
    // Boxes of 8 rows and more that tiles consist of.
    for (int r = kKeys; r >= 8 && p.box == 0; r /= 2)
      if (cache->page_size % r == 0 && (r == kKeys || cache->page_size == r)) p.box = r;
    CUtensorMap maps[2] = {};
    if (dim % 64 || p.box == 0 || !box_map(*cache, cache->k, p.box, false, &maps[0]) || !box_map(*cache, cache->v, p.box, false, &maps[1]))
      p.box = 0;
    if (int rc = prefix_mma(p, maps, stream)) return rc;
    if (int rc = decode(plan, static_cast<const DecodeArgs &>(own), stream)) return rc;
    return join_partials(p, j, stream);
  }
  if (int rc = decode(plan, prefix, stream)) return rc;
  if (int rc = decode(plan, static_cast<const DecodeArgs &>(own), stream)) return rc;
  return join_prefix(j, stream);
}

}  // extern "C"
