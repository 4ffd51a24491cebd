// Decode attention: plans, workspaces, checks of arguments, choice of the kernel.
#include <algorithm>
#include <climits>
#include <cmath>
#include <new>

#include "decode_mma.cuh"

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

// Rows of a unit of the line: as many as it takes for the whole line, each item counted twice at most, to stay below 2^30
// units, or 0 where 2^15 do not.
int unit_of(int64_t items, int most_rows) {
  for (int unit = 64; unit <= 32768; unit *= 2)
    if (items * (most_rows / unit + 3) * 2 < 1 << 30) return unit;
  return 0;
}

// The tensor-core kernels copy 16-byte chunks.
bool takes_mma(const gar_kv_cache &c, const void *q, int64_t q_batch_stride, int64_t q_head_stride, int q_dtype) {
  const int64_t n = 16 / element_size(c.dtype), m = 16 / element_size(q_dtype);
  return (uintptr_t)q % 16 == 0 && q_batch_stride % m == 0 && q_head_stride % m == 0 && (uintptr_t)c.k % 16 == 0 &&
         (uintptr_t)c.v % 16 == 0 && c.dim % n == 0 && c.page_stride % n == 0 && c.head_stride % n == 0 &&
         c.token_stride % n == 0;
}

}  // namespace

bool box_map(const gar_kv_cache &c, void *base, int rows, CUtensorMap *map) {
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
  const cuuint32_t box[5] = {line, (cuuint32_t)rows, lines, 1, 1}, step[5] = {1, 1, 1, 1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 5, base, extent, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

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
  if (plan == nullptr) return refuse("null plan");
  if (int rc = check_cache(cache)) return rc;
  if (cache->heads != plan->kv_heads || cache->dim != plan->dim) return refuse("the cache's heads or dim are not the plan's");
  if (!float_type(q_dtype)) return refuse("q is GAR_F32, GAR_BF16 or GAR_F16");
  if (float_type(cache->dtype) && cache->dtype != q_dtype) return refuse("a cache of float type goes with queries of its type");
  if (out_dtype != q_dtype && out_dtype != GAR_F32) return refuse("out is of q's type or GAR_F32");
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
  // Row numbers stay below 2^31 with room for a tile past the end.
  const int most_rows = (int)std::min<int64_t>((int64_t)table_width * cache->page_size, 0x7fffffff - 65536);
  const int group = plan->q_heads / plan->kv_heads;
  const int unit = unit_of((int64_t)batch * plan->kv_heads * ((group + 7) / 8), most_rows);
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
  DecodeArgs a{};
  a.c = *cache;
  a.q = q, a.out = out, a.lse = lse;
  a.qb = q_batch_stride, a.qh = q_head_stride, a.ob = out_batch_stride, a.oh = out_head_stride;
  a.table = page_table, a.table_stride = table_stride, a.lengths = lengths;
  a.page = divide_by((uint32_t)cache->page_size);
  a.most_rows = most_rows, a.batch = batch, a.q_heads = plan->q_heads, a.group = group;
  a.q_dtype = q_dtype, a.out_dtype = out_dtype, a.window = window;
  a.scale_log2 = (float)((double)scale * 1.4426950408889634);
  char *ws = static_cast<char *>(plan->ws);
  a.count = reinterpret_cast<unsigned *>(ws);
  a.part_ml = reinterpret_cast<float2 *>(ws + kCounterBytes);
  a.part_o = reinterpret_cast<float *>(a.part_ml + (size_t)kMaxCtas * 2 * kMaxGroup);
  a.dim_pad = dim_pad(plan->dim), a.device = dev, a.give_up = plan->give_up;
  a.out_wide = (uintptr_t)out % (4 * element_size(out_dtype)) == 0 && plan->dim % 4 == 0 && out_batch_stride % 4 == 0 &&
               out_head_stride % 4 == 0;
  a.unit = unit;
  a.slack = std::max(1, 196608 / (128 * cache->dim * element_size(cache->dtype)));
  if (!takes_mma(*cache, q, q_batch_stride, q_head_stride, q_dtype)) return decode_general(a, plan->sms, stream);
  const bool q32 = q_dtype == GAR_F32;
  switch (cache->dtype) {
    case GAR_F32: return decode_mma_f32(a, plan->sms, stream);
    case GAR_BF16: return decode_mma_bf16(a, plan->sms, stream);
    case GAR_F16: return decode_mma_f16(a, plan->sms, stream);
    case GAR_I8: return (q32 ? decode_mma_i8_f32 : decode_mma_i8)(a, plan->sms, stream);
    default: return (q32 ? decode_mma_e4m3_f32 : decode_mma_e4m3)(a, plan->sms, stream);
  }
}

}  // extern "C"
