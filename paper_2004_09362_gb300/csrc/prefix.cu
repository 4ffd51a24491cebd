// Attention of a batch over a prefix that its sequences share, joined with that over their own rows.
#include "prefix.cuh"

namespace gar {
namespace {

constexpr int kThreads = 256;

template <typename T> __device__ __forceinline__ void put(void *out, int64_t at, float x) {
  static_cast<T *>(out)[at] = from_f32<T>(x);
}

// A warp joins a query's two results:  out = (2^(l0 - l) out0 + 2^(l1 - l) out1),  l = log2(2^l0 + 2^l1).
__global__ void __launch_bounds__(kThreads) join_kernel(const JoinArgs a) {
  after_earlier_kernels();
  const int64_t i = (int64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
  if (i >= a.rows) return;
  const int lane = threadIdx.x & 31;
  const int64_t b = i / a.heads, g = b / a.share;
  const int h = (int)(i - b * a.heads), kv = h / a.group;
  const int64_t j = (g * (a.heads / a.group) + kv) * ((int64_t)a.share * a.group) + (b - g * a.share) * a.group + (h - kv * a.group);
  const float x = __ldcg(a.parts[0].lse + i), y = __ldcg(a.parts[1].lse + j), top = fmaxf(x, y);
  const float off = top == -INFINITY ? 0.f : top;
  float wx = expf(x - off), wy = expf(y - off);
  const float sum = wx + wy;
  if (a.lse && lane == 0) a.lse[i] = top == -INFINITY ? top : off + logf(sum);
  if (sum > 0.f) wx /= sum, wy /= sum;
  const float *const p = a.parts[0].out + i * a.parts[0].row, *const q = a.parts[1].out + j * a.parts[1].row;
  for (int d = lane; d < a.dim; d += 32) {
    // (a part without rows holds zeros)
    const float z = wx * __ldcg(p + d) + wy * __ldcg(q + d);
    const int64_t at = b * a.ob + h * a.oh + d;
    if (a.out_dtype == GAR_F32)
      put<float>(a.out, at, z);
    else if (a.out_dtype == GAR_BF16)
      put<__nv_bfloat16>(a.out, at, z);
    else
      put<__half>(a.out, at, z);
  }
}

}  // namespace

size_t prefix_workspace(int batch, int heads, int dim, char *base, PrefixParts *parts) {
  const int64_t rows = (int64_t)batch * heads, row = (dim + 3) / 4 * 4;
  const size_t outs = (size_t)(rows * row) * sizeof(float), sums = ((size_t)rows * sizeof(float) + 15) / 16 * 16;
  if (parts)
    for (int i = 0; i < 2; ++i) {
      char *const at = base + i * (outs + sums);
      parts[i] = {reinterpret_cast<float *>(at), reinterpret_cast<float *>(at + outs), row};
    }
  return 2 * (outs + sums);
}

int join_prefix(const JoinArgs &a, gar_stream_t stream) {
  return launch("gar_prefix_attention", join_kernel, (a.rows + kThreads / 32 - 1) / (kThreads / 32), kThreads, 0, stream, a);
}

}  // namespace gar
