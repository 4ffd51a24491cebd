// Rotary positions: the table of rotations, and the kernel that applies it.
#include <algorithm>
#include <cmath>

#include "gar_device.cuh"

namespace gar {
namespace {

struct Frequencies {
  double f[GAR_MAX_HEAD_DIM / 2];
};

// One thread per entry.  64-bit sincos: this GPU is slow at it, and a table is made once.
__global__ void rope_table_kernel(float2 *table, int64_t first, int64_t count, int pairs, double magnitude,
                                  const __grid_constant__ Frequencies fr) {
  after_earlier_kernels();
  const int64_t n = count * pairs, step = (int64_t)gridDim.x * blockDim.x;
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += step) {
    const int64_t row = i / pairs;
    double s, c;
    sincos((double)(first + row) * fr.f[i - row * pairs], &s, &c);
    table[i] = make_float2((float)(c * magnitude), (float)(s * magnitude));
  }
}

struct RopeArgs {
  const void *x;
  void *out;
  int64_t xt, xh, ot, oh;  // strides
  int64_t tokens;
  const void *positions;
  const float2 *table;
  int64_t table_rows;
  int heads, dim, rot;
  int units;         // per (token, head): vectors of pairs, then vectors that are copied
  int pair_units;
  int lanes;         // threads that share a (token, unit), each with every lanes-th head
  int block_tokens;
  int wide_positions;
  float sign;        // -1 turns back
};

__device__ __forceinline__ int64_t position(const RopeArgs &a, int64_t token) {
  return a.wide_positions ? static_cast<const int64_t *>(a.positions)[token]
                          : (int64_t) static_cast<const int32_t *>(a.positions)[token];
}

// out = x rotated.  Bound by memory: every element is read and written once.
//
// A unit is the work of one thread at one head: with the half layout V channels of the
// first half and the V that pair with them (two 16-byte accesses each way), with the interleaved
// layout V channels that hold V/2 pairs; the channels past `rot` are copied in units of V.  The
// rotation depends on token and channel only, so a thread keeps its unit's table entries in
// registers and takes several heads; kUnroll heads' loads are in flight at once, the first of
// them before the token's position is known (two in flight 53 us, four 52, eight 59 at the size below).
// 16384 tokens x 40 heads x 128 bf16: 52 us, 6.6 TB/s, 0.98 of what a copy reaches; one token 1.7 us, which
// is the launch and two round trips to memory.
template <typename T, bool INTERLEAVED> __global__ void __launch_bounds__(256) rope_kernel(const RopeArgs a) {
  constexpr int kUnroll = 4;
  using chunk = chunk16<T>;
  constexpr int V = chunk::N, PAIRS = INTERLEAVED ? V / 2 : V;
  after_earlier_kernels();
  const int per_token = a.lanes * a.units;
  for (int i = threadIdx.x; i < a.block_tokens * per_token; i += blockDim.x) {
    const int bt = i / per_token, r = i - bt * per_token;
    const int lane = r / a.units, unit = r - lane * a.units;
    const int64_t token = (int64_t)blockIdx.x * a.block_tokens + bt;
    if (token >= a.tokens) return;
    const bool copy = unit >= a.pair_units;
    const int at = copy ? a.rot + (unit - a.pair_units) * V : unit * V;
    const T *x = static_cast<const T *>(a.x) + token * a.xt + at;
    T *out = static_cast<T *>(a.out) + token * a.ot + at;
    const int half = a.rot / 2;
    chunk p[kUnroll], q[kUnroll];
    const auto load = [&](int h0) {
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        const int h = h0 + k * a.lanes;
        if (h >= a.heads) break;
        p[k] = *reinterpret_cast<const chunk *>(x + h * a.xh);
        if (!INTERLEAVED && !copy) q[k] = *reinterpret_cast<const chunk *>(x + h * a.xh + half);
      }
    };
    load(lane);
    float c[PAIRS], s[PAIRS];
    if (!copy) {
      const int64_t pos = position(a, token);
      const bool good = (uint64_t)pos < (uint64_t)a.table_rows;
      load_rotation<PAIRS, true>(a.table + (good ? pos * half + unit * PAIRS : 0), good, c, s);
#pragma unroll
      for (int k = 0; k < PAIRS; ++k) s[k] *= a.sign;
    }
    for (int h0 = lane; h0 < a.heads;) {
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        const int h = h0 + k * a.lanes;
        if (h >= a.heads) break;
        if (!copy) {
          float u[V], v[V];
          unpack(p[k], u);
          if (!INTERLEAVED) unpack(q[k], v);
#pragma unroll
          for (int e = 0; e < PAIRS; ++e) {
            float &y = INTERLEAVED ? u[2 * e] : u[e], &z = INTERLEAVED ? u[2 * e + 1] : v[e];
            const float y0 = y, z0 = z;
            y = __fsub_rn(__fmul_rn(y0, c[e]), __fmul_rn(z0, s[e]));
            z = __fadd_rn(__fmul_rn(z0, c[e]), __fmul_rn(y0, s[e]));
          }
          p[k] = packed<T>(u);
          if (!INTERLEAVED) *reinterpret_cast<chunk *>(out + h * a.oh + half) = packed<T>(v);
        }
        *reinterpret_cast<chunk *>(out + h * a.oh) = p[k];
      }
      h0 += kUnroll * a.lanes;
      load(h0);
    }
  }
}

// The same where 16-byte accesses do not fit: one pair, or one copied channel, of every lanes-th head.
template <typename T> __global__ void __launch_bounds__(256) rope_narrow_kernel(const RopeArgs a, bool interleaved) {
  after_earlier_kernels();
  const int per_token = a.lanes * a.units;
  for (int i = threadIdx.x; i < a.block_tokens * per_token; i += blockDim.x) {
    const int bt = i / per_token, r = i - bt * per_token;
    const int lane = r / a.units, unit = r - lane * a.units;
    const int64_t token = (int64_t)blockIdx.x * a.block_tokens + bt;
    if (token >= a.tokens) return;
    const T *x = static_cast<const T *>(a.x) + token * a.xt;
    T *out = static_cast<T *>(a.out) + token * a.ot;
    if (unit >= a.pair_units) {
      const int at = a.rot + unit - a.pair_units;
      for (int h = lane; h < a.heads; h += a.lanes) out[h * a.oh + at] = x[h * a.xh + at];
      continue;
    }
    const int64_t pos = position(a, token);
    const bool good = (uint64_t)pos < (uint64_t)a.table_rows;
    float c[1], s[1];
    load_rotation<1, false>(a.table + (good ? pos * (a.rot / 2) + unit : 0), good, c, s);
    s[0] *= a.sign;
    const int at = interleaved ? 2 * unit : unit, to = interleaved ? at + 1 : at + a.rot / 2;
    for (int h = lane; h < a.heads; h += a.lanes) {
      const float u = to_f32(x[h * a.xh + at]), v = to_f32(x[h * a.xh + to]);
      out[h * a.oh + at] = from_f32<T>(__fsub_rn(__fmul_rn(u, c[0]), __fmul_rn(v, s[0])));
      out[h * a.oh + to] = from_f32<T>(__fadd_rn(__fmul_rn(v, c[0]), __fmul_rn(u, s[0])));
    }
  }
}

template <typename T> int launch_rope(RopeArgs a, int layout, bool in_place, bool wide, gar_stream_t stream) {
  const bool inter = layout == GAR_ROPE_INTERLEAVED;
  const int v = wide ? chunk16<T>::N : 1;
  a.pair_units = inter && wide ? a.rot / v : a.rot / 2 / v;
  a.units = a.pair_units + (in_place ? 0 : (a.dim - a.rot) / v);
  // Eight heads to a thread once there are enough threads to fill the GPU without (16384 tokens x 40 heads x 128
  // bf16: 52 us with eight, 115 with one, 75 with two, 58 with four, 53 with sixteen, 61 with all; one token x 8
  // heads: 1.7 us with one, 2.0 with four).
  const int64_t all = a.tokens * a.heads * a.units;
  a.lanes = all > (int64_t)152 * 2048 * 4 ? (a.heads + 7) / 8 : a.heads;
  a.block_tokens = std::max(1, 256 / (a.lanes * a.units));
  const int64_t blocks = (a.tokens + a.block_tokens - 1) / a.block_tokens;
  if (blocks > 0x7fffffff) return refuse("too many tokens");
  const int threads = std::min(256, (a.block_tokens * a.lanes * a.units + 31) / 32 * 32);
  if (!wide) return launch("gar_rope", rope_narrow_kernel<T>, blocks, threads, 0, stream, a, inter);
  return launch("gar_rope", inter ? rope_kernel<T, true> : rope_kernel<T, false>, blocks, threads, 0, stream, a);
}

}  // namespace
}  // namespace gar

using namespace gar;

extern "C" {

int gar_rope_frequencies(int rot, double base, int scaling, double factor, double original, double *frequencies,
                         double *magnitude) {
  if (rot < 2 || rot > GAR_MAX_HEAD_DIM || rot % 2 || frequencies == nullptr || magnitude == nullptr)
    return refuse("rot must be even, 2..256, and the outputs not null");
  if (!(base > 1) || !std::isfinite(base)) return refuse("base must be a number above 1");
  if (scaling < GAR_ROPE_PLAIN || scaling > GAR_ROPE_PARTS) return refuse("unknown scaling");
  if (scaling != GAR_ROPE_PLAIN && (!(factor >= 1) || !std::isfinite(factor))) return refuse("factor must be a number of at least 1");
  if (scaling == GAR_ROPE_PARTS && !(original > 0)) return refuse("the original length must be positive");
  if (scaling == GAR_ROPE_BASE) {
    if (rot < 4) return refuse("a scaled base needs rot of at least 4");
    base *= std::pow(factor, (double)rot / (rot - 2));
  }
  for (int i = 0; i < rot / 2; ++i) {
    double f = std::pow(base, -2.0 * i / rot);
    if (scaling == GAR_ROPE_LINEAR) f /= factor;
    if (scaling == GAR_ROPE_PARTS) {
      const double turns = original * f / (2 * 3.14159265358979323846);
      const double keep = std::min(1.0, std::max(0.0, (turns - 1.0) / (32.0 - 1.0)));
      f = f * keep + f / factor * (1 - keep);
    }
    frequencies[i] = f;
  }
  *magnitude = scaling == GAR_ROPE_PARTS ? 0.1 * std::log(factor) + 1.0 : 1.0;
  return GAR_OK;
}

int gar_rope_table(float *table, int64_t first, int64_t count, int rot, const double *frequencies, double magnitude,
                   gar_stream_t stream) {
  if (rot < 2 || rot > GAR_MAX_HEAD_DIM || rot % 2) return refuse("rot must be even, 2..256");
  if (count < 0 || first < 0 || frequencies == nullptr || (count > 0 && table == nullptr))
    return refuse("negative count or first position, or a null pointer");
  if ((uintptr_t)table % 8) {
    set_error("the table must be 8-byte aligned");
    return GAR_EALIGN;
  }
  if (count == 0) return GAR_OK;
  Frequencies fr{};
  std::copy(frequencies, frequencies + rot / 2, fr.f);
  const int64_t blocks = std::min<int64_t>((count * (rot / 2) + 255) / 256, 152 * 64);
  return launch("gar_rope_table", rope_table_kernel, blocks, 256, 0, stream, reinterpret_cast<float2 *>(table), first, count,
                rot / 2, magnitude, fr);
}

int gar_rope(const void *x, int64_t x_token_stride, int64_t x_head_stride, void *out, int64_t out_token_stride,
             int64_t out_head_stride, int dtype, int64_t tokens, int heads, int dim, int rot, const void *positions,
             int position_bytes, const float *table, int64_t table_rows, int layout, int inverse,
             gar_stream_t stream) {
  if (!float_type(dtype)) return refuse("gar_rope takes GAR_F32, GAR_BF16 or GAR_F16");
  if (tokens < 0 || heads < 0 || dim < 1 || dim > GAR_MAX_HEAD_DIM) return refuse("bad tokens, heads or dim");
  if (heads > 1 << 20) return refuse("too many heads");
  if (rot < 2 || rot % 2 || rot > dim) return refuse("rot must be even, 2..dim");
  if (layout != GAR_ROPE_HALF && layout != GAR_ROPE_INTERLEAVED) return refuse("unknown layout");
  if (position_bytes != 4 && position_bytes != 8) return refuse("positions are 4 or 8 bytes wide");
  if (table_rows < 0) return refuse("negative table_rows");
  if (tokens == 0 || heads == 0) return GAR_OK;
  if (x == nullptr || out == nullptr || positions == nullptr || (table == nullptr && table_rows > 0))
    return refuse("null pointer");
  const int size = element_size(dtype);
  if ((uintptr_t)x % size || (uintptr_t)out % size || (uintptr_t)positions % position_bytes || (uintptr_t)table % 8) {
    set_error("a buffer is not aligned to its elements (the table to 8 bytes)");
    return GAR_EALIGN;
  }
  const bool in_place = x == out;
  if (in_place && (x_token_stride != out_token_stride || x_head_stride != out_head_stride))
    return refuse("in place needs equal strides");
  RopeArgs a{};
  a.x = x, a.out = out, a.xt = x_token_stride, a.xh = x_head_stride, a.ot = out_token_stride, a.oh = out_head_stride;
  a.tokens = tokens, a.positions = positions, a.table = reinterpret_cast<const float2 *>(table);
  a.table_rows = table_rows, a.heads = heads, a.dim = dim, a.rot = rot;
  a.wide_positions = position_bytes == 8, a.sign = inverse ? -1.f : 1.f;
  // The widest vector (16 bytes, else one element) that every address, half and remainder is a multiple of.
  const int v = 16 / size;
  const auto fits = [&](int64_t n) { return n % v == 0; };
  const bool wide = (uintptr_t)x % 16 == 0 && (uintptr_t)table % 16 == 0 && (uintptr_t)out % 16 == 0 &&
                    fits(x_token_stride) && fits(x_head_stride) && fits(out_token_stride) && fits(out_head_stride) &&
                    fits(dim) && fits(layout == GAR_ROPE_HALF ? rot / 2 : rot);
  return with_float(dtype, [&](auto tag) {
    using T = typename decltype(tag)::type;
    return launch_rope<T>(a, layout, in_place, wide, stream);
  });
}

}  // extern "C"
