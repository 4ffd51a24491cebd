// Decode attention on tensor cores: a cache of this type.
#include <algorithm>

#include "decode_mma.cuh"

namespace gar {
int decode_mma_bf16(const DecodeArgs &a, int sms, gar_stream_t stream) { return decode_mma<__nv_bfloat16, false>(a, sms, stream); }
}  // namespace gar
