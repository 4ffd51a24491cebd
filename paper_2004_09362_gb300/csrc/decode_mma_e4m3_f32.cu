// Decode attention on tensor cores: 32-bit queries over a cache of 8-bit codes.
#include <algorithm>

#include "decode_mma.cuh"

namespace gar {
int decode_mma_e4m3_f32(const DecodeArgs &a, int sms, gar_stream_t stream) { return decode_mma<e4m3, true>(a, sms, stream); }
}  // namespace gar
