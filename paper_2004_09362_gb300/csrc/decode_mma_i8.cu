// Decode attention on tensor cores: a cache of this type.
#include <algorithm>

#include "decode_mma.cuh"

namespace gar {
int decode_mma_i8(const DecodeArgs &a, int sms, gar_stream_t stream) { return decode_mma<i8, false>(a, sms, stream); }
}  // namespace gar
