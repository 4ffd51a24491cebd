// Decode attention on tensor cores: a cache of this type.
#include <algorithm>

#include "decode_mma.cuh"

namespace gar {
int decode_mma_e4m3(const DecodeArgs &a, int sms, gar_stream_t stream) { return decode_mma<e4m3, false>(a, sms, stream); }
}  // namespace gar
