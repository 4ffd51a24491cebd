// Attention of batches that share rows, on tensor cores: a cache of this type.
#include <algorithm>

#include "decode_mma.cuh"

namespace gar {
int decode_mma_f32(const ServingArgs &a, int sms, gar_stream_t stream) { return decode_mma<float, true>(a, sms, stream); }
}  // namespace gar
