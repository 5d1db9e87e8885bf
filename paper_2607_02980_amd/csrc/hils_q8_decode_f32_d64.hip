// Decode over the 8-bit cache, f32 queries, head dim 64 (kernels and dispatch: hils_q8_decode.hpp).
#include "hils_q8_decode.hpp"

namespace hils {
hipError_t launch_q8_decode_f32_d64(const Q8DecodeArgs& a, hipStream_t s) { return dispatch_q8_decode<float, 64>(a, s); }
}  // namespace hils
