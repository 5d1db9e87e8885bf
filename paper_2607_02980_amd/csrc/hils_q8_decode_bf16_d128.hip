// Decode over the 8-bit cache, bf16 queries, head dim 128 (kernels and dispatch: hils_q8_decode.hpp).
#include "hils_q8_decode.hpp"

namespace hils {
hipError_t launch_q8_decode_bf16_d128(const Q8DecodeArgs& a, hipStream_t s) { return dispatch_q8_decode<bf16, 128>(a, s); }
}  // namespace hils
