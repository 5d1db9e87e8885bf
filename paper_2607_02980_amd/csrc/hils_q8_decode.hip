// Host side of the decode over the 8-bit cache: workspace size and dispatch over the storage
// type and the head dim.
#include "hils_q8_decode.hpp"

namespace hils {

size_t q8_decode_workspace_bytes(int B, int N, int Hkv, int G, int d, int L, int K, int W) {
    return q8_layout(B, N, Hkv, G, d, L, K, W, false).total;  // (the same with shared landmarks)
}

hipError_t launch_q8_decode(const Q8DecodeArgs& a, hipStream_t s) {
    if (a.f.d == 64) return a.f.bf16 ? launch_q8_decode_bf16_d64(a, s) : launch_q8_decode_f32_d64(a, s);
    if (a.f.d == 128) return a.f.bf16 ? launch_q8_decode_bf16_d128(a, s) : launch_q8_decode_f32_d128(a, s);
    return hipErrorInvalidValue;
}

}  // namespace hils
