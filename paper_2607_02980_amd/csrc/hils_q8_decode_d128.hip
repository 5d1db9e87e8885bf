// Decode over the 8-bit cache, head dim 128 (kernels and dispatch: hils_q8_decode.hpp), and the
// host side of both head dims.
#include "hils_q8_decode.hpp"

namespace hils {

hipError_t launch_q8_decode_d128(const Q8DecodeArgs& a, hipStream_t s) { return dispatch_q8_decode<128>(a, s); }

size_t q8_decode_workspace_bytes(int B, int N, int Hkv, int G, int d, int L, int K, int W) {
    return q8_layout(B, N, Hkv, G, d, L, K, W, false).total;
}

hipError_t launch_q8_decode(const Q8DecodeArgs& a, hipStream_t s) {
    if (a.f.d == 64) return launch_q8_decode_d64(a, s);
    if (a.f.d == 128) return launch_q8_decode_d128(a, s);
    return hipErrorInvalidValue;
}

}  // namespace hils
