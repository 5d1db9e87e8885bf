// The 8-bit cache: e4m3 conversions and MFMA operands (gfx950), launch interface.
//
// A page holds one chunk (64 tokens) of one sequence for every KV head:
//   k_pages  [P, Hkv, 64, d]  e4m3, key-major
//   v_pages  [P, Hkv, d, 64]  e4m3, dim-major: 16 keys of a dim are one 16-byte load and, as
//                             bf16, one row of the A operand of O^T = V^T P^T, so that values
//                             need no transposition through LDS
//   kv_scale [P, Hkv, 2]      f32: a stored x stands for x * scale (K's, V's)
//   lmk_pages [P, Hl, d]      e4m3 in units of the page's K scale: k'_c is a convex combination
//                             of the chunk's keys, so it fits in their range
//   bias_pages [P, Hl]        f32
// e4m3 values are exact in bf16 and float16 (4 significant bits, 2^-9 to 448), so products run on
// the 16-bit MFMAs with the other operand, queries or weights, as several terms of that type; the
// scales multiply float32 results.
#pragma once

#include "hils_device.hpp"
#include "hils_internal.hpp"
#include "hils_mfma.hpp"

namespace hils {

// Four e4m3 codes of a dword as a float each, and back (round to nearest, ties to even; |x|
// <= 448 or NaN).  The conversions agree with the format's table for all 256 codes.
__device__ __forceinline__ void e4m3_to_f32x4(uint32_t u, float* o) {
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(u, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(u, true);
    o[0] = a[0]; o[1] = a[1]; o[2] = b[0]; o[3] = b[1];
}
__device__ __forceinline__ uint32_t f32x4_to_e4m3(float a, float b, float c, float d) {
    const int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}

// Eight e4m3 codes as an MFMA operand (exact).
__device__ __forceinline__ bf16x8 bf16x8_of_e4m3(uint32_t lo, uint32_t hi) {
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// x as the sum of S bf16 values, largest first: S = 3 holds a float32 to its last bit
// (3 x 8 significant bits).
template <int S>
__device__ __forceinline__ void split_bf16x8(const float* x, bf16x8 (&o)[S]) {
    float r[8];
#pragma unroll
    for (int t = 0; t < 8; ++t) r[t] = x[t];
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            o[s][t] = static_cast<__bf16>(r[t]);
            r[t] -= (float)o[s][t];
        }
}

// Softmax weights (0 <= w <= 1) as operands: 4096 w as the sum of two float16 values, to 2^-23 of it, a
// float32's last bit, and to 2^-37 of 1 (below 2^-26 the terms are subnormal).  Two terms of bf16 hold
// 2^-17 of w, which shows where a sum cancels; three hold it whole for half as many products again.
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
constexpr float kWeightUnit = 1.f / 4096;
__device__ __forceinline__ f16x8 f16x8_of_e4m3(uint32_t lo, uint32_t hi) {
    typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
    const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false);
    const f16x2 b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true);
    const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false);
    const f16x2 d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true);
    return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
struct WeightOperand {
    f16x8 t[2];
    __device__ __forceinline__ explicit WeightOperand(const float* w) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
            const float x0 = w[i] * (1.f / kWeightUnit), x1 = w[i + 1] * (1.f / kWeightUnit);
            f16x2 h = {static_cast<_Float16>(x0), static_cast<_Float16>(x1)};
            asm("" : "+v"(h));  // (one conversion of both, not another of each for the difference)
            t[0][i] = h[0];
            t[0][i + 1] = h[1];
            t[1][i] = static_cast<_Float16>(x0 - (float)h[0]);
            t[1][i + 1] = static_cast<_Float16>(x1 - (float)h[1]);
        }
    }
};
// The sum of two products x w of e4m3 values and weights, in units of kWeightUnit, the smaller terms first.
__device__ __forceinline__ f32x4 mfma_weights(const f16x8& x0, const WeightOperand& w0, const f16x8& x1,
                                              const WeightOperand& w1) {
    f32x4 o = zero4();
#pragma unroll
    for (int t = 1; t >= 0; --t) {
        o = __builtin_amdgcn_mfma_f32_16x16x32_f16(x0, w0.t[t], o, 0, 0, 0);
        o = __builtin_amdgcn_mfma_f32_16x16x32_f16(x1, w1.t[t], o, 0, 0, 0);
    }
    return o;
}

// Eight consecutive elements of a caller's array, aligned as its elements are.
__device__ __forceinline__ bf16x8 load8_unaligned(const bf16* p) {
    bf16x8 r;
    __builtin_memcpy(&r, p, sizeof r);
    return r;
}
__device__ __forceinline__ void load8_unaligned(const float* p, float* o) { __builtin_memcpy(o, p, 8 * sizeof(float)); }

// A row of D query elements as MFMA operands against 16-byte loads of an e4m3 row: the lane
// group lg holds dims 64 j + 16 lg + 0..15 of the row, so operand ks = 2 j + t takes dims
// 64 j + 16 lg + 8 t + 0..7 (the contraction may run over the dims in any order).
template <typename T, int D>
struct QRow {
    static constexpr int S = sizeof(T) == 2 ? 1 : 3, KS = D / 32;
    bf16x8 x[KS][S];
    __device__ __forceinline__ void load(const T* row, int lg, bool valid) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const T* src = row + (ks / 2) * 64 + lg * 16 + (ks % 2) * 8;
            if constexpr (sizeof(T) == 2) {
                const bf16x8 y = load8_unaligned(src);
                x[ks][0] = valid ? y : as_bf16x8(make_uint4(0, 0, 0, 0));
            } else {
                float y[8];
                load8_unaligned(src, y);
#pragma unroll
                for (int t = 0; t < 8; ++t) y[t] = valid ? y[t] : 0.f;
                split_bf16x8<S>(y, x[ks]);
            }
        }
    }
};

// D += A B over one e4m3 row piece per lane (16 rows x D), the smallest terms first.
template <typename T, int D>
__device__ __forceinline__ f32x4 mfma_row(const uint4 (&a)[D / 64], const QRow<T, D>& q, f32x4 acc) {
#pragma unroll
    for (int j = 0; j < D / 64; ++j) {
        const bf16x8 a0 = bf16x8_of_e4m3(a[j].x, a[j].y), a1 = bf16x8_of_e4m3(a[j].z, a[j].w);
#pragma unroll
        for (int s = QRow<T, D>::S - 1; s >= 0; --s) {
            acc = mfma16x16x32(a0, q.x[2 * j][s], acc);
            acc = mfma16x16x32(a1, q.x[2 * j + 1][s], acc);
        }
    }
    return acc;
}

// Tokens of sequence b and how many of them are new (at most N of the last ones).
template <typename A>
__device__ __forceinline__ int q8_tokens(const A& a, int b, int& fresh) {
    int len = a.seqlens ? a.seqlens[b] : a.L;
    len = len < 0 ? 0 : (len > a.L ? a.L : len);
    int n = a.newlens ? a.newlens[b] : a.N;
    n = n < 0 ? 0 : (n > a.N ? a.N : n);
    fresh = n > len ? len : n;
    return len;
}

}  // namespace hils
