// Writing the 8-bit cache (gfx950): new tokens' keys and values, and the landmark rows of the
// chunks that they complete.  Layout of the cache: hils_q8.hpp.
#include <type_traits>

#include "hils_dispatch.hpp"
#include "hils_q8.hpp"

namespace hils {

namespace {

constexpr int kBlock = 256;
constexpr int kWaves = kBlock / kWave;

// Smallest e >= -100 with amax <= 448 * 2^e, from the float's exponent and whether its
// significand is above 448 / 256; 2^e and 2^-e are then normal floats for every finite amax.
__device__ __forceinline__ float scale_for(float amax) {
    const uint32_t u = __float_as_uint(amax);
    const int ex = (int)(u >> 23) - 127;
    int e = (u & 0x7fffffu) > 0x600000u ? ex - 7 : ex - 8;
    e = e < -100 ? -100 : e;
    return __uint_as_float((uint32_t)(e + 127) << 23);
}
__device__ __forceinline__ float finite_abs(float x) { return fabsf(x) < INFINITY ? fabsf(x) : 0.f; }
// W / 2 (or W) neighbouring elements as they lie in memory, in W words.
template <typename T, int W>
struct Raw {
    uint32_t u[W];
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(u[i]);
        else return __uint_as_float(i & 1 ? u[i / 2] & 0xffff0000u : u[i / 2] << 16);
    }
};
template <typename T>
using Pair = Raw<T, sizeof(T) / 2>;
template <typename T>
using Oct = Raw<T, 2 * sizeof(T)>;
// (elements that are read once: not kept in the caches; of the alignment of bf16 elements at least)
template <typename R, typename T>
__device__ __forceinline__ R load_stream(const T* p) {
    R r;
    if constexpr (sizeof(R) == 4) {
        typedef uint32_t u32 __attribute__((aligned(2)));
        r.u[0] = __builtin_nontemporal_load(reinterpret_cast<const u32*>(p));
    } else if constexpr (sizeof(R) == 8) {
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2), aligned(2)));
        const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p));
        r.u[0] = x[0];
        r.u[1] = x[1];
    } else {
        typedef uint32_t u32x4 __attribute__((ext_vector_type(4), aligned(2)));
#pragma unroll
        for (int i = 0; i < (int)sizeof(R) / 16; ++i) {
            const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p) + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) r.u[4 * i + e] = x[e];
        }
    }
    return r;
}

// ---- new tokens ------------------------------------------------------------------
//
// One wave per (sequence, chunk that gets tokens, KV head, K or V).  With a the largest finite
// magnitude among the chunk's new rows, s = scale_for(a), or the scale the chunk has if it
// holds older tokens and that one is larger; new x -> e4m3(x / s).  Where s grew, older codes
// y -> e4m3(y * s_old / s): powers of two, so exact unless the result falls below e4m3's
// normal range.  Infinities, which e4m3 lacks, become NaN, as the conversion makes them.  Bytes of
// rows at or past the sequence's end are left as they were; tokens of a chunk without a page
// (a table entry outside the pool) are dropped.
//
// Bound by memory: 2 (es + 1) d bytes per token and head.  A whole chunk's values stay in
// registers, as they came, between the maximum and the conversion: of K 8 neighbouring dims per
// lane and load; of V two dims of all rows (d = 64: of half the rows) per lane, so that a
// dim-major row of 64 keys is 64 contiguous bytes of one lane.  (65536 tokens of 8 heads, d = 128:
// 75 to 80 us, 5.0 to 5.4 TB/s where a copy of 1 GiB takes 4.8; K by two dims per lane and kept as floats 86.)
template <typename T, int D>
__global__ __launch_bounds__(kBlock) void k_q8_append(Q8AppendArgs a, int most) {
    constexpr int LPR = D / 2, TH = kWave / LPR, ROWS = kChunk / TH;  // lanes per row, row groups, rows per lane
    const int lane = threadIdx.x % kWave, dd = (lane % LPR) * 2, th = lane / LPR;
    // unit: (sequence, head, chunk, K or V), the last fastest
    const long unit = (long)blockIdx.x * kWaves + wave_id();
    const int which = unit & 1;
    long u = unit >> 1;
    const int j = (int)(u % most);
    u /= most;
    const int g = (int)(u % a.Hkv), b = (int)(u / a.Hkv);
    if (b >= a.B) return;
    int fresh;
    const int len = q8_tokens(a, b, fresh), start = len - fresh;
    const int c = start / kChunk + j;
    const int r0 = j == 0 ? start % kChunk : 0, r1 = min(kChunk, len - c * kChunk);  // the chunk's new rows
    if (fresh == 0 || r1 <= r0) return;
    const int entry = a.block_table[(size_t)b * (a.L / kChunk) + c];
    if (entry < 0 || entry >= a.num_pages) return;  // (no page: another sequence's stays as it is)
    const size_t page = entry;
    const size_t pg = page * a.Hkv + g;
    uint8_t* dst = static_cast<uint8_t*>(which ? a.v_pages : a.k_pages) + pg * kChunk * D;
    float* scale = a.kv_scale + pg * 2 + which;
    // row r of the chunk is new token c * 64 + r - start
    const T* src = as<T>(which ? a.v_new : a.k_new) + ((size_t)b * a.Hkv + g) * a.N * D +
                   ((long)c * kChunk - start) * D + dd;
    if (r0 == 0 && r1 == kChunk) {  // a whole chunk, in registers as it came
        float m = 0.f;
        if (which) {
            Pair<T> x[ROWS];
#pragma unroll
            for (int r = 0; r < ROWS; ++r) x[r] = load_stream<Pair<T>>(src + (size_t)(th * ROWS + r) * D);
#pragma unroll
            for (int r = 0; r < ROWS; ++r) m = fmaxf(m, fmaxf(finite_abs(x[r].get(0)), finite_abs(x[r].get(1))));
            const float s = scale_for(wave_max(m)), inv = 1.f / s;
            if (lane == 0) *scale = s;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < ROWS; r += 16) {
                    uint32_t w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const Pair<T>* y = x + r + 4 * i;
                        w[i] = f32x4_to_e4m3(y[0].get(t) * inv, y[1].get(t) * inv, y[2].get(t) * inv, y[3].get(t) * inv);
                    }
                    *reinterpret_cast<uint4*>(dst + (dd + t) * kChunk + th * ROWS + r) =
                        make_uint4(w[0], w[1], w[2], w[3]);
                }
        } else {  // K: 8 neighbouring dims of a row per lane and load
            constexpr int LP8 = D / 8, RPL = kWave / LP8, NL = kChunk / RPL;
            const T* src8 = src - dd + (size_t)(lane / LP8) * D + lane % LP8 * 8;
            Oct<T> x[NL];
#pragma unroll
            for (int i = 0; i < NL; ++i) x[i] = load_stream<Oct<T>>(src8 + (size_t)i * RPL * D);
#pragma unroll
            for (int i = 0; i < NL; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) m = fmaxf(m, finite_abs(x[i].get(e)));
            const float s = scale_for(wave_max(m)), inv = 1.f / s;
            if (lane == 0) *scale = s;
#pragma unroll
            for (int i = 0; i < NL; ++i)
                *reinterpret_cast<uint2*>(dst + (i * RPL + lane / LP8) * D + lane % LP8 * 8) = make_uint2(
                    f32x4_to_e4m3(x[i].get(0) * inv, x[i].get(1) * inv, x[i].get(2) * inv, x[i].get(3) * inv),
                    f32x4_to_e4m3(x[i].get(4) * inv, x[i].get(5) * inv, x[i].get(6) * inv, x[i].get(7) * inv));
        }
        return;
    }
    // Part of a chunk, NB row steps of TH rows at a time (rows past the last one are the last one again).
    auto partial = [&](auto nb_tag) {
        constexpr int NB = decltype(nb_tag)::value;
        Pair<T> x[NB];
        auto row_at = [&](int base, int i) { return r0 + base + i * TH + th; };
        auto load = [&](int base) {
#pragma unroll
            for (int i = 0; i < NB; ++i) x[i] = load_stream<Pair<T>>(src + (long)min(row_at(base, i), r1 - 1) * D);
        };
        float m = 0.f;
        for (int base = 0; base < r1 - r0; base += NB * TH) {
            load(base);
#pragma unroll
            for (int i = 0; i < NB; ++i) m = fmaxf(m, fmaxf(finite_abs(x[i].get(0)), finite_abs(x[i].get(1))));
        }
        float s = scale_for(wave_max(m));
        if (r0 > 0) {
            const float old = *scale;
            s = fmaxf(s, old);
            if (s != old) {  // the older codes at the new scale
                const float f = old / s;
                auto moved = [&](uint32_t w) {
                    float y[4];
                    e4m3_to_f32x4(w, y);
                    return f32x4_to_e4m3(y[0] * f, y[1] * f, y[2] * f, y[3] * f);
                };
                if (which) {
                    const int quads = (r0 + 3) / 4;  // dwords of a dim's row with older keys
                    for (int e = lane; e < quads * D; e += kWave) {
                        uint32_t* w = reinterpret_cast<uint32_t*>(dst + (e % D) * kChunk) + e / D;
                        const int n = r0 - e / D * 4;
                        const uint32_t keep = n >= 4 ? 0xffffffffu : (1u << (8 * n)) - 1u, was = *w;
                        *w = (moved(was) & keep) | (was & ~keep);
                    }
                } else {
                    uint32_t* w = reinterpret_cast<uint32_t*>(dst);
                    for (int e = lane; e < r0 * D / 4; e += kWave) w[e] = moved(w[e]);
                }
                // the new keys' bytes may share a dword with the older ones'
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            }
        }
        if (lane == 0) *scale = s;
        const float inv = 1.f / s;
        for (int base = 0; base < r1 - r0; base += NB * TH) {
            if (r1 - r0 > NB * TH) load(base);  // (otherwise they are still there)
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const int r = row_at(base, i);
                if (r >= r1) continue;
                const uint32_t w = f32x4_to_e4m3(x[i].get(0) * inv, x[i].get(1) * inv, 0.f, 0.f);
                if (which) {
                    dst[dd * kChunk + r] = (uint8_t)w;
                    dst[(dd + 1) * kChunk + r] = (uint8_t)(w >> 8);
                } else {
                    *reinterpret_cast<uint16_t*>(dst + r * D + dd) = (uint16_t)w;
                }
            }
        }
    };
    if (r1 - r0 <= TH) partial(std::integral_constant<int, 1>{});  // a decode step's one token
    else partial(std::integral_constant<int, 16>{});
}

// ---- landmark rows -----------------------------------------------------------------
//
// Prop. 3.1 on the stored keys k_j = x_j ks: one wave per (sequence, completed chunk, KV head),
// the group's GL landmark heads as MFMA columns: S^T = K Q'^T from K rows as they lie in the
// page, the softmax over the lane groups, b' = log l - sum_j p_j s_j (s from its maximum), and
// k' / ks = X^T P^T with X^T by transposing reads of the rows, as float16, in the wave's LDS tile
// and P in two float16 terms (512 chunks of 32 heads 12.3 us; in two bf16 terms, 2^-17 of it, 11.8,
// in three 12.5).  Bound by memory: 64 d + GL (d + 4) bytes per wave.  (Products with P on the vector unit, key by key from LDS: 512
// chunks of 32 heads 18 us, 24 chunks 12 us.)
template <int D>
struct LmkTile {
    static constexpr int ROW = D + 16;  // (transposing reads of padded rows meet two addresses per bank)
    _Float16 x[kChunk * ROW];
};
template <typename T, int D, int GL>
__global__ __launch_bounds__(kBlock) void k_q8_landmark(Q8LandmarkArgs a, int most) {
    constexpr int DJ = D / 64, DB = D / 16, ROW = LmkTile<D>::ROW;
    __shared__ __align__(16) LmkTile<D> tiles[kWaves];
    _Float16* tile = tiles[wave_id()].x;
    const int lane = threadIdx.x % kWave, lg = lane / 16, n16 = lane % 16;
    const long unit = (long)blockIdx.x * kWaves + wave_id();
    const int g = (int)(unit % a.Hkv);
    const int j = (int)(unit / a.Hkv % most), b = (int)(unit / a.Hkv / most);
    if (b >= a.B) return;
    int fresh;
    const int len = q8_tokens(a, b, fresh);
    const int c = (len - fresh) / kChunk + j;
    if (c >= len / kChunk) return;
    const int entry = a.block_table[(size_t)b * (a.L / kChunk) + c];
    if (entry < 0 || entry >= a.num_pages) return;  // (no page: another sequence's stays as it is)
    const size_t page = entry;
    const uint8_t* kp = static_cast<const uint8_t*>(a.k_pages) + (page * a.Hkv + g) * kChunk * D;
    const int hl0 = g * GL;
    QRow<T, D> q;
    {
        const int hl = hl0 + min(n16, GL - 1);
        const size_t row = a.shared ? hl : ((size_t)b * a.Hl + hl) * most + j;
        q.load(as<T>(a.lq) + row * D, lg, n16 < GL);
    }
    uint4 kx[4][DJ];
#pragma unroll
    for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int t = 0; t < DJ; ++t)
            kx[kb][t] = *reinterpret_cast<const uint4*>(kp + (kb * 16 + n16) * D + t * 64 + lg * 16);
    const float c1 = a.scale * a.kv_scale[(page * a.Hkv + g) * 2];
    // S^T (lane: head n16, keys 16 kb + 4 lg + i)
    float s[16], mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
        f32x4 st = zero4();
#pragma unroll
        for (int t = 0; t < DJ; ++t) {
            const bf16x8 k0 = bf16x8_of_e4m3(kx[kb][t].x, kx[kb][t].y), k1 = bf16x8_of_e4m3(kx[kb][t].z, kx[kb][t].w);
            _Float16* dst = tile + (kb * 16 + n16) * ROW + t * 64 + lg * 16;
            *reinterpret_cast<f16x8*>(dst) = f16x8_of_e4m3(kx[kb][t].x, kx[kb][t].y);
            *reinterpret_cast<f16x8*>(dst + 8) = f16x8_of_e4m3(kx[kb][t].z, kx[kb][t].w);
#pragma unroll
            for (int r = QRow<T, D>::S - 1; r >= 0; --r) {
                st = mfma16x16x32(k0, q.x[2 * t][r], st);
                st = mfma16x16x32(k1, q.x[2 * t + 1][r], st);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[kb * 4 + i] = st[i] * c1;
            mx = fmaxf(mx, s[kb * 4 + i]);
        }
    }
    mx = group4_max(mx);
    float l = 0.f, ps = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float t = s[i] - mx;
        s[i] = fexp2(t * kLog2e);
        l += s[i];
        ps += s[i] * t;
    }
    l = group4_sum(l);
    ps = group4_sum(ps);
    const float inv = 1.f / l;
    if (n16 < GL && lg == 0) a.bias_pages[page * a.Hl + hl0 + n16] = logf(l) - ps * inv;
    const WeightOperand p0(s), p1(s + 8);
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    // (lane: head n16, dims 16 db + 4 lg + i; a convex combination of codes: above 448 by the
    // sum's rounding at most, which rounds back to it)
    f32x4 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) {
        const f16x8 x0 = __builtin_bit_cast(f16x8, tr_operand_perm(tile, ROW, 0, db * 16, lane));
        const f16x8 x1 = __builtin_bit_cast(f16x8, tr_operand_perm(tile, ROW, 32, db * 16, lane));
        o[db] = mfma_weights(x0, p0, x1, p1) * kWeightUnit;
    }
    if (n16 < GL) {
        uint8_t* dst = static_cast<uint8_t*>(a.lmk_pages) + (page * a.Hl + hl0 + n16) * D + lg * 4;
#pragma unroll
        for (int db = 0; db < DB; ++db)
            *reinterpret_cast<uint32_t*>(dst + db * 16) =
                f32x4_to_e4m3(o[db][0] * inv, o[db][1] * inv, o[db][2] * inv, o[db][3] * inv);
    }
}

}  // namespace

hipError_t launch_q8_append(const Q8AppendArgs& a, hipStream_t s) {
    const int most = (a.N + 62) / kChunk + 1;  // chunks that N tokens reach into
    const long waves = (long)a.B * a.Hkv * most * 2;
    const dim3 grid((unsigned)((waves + kWaves - 1) / kWaves)), block(kBlock);
    if (a.bf16) {
        if (a.d == 64) HILS_LAUNCH("k_q8_append", (k_q8_append<bf16, 64>), grid, block, 0, s, a, most);
        else HILS_LAUNCH("k_q8_append", (k_q8_append<bf16, 128>), grid, block, 0, s, a, most);
    } else {
        if (a.d == 64) HILS_LAUNCH("k_q8_append", (k_q8_append<float, 64>), grid, block, 0, s, a, most);
        else HILS_LAUNCH("k_q8_append", (k_q8_append<float, 128>), grid, block, 0, s, a, most);
    }
    return hipGetLastError();
}

namespace {
struct Q8LandmarkRun {
    template <typename T, int D, int G>
    static hipError_t run(const Q8LandmarkArgs& a, hipStream_t s) {
        const int most = (a.N + kChunk - 1) / kChunk;  // chunks that N tokens complete, at most
        const long waves = (long)a.B * a.Hkv * most;
        const dim3 grid((unsigned)((waves + kWaves - 1) / kWaves)), block(kBlock);
        if (a.Hl == a.Hkv)
            HILS_LAUNCH("k_q8_landmark", (k_q8_landmark<T, D, 1>), grid, block, 0, s, a, most);
        else
            HILS_LAUNCH("k_q8_landmark", (k_q8_landmark<T, D, G>), grid, block, 0, s, a, most);
        return hipGetLastError();
    }
};
}  // namespace

hipError_t launch_q8_landmark(const Q8LandmarkArgs& a, hipStream_t s) {
    return dispatch<Q8LandmarkRun>(a.bf16, a.d, a.G, a, s);
}

}  // namespace hils
