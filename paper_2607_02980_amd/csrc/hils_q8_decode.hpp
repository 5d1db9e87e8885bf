// HiLS attention decode over the 8-bit cache (layout: hils_q8.hpp), gfx950; compiled once per
// storage type and head dim.  N >= 1 new queries per sequence, each a row (b, g, n) of its own position.
//
//   A  k_q8_scan     a workgroup per (slice of candidate chunks, KV group, query group): s^ for the
//                    group's heads, max over heads, the slice's top-K
//   B  k_q8_row      one or more workgroups per row: top-K over the slices' survivors -> idx; the
//                    intra-chunk softmax of the selected chunks and the pieces of the window,
//                    their fusion -> out, lse and each part's weight
//
// Memory-bound: a row reads G d bytes of landmarks per candidate (one head's: d) and 128 d per
// part.  S^T = K Q^T leaves lane group lg with keys 16 lg + 0..15 when key 16 a + 4 kb + i is row
// 4 a + i of block kb, and V^T's 16-byte pieces hold those keys: P^T goes from the accumulators
// into O^T = V^T P^T without leaving its lane, and nothing of a part passes through LDS.
// (Several new queries of a sequence are rows of their own: their windows meet in an XCD's L2,
// which all rows of a KV group share with Hkv a multiple of 8, and a value behind a query never
// meets its products.  One tile for the window of 4 queries, 8 sequences of 64K: parts and fusion 25 us, now 21.)
#pragma once

#include "hils_decode.hpp"
#include "hils_q8.hpp"

namespace hils {

namespace {

// Workgroups that may share a row, and rows (b, g, n) up to which they do.
constexpr int kQ8MaxSplit = 8, kQ8SplitRows = 128;

// Floats of a shared row's records: {M, Z, -, -, numerator[d]} per workgroup and head, then z of
// each part and head.  The first record's last header word is the row's arrival counter.
__host__ __device__ __forceinline__ int q8_row_floats(int nparts, int G, int d) {
    return kQ8MaxSplit * G * (4 + d) + (nparts * G + 3) / 4 * 4;
}

// Workspace: the slices' survivors (as in dec_layout), then the records.  Room for the finest
// slices and for every shared row, so that the size never falls as a call grows.
inline DecLayout q8_layout(int B, int N, int Hkv, int G, int d, int L, int K, int W, bool shared) {
    DecLayout o = {};
    o.nC = L / kChunk;
    o.nlocal = local_pieces_max(W);
    o.nparts = K + o.nlocal;
    const size_t rows = (size_t)B * N * Hkv;
    // slices of 256 chunks, halved while fewer than four workgroups per CU would scan (two where the
    // group shares its landmarks and a slice is a quarter of the bytes) and a row's survivors stay
    // within one selection of a wave (steps with 256, 512, 1024 and 2048 workgroups: 8 sequences of
    // 64K 23.0, 22.3, 21.8 and 21.7 us, 16 of 64K and 4 new tokens 59.3, 59.2, 58.1 and 56.7, 48 of
    // 30K 58.7, 58.5, 56.2 and 58.2; 24 of 60K, shared landmarks, 30.8, 29.8, 31.3 and 33.4)
    o.slice = kSlice;
    const long sgroups = (long)B * ((N + 3) / 4) * Hkv, full = shared ? 512 : 1024;
    while (o.slice > 64 && sgroups * ((o.nC + o.slice - 1) / o.slice) < full &&
           (o.nC + o.slice / 2 - 1) / (o.slice / 2) * K <= 4 * kWave)
        o.slice /= 2;
    o.nslices = (o.nC + o.slice - 1) / o.slice;
    o.cand = 0;
    o.parts = align256(rows * ((o.nC + 63) / 64) * K * 8);
    o.total = o.parts + align256(std::min(rows, (size_t)kQ8SplitRows) * q8_row_floats(o.nparts, G, d) * 4);
    return o;
}

__device__ __forceinline__ float* q8_record(const FwdArgs& a, const DecLayout& ly, size_t rg, int G, int d) {
    return reinterpret_cast<float*>(static_cast<char*>(a.ws) + ly.parts) + rg * q8_row_floats(ly.nparts, G, d);
}

// New queries whose scores a scan workgroup takes from one read of the landmarks.
template <int G>
constexpr int scan_queries(bool many) {
    return !many ? 1 : (G == 8 ? 2 : 4);
}

template <int G, int NQ>
struct __align__(16) Q8ScanSmem {
    float score[NQ][G][kSlice];
    float sig[NQ][kSlice];
    float osc[NQ][64], tsc[NQ][64];
    int page[kSlice];
    int oid[NQ][64], tid[NQ][64];
};

// One query, landmarks per head: plain products of 64 rows (scales and biases come later).  D / 16
// lanes read a row, so that a load covers whole 128-byte lines, non-temporal because a step reads
// each line once.  (32 sequences of 131K: 48 us, 5.6 TB/s of landmarks; as MFMA operands, half a
// row per load and lane group, 62, and 83 non-temporal, every line fetched twice; the next 64 rows
// loaded ahead, 54.)
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
template <typename T, int D>
struct ScanRows {
    static constexpr int LPR = D / 16, RPL = kWave / LPR, NL = 64 / RPL;  // lanes per row, rows per load, loads
    static constexpr int S = sizeof(T) == 2 ? 1 : 3;                      // bf16 terms of a query element
    static_assert(NL == LPR, "a row's lanes end with one row each");
    uint4 x[NL];
    __device__ __forceinline__ void load(const uint8_t* lmk, const int* page, int r0, int len, int Hl, int hl, int lane) {
#pragma unroll
        for (int i = 0; i < NL; ++i)
            x[i] = ld_stream16(lmk + ((size_t)page[min(r0 + i * RPL + lane / LPR, len - 1)] * Hl + hl) * D +
                               lane % LPR * 16);
    }
    // The lane's 16 products are the diagonal of a 4 x 4 block of v_mfma_f32_4x4x4_16b (lane l: row and
    // column l % 4 of block l / 4), half the vector instructions of multiplying them there; the
    // sums over a row's lanes halve the rows that a lane still carries each time, down to one.
    __device__ __forceinline__ void dot(const bf16x4 (&q)[S][4], float* score, int lane) const {
        float part[NL];
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const bf16x8 lo = bf16x8_of_e4m3(x[i].x, x[i].y), hi = bf16x8_of_e4m3(x[i].z, x[i].w);
            const bf16x4 a[4] = {bf16x4{lo[0], lo[1], lo[2], lo[3]}, bf16x4{lo[4], lo[5], lo[6], lo[7]},
                                 bf16x4{hi[0], hi[1], hi[2], hi[3]}, bf16x4{hi[4], hi[5], hi[6], hi[7]}};
            f32x4 d = zero4();
#pragma unroll
            for (int s = S - 1; s >= 0; --s)
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    d = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(__builtin_bit_cast(v4i16, a[t]),
                                                               __builtin_bit_cast(v4i16, q[s][t]), d, 0, 0, 0);
            const float e0 = lane & 1 ? d[1] : d[0], e1 = lane & 1 ? d[3] : d[2];
            part[i] = lane & 2 ? e1 : e0;
        }
        int row = lane / LPR;  // of the load that the lane ends with: load number times RPL more
        if constexpr (NL == 8) {
            const bool up = lane & 4;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float keep = up ? part[i + 4] : part[i], send = up ? part[i] : part[i + 4];
                part[i] = keep + dpp<0x141>(send);  // the other quad of the 8 lanes, mirrored
            }
            row += up ? 4 * RPL : 0;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float keep = lane & 2 ? part[i + 2] : part[i], send = lane & 2 ? part[i] : part[i + 2];
            part[i] = keep + dpp<0x4E>(send);  // lane ^ 2
        }
        const float keep = lane & 1 ? part[1] : part[0], send = lane & 1 ? part[0] : part[1];
        row += (lane & 2 ? 2 * RPL : 0) + (lane & 1 ? RPL : 0);
        score[row] = keep + dpp<0xB1>(send);  // lane ^ 1
    }
    // the lane's piece of a query
    static __device__ __forceinline__ void load_q(const T* src, bf16x4 (&q)[S][4]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            bf16x8 y[S];
            if constexpr (S == 1) {
                y[0] = load8_unaligned(src + h * 8);
            } else {
                float f[8];
                load8_unaligned(src + h * 8, f);
                split_bf16x8<S>(f, y);
            }
#pragma unroll
            for (int s = 0; s < S; ++s) {
                q[s][2 * h] = bf16x4{y[s][0], y[s][1], y[s][2], y[s][3]};
                q[s][2 * h + 1] = bf16x4{y[s][4], y[s][5], y[s][6], y[s][7]};
            }
        }
    }
};

// Several queries, or landmarks shared by the group: 64 rows as 4 MFMA tiles against a column per
// query or (query, head).  (On the vector unit a product per query and element: 4 queries, 8
// sequences of 64K, 2 us more.)
template <int D>
struct LmkBlock {
    uint4 x[4][D / 64];
    __device__ __forceinline__ void load(const uint8_t* lmk, const int* page, int r0, int len, int Hl, int hl, int lg,
                                         int n16) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const uint8_t* src = lmk + ((size_t)page[min(r0 + t * 16 + n16, len - 1)] * Hl + hl) * D + lg * 16;
#pragma unroll
            for (int j = 0; j < D / 64; ++j) x[t][j] = *reinterpret_cast<const uint4*>(src + j * 64);
        }
    }
};

template <typename T, int D, int G, int NQ>
__global__ __launch_bounds__(kBlock) void k_q8_scan(Q8DecodeArgs qa, DecLayout ly, int counters) {
    const FwdArgs& a = qa.f;
    const int ngrp = (a.N + NQ - 1) / NQ;
    // (slice, query group) pairs are dealt to the XCDs (block x runs on XCD x mod 8), a pair's KV
    // groups one after the other on one: a page's scales of all heads are one line, its
    // landmarks 4 KB in one place (slices fastest: scan of 32 sequences of 131K 74 us against 59)
    const int xcd = blockIdx.x % 8, seq = blockIdx.x / 8, g = seq % a.Hkv, pair = seq / a.Hkv * 8 + xcd;
    const int slice = pair % ly.nslices, bz = pair / ly.nslices;
    const int b = bz / ngrp, n0 = (bz % ngrp) * NQ;
    if (b >= a.B) return;
    const int nq = min(NQ, a.N - n0);
    __shared__ Q8ScanSmem<G, NQ> ss;
    const int tid = threadIdx.x, wave = wave_id(), lane = tid % kWave, lg = lane / 16, n16 = lane % 16;
    const int c0 = slice * ly.slice;
    float* cand_sc = reinterpret_cast<float*>(static_cast<char*>(a.ws) + ly.cand);
    int* cand_id = reinterpret_cast<int*>(cand_sc + (size_t)a.B * a.N * a.Hkv * ly.nslices * a.K);
    auto row_of = [&](int q) { return ((size_t)b * a.Hkv + g) * a.N + n0 + q; };
    auto len_of = [&](int q) {
        return q < nq ? max(0, min(ly.slice, n_candidates(decode_position(a, b, n0 + q), a.W) - c0)) : 0;
    };
    auto clear_counters = [&]() {
        if (counters && slice == 0 && tid < nq) *reinterpret_cast<int*>(q8_record(a, ly, row_of(tid), G, D) + 3) = 0;
    };
    int len = 0;
#pragma unroll
    for (int q = 0; q < NQ; ++q) len = max(len, len_of(q));
    for (int q = 0; q < nq; ++q) {
        if (len_of(q) > 0) continue;
        const size_t cbase = (row_of(q) * ly.nslices + slice) * a.K;
        for (int t = tid; t < a.K; t += kBlock) {
            cand_sc[cbase + t] = -INFINITY;
            cand_id[cbase + t] = -1;
        }
    }
    if (len <= 0) {
        clear_counters();
        return;
    }
    // thread r: chunk c0 + r's page, and what its score needs besides the products
    const bool shared = a.Hl != a.Hq;
    float ks = 0.f, bias[G];
#pragma unroll
    for (int h = 0; h < G; ++h) bias[h] = 0.f;
    int page = 0;
    if (tid < len) {
        page = page_of(a, ly.nC, b, c0 + tid);
        ss.page[tid] = page;
    }
    __syncthreads();
    if (tid < len) {
        ks = qa.kv_scale[((size_t)page * a.Hkv + g) * 2];
        if (a.bias) {
#pragma unroll
            for (int h = 0; h < G; ++h) bias[h] = a.bias[(size_t)page * a.Hl + (shared ? g : g * G + h)];
        }
    }
    const uint8_t* lmk = static_cast<const uint8_t*>(a.lmk);
    const T* qsrc = as<T>(a.q_route ? a.q_route : a.q);
    const int nblk = (len + 63) / 64, gl = shared ? 1 : G;  // blocks of 64 chunks; landmark heads of the group
    // units of (head, block): wave, wave + 4, ..., the head fastest, so that with four heads or more
    // a wave keeps its queries
    const int nunits = gl * nblk;
    auto head_of = [&](int u) { return shared ? 0 : u % G; };
    auto row_at = [&](int u) { return (shared ? u : u / G) * 64; };
    if (NQ == 1 && !shared) {
        using Rows = ScanRows<T, D>;
        const int seg = lane % Rows::LPR;
        if (wave < nunits) {
            Rows cur;
            bf16x4 q[Rows::S][4];
            int qh = -1;
            for (int u = wave; u < nunits; u += kBlock / kWave) {
                const int hh = head_of(u);
                cur.load(lmk, ss.page, row_at(u), len, a.Hl, g * G + hh, lane);
                if (hh != qh) {
                    Rows::load_q(qsrc + q_row(a, b, g * G + hh, n0) * D + seg * 16, q);
                    qh = hh;
                }
                cur.dot(q, &ss.score[0][hh][row_at(u)], lane);
            }
        }
    } else if (wave < nunits) {
        // columns: the queries of one head, or, the landmarks shared by the group, (query, head)
        const int ncol = shared ? nq * G : nq, col = min(n16, ncol - 1);
        QRow<T, D> q;
        LmkBlock<D> cur;
        int qh = -1;
        for (int u = wave; u < nunits; u += kBlock / kWave) {
            const int hh = head_of(u);
            cur.load(lmk, ss.page, row_at(u), len, a.Hl, g * gl + hh, lg, n16);
            if (hh != qh) {
                const int qq = shared ? col / G : col, h = shared ? col % G : hh;
                q.load(qsrc + q_row(a, b, g * G + h, n0 + qq) * D, lg, true);
                qh = hh;
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const f32x4 sc = mfma_row<T, D>(cur.x[t], q, zero4());
                if (n16 < ncol)
                    *reinterpret_cast<f32x4*>(
                        &ss.score[shared ? n16 / G : n16][shared ? n16 % G : hh][row_at(u) + t * 16 + lg * 4]) = sc;
            }
        }
    }
    __syncthreads();
    if (tid < len) {
        const float c = a.scale * ks;
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            float m = -INFINITY;
#pragma unroll
            for (int h = 0; h < G; ++h) m = fmaxf(m, c * ss.score[q][h][tid] + bias[h]);
            ss.sig[q][tid] = m + 0.f;  // (-0 as 0: equal scores rank by index)
        }
    }
    __syncthreads();
    if (wave < nq) {
        const int q = wave, lq = len_of(q);
        if (lq > 0) {
            constexpr int E = kSlice / kWave;
            float sc[E];
            int id[E];
            bool ok[E];
#pragma unroll
            for (int r = 0; r < E; ++r) {
                const int e = r * kWave + lane;
                ok[r] = e < lq;
                sc[r] = ok[r] ? ss.sig[q][e] : 0.f;
                id[r] = ok[r] ? c0 + e : -1;
            }
            const int m = wave_topk_reg<E, kTopkNatural>(sc, id, ok, a.K, ss.oid[q], ss.osc[q], ss.tid[q], ss.tsc[q]);
            const size_t cbase = (row_of(q) * ly.nslices + slice) * a.K;
            for (int t = lane; t < a.K; t += kWave) {
                cand_sc[cbase + t] = t < m ? ss.osc[q][t] : -INFINITY;
                cand_id[cbase + t] = t < m ? ss.oid[q][t] : -1;
            }
        }
    }
    clear_counters();
}

// a b, 0 if b is 0, whatever a is.
extern "C" __device__ float hils_mul_legacy(float, float) __asm("llvm.amdgcn.fmul.legacy");
__device__ __forceinline__ float mul_0(float a, float b) { return hils_mul_legacy(a, b); }

// Bytes of a dword of keys k0 .. k0 + 3 that lie below nk.
__device__ __forceinline__ uint32_t keys_below(int k0, int nk) {
    const int n = nk - k0;
    return n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << (8 * n)) - 1u;
}

// The K best of more survivors than a wave takes in one round, by the whole workgroup of row rg:
// histograms of 1024 steps of the keys' range (keys fall into its steps in order, so everything
// above the step that holds the K-th is in, everything below it out), narrowed to that step
// until at most 64 entries are left at or above it, which one wave ranks exactly.  More equal keys than
// that go the way of the smaller selections.  (2048 survivors: one wave, two rounds of 1024,
// 1M x 4 step 85 us, with the histograms 75.)
struct __align__(16) Q8BlockMerge {
    uint32_t lo[kBlock / kWave], hi[kBlock / kWave];
    int hist[1024];
    int id[64], oid[64], tid[64];
    float sc[64], osc[64], tsc[64];
    int count, kept, step, above;
};
template <typename MS>
__device__ int q8_merge_block(const FwdArgs& a, const DecLayout& ly, size_t rg, Q8BlockMerge& bm, MS& ms) {
    constexpr int E = 8;
    const int tid = threadIdx.x, w = wave_id(), lane = tid % kWave;
    const float* cand_sc = reinterpret_cast<const float*>(static_cast<const char*>(a.ws) + ly.cand);
    const int* cand_id = reinterpret_cast<const int*>(cand_sc + (size_t)a.B * a.N * a.Hkv * ly.nslices * a.K);
    const size_t base = rg * ly.nslices * a.K;
    const int total = ly.nslices * a.K;
    // key 0: no entry.  The first kBlock * E survivors stay in registers, the others are read again.
    uint32_t key0[E];
    auto key_at = [&](int e) {
        if (e >= total || cand_id[base + e] < 0) return 0u;
        const uint32_t k = ordered_key(cand_sc[base + e]);
        return k ? k : 1u;
    };
    uint32_t lo = 0xffffffffu, hi = 0;
    int n = 0;
#pragma unroll
    for (int r = 0; r < E; ++r) key0[r] = key_at(r * kBlock + tid);
    auto each = [&](auto&& f) {
#pragma unroll
        for (int r = 0; r < E; ++r) f(key0[r], r * kBlock + tid);
        for (int e = E * kBlock + tid; e - tid < total; e += kBlock) f(key_at(e), e);
    };
    each([&](uint32_t k, int) {
        if (k) {
            lo = min(lo, k);
            hi = max(hi, k);
            ++n;
        }
    });
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        lo = min(lo, (uint32_t)__shfl_xor((int)lo, o, kWave));
        hi = max(hi, (uint32_t)__shfl_xor((int)hi, o, kWave));
        n += __shfl_xor(n, o, kWave);
    }
    if (tid == 0) bm.count = bm.kept = 0;
    __syncthreads();
    if (lane == 0) {
        bm.lo[w] = lo;
        bm.hi[w] = hi;
        atomicAdd(&bm.count, n);
    }
    __syncthreads();
    n = bm.count;
#pragma unroll
    for (int i = 0; i < kBlock / kWave; ++i) {
        lo = min(lo, bm.lo[i]);
        hi = max(hi, bm.hi[i]);
    }
    const int m = min(n, a.K);
    uint32_t from = 1;  // entries with key >= from are left
    int left = n, want = m;  // of which `want` of the ones within [lo, hi] are among the m best
    while (left > 64) {
        const int shift = max(0, 22 - __clz(hi - lo | 1u));  // (hi - lo) >> shift < 1024
        for (int i = tid; i < 1024; i += kBlock) bm.hist[i] = 0;
        __syncthreads();
        each([&](uint32_t k, int) {
            if (k >= lo && k <= hi) atomicAdd(&bm.hist[(k - lo) >> shift], 1);
        });
        __syncthreads();
        if (w == 0) {  // the step where the count from the top reaches `want`; lane l: steps 1023 - 16 l and down
            int h[16], sum = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                h[i] = bm.hist[1023 - 16 * lane - i];
                sum += h[i];
            }
            int incl = sum;
#pragma unroll
            for (int o = 1; o < kWave; o <<= 1) {
                const int y = __shfl_up(incl, o, kWave);
                if (lane >= o) incl += y;
            }
            int at = incl - sum;
            if (at < want && want <= incl) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    if (at < want && want <= at + h[i]) {
                        bm.step = 1023 - 16 * lane - i;
                        bm.above = at;
                        bm.count = at + h[i];
                    }
                    at += h[i];
                }
            }
        }
        __syncthreads();
        left = m - want + bm.count;  // the ones above the range, and the range's down to that step
        want -= bm.above;
        lo += (uint32_t)bm.step << shift;
        from = lo;
        hi = min(hi, lo + ((1u << shift) - 1u));
        __syncthreads();
        if (shift == 0 && left > 64) break;
    }
    if (left > 64) {  // ties
        merge_row<E, kBlock / kWave>(a, ly, rg, ms, w);
        if (tid < ms.nbest) bm.oid[tid] = ms.bid[tid];
        __syncthreads();
        return ms.nbest;
    }
    each([&](uint32_t k, int e) {
        if (k >= from) {  // (counted apart: a wave may be here before another has read the first count)
            const int at = atomicAdd(&bm.kept, 1);
            bm.id[at] = cand_id[base + e];
            bm.sc[at] = cand_sc[base + e];
        }
    });
    __syncthreads();
    if (w == 0) {
        const bool ok[1] = {lane < left};
        const float sc[1] = {ok[0] ? bm.sc[lane] : 0.f};
        const int id[1] = {ok[0] ? bm.id[lane] : -1};
        wave_topk_reg<1>(sc, id, ok, a.K, bm.oid, bm.osc, bm.tid, bm.tsc);
    }
    __syncthreads();
    return m;
}

// gridDim.z workgroups of four waves share the parts of a row.  In a workgroup the last wave selects
// while the others take their share of the window's pieces, then the selected chunks are spread
// over all four.  A wave adds its parts into one running
// (maximum, sum, numerator) per head: part t enters with weight exp(z_t - M), z = s^_c for a chunk,
// whose P is divided by its own sum, and z = m + log l for a piece of the window.  With a row to
// itself a workgroup has many parts per wave, and the next one's K, landmark row and V are loaded as
// soon as the current one is done with their registers (the loads are the same in every
// iteration, so that the compiler counts the outstanding ones; float32 with routing queries, d = 128,
// spills 20 to 60 bytes a lane for it); with few there is nothing to load ahead (1024 rows 79 us when
// measured, without 83; a step of 32 rows the other way round, 19.9 and 18.3).
// The waves' results meet in LDS, those of several workgroups in the last of them to arrive.
// (A wave per part with its record in memory and the fusion in a launch of its own: 1024 rows of
// 25 parts 95 + 10 us, now 76.)
constexpr int kQ8RowWaves = 4;
template <typename T>
__device__ __forceinline__ void q8_store_out(const FwdArgs& a, size_t at, const f32x4& o) {
    if constexpr (sizeof(T) == 2)
        store_unaligned(as_mut<bf16>(a.out) + at, make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])));
    else
        __builtin_memcpy(as_mut<float>(a.out) + at, &o, 16);
}
template <typename T, int D, int G>
struct Q8RowSmem {
    float acc[kQ8RowWaves][G][D];
    float m[kQ8RowWaves][G], z[kQ8RowWaves][G];
    float part[kMaxParts][G];  // z of each part, log2 units
    float lse[G];
    union {
        MergeSmem<1> ms;
        MergeSmem<kQ8RowWaves> msb;
    };
    int page[64];      // of each slot
    float ks[64], vs[64];
};
template <typename T, int D, int G, int E, bool ROUTE, bool SPLIT>
__global__ __launch_bounds__(kQ8RowWaves * kWave, 2) void k_q8_row(Q8DecodeArgs qa, DecLayout ly) {
    constexpr int NW = kQ8RowWaves, DJ = D / 64, DB = D / 16;
    constexpr bool kAhead = !SPLIT;
    __shared__ __align__(16) Q8RowSmem<T, D, G> sm;
    __shared__ Q8BlockMerge bm;
    const FwdArgs& a = qa.f;
    const int ns = SPLIT ? gridDim.z : 1, split = SPLIT ? blockIdx.z : 0;
    const int g = blockIdx.x, b = blockIdx.y / a.N, n = blockIdx.y % a.N;
    const int tid = threadIdx.x, w = wave_id(), lane = tid % kWave, lg = lane / 16, n16 = lane % 16;
    const size_t rg = ((size_t)b * a.Hkv + g) * a.N + n;
    const int pos = decode_position(a, b, n), ncand = n_candidates(pos, a.W);
    const int hh = min(n16, G - 1), hl = a.Hl == a.Hq ? g * G + hh : g;
    QRow<T, D> q, qr_;
    q.load(as<T>(a.q) + q_row(a, b, g * G + hh, n) * D, lg, n16 < G);
    if constexpr (ROUTE) qr_.load(as<T>(a.q_route) + q_row(a, b, g * G + hh, n) * D, lg, n16 < G);
    const QRow<T, D>& qr = ROUTE ? qr_ : q;
    f32x4 acc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[db] = zero4();
    float M = -INFINITY, Z = 0.f;

    struct Regs {
        uint4 k[4][DJ], l[DJ], v[DB];
        float bias;
    } x;
    // (past a wave's last part `on` is 0 and the lanes of a load read one 16-byte piece; a
    // multiplication, because the compiler makes a choice a branch, with a wait, around each load)
    const int koff = ((n16 / 4) * 16 + n16 % 4) * D + lg * 16, voff = n16 * kChunk + lg * 16;
    auto load_k = [&](size_t page, int on) {
        const uint8_t* kp = static_cast<const uint8_t*>(a.k) + (page * a.Hkv + g) * kChunk * D;
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
#pragma unroll
            for (int j = 0; j < DJ; ++j)
                x.k[kb][j] = *reinterpret_cast<const uint4*>(kp + koff * on + kb * 4 * D + j * 64);
    };
    auto load_l = [&](size_t page, int on) {
        const uint8_t* lr = static_cast<const uint8_t*>(a.lmk) + (page * a.Hl + hl) * D;
#pragma unroll
        for (int j = 0; j < DJ; ++j) x.l[j] = *reinterpret_cast<const uint4*>(lr + lg * 16 * on + j * 64);
        // (branch-free: without biases a scale is read and not used)
        x.bias = *(a.bias ? a.bias + page * a.Hl + hl : qa.kv_scale + (page * a.Hkv + g) * 2);
    };
    auto load_v = [&](size_t page, int on) {
        const uint8_t* vp = static_cast<const uint8_t*>(a.v) + (page * a.Hkv + g) * kChunk * D;
#pragma unroll
        for (int db = 0; db < DB; ++db)
            x.v[db] = *reinterpret_cast<const uint4*>(vp + voff * on + db * 16 * kChunk);
    };
    // a part's page (-1: nothing there) and scales
    struct Where {
        int page;
        float ks, vs;
    };
    auto where = [&](int c) {
        Where r = {-1, 0.f, 0.f};
        if (c >= 0) {
            r.page = page_of(a, ly.nC, b, c);
            const float* sc = qa.kv_scale + ((size_t)r.page * a.Hkv + g) * 2;
            r.ks = sc[0];
            r.vs = sc[1];
        }
        return r;
    };

    // the workgroup's share: window pieces split, split + ns, ... and slots likewise
    const int npiece = (ly.nlocal - split + ns - 1) / ns, nslot = (a.K - split + ns - 1) / ns;
    int nsel = 0;
    if constexpr (E > kSoloE) nsel = q8_merge_block(a, ly, rg, bm, sm.msb);
    for (int phase = 0; phase < 2; ++phase) {
        if (phase == 0 && w == NW - 1 && nslot > 0) {
            int c = -1;  // lane t: the chunk of slot t (K <= 64)
            if constexpr (E > kSoloE) {
                c = lane < nsel ? bm.oid[lane] : -1;
                if (split == 0 && lane < a.K) a.idx[rg * a.K + lane] = c;
            } else if constexpr (E > 0) {
                merge_row_wave<E>(a, ly, rg, sm.ms);
                c = lane < sm.ms.nbest ? sm.ms.bid[lane] : -1;
                if (split == 0 && lane < a.K) a.idx[rg * a.K + lane] = c;
            } else {
                const int32_t* irow = a.idx + rg * a.K;
                if (lane < a.K && idx_entry_valid(irow, lane, ncand)) c = irow[lane];
            }
            const Where r = where(c);
            sm.page[lane] = r.page;
            sm.ks[lane] = r.ks;
            sm.vs[lane] = r.vs;
        }
        if (phase == 1) __syncthreads();  // the selection is made
        const int j0 = phase == 0 && w == NW - 1 ? npiece : w, step = phase == 0 ? NW - 1 : NW;
        const int nj = phase == 0 ? npiece : nslot;
        if (j0 >= nj) continue;
        // lane t: the wave's t-th part (at most 64 pieces or slots, over three or four waves)
        Where mine = {-1, 0.f, 0.f};
        {
            const int j = j0 + lane * step, at = split + j * ns;
            if (j < nj) {
                if (phase == 0)
                    mine = where(ncand + at <= pos / kChunk ? ncand + at : -1);
                else
                    mine = {sm.page[at], sm.ks[at], sm.vs[at]};
            }
        }
        if constexpr (kAhead) {
            const int page = max(0, __builtin_amdgcn_readlane(mine.page, 0));
            load_k(page, 1);
            load_l(page, 1);
            load_v(page, 1);
        }
        for (int j = j0, it = 0; j < nj; j += step, ++it) {
            const int pg = __builtin_amdgcn_readlane(mine.page, it);
            const float ks = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(mine.ks), it));
            const float vs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(mine.vs), it));
            const int at = split + j * ns, slot = phase == 0 ? a.K + at : at;
            const int nk = pg < 0 ? 0 : phase == 0 ? min(kChunk, pos - (ncand + at) * kChunk + 1) : kChunk;
            const int on = kAhead ? __builtin_amdgcn_readfirstlane((int)(j + step < nj)) : 1;
            const int page = max(0, kAhead ? __builtin_amdgcn_readlane(mine.page, it + on) : pg);
            if constexpr (!kAhead) {
                load_k(page, 1);
                load_l(page, 1);
                load_v(page, 1);
            }
            // S^T (lane: column n16, keys 16 lg + 4 kb + i), in log2 units; the next K
            const float c1 = a.scale * ks * kLog2e;
            float st[16], mx = -INFINITY;
#pragma unroll
            for (int kb = 0; kb < 4; ++kb) {
                const f32x4 s4 = mfma_row<T, D>(x.k[kb], q, zero4());
#pragma unroll
                for (int i = 0; i < 4; ++i) st[kb * 4 + i] = s4[i] * c1;
            }
            if constexpr (kAhead) load_k(page, on);
            // s^ of head n16: the diagonal of (landmark rows) x q^, held by lane group n16 / 4
            const f32x4 d4 = mfma_row<T, D>(x.l, qr, zero4());
            float dg = d4[0];
#pragma unroll
            for (int i = 1; i < 4; ++i)
                if (n16 % 4 == i) dg = d4[i];
            // (a bias of -inf is a mask, though the landmark be NaN)
            const float bias = a.bias ? x.bias : 0.f, score = c1 * __shfl(dg, n16 + 16 * (n16 / 4), kWave) + bias * kLog2e;
            const float sh = bias == -INFINITY ? bias : score;
            // (with loads ahead the compiler would move this score's product in among the exps: 8 sequences of
            // 64K, 4 new tokens, pages not in a cache, 39.4 us, now 38.6; 32 of 131K 75.7, now 75.2)
            if constexpr (kAhead) __builtin_amdgcn_sched_barrier(0);
            if constexpr (kAhead) load_l(page, on);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                st[i] = lg * 16 + i < nk ? st[i] : -INFINITY;
                mx = fmaxf(mx, st[i]);
            }
            mx = group4_max(mx);
            const float ref = mx == -INFINITY ? 0.f : mx;
            float l = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                st[i] = fexp2(st[i] - ref);
                l += st[i];
            }
            l = group4_sum(l);
            // the part enters the running sums
            const float z = l == 0.f ? -INFINITY : phase ? sh : mx + __builtin_amdgcn_logf(l);
            const float Mn = fmaxf(M, z), base = Mn == -INFINITY ? 0.f : Mn;
            const float corr = fexp2(M - base), zin = fexp2(z - base);
            const float f = zin == 0.f ? 0.f : vs * kWeightUnit * (phase ? zin / l : fexp2(mx - base));
            Z = Z * corr + zin;
            M = Mn;
            if (n16 < G && lg == 0) sm.part[slot][n16] = z;
            // (a part masked for every head, z = -inf, adds nothing, whatever its keys and values; one
            // masked for some heads adds nothing to them whatever its keys)
            if (__ballot(n16 < G && f != 0.f) != 0) {
                const WeightOperand p0(st), p1(st + 8);
                uint32_t keep[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) keep[i] = keys_below(lg * 16 + i * 4, nk);
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    const f16x8 v0 = f16x8_of_e4m3(x.v[db].x & keep[0], x.v[db].y & keep[1]);
                    const f16x8 v1 = f16x8_of_e4m3(x.v[db].z & keep[2], x.v[db].w & keep[3]);
                    const f32x4 o = mfma_weights(v0, p0, v1, p1);
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[db][i] = acc[db][i] * corr + mul_0(o[i], f);
                }
            } else {
#pragma unroll
                for (int db = 0; db < DB; ++db) acc[db] *= corr;
            }
            if constexpr (kAhead) load_v(page, on);
        }
    }
    // ---- the waves' sums, then the workgroups' ----
    if (n16 < G) {
#pragma unroll
        for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4*>(&sm.acc[w][n16][db * 16 + lg * 4]) = acc[db];
        if (lg == 0) {
            sm.m[w][n16] = M;
            sm.z[w][n16] = Z;
        }
    }
    __syncthreads();
    constexpr int RECF = 4 + D;
    const Recs<true> recs(q8_record(a, ly, SPLIT ? rg : 0, G, D), (size_t)q8_row_floats(ly.nparts, G, D));
    constexpr int zoff = kQ8MaxSplit * G * RECF;
    for (int e = tid; e < G * D / 4; e += NW * kWave) {
        const int h = e / (D / 4), d0 = e % (D / 4) * 4;
        float m = -INFINITY, z = 0.f;
#pragma unroll
        for (int i = 0; i < NW; ++i) m = fmaxf(m, sm.m[i][h]);
        const float base = m == -INFINITY ? 0.f : m;
        f32x4 o = zero4();
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const float c = fexp2(sm.m[i][h] - base);
            z += c * sm.z[i][h];
            o += c * *reinterpret_cast<const f32x4*>(&sm.acc[i][h][d0]);
        }
        if constexpr (SPLIT) {
            recs.store4((split * G + h) * RECF + 4 + d0, o);
            if (d0 == 0) recs.store3((split * G + h) * RECF, m, z, 0.f);
        } else {
            q8_store_out<T>(a, q_row(a, b, g * G + h, n) * D + d0, o * (1.f / z));
            if (d0 == 0) {
                sm.lse[h] = m + __builtin_amdgcn_logf(z);
                a.lse[q_row(a, b, g * G + h, n)] = (m + __builtin_amdgcn_logf(z)) * (1.f / kLog2e);
            }
        }
    }
    if constexpr (SPLIT) {
        auto z_at = [&](int e) { return (zoff + e) * 4; };
        for (int e = tid; e < ly.nparts * G; e += NW * kWave) {
            const int pt = e / G;
            if ((pt < a.K ? pt : pt - a.K) % ns == split)
                __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint((&sm.part[0][0])[e]), recs.r, z_at(e), 0, Recs<true>::kAux);
        }
        if (!last_to_arrive(reinterpret_cast<int*>(q8_record(a, ly, rg, G, D) + 3), ns)) return;
        for (int e = tid; e < G * D / 4; e += NW * kWave) {
            const int h = e / (D / 4), d0 = e % (D / 4) * 4;
            f32x4 head[kQ8MaxSplit], num[kQ8MaxSplit];
#pragma unroll
            for (int i = 0; i < kQ8MaxSplit; ++i) {
                const int r = (min(i, ns - 1) * G + h) * RECF;
                head[i] = recs.load4(r);
                num[i] = recs.load4(r + 4 + d0);
            }
            float m = -INFINITY, z = 0.f;
#pragma unroll
            for (int i = 0; i < kQ8MaxSplit; ++i) m = fmaxf(m, head[i][0]);
            const float base = m == -INFINITY ? 0.f : m;
            f32x4 o = zero4();
#pragma unroll
            for (int i = 0; i < kQ8MaxSplit; ++i)
                if (i < ns) {
                    const float c = fexp2(head[i][0] - base);
                    z += c * head[i][1];
                    o += c * num[i];
                }
            q8_store_out<T>(a, q_row(a, b, g * G + h, n) * D + d0, o * (1.f / z));
            if (d0 == 0) {
                sm.lse[h] = m + __builtin_amdgcn_logf(z);
                a.lse[q_row(a, b, g * G + h, n)] = (m + __builtin_amdgcn_logf(z)) * (1.f / kLog2e);
            }
        }
        if (qa.weights)
            for (int e = tid; e < ly.nparts * G; e += NW * kWave)
                (&sm.part[0][0])[e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(recs.r, z_at(e), 0, Recs<true>::kAux));
    }
    if (qa.weights) {
        __syncthreads();
        for (int pt = tid; pt < ly.nparts; pt += NW * kWave) {
            float sum = 0.f;
#pragma unroll
            for (int h = 0; h < G; ++h) sum += fexp2(sm.part[pt][h] - sm.lse[h]);
            qa.weights[rg * ly.nparts + pt] = sum;
        }
    }
}

struct Q8DecRun {
    template <typename T, int D, int G>
    static hipError_t run(const Q8DecodeArgs& qa, hipStream_t s) {
        const FwdArgs& a = qa.f;
        const DecLayout ly = q8_layout(a.B, a.N, a.Hkv, G, D, a.L, a.K, a.W, a.Hl != a.Hq);
        const int R = a.B * a.N, cus = device_cus(), surv = ly.nslices * a.K;
        auto scan = [&](auto many_tag, int counters) {
            constexpr int NQ = scan_queries<G>(decltype(many_tag)::value);
            const int pairs = ly.nslices * a.B * ((a.N + NQ - 1) / NQ);
            if (!a.given_idx)
                HILS_LAUNCH("k_q8_scan", (k_q8_scan<T, D, G, NQ>), dim3((pairs + 7) / 8 * 8 * a.Hkv), dim3(kBlock), 0, s,
                            qa, ly, counters);
        };
        // Above 128 rows a workgroup each; up to 128 four or more each, one per CU but no more than one
        // per four parts (256 rows: 1 workgroup per row 67.1 us a step, 2 70.9; 160 rows 30.3 and 31.3; 128
        // rows: 4 23.1, 2 24.9, 6 27.5; 64 rows: 4 22.9, 7 23.7).  (A given selection comes without the scan
        // that clears the arrival counters: one workgroup per row.)
        const int rows = R * a.Hkv;
        const int ns = a.given_idx || rows > kQ8SplitRows
                           ? 1
                           : std::max(1, std::min({kQ8MaxSplit, (ly.nparts + 3) / 4, std::max(4, cus / rows)}));
        if (a.N == 1)
            scan(std::false_type{}, ns > 1);
        else
            scan(std::true_type{}, ns > 1);
        const dim3 grid(a.Hkv, R, ns), block(kQ8RowWaves * kWave);
        auto row = [&](auto e_tag, auto route_tag) {
            constexpr int EE = decltype(e_tag)::value;
            constexpr bool RR = decltype(route_tag)::value;
            if constexpr (EE > 0)
                if (ns > 1) {
                    HILS_LAUNCH("k_q8_row", (k_q8_row<T, D, G, EE, RR, true>), grid, block, 0, s, qa, ly);
                    return;
                }
            HILS_LAUNCH("k_q8_row", (k_q8_row<T, D, G, EE, RR, false>), grid, block, 0, s, qa, ly);
        };
        auto by_route = [&](auto e_tag) {
            if (a.q_route) row(e_tag, std::true_type{});
            else row(e_tag, std::false_type{});
        };
        if (a.given_idx)
            by_route(std::integral_constant<int, 0>{});
        else if (surv <= kWave * kSoloE)
            by_route(std::integral_constant<int, kSoloE>{});
        else
            by_route(std::integral_constant<int, 2 * kSoloE>{});
        return hipGetLastError();
    }
};

template <typename T, int D>
hipError_t dispatch_q8_decode(const Q8DecodeArgs& qa, hipStream_t s) {
    const int G = qa.f.Hq / qa.f.Hkv;
#define HILS_CASE(GG) \
    if (G == GG) return Q8DecRun::run<T, D, GG>(qa, s);
    HILS_CASE(1) HILS_CASE(2) HILS_CASE(4) HILS_CASE(8)
#undef HILS_CASE
    return hipErrorInvalidValue;
}

}  // namespace

}  // namespace hils
