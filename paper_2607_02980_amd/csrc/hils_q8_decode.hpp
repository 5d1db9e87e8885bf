// HiLS attention decode over the 8-bit cache (layout: hils_q8.hpp), gfx950; compiled once per
// head dim.  N >= 1 new queries per sequence, each a row (b, g, n) of its own position.
//
//   A  k_q8_scan     grid (slices, Hkv, B x query groups): s^ of a slice of candidate chunks for
//                    a KV group's heads on MFMA, A operand the landmark rows as they lie in the
//                    pages, columns the queries; max over heads, the slice's top-K
//   B  merge         top-K over the slices' survivors, by each wave that needs it
//   C  k_q8_parts    a wave per part: a selected chunk of one query, or one piece of the window
//                    for all the queries of a group (16 / G of them, whose (query, head) pairs
//                    are the MFMA columns).  Record {m, l, s^, o[d]} per (row, part, head)
//   D  fusion        softmax over the parts -> out, lse and each part's weight; by the last
//                    workgroup of a group to arrive, or k_q8_combine
//
// Memory-bound: a row reads G d bytes of landmarks per candidate (one head's, d) and 128 d per
// part.  S^T = K Q^T leaves lane group lg with keys 16 lg + 0..15 when key 16 a + 4 kb + i is row
// 4 a + i of block kb, and V^T's 16-byte pieces hold those keys: P^T goes from the accumulators
// into O^T = V^T P^T without leaving its lane, and nothing of a part passes through LDS.
#pragma once

#include "hils_decode.hpp"
#include "hils_q8.hpp"

namespace hils {

namespace {

inline DecLayout q8_layout(int B, int N, int Hkv, int G, int d, int L, int K, int W, bool shared) {
    DecLayout o = {};
    o.nC = L / kChunk;
    o.nlocal = local_pieces_max(W);
    o.nparts = K + o.nlocal;
    const size_t bg = (size_t)B * N * Hkv;
    const size_t parts = align256(bg * o.nparts * G * (4 + d) * 4);
    o.slice = kSlice;
    const long sgroups = (long)B * ((N + 3) / 4) * Hkv;
    while (o.slice > 64 && sgroups * ((o.nC + o.slice - 1) / o.slice) < 1024 &&
           (o.nC + o.slice / 2 - 1) / (o.slice / 2) * K <= 4 * kWave)
        o.slice /= 2;
    o.nslices = (o.nC + o.slice - 1) / o.slice;
    o.cand = 0;
    // sized for the finest slices, so that the size never falls as a call grows
    o.parts = align256(bg * ((o.nC + 63) / 64) * K * 8);
    o.total = o.parts + parts;
    return o;
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

// Landmark rows of 64 chunks (4 MFMA tiles) of one landmark head against the columns of q.
template <typename T, int D>
struct LmkBlock {
    uint4 x[4][D / 64];
    __device__ __forceinline__ void load(const uint8_t* lmk, const int* page, int r0, int len, int Hl, int hl, int lg,
                                         int n16, bool stream) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const uint8_t* src = lmk + ((size_t)page[min(r0 + t * 16 + n16, len - 1)] * Hl + hl) * D + lg * 16;
#pragma unroll
            for (int j = 0; j < D / 64; ++j)
                x[t][j] = stream ? ld_stream16(src + j * 64) : *reinterpret_cast<const uint4*>(src + j * 64);
        }
    }
};

template <typename T, int D, int G, int NQ>
__global__ __launch_bounds__(kBlock) void k_q8_scan(Q8DecodeArgs qa, DecLayout ly, int counters) {
    const FwdArgs& a = qa.f;
    const int ngrp = (a.N + NQ - 1) / NQ;
    const int b = blockIdx.z / ngrp, n0 = (blockIdx.z % ngrp) * NQ, g = blockIdx.y;
    const int nq = min(NQ, a.N - n0);
    __shared__ Q8ScanSmem<G, NQ> ss;
    const int tid = threadIdx.x, wave = wave_id(), lane = tid % kWave, lg = lane / 16, n16 = lane % 16;
    const int c0 = blockIdx.x * ly.slice;
    float* cand_sc = reinterpret_cast<float*>(static_cast<char*>(a.ws) + ly.cand);
    int* cand_id = reinterpret_cast<int*>(cand_sc + (size_t)a.B * a.N * a.Hkv * ly.nslices * a.K);
    auto row_of = [&](int q) { return ((size_t)b * a.Hkv + g) * a.N + n0 + q; };
    auto len_of = [&](int q) {
        return q < nq ? max(0, min(ly.slice, n_candidates(decode_position(a, b, n0 + q), a.W) - c0)) : 0;
    };
    auto clear_counters = [&]() {
        if (counters && blockIdx.x == 0 && tid < nq) *part_counter<D>(a, ly, row_of(tid), G) = 0;
    };
    int len = 0;
#pragma unroll
    for (int q = 0; q < NQ; ++q) len = max(len, len_of(q));
    for (int q = 0; q < nq; ++q) {
        if (len_of(q) > 0) continue;
        const size_t cbase = (row_of(q) * ly.nslices + blockIdx.x) * a.K;
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
    const bool stream = a.N <= NQ;
    // column n16: query n16 of one head, or, the landmarks shared by the group, (query, head)
    const int gl = shared ? 1 : G;       // landmark heads of the group
    const int ncol = shared ? nq * G : nq;
    // units of (landmark head, 64 chunks): wave, wave + 4, ..., the head fastest, so that with
    // four heads or more a wave keeps its queries
    const int nblk = (len + 63) / 64, nunits = gl * nblk;
    if (wave < nunits) {
        LmkBlock<T, D> cur;
        QRow<T, D> q;
        int qh = -1;
        cur.load(lmk, ss.page, wave / gl * 64, len, a.Hl, shared ? g : g * G + wave % gl, lg, n16, stream);
        for (int u = wave; u < nunits; u += kBlock / kWave) {
            const int hh = u % gl, r0 = u / gl * 64;
            if (hh != qh) {
                const int col = min(n16, ncol - 1), qq = shared ? col / G : col, h = shared ? col % G : hh;
                q.load(qsrc + q_row(a, b, g * G + h, n0 + qq) * D, lg, true);
                qh = hh;
            }
            LmkBlock<T, D> nxt;
            const int un = min(u + kBlock / kWave, nunits - 1);  // (past the end: a block again, discarded)
            nxt.load(lmk, ss.page, un / gl * 64, len, a.Hl, shared ? g : g * G + un % gl, lg, n16, stream);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const f32x4 s = mfma_row<T, D>(cur.x[t], q, zero4());
                if (n16 < ncol)
                    *reinterpret_cast<f32x4*>(&ss.score[shared ? n16 / G : n16][shared ? n16 % G : hh][r0 + t * 16 + lg * 4]) = s;
            }
            cur = nxt;
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
            ss.sig[q][tid] = m;
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
            const size_t cbase = (row_of(q) * ly.nslices + blockIdx.x) * a.K;
            for (int t = lane; t < a.K; t += kWave) {
                cand_sc[cbase + t] = t < m ? ss.osc[q][t] : -INFINITY;
                cand_id[cbase + t] = t < m ? ss.oid[q][t] : -1;
            }
        }
    }
    clear_counters();
}

// Bytes of a dword of keys k0 .. k0 + 3 that lie below nk.
__device__ __forceinline__ uint32_t keys_below(int k0, int nk) {
    const int n = nk - k0;
    return n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << (8 * n)) - 1u;
}

// The columns of a part: lane l % 16 is (query rq, head rh) of the group's tile, on if it takes
// part; its first nk keys count, its record is rec (-1: none).
struct PartCol {
    int nk, rec;
    bool on;
};

// One part (chunk c) for the lanes' columns.  l = 0 marks a part without keys.  P is split into
// bf16 terms (two, three for float32 outputs), so that O has the sums' precision, not P's.
// uniform: every column that is on has the same nk; otherwise the values are masked for one
// query after the other (a value behind a query must not reach it, not even as 0 * NaN).
template <typename T, int D, int G, typename R>
__device__ __forceinline__ void q8_part(const Q8DecodeArgs& qa, const DecLayout& ly, const R& recs, int b, int g, int c,
                                        const T* qrow, const T* rrow, int hl, const PartCol& col, bool is_chunk,
                                        int nq, int rq) {
    constexpr int DJ = D / 64, DB = D / 16, PS = sizeof(T) == 2 ? 2 : 3;
    const FwdArgs& a = qa.f;
    const int lane = threadIdx.x % kWave, lg = lane / 16, n16 = lane % 16;
    const size_t page = page_of(a, ly.nC, b, c), pg = page * a.Hkv + g;
    const uint8_t* kp = static_cast<const uint8_t*>(a.k) + pg * kChunk * D;
    const uint8_t* vp = static_cast<const uint8_t*>(a.v) + pg * kChunk * D;
    uint4 kx[4][DJ], vx[DB];
#pragma unroll
    for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int j = 0; j < DJ; ++j)
            kx[kb][j] =
                *reinterpret_cast<const uint4*>(kp + ((n16 / 4) * 16 + kb * 4 + n16 % 4) * D + j * 64 + lg * 16);
#pragma unroll
    for (int db = 0; db < DB; ++db)
        vx[db] = *reinterpret_cast<const uint4*>(vp + (db * 16 + n16) * kChunk + lg * 16);
    const float ks = qa.kv_scale[pg * 2], vs = qa.kv_scale[pg * 2 + 1];
    QRow<T, D> q;
    q.load(qrow, lg, col.on);
    // s^ of the column's head: q^ . k' over the lane's 16 dims per 64, summed over the lane groups
    float sh = -INFINITY;
    if (is_chunk) {  // uniform over the wave
        const uint8_t* lr = static_cast<const uint8_t*>(a.lmk) + (page * a.Hl + hl) * D;
        float acc = 0.f;
#pragma unroll
        for (int j = 0; j < DJ; ++j) {
            const uint4 lx = *reinterpret_cast<const uint4*>(lr + j * 64 + lg * 16);
            const uint32_t w[4] = {lx.x, lx.y, lx.z, lx.w};
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                float x[8], y[8];
                e4m3_to_f32x4(w[2 * t], x);
                e4m3_to_f32x4(w[2 * t + 1], x + 4);
                load8(rrow + j * 64 + lg * 16 + t * 8, y);
#pragma unroll
                for (int e = 0; e < 8; ++e) acc += x[e] * y[e];
            }
        }
        sh = a.scale * ks * group4_sum(acc) + (a.bias ? a.bias[page * a.Hl + hl] : 0.f);
    }
    // S^T (lane: column n16, keys 16 lg + 4 kb + i), in log2 units
    const float c1 = a.scale * ks * kLog2e;
    float st[16], mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
        const f32x4 s4 = mfma_row<T, D>(kx[kb], q, zero4());
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            st[kb * 4 + i] = lg * 16 + kb * 4 + i < col.nk ? s4[i] * c1 : -INFINITY;
            mx = fmaxf(mx, st[kb * 4 + i]);
        }
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
    if (col.rec >= 0 && lg == 0) recs.store3(col.rec, mx * (1.f / kLog2e), l, sh);
    bf16x8 p0[PS], p1[PS];
    split_bf16x8<PS>(st, p0);
    split_bf16x8<PS>(st + 8, p1);
    auto values = [&](int nk, bool store) {
        uint32_t keep[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) keep[w] = keys_below(lg * 16 + w * 4, nk);
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            const bf16x8 v0 = bf16x8_of_e4m3(vx[db].x & keep[0], vx[db].y & keep[1]);
            const bf16x8 v1 = bf16x8_of_e4m3(vx[db].z & keep[2], vx[db].w & keep[3]);
            f32x4 o = zero4();
#pragma unroll
            for (int s = PS - 1; s >= 0; --s) {
                o = mfma16x16x32(v0, p0[s], o);
                o = mfma16x16x32(v1, p1[s], o);
            }
            if (store) recs.store4(col.rec + 4 + db * 16 + lg * 4, o * vs);
        }
    };
    // the keys of each query (uniform: the same for all)
    auto keys_of = [&](int q) { return __builtin_amdgcn_readlane(col.nk, q * G); };
    if (is_chunk) {
        values(kChunk, col.rec >= 0);
        return;
    }
    bool uniform = true;
    for (int q = 1; q < nq; ++q) uniform = uniform && keys_of(q) == keys_of(0);
    if (uniform) {
        values(keys_of(0), col.rec >= 0 && col.nk > 0);
    } else {
        for (int q = 0; q < nq; ++q) values(keys_of(q), col.rec >= 0 && col.nk > 0 && rq == q);
    }
}

// Fusion of row (b, g, n), records from float offset `off` of recs, by a workgroup of four waves:
// wave w takes heads w, w + 4, ...  With lambda0 the log mass of the window's pieces, z the scores
// of the chunks and L = LSE({z} U {lambda0}): a chunk weighs exp(z - L), a piece its share
// exp(m + log l - L) of the window; out = sum of weight * o / l.  A part's weights are added
// over the group's heads.
template <int G>
struct __align__(16) Q8FuseSmem {
    float w[G][kMaxParts];     // weight / l
    float mass[G][kMaxParts];  // weight
};
template <typename T, int D, int G, bool SHARED>
__device__ void q8_fuse(const Q8DecodeArgs& qa, const DecLayout& ly, Q8FuseSmem<G>& fs, const Recs<SHARED>& recs,
                        int off, int b, int n, int g) {
    constexpr int P = kMaxParts / kWave;
    constexpr int RECF = 4 + D, LPP = D / 4, PPL = kWave / LPP, BATCH = 16;
    const FwdArgs& a = qa.f;
    const int lane = threadIdx.x % kWave, d0 = (lane % LPP) * 4, sub = lane / LPP;
    for (int hh = wave_id(); hh < G; hh += kBlock / kWave) {
        auto part = [&](int j) {
            return recs.load4(off + (min(sub + PPL * j, ly.nparts - 1) * G + hh) * RECF + 4 + d0);
        };
        f32x4 h[P], v[BATCH];
#pragma unroll
        for (int t = 0; t < P; ++t) h[t] = recs.load4(off + (min(lane + t * kWave, ly.nparts - 1) * G + hh) * RECF);
#pragma unroll
        for (int j = 0; j < BATCH; ++j) v[j] = part(j);
        float m0 = -INFINITY, z = -INFINITY;
#pragma unroll
        for (int t = 0; t < P; ++t) {
            const int pt = lane + t * kWave;
            if (pt >= ly.nparts) h[t][1] = 0.f;
            if (h[t][1] != 0.f) {
                if (pt >= a.K)
                    m0 = fmaxf(m0, h[t][0]);
                else
                    z = fmaxf(z, h[t][2]);
            }
        }
        m0 = wave_max(m0);
        float l0 = 0.f;
#pragma unroll
        for (int t = 0; t < P; ++t)
            if (lane + t * kWave >= a.K && h[t][1] != 0.f) l0 += h[t][1] * expf(h[t][0] - m0);
        l0 = wave_sum(l0);
        const float lam0 = m0 + logf(l0);
        const float M = fmaxf(wave_max(z), lam0);
        float Z = 0.f;
#pragma unroll
        for (int t = 0; t < P; ++t)
            if (lane + t * kWave < a.K && h[t][1] != 0.f) Z += expf(h[t][2] - M);
        Z = wave_sum(Z) + expf(lam0 - M);
        const float L = M + logf(Z), a0 = expf(lam0 - L) / l0;
#pragma unroll
        for (int t = 0; t < P; ++t) {
            const int pt = lane + t * kWave;
            const float l = h[t][1];
            const float w = l == 0.f ? 0.f : pt >= a.K ? a0 * expf(h[t][0] - m0) : expf(h[t][2] - L) / l;
            fs.w[hh][pt] = w;
            fs.mass[hh][pt] = l == 0.f ? 0.f : w * l;
        }
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        f32x4 acc = zero4();
        for (int j0 = 0; j0 * PPL < ly.nparts; j0 += BATCH) {
            if (j0 > 0)
#pragma unroll
                for (int j = 0; j < BATCH; ++j) v[j] = part(j0 + j);
#pragma unroll
            for (int j = 0; j < BATCH; ++j) {
                const int pt = sub + PPL * (j0 + j);
                const float w = pt < ly.nparts ? fs.w[hh][pt] : 0.f;
                if (w != 0.f) acc += w * v[j];
            }
        }
#pragma unroll
        for (int o = LPP; o < kWave; o <<= 1)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] += __shfl_xor(acc[i], o, kWave);
        const size_t row = q_row(a, b, g * G + hh, n);
        if (sub == 0) {
            if constexpr (sizeof(T) == 2)
                store_unaligned(as_mut<bf16>(a.out) + row * D + d0,
                                make_uint2(pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3])));
            else
                __builtin_memcpy(as_mut<float>(a.out) + row * D + d0, &acc, 16);
        }
        if (lane == 0) a.lse[row] = L;
    }
    if (qa.weights) {
        __syncthreads();
        const size_t rg = ((size_t)b * a.Hkv + g) * a.N + n;
        for (int pt = threadIdx.x; pt < ly.nparts; pt += kBlock) {
            float m = 0.f;
#pragma unroll
            for (int hh = 0; hh < G; ++hh) m += fs.mass[hh][pt];
            qa.weights[rg * ly.nparts + pt] = m;
        }
        __syncthreads();  // the next row's weights may follow in fs
    }
}

// Four parts per workgroup, one per wave; units of a query group: KP = K rounded up to 4 per
// query, then the window's pieces.  E as in k_dec_parts_w: > 0, the waves of selected chunks
// merge the scan's survivors themselves (kSoloE: each alone; more: its workgroup, all of one
// query); 0: idx given.
template <typename T, int D, int G, int NQP, int E, bool FUSE>
__global__ __launch_bounds__(kBlock) void k_q8_parts(Q8DecodeArgs qa, DecLayout ly) {
    constexpr int NW = kBlock / kWave;
    constexpr int kScratch = E > kSoloE ? (int)sizeof(MergeSmem<NW>) : (int)sizeof(MergeSmem<1>) * NW;
    constexpr int kBytes = FUSE && (int)sizeof(Q8FuseSmem<G>) > kScratch ? (int)sizeof(Q8FuseSmem<G>) : kScratch;
    __shared__ __align__(16) unsigned char s_raw[kBytes];
    const FwdArgs& a = qa.f;
    const int w = wave_id(), lane = threadIdx.x % kWave, n16 = lane % 16;
    const int ngrp = (a.N + NQP - 1) / NQP;
    const int g = blockIdx.y, b = blockIdx.z / ngrp, n0 = (blockIdx.z % ngrp) * NQP;
    const int nq = min(NQP, a.N - n0);
    const int KP = (a.K + NW - 1) / NW * NW;
    const int unit = blockIdx.x * NW + w, rq_unit = unit / KP;
    const size_t rg0 = ((size_t)b * a.Hkv + g) * a.N + n0;  // the group's first row; the others follow
    const Recs<FUSE> recs(part_record<D>(a, ly, rg0, 0, 0, G), (size_t)nq * ly.nparts * G * (4 + D));
    const int rowf = ly.nparts * G * (4 + D);  // floats of a row's records
    auto record = [&](int q, int part, int h) { return q * rowf + (part * G + h) * (4 + D); };
    if (rq_unit < nq) {  // a slot of query rq_unit (uniform over the workgroup)
        const int slot = unit % KP, n = n0 + rq_unit;
        const size_t rg = rg0 + rq_unit;
        int csel = -1;
        if constexpr (E == kSoloE) {
            if (slot < a.K) {
                auto& ms = reinterpret_cast<MergeSmem<1>*>(s_raw)[w];
                merge_row_wave<E>(a, ly, rg, ms);
                const int nb = ms.nbest;
                if (slot == 0)
                    for (int t = lane; t < a.K; t += kWave) a.idx[rg * a.K + t] = t < nb ? ms.bid[t] : -1;
                csel = slot < nb ? ms.bid[slot] : -1;
            }
        } else if constexpr (E > 0) {
            auto& ms = *reinterpret_cast<MergeSmem<NW>*>(s_raw);
            merge_row<E, NW>(a, ly, rg, ms, w);
            const int nb = ms.nbest;
            if (unit % KP < NW)
                for (int t = threadIdx.x; t < a.K; t += kBlock) a.idx[rg * a.K + t] = t < nb ? ms.bid[t] : -1;
            if (slot < a.K) csel = slot < nb ? ms.bid[slot] : -1;
        } else {
            const int32_t* irow = a.idx + rg * a.K;
            if (slot < a.K && idx_entry_valid(irow, slot, n_candidates(decode_position(a, b, n), a.W)))
                csel = irow[slot];
        }
        const int c = __builtin_amdgcn_readfirstlane(csel);
        const int hh = min(n16, G - 1);
        if (slot < a.K && c >= 0) {
            const size_t row = q_row(a, b, g * G + hh, n);
            const PartCol col = {kChunk, n16 < G ? record(rq_unit, slot, hh) : -1, n16 < G};
            q8_part<T, D, G>(qa, ly, recs, b, g, c, as<T>(a.q) + row * D,
                             as<T>(a.q_route ? a.q_route : a.q) + row * D, a.Hl == a.Hq ? g * G + hh : g, col, true, 1, 0);
        } else if (slot < a.K && lane < G) {
            recs.store3(record(rq_unit, slot, lane), -INFINITY, 0.f, -INFINITY);
        }
    } else if (unit >= NQP * KP) {  // a piece of the window, for the group's queries
        const int first = decode_position(a, b, n0), c = n_candidates(first, a.W) + (unit - NQP * KP);
        const int rq = n16 / G, rh = n16 % G;
        const int pos = first + min(rq, nq - 1), piece = c - n_candidates(pos, a.W);
        const bool mine = rq < nq && piece >= 0 && piece < ly.nlocal;
        const int nk = mine ? max(0, min(kChunk, pos - c * kChunk + 1)) : 0;
        const int rec = mine ? record(rq, piece + a.K, rh) : -1;
        if (c <= (first + nq - 1) / kChunk) {  // some query reaches it
            const size_t row = q_row(a, b, g * G + rh, n0 + min(rq, nq - 1));
            q8_part<T, D, G>(qa, ly, recs, b, g, c, as<T>(a.q) + row * D, as<T>(a.q), 0, PartCol{nk, rec, rq < nq},
                             false, nq, rq);
        } else if (rec >= 0 && lane < 16) {
            recs.store3(rec, -INFINITY, 0.f, -INFINITY);
        }
    }
    if constexpr (FUSE) {
        if (last_to_arrive(part_counter<D>(a, ly, rg0, G), gridDim.x))
            for (int q = 0; q < nq; ++q)
                q8_fuse<T, D, G>(qa, ly, *reinterpret_cast<Q8FuseSmem<G>*>(s_raw), recs, q * rowf, b, n0 + q, g);
    }
}

template <typename T, int D, int G>
__global__ __launch_bounds__(kBlock) void k_q8_combine(Q8DecodeArgs qa, DecLayout ly) {
    __shared__ Q8FuseSmem<G> fs;
    const FwdArgs& a = qa.f;
    const int g = blockIdx.x, b = blockIdx.y / a.N, n = blockIdx.y % a.N;
    const size_t rg = ((size_t)b * a.Hkv + g) * a.N + n;
    const Recs<false> recs(part_record<D>(a, ly, rg, 0, 0, G), (size_t)ly.nparts * G * (4 + D));
    q8_fuse<T, D, G>(qa, ly, fs, recs, 0, b, n, g);
}

struct Q8DecRun {
    template <typename T, int D, int G, int NQS, int NQP>
    static hipError_t go(const Q8DecodeArgs& qa, hipStream_t s) {
        const FwdArgs& a = qa.f;
        const DecLayout ly = q8_layout(a.B, a.N, a.Hkv, G, D, a.L, a.K, a.W, a.Hl != a.Hq);
        const int R = a.B * a.N, cus = device_cus();
        constexpr int NW = kBlock / kWave;
        const int KP = (a.K + NW - 1) / NW * NW;
        const bool fuse = !a.given_idx && (long)R * a.Hkv * ly.nparts <= 8l * cus;
        if (!a.given_idx)
            HILS_LAUNCH("k_q8_scan", (k_q8_scan<T, D, G, NQS>),
                        dim3(ly.nslices, a.Hkv, a.B * ((a.N + NQS - 1) / NQS)), dim3(kBlock), 0, s, qa, ly, fuse);
        // (queries of a group sit within one chunk's length of each other: one more piece at most)
        const int units = NQP * KP + ly.nlocal + (NQP > 1 ? 1 : 0);
        const dim3 grid((units + NW - 1) / NW, a.Hkv, a.B * ((a.N + NQP - 1) / NQP));
        auto parts = [&](auto e_tag) {
            constexpr int EE = decltype(e_tag)::value;
            if constexpr (EE > 0) {
                if (fuse) {
                    HILS_LAUNCH("k_q8_parts", (k_q8_parts<T, D, G, NQP, EE, true>), grid, dim3(kBlock), 0, s, qa, ly);
                    return;
                }
            }
            HILS_LAUNCH("k_q8_parts", (k_q8_parts<T, D, G, NQP, EE, false>), grid, dim3(kBlock), 0, s, qa, ly);
            HILS_LAUNCH("k_q8_combine", (k_q8_combine<T, D, G>), dim3(a.Hkv, R), dim3(kBlock), 0, s, qa, ly);
        };
        const int surv = ly.nslices * a.K;
        if (a.given_idx)
            parts(std::integral_constant<int, 0>{});
        else if (surv <= kWave * kSoloE)
            parts(std::integral_constant<int, kSoloE>{});
        else if (surv <= kBlock * 8)
            parts(std::integral_constant<int, 8>{});
        else
            parts(std::integral_constant<int, 16>{});
        return hipGetLastError();
    }
    template <typename T, int D, int G>
    static hipError_t run(const Q8DecodeArgs& qa, hipStream_t s) {
        if (qa.f.N == 1) return go<T, D, G, 1, 1>(qa, s);
        return go<T, D, G, scan_queries<G>(true), MqCfg<G>::NQ>(qa, s);
    }
};

template <int D>
hipError_t dispatch_q8_decode(const Q8DecodeArgs& qa, hipStream_t s) {
    const int G = qa.f.Hq / qa.f.Hkv;
#define HILS_CASE(GG) \
    if (G == GG) return qa.f.bf16 ? Q8DecRun::run<bf16, D, GG>(qa, s) : Q8DecRun::run<float, D, GG>(qa, s);
    HILS_CASE(1) HILS_CASE(2) HILS_CASE(4) HILS_CASE(8)
#undef HILS_CASE
    return hipErrorInvalidValue;
}

}  // namespace

}  // namespace hils
