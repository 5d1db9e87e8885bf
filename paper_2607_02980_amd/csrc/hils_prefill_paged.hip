// Attention of a chunk of new tokens over a paged cache (f32 and bf16 storage, fp32 sums), gfx950.
//
// Row n < fresh_b of sequence b is the query at position len_b - fresh_b + n; everything else
// is the prefill's (Eqs. (1), (9), (10)), with chunk c of sequence b in page block_table[b, c]:
//
//   k_pp_score    sigma_ic = max_h s^_hc of 64 to 256 rows of a KV group against a slice of the
//                 candidates, on MFMA tiles; to the workspace, a block of rows at a time; where
//                 candidates are many, with the maxima of blocks of 16
//   k_pp_select   the K best of each row (exact radix select, ties to the smaller chunk; many
//                 candidates: the best blocks first, then theirs); each chosen chunk counts the
//                 row and gives it a rank
//   k_pp_plan     per (b, g): where each chunk's rows start, and the work items
//   k_pp_fill     the rows of every chunk, by offset and rank (few rows: k_pp_plan does it; very
//                 few: k_pp_select does the work of both)
//   k_pp_chunks   chunk-major: a chunk's K and V are read once and attended by all the rows that
//                 chose it, 16 (row, head) columns at a time; o_c and s^ of every (row, slot,
//                 head) go to the workspace as records
//   k_pp_local    the window [l(i), i] of 16 * 8 / G rows x G heads per workgroup, and the
//                 fusion with the records
//   k_pp_join     instead, where there are few rows: the blocks of the windows have been work items
//                 of k_pp_chunks too, and only records are left to be added up
//
// A row is computed the same way wherever the rows are cut; the order of a chunk's rows, which
// depends on atomics, decides only which of them share a matrix instruction, and columns of one
// do not meet, so results repeat bit for bit.
//
// Operands: a 16-byte piece of a row-major row is an MFMA operand in either type.  bf16: 8 of
// the 32 k-values of v_mfma_f32_16x16x32_bf16; f32: four k-values, one for each of four
// v_mfma_f32_16x16x4_f32, which take the contraction index in any order as long as both
// operands agree.  S^T = K Q^T leaves 4 consecutive keys of a column in each lane, the other
// product's B operand.  O^T = V^T P^T: V by transposing LDS reads (bf16), or as
// 16-byte reads that each feed four products, accumulator [4 dd + j][i] being dim
// 64 dd + 16 lg + 4 i + j (f32; lg = l / 16 of lane l).
#include <algorithm>
#include <type_traits>

#include "hils_device.hpp"
#include "hils_dispatch.hpp"
#include "hils_internal.hpp"
#include "hils_mfma.hpp"

namespace hils {

namespace {

// Waves of a score tile, 16 rows each (f32: its products take 8 times as long, and short calls have few tiles).
constexpr int score_waves(bool bf16) { return bf16 ? 8 : 4; }
constexpr int kScoreRows = 16 * score_waves(true);
constexpr int kScoreCand = 64;                // candidates of a staged landmark block
constexpr int kScoreSlice = 2048;             // candidates of a workgroup, at most
constexpr int kSelWaves = 4;
constexpr int kChunkWaves = 4;
// Rows of a work item, at most.  f32: 128 columns, as 16 of them take a wave 3 us (an item of 64 rows x 8 heads
// alone 25 us).
constexpr int seg_rows(bool bf16, int G) { return bf16 ? 64 : std::min(64, 128 / G); }
constexpr int kLocalWaves = 8;

// 16 bytes of global memory of which only the elements' alignment is known (one instruction).
template <typename T>
__device__ __forceinline__ uint4 ld16(const T* p) {
    uint4 x;
    __builtin_memcpy(&x, p, 16);
    return x;
}
__device__ __forceinline__ uint4 lds16(const char* p) { return *reinterpret_cast<const uint4*>(p); }

template <typename T, int D>
struct Cfg {
    static constexpr int ES = sizeof(T);
    static constexpr int KS = D * ES / 64;          // operands of a row (64 bytes of it each, over the lane groups)
    static constexpr int EP = 16 / ES;              // elements of a 16-byte piece
    static constexpr int DB = D / 16;               // accumulators of O^T
    static constexpr int KROW = D * ES + 16;        // bytes of a K (landmark) row in LDS
    static constexpr int VROW = D * ES + (ES == 2 ? 32 : 16);  // and of a V row
};

template <typename T>
__device__ __forceinline__ f32x4 mma(const uint4& a, const uint4& b, f32x4 c) {
    if constexpr (sizeof(T) == 2) {
        return mfma16x16x32(as_bf16x8(a), as_bf16x8(b), c);
    } else {
        const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], c, 0, 0, 0);
        return c;
    }
}

// o += V^T P^T for the 64 keys of a V tile in LDS, P as the accumulators st of S^T hold it.  bf16:
// the weights (unnormalised, at most 1) are rounded to bf16, at most 2^-8 of each, the type they
// are multiplied in.
template <typename T, int D>
__device__ __forceinline__ void add_pv(const char* s_v, const f32x4 (&st)[4], f32x4 (&o)[D / 16], int lane) {
    using C = Cfg<T, D>;
    if constexpr (sizeof(T) == 2) {
        const bf16* v = reinterpret_cast<const bf16*>(s_v);
        bf16x8 pb[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const float x[8] = {st[2 * t][0],     st[2 * t][1],     st[2 * t][2],     st[2 * t][3],
                                st[2 * t + 1][0], st[2 * t + 1][1], st[2 * t + 1][2], st[2 * t + 1][3]};
            pb[t] = pack_bf16x8(x);
        }
#pragma unroll
        for (int db = 0; db < C::DB; ++db) {
            o[db] = mfma16x16x32(tr_operand_perm(v, C::VROW / 2, 0, db * 16, lane), pb[0], o[db]);
            o[db] = mfma16x16x32(tr_operand_perm(v, C::VROW / 2, 32, db * 16, lane), pb[1], o[db]);
            if (db % 2 == 1) __builtin_amdgcn_sched_barrier(0);
        }
    } else {
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const char* row = s_v + (16 * kb + 4 * (lane / 16) + i) * C::VROW + 16 * (lane % 16);
#pragma unroll
                for (int dd = 0; dd < D / 64; ++dd) {
                    const f32x4 v = *reinterpret_cast<const f32x4*>(row + 256 * dd);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        o[4 * dd + j] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[j], st[kb][i], o[4 * dd + j], 0, 0, 0);
                }
            }
    }
}

// Dim of accumulator element [db][i] of lane group lg.
template <typename T>
__device__ __forceinline__ int dim_of(int db, int i, int lg) {
    return sizeof(T) == 2 ? 16 * db + 4 * lg + i : 64 * (db / 4) + 16 * lg + 4 * i + db % 4;
}

// No infinity or NaN among the elements of a 16-byte piece.
template <typename T>
__device__ __forceinline__ bool all_finite(const uint4& v) {
    const uint32_t y[4] = {v.x, v.y, v.z, v.w};
    bool ok = true;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        ok &= (y[i] & 0x7f800000u) != 0x7f800000u;
        if constexpr (sizeof(T) == 2) ok &= (y[i] & 0x7f80u) != 0x7f80u;
    }
    return ok;
}

// add_pv one key at a time, for a block with values that are not finite: keys past `last` or before `first`
// (of the column's row) are left out, where 0 times them would not be.
template <typename T, int D>
__device__ __forceinline__ void add_pv_by_key(const char* s_v, const f32x4 (&st)[4], f32x4 (&o)[D / 16], int lane,
                                              int last, int first) {
    using C = Cfg<T, D>;
#pragma unroll 1
    for (int j = 0; j < kChunk; ++j) {
        float mine = 0.f;
#pragma unroll
        for (int x = 0; x < 16; ++x) mine = j / 16 * 4 + j % 4 == x ? st[x / 4][x % 4] : mine;
        const float p = __shfl(mine, (j % 16) / 4 * 16 + lane % 16, kWave);
        const bool sees = (j <= last) & (j >= first);
        const T* v = reinterpret_cast<const T*>(s_v + j * C::VROW);
#pragma unroll
        for (int db = 0; db < C::DB; ++db) {
#pragma unroll
            for (int y = 0; y < 4; ++y)
                o[db][y] = sees ? fmaf(p, to_f32(v[dim_of<T>(db, y, lane / 16)]), o[db][y]) : o[db][y];
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// Records: a chunk's output o_c for one (row, head), as the accumulators hold it, with s^ in log2 units and the unit it
// is held in (bf16 calls) or the sum it stands for (f32: 1 for a chunk, a block's own for a piece of the window).
// They are written once and read once, a pass's largest traffic, so that bf16 calls keep them in
// float16, in units of the power of two below the vector's largest finite element: 2^-11 of that
// at most is lost, a fraction of what rounding the weights to bf16 loses (in bf16, 2^-8, it would be
// as much again).  f32 calls keep floats.
template <typename T, int D>
struct Record {
    static constexpr int BYTES = sizeof(T) == 2 ? 2 * D : 4 * D;
    static constexpr int PIECES = BYTES / 64;  // 16-byte pieces of a lane
    uint4 x[PIECES];

    __device__ __forceinline__ void load(const char* rec, int lg) {
#pragma unroll
        for (int t = 0; t < PIECES; ++t) x[t] = *reinterpret_cast<const uint4*>(rec + 64 * t + 16 * lg);
    }
    // acc = acc * rs + w * record (of which any bits are possible where w is to add nothing: ok)
    __device__ __forceinline__ void add(f32x4 (&acc)[D / 16], float rs, float w, bool ok) const {
#pragma unroll
        for (int t = 0; t < PIECES; ++t) {
            const uint4 y = ok ? x[t] : make_uint4(0, 0, 0, 0);
            if constexpr (sizeof(T) == 2) {
                typedef _Float16 h8 __attribute__((ext_vector_type(8)));
                const h8 h = __builtin_bit_cast(h8, y);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    acc[2 * t + i / 4][i % 4] = fmaf((float)h[i], w, acc[2 * t + i / 4][i % 4] * rs);
            } else {
                const f32x4 h = __builtin_bit_cast(f32x4, y);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[t][i] = fmaf(h[i], w, acc[t][i] * rs);
            }
        }
    }
    // Stores o * inv; the scale that the record is in units of.
    static __device__ __forceinline__ float store(char* rec, const f32x4 (&o)[D / 16], float inv, int lg, bool live) {
        if constexpr (sizeof(T) == 2) {
            float top = 0.f;
#pragma unroll
            for (int db = 0; db < D / 16; ++db)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float a = fabsf(o[db][i]);
                    top = fmaxf(top, a < INFINITY ? a : 0.f);
                }
            top = group4_max(top * inv);
            // 2^e <= top (2^-126 for less, 2^126 for more), and 2^-e
            const uint32_t e = min(max(__float_as_uint(top) >> 23, 1u), 253u);
            const float unit = __uint_as_float(e << 23), down = inv * __uint_as_float((254u - e) << 23);
            if (live) {
                typedef _Float16 h8 __attribute__((ext_vector_type(8)));
#pragma unroll
                for (int t = 0; t < PIECES; ++t) {
                    h8 h;
#pragma unroll
                    for (int i = 0; i < 8; ++i) h[i] = static_cast<_Float16>(o[2 * t + i / 4][i % 4] * down);
                    *reinterpret_cast<h8*>(rec + 64 * t + 16 * lg) = h;
                }
            }
            return unit;
        } else {
            if (live) {
#pragma unroll
                for (int db = 0; db < D / 16; ++db) *reinterpret_cast<f32x4*>(rec + 64 * db + 16 * lg) = o[db] * inv;
            }
            return 1.f;
        }
    }
};

// s^ in log2 units, and back.  log2 e times a bias near float32's largest value would pass it, so from 2^127 on the
// units are halves of s^ itself: still in order, and no two such logits need their difference but to be told apart (it is
// 0 or at least 2^104).
constexpr float kFarLogit = 0x1p127f;
__device__ __forceinline__ float to_log2(float s) {
    return s < kFarLogit ? s * kLog2e : kFarLogit * kLog2e + (s - kFarLogit) * 0.5f;
}
__device__ __forceinline__ float from_log2(float x) {
    return x < kFarLogit * kLog2e ? x * (1.f / kLog2e) : kFarLogit + (x - kFarLogit * kLog2e) * 2.f;
}

// Adds NR records to a running softmax (maximum m in log2 units, sum l, numerator o).
template <typename T, int D, int NR>
__device__ __forceinline__ void add_records(const Record<T, D> (&r)[NR], const float2 (&sv)[NR], const bool (&valid)[NR],
                                            f32x4 (&o)[D / 16], float& m, float& l) {
    // (a logit in log2 units is -inf for a bias of the lowest value too, whose weight is 0 beside any token of the window)
    float mnew = m;
    bool ok[NR];
#pragma unroll
    for (int u = 0; u < NR; ++u) {
        ok[u] = valid[u] && sv[u].x != -INFINITY;  // (a masked chunk's record may hold anything)
        mnew = ok[u] ? fmaxf(mnew, sv[u].x) : mnew;
    }
    float rs = mnew == m ? 1.f : fexp2(m - mnew);
    m = mnew;
    l *= rs;
#pragma unroll
    for (int u = 0; u < NR; ++u) {
        const float wk = ok[u] ? fexp2(sv[u].x - m) : 0.f, wy = ok[u] ? wk * sv[u].y : 0.f;
        l += sizeof(T) == 4 ? wy : wk;
        r[u].add(o, rs, sizeof(T) == 4 ? wk : wy, ok[u]);
        rs = 1.f;
    }
}

// New tokens of a sequence: `fresh` of them, the last of `len`.
struct Seq {
    int len, fresh, pos0;
};
__device__ __forceinline__ Seq sequence(const FwdArgs& f, const int32_t* newlens, int b) {
    Seq s;
    s.len = f.seqlens ? min(max(f.seqlens[b], 0), f.L) : f.L;
    s.fresh = min(newlens ? min(max(newlens[b], 0), f.N) : f.N, s.len);
    s.pos0 = s.len - s.fresh;
    return s;
}
__device__ __forceinline__ size_t page_of(const FwdArgs& f, int b, int c) {
    return (size_t)min(max(f.block_table[(size_t)b * (f.L / kChunk) + c], 0), f.num_pages - 1);
}

// Workspace of one segment of rows n0 .. n0 + Ns - 1 of every sequence.
struct Ws {
    int* counts;   // [bg][nC] rows of each chunk, then one word: the work items
    int* offs;     // [bg][nC] start of its rows in list
    int* ranks;    // [bg][Ns][K] rank of a row among its chunk's, -1: no chunk
    int* list;     // [bg][Ns * K] row << 6 | slot
    int4* work;    // (bg, chunk, offset, rows)
    float* sigma;  // [bg][Rs][nS], nS: nC in whole blocks
    float* bmax;   // [bg][Rs][nS / kBlock] the maxima of its blocks
    float2* rec_s; // [bg][Ns][slots][G] logit in log2 units, and the record's unit or sum
    char* rec_o;   // [bg][Ns][slots][G] records
};
struct Layout {
    size_t counts, offs, ranks, list, work, sigma, bmax, rec_s, rec_o, total;
    int Ns, Rs, slots;  // records of a (row, head)
    bool few;           // the windows' pieces among them
};

// Scores of so many candidates in a row have their maximum beside them.
constexpr int kBlock = 16;
__host__ __device__ constexpr int score_stride(int nC) { return (nC + kBlock - 1) / kBlock * kBlock; }

// sigma of a block of rows, in whole score tiles (4096 rows over 131K, 270 MB: in one block 123 us of scores and 65 of
// selection; in two of 135 MB 143 and 72).
constexpr size_t kSigmaBytes = size_t(512) << 20;

// Calls of so many records or fewer, those of the windows' pieces among them, take the windows as
// work items too (k_pp_join instead of k_pp_local, whose workgroups, each with all blocks of its rows' windows one
// after the other, take some 35 us however few they are).  Whole calls, K = 16, W = 512, k_pp_join and
// k_pp_local in us: bf16, 32 heads in groups of 4, d = 128, over 16000 tokens: 16 new tokens (12K records) 50 and
// 70, 256 (200K) 89 and 97, 512 (400K) 118 and 117, 1024 (800K) 218 and 185; f32: 512 291 and 314, 1024
// 565 and 497; f32, 16 heads in groups of 8, d = 64: 1024 (400K) 188 and 212.
constexpr size_t kFewRecords = size_t(5) << 16;
constexpr size_t kMaxRows = size_t(1) << 24;  // rows of a segment: a row and a slot in 31 bits, and their entries

Layout layout(int B, int Hq, int Hkv, int N, int L, int d, int K, int W, int bf16) {
    Layout w;
    const size_t nC = L / kChunk, bg = (size_t)B * Hkv, columns = (size_t)B * Hq * N;
    const size_t pieces = ((size_t)W + 62) / kChunk + 1;
    w.few = columns * (K + pieces) <= kFewRecords;
    w.slots = w.few ? K + (int)pieces : K;
    const size_t rec = (bf16 ? 2 : 4) * (size_t)d + sizeof(float2), per_row = (size_t)B * Hq * w.slots * rec;
    const size_t cap = prefill_record_cap(0);
    size_t ns = std::min<size_t>(N, kMaxRows);
    if (ns * per_row > cap) ns = std::min(ns, std::max<size_t>(kScoreRows, cap / per_row / kScoreRows * kScoreRows));
    const size_t nS = score_stride((int)nC);
    size_t rs = kSigmaBytes / (bg * nS * sizeof(float)) / kScoreRows * kScoreRows;
    rs = std::max<size_t>(rs, kScoreRows);
    const size_t parts = (ns + rs - 1) / rs;  // as equal as whole tiles allow
    rs = std::min(ns, (ns + parts * kScoreRows - 1) / (parts * kScoreRows) * kScoreRows);
    w.Ns = (int)ns;
    w.Rs = (int)rs;
    // Sizes by what any call of as many sequences, rows and tokens or fewer may need: bg * Ns is at most rows(slots)
    // and sigma at most kSigmaBytes, or their smallest blocks.
    const size_t G = Hq / Hkv, smallest = bg * std::min<size_t>(N, kScoreRows);
    auto rows = [&](size_t slots) {
        return std::min(bg * std::min<size_t>(N, kMaxRows), std::max(cap / (G * slots * rec), smallest));
    };
    const size_t most = rows(K), entries = most * K;
    const size_t scores = std::min(most * nS, std::max(kSigmaBytes / sizeof(float), smallest * nS));
    const size_t few_records = std::min(kFewRecords, rows(K + pieces) * G * (K + pieces));
    const size_t records = w.few ? few_records : std::max(most * G * K, few_records);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at = align256(at + bytes);
        return here;
    };
    w.counts = take((bg * nC + 1) * sizeof(int));
    w.offs = take(bg * nC * sizeof(int));
    w.ranks = take(entries * sizeof(int));
    w.list = take(entries * sizeof(int));
    w.work = take((std::min(bg * nC, entries) + entries / seg_rows(bf16, (int)G)) * sizeof(int4));
    w.sigma = take(scores * sizeof(float));
    w.rec_s = take(records * sizeof(float2));
    w.rec_o = take(records * (rec - sizeof(float2)));
    w.bmax = take(scores / kBlock * sizeof(float));
    w.total = at;
    return w;
}

// ---------------------------------------------------------------------------
// scores
// ---------------------------------------------------------------------------
// The value of the lane that PERM names among the four of a group.
template <int PERM>
__device__ __forceinline__ float quad_perm(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), PERM, 0xf, 0xf, true));
}

// A workgroup takes 16 RT rows per wave of a KV group (f32 64, bf16 128, or 256 with two row tiles a wave) and
// `slice` candidates; 64 landmark rows of one head at a time come through LDS (double-buffered) and serve all rows;
// the maximum over the heads stays in registers until a block of candidates is done.  It also
// clears the words that the next launches count in.
template <typename T, int D, int G, int RT>
__global__ __launch_bounds__(score_waves(sizeof(T) == 2) * kWave, sizeof(T) == 2 && RT * G * D <= 512 ? 4 : 1) void k_pp_score(FwdArgs f, const int32_t* newlens,
                                                                                 float* sigma, float* bmax, int r0, int Rs, int slice,
                                                                                 int nslices, int* counts, size_t nclear) {
    using C = Cfg<T, D>;
    constexpr int NW = score_waves(C::ES == 2), NT = NW * kWave, WROWS = 16 * RT, ROWS = WROWS * NW;
    constexpr int PPT = kScoreCand * D * C::ES / 16 / NT;
    constexpr bool kHold = C::ES == 2;  // the query operands of all heads fit in registers
    static_assert(PPT >= 1 && PPT * NT * 16 == kScoreCand * D * C::ES, "landmark blocks split evenly over the threads");
    __shared__ __align__(16) char s_l[2][kScoreCand * C::KROW];
    __shared__ float s_b[2][kScoreCand];
    __shared__ int s_pg[kScoreSlice];  // the candidates' pages: a step's loads do not wait for them
    const int tid = threadIdx.x, w = wave_id(), lane = tid % kWave, lg = lane / 16;
    const int ntiles = (Rs + ROWS - 1) / ROWS;
    for (size_t i = (size_t)blockIdx.x * NT + tid; i < nclear; i += (size_t)gridDim.x * NT) counts[i] = 0;
    int at = blockIdx.x;
    const int g = at % f.Hkv;
    at /= f.Hkv;
    const int part = at % nslices;
    at /= nslices;
    const int tile = at % ntiles, b = at / ntiles;
    const Seq sq = sequence(f, newlens, b);
    const int q0 = r0 + tile * ROWS;
    const int qend = min(min(q0 + ROWS, r0 + Rs), sq.fresh);
    if (q0 >= qend) return;
    const int nS = score_stride(f.L / kChunk);
    const int c_beg = part * slice, c_end = min(n_candidates(sq.pos0 + qend - 1, f.W), c_beg + slice);
    if (c_beg >= c_end) return;
    const bool shared_lmk = f.Hl != f.Hq;
    const int NH = shared_lmk ? 1 : G;
    const T* qr = as<T>(f.q_route ? f.q_route : f.q);
    auto q_operand = [&](int hh, int rt, int ks) {
        const int qa = min(q0 + WROWS * w + 16 * rt + lane % 16, qend - 1);
        return ld16(qr + (((size_t)b * f.Hq + g * G + hh) * f.N + qa) * D + ks * 4 * C::EP + lg * C::EP);
    };
    uint4 aq[kHold ? G : 2][RT][C::KS];
    if constexpr (kHold) {
#pragma unroll
        for (int hh = 0; hh < G; ++hh)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int ks = 0; ks < C::KS; ++ks) aq[hh][rt][ks] = q_operand(hh, rt, ks);
    }
    struct Regs {
        uint4 x[PPT];
        float bv;
    };
    const int nsteps = (c_end - c_beg + kScoreCand - 1) / kScoreCand * NH;
    // step t: candidate block t / NH, landmark head t % NH
    for (int i = tid; i < c_end - c_beg; i += NT) s_pg[i] = (int)page_of(f, b, c_beg + i);
    __syncthreads();
    auto fetch = [&](int t) {
        t = min(t, nsteps - 1);
        const int hl = shared_lmk ? g : g * G + t % NH, c0 = (t / NH) * kScoreCand, last = c_end - c_beg - 1;
        Regs r;
#pragma unroll
        for (int u = 0; u < PPT; ++u) {
            const int e = tid + u * NT, j = e / (D / C::EP), d0 = (e % (D / C::EP)) * C::EP;
            r.x[u] = ld16(as<T>(f.lmk) + ((size_t)s_pg[min(c0 + j, last)] * f.Hl + hl) * D + d0);
        }
        r.bv = f.bias && tid < kScoreCand ? f.bias[(size_t)s_pg[min(c0 + tid, last)] * f.Hl + hl] : 0.f;
        return r;
    };
    // candidate j of a block as row 16 (j % 4) + j / 4, so that a lane's four results are neighbours
    auto place = [](int j) { return j % 4 * 16 + j / 4; };
    auto store = [&](int buf, const Regs& r) {
#pragma unroll
        for (int u = 0; u < PPT; ++u) {
            const int e = tid + u * NT, j = e / (D / C::EP), d0 = (e % (D / C::EP)) * C::EP;
            *reinterpret_cast<uint4*>(&s_l[buf][place(j) * C::KROW + d0 * C::ES]) = r.x[u];
        }
        if (tid < kScoreCand) s_b[buf][place(tid)] = r.bv;
    };
    const size_t bg = (size_t)b * f.Hkv + g;
    f32x4 sg[RT][4];
    // step t computes from buffer t % 2; the rows of the next two steps are in flight
    auto step = [&](int t, const Regs& next, Regs& after) {
        const int buf = t & 1, lh = t % NH;
        after = fetch(t + 2);
        if (lh == 0)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int nb = 0; nb < 4; ++nb) sg[rt][nb] = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        auto head = [&](const uint4 (&q)[RT][C::KS]) {
#pragma unroll
            for (int nb = 0; nb < 4; ++nb) {
                f32x4 acc[RT];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) acc[rt] = zero4();
#pragma unroll
                for (int ks = 0; ks < C::KS; ++ks) {
                    const uint4 x = lds16(&s_l[buf][(nb * 16 + lane % 16) * C::KROW + ks * 64 + lg * 16]);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) acc[rt] = mma<T>(q[rt][ks], x, acc[rt]);
                }
                const float bv = s_b[buf][nb * 16 + lane % 16];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sg[rt][nb][i] = fmaxf(sg[rt][nb][i], f.scale * acc[rt][i] + bv);  // (a NaN loses)
            }
        };
        if constexpr (kHold) {
#pragma unroll
            for (int hh = 0; hh < G; ++hh)
                if (shared_lmk || hh == lh) head(aq[hh]);
        } else {
            // one head's operands at a time, the next one's in flight
            auto load = [&](int hh, uint4 (&q)[RT][C::KS]) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int ks = 0; ks < C::KS; ++ks) q[rt][ks] = q_operand(min(hh, G - 1), rt, ks);
            };
            const int h0 = shared_lmk ? 0 : lh, h1 = shared_lmk ? G : lh + 1;
            load(h0, aq[0]);
            for (int hh = h0; hh < h1; hh += 2) {
                load(hh + 1, aq[1]);
                head(aq[0]);
                if (hh + 1 >= h1) break;
                load(hh + 2, aq[0]);
                head(aq[1]);
            }
        }
        if (lh == NH - 1) {
            // (past c_end up to a whole block: nobody reads these)
            const int c = c_beg + (t / NH) * kScoreCand + 4 * (lane % 16);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int n = q0 + WROWS * w + 16 * rt + 4 * lg + i;
                    const bool in = n < qend && c < c_end;
                    // (-0 as 0: equal scores rank by index)
                    const f32x4 x = {sg[rt][0][i] + 0.f, sg[rt][1][i] + 0.f, sg[rt][2][i] + 0.f, sg[rt][3][i] + 0.f};
                    const size_t at = (bg * Rs + (n - r0)) * nS + c;
                    if (!bmax) {
                        if (in) *reinterpret_cast<f32x4*>(sigma + at) = x;
                        continue;
                    }
                    // (few of them will be read: past the last-level cache, whose lines the chunks' pass would
                    // have to write back: 4096 rows over 131K, that pass 291 -> 277 us)
                    if (in) __builtin_nontemporal_store(x, reinterpret_cast<f32x4*>(sigma + at));
                    float top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
                    top = fmaxf(top, quad_perm<0xb1>(top));  // lane ^ 1
                    top = fmaxf(top, quad_perm<0x4e>(top));  // lane ^ 2
                    if (in && lane % 4 == 0) bmax[at / kBlock] = top;
                }
        }
        store(buf ^ 1, next);
        __syncthreads();
    };
    Regs ra = fetch(0), rb = fetch(1);
    store(0, ra);
    __syncthreads();
    for (int t = 0; t < nsteps; t += 2) {
        step(t, rb, ra);
        if (t + 1 >= nsteps) break;
        step(t + 1, ra, rb);
    }
}

__global__ __launch_bounds__(256) void k_pp_clear(int* p, size_t n) {
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) p[i] = 0;
}

// Exclusive prefix sum of pairs (rows, and work items in the upper half) over NW waves; `all` is the total.
template <int NW>
__device__ __forceinline__ unsigned long long scan_pairs(unsigned long long mine, unsigned long long* s_sum,
                                                         unsigned long long& all) {
    const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave;
    unsigned long long incl = mine;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const unsigned long long y = __shfl_up(incl, o, kWave);
        if (lane >= o) incl += y;
    }
    if (lane == kWave - 1) s_sum[w] = incl;
    __syncthreads();
    unsigned long long at = incl - mine;
    all = 0;
    for (int i = 0; i < NW; ++i) {
        at += i < w ? s_sum[i] : 0;
        all += s_sum[i];
    }
    return at;
}
__device__ __forceinline__ unsigned long long pair_of(int rows, int seg) {
    return (unsigned long long)((rows + seg - 1) / seg) << 32 | (unsigned)rows;
}

// One wave per row: the K best of its candidates (E registers of 64 at a time, the best so far
// beside them), or the valid entries of a given selection; each counts the row for its chunk.
// kMany: a workgroup of 16 waves takes 64 rows of a (b, g) and counts in LDS first, with one atomic per
// chunk that any of them chose, which pays where many rows share a counter: K = 16, 4096 rows over
// 1000 tokens (820 entries a chunk) 157 us without, 30 with; over 16000 (209) 148 and 45; over 64000 (61) 87
// and 78; over 131K (31) 85 and 112.
// kPlanToo: where a segment has so few rows that one such workgroup takes all of a (b, g), it goes on with
// what is left for k_pp_plan and k_pp_fill otherwise, from the counts and ranks in LDS.  Whole calls, bf16, K = 16, with
// k_pp_plan and so: 16 rows over 15 candidates 30.1 and 27.5 us, 64 41.9 and 41.1; 16 over 242 39.6 and 37.9, 33 47.1
// and 48.2, 64 53.6 and 58.8 (one CU selects for all); 1 over 2040 34.9 and 33.0, 16 49.0 and 49.8.
constexpr int kSelHist = 4096;  // chunks counted in LDS
enum Select { kPerRow, kMany, kPlanToo };
// Candidates above which a row's blocks are looked at first: more than one pass over all of them takes, and of which
// the blocks hold half or fewer (K = 16, selection: 4096 rows over 131K 92 -> 67 us, 512 over 1M 71 -> 14, 16 over
// 1M 45 -> 10; 16 x 512 rows over up to 500 candidates 47 -> 52).
constexpr int kBlocks = 0;  // as E: by blocks
__host__ __device__ constexpr int blocks_above(int K) { return K <= 32 ? 16 * kWave : 32 * K; }
constexpr int kPlanTooScores = 4096;  // of a (b, g), at most
// kPlanToo: what a row's slot chose, in a word of LDS: the chunk, and the rank among its uses.  The uses of a chunk may be more
// than the rows: a given row that does not ascend ([4, -1, 4, ...]) uses it several times.
constexpr int kPlanRows = 64, kMaxSlots = 64;
constexpr int kRankBits = 12;
constexpr int plan_entry(int chunk, int rank) { return chunk << kRankBits | rank; }
constexpr int entry_chunk(int x) { return x >> kRankBits; }
constexpr int entry_rank(int x) { return x & ((1 << kRankBits) - 1); }
static_assert(entry_chunk(plan_entry(kSelHist - 1, kPlanRows * kMaxSlots - 1)) == kSelHist - 1 &&
                  entry_rank(plan_entry(kSelHist - 1, kPlanRows * kMaxSlots - 1)) == kPlanRows * kMaxSlots - 1 &&
                  plan_entry(kSelHist - 1, kPlanRows * kMaxSlots - 1) >= 0,
              "a chunk and a rank fit side by side, and -1 is neither");
template <int E, Select MODE>
__global__ __launch_bounds__((MODE != kPerRow ? 16 : kSelWaves) * kWave) void k_pp_select(
    FwdArgs f, const int32_t* newlens, const float* sigma, const float* bmax, int* counts, int* ranks, int n0, int Ns,
    int r0, int Rs, int* nwork, int4* work, int* list, int seg) {
    constexpr bool MANY = MODE != kPerRow;
    constexpr int NW = MANY ? 16 : kSelWaves, ROWS = MANY ? 64 : kSelWaves;
    __shared__ int s_tid[NW][kWave];
    __shared__ __align__(16) float s_tsc[NW][kWave];
    __shared__ int s_oid[NW][kWave];
    __shared__ float s_osc[NW][kWave];
    extern __shared__ int s_cnt[];  // MANY: rows of each chunk, then where they begin
    int* s_ent = s_cnt + (MODE == kPlanToo ? f.L / kChunk : 0);  // kPlanToo: plan_entry of a row's slot, or -1
    const int tid = threadIdx.x, w = wave_id(), lane = tid % kWave, nC = f.L / kChunk;
    const int tiles = (Rs + ROWS - 1) / ROWS, first = r0 + (int)(blockIdx.x % tiles) * ROWS;
    const size_t bg = blockIdx.x / tiles;
    const int b = (int)(bg / f.Hkv);
    const Seq sq = sequence(f, newlens, b);
    const int end = min(min(first + ROWS, r0 + Rs), sq.fresh);
    if (first >= end) return;
    const int chunks = min(nC, n_candidates(sq.pos0 + end - 1, f.W));  // that any row may choose
    if constexpr (MANY) {
        for (int c = tid; c < chunks; c += NW * kWave) s_cnt[c] = 0;
        __syncthreads();
    }
    for (int n = first + w; n < end; n += NW) {
        const int lim = n_candidates(sq.pos0 + n, f.W);
        int32_t* orow = f.idx + (bg * f.N + n) * f.K;
        int c = -1;
        if (f.given_idx) {
            if (lane < f.K && idx_entry_valid(orow, lane, lim)) c = orow[lane];
        } else {
            const float* row = sigma + (bg * Rs + (n - r0)) * score_stride(nC);
            int m = 0;
            // the K best of `src` at id_of(0 .. count - 1), in ascending order, to s_oid
            auto best_of = [&](auto e_tag, int count, auto id_of, const float* src) {
                constexpr int EE = decltype(e_tag)::value;
                m = 0;
                for (int c0 = 0; c0 < count; c0 += EE * kWave) {
                    float sc[EE + 1];
                    int id[EE + 1];
                    bool ok[EE + 1];
#pragma unroll
                    for (int e = 0; e < EE; ++e) {
                        const int at = c0 + e * kWave + lane;
                        ok[e] = at < count;
                        id[e] = id_of(at);
                        sc[e] = ok[e] ? src[id[e]] : 0.f;
                    }
                    ok[EE] = lane < m;
                    sc[EE] = ok[EE] ? s_osc[w][lane] : 0.f;
                    id[EE] = ok[EE] ? s_oid[w][lane] : -1;
                    m = wave_topk_reg<EE + 1, EE>(sc, id, ok, f.K, s_oid[w], s_osc[w], s_tid[w], s_tsc[w]);
                    __builtin_amdgcn_wave_barrier();
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                }
            };
            // (the row's own candidates may be far fewer than the call's)
            auto all_of = [](int i) { return i; };
            if constexpr (E != kBlocks) {
                if (E >= 4 && lim <= kWave)
                    best_of(std::integral_constant<int, 1>{}, lim, all_of, row);
                else if (E >= 16 && lim <= 4 * kWave)
                    best_of(std::integral_constant<int, 4>{}, lim, all_of, row);
                else
                    best_of(std::integral_constant<int, E>{}, lim, all_of, row);
            } else {
                // The K best are in the K blocks of the largest maxima (ties: the smaller; whatever is in another
                // has K before it), or past the whole blocks.
                const bool two = lim > blocks_above(f.K);
                const int whole = lim / kBlock, count = two ? whole : lim;
                const float* src = two ? bmax + (bg * Rs + (n - r0)) * (score_stride(nC) / kBlock) : row;
                if (count <= 5 * kWave)
                    best_of(std::integral_constant<int, 5>{}, count, all_of, src);
                else
                    best_of(std::integral_constant<int, 16>{}, count, all_of, src);
                if (two) {
                    const int blocks = m, picked = m * kBlock, held = s_oid[w][min(lane, m - 1)];
                    best_of(std::integral_constant<int, 5>{}, picked + lim - whole * kBlock, [&](int i) {
                        const int b = __shfl(held, min(i / kBlock, blocks - 1), kWave);
                        return i < picked ? b * kBlock + i % kBlock : whole * kBlock + i - picked;
                    }, row);
                }
            }
            if (lane < m) c = s_oid[w][lane];
            if (lane < f.K) orow[lane] = c;
        }
        if (lane < f.K) {
            const int rank = c < 0 ? -1 : atomicAdd(MANY ? &s_cnt[c] : &counts[bg * nC + c], 1);
            if constexpr (MODE == kPlanToo)
                s_ent[(n - first) * f.K + lane] = c < 0 ? -1 : plan_entry(c, rank);
            else
                ranks[(bg * Ns + (n - n0)) * f.K + lane] = rank;
        }
        __builtin_amdgcn_wave_barrier();
    }
    if constexpr (MODE == kPlanToo) {
        __shared__ unsigned long long s_sum[NW];
        __shared__ int s_base;
        __syncthreads();
        int rows0 = 0;
        for (int c0 = 0; c0 < chunks; c0 += NW * kWave) {
            const int c = c0 + tid, cnt = c < chunks ? s_cnt[c] : 0;
            unsigned long long all;
            const unsigned long long at = scan_pairs<NW>(pair_of(cnt, seg), s_sum, all);
            if (tid == 0) s_base = atomicAdd(nwork, (int)(all >> 32));
            __syncthreads();
            const int row = rows0 + (int)(unsigned)at;
            int item = s_base + (int)(at >> 32);
            if (c < chunks) s_cnt[c] = row;
            for (int k = 0; k < cnt; k += seg) work[item++] = make_int4((int)bg, c, row + k, min(seg, cnt - k));
            rows0 += (int)(unsigned)all;
        }
        __syncthreads();
        for (int e = tid; e < (end - first) * f.K; e += NW * kWave) {
            const int x = s_ent[e];
            if (x >= 0) list[bg * Ns * f.K + s_cnt[entry_chunk(x)] + entry_rank(x)] = (first - n0 + e / f.K) << 6 | e % f.K;
        }
    } else if constexpr (MANY) {
        __syncthreads();
        for (int c = tid; c < chunks; c += NW * kWave) {
            const int x = s_cnt[c];
            s_cnt[c] = x ? atomicAdd(&counts[bg * nC + c], x) : 0;
        }
        __syncthreads();
        for (int e = tid; e < (end - first) * f.K; e += NW * kWave) {
            const int n = first + e / f.K, slot = e % f.K;
            int& rank = ranks[(bg * Ns + (n - n0)) * f.K + slot];
            if (rank >= 0) rank += s_cnt[f.idx[(bg * f.N + n) * f.K + slot]];
        }
    }
}

// ---------------------------------------------------------------------------
// rows of every chunk
// ---------------------------------------------------------------------------
// One workgroup per (b, g): offsets of the chunks' rows in the list, and the work items (runs of
// up to `seg` rows of a chunk), which take ranges of `work` in any order; few rows are put in
// the list right here.
constexpr int kPlanThreads = 1024;
constexpr size_t kPlanFill = 16 * kPlanThreads;  // entries of a (b, g) that are not worth a launch
__device__ __forceinline__ void put_in_list(const FwdArgs& f, const int* offs, const int* ranks, int* list, size_t bg,
                                            int n0, int Ns, int fresh, int e) {  // entry e of (b, g)
    const int n = e / f.K, slot = e % f.K;
    if (n0 + n >= fresh) return;
    const int rank = ranks[bg * Ns * f.K + e];
    if (rank < 0) return;
    const int c = f.idx[(bg * f.N + n0 + n) * f.K + slot];
    list[bg * Ns * f.K + offs[bg * (f.L / kChunk) + c] + rank] = n << 6 | slot;
}
// PER chunks of a thread at a time: 1 where all fit, else 8 (16384 chunks: 84 -> 54 us).
template <int PER>
__global__ __launch_bounds__(kPlanThreads) void k_pp_plan(FwdArgs f, const int32_t* newlens, const int* counts,
                                                         int* offs, int4* work, int* nwork, const int* ranks,
                                                         int* list, int n0, int Ns, int fill, int seg) {
    constexpr int NW = kPlanThreads / kWave;
    __shared__ unsigned long long s_sum[NW];
    __shared__ int s_base;
    const int bg = blockIdx.x, tid = threadIdx.x, nC = f.L / kChunk;
    const int* cnt = counts + (size_t)bg * nC;
    int rows0 = 0;
    for (int c0 = 0; c0 < nC; c0 += kPlanThreads * PER) {
        int n[PER];
        unsigned long long mine = 0;  // rows, and items in the upper half
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = c0 + tid * PER + i;
            n[i] = c < nC ? cnt[c] : 0;
            mine += pair_of(n[i], seg);
        }
        unsigned long long all;
        const unsigned long long at = scan_pairs<NW>(mine, s_sum, all);
        if (tid == 0) s_base = atomicAdd(nwork, (int)(all >> 32));
        __syncthreads();
        int row = rows0 + (int)(unsigned)at, item = s_base + (int)(at >> 32);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = c0 + tid * PER + i;
            if (c < nC) offs[(size_t)bg * nC + c] = row;
            for (int k = 0; k < n[i]; k += seg) work[item++] = make_int4(bg, c, row + k, min(seg, n[i] - k));
            row += n[i];
        }
        rows0 += (int)(unsigned)all;
    }
    __syncthreads();  // (the offsets are written, s_base and s_sum read)
    if (!fill) return;
    const int fresh = sequence(f, newlens, bg / f.Hkv).fresh;
    for (int e = tid; e < Ns * f.K; e += kPlanThreads) put_in_list(f, offs, ranks, list, bg, n0, Ns, fresh, e);
}

__global__ __launch_bounds__(256) void k_pp_fill(FwdArgs f, const int32_t* newlens, const int* offs, const int* ranks,
                                                 int* list, int n0, int Ns) {
    const size_t e = (size_t)blockIdx.x * 256 + threadIdx.x, per = (size_t)Ns * f.K;
    if (e >= (size_t)f.B * f.Hkv * per) return;
    const size_t bg = e / per;
    put_in_list(f, offs, ranks, list, bg, n0, Ns, sequence(f, newlens, (int)(bg / f.Hkv)).fresh, (int)(e % per));
}

// ---------------------------------------------------------------------------
// retrieved chunks
// ---------------------------------------------------------------------------
// A workgroup takes one work item after the other: K and V of the chunk and the landmark rows of
// the group's heads in LDS, then columns p = (entry p / G, head p % G), 16 to a wave at a
// time, so that a chunk with few rows still fills its instructions with their heads.
// WINDOW: blocks of the rows' windows are items too, SEG rows and a block each, with records of
// their own (slots K .. K + P - 1 of a row are the pieces of its window, s^ is then the
// log-sum-exp).  Values that some row must not see: as in k_pp_local.
template <typename T, int D, int G, bool WINDOW>
__global__ __launch_bounds__(kChunkWaves * kWave, sizeof(T) == 2 ? 4 : 2) void k_pp_chunks(FwdArgs f,
                                                                                          const int32_t* newlens,
                                                                                          Ws ws, const int* nwork,
                                                                                          int n0, int Ns, int slots,
                                                                                          int blocks) {
    using C = Cfg<T, D>;
    constexpr int NT = kChunkWaves * kWave;
    constexpr int PPT = kChunk * D * C::ES / 16 / NT;
    __shared__ __align__(16) char s_k[kChunk * C::KROW];
    __shared__ __align__(16) char s_v[kChunk * C::VROW];
    __shared__ __align__(16) char s_l[G * D * C::ES];
    __shared__ float s_b[G];
    const int tid = threadIdx.x, w = wave_id(), lane = tid % kWave, lg = lane / 16;
    const int col = lane % 16, hh = col % G;
    constexpr int SEG = seg_rows(C::ES == 2, G);
    const int segs = (Ns + SEG - 1) / SEG;
    const int listed = nwork ? *nwork : 0, items = listed + (WINDOW ? f.B * f.Hkv * segs * blocks : 0);
    const float c1 = f.scale * kLog2e;
    for (int it = blockIdx.x; it < items; it += gridDim.x) {
        const bool win = WINDOW && it >= listed;  // uniform
        int bgi, c, len, first = 0;               // first: the item's first row, or place in the list
        Seq sq = {};
        if (win) {
            const int x = it - listed;
            bgi = x / (segs * blocks);
            sq = sequence(f, newlens, bgi / f.Hkv);
            first = x / blocks % segs * SEG;
            len = min(min(SEG, Ns - first), sq.fresh - n0 - first);
            if (len <= 0) continue;
            c = n_candidates(sq.pos0 + n0 + first, f.W) + x % blocks;
            if (c > (sq.pos0 + n0 + first + len - 1) / kChunk) continue;
        } else {
            const int4 wi = ws.work[it];
            bgi = wi.x;
            c = wi.y;
            first = wi.z;
            len = wi.w;
        }
        const int b = bgi / f.Hkv, g = bgi % f.Hkv;
        const size_t bg = bgi, pg = page_of(f, b, c);
        // a window's block that some row of the item sees only part of
        const bool part = win && (c < n_candidates(sq.pos0 + n0 + first + len - 1, f.W) ||
                                  c * kChunk + kChunk - 1 > sq.pos0 + n0 + first);
        bool bad = false;
        {
            const T* k = as<T>(f.k) + (pg * f.Hkv + g) * kChunk * D;
            const T* v = as<T>(f.v) + (pg * f.Hkv + g) * kChunk * D;
            uint4 kr[PPT], vr[PPT];
#pragma unroll
            for (int u = 0; u < PPT; ++u) {
                kr[u] = ld16(k + (size_t)(tid + u * NT) * C::EP);
                vr[u] = ld16(v + (size_t)(tid + u * NT) * C::EP);
            }
            if (part)
#pragma unroll
                for (int u = 0; u < PPT; ++u) {
                    if (c * kChunk + (tid + u * NT) / (D / C::EP) >= sq.len) vr[u] = make_uint4(0, 0, 0, 0);
                    bad |= !all_finite<T>(vr[u]);
                }
            __syncthreads();  // the previous item has been read
            if (!win) for (int e = tid; e < G * D / C::EP; e += NT) {
                const int h = e / (D / C::EP), d0 = (e % (D / C::EP)) * C::EP;
                const size_t lrow = pg * f.Hl + (f.Hl == f.Hq ? g * G + h : g);
                *reinterpret_cast<uint4*>(s_l + h * D * C::ES + d0 * C::ES) = ld16(as<T>(f.lmk) + lrow * D + d0);
                if (d0 == 0) s_b[h] = f.bias ? f.bias[lrow] : 0.f;
            }
#pragma unroll
            for (int u = 0; u < PPT; ++u) {
                const int e = tid + u * NT, j = e / (D / C::EP), at = (e % (D / C::EP)) * 16;
                *reinterpret_cast<uint4*>(s_k + j * C::KROW + at) = kr[u];
                *reinterpret_cast<uint4*>(s_v + j * C::VROW + at) = vr[u];
            }
        }
        if (WINDOW)
            bad = __syncthreads_or(bad);
        else
            __syncthreads();
        const int* seg = ws.list + bg * (size_t)Ns * f.K + first;
        const int units = (len * G + 15) / 16;
        for (int u = w; u < units; u += kChunkWaves) {
            const int e = u * (16 / G) + col / G;
            const bool live = e < len;
            int n = first + min(e, len - 1), slot = 0;
            if (!win) {
                const int ent = seg[min(e, len - 1)];
                n = ent >> 6;
                slot = ent & 63;
            }
            const size_t qrow = (((size_t)b * f.Hq + g * G + hh) * f.N + n0 + n) * D;
            uint4 q[C::KS];
#pragma unroll
            for (int ks = 0; ks < C::KS; ++ks) q[ks] = ld16(as<T>(f.q) + qrow + ks * 4 * C::EP + lg * C::EP);
            float shat = 0.f;
            if (!win) {
                // s^: the heads' landmark rows are rows 0 .. G - 1 of the A operand, so column p's is
                // accumulator row p % G, which lane group hh / 4 holds as element hh % 4
                f32x4 sh = zero4();
#pragma unroll
                for (int ks = 0; ks < C::KS; ++ks) {
                    uint4 al = lds16(s_l + min(col, G - 1) * D * C::ES + ks * 64 + lg * 16);
                    if (col >= G) al = make_uint4(0, 0, 0, 0);
                    const uint4 qs = f.q_route ? ld16(as<T>(f.q_route) + qrow + ks * 4 * C::EP + lg * C::EP) : q[ks];
                    sh = mma<T>(al, qs, sh);
                }
                const int hi = hh & 3;
                const float shv = hi == 0 ? sh[0] : hi == 1 ? sh[1] : hi == 2 ? sh[2] : sh[3];
                const float shr = __shfl(shv, (hh >> 2) * 16 + col, kWave);
                const float bias = s_b[hh];
                shat = bias == -INFINITY ? -INFINITY : f.scale * shr + bias;
            }
            f32x4 st[4];
#pragma unroll
            for (int kb = 0; kb < 4; ++kb) {
                st[kb] = zero4();
#pragma unroll
                for (int ks = 0; ks < C::KS; ++ks)
                    st[kb] = mma<T>(lds16(s_k + (kb * 16 + col) * C::KROW + ks * 64 + lg * 16), q[ks], st[kb]);
                __builtin_amdgcn_sched_barrier(0);
            }
            const int pos = sq.pos0 + n0 + n, ell = n_candidates(pos, f.W) * kChunk;  // (of a window's row)
            float mx = -INFINITY, sum = 0.f;
#pragma unroll
            for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    st[kb][i] *= c1;
                    if (part) {
                        const int j = c * kChunk + kb * 16 + lg * 4 + i;
                        const bool sees = (j <= pos) & (j >= ell);
                        st[kb][i] = sees ? st[kb][i] : -INFINITY;
                    }
                    mx = fmaxf(mx, st[kb][i]);
                }
            mx = group4_max(mx);
            const float muse = mx == -INFINITY ? 0.f : mx;
#pragma unroll
            for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    st[kb][i] = fexp2(st[kb][i] - muse);
                    sum += st[kb][i];
                }
            sum = group4_sum(sum);
            f32x4 o[C::DB];
#pragma unroll
            for (int db = 0; db < C::DB; ++db) o[db] = zero4();
            if (WINDOW && bad)
                add_pv_by_key<T, D>(s_v, st, o, lane, pos - c * kChunk, ell - c * kChunk);
            else
                add_pv<T, D>(s_v, st, o, lane);
            float inv = sum > 0.f ? 1.f / sum : 0.f, logit = to_log2(shat), mass = 1.f;
            bool keep = live;
            if (win) {
                slot = f.K + c - ell / kChunk;
                keep = live && slot >= f.K && c <= pos / kChunk;
                if constexpr (C::ES == 4) {  // (the sum beside the maximum: a rounded logarithm of it would cost 2^-22)
                    inv = 1.f;
                    logit = sum > 0.f ? mx : sum == 0.f ? -INFINITY : sum;
                    mass = sum;
                } else {
                    logit = mx + __log2f(sum);
                }
            }
            const size_t rec = ((bg * Ns + n) * slots + slot) * G + hh;
            const float unit = Record<T, D>::store(ws.rec_o + rec * Record<T, D>::BYTES, o, inv, lg, keep);
            if (keep && lg == 0) ws.rec_s[rec] = make_float2(logit, C::ES == 4 ? mass : unit);
        }
    }
}

// ---------------------------------------------------------------------------
// window and fusion
// ---------------------------------------------------------------------------
template <int G>
struct Tile {
    static constexpr int WR = 16 / G;            // rows of a wave (x G heads: 16 columns)
    static constexpr int QT = WR * kLocalWaves;  // rows of a workgroup
};

// Of the fusion's softmax a record is one more key, with logit s^ and value o_c, so that window and
// records go through one running (maximum, sum, numerator) per (row, head), in either order.  The
// window keeps the matrix cores busy (its 64-key blocks are double-buffered in LDS and shared
// by the waves), the records the memory; workgroups that share a CU take them in opposite order.
// Rows of V at or past the length are staged as zeros (nobody has written them).  Where a block
// holds an infinity or a NaN among values that some row of the tile must not see, 0 * it
// would reach that row: such a block's values are added one key at a time.
template <typename T, int D, int G>
__global__ __launch_bounds__(kLocalWaves * kWave, D * sizeof(T) <= 256 ? 4 : 2) void k_pp_local(FwdArgs f,
                                                                                         const int32_t* newlens,
                                                                                         const float2* rec_s,
                                                                                         const char* rec_o, int n0,
                                                                                         int Ns, int cus) {
    using C = Cfg<T, D>;
    constexpr int NT = kLocalWaves * kWave, QT = Tile<G>::QT, WR = Tile<G>::WR;
    constexpr int PPT = kChunk * D * C::ES / 16 / NT;
    __shared__ __align__(16) char s_k[2][kChunk * C::KROW];
    __shared__ __align__(16) char s_v[2][kChunk * C::VROW];
    __shared__ int s_bad[2];  // first key of the block in the buffer if its values are not all finite
    const int tid = threadIdx.x, w = wave_id(), lane = tid % kWave, lg = lane / 16;
    const int col = lane % 16, hh = col % G;
    const int ntiles = (Ns + QT - 1) / QT;
    int at = blockIdx.x;
    const int g = at % f.Hkv;
    at /= f.Hkv;
    const int tile = at % ntiles, b = at / ntiles;
    const Seq sq = sequence(f, newlens, b);
    const int q0 = n0 + tile * QT, qend = min(min(q0 + QT, n0 + Ns), sq.fresh);
    if (q0 >= qend) return;
    const size_t bg = (size_t)b * f.Hkv + g;
    const int n = min(q0 + w * WR + col / G, qend - 1), pos = sq.pos0 + n;
    const bool live = q0 + w * WR + col / G < qend;
    const int ncand = n_candidates(pos, f.W), ell = ncand * kChunk;
    const int kbeg = n_candidates(sq.pos0 + q0, f.W) * kChunk, klast = sq.pos0 + qend - 1;
    const int kfull = n_candidates(klast, f.W) * kChunk;  // keys from here to pos0 + q0 are in every row's window
    const size_t row = ((size_t)b * f.Hq + g * G + hh) * f.N + n;
    const float c1 = f.scale * kLog2e;
    if (tid < 2) s_bad[tid] = -1;
    // (not by the tile's place in the launch: the same bits however the rows are cut)
    const bool records_first = (q0 / QT + (size_t)b * ((f.N + QT - 1) / QT)) * f.Hkv / cus % 2;

    struct KV {
        uint4 k[PPT], v[PPT];
    };
    auto fetch = [&](int j0) {
        const size_t base = (page_of(f, b, j0 / kChunk) * f.Hkv + g) * kChunk * D;
        KV x;
#pragma unroll
        for (int u = 0; u < PPT; ++u) {
            x.k[u] = ld16(as<T>(f.k) + base + (size_t)(tid + u * NT) * C::EP);
            x.v[u] = ld16(as<T>(f.v) + base + (size_t)(tid + u * NT) * C::EP);
        }
        return x;
    };
    auto masked = [&](int j0) { return j0 < kfull || j0 + kChunk - 1 > sq.pos0 + q0; };
    auto stage = [&](int buf, int j0, const KV& x) {
        bool bad = false;
#pragma unroll
        for (int u = 0; u < PPT; ++u) {
            const int e = tid + u * NT, j = e / (D / C::EP), piece = (e % (D / C::EP)) * 16;
            uint4 v = x.v[u];
            if (j0 + j >= sq.len) v = make_uint4(0, 0, 0, 0);
            *reinterpret_cast<uint4*>(&s_k[buf][j * C::KROW + piece]) = x.k[u];
            *reinterpret_cast<uint4*>(&s_v[buf][j * C::VROW + piece]) = v;
            bad |= !all_finite<T>(v);
        }
        if (bad && masked(j0)) s_bad[buf] = j0;
    };

    uint4 q[C::KS];
#pragma unroll
    for (int ks = 0; ks < C::KS; ++ks) q[ks] = ld16(as<T>(f.q) + row * D + ks * 4 * C::EP + lg * C::EP);
    f32x4 o[C::DB];
#pragma unroll
    for (int db = 0; db < C::DB; ++db) o[db] = zero4();
    float m = -INFINITY, l = 0.f;  // running maximum (log2 units) and sum
    auto records = [&] {
        // the row's records, slots in idx order (lane: its column's dims)
        const int32_t* irow = f.idx + (bg * f.N + n) * f.K;
        const size_t rec0 = (bg * Ns + (n - n0)) * f.K;
        constexpr int SB = D == 128 ? 2 : 4;  // slots in flight together
        int prev = -1;
        for (int k0 = 0; k0 < f.K; k0 += SB) {
            Record<T, D> r[SB];
            float2 sv[SB];
            bool ok[SB];
#pragma unroll
            for (int u = 0; u < SB; ++u) {
                const int k = min(k0 + u, f.K - 1), c = irow[k];
                const size_t rec = (rec0 + k) * G + hh;
                sv[u] = rec_s[rec];  // (addresses that do not depend on c, so that all loads are issued at once)
                r[u].load(rec_o + rec * Record<T, D>::BYTES, lg);
                ok[u] = (k0 + u < f.K) & (c >= 0) & (c < ncand) & (c > prev);  // as idx_entry_valid
                prev = c;
            }
            add_records<T, D, SB>(r, sv, ok, o, m, l);
        }
    };
    bool seen_bad = false;  // uniform
    auto window = [&](auto careful_tag) {
        constexpr bool careful = decltype(careful_tag)::value;
        KV nx = fetch(kbeg);
        stage(0, kbeg, nx);
        __syncthreads();
        int buf = 0;
        for (int j0 = kbeg; j0 <= klast; j0 += kChunk, buf ^= 1) {
            const bool more = j0 + kChunk <= klast;  // uniform
            if (more) nx = fetch(j0 + kChunk);
            f32x4 st[4];
#pragma unroll
            for (int kb = 0; kb < 4; ++kb) {
                st[kb] = zero4();
#pragma unroll
                for (int ks = 0; ks < C::KS; ++ks)
                    st[kb] = mma<T>(lds16(&s_k[buf][(kb * 16 + col) * C::KROW + ks * 64 + lg * 16]), q[ks], st[kb]);
                __builtin_amdgcn_sched_barrier(0);
            }
            const bool part = masked(j0);
#pragma unroll
            for (int kb = 0; kb < 4; ++kb) st[kb] *= c1;
            if (part) {
#pragma unroll
                for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int j = j0 + kb * 16 + lg * 4 + i;
                        const bool sees = (j <= pos) & (j >= ell);
                        st[kb][i] = sees ? st[kb][i] : -INFINITY;
                    }
            }
            float mx = -INFINITY;
#pragma unroll
            for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                for (int i = 0; i < 4; ++i) mx = fmaxf(mx, st[kb][i]);
            mx = group4_max(mx);
            const float mnew = fmaxf(m, mx), muse = mnew == -INFINITY ? 0.f : mnew;
            const float alpha = fexp2(m - muse);
            float psum = 0.f;
#pragma unroll
            for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    st[kb][i] = fexp2(st[kb][i] - muse);
                    psum += st[kb][i];
                }
            psum = group4_sum(psum);
            l = l * alpha + psum;
            m = mnew;
#pragma unroll
            for (int db = 0; db < C::DB; ++db) o[db] *= alpha;
            if (careful && part && s_bad[buf] == j0) {  // uniform
                add_pv_by_key<T, D>(s_v[buf], st, o, lane, pos - j0, ell - j0);
            } else {
                add_pv<T, D>(s_v[buf], st, o, lane);
            }
            seen_bad |= part && s_bad[buf] == j0;
            if (more) stage(buf ^ 1, j0 + kChunk, nx);
            __syncthreads();
        }
    };
    __syncthreads();  // s_bad is set
    if (records_first) {
        records();
        window(std::false_type{});
    } else {
        window(std::false_type{});
        records();
    }
    // Once more, apart from the usual way.  It is in the same kernel all the same, and the register allocation spills around it:
    // bf16, d = 128 43 to 44 registers, f32, d = 64 9 to 11; without it 0, and 5 to 7.
    if (seen_bad) {
#pragma unroll
        for (int db = 0; db < C::DB; ++db) o[db] = zero4();
        m = -INFINITY;
        l = 0.f;
        window(std::true_type{});
        records();
    }
    if (!live) return;
    const float inv = 1.f / l;  // (the query's own key is in its window: l is 0 only where all logits are -inf)
    T* out = as_mut<T>(f.out) + row * D;
#pragma unroll
    for (int db = 0; db < C::DB; ++db) {
        if constexpr (C::ES == 2) {
            const f32x4 r = o[db] * inv;
            store_unaligned(out + 16 * db + 4 * lg, make_uint2(pack_bf16x2(r[0], r[1]), pack_bf16x2(r[2], r[3])));
        } else {
            const int dd = db / 4, i = db % 4;  // element i of the four accumulators of block dd: four dims in a row
            const f32x4 r = {o[4 * dd][i] * inv, o[4 * dd + 1][i] * inv, o[4 * dd + 2][i] * inv, o[4 * dd + 3][i] * inv};
            __builtin_memcpy(out + 64 * dd + 16 * lg + 4 * i, &r, 16);
        }
    }
    if (lg == 0) f.lse[row] = from_log2(m + __log2f(l));
}

// ---------------------------------------------------------------------------
// records of chunks and window, joined
// ---------------------------------------------------------------------------
// A wave per (row, head): each 16 lanes take every fourth record, a sixteenth of it per lane, in
// whole lines and independent of each other, and the four join at the end.
constexpr int kJoinWaves = 4;
template <typename T, int D>
__global__ __launch_bounds__(kJoinWaves * kWave) void k_pp_join(FwdArgs f, const int32_t* newlens, const float2* rec_s,
                                                               const char* rec_o, int n0, int Ns, int slots) {
    using C = Cfg<T, D>;
    // 16-byte pieces of a lane (a bf16 record of d = 64 has 8: the other 8 lanes read them too)
    constexpr int BYTES = Record<T, D>::BYTES, PCS = (BYTES / 16 + 15) / 16;
    constexpr int EPP = C::ES == 2 ? 8 : 4;  // elements of a piece
    const int G = f.Hq / f.Hkv, lane = threadIdx.x % kWave, sub = lane % 16, part = lane / 16;
    const size_t pair = (size_t)blockIdx.x * kJoinWaves + wave_id();  // (b, g, n, head)
    if (pair >= (size_t)f.B * f.Hkv * Ns * G) return;
    const int hh = (int)(pair % G), n = n0 + (int)(pair / G % Ns);
    const size_t bg = pair / G / Ns;
    const int b = (int)(bg / f.Hkv), g = (int)(bg % f.Hkv);
    const Seq sq = sequence(f, newlens, b);
    if (n >= sq.fresh) return;
    const int pos = sq.pos0 + n, ncand = n_candidates(pos, f.W), nrec = f.K + pos / kChunk + 1 - ncand;
    const int32_t* irow = f.idx + (bg * f.N + n) * f.K;
    const size_t rec0 = (bg * Ns + (n - n0)) * slots;
    float acc[PCS][EPP] = {}, m = -INFINITY, l = 0.f;
    constexpr int SB = 4;  // records of a lane in flight together
    for (int k0 = part; k0 < nrec; k0 += 4 * SB) {
        uint4 x[SB][PCS];
        float2 sv[SB];
        bool ok[SB];
#pragma unroll
        for (int u = 0; u < SB; ++u) {
            const int k = min(k0 + 4 * u, nrec - 1);
            const size_t rec = (rec0 + k) * G + hh;
            sv[u] = rec_s[rec];
#pragma unroll
            for (int t = 0; t < PCS; ++t)
                x[u][t] = *reinterpret_cast<const uint4*>(rec_o + rec * BYTES + (sub * PCS + t) * 16 % BYTES);
            ok[u] = k0 + 4 * u < nrec && (k >= f.K || idx_entry_valid(irow, k, ncand));
        }
        float mnew = m;
#pragma unroll
        for (int u = 0; u < SB; ++u) {
            ok[u] = ok[u] && sv[u].x != -INFINITY;  // (as in add_records)
            mnew = ok[u] ? fmaxf(mnew, sv[u].x) : mnew;
        }
        float rs = mnew == m ? 1.f : fexp2(m - mnew);
        m = mnew;
        l *= rs;
#pragma unroll
        for (int u = 0; u < SB; ++u) {
            const float wk = ok[u] ? fexp2(sv[u].x - m) : 0.f, wy = ok[u] ? wk * sv[u].y : 0.f;
            const float wu = C::ES == 4 ? wk : wy;
            l += C::ES == 4 ? wy : wk;
#pragma unroll
            for (int t = 0; t < PCS; ++t) {
                const uint4 y = ok[u] ? x[u][t] : make_uint4(0, 0, 0, 0);
                if constexpr (C::ES == 2) {
                    typedef _Float16 h8 __attribute__((ext_vector_type(8)));
                    const h8 h = __builtin_bit_cast(h8, y);
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[t][e] = fmaf((float)h[e], wu, acc[t][e] * rs);
                } else {
                    const f32x4 h = __builtin_bit_cast(f32x4, y);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[t][e] = fmaf(h[e], wu, acc[t][e] * rs);
                }
            }
            rs = 1.f;
        }
    }
    const float M = group4_max(m), to = m == M ? 1.f : fexp2(m - M);
    l = group4_sum(l * to);
    const float inv = 1.f / l;
#pragma unroll
    for (int t = 0; t < PCS; ++t)
#pragma unroll
        for (int e = 0; e < EPP; ++e) acc[t][e] = group4_sum(acc[t][e] * to) * inv;
    if (part != 0) return;
    const size_t row = ((size_t)b * f.Hq + g * G + hh) * f.N + n;
    T* out = as_mut<T>(f.out) + row * D;
#pragma unroll
    for (int t = 0; t < PCS; ++t) {
        const int piece = sub * PCS + t, pt = piece / 4, lg = piece % 4;  // piece 4 pt + lg of the record
        if (piece >= BYTES / 16) break;
        if constexpr (C::ES == 2) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                store_unaligned(out + dim_of<T>(2 * pt + h, 0, lg),
                                make_uint2(pack_bf16x2(acc[t][4 * h], acc[t][4 * h + 1]),
                                           pack_bf16x2(acc[t][4 * h + 2], acc[t][4 * h + 3])));
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) out[dim_of<T>(pt, i, lg)] = acc[t][i];
        }
    }
    if (sub == 0) f.lse[row] = from_log2(M + __log2f(l));
}

struct Run {
    template <typename T, int D, int G>
    static hipError_t run(const PrefillPagedArgs& a, hipStream_t s) {
        const FwdArgs& f = a.f;
        const Layout ly = layout(f.B, f.Hq, f.Hkv, f.N, f.L, D, f.K, f.W, f.bf16);
        char* base = static_cast<char*>(f.ws);
        Ws ws;
        ws.counts = reinterpret_cast<int*>(base + ly.counts);
        ws.offs = reinterpret_cast<int*>(base + ly.offs);
        ws.ranks = reinterpret_cast<int*>(base + ly.ranks);
        ws.list = reinterpret_cast<int*>(base + ly.list);
        ws.work = reinterpret_cast<int4*>(base + ly.work);
        ws.sigma = reinterpret_cast<float*>(base + ly.sigma);
        ws.bmax = reinterpret_cast<float*>(base + ly.bmax);
        ws.rec_s = reinterpret_cast<float2*>(base + ly.rec_s);
        ws.rec_o = base + ly.rec_o;
        const int nC = f.L / kChunk, maxc = n_candidates(f.L - 1, f.W);  // candidates of any row, at most
        const size_t bg = (size_t)f.B * f.Hkv, ncount = bg * nC;
        const int cus = device_cus(), seg = seg_rows(f.bf16, G);
        int* nwork = ws.counts + ncount;
        for (int n0 = 0; n0 < f.N; n0 += ly.Ns) {
            const int Ns = std::min(ly.Ns, f.N - n0);
            const bool plan_too = Ns <= kPlanRows && nC <= kSelHist && Ns * maxc <= kPlanTooScores;
            if (f.given_idx && maxc > 0)
                HILS_LAUNCH("k_pp_clear", k_pp_clear, dim3((unsigned)std::min<size_t>((ncount + 256) / 256, 4096)),
                            dim3(256), 0, s, ws.counts, ncount + 1);
            for (int r0 = n0; r0 < n0 + Ns; r0 += ly.Rs) {
                const int Rs = std::min(ly.Rs, n0 + Ns - r0);
                if (!f.given_idx && maxc > 0) {
                    // slices of candidates, so that the workgroups are one round of the chip
                    auto score = [&](auto rt_tag) {
                        constexpr int RT = decltype(rt_tag)::value, waves = score_waves(sizeof(T) == 2), rows = 16 * RT * waves;
                        const size_t tiles = bg * ((Rs + rows - 1) / rows);
                        const size_t want = std::max<size_t>(1, (2 / RT) * (size_t)cus / tiles);
                        const int blocks = (maxc + kScoreCand - 1) / kScoreCand;
                        const int slice = std::min(kScoreSlice, kScoreCand * (int)((blocks + want - 1) / want));
                        const int nslices = (maxc + slice - 1) / slice;
                        HILS_LAUNCH("k_pp_score", (k_pp_score<T, D, G, RT>), dim3((unsigned)(tiles * nslices)),
                                    dim3(waves * kWave), 0, s, f, a.newlens, ws.sigma, maxc > blocks_above(f.K) ? ws.bmax : nullptr, r0, Rs, slice, nslices, ws.counts,
                                    r0 == n0 ? ncount + 1 : 0);
                    };
                    // two row tiles per wave, each landmark operand feeding two products, where the heads' queries
                    // just fill the registers (4096 rows over 131K, groups of 4: 142 -> 121 us; groups of 2
                    // spill for no gain: 24 -> 43 us for 4 x 1500 rows over 8000)
                    constexpr int kTwo = sizeof(T) == 2 && G * D == 512 ? 2 : 1;
                    if (Rs > 16 * score_waves(sizeof(T) == 2))
                        score(std::integral_constant<int, kTwo>{});
                    else
                        score(std::integral_constant<int, 1>{});
                }
                auto select = [&](auto e_tag) {
                    constexpr int E = decltype(e_tag)::value;
                    auto launch = [&](auto mode_tag, int rows, int waves, size_t lds) {
                        constexpr Select MODE = decltype(mode_tag)::value;
                        HILS_LAUNCH("k_pp_select", (k_pp_select<E, MODE>), dim3((unsigned)(bg * ((Rs + rows - 1) / rows))),
                                    dim3(waves * kWave), lds, s, f, a.newlens, (const float*)ws.sigma,
                                    (const float*)ws.bmax, ws.counts, ws.ranks, n0, Ns, r0, Rs, nwork, ws.work, ws.list,
                                    seg);
                    };
                    if (plan_too)
                        launch(std::integral_constant<Select, kPlanToo>{}, kPlanRows, 16, (nC + kPlanRows * f.K) * sizeof(int));
                    else if ((size_t)Rs * f.K >= 64 * (size_t)nC && Rs >= 64 && nC <= kSelHist)
                        launch(std::integral_constant<Select, kMany>{}, 64, 16, nC * sizeof(int));
                    else
                        launch(std::integral_constant<Select, kPerRow>{}, kSelWaves, kSelWaves, 0);
                };
                if (maxc <= kWave)
                    select(std::integral_constant<int, 1>{});
                else if (maxc <= 4 * kWave)
                    select(std::integral_constant<int, 4>{});
                else if (maxc <= blocks_above(f.K))
                    select(std::integral_constant<int, 16>{});
                else
                    select(std::integral_constant<int, kBlocks>{});
            }
            const size_t most = bg * (std::min<size_t>(maxc, (size_t)Ns * f.K) + (size_t)Ns * f.K / seg);
            if (maxc > 0 && !plan_too) {
                const bool fill = (size_t)Ns * f.K <= kPlanFill;
                auto plan = [&](auto per_tag) {
                    constexpr int PER = decltype(per_tag)::value;
                    HILS_LAUNCH("k_pp_plan", k_pp_plan<PER>, dim3((unsigned)bg), dim3(kPlanThreads), 0, s, f, a.newlens,
                                (const int*)ws.counts, ws.offs, ws.work, nwork, (const int*)ws.ranks, ws.list, n0, Ns,
                                (int)fill, seg);
                };
                if (nC <= kPlanThreads)
                    plan(std::integral_constant<int, 1>{});
                else
                    plan(std::integral_constant<int, 8>{});
                if (!fill)
                    HILS_LAUNCH("k_pp_fill", k_pp_fill, dim3((unsigned)((bg * Ns * f.K + 255) / 256)), dim3(256), 0, s, f,
                                a.newlens, (const int*)ws.offs, (const int*)ws.ranks, ws.list, n0, Ns);
            }
            const size_t chunk_grid = 16 * (size_t)cus;
            if (ly.few) {
                const int blocks = (f.W + 61 + seg) / kChunk + 1;  // that the windows of `seg` rows reach into, at most
                const size_t wins = bg * ((Ns + seg - 1) / seg) * blocks;
                HILS_LAUNCH("k_pp_chunks", (k_pp_chunks<T, D, G, true>), dim3((unsigned)std::min(most + wins, chunk_grid)),
                            dim3(kChunkWaves * kWave), 0, s, f, a.newlens, ws, maxc > 0 ? (const int*)nwork : nullptr, n0, Ns,
                            ly.slots, blocks);
                const size_t pairs = bg * Ns * G;
                HILS_LAUNCH("k_pp_join", (k_pp_join<T, D>), dim3((unsigned)((pairs + kJoinWaves - 1) / kJoinWaves)),
                            dim3(kJoinWaves * kWave), 0, s, f, a.newlens, (const float2*)ws.rec_s, (const char*)ws.rec_o, n0,
                            Ns, ly.slots);
                continue;
            }
            if (maxc > 0)
                HILS_LAUNCH("k_pp_chunks", (k_pp_chunks<T, D, G, false>), dim3((unsigned)std::min(most, chunk_grid)),
                            dim3(kChunkWaves * kWave), 0, s, f, a.newlens, ws, (const int*)nwork, n0, Ns, ly.slots, 0);
            const int ntiles = (Ns + Tile<G>::QT - 1) / Tile<G>::QT;
            HILS_LAUNCH("k_pp_local", (k_pp_local<T, D, G>), dim3((unsigned)(bg * ntiles)), dim3(kLocalWaves * kWave), 0,
                        s, f, a.newlens, (const float2*)ws.rec_s, (const char*)ws.rec_o, n0, Ns, cus);
        }
        return hipGetLastError();
    }
};

}  // namespace

size_t prefill_paged_workspace_bytes(int B, int Hq, int Hkv, int N, int L, int d, int K, int W, int bf16) {
    return layout(B, Hq, Hkv, N, L, d, K, W, bf16).total;
}

hipError_t launch_prefill_paged(const PrefillPagedArgs& a, hipStream_t s) {
    return dispatch<Run>(a.f.bf16, a.f.d, a.f.Hq / a.f.Hkv, a, s);
}

}  // namespace hils
