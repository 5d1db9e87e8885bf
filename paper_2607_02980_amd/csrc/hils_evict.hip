// Eviction from a paged cache by accumulated attention weight (gfx950).
//
// A chunk's total is the attention weight that it has received: acc[c] += sum over KV groups and
// new queries of the weights that a decode call reported for it.  A sequence that holds more than
// `budget` candidate chunks (those before the last query's window) loses the ones with the least
// totals, ties to the lower index, the first `sink` chunks never.  Its table and totals close up
// over them and its length falls by 64 per chunk: chunks are whole, so every later position keeps
// its place inside its chunk.
//
// One workgroup per sequence.  What bounds it is latency: a step's work is a few kilobytes per
// sequence, a dozen dependent phases, and before them a thread's loads, each waited for before the
// next.  Up to kMaxHeld chunks a sequence's totals stay in LDS and its table in registers between the
// phases (k_evict; above 8192 chunks 18 registers of it spill); longer ones are read again from the
// L2 in each (k_evict_long).  Four sequences cut to 4096 chunks: of 16384 21 us, of 20480 22, of
// 20481 63; eight of 8191 12.5.
#include <climits>

#include "hils_dispatch.hpp"
#include "hils_internal.hpp"

namespace hils {

namespace {

constexpr int kEvictBlock = 1024;
constexpr int kEvictWaves = kEvictBlock / kWave;
constexpr int kMaxHeld = 20 * kEvictBlock;  // chunks (1.3M tokens): totals of 80 KB in LDS

// Tokens of sequence b.
__device__ __forceinline__ int evict_tokens(const EvictArgs& a, int b) {
    const int len = a.seqlens ? a.seqlens[b] : a.L;
    return len < 0 ? 0 : (len > a.L ? a.L : len);
}

// How many lanes below have x, and how many of the wave.
__device__ __forceinline__ int below(bool x, int& all) {
    const uint64_t m = __ballot(x);
    all = popc64(m);
    return popc64(m & ((1ull << __lane_id()) - 1ull));
}

// Order of the totals: -0 as 0, a NaN above every number (such a chunk stays while another can go);
// below 0xffffffff.  And the total of a number's key.
__device__ __forceinline__ uint32_t total_key(float x) { return x != x ? 0xfffffffeu : ordered_key(x + 0.f); }
__device__ __forceinline__ float key_total(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// Whether slot t of a selection row does not follow on the one before it.  A row without such a slot
// ascends and then is padded, so it names a chunk once; a given one may name a chunk again behind
// another entry ([5, -1, 5]: both slots count, as they do in decode), and its weights are then added
// one slot after the other, not by two threads at a time.
__device__ __forceinline__ bool out_of_order(const int32_t* row, int t) {
    return t > 0 && row[t] >= 0 && row[t] <= (row[t - 1] < 0 ? INT_MAX : row[t - 1]);
}

__global__ __launch_bounds__(kEvictBlock) void k_evict_long(EvictArgs a) {
    __shared__ int s_hist[256];
    __shared__ int s_bin, s_k, s_odd;
    __shared__ int s_tie[kEvictWaves], s_gone[kEvictWaves];
    const int b = blockIdx.x, tid = threadIdx.x, w = wave_id(), lane = tid % kWave;
    const int nC = a.L / kChunk;
    const int len0 = evict_tokens(a, b), len = max(len0, a.N);  // (len: the decode call's positions)
    const float* acc_in = a.acc + (size_t)b * nC;
    float* acc = a.acc_out + (size_t)b * nC;
    const int32_t* table_in = a.table + (size_t)b * nC;
    int32_t* table = a.table_out + (size_t)b * nC;
    int32_t* freed = a.freed ? a.freed + (size_t)b * a.most : nullptr;

    // ---- the totals ----
    if (tid == 0) s_odd = 0;
    if (acc != acc_in)
        for (int c = tid; c < nC; c += kEvictBlock) acc[c] = acc_in[c];
    __syncthreads();  // (also: every wave has read the length that seqlens_out may replace)
    if (a.weights) {
        const int pieces = (a.W + 62) / kChunk + 1, per = a.K + pieces;
        // row after row, so that a total is one sum in one order; a thread per weight of a row (at most
        // 64 slots and 64 pieces)
        for (int r = 0; r < a.Hkv * a.N; ++r) {
            const int g = r / a.N, n = r % a.N, pos = len - a.N + n, ncand = n_candidates(pos, a.W), t = tid;
            const size_t rg = ((size_t)b * a.Hkv + g) * a.N + n;
            const int32_t* row = a.idx + rg * a.K;
            int c = -1;
            if (t < a.K) {
                if (idx_entry_valid(row, t, ncand)) c = row[t];
                if (out_of_order(row, t)) s_odd = 1;
            } else if (t < per && ncand + t - a.K <= pos / kChunk) {
                c = ncand + t - a.K;
            }
            __syncthreads();
            const int steps = s_odd ? a.K : 1;  // (from the first such row on)
            for (int u = 0; u < steps; ++u) {
                if (c >= 0 && (steps == 1 || (t < a.K ? t : 0) == u)) acc[c] += a.weights[rg * per + t];
                __syncthreads();
            }
        }
    }
    const int last = n_candidates(len0 - 1, a.W), able = max(0, last - a.sink);
    const int drop = min(min(max(0, last - a.budget), able), a.most);
    if (tid == 0) {
        a.seqlens_out[b] = len0 - drop * kChunk;
        a.nfreed[b] = drop;
    }
    for (int t = drop + tid; t < a.most; t += kEvictBlock) freed[t] = -1;
    if (drop == 0) {
        if (table != table_in)
            for (int c = tid; c < nC; c += kEvictBlock) table[c] = table_in[c];
        return;
    }
    __syncthreads();

    // ---- the drop-th smallest total of chunks sink .. last - 1, eight bits of its key at a time ----
    auto key_of = [&](int c) { return total_key(acc[c]); };
    uint32_t T = 0, mask = 0;
    int k = drop;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int t = tid; t < 256; t += kEvictBlock) s_hist[t] = 0;
        __syncthreads();
        for (int c = a.sink + tid; c < last; c += kEvictBlock) {
            const uint32_t key = key_of(c);
            if ((key & mask) == T) atomicAdd(&s_hist[(key >> shift) & 255], 1);
        }
        __syncthreads();
        if (w == 0) {
            int h[4], sum = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                h[i] = s_hist[lane * 4 + i];
                sum += h[i];
            }
            int incl = sum;
#pragma unroll
            for (int o = 1; o < kWave; o <<= 1) {
                const int y = __shfl_up(incl, o, kWave);
                if (lane >= o) incl += y;
            }
            int at = incl - sum;
            if (at < k && k <= incl) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (at < k && k <= at + h[i]) {
                        s_bin = lane * 4 + i;
                        s_k = k - at;
                    }
                    at += h[i];
                }
            }
        }
        __syncthreads();
        T |= (uint32_t)s_bin << shift;
        mask |= 255u << shift;
        k = s_k;
        __syncthreads();
    }

    // ---- the table and the totals close up: chunks below the threshold, and its first k ties, go ----
    int ties = 0, gone = 0;  // before this tile
    for (int c0 = 0; c0 < nC; c0 += kEvictBlock) {
        const int c = c0 + tid;
        const bool in = c < nC;
        const float total = in ? acc[c] : 0.f;
        const int32_t page = in ? table_in[c] : -1;
        const bool free_ = c >= a.sink && c < last;
        const uint32_t key = total_key(total);
        const bool tie = free_ && key == T;
        int nt, ng;
        int before = below(tie, nt);
        if (lane == 0) s_tie[w] = nt;
        __syncthreads();
        for (int i = 0; i < w; ++i) before += s_tie[i];
        const bool go = free_ && (key < T || (tie && ties + before < k));
        int at = below(go, ng);
        if (lane == 0) s_gone[w] = ng;
        __syncthreads();
        for (int i = 0; i < w; ++i) at += s_gone[i];
        at += gone;
        if (go) {
            freed[at] = page;
        } else if (in) {  // (to a place that no later tile reads)
            acc[c - at] = total;
            table[c - at] = page;
        }
        for (int i = 0; i < kEvictWaves; ++i) {
            ties += s_tie[i];
            gone += s_gone[i];
        }
        __syncthreads();
    }
    for (int c = nC - drop + tid; c < nC; c += kEvictBlock) {
        acc[c] = 0.f;
        table[c] = -1;
    }
}

// The totals of up to 1024 EPT chunks in LDS.  With nr chunks per thread, wave w owns chunks
// 64 nr w + 64 r + lane, r < nr.
template <int EPT>
__global__ __launch_bounds__(kEvictBlock) void k_evict(EvictArgs a) {
    constexpr int NW = kEvictWaves, kSteps = 1024;
    __shared__ float s_tot[EPT * kEvictBlock];
    __shared__ int s_hist[kSteps];
    __shared__ uint32_t s_lo[NW], s_hi[NW], s_list[kWave];
    __shared__ int s_step, s_below, s_in, s_ties[NW], s_gone[NW], s_odd[2][NW];
    const int b = blockIdx.x, tid = threadIdx.x, w = wave_id(), lane = tid % kWave;
    const int nC = a.L / kChunk, nr = (nC + kEvictBlock - 1) / kEvictBlock, first = w * kWave * nr + lane;
    const float* acc_in = a.acc + (size_t)b * nC;
    float* acc = a.acc_out + (size_t)b * nC;
    const int32_t* table_in = a.table + (size_t)b * nC;
    int32_t* table = a.table_out + (size_t)b * nC;
    const int len0 = evict_tokens(a, b), len = max(len0, a.N);  // (len: the decode call's positions)
    int32_t page[EPT];
#pragma unroll
    for (int r = 0; r < EPT; ++r) {
        if (r >= nr) continue;
        const int c = first + r * kWave;
        s_tot[c] = c < nC ? acc_in[c] : 0.f;
        page[r] = c < nC ? table_in[c] : -1;
    }
    if (a.weights) {
        // row after row (g, n), so that a total is one sum in one order
        const int per = a.K + (a.W + 62) / kChunk + 1, total = a.Hkv * a.N * per;
        for (int e0 = 0; e0 < total; e0 += kEvictBlock) {
            const int e = e0 + tid, r = e / per, t = e % per;
            int c = -1;
            float x = 0.f;
            bool odd = false;
            if (e < total) {
                const int pos = len - a.N + r % a.N, ncand = n_candidates(pos, a.W);
                const size_t rg = (size_t)b * a.Hkv * a.N + r;
                const int32_t* row = a.idx + rg * a.K;
                x = a.weights[rg * per + t];
                if (t < a.K) {
                    if (idx_entry_valid(row, t, ncand)) c = row[t];
                    odd = out_of_order(row, t);
                } else if (ncand + t - a.K <= pos / kChunk) {
                    c = ncand + t - a.K;
                }
            }
            const int r0 = e0 / per, r1 = min(total - 1, e0 + kEvictBlock - 1) / per;
            int* odds = s_odd[(e0 / kEvictBlock) & 1];  // (the last round's may still be being read)
            odd = __ballot(odd) != 0;
            if (lane == 0) odds[w] = odd;
            __syncthreads();
            odd = false;
#pragma unroll
            for (int i = 0; i < NW; ++i) odd |= odds[i] != 0;
            if (!odd) {
                for (int row = r0; row <= r1; ++row) {
                    if (c >= 0 && r == row) s_tot[c] += x;
                    if (row < r1) __syncthreads();
                }
            } else {
                for (int row = r0; row <= r1; ++row)
                    for (int u = 0; u < a.K; ++u) {
                        if (c >= 0 && r == row && (t < a.K ? t : 0) == u) s_tot[c] += x;
                        __syncthreads();
                    }
            }
        }
    }
    __syncthreads();  // the totals; and every wave has read what the outputs may replace
    const int last = n_candidates(len0 - 1, a.W), able = max(0, last - a.sink);
    const int drop = min(min(max(0, last - a.budget), able), a.most);
    if (tid == 0) {
        a.seqlens_out[b] = len0 - drop * kChunk;
        a.nfreed[b] = drop;
    }
    int32_t* freed = a.freed + (size_t)b * a.most;  // (not touched if most is 0)
    for (int t = drop + tid; t < a.most; t += kEvictBlock) freed[t] = -1;
    if (drop == 0) {
#pragma unroll
        for (int r = 0; r < EPT; ++r) {
            if (r >= nr) continue;
            const int c = first + r * kWave;
            if (c < nC) {
                acc[c] = s_tot[c];
                table[c] = page[r];
            }
        }
        return;
    }
    // keys of the chunks that may go; kStays for the others
    constexpr uint32_t kStays = 0xffffffffu;
    uint32_t key[EPT];
    uint32_t lo = kStays, hi = 0;
#pragma unroll
    for (int r = 0; r < EPT; ++r) {
        const int c = first + r * kWave;
        const bool may = r < nr && c >= a.sink && c < last;
        key[r] = may ? total_key(s_tot[c]) : kStays;
        lo = min(lo, key[r]);
        hi = max(hi, may ? key[r] : 0u);
    }
    // least and greatest key within [from, to]
    auto range = [&]() {
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) {
            lo = min(lo, (uint32_t)__shfl_xor((int)lo, o, kWave));
            hi = max(hi, (uint32_t)__shfl_xor((int)hi, o, kWave));
        }
        if (lane == 0) {
            s_lo[w] = lo;
            s_hi[w] = hi;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            lo = min(lo, s_lo[i]);
            hi = max(hi, s_hi[i]);
        }
    };
    range();
    // The drop-th smallest key, by histograms of 1024 steps of the range that it is in, narrowed to
    // one step until 64 keys are left.  Steps of the totals themselves first: equal steps of their
    // keys, which grow with the logarithm, put most totals into a few of them, and a wave's
    // additions to one counter take one cycle each (16385 chunks: 10 of 27 us).  Any step that
    // grows with the key is as good: what lies below the chosen one goes, above it stays.
    const float f0 = key_total(lo), f1 = key_total(hi);
    bool by_value = f1 - f0 > 0.f && f1 - f0 < INFINITY;  // (not with a NaN or an infinity among them)
    int want = drop, ties;  // the want-th of the keys within [lo, hi]; keys equal to it
    for (;;) {
        const int shift = max(0, 22 - __clz((hi - lo) | 1u));  // (hi - lo) >> shift < 1024
        const float per = 1023.f / (f1 - f0);
        auto step_of = [&](uint32_t k) {
            return by_value ? min(1023, (int)((key_total(k) - f0) * per)) : (int)((k - lo) >> shift);
        };
        s_hist[tid] = 0;
        if (tid == 0) s_in = 0;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < EPT; ++r)
            if (key[r] >= lo && key[r] <= hi) atomicAdd(&s_hist[step_of(key[r])], 1);
        __syncthreads();
        if (w == 0) {
            int h[kSteps / kWave], sum = 0;
#pragma unroll
            for (int i = 0; i < kSteps / kWave; ++i) {
                h[i] = s_hist[lane * (kSteps / kWave) + i];
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
                for (int i = 0; i < kSteps / kWave; ++i) {
                    if (at < want && want <= at + h[i]) {
                        s_step = lane * (kSteps / kWave) + i;
                        s_below = at;
                    }
                    at += h[i];
                }
            }
        }
        __syncthreads();
        const int step = s_step, in = s_hist[step];
        want -= s_below;
        const uint32_t from = lo, to = hi;
        lo = kStays;
        hi = 0;
        if (in <= kWave) {  // few: one wave ranks them
#pragma unroll
            for (int r = 0; r < EPT; ++r)
                if (key[r] >= from && key[r] <= to && (by_value ? step_of(key[r]) : (int)((key[r] - from) >> shift)) == step)
                    s_list[atomicAdd(&s_in, 1)] = key[r];
            __syncthreads();
            const uint32_t mine = s_list[lane];
            int less = 0, upto = 0;
            for (int i = 0; i < in; ++i) {
                const uint32_t x = s_list[i];
                less += x < mine;
                upto += x <= mine;
            }
            const uint64_t hit = __ballot(lane < in && less < want && want <= upto);
            const int src = __ffsll((unsigned long long)hit) - 1;
            lo = (uint32_t)__shfl((int)mine, src, kWave);
            ties = __shfl(upto - less, src, kWave);
            want -= __shfl(less, src, kWave);
            break;
        }
#pragma unroll
        for (int r = 0; r < EPT; ++r)
            if (key[r] >= from && key[r] <= to && (by_value ? step_of(key[r]) : (int)((key[r] - from) >> shift)) == step) {
                lo = min(lo, key[r]);
                hi = max(hi, key[r]);
            }
        range();
        by_value = false;
        if (lo == hi) {
            ties = in;
            break;
        }
    }
    // keys below lo go, and the first `want` of the ties with it
    uint32_t go = 0;  // bit r
    if (ties == want) {
#pragma unroll
        for (int r = 0; r < EPT; ++r) go |= (uint32_t)(key[r] <= lo && key[r] != kStays) << r;
    } else {
        int before = 0, all;
#pragma unroll
        for (int r = 0; r < EPT; ++r) {
            below(key[r] == lo, all);
            before += all;
        }
        if (lane == 0) s_ties[w] = before;
        __syncthreads();
        before = 0;
        for (int i = 0; i < w; ++i) before += s_ties[i];
#pragma unroll
        for (int r = 0; r < EPT; ++r) {
            const bool tie = key[r] == lo;
            const int at = before + below(tie, all);
            before += all;
            go |= (uint32_t)(key[r] < lo || (tie && at < want)) << r;
        }
    }
    int gone = __popc(go), all;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) gone += __shfl_xor(gone, o, kWave);
    if (lane == 0) s_gone[w] = gone;
    __syncthreads();
    gone = 0;
    for (int i = 0; i < w; ++i) gone += s_gone[i];
#pragma unroll
    for (int r = 0; r < EPT; ++r) {
        const int c = first + r * kWave;
        const bool out = (go >> r) & 1u;
        const int at = gone + below(out, all);
        gone += all;
        if (out) {
            freed[at] = page[r];
        } else if (r < nr && c < nC) {
            acc[c - at] = s_tot[c];
            table[c - at] = page[r];
        }
    }
    for (int c = nC - drop + tid; c < nC; c += kEvictBlock) {
        acc[c] = 0.f;
        table[c] = -1;
    }
}

}  // namespace

hipError_t launch_evict(const EvictArgs& a, hipStream_t s) {
    const int nC = a.L / kChunk;
    const dim3 grid(a.B), block(kEvictBlock);
    if (nC <= kEvictBlock)
        HILS_LAUNCH("k_evict", k_evict<1>, grid, block, 0, s, a);
    else if (nC <= 8 * kEvictBlock)
        HILS_LAUNCH("k_evict", k_evict<8>, grid, block, 0, s, a);
    else if (nC <= kMaxHeld)
        HILS_LAUNCH("k_evict", k_evict<20>, grid, block, 0, s, a);
    else
        HILS_LAUNCH("k_evict_long", k_evict_long, grid, block, 0, s, a);
    return hipGetLastError();
}

}  // namespace hils
