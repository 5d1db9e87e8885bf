// Eviction from a paged cache by accumulated attention weight (gfx950).
//
// A chunk's total is the attention weight that it has received: acc[c] += sum over KV groups and
// new queries of the weights that a decode call reported for it.  A sequence that holds more than
// `budget` candidate chunks (those before the last query's window) loses the ones with the least
// totals, ties to the lower index, the first `sink` chunks never.  Its table and totals close up
// over them and its length falls by 64 per chunk: chunks are whole, so every later position keeps
// its place inside its chunk.
//
// One workgroup per sequence; a sequence's totals and table are read and written once (16 bytes
// per chunk) and come from the L2 in between.
#include "hils_dispatch.hpp"
#include "hils_internal.hpp"

namespace hils {

namespace {

constexpr int kEvictBlock = 1024;
constexpr int kEvictWaves = kEvictBlock / kWave;

// How many lanes below have x, and how many of the wave.
__device__ __forceinline__ int below(bool x, int& all) {
    const uint64_t m = __ballot(x);
    all = popc64(m);
    return popc64(m & ((1ull << __lane_id()) - 1ull));
}

__global__ __launch_bounds__(kEvictBlock) void k_evict(EvictArgs a) {
    __shared__ int s_hist[256];
    __shared__ int s_bin, s_k;
    __shared__ int s_tie[kEvictWaves], s_gone[kEvictWaves];
    const int b = blockIdx.x, tid = threadIdx.x, w = wave_id(), lane = tid % kWave;
    const int nC = a.L / kChunk;
    int len = a.seqlens ? a.seqlens[b] : a.L;
    len = len < a.N ? a.N : (len > a.L ? a.L : len);
    const float* acc_in = a.acc + (size_t)b * nC;
    float* acc = a.acc_out + (size_t)b * nC;
    const int32_t* table_in = a.table + (size_t)b * nC;
    int32_t* table = a.table_out + (size_t)b * nC;
    int32_t* freed = a.freed ? a.freed + (size_t)b * a.most : nullptr;

    // ---- the totals ----
    if (acc != acc_in)
        for (int c = tid; c < nC; c += kEvictBlock) acc[c] = acc_in[c];
    __syncthreads();  // (also: every wave has read the length that seqlens_out may replace)
    if (a.weights) {
        const int pieces = (a.W + 62) / kChunk + 1, per = a.K + pieces;
        // row after row, so that a total is one sum in one order; a row names a chunk once
        for (int r = 0; r < a.Hkv * a.N; ++r) {
            const int g = r / a.N, n = r % a.N, pos = len - a.N + n, ncand = n_candidates(pos, a.W);
            const size_t rg = ((size_t)b * a.Hkv + g) * a.N + n;
            for (int t = tid; t < per; t += kEvictBlock) {
                int c = -1;
                if (t < a.K) {
                    if (idx_entry_valid(a.idx + rg * a.K, t, ncand)) c = a.idx[rg * a.K + t];
                } else if (ncand + t - a.K <= pos / kChunk) {
                    c = ncand + t - a.K;
                }
                if (c >= 0) acc[c] += a.weights[rg * per + t];
            }
            __syncthreads();
        }
    }
    const int last = n_candidates(len - 1, a.W), able = max(0, last - a.sink);
    const int drop = min(min(max(0, last - a.budget), able), a.most);
    if (tid == 0) {
        a.seqlens_out[b] = len - drop * kChunk;
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
    // (a total of -0 counts as 0; a NaN is above every number and stays)
    auto key_of = [&](int c) { return ordered_key(acc[c] + 0.f); };
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
        const uint32_t key = ordered_key(total + 0.f);
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

}  // namespace

hipError_t launch_evict(const EvictArgs& a, hipStream_t s) {
    HILS_LAUNCH("k_evict", k_evict, dim3(a.B), dim3(kEvictBlock), 0, s, a);
    return hipGetLastError();
}

}  // namespace hils
