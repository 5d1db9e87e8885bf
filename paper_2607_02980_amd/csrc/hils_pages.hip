// The pages of a cache as a resource: giving sequences pages to write to (copy on write), forking,
// freeing and compacting.  Integers and copies only.
//
// State: a table row of pages per sequence, its length, and page_refs[page], how many table
// entries name the page; a count of 0 (or less) marks a free page.  Every choice is by lowest index
// first, so that results do not depend on the order in which threads run (the counts'
// atomics are integer sums).
#include <algorithm>

#include "hils_device.hpp"
#include "hils_internal.hpp"

namespace hils {

namespace {

constexpr int kThreads = 256;
constexpr int kPlan = 1024;             // threads of the one workgroup that plans
constexpr int kPlanWaves = kPlan / kWave;
constexpr int kPer = 16, kFewPer = 4;   // pages of a thread per step of a scan over the pool (small pools: few)
constexpr size_t kSlice = 16 * 1024;    // bytes of a page that a workgroup copies at a time
constexpr int kPools = 16;              // pools of one copying launch

__device__ __forceinline__ int length_of(const int32_t* seqlens, int b, int L) {
    return seqlens ? min(max(seqlens[b], 0), L) : L;
}
__device__ __forceinline__ int chunks_of(int tokens) { return (tokens + kChunk - 1) / kChunk; }

// Exclusive prefix sum over the planning workgroup; `all` is the total.
__device__ __forceinline__ int block_scan(int x, int* s_sum, int& all) {
    const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave;
    int incl = x;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const int y = __shfl_up(incl, o, kWave);
        if (lane >= o) incl += y;
    }
    __syncthreads();  // the last call's sums have been read
    if (lane == kWave - 1) s_sum[w] = incl;
    __syncthreads();
    int before = incl - x;
    all = 0;
    for (int i = 0; i < kPlanWaves; ++i) {
        before += i < w ? s_sum[i] : 0;
        all += s_sum[i];
    }
    return before;
}

__global__ __launch_bounds__(kThreads) void k_cache_copy_state(const int32_t* table, int32_t* table_out, size_t nt,
                                                              const int32_t* refs, int32_t* refs_out, size_t np) {
    const size_t step = (size_t)gridDim.x * kThreads;
    for (size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x; i < nt; i += step) table_out[i] = table[i];
    for (size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x; i < np; i += step) refs_out[i] = refs[i];
}

// ---------------------------------------------------------------------------
// pages for new tokens
// ---------------------------------------------------------------------------
// One workgroup.  First what every sequence needs: a copy of the page that its first new token
// goes to, if others have it too, and a page for every chunk that begins; then, if the
// pool holds as many, the free pages by index, the r-th for the sequence whose range of needs
// r lies in.  A chain of dependent steps, so what they exchange is in LDS: per sequence a state and where its
// needs begin (more than kLdsSeqs sequences: in `copied`).  64 sequences, 992 pages: 14 us with all of it in
// memory, 8 now.
constexpr int kNone = -1, kNew = -2;  // no page to copy; (kNew: the entry names no page, a fresh one takes its place)
constexpr int kLdsSeqs = 2048;
constexpr size_t kSmallState = 16 * 1024;  // entries of a table and counts that are copied on the way

// The threads' free pages of a step: PER in a row each, as bits.
template <int PER>
__device__ __forceinline__ unsigned free_bits(const int32_t* refs, int P, int p0) {
    unsigned bits = 0;
    int r[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) r[i] = refs[min(p0 + i, P - 1)];
#pragma unroll
    for (int i = 0; i < PER; ++i) bits |= (unsigned)(p0 + i < P && r[i] <= 0) << i;
    return bits;
}

template <bool LDS, int PER>
__global__ __launch_bounds__(kPlan) void k_cache_reserve(ReserveArgs a, size_t nt, size_t np) {
    __shared__ int s_sum[kPlanWaves];
    __shared__ int s_state[LDS ? 2 * kLdsSeqs : 2], s_chunk[LDS ? kLdsSeqs : 1];  // s_chunk: the first need's chunk
    const int tid = threadIdx.x, C = a.L / kChunk;
    int* st = LDS ? s_state : a.copied;  // st[2 b]: page to copy, or kNone, kNew, or -3 - a page of its own; st[2 b + 1]: needs before
    auto seq = [&](int b, int& len, int& start) {
        len = length_of(a.seqlens, b, a.L);
        start = len - min(a.newlens ? min(max(a.newlens[b], 0), a.N) : a.N, len);
    };
    for (size_t i = tid; i < nt; i += kPlan) a.table_out[i] = a.table[i];
    for (size_t i = tid; i < np; i += kPlan) a.refs_out[i] = a.refs[i];
    for (int b = tid; b < a.B; b += kPlan) {
        int len, start, src = kNone;
        seq(b, len, start);
        if (len > start && start % kChunk) {
            src = a.table[(size_t)b * C + start / kChunk];
            if (src < 0 || src >= a.P) src = kNew;
        }
        st[2 * b] = src;
    }
    __syncthreads();
    const unsigned first_bits = free_bits<PER>(a.refs, a.P, tid * PER);
    int total = 0;
    for (int b0 = 0; b0 < a.B; b0 += kPlan) {
        const int b = b0 + tid;
        int need = 0, src = kNone;
        if (b < a.B) {
            int len, start;
            seq(b, len, start);
            src = st[2 * b];
            if (src >= 0) {
                // the first of the sequences that write to the page keeps it if no others have it
                const int refs = a.refs[src];
                int writers = 0;
                bool first = true;
                if (refs > 1)
                    for (int o = 0; o < a.B; ++o) {
                        const int x = st[2 * o];
                        const bool same = x == src || x == -3 - src;
                        writers += same;
                        first = first && !(same && o < b);
                    }
                if (refs <= 1 || (first && writers >= refs)) src = -3 - src;  // its own
            }
            const bool replaced = src >= 0 || src == kNew;  // the page in use comes first
            need = chunks_of(len) - chunks_of(start) + replaced;
            if (LDS) s_chunk[b] = replaced ? start / kChunk : chunks_of(start);
        }
        int all;
        const int before = block_scan(need, s_sum, all);  // (its barriers are behind the loop over the others' states)
        if (b < a.B) {
            if (src < kNew) st[2 * b] = src;
            st[2 * b + 1] = total + before;
        }
        total += all;
    }
    // free pages, up to as many as are needed
    int found = 0, first_before = 0;
    for (int p0 = 0; p0 < a.P && found < total; p0 += kPlan * PER) {
        const unsigned bits = p0 ? free_bits<PER>(a.refs, a.P, p0 + tid * PER) : first_bits;
        int all;
        const int before = block_scan(__popc(bits), s_sum, all);
        if (p0 == 0) first_before = before;
        found += all;
    }
    const bool enough = found >= total;
    if (tid == 0) {
        a.counts[0] = total;
        a.counts[1] = min(found, total);
    }
    if (!enough) {
        __syncthreads();
        for (int b = tid; b < a.B; b += kPlan) a.copied[2 * b] = a.copied[2 * b + 1] = -1;
        return;
    }
    __syncthreads();
    int given = 0;
    for (int p0 = 0; p0 < a.P && given < total; p0 += kPlan * PER) {
        unsigned bits = first_bits;
        int all = 0, r = first_before;
        if (p0 || a.P > kPlan * PER) {
            bits = free_bits<PER>(a.refs, a.P, p0 + tid * PER);
            r = given + block_scan(__popc(bits), s_sum, all);
        }
        given += all;
        for (; bits && r < total; bits &= bits - 1, ++r) {
            const int p = p0 + tid * PER + __ffs(bits) - 1;
            int lo = 0, hi = a.B - 1;  // the last sequence whose needs begin at or before r
            while (lo < hi) {
                const int mid = (lo + hi + 1) / 2;
                if (st[2 * mid + 1] <= r)
                    lo = mid;
                else
                    hi = mid - 1;
            }
            int c0;
            if constexpr (LDS) {
                c0 = s_chunk[lo];
            } else {
                int len, start;
                seq(lo, len, start);
                c0 = st[2 * lo] >= 0 || st[2 * lo] == kNew ? start / kChunk : chunks_of(start);
            }
            a.table_out[(size_t)lo * C + c0 + r - st[2 * lo + 1]] = p;
            a.refs_out[p] = 1;
        }
    }
    __syncthreads();
    for (int b = tid; b < a.B; b += kPlan) {
        const int src = st[2 * b];
        int len, start;
        seq(b, len, start);
        if (src >= 0) atomicSub(&a.refs_out[src], 1);
        const int dst = src >= 0 ? a.table_out[(size_t)b * C + start / kChunk] : -1;
        a.copied[2 * b] = src >= 0 ? src : -1;
        a.copied[2 * b + 1] = dst;
    }
}

// ---------------------------------------------------------------------------
// copies of pages
// ---------------------------------------------------------------------------
struct PoolList {
    char* data[kPools];
    size_t bytes[kPools];
    int slices[kPools + 1];  // slices of the pools before
    int n;
};
// Copy i of *count (or n_max): page from[i * stride] to page to[...]; MAP: to[the source page].
struct CopyList {
    const int32_t* from;
    const int32_t* to;
    const int32_t* count;  // nullable: n_max
    int n_max, stride, map;
};
__device__ __forceinline__ void copy_listed(const PoolList& pools, const CopyList& list, int P) {
    const int n = list.count ? min(*list.count, list.n_max) : list.n_max;
    const int per = pools.slices[pools.n];
    for (size_t u = blockIdx.x; u < (size_t)n * per; u += gridDim.x) {
        const int i = (int)(u / per), part = (int)(u % per);
        const int src = list.from[(size_t)i * list.stride];
        if (src < 0 || src >= P) continue;
        const int dst = list.map ? list.to[src] : list.to[(size_t)i * list.stride];
        if (dst < 0 || dst >= P) continue;
        int k = 0;
        while (part >= pools.slices[k + 1]) ++k;
        const size_t bytes = pools.bytes[k], at = (size_t)(part - pools.slices[k]) * kSlice;
        const size_t len = min(kSlice, bytes - at);
        const char* x = pools.data[k] + (size_t)src * bytes + at;
        char* y = pools.data[k] + (size_t)dst * bytes + at;
        if ((((size_t)pools.data[k] | bytes) & 15) == 0) {
            // (non-temporal stores leave the caches to the reads: 350 pages of 270 KB 47.5 -> 39.3 us a call; the loads
            // too: 42.5, the loads alone: 39.8)
            typedef int v4i __attribute__((ext_vector_type(4)));
            for (size_t j = threadIdx.x; j < len / 16; j += kThreads)
                __builtin_nontemporal_store(reinterpret_cast<const v4i*>(x)[j], reinterpret_cast<v4i*>(y) + j);
        } else if ((((size_t)pools.data[k] | bytes) & 3) == 0) {
            for (size_t j = threadIdx.x; j < len / 4; j += kThreads)
                reinterpret_cast<uint32_t*>(y)[j] = reinterpret_cast<const uint32_t*>(x)[j];
        } else {
            for (size_t j = threadIdx.x; j < len; j += kThreads) y[j] = x[j];
        }
    }
}

__global__ __launch_bounds__(kThreads) void k_cache_copy_pages(PoolList pools, CopyList list, int P) {
    copy_listed(pools, list, P);
}

// ---------------------------------------------------------------------------
// forking
// ---------------------------------------------------------------------------
__device__ __forceinline__ void fork_rows(const ForkArgs& a, size_t at, size_t step) {
    const int C = a.L / kChunk;
    for (size_t i = at; i < (size_t)a.rows * C; i += step) {
        const int b = (int)(i / C), c = (int)(i % C), u = a.parent[b];
        const bool lives = u >= 0 && u < a.B;
        const int len = lives ? length_of(a.seqlens, u, a.L) : 0;
        a.table_out[i] = c < chunks_of(len) ? a.table[(size_t)u * C + c] : -1;
        if (c == 0) a.seqlens_out[b] = len;
    }
    if (a.refs_out != a.refs)
        for (size_t i = at; i < (size_t)a.P; i += step) a.refs_out[i] = a.refs[i];
}
__device__ __forceinline__ void add_refs(const ForkArgs& a, size_t entry, int change) {
    const int p = a.table[entry];
    if (change != 0 && p >= 0 && p < a.P) atomicAdd(&a.refs_out[p], change);
}
__global__ __launch_bounds__(kThreads) void k_cache_fork_rows(ForkArgs a) {
    fork_rows(a, (size_t)blockIdx.x * kThreads + threadIdx.x, (size_t)gridDim.x * kThreads);
}
// A workgroup per (input row, range of its chunks): the row's pages gain a reference for every
// row that goes on from it and lose the row's own.
__global__ __launch_bounds__(kThreads) void k_cache_fork_refs(ForkArgs a, int per) {
    __shared__ int s_times;
    const int b = blockIdx.y, C = a.L / kChunk, n = chunks_of(length_of(a.seqlens, b, a.L));
    const int c0 = blockIdx.x * per;
    if (c0 >= n) return;
    if (threadIdx.x == 0) s_times = 0;
    __syncthreads();
    int t = 0;
    for (int i = threadIdx.x; i < a.rows; i += kThreads) t += a.parent[i] == b;
    if (t) atomicAdd(&s_times, t);
    __syncthreads();
    const int change = s_times - 1;
    if (change == 0) return;
    for (int c = c0 + threadIdx.x; c < min(n, c0 + per); c += kThreads) add_refs(a, (size_t)b * C + c, change);
}
// Both in one workgroup, for few entries: a call is the host's time then, 2 us a launch (32 beams, 9K
// entries and counts: 10.3 us a call with two launches, 8.7 with one).
constexpr int kSmallRows = 1024;
__global__ __launch_bounds__(kPlan) void k_cache_fork(ForkArgs a) {
    __shared__ int s_change[kSmallRows];
    const int tid = threadIdx.x, C = a.L / kChunk;
    for (int b = tid; b < a.B; b += kPlan) s_change[b] = -1;
    fork_rows(a, tid, kPlan);
    __syncthreads();
    for (int i = tid; i < a.rows; i += kPlan) {
        const int u = a.parent[i];
        if (u >= 0 && u < a.B) atomicAdd(&s_change[u], 1);
    }
    __syncthreads();
    for (int i = tid; i < a.B * C; i += kPlan) {
        const int b = i / C;
        if (i % C < chunks_of(length_of(a.seqlens, b, a.L))) add_refs(a, i, s_change[b]);
    }
}

// ---------------------------------------------------------------------------
// freeing
// ---------------------------------------------------------------------------
__device__ __forceinline__ void lose_ref(const FreeArgs& a, int p) {
    if (p >= 0 && p < a.P) atomicSub(&a.refs_out[p], 1);
}
// Entry i of the table, of a row with chunks beg .. end - 1 to give up.
__device__ __forceinline__ void free_entry(const FreeArgs& a, size_t i, int c, int beg, int end) {
    const int p = a.table[i];
    const bool gone = c >= beg && c < end;
    if (gone) lose_ref(a, p);
    if (gone || a.table_out != a.table) a.table_out[i] = gone ? -1 : p;
}
// A workgroup per sequence (a length may be overwritten in place: read once, first).
__global__ __launch_bounds__(kPlan) void k_cache_free(FreeArgs a) {
    const int b = blockIdx.x, C = a.L / kChunk;
    const int len = length_of(a.seqlens, b, a.L), kept = min(len, max(a.keep[b], 0));
    __syncthreads();
    if (threadIdx.x == 0) a.seqlens_out[b] = kept;
    const int beg = chunks_of(kept), end = chunks_of(len);
    for (int c = threadIdx.x; c < C; c += kPlan) free_entry(a, (size_t)b * C + c, c, beg, end);
    if (a.pages) {
        const int n = a.npages ? min(max(a.npages[b], 0), a.most) : a.most;
        for (int i = threadIdx.x; i < n; i += kPlan) lose_ref(a, a.pages[(size_t)b * a.most + i]);
    }
}
// All sequences in one workgroup and the counts copied on the way, for few entries (as k_cache_fork; 64
// sequences, 11K entries and counts: 10.5 us a call with two launches, 8.6 with one).
__global__ __launch_bounds__(kPlan) void k_cache_free_small(FreeArgs a) {
    __shared__ int s_beg[kSmallRows], s_end[kSmallRows];
    const int tid = threadIdx.x, C = a.L / kChunk;
    for (int b = tid; b < a.B; b += kPlan) {
        const int len = length_of(a.seqlens, b, a.L), kept = min(len, max(a.keep[b], 0));
        s_beg[b] = chunks_of(kept);
        s_end[b] = chunks_of(len);
        a.seqlens_out[b] = kept;
    }
    for (int i = tid; i < a.P; i += kPlan) a.refs_out[i] = a.refs[i];
    __syncthreads();
    for (int i = tid; i < a.B * C; i += kPlan) free_entry(a, i, i % C, s_beg[i / C], s_end[i / C]);
    if (a.pages)
        for (int i = tid; i < a.B * a.most; i += kPlan)
            if (!a.npages || i % a.most < a.npages[i / a.most]) lose_ref(a, a.pages[i]);
}

// ---------------------------------------------------------------------------
// compacting
// ---------------------------------------------------------------------------
// One workgroup: n pages are in use; the i-th used page at or past n goes to the i-th free one
// before it.  Both lists are as long, at most half of the pool: the free pages are listed in the
// second half of `moved` until the pairs are made.
template <int PER>
__global__ __launch_bounds__(kPlan) void k_cache_compact(CompactArgs a) {
    __shared__ int s_sum[kPlanWaves];
    const int tid = threadIdx.x, half = (a.P + 1) / 2;
    int used = 0;
    for (int p0 = 0; p0 < a.P; p0 += kPlan * PER) {
        int all;
        (void)block_scan(__popc(free_bits<PER>(a.refs, a.P, p0 + tid * PER)), s_sum, all);
        used += min(a.P - p0, kPlan * PER) - all;
    }
    int movers = 0, holes = 0;
    for (int p0 = 0; p0 < a.P; p0 += kPlan * PER) {
        int r[PER], n = 0, h = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) r[i] = a.refs[min(p0 + tid * PER + i, a.P - 1)];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int p = p0 + tid * PER + i;
            n += p < a.P && p >= used && r[i] > 0;
            h += p < used && r[i] <= 0;
        }
        int all;  // (both at once: a step has at most 2^14 of each)
        const int before = block_scan(n << 16 | h, s_sum, all);
        int at = movers + (before >> 16), to = holes + (before & 0xffff);
        movers += all >> 16;
        holes += all & 0xffff;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int p = p0 + tid * PER + i;
            if (p >= a.P) continue;
            a.new_page[p] = r[i] > 0 ? p : -1;
            // (in place too: all have counted the used pages by now, and from here each thread uses its own counts only)
            if (a.refs_out != a.refs || r[i] < 0) a.refs_out[p] = max(r[i], 0);
            if (p >= used && r[i] > 0) a.moved[at++] = p;
            if (p < used && r[i] <= 0) a.moved[half + to++] = p;
        }
    }
    __syncthreads();
    for (int i = tid; i < movers; i += kPlan) {
        const int src = a.moved[i], dst = a.moved[half + i];
        a.new_page[src] = dst;
        const int r = a.refs_out[src];  // (a copy of refs, or refs themselves)
        a.refs_out[dst] = r;
        a.refs_out[src] = 0;
    }
    __syncthreads();
    for (int i = movers + tid; i < a.P; i += kPlan) a.moved[i] = -1;
    if (tid == 0) {
        a.counts[0] = used;
        a.counts[1] = movers;
    }
}
// The tables follow the pages, and (the first pools of) the pages move.
__global__ __launch_bounds__(kThreads) void k_cache_move(CompactArgs a, PoolList pools, CopyList list) {
    const int C = a.L / kChunk;
    const size_t step = (size_t)gridDim.x * kThreads;
    for (size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x; i < (size_t)a.B * C; i += step) {
        const int b = (int)(i / C), c = (int)(i % C), p = a.table[i];
        const bool held = c < chunks_of(length_of(a.seqlens, b, a.L)) && p >= 0 && p < a.P;
        a.table_out[i] = held ? a.new_page[p] : p;
    }
    copy_listed(pools, list, a.P);
}

unsigned blocks_for(size_t items, size_t per = kThreads, size_t most = 4096) {
    return (unsigned)std::max<size_t>(1, std::min(most, (items + per - 1) / per));
}

PoolList pool_list(const PoolArg* pools, int n) {
    PoolList x;
    x.n = n;
    x.slices[0] = 0;
    for (int k = 0; k < n; ++k) {
        x.data[k] = static_cast<char*>(pools[k].data);
        x.bytes[k] = pools[k].page_bytes;
        x.slices[k + 1] = x.slices[k] + (int)((x.bytes[k] + kSlice - 1) / kSlice);
    }
    return x;
}
unsigned copy_blocks(const PoolList& x, const CopyList& list) {
    return blocks_for((size_t)list.n_max * x.slices[x.n], 1, 8 * (size_t)device_cus());
}
void copy_pages(const PoolArg* pools, int num_pools, int P, const CopyList& list, hipStream_t s) {
    for (int k = 0; k < num_pools; k += kPools) {
        const PoolList x = pool_list(pools + k, std::min(kPools, num_pools - k));
        HILS_LAUNCH("k_cache_copy_pages", k_cache_copy_pages, dim3(copy_blocks(x, list)), dim3(kThreads), 0, s, x, list, P);
    }
}

}  // namespace

hipError_t launch_reserve(const ReserveArgs& a, const PoolArg* pools, int num_pools, hipStream_t s) {
    size_t nt = a.table_out != a.table ? (size_t)a.B * (a.L / kChunk) : 0;
    size_t np = a.refs_out != a.refs ? (size_t)a.P : 0;
    const bool small = nt + np <= kSmallState;
    if (!small)
        HILS_LAUNCH("k_cache_copy_state", k_cache_copy_state, dim3(blocks_for(std::max(nt, np))), dim3(kThreads), 0, s,
                    a.table, a.table_out, nt, a.refs, a.refs_out, np);
    nt = small ? nt : 0;
    np = small ? np : 0;
    if (a.B > kLdsSeqs)
        HILS_LAUNCH("k_cache_reserve", (k_cache_reserve<false, kPer>), dim3(1), dim3(kPlan), 0, s, a, nt, np);
    else if (a.P > kFewPer * kPlan)
        HILS_LAUNCH("k_cache_reserve", (k_cache_reserve<true, kPer>), dim3(1), dim3(kPlan), 0, s, a, nt, np);
    else
        HILS_LAUNCH("k_cache_reserve", (k_cache_reserve<true, kFewPer>), dim3(1), dim3(kPlan), 0, s, a, nt, np);
    copy_pages(pools, num_pools, a.P, CopyList{a.copied, a.copied + 1, nullptr, a.B, 2, 0}, s);
    return hipGetLastError();
}

hipError_t launch_fork(const ForkArgs& a, hipStream_t s) {
    const int C = a.L / kChunk;
    const size_t np = a.refs_out != a.refs ? (size_t)a.P : 0, items = std::max((size_t)a.rows * C, np);
    if (((size_t)a.rows + a.B) * C + np <= kSmallState && a.B <= kSmallRows && a.rows <= (int)kSmallState) {
        HILS_LAUNCH("k_cache_fork", k_cache_fork, dim3(1), dim3(kPlan), 0, s, a);
        return hipGetLastError();
    }
    HILS_LAUNCH("k_cache_fork_rows", k_cache_fork_rows, dim3(blocks_for(items)), dim3(kThreads), 0, s, a);
    const int per = 4 * kThreads;
    HILS_LAUNCH("k_cache_fork_refs", k_cache_fork_refs, dim3((C + per - 1) / per, a.B), dim3(kThreads), 0, s, a, per);
    return hipGetLastError();
}

hipError_t launch_free(const FreeArgs& a, hipStream_t s) {
    const size_t np = a.refs_out != a.refs ? (size_t)a.P : 0;
    if (np && a.B <= kSmallRows && (size_t)a.B * (a.L / kChunk) + np + (size_t)a.B * a.most <= kSmallState) {
        HILS_LAUNCH("k_cache_free", k_cache_free_small, dim3(1), dim3(kPlan), 0, s, a);
        return hipGetLastError();
    }
    if (np)
        HILS_LAUNCH("k_cache_copy_state", k_cache_copy_state, dim3(blocks_for(np)), dim3(kThreads), 0, s, a.table,
                    a.table_out, (size_t)0, a.refs, a.refs_out, np);
    HILS_LAUNCH("k_cache_free", k_cache_free, dim3(a.B), dim3(kPlan), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_compact(const CompactArgs& a, const PoolArg* pools, int num_pools, hipStream_t s) {
    if (a.P > kFewPer * kPlan)
        HILS_LAUNCH("k_cache_compact", k_cache_compact<kPer>, dim3(1), dim3(kPlan), 0, s, a);
    else
        HILS_LAUNCH("k_cache_compact", k_cache_compact<kFewPer>, dim3(1), dim3(kPlan), 0, s, a);
    const CopyList list{a.moved, a.new_page, a.counts + 1, a.P / 2, 1, 1};
    const int first = std::min(num_pools, kPools);
    const PoolList x = pool_list(pools, first);
    HILS_LAUNCH("k_cache_move", k_cache_move, dim3(std::max(blocks_for((size_t)a.B * (a.L / kChunk)), copy_blocks(x, list))),
                dim3(kThreads), 0, s, a, x, list);
    copy_pages(pools + first, num_pools - first, a.P, list, s);
    return hipGetLastError();
}

}  // namespace hils
