// C-ABI of libhils.so: argument validation, workspace sizing and dispatch.
// Every check runs on the host before any HIP call.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <string>
#include <vector>

#include "../../include/hils.h"
#include "hils_internal.hpp"

namespace {

thread_local std::string g_err;

struct TimedLaunch {
    const char* name;
    hipEvent_t e0, e1;
};
thread_local bool g_timing = false;
thread_local std::vector<TimedLaunch> g_launches;

void release_launches() {
    for (auto& t : g_launches) {
        (void)hipEventDestroy(t.e0);
        (void)hipEventDestroy(t.e1);
    }
    g_launches.clear();
}

int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int fail(int code, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    g_err = buf;
    return code;
}

int ok() {
    g_err.clear();
    return HILS_OK;
}

int check_params(const hils_params* p, int op) {
    if (!p) return fail(HILS_ERR_INVALID, "params is NULL");
    if (op < HILS_OP_PREFILL || op > HILS_OP_CACHE_COMPACT)
        return fail(HILS_ERR_INVALID, "unknown op %d", op);
    if (p->B < 1 || p->Hq < 1 || p->Hkv < 1 || p->N < 1 || p->L < 1 || p->d < 1)
        return fail(HILS_ERR_INVALID, "B, Hq, Hkv, N, L and d must be >= 1 (B=%d Hq=%d Hkv=%d N=%d L=%d d=%d)",
                    p->B, p->Hq, p->Hkv, p->N, p->L, p->d);
    if (p->chunk < 1 || p->topk < 1 || p->window < 1)
        return fail(HILS_ERR_INVALID, "chunk, topk and window must be >= 1 (chunk=%d topk=%d window=%d)", p->chunk,
                    p->topk, p->window);
    if (p->Hq % p->Hkv) return fail(HILS_ERR_INVALID, "Hq=%d is not a multiple of Hkv=%d", p->Hq, p->Hkv);
    if (p->Hl != p->Hq && p->Hl != p->Hkv)
        return fail(HILS_ERR_INVALID, "Hl=%d must equal Hq=%d or Hkv=%d", p->Hl, p->Hq, p->Hkv);
    if (p->L % p->chunk) return fail(HILS_ERR_INVALID, "L=%d is not a multiple of chunk=%d", p->L, p->chunk);
    // the field's bits as an int: a C caller may store any value there, and loading
    // one outside the enumerators as the enum type is undefined in C++
    int dtype_raw = 0;
    static_assert(sizeof(p->dtype) == sizeof(int), "hils_dtype has the size of an int");
    memcpy(&dtype_raw, &p->dtype, sizeof dtype_raw);
    if (dtype_raw != HILS_F32 && dtype_raw != HILS_BF16) return fail(HILS_ERR_INVALID, "unknown dtype %d", dtype_raw);
    if (!isfinite(p->scale)) return fail(HILS_ERR_INVALID, "scale is not finite");
    if (p->flags & ~(HILS_FLAG_GIVEN_IDX | HILS_FLAG_SHARED_LMK_QUERY | HILS_FLAG_HEAD_NORM_SELECT |
                     HILS_FLAG_UNION_PACKING))
        return fail(HILS_ERR_INVALID, "unknown flags 0x%x", p->flags);
    const bool pages = op >= HILS_OP_CACHE_RESERVE;
    const bool q8_cache = op == HILS_OP_Q8_APPEND || op == HILS_OP_Q8_LANDMARK || op == HILS_OP_CACHE_EVICT || pages;
    // (the cache's own operators take the decode call's parameters, whose forward flags mean nothing to them)
    const unsigned q8_flags = op == HILS_OP_Q8_LANDMARK ? HILS_FLAG_SHARED_LMK_QUERY
                              : op == HILS_OP_CACHE_EVICT || pages
                                  ? HILS_FLAG_GIVEN_IDX | HILS_FLAG_HEAD_NORM_SELECT | HILS_FLAG_UNION_PACKING
                                  : 0u;
    if (q8_cache && (p->flags & ~q8_flags))
        return fail(HILS_ERR_INVALID, "flags 0x%x do not apply to this entry point", p->flags);
    if ((p->flags & HILS_FLAG_HEAD_NORM_SELECT) && op == HILS_OP_LANDMARK)
        return fail(HILS_ERR_INVALID, "HILS_FLAG_HEAD_NORM_SELECT does not apply to the landmark compression");
    if ((p->flags & HILS_FLAG_SHARED_LMK_QUERY) && op != HILS_OP_LANDMARK && op != HILS_OP_Q8_LANDMARK)
        return fail(HILS_ERR_INVALID, "HILS_FLAG_SHARED_LMK_QUERY applies to the landmark compression only");
    if ((p->flags & HILS_FLAG_GIVEN_IDX) && op == HILS_OP_LANDMARK)
        return fail(HILS_ERR_INVALID, "HILS_FLAG_GIVEN_IDX does not apply to the landmark compression");
    const bool decode = op == HILS_OP_DECODE || op == HILS_OP_DECODE_Q8;
    if (q8_cache && p->N > p->L)
        return fail(HILS_ERR_INVALID, "N <= L new tokens per sequence are needed (N=%d L=%d)", p->N, p->L);
    if (decode && p->N > p->L)
        return fail(HILS_ERR_INVALID, "decode needs N <= L new queries per sequence (N=%d L=%d)", p->N, p->L);
    if (decode && (long)p->B * p->N > 65535)
        return fail(HILS_ERR_INVALID, "decode needs B * N <= 65535 (B=%d N=%d)", p->B, p->N);
    if (!decode && !q8_cache && op != HILS_OP_LANDMARK && p->N > p->L)
        return fail(HILS_ERR_INVALID, "prefill/backward need N <= L (N=%d L=%d)", p->N, p->L);
    if (p->B > 65535 || p->Hkv > 65535) return fail(HILS_ERR_INVALID, "B and Hkv must be <= 65535");
    if (op == HILS_OP_BWD && (p->flags & HILS_FLAG_GIVEN_IDX))
        return fail(HILS_ERR_INVALID, "HILS_FLAG_GIVEN_IDX is a forward flag (the backward always reads idx)");
    // kernel coverage
    if (p->chunk != 64) return fail(HILS_ERR_UNSUPPORTED, "chunk=%d: kernels exist for chunk 64 only", p->chunk);
    if (p->d != 64 && p->d != 128) return fail(HILS_ERR_UNSUPPORTED, "d=%d: kernels exist for d in {64, 128}", p->d);
    const int G = p->Hq / p->Hkv;
    if (G != 1 && G != 2 && G != 4 && G != 8)
        return fail(HILS_ERR_UNSUPPORTED, "group size G=%d: kernels exist for G in {1, 2, 4, 8}", G);
    if (p->topk > 64) return fail(HILS_ERR_UNSUPPORTED, "topk=%d: kernels exist for topk <= 64", p->topk);
    if ((decode || op == HILS_OP_CACHE_EVICT) && p->window > 4032)
        return fail(HILS_ERR_UNSUPPORTED, "window=%d: the decode kernels cover windows <= 4032", p->window);
    if (op == HILS_OP_DECODE_Q8 && (p->flags & HILS_FLAG_HEAD_NORM_SELECT))
        return fail(HILS_ERR_UNSUPPORTED, "HILS_FLAG_HEAD_NORM_SELECT: no kernel over the 8-bit cache");
    if (op == HILS_OP_PREFILL_PAGED && (p->flags & HILS_FLAG_HEAD_NORM_SELECT))
        return fail(HILS_ERR_UNSUPPORTED, "HILS_FLAG_HEAD_NORM_SELECT: no kernel for new tokens over a paged cache");
    // (64 threads a row, or 64 entries, in one-dimensional grids)
    if (op == HILS_OP_PREFILL_PAGED && 64. * p->B * p->Hkv * (p->N + 127.) > 4294967295.)
        return fail(HILS_ERR_UNSUPPORTED, "B=%d Hkv=%d N=%d: more workgroups than one grid holds", p->B, p->Hkv, p->N);
    return HILS_OK;
}

size_t ws_bytes_for(const hils_params* p, int op) {
    switch (op) {
        case HILS_OP_LANDMARK:
            return hils::landmark_workspace_bytes(p->B, p->Hl, p->L / p->chunk, p->d,
                                                  (p->flags & HILS_FLAG_SHARED_LMK_QUERY) != 0);
        case HILS_OP_BWD:
            if (p->dtype == HILS_BF16)
                return hils::bwd_mfma_workspace_bytes(p->B, p->Hq, p->Hkv, p->N, p->L, p->d, p->topk);
            return hils::bwd_f32_workspace_bytes(p->B, p->Hq, p->Hkv, p->N, p->L, p->d, p->topk, p->window);
        case HILS_OP_DECODE:
            return hils::decode_workspace_bytes(p->B, p->N, p->Hkv, p->Hq / p->Hkv, p->d, p->L, p->topk, p->window,
                                                (p->flags & HILS_FLAG_HEAD_NORM_SELECT) != 0);
        case HILS_OP_DECODE_Q8:
            return hils::q8_decode_workspace_bytes(p->B, p->N, p->Hkv, p->Hq / p->Hkv, p->d, p->L, p->topk, p->window);
        case HILS_OP_Q8_APPEND:
        case HILS_OP_Q8_LANDMARK:
        case HILS_OP_CACHE_EVICT:
        case HILS_OP_CACHE_RESERVE:
        case HILS_OP_CACHE_FORK:
        case HILS_OP_CACHE_FREE:
        case HILS_OP_CACHE_COMPACT:
            return 0;
        case HILS_OP_PREFILL_PAGED:
            return hils::prefill_paged_workspace_bytes(p->B, p->Hq, p->Hkv, p->N, p->L, p->d, p->topk,
                                                       p->window, p->dtype == HILS_BF16);
        default:
            return hils::prefill_workspace_bytes(p->B, p->Hq, p->Hkv, p->N, p->L, p->d, p->topk,
                                                 p->dtype == HILS_BF16,
                                                 (p->flags & HILS_FLAG_UNION_PACKING) != 0);
    }
}

int check_ws(const hils_params* p, int op, const void* ws, size_t bytes) {
    const size_t need = ws_bytes_for(p, op);
    if (need == 0) return HILS_OK;
    if (!ws) return fail(HILS_ERR_WORKSPACE, "workspace is NULL but %zu bytes are needed", need);
    if (bytes < need) return fail(HILS_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", bytes, need);
    return HILS_OK;
}

int hip_status(hipError_t e, const char* what) {
    if (e != hipSuccess) return fail(HILS_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
    return ok();
}

#define REQUIRE(ptr) \
    if (!(ptr)) return fail(HILS_ERR_INVALID, "required pointer '%s' is NULL", #ptr)

#define REQUIRE_ALIGNED(ptr, n) \
    if ((uintptr_t)(ptr) % (n)) return fail(HILS_ERR_INVALID, "'%s' is not %d-byte aligned", #ptr, n)

// Workgroups of 256 threads in a one-dimensional grid.
int check_q8_grid(const hils_params* p, double blocks) {
    if (blocks > 0xffffff)  // 2^32 threads
        return fail(HILS_ERR_UNSUPPORTED, "B=%d Hkv=%d N=%d: more workgroups than one grid holds", p->B, p->Hkv, p->N);
    return HILS_OK;
}

hils::FwdArgs fwd_args(const hils_params* p, const void* q, const void* k, const void* v, const void* lmk,
                       const float* bias, const void* q_route, const int32_t* seqlens, void* out, float* lse,
                       int32_t* idx, void* ws, size_t ws_bytes) {
    hils::FwdArgs a;
    a.q = q; a.k = k; a.v = v; a.lmk = lmk; a.bias = bias; a.q_route = q_route; a.seqlens = seqlens;
    a.block_table = nullptr; a.num_pages = 0;
    a.out = out; a.lse = lse; a.idx = idx;
    a.B = p->B; a.Hq = p->Hq; a.Hkv = p->Hkv; a.Hl = p->Hl; a.N = p->N; a.L = p->L; a.d = p->d;
    a.K = p->topk; a.W = p->window; a.scale = p->scale;
    a.bf16 = p->dtype == HILS_BF16;
    a.given_idx = (p->flags & HILS_FLAG_GIVEN_IDX) ? 1 : 0;
    a.head_norm = (p->flags & HILS_FLAG_HEAD_NORM_SELECT) ? 1 : 0;
    a.union_pack = (p->flags & HILS_FLAG_UNION_PACKING) ? 1 : 0;
    a.ws = ws; a.ws_bytes = ws_bytes;
    return a;
}

// Pools that a call copies pages of; the launchers take them as they are.
static_assert(sizeof(hils_pool) == sizeof(hils::PoolArg) && offsetof(hils_pool, data) == offsetof(hils::PoolArg, data) &&
                  offsetof(hils_pool, page_bytes) == offsetof(hils::PoolArg, page_bytes),
              "a pool has one layout");
int check_page_count(int num_pages) {
    if (num_pages < 1) return fail(HILS_ERR_INVALID, "num_pages must be >= 1 (got %d)", num_pages);
    if (num_pages > 1 << 30) return fail(HILS_ERR_UNSUPPORTED, "num_pages=%d: more than 2^30", num_pages);
    return HILS_OK;
}
int check_pools(const hils_pool* pools, int num_pools) {
    if (num_pools < 0 || num_pools > 65536)
        return fail(HILS_ERR_INVALID, "num_pools=%d: 0 to 65536 are possible", num_pools);
    if (num_pools > 0 && !pools) return fail(HILS_ERR_INVALID, "num_pools=%d, so pools must be non-NULL", num_pools);
    for (int i = 0; i < num_pools; ++i) {
        if (!pools[i].data) return fail(HILS_ERR_INVALID, "pool %d is NULL", i);
        if (pools[i].page_bytes == 0 || pools[i].page_bytes > ((size_t)1 << 32))
            return fail(HILS_ERR_INVALID, "pool %d: a page has %zu bytes (1 to 2^32 are possible)", i, pools[i].page_bytes);
    }
    return HILS_OK;
}

}  // namespace

namespace hils {
bool timing_on() { return g_timing; }
void timing_begin(const char* name, hipStream_t s) {
    TimedLaunch t{name, nullptr, nullptr};
    if (hipEventCreate(&t.e0) != hipSuccess || hipEventCreate(&t.e1) != hipSuccess) return;
    (void)hipEventRecord(t.e0, s);
    g_launches.push_back(t);
}
void timing_end(hipStream_t s) {
    if (!g_launches.empty()) (void)hipEventRecord(g_launches.back().e1, s);
}
}  // namespace hils

extern "C" {

int hils_timing_enable(int on) {
    g_timing = on != 0;
    if (!g_timing) release_launches();
    return ok();
}

int hils_timing_read(char* names, size_t names_len, float* total_ms, int* launches, int max_kernels,
                     int* n_kernels) {
    if (!n_kernels) return fail(HILS_ERR_INVALID, "n_kernels is NULL");
    std::vector<std::string> order;
    std::vector<float> tot;
    std::vector<int> cnt;
    for (auto& t : g_launches) {
        float ms = 0.f;
        if (hipEventSynchronize(t.e1) != hipSuccess || hipEventElapsedTime(&ms, t.e0, t.e1) != hipSuccess) {
            release_launches();
            return fail(HILS_ERR_HIP, "reading kernel timing events failed");
        }
        size_t k = 0;
        while (k < order.size() && order[k] != t.name) ++k;
        if (k == order.size()) {
            order.push_back(t.name);
            tot.push_back(0.f);
            cnt.push_back(0);
        }
        tot[k] += ms;
        cnt[k] += 1;
    }
    release_launches();
    *n_kernels = (int)order.size();
    std::string joined;
    for (size_t k = 0; k < order.size() && (int)k < max_kernels; ++k) {
        if (total_ms) total_ms[k] = tot[k];
        if (launches) launches[k] = cnt[k];
        joined += order[k];
        joined += '\n';
    }
    if (names && names_len) {
        const size_t n = joined.size() < names_len - 1 ? joined.size() : names_len - 1;
        memcpy(names, joined.data(), n);
        names[n] = 0;
    }
    return ok();
}


int hils_version(void) { return 100; }

size_t hils_prefill_record_cap(size_t bytes) { return hils::prefill_record_cap(bytes); }

const char* hils_last_error(void) { return g_err.c_str(); }

int hils_workspace_size(const hils_params* p, int op, size_t* bytes) {
    int rc = check_params(p, op);
    if (rc) return rc;
    if (!bytes) return fail(HILS_ERR_INVALID, "bytes is NULL");
    *bytes = ws_bytes_for(p, op);
    return ok();
}

int hils_prefill_fwd(const hils_params* p, const void* q, const void* k, const void* v, const void* lmk,
                     const float* lmk_bias, const void* q_route, void* out, float* lse, int32_t* idx,
                     void* workspace, size_t ws_bytes, void* stream) {
    int rc = check_params(p, HILS_OP_PREFILL);
    if (rc) return rc;
    REQUIRE(q); REQUIRE(k); REQUIRE(v); REQUIRE(lmk); REQUIRE(out); REQUIRE(lse); REQUIRE(idx);
    rc = check_ws(p, HILS_OP_PREFILL, workspace, ws_bytes);
    if (rc) return rc;
    const hils::FwdArgs a = fwd_args(p, q, k, v, lmk, lmk_bias, q_route, nullptr, out, lse, idx, workspace,
                                     ws_bytes);
    return hip_status(hils::launch_prefill_fwd(a, (hipStream_t)stream), "hils_prefill_fwd launch");
}

int hils_decode_fwd(const hils_params* p, const void* q, const void* k_cache, const void* v_cache,
                    const void* lmk_cache, const float* lmk_bias, const void* q_route, const int32_t* seqlens,
                    void* out, float* lse, int32_t* idx, void* workspace, size_t ws_bytes, void* stream) {
    int rc = check_params(p, HILS_OP_DECODE);
    if (rc) return rc;
    REQUIRE(q); REQUIRE(k_cache); REQUIRE(v_cache); REQUIRE(lmk_cache); REQUIRE(out); REQUIRE(lse); REQUIRE(idx);
    rc = check_ws(p, HILS_OP_DECODE, workspace, ws_bytes);
    if (rc) return rc;
    const hils::FwdArgs a = fwd_args(p, q, k_cache, v_cache, lmk_cache, lmk_bias, q_route, seqlens, out, lse, idx,
                                     workspace, ws_bytes);
    return hip_status(hils::launch_decode_fwd(a, (hipStream_t)stream), "hils_decode_fwd launch");
}

int hils_decode_fwd_noalloc(const hils_params* p, const void* q, const void* k_cache, const void* v_cache,
                            const void* lmk_cache, const float* lmk_bias, const void* q_route,
                            const int32_t* seqlens, void* out, float* lse, int32_t* idx, void* stream) {
    int rc = check_params(p, HILS_OP_DECODE);
    if (rc) return rc;
    REQUIRE(q); REQUIRE(k_cache); REQUIRE(v_cache); REQUIRE(lmk_cache); REQUIRE(out); REQUIRE(lse); REQUIRE(idx);
    const size_t need = ws_bytes_for(p, HILS_OP_DECODE);
    const size_t cap = hils::decode_noalloc_capacity();
    if (need > cap)
        return fail(HILS_ERR_WORKSPACE,
                    "hils_decode_fwd_noalloc: this call needs %zu bytes of workspace, above the library's fixed "
                    "%zu-byte array (use hils_decode_fwd with a workspace, or fewer sequences/new tokens)",
                    need, cap);
    void* ws = nullptr;
    rc = hip_status(hils::decode_noalloc_scratch(&ws), "hils_decode_fwd_noalloc: device address of the array");
    if (rc) return rc;
    const hils::FwdArgs a = fwd_args(p, q, k_cache, v_cache, lmk_cache, lmk_bias, q_route, seqlens, out, lse, idx,
                                     ws, cap);
    return hip_status(hils::launch_decode_fwd(a, (hipStream_t)stream), "hils_decode_fwd_noalloc launch");
}

int hils_decode_paged_fwd(const hils_params* p, const void* q, const void* k_pages, const void* v_pages,
                          const void* lmk_pages, const float* bias_pages, const void* q_route,
                          const int32_t* block_table, int num_pages, const int32_t* seqlens, void* out, float* lse,
                          int32_t* idx, void* workspace, size_t ws_bytes, void* stream) {
    int rc = check_params(p, HILS_OP_DECODE);
    if (rc) return rc;
    REQUIRE(q); REQUIRE(k_pages); REQUIRE(v_pages); REQUIRE(lmk_pages); REQUIRE(block_table);
    REQUIRE(out); REQUIRE(lse); REQUIRE(idx);
    if (num_pages < 1) return fail(HILS_ERR_INVALID, "num_pages must be >= 1 (got %d)", num_pages);
    rc = check_ws(p, HILS_OP_DECODE, workspace, ws_bytes);
    if (rc) return rc;
    hils::FwdArgs a = fwd_args(p, q, k_pages, v_pages, lmk_pages, bias_pages, q_route, seqlens, out, lse, idx,
                               workspace, ws_bytes);
    a.block_table = block_table;
    a.num_pages = num_pages;
    return hip_status(hils::launch_decode_fwd(a, (hipStream_t)stream), "hils_decode_paged_fwd launch");
}

int hils_prefill_paged_fwd(const hils_params* p, const void* q, const void* k_pages, const void* v_pages,
                           const void* lmk_pages, const float* bias_pages, const void* q_route,
                           const int32_t* block_table, int num_pages, const int32_t* seqlens, const int32_t* newlens,
                           void* out, float* lse, int32_t* idx, void* workspace, size_t ws_bytes, void* stream) {
    int rc = check_params(p, HILS_OP_PREFILL_PAGED);
    if (rc) return rc;
    REQUIRE(q); REQUIRE(k_pages); REQUIRE(v_pages); REQUIRE(lmk_pages); REQUIRE(block_table);
    REQUIRE(out); REQUIRE(lse); REQUIRE(idx);
    if (num_pages < 1) return fail(HILS_ERR_INVALID, "num_pages must be >= 1 (got %d)", num_pages);
    rc = check_ws(p, HILS_OP_PREFILL_PAGED, workspace, ws_bytes);
    if (rc) return rc;
    REQUIRE_ALIGNED(workspace, 16);
    hils::PrefillPagedArgs a;
    a.f = fwd_args(p, q, k_pages, v_pages, lmk_pages, bias_pages, q_route, seqlens, out, lse, idx, workspace, ws_bytes);
    a.f.block_table = block_table;
    a.f.num_pages = num_pages;
    a.newlens = newlens;
    return hip_status(hils::launch_prefill_paged(a, (hipStream_t)stream), "hils_prefill_paged_fwd launch");
}

int hils_bwd(const hils_params* p, const void* dout, const void* q, const void* k, const void* v, const void* lmk,
             const float* lmk_bias, const void* q_route, const void* out, const float* lse, const int32_t* idx,
             void* dq, void* dk, void* dv, void* dlmk, float* dlmk_bias, void* dq_route, void* workspace,
             size_t ws_bytes, void* stream) {
    int rc = check_params(p, HILS_OP_BWD);
    if (rc) return rc;
    REQUIRE(dout); REQUIRE(q); REQUIRE(k); REQUIRE(v); REQUIRE(lmk); REQUIRE(out); REQUIRE(lse); REQUIRE(idx);
    REQUIRE(dq); REQUIRE(dk); REQUIRE(dv); REQUIRE(dlmk);
    if (q_route && !dq_route)
        return fail(HILS_ERR_INVALID, "q_route is given, so dq_route must be non-NULL");
    rc = check_ws(p, HILS_OP_BWD, workspace, ws_bytes);
    if (rc) return rc;
    hils::BwdArgs a;
    a.dout = dout; a.q = q; a.k = k; a.v = v; a.lmk = lmk; a.bias = lmk_bias; a.q_route = q_route;
    a.out = out; a.lse = lse; a.idx = idx;
    a.dq = dq; a.dk = dk; a.dv = dv; a.dlmk = dlmk; a.dbias = dlmk_bias; a.dq_route = q_route ? dq_route : nullptr;
    a.B = p->B; a.Hq = p->Hq; a.Hkv = p->Hkv; a.Hl = p->Hl; a.N = p->N; a.L = p->L; a.d = p->d;
    a.K = p->topk; a.W = p->window; a.scale = p->scale;
    a.bf16 = p->dtype == HILS_BF16;
    a.ws = workspace; a.ws_bytes = ws_bytes;
    return hip_status(hils::launch_bwd(a, (hipStream_t)stream), "hils_bwd launch");
}

static hils::LmkArgs lmk_args(const hils_params* p) {
    hils::LmkArgs a = {};
    a.B = p->B; a.Hkv = p->Hkv; a.Hl = p->Hl; a.L = p->L; a.d = p->d;
    a.scale = p->scale;
    a.bf16 = p->dtype == HILS_BF16;
    a.shared = (p->flags & HILS_FLAG_SHARED_LMK_QUERY) != 0;
    return a;
}

int hils_landmark_fwd(const hils_params* p, const void* lq, const void* k, void* lmk, float* lmk_bias,
                      void* stream) {
    int rc = check_params(p, HILS_OP_LANDMARK);
    if (rc) return rc;
    REQUIRE(lq); REQUIRE(k); REQUIRE(lmk); REQUIRE(lmk_bias);
    hils::LmkArgs a = lmk_args(p);
    a.lq = lq; a.k = k; a.lmk = lmk; a.bias = lmk_bias;
    return hip_status(hils::launch_landmark_fwd(a, (hipStream_t)stream), "hils_landmark_fwd launch");
}

int hils_landmark_bwd(const hils_params* p, const void* lq, const void* k, const void* dlmk,
                      const float* dlmk_bias, void* dlq, void* dk, void* workspace, size_t ws_bytes,
                      void* stream) {
    int rc = check_params(p, HILS_OP_LANDMARK);
    if (rc) return rc;
    REQUIRE(lq); REQUIRE(k); REQUIRE(dlmk); REQUIRE(dlq); REQUIRE(dk);
    rc = check_ws(p, HILS_OP_LANDMARK, workspace, ws_bytes);
    if (rc) return rc;
    hils::LmkArgs a = lmk_args(p);
    a.lq = lq; a.k = k; a.dlmk = dlmk; a.dbias = dlmk_bias; a.dlq = dlq; a.dk = dk;
    a.ws = static_cast<float*>(workspace);
    return hip_status(hils::launch_landmark_bwd(a, (hipStream_t)stream), "hils_landmark_bwd launch");
}

int hils_q8_append(const hils_params* p, const void* k_new, const void* v_new, void* k_pages, void* v_pages,
                   float* kv_scale, const int32_t* block_table, int num_pages, const int32_t* seqlens,
                   const int32_t* newlens, void* stream) {
    int rc = check_params(p, HILS_OP_Q8_APPEND);
    if (rc) return rc;
    REQUIRE(k_new); REQUIRE(v_new); REQUIRE(k_pages); REQUIRE(v_pages); REQUIRE(kv_scale); REQUIRE(block_table);
    REQUIRE_ALIGNED(k_pages, 16); REQUIRE_ALIGNED(v_pages, 16); REQUIRE_ALIGNED(kv_scale, 8);
    if (num_pages < 1) return fail(HILS_ERR_INVALID, "num_pages must be >= 1 (got %d)", num_pages);
    rc = check_q8_grid(p, .5 * p->B * p->Hkv * ((p->N + 62l) / 64 + 1));
    if (rc) return rc;
    hils::Q8AppendArgs a;
    a.k_new = k_new; a.v_new = v_new; a.k_pages = k_pages; a.v_pages = v_pages; a.kv_scale = kv_scale;
    a.block_table = block_table; a.seqlens = seqlens; a.newlens = newlens;
    a.num_pages = num_pages; a.B = p->B; a.Hkv = p->Hkv; a.N = p->N; a.L = p->L; a.d = p->d;
    a.bf16 = p->dtype == HILS_BF16;
    return hip_status(hils::launch_q8_append(a, (hipStream_t)stream), "hils_q8_append launch");
}

int hils_q8_landmark_fwd(const hils_params* p, const void* lq, const void* k_pages, const float* kv_scale,
                         const int32_t* block_table, int num_pages, const int32_t* seqlens, const int32_t* newlens,
                         void* lmk_pages, float* bias_pages, void* stream) {
    int rc = check_params(p, HILS_OP_Q8_LANDMARK);
    if (rc) return rc;
    REQUIRE(lq); REQUIRE(k_pages); REQUIRE(kv_scale); REQUIRE(block_table); REQUIRE(lmk_pages); REQUIRE(bias_pages);
    REQUIRE_ALIGNED(k_pages, 16); REQUIRE_ALIGNED(lmk_pages, 16); REQUIRE_ALIGNED(kv_scale, 8);
    if (num_pages < 1) return fail(HILS_ERR_INVALID, "num_pages must be >= 1 (got %d)", num_pages);
    rc = check_q8_grid(p, .25 * p->B * p->Hkv * ((p->N + 63l) / 64));
    if (rc) return rc;
    hils::Q8LandmarkArgs a;
    a.lq = lq; a.k_pages = k_pages; a.kv_scale = kv_scale; a.lmk_pages = lmk_pages; a.bias_pages = bias_pages;
    a.block_table = block_table; a.seqlens = seqlens; a.newlens = newlens;
    a.num_pages = num_pages; a.B = p->B; a.Hkv = p->Hkv; a.Hl = p->Hl; a.G = p->Hq / p->Hkv; a.N = p->N; a.L = p->L;
    a.d = p->d; a.bf16 = p->dtype == HILS_BF16; a.shared = (p->flags & HILS_FLAG_SHARED_LMK_QUERY) != 0;
    a.scale = p->scale;
    return hip_status(hils::launch_q8_landmark(a, (hipStream_t)stream), "hils_q8_landmark_fwd launch");
}

int hils_decode_q8_fwd(const hils_params* p, const void* q, const void* k_pages, const void* v_pages,
                       const float* kv_scale, const void* lmk_pages, const float* bias_pages, const void* q_route,
                       const int32_t* block_table, int num_pages, const int32_t* seqlens, void* out, float* lse,
                       int32_t* idx, float* weights, void* workspace, size_t ws_bytes, void* stream) {
    int rc = check_params(p, HILS_OP_DECODE_Q8);
    if (rc) return rc;
    REQUIRE(q); REQUIRE(k_pages); REQUIRE(v_pages); REQUIRE(kv_scale); REQUIRE(lmk_pages); REQUIRE(block_table);
    REQUIRE(out); REQUIRE(lse); REQUIRE(idx);
    REQUIRE_ALIGNED(k_pages, 16); REQUIRE_ALIGNED(v_pages, 16); REQUIRE_ALIGNED(lmk_pages, 16); REQUIRE_ALIGNED(kv_scale, 8);
    if (num_pages < 1) return fail(HILS_ERR_INVALID, "num_pages must be >= 1 (got %d)", num_pages);
    rc = check_q8_grid(p, ((p->L / 64 + 255) / 256 + 8.) * p->B * p->N * p->Hkv);  // the scan's
    if (rc) return rc;
    rc = check_ws(p, HILS_OP_DECODE_Q8, workspace, ws_bytes);
    if (rc) return rc;
    REQUIRE_ALIGNED(workspace, 16);
    hils::Q8DecodeArgs a;
    a.f = fwd_args(p, q, k_pages, v_pages, lmk_pages, bias_pages, q_route, seqlens, out, lse, idx, workspace, ws_bytes);
    a.f.block_table = block_table;
    a.f.num_pages = num_pages;
    a.kv_scale = kv_scale;
    a.weights = weights;
    return hip_status(hils::launch_q8_decode(a, (hipStream_t)stream), "hils_decode_q8_fwd launch");
}

int hils_cache_evict(const hils_params* p, const float* acc, const int32_t* block_table, const int32_t* seqlens,
                     const float* weights, const int32_t* idx, int budget, int sink, int max_evict, float* acc_out,
                     int32_t* table_out, int32_t* seqlens_out, int32_t* freed, int32_t* nfreed, void* stream) {
    int rc = check_params(p, HILS_OP_CACHE_EVICT);
    if (rc) return rc;
    REQUIRE(acc); REQUIRE(block_table); REQUIRE(acc_out); REQUIRE(table_out); REQUIRE(seqlens_out); REQUIRE(nfreed);
    if (weights && !idx) return fail(HILS_ERR_INVALID, "weights are given, so idx must be non-NULL");
    if (budget < 0 || sink < 0 || max_evict < 0)
        return fail(HILS_ERR_INVALID, "budget, sink and max_evict must be >= 0 (budget=%d sink=%d max_evict=%d)", budget,
                    sink, max_evict);
    if (weights && ((double)p->Hkv * p->N * (p->topk + (p->window + 62) / 64 + 1) > 0x7ffffbff))  // (and a step of 1024)
        return fail(HILS_ERR_UNSUPPORTED, "Hkv=%d N=%d topk=%d: more weights per sequence than 2^31", p->Hkv, p->N,
                    p->topk);
    if (max_evict > 0 && !freed) return fail(HILS_ERR_INVALID, "max_evict=%d, so freed must be non-NULL", max_evict);
    hils::EvictArgs a;
    a.acc = acc; a.table = block_table; a.seqlens = seqlens; a.weights = weights; a.idx = idx;
    a.acc_out = acc_out; a.table_out = table_out; a.seqlens_out = seqlens_out; a.freed = freed; a.nfreed = nfreed;
    a.B = p->B; a.Hkv = p->Hkv; a.N = p->N; a.L = p->L; a.K = p->topk; a.W = p->window;
    a.budget = budget; a.sink = sink; a.most = max_evict;
    return hip_status(hils::launch_evict(a, (hipStream_t)stream), "hils_cache_evict launch");
}

int hils_cache_reserve(const hils_params* p, const int32_t* block_table, const int32_t* page_refs, int num_pages,
                       const int32_t* seqlens, const int32_t* newlens, const hils_pool* pools, int num_pools,
                       int32_t* table_out, int32_t* refs_out, int32_t* copied, int32_t* counts, void* stream) {
    int rc = check_params(p, HILS_OP_CACHE_RESERVE);
    if (rc) return rc;
    REQUIRE(block_table); REQUIRE(page_refs); REQUIRE(table_out); REQUIRE(refs_out); REQUIRE(copied); REQUIRE(counts);
    rc = check_page_count(num_pages);
    if (rc) return rc;
    if ((double)p->B * (p->L / 64) > 0x7fffffff)
        return fail(HILS_ERR_UNSUPPORTED, "B=%d L=%d: more than 2^31 table entries", p->B, p->L);
    rc = check_pools(pools, num_pools);
    if (rc) return rc;
    const hils::ReserveArgs a{block_table, page_refs, seqlens, newlens, table_out, refs_out, copied, counts,
                              num_pages, p->B, p->N, p->L};
    return hip_status(hils::launch_reserve(a, reinterpret_cast<const hils::PoolArg*>(pools), num_pools, (hipStream_t)stream), "hils_cache_reserve launch");
}

int hils_cache_fork(const hils_params* p, const int32_t* parent, int rows, const int32_t* block_table,
                    const int32_t* page_refs, int num_pages, const int32_t* seqlens, int32_t* table_out,
                    int32_t* seqlens_out, int32_t* refs_out, void* stream) {
    int rc = check_params(p, HILS_OP_CACHE_FORK);
    if (rc) return rc;
    REQUIRE(parent); REQUIRE(block_table); REQUIRE(page_refs); REQUIRE(table_out); REQUIRE(seqlens_out); REQUIRE(refs_out);
    rc = check_page_count(num_pages);
    if (rc) return rc;
    if (rows < 1 || rows > 65535) return fail(HILS_ERR_INVALID, "rows=%d: 1 to 65535 are possible", rows);
    if (table_out == block_table || (seqlens && seqlens_out == seqlens))
        return fail(HILS_ERR_INVALID, "a fork's rows and lengths cannot be written in place");
    const hils::ForkArgs a{parent, block_table, page_refs, seqlens, table_out, seqlens_out, refs_out, num_pages, p->B,
                           p->L, rows};
    return hip_status(hils::launch_fork(a, (hipStream_t)stream), "hils_cache_fork launch");
}

int hils_cache_free(const hils_params* p, const int32_t* keep, const int32_t* pages, const int32_t* npages,
                    int max_pages, const int32_t* block_table, const int32_t* page_refs, int num_pages,
                    const int32_t* seqlens, int32_t* table_out, int32_t* seqlens_out, int32_t* refs_out, void* stream) {
    int rc = check_params(p, HILS_OP_CACHE_FREE);
    if (rc) return rc;
    REQUIRE(keep); REQUIRE(block_table); REQUIRE(page_refs); REQUIRE(table_out); REQUIRE(seqlens_out); REQUIRE(refs_out);
    rc = check_page_count(num_pages);
    if (rc) return rc;
    if (max_pages < 0 || max_pages > 1 << 30)
        return fail(HILS_ERR_INVALID, "max_pages=%d: 0 to 2^30 are possible", max_pages);
    if (npages && !pages) return fail(HILS_ERR_INVALID, "npages is given, so pages must be non-NULL");
    const hils::FreeArgs a{keep, max_pages ? pages : nullptr, npages, block_table, page_refs, seqlens, table_out,
                           seqlens_out, refs_out, num_pages, p->B, p->L, max_pages};
    return hip_status(hils::launch_free(a, (hipStream_t)stream), "hils_cache_free launch");
}

int hils_cache_compact(const hils_params* p, const int32_t* block_table, const int32_t* page_refs, int num_pages,
                       const int32_t* seqlens, const hils_pool* pools, int num_pools, int32_t* table_out,
                       int32_t* refs_out, int32_t* new_page, int32_t* moved, int32_t* counts, void* stream) {
    int rc = check_params(p, HILS_OP_CACHE_COMPACT);
    if (rc) return rc;
    REQUIRE(block_table); REQUIRE(page_refs); REQUIRE(table_out); REQUIRE(refs_out); REQUIRE(new_page); REQUIRE(moved);
    REQUIRE(counts);
    rc = check_page_count(num_pages);
    if (rc) return rc;
    rc = check_pools(pools, num_pools);
    if (rc) return rc;
    const hils::CompactArgs a{block_table, page_refs, seqlens, table_out, refs_out, new_page, moved, counts, num_pages,
                              p->B, p->L};
    return hip_status(hils::launch_compact(a, reinterpret_cast<const hils::PoolArg*>(pools), num_pools, (hipStream_t)stream), "hils_cache_compact launch");
}

}  // extern "C"
