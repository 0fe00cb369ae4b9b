// C ABI of window attention, of the paged cache and of key weights (see include/rr_attn.h): argument checks on the host, then
// launches.
#include "rr_common.hpp"
#include "rr_cache.hpp"
#include "rr_check.hpp"

#include <algorithm>

namespace {

using namespace rr;

constexpr int kMostPositions = 1 << 30;         // blocks and strides behind the last position still have 32-bit positions

// The layout that outputs are written in gives every element a place of its own
bool outputs_distinct(const rr_shape* s, int rows) {
    return (rows == 1 || s->q_stride_l >= s->d) && (s->Hq == 1 || s->q_stride_h > 0) && (s->batch == 1 || s->q_stride_b > 0);
}

int check_window(const rr_shape* shape, int window, int sinks, Geom* g) {
    const int rc = check_shape(shape, g);
    if (rc != RR_OK) return rc;
    if (g->L > kMostPositions || !outputs_distinct(shape, g->Lq)) return RR_ERR_SHAPE;
    if (window < 1 || sinks < 0) return RR_ERR_PARAM;
    return RR_OK;
}

int check_key_weights(const rr_shape* shape, Geom* g) {
    const int rc = check_shape(shape, g);
    if (rc != RR_OK) return rc;
    // the indexes of a launch (tiles of 128 keys and more), and of a KV head's stages of 32 rows, are 32 bits
    if (g->L > kMostPositions || (long long)g->batch * g->Hkv > 0x7fffffff || (long long)g->G * ((g->Lq + 31) / 32) > 0x3fffffff ||
        (long long)g->batch * g->Hkv * ((g->L + 127) / 128) > 0x7fffff)
        return RR_ERR_SHAPE;
    return RR_OK;
}

// A step of few rows per KV head whose keys are shared out among workgroups, contiguous form of the cache kernels
bool window_step(const Geom& g, int dtype, int window, int sinks, CacheArgs* c, CachePlan* plan) {
    if (g.Lq > 16 || g.G * g.Lq > 32) return false;
    *c = CacheArgs{};
    c->batch = g.batch; c->Hq = g.Hq; c->Hkv = g.Hkv; c->G = g.G; c->d = g.d;
    c->T = g.Lq;
    c->L = g.L;
    c->qsb = g.qsb; c->qsh = g.qsh; c->qsl = g.qsl;
    c->psb = g.ksb; c->ksh = g.ksh; c->ksl = g.ksl;
    c->window = std::min(window, g.L); c->sinks = std::min(sinks, g.L);
    c->scale_log2 = (float)(1.4426950408889634 / sqrt((double)g.d));
    if (!cache_attn_plan(*c, dtype, false, plan)) return false;
    c->row_tiles = plan->row_tiles;
    c->whole = plan->whole;
    return true;
}

// The cache of a call: `rows` query (or new) positions at the end of every sequence
int check_cache(const rr_shape* shape, const rr_paged_cache* cache, CacheArgs* c, bool sizes_only = false) {
    Geom g;
    const int rc = check_shape(shape, &g);
    if (rc != RR_OK) return rc;
    if (!cache || (!sizes_only && (!cache->K || !cache->V || !cache->table || !cache->length))) return RR_ERR_NULL;
    if (cache->page < 16 || cache->page % 16 || cache->num_pages < 1 || cache->width < 1) return RR_ERR_SHAPE;
    if (g.L > kMostPositions || (long long)cache->width * cache->page < g.L) return RR_ERR_SHAPE;
    if (!aligned16(cache->K) || !aligned16(cache->V)) return RR_ERR_SHAPE;
    *c = CacheArgs{};
    c->batch = g.batch; c->Hq = g.Hq; c->Hkv = g.Hkv; c->G = g.G; c->d = g.d;
    c->T = g.Lq;
    c->L = g.L;
    c->qsb = g.qsb; c->qsh = g.qsh; c->qsl = g.qsl;
    c->psb = g.ksb; c->ksh = g.ksh; c->ksl = g.ksl;
    c->K = cache->K; c->V = cache->V; c->weight = cache->weight;
    c->table = cache->table; c->length = cache->length;
    set_page(c, cache->page);
    c->num_pages = cache->num_pages; c->width = cache->width;
    c->scale_log2 = (float)(1.4426950408889634 / sqrt((double)g.d));
    return RR_OK;
}

int set_window(CacheArgs* c, int window, int sinks) {
    if (window < 0 || sinks < 0) return RR_ERR_PARAM;
    // no window: one that reaches over everything from any query
    const long long whole = (long long)c->L + c->T;
    if (whole > 0x7fffffffLL) return RR_ERR_SHAPE;
    c->window = window == 0 || window > whole ? (int)whole : window;
    c->sinks = std::min(sinks, c->L);
    return RR_OK;
}

void set_workspace(CacheArgs* c, const CachePlan& plan, void* workspace) {
    unsigned char* ws = reinterpret_cast<unsigned char*>(workspace);
    c->part_O = reinterpret_cast<float*>(ws);
    c->part_lse = c->part_O + plan.part_rows * c->d;
    c->front = reinterpret_cast<int*>(c->part_lse + plan.part_rows);
    c->scores = plan.score_bytes ? reinterpret_cast<float*>(ws + plan.part_bytes) : nullptr;
    c->row_lse = plan.row_bytes ? reinterpret_cast<float*>(ws + plan.part_bytes + plan.score_bytes) : nullptr;
}

bool misaligned256(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 255u) != 0; }

}  // namespace

#define RR_API __attribute__((visibility("default")))

extern "C" {

RR_API size_t rr_window_workspace_bytes(const rr_shape* shape, int window, int sinks) {
    Geom g;
    CacheArgs c;
    CachePlan plan;
    if (check_window(shape, window, sinks, &g) != RR_OK || !window_step(g, shape->dtype, window, sinks, &c, &plan)) return 0;
    return plan.total();
}

RR_API int rr_window_attn(const rr_shape* shape, const void* Q, const void* K, const void* V, int window, int sinks,
                          const int32_t* seq_first, int B, void* O, float* lse, void* workspace, size_t workspace_bytes,
                          void* hip_stream) {
    Geom g;
    const int rc = check_window(shape, window, sinks, &g);
    if (rc != RR_OK) return rc;
    if (!Q || !K || !V || !O) return RR_ERR_NULL;
    if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O)) return RR_ERR_SHAPE;
    if (seq_first) {
        if (B < 16 || B > 128 || B % 16) return RR_ERR_SHAPE;
        if (g.q0 != 0) return RR_ERR_PARAM;                  // packed sequences and a query chunk do not combine
    }
    CacheArgs c;
    CachePlan plan;
    hipError_t e;
    if (!seq_first && window_step(g, shape->dtype, window, sinks, &c, &plan) && (workspace || plan.total() == 0)) {
        if (plan.total() && (workspace_bytes < plan.total() || misaligned256(workspace))) return RR_ERR_WORKSPACE;
        c.Q = Q; c.K = K; c.V = V; c.O = O; c.lse = lse;
        set_workspace(&c, plan, workspace);
        e = launch_cache_attn(c, shape->dtype, plan, (hipStream_t)hip_stream);
    } else {
        const WindowArgs a = {Q, K, V, O, lse, std::min(window, g.L), std::min(sinks, g.L), seq_first, B};
        e = window_mfma_takes(g, shape->dtype, seq_first, B) ? launch_window_mfma(g, a, (hipStream_t)hip_stream)
                                                             : launch_window_generic(g, shape->dtype, a, (hipStream_t)hip_stream);
    }
    return e == hipSuccess ? RR_OK : RR_ERR_LAUNCH;
}

RR_API size_t rr_paged_workspace_bytes(const rr_shape* shape, const rr_paged_cache* cache, int window, int sinks, uint32_t flags) {
    CacheArgs c;
    CachePlan plan;
    if (check_cache(shape, cache, &c, true) != RR_OK || set_window(&c, window, sinks) != RR_OK) return 0;
    if (flags & ~RR_FLAG_ACCUMULATE) return 0;
    return cache_attn_plan(c, shape->dtype, (flags & RR_FLAG_ACCUMULATE) != 0, &plan) ? plan.total() : 0;
}

RR_API int rr_paged_attn(const rr_shape* shape, const void* Q, const rr_paged_cache* cache, int window, int sinks, uint32_t flags,
                         void* O, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
    CacheArgs c;
    int rc = check_cache(shape, cache, &c);
    if (rc != RR_OK) return rc;
    if (!Q || !O) return RR_ERR_NULL;
    if (flags & ~RR_FLAG_ACCUMULATE) return RR_ERR_PARAM;
    const bool accumulate = (flags & RR_FLAG_ACCUMULATE) != 0;
    if (accumulate && !cache->weight) return RR_ERR_NULL;
    if (accumulate && !aligned16(cache->weight)) return RR_ERR_SHAPE;
    if (!aligned16(Q) || !aligned16(O) || !outputs_distinct(shape, c.T)) return RR_ERR_SHAPE;
    rc = set_window(&c, window, sinks);
    if (rc != RR_OK) return rc;
    CachePlan plan;
    if (!cache_attn_plan(c, shape->dtype, accumulate, &plan)) return RR_ERR_SHAPE;
    if (plan.total() && (!workspace || workspace_bytes < plan.total() || misaligned256(workspace))) return RR_ERR_WORKSPACE;
    c.Q = Q; c.O = O; c.lse = lse;
    c.row_tiles = plan.row_tiles;
    c.whole = plan.whole;
    set_workspace(&c, plan, workspace);
    return launch_cache_attn(c, shape->dtype, plan, (hipStream_t)hip_stream) == hipSuccess ? RR_OK : RR_ERR_LAUNCH;
}

RR_API int rr_paged_write(const rr_shape* shape, const rr_paged_cache* cache, const void* K, const void* V, const int32_t* count,
                          const float* weight, void* hip_stream) {
    CacheArgs c;
    const int rc = check_cache(shape, cache, &c);
    if (rc != RR_OK) return rc;
    if (!K || !V) return RR_ERR_NULL;
    if (weight && !cache->weight) return RR_ERR_NULL;
    if (!aligned16(K) || !aligned16(V) || (long long)c.batch * c.Hkv > 65535) return RR_ERR_SHAPE;
    const CacheWriteArgs a = {K, V, weight, count};
    return launch_cache_write(c, shape->dtype, a, cache->K, cache->V, (hipStream_t)hip_stream) == hipSuccess ? RR_OK : RR_ERR_LAUNCH;
}

RR_API size_t rr_cache_evict_workspace_bytes(const rr_shape* shape, const rr_paged_cache* cache) {
    CacheArgs c;
    return check_cache(shape, cache, &c, true) == RR_OK && (long long)c.batch * c.Hkv <= 65535 ? cache_evict_bytes(c) : 0;
}

RR_API int rr_cache_evict(const rr_shape* shape, const rr_paged_cache* cache, int keep, int sinks, int recent, const int32_t* to_table,
                          int to_width, int32_t* to_length, int32_t* kept, void* workspace, size_t workspace_bytes, void* hip_stream) {
    CacheArgs c;
    const int rc = check_cache(shape, cache, &c);
    if (rc != RR_OK) return rc;
    if (!cache->weight || !to_table || !to_length || !kept) return RR_ERR_NULL;
    if (keep < 1 || sinks < 0 || recent < 0 || (long long)sinks + recent > keep) return RR_ERR_PARAM;
    // a target holds what is kept of the longest sequence
    if (to_width < 1 || (long long)to_width * c.page < std::min(keep, c.L)) return RR_ERR_SHAPE;
    if (!aligned16(cache->weight) || (long long)c.batch * c.Hkv > 65535) return RR_ERR_SHAPE;
    const size_t need = cache_evict_bytes(c);
    if (need && (!workspace || workspace_bytes < need || misaligned256(workspace))) return RR_ERR_WORKSPACE;
    const CacheEvictArgs a = {keep, sinks, recent, to_table, to_width, to_length, kept};
    return launch_cache_evict(c, shape->dtype, a, cache->K, cache->V, workspace, (hipStream_t)hip_stream) == hipSuccess ? RR_OK : RR_ERR_LAUNCH;
}

RR_API size_t rr_key_weights_workspace_bytes(const rr_shape* shape) {
    Geom g;
    return check_key_weights(shape, &g) == RR_OK ? key_weights_bytes(g, shape->dtype) : 0;
}

RR_API int rr_key_weights(const rr_shape* shape, const void* Q, const void* K, const float* lse, float* weight, void* workspace,
                          size_t workspace_bytes, void* hip_stream) {
    Geom g;
    const int rc = check_key_weights(shape, &g);
    if (rc != RR_OK) return rc;
    if (!Q || !K || !lse || !weight) return RR_ERR_NULL;
    if (!aligned16(Q) || !aligned16(K)) return RR_ERR_SHAPE;
    const size_t need = key_weights_bytes(g, shape->dtype);
    if (need && (!workspace || workspace_bytes < need || misaligned256(workspace))) return RR_ERR_WORKSPACE;
    return launch_key_weights(g, shape->dtype, Q, K, lse, weight, workspace, (hipStream_t)hip_stream) == hipSuccess ? RR_OK : RR_ERR_LAUNCH;
}

}  // extern "C"
