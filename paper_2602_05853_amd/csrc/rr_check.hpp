// Argument checks that the entry points share.
#pragma once
#include "rr_common.hpp"

namespace rr {

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

inline int check_shape(const rr_shape* s, Geom* g) {
    if (!s) return RR_ERR_NULL;
    if (s->dtype != RR_BF16 && s->dtype != RR_F32) return RR_ERR_DTYPE;
    if (s->batch < 1 || s->L < 1 || s->Hq < 1 || s->Hkv < 1 || s->d < 8) return RR_ERR_SHAPE;
    if (s->Hq % s->Hkv) return RR_ERR_SHAPE;
    if (s->d % 8 || s->d > 256) return RR_ERR_SHAPE;
    const int64_t row = s->dtype == RR_BF16 ? 8 : 4;          // elements per 16 bytes
    const int64_t st[6] = {s->q_stride_b, s->q_stride_h, s->q_stride_l,
                           s->kv_stride_b, s->kv_stride_h, s->kv_stride_l};
    for (int i = 0; i < 6; ++i)
        if (st[i] < 0 || st[i] % row) return RR_ERR_SHAPE;
    if (s->q_stride_l < s->d || s->kv_stride_l < s->d) return RR_ERR_SHAPE;
    g->batch = s->batch; g->L = s->L; g->Hq = s->Hq; g->Hkv = s->Hkv; g->d = s->d;
    g->G = s->Hq / s->Hkv;
    if (s->Lq < 0 || s->Lq > s->L) return RR_ERR_SHAPE;
    g->Lq = s->Lq ? s->Lq : s->L;
    g->q0 = g->L - g->Lq;
    g->qoff = 0;
    g->Lr = g->L;
    g->qsb = s->q_stride_b; g->qsh = s->q_stride_h; g->qsl = s->q_stride_l;
    g->ksb = s->kv_stride_b; g->ksh = s->kv_stride_h; g->ksl = s->kv_stride_l;
    return RR_OK;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace rr
