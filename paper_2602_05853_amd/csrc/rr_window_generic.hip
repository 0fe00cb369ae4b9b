// Causal attention with a sliding window and sinks on 16 x 16 matrix tiles: O_i = softmax over the keys j <= i with j > i - window
// or j - s0 < sinks (s0 the first position of i's sequence) of q_i k_j / sqrt(d), times V.  Every shape that the bf16 d = 128
// kernel does not take: fp32 tensors, any d (a multiple of 8 up to 256), packed sequences of any block size.
//
// Work split as in the generic block-sparse attention: one workgroup per 16 QT queries of a head, whose KW waves share the keys,
// each with an online softmax of its own, joined in LDS at the end.  The keys are two runs of 16-key tiles, the sinks' and the
// window's; only tiles at a border (of the window, the sinks, the sequence, causality) are masked key by key.
// Arithmetic: nothing is held in fewer than 32 bits (rr_attn_frag.hpp).
//
// Measured (window 1024, 4 sinks): bf16, 8192 tokens, 16 / 4 heads of 64 129 us (251 TFLOP/s; every probability is three terms, so 500 of
// products), of 96 164; fp32, 6000 tokens, 8 / 2 heads of 128 296 us (78 TFLOP/s, half of what a large fp32 product reaches).
#include "rr_attn_frag.hpp"

#include <algorithm>
#include <type_traits>

namespace rr {

namespace {

__device__ __forceinline__ void store_row4(float* p, const f32x4& v) { *reinterpret_cast<f32x4*>(p) = v; }
__device__ __forceinline__ void store_row4(bf16_t* p, const f32x4& v) {
    const u32x2 o = {f32_to_bf16_bits(v[0]) | (f32_to_bf16_bits(v[1]) << 16),
                     f32_to_bf16_bits(v[2]) | (f32_to_bf16_bits(v[3]) << 16)};
    *reinterpret_cast<u32x2*>(p) = o;
}

// D: d where it fills the matrix tiles, so that a row's last channels need no check (which would wait for the keys in front of
// the work they are requested ahead of), or 0.
template <typename T, int NT, int D, int QT, int TL, int KW, int OCC>
__global__ void __launch_bounds__(64 * KW, OCC)
k_window_generic(Geom g, WindowArgs a, float scale_log2, int tiles_q) {
    using F = Frag<T, NT, TL>;
    constexpr int kQ = 16 * QT, kPitch = 16 * NT + 4, kThreads = 64 * KW;
    __shared__ __align__(16) float s_o[KW][kQ][kPitch];
    __shared__ float s_ref[KW][kQ], s_l[KW][kQ];
    const float NEG_INF = -__builtin_huge_valf();
    const int t = threadIdx.x, lane = t & 63, x = lane & 15, gq = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(t >> 6);
    const int d = D ? D : g.d;

    // heads fastest, and of those the KV head: the XCDs, which take consecutive workgroups in turn, each keep the keys of few
    // KV heads in L2; the last queries, which see most, first
    int id = (int)blockIdx.x;
    const int hx = id % g.Hq, hl = hx / g.Hkv, kv = hx - hl * g.Hkv, h = kv * g.G + hl;
    id /= g.Hq;
    const int b = id / tiles_q;
    // tiles of queries begin at multiples of 16 positions of the context, so that none holds two sequences' queries
    const int p_tile = g.q0 / 16 * 16 + kQ * (tiles_q - 1 - (id - b * tiles_q));
    const int p_lo = max(p_tile, g.q0), p_hi = min(p_tile + kQ, g.L) - 1;
    if (p_lo > p_hi) return;

    const T* Q = reinterpret_cast<const T*>(a.Q) + b * g.qsb + h * g.qsh;
    const T* K = reinterpret_cast<const T*>(a.K) + b * g.ksb + kv * g.ksh;
    const T* V = reinterpret_cast<const T*>(a.V) + b * g.ksb + kv * g.ksh;

    // the sequence of a query's tile of 16 (a workgroup's queries may belong to several sequences: QT > 1 of packed ones)
    int s0[QT], qpos[QT];
    int s0_first = 0;
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        const int at = min(p_tile + 16 * u, g.L - 1);
        s0[u] = 0;
        if (a.seq_first) {
            const int m = at / a.B, f = a.seq_first[m];
            s0[u] = (f < 0 ? 0 : (f > m ? m : f)) * a.B;
        }
        s0[u] = __builtin_amdgcn_readfirstlane(s0[u]);
        if (u == 0) s0_first = s0[0];
        qpos[u] = min(max(p_tile + 16 * u + x, p_lo), p_hi);            // rows that do not exist: a copy of the nearest real one
    }

    F qf[QT];
#pragma unroll
    for (int u = 0; u < QT; ++u) qf[u].load(Q + (long long)(qpos[u] - g.q0) * g.qsl, d, gq);

    // tiles of the sinks that lie in front of the window's, then the window's
    const int w_lo = max((long long)s0_first, (long long)p_lo - a.window + 1) >> 4, w_hi = p_hi >> 4;
    // (of several sequences in a workgroup the later ones begin behind p_lo's window: their sinks are among its tiles)
    const int sink_lo = s0_first >> 4;
    const int n_sink = (int)max(0ll, min((long long)w_lo, ((long long)s0_first + a.sinks + 15) >> 4) - sink_lo);
    const int tiles = n_sink + w_hi - w_lo + 1, steps = (tiles + TL - 1) / TL;
    auto tile_at = [&](int i) { return i < n_sink ? sink_lo + i : w_lo + i - n_sink; };

    const long long k_off = (long long)x * g.ksl;
    long long v_off[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) v_off[r] = (long long)(4 * gq + r) * g.ksl;
    F kf[TL];
    int key0[TL], last[TL];                                             // first key of a tile; the last that exists, -1: no such tile
    auto load_keys = [&](int st) {
#pragma unroll
        for (int tl = 0; tl < TL; ++tl) {
            const int i = st * TL + tl;
            key0[tl] = 16 * tile_at(min(i, tiles - 1));
            last[tl] = i < tiles ? min(15, g.L - 1 - key0[tl]) : -1;
            const T* base = K + (long long)key0[tl] * g.ksl;
            kf[tl].load(last[tl] == 15 ? base + k_off : base + (long long)min(x, max(last[tl], 0)) * g.ksl, d, gq);
        }
    };
    f32x4 acc[QT][NT];
    float ref[QT], lsum[QT];
    auto walk = [&](auto careful) {
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        ref[u] = NEG_INF;
        lsum[u] = 0.f;
#pragma unroll
        for (int c = 0; c < NT; ++c) acc[u][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if (w < steps) load_keys(w);
    for (int st = w; st < steps; st += KW) {
        typename F::V vf;
#pragma unroll
        for (int tl = 0; tl < TL; ++tl) {
            const T* base = V + (long long)key0[tl] * g.ksl;
#pragma unroll
            for (int r = 0; r < 4; ++r)
                F::load_v(vf, 4 * tl + r, last[tl] == 15 ? base + v_off[r] : base + (long long)min(4 * gq + r, max(last[tl], 0)) * g.ksl, d, x);
        }
        f32x4 s[QT][TL];
#pragma unroll
        for (int u = 0; u < QT; ++u)
#pragma unroll
            for (int tl = 0; tl < TL; ++tl) s[u][tl] = f32x4{0.f, 0.f, 0.f, 0.f};
        F::template qk<QT>(s, kf, qf);
        int key_now[TL], last_now[TL];
#pragma unroll
        for (int tl = 0; tl < TL; ++tl) {
            key_now[tl] = key0[tl];
            last_now[tl] = last[tl];
#pragma unroll
            for (int u = 0; u < QT; ++u) {
                const int first_q = min(max(p_tile + 16 * u, p_lo), p_hi), last_q = min(p_tile + 16 * u + 15, p_hi);
                const bool whole = last[tl] == 15 && key0[tl] >= s0[u] && key0[tl] + 15 <= first_q &&
                                   (key0[tl] > last_q - a.window || key0[tl] + 15 - s0[u] < a.sinks);
                if (!whole) {
                    f32x4 v = s[u][tl];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int k = 4 * gq + r, key = key0[tl] + k;
                        const bool sees = k <= last[tl] && key >= s0[u] && key <= qpos[u] &&
                                          (key > qpos[u] - a.window || key - s0[u] < a.sinks);
                        v[r] = sees ? v[r] : NEG_INF;
                    }
                    s[u][tl] = v;
                }
            }
        }
        // the next step's keys travel during the softmax and the second product
        if (st + KW < steps) load_keys(st + KW);
        float p[QT][4 * TL];
#pragma unroll
        for (int u = 0; u < QT; ++u) frag_softmax<TL, NT>(s[u], scale_log2, ref[u], lsum[u], acc[u], p[u]);
        if constexpr (decltype(careful)::value) {
            // values of keys that none of the workgroup's rows sees are left out
#pragma unroll
            for (int tl = 0; tl < TL; ++tl)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int k = 4 * gq + r, key = key_now[tl] + k;
                    F::drop(vf, 4 * tl + r, k > last_now[tl] || key > p_hi || key < s0_first ||
                                            !((long long)key > (long long)p_lo - a.window || key - s0_first < a.sinks));
                }
        }
        F::template pv<QT, decltype(careful)::value>(acc, vf, p);
    }
    };
    walk(std::false_type{});
    if (has_nan(acc)) walk(std::true_type{});

    // ---- the waves' shares, brought to one reference ----
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        float l = lsum[u];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        const int q = 16 * u + x;
        if (gq == 0) { s_ref[w][q] = ref[u]; s_l[w][q] = l; }
        frag_store<F::kW, NT>(acc[u], &s_o[w][q][0], gq);
    }
    __syncthreads();
    T* O = reinterpret_cast<T*>(a.O) + b * g.qsb + h * g.qsh;
    float* lse = a.lse ? a.lse + ((long long)b * g.Hq + h) * g.Lq : nullptr;
    for (int idx = t; idx < kQ * 4 * NT; idx += kThreads) {
        const int q = idx / (4 * NT), c = 4 * (idx - q * (4 * NT));
        const int pos = p_tile + q;
        if (pos < p_lo || pos > p_hi || c >= d) continue;
        float top = NEG_INF;
#pragma unroll
        for (int i = 0; i < KW; ++i) top = fmaxf(top, s_ref[i][q]);
        float l = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KW; ++i) {
            const float f = s_ref[i][q] == NEG_INF ? 0.f : __builtin_amdgcn_exp2f(s_ref[i][q] - top);
            l = fmaf(f, s_l[i][q], l);
            const f32x4 v = *reinterpret_cast<const f32x4*>(&s_o[i][q][c]);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = fmaf(f, v[e], o[e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = l > 0.f ? o[e] / l : 0.f;
        store_row4(O + (long long)(pos - g.q0) * g.qsl + c, o);
        if (lse && c == 0) lse[pos - g.q0] = l > 0.f ? top * 0.6931471805599453f + logf(l) : NEG_INF;
    }
}

}  // namespace

hipError_t launch_window_generic(const Geom& g, int dtype, const WindowArgs& a, hipStream_t st) {
    const float scale_log2 = (float)(1.4426950408889634 / sqrt((double)g.d));
    auto launch = [&](auto kernel, int queries, int waves) -> hipError_t {
        const long long tiles_q = ((long long)g.L - g.q0 / 16 * 16 + queries - 1) / queries;
        const long long blocks = tiles_q * g.Hq * g.batch;
        if (blocks * 64 * waves > 0xFFFFFFFFll) return hipErrorInvalidValue;
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(64 * waves), 0, st, g, a, scale_log2, (int)tiles_q);
        return hipGetLastError();
    };
    auto pick = [&](auto tiles, auto full) -> hipError_t {
        constexpr int N = decltype(tiles)::value, D = decltype(full)::value;
        const long long rows = (long long)g.batch * g.Hq * g.Lq;
        if constexpr (N > 8) {
            return dtype == RR_BF16 ? launch(k_window_generic<bf16_t, N, D, 1, 2, 4, 1>, 16, 4)
                                    : launch(k_window_generic<float, N, D, 1, 1, 4, 1>, 16, 4);
        } else {
            if (dtype == RR_BF16) {
                if constexpr (N <= 4)
                    if (rows >= 64 * 512) return launch(k_window_generic<bf16_t, N, D, 4, 2, 4, 2>, 64, 4);
                // (a few queries deep in a context end when the longest workgroup does: 16 queries on eight waves while those fill the
                // chip once; d = 128, us, this / 32 on four waves: 100 of 24000, window 4096, 32 heads (224 workgroups) 42 / 53, 200
                // (416) 80 / 55; 500, window 512, 8 heads (256) 11.0 / 15.1; 1024 positions, 8 heads (512) 19.8 / 19.4)
                if (rows <= 16 * 256) return launch(k_window_generic<bf16_t, N, D, 1, 2, 8, 2>, 16, 8);
                return launch(k_window_generic<bf16_t, N, D, 2, 2, 4, 2>, 32, 4);
            }
            // (1511 positions, 8 heads of 80, window 200, 95 tiles of 16 queries to a head, us: 16 queries on eight waves 20.0, on four
            // 18.7, 32 on eight 24.9, on four 21.8: half the reads, but the workgroups no longer fill the chip)
            if (rows >= 32 * 512) return launch(k_window_generic<float, N, D, 2, 1, 8, 2>, 32, 8);
            return launch(k_window_generic<float, N, D, 1, 1, 4, 2>, 16, 4);
        }
    };
    using std::integral_constant;
    switch ((g.d + 15) / 16) {
#define RR_WINDOW_CASE(N) case N: return g.d == 16 * N ? pick(integral_constant<int, N>{}, integral_constant<int, 16 * N>{}) \
                                                : pick(integral_constant<int, N>{}, integral_constant<int, 0>{})
        RR_WINDOW_CASE(1); RR_WINDOW_CASE(2); RR_WINDOW_CASE(3); RR_WINDOW_CASE(4);
        RR_WINDOW_CASE(5); RR_WINDOW_CASE(6); RR_WINDOW_CASE(7); RR_WINDOW_CASE(8);
        RR_WINDOW_CASE(9); RR_WINDOW_CASE(10); RR_WINDOW_CASE(11); RR_WINDOW_CASE(12);
        RR_WINDOW_CASE(13); RR_WINDOW_CASE(14); RR_WINDOW_CASE(15); RR_WINDOW_CASE(16);
#undef RR_WINDOW_CASE
        default: return hipErrorInvalidValue;
    }
}

}  // namespace rr
