// Softmax weights that every key gets from the queries of a call: w_j = sum over the heads h of a KV group and the query rows i of
// exp(q_i k_j / sqrt(d) - lse_i) where j <= i's position; lse is what the attention of the same call has written.
//
// One product per (query, key) pair and no second one: half the operations of attention.  The keys of a workgroup stay in
// registers (rows of the matrix tiles), its waves take the queries' tiles (columns) in turn, so a query tile is read once per
// workgroup of keys; every lane adds up its own columns, and columns and waves meet once, at the end, in a fixed order.
#include "rr_attn_frag.hpp"

#include <algorithm>
#include <type_traits>

namespace rr {

namespace {

template <typename T, int NT, int PAIRS, int KW, int OCC>
__global__ void __launch_bounds__(64 * KW, OCC)
k_key_weights(Geom g, const T* Qp, const T* Kp, const float* lse, float* out, float scale_log2) {
    using F = Frag<T, NT, 2>;
    constexpr int kKeys = 32 * PAIRS;
    __shared__ float s_sum[KW][kKeys];
    const int t = threadIdx.x, lane = t & 63, x = lane & 15, gq = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(t >> 6);
    const float INF = __builtin_huge_valf();
    const int kv = blockIdx.y, b = blockIdx.z;
    const int key0 = (int)blockIdx.x * kKeys;              // the first keys are seen by most queries: heaviest first
    const T* K = Kp + b * g.ksb + kv * g.ksh;
    F kf[PAIRS][2];
#pragma unroll
    for (int i = 0; i < PAIRS; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) kf[i][e].load(K + (long long)min(key0 + 32 * i + 16 * e + x, g.L - 1) * g.ksl, g.d, gq);
    f32x4 sum[PAIRS][2];
#pragma unroll
    for (int i = 0; i < PAIRS; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) sum[i][e] = f32x4{0.f, 0.f, 0.f, 0.f};

    // tiles of 16 query rows from the first that sees a key of the workgroup, head by head
    const int r0 = max(0, key0 - g.q0) & ~15, per_head = (g.Lq - r0 + 15) >> 4;
    int hl = 0, tile = w;
    F qf[1];
    float l2;                                               // this lane's query, log2 units; +inf: no such query, or one without a key
    auto load_rows = [&]() {
        const int h = kv * g.G + hl, row = r0 + 16 * tile + x, at = min(row, g.Lq - 1);
        qf[0].load(Qp + b * g.qsb + h * g.qsh + (long long)at * g.qsl, g.d, gq);
        const float l = lse[((long long)b * g.Hq + h) * g.Lq + at];
        l2 = row < g.Lq && l != -INF ? l * 1.4426950408889634f : INF;
    };
    auto settle = [&]() {                                   // tiles past a head's end are the next head's
        while (tile >= per_head && hl < g.G) { tile -= per_head; ++hl; }
    };
    settle();
    if (hl < g.G) load_rows();
    while (hl < g.G) {
        f32x4 s[PAIRS][1][2];
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
#pragma unroll
            for (int e = 0; e < 2; ++e) s[i][0][e] = f32x4{0.f, 0.f, 0.f, 0.f};
            F::template qk<1>(s[i], kf[i], qf);
        }
        const float l_now = l2;
        const int first = g.q0 + r0 + 16 * tile;            // position of the tile's first query
        tile += KW;
        settle();
        if (hl < g.G) load_rows();
        if (first >= key0 + kKeys - 1) {
#pragma unroll
            for (int i = 0; i < PAIRS; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sum[i][e][r] += __builtin_amdgcn_exp2f(fmaf(s[i][0][e][r], scale_log2, -l_now));
        } else {
#pragma unroll
            for (int i = 0; i < PAIRS; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float p = __builtin_amdgcn_exp2f(fmaf(s[i][0][e][r], scale_log2, -l_now));
                        sum[i][e][r] += key0 + 32 * i + 16 * e + 4 * gq + r <= first + x ? p : 0.f;
                    }
        }
    }
#pragma unroll
    for (int i = 0; i < PAIRS; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float v = sum[i][e][r];
#pragma unroll
                for (int o = 1; o < 16; o <<= 1) v += __shfl_xor(v, o);
                if (x == 0) s_sum[w][32 * i + 16 * e + 4 * gq + r] = v;
            }
    __syncthreads();
    for (int k = t; k < kKeys; k += 64 * KW) {
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < KW; ++i) v += s_sum[i][k];
        if (key0 + k < g.L) out[((long long)b * g.Hkv + kv) * g.L + key0 + k] = v;
    }
}

}  // namespace

// expects batch and Hkv within 65535
hipError_t launch_key_weights(const Geom& g, int dtype, const void* Q, const void* K, const float* lse, float* out, hipStream_t st) {
    const float scale_log2 = (float)(1.4426950408889634 / sqrt((double)g.d));
    auto launch = [&](auto kernel, auto type, int keys, int waves) -> hipError_t {
        typedef decltype(type) T;
        hipLaunchKernelGGL(kernel, dim3((unsigned)((g.L + keys - 1) / keys), (unsigned)g.Hkv, (unsigned)g.batch), dim3(64 * waves), 0, st, g,
                           reinterpret_cast<const T*>(Q), reinterpret_cast<const T*>(K), lse, out, scale_log2);
        return hipGetLastError();
    };
    auto pick = [&](auto tiles) -> hipError_t {
        constexpr int N = decltype(tiles)::value;
        constexpr int kBf16 = N <= 8 ? 4 : 2, kF32 = N <= 4 ? 2 : 1, kOcc = N <= 8 ? 2 : 1;
        return dtype == RR_BF16 ? launch(k_key_weights<bf16_t, N, kBf16, 4, kOcc>, bf16_t{}, 32 * kBf16, 4)
                                : launch(k_key_weights<float, N, kF32, 4, kOcc>, float{}, 32 * kF32, 4);
    };
    using std::integral_constant;
    switch ((g.d + 15) / 16) {
#define RR_WEIGHTS_CASE(N) case N: return pick(integral_constant<int, N>{})
        RR_WEIGHTS_CASE(1); RR_WEIGHTS_CASE(2); RR_WEIGHTS_CASE(3); RR_WEIGHTS_CASE(4);
        RR_WEIGHTS_CASE(5); RR_WEIGHTS_CASE(6); RR_WEIGHTS_CASE(7); RR_WEIGHTS_CASE(8);
        RR_WEIGHTS_CASE(9); RR_WEIGHTS_CASE(10); RR_WEIGHTS_CASE(11); RR_WEIGHTS_CASE(12);
        RR_WEIGHTS_CASE(13); RR_WEIGHTS_CASE(14); RR_WEIGHTS_CASE(15); RR_WEIGHTS_CASE(16);
#undef RR_WEIGHTS_CASE
        default: return hipErrorInvalidValue;
    }
}

}  // namespace rr
