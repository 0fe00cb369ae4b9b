// Causal attention with a sliding window and sinks on the gfx950 matrix cores, bf16, d = 128: the pipeline of the block-sparse
// kernel (rr_attn_pipe.hpp; rr_attn_mfma.hip describes it) over the key blocks that all of a workgroup's 128 queries see, and
// a plain masked pass over those that some of them see.
//
// Query block m (positions 128 m .. +127) sees in full the blocks 128 n > 128 m + 127 - window, n < m, and in front of them those
// that hold nothing but sinks; in part the diagonal one, the one or two that the windows' first keys fall into, and the one that
// the sinks end in.  What bounds it: the matrix pipe (4 d operations a visible pair); the partial blocks, three or four at most, cost
// about twice a whole one, a window of 4096 positions has 31 of those.
//
// Not taken (us, 8192 tokens, 32 / 8 heads; windows of 128, 256, 512, 1000: 73, 82, 106, 163): the masked tiles staged a half ahead of their
// use 77, 87, 111, 171; 32 positions of a KV group's four heads to a workgroup, whose windows differ by less, 66, 93, 122, 185 (every
// wave then meets every masked key, where with 128 positions a wave skips most of those that are not its queries').
//
// Rows are dealt to the XCDs in eight runs, group after group, the heads of a group next to each other and then the query blocks:
// rows that run on an XCD at the same time then walk nearly the same window (2 MB of K and V for 4096 positions) in its 4 MB of L2.
//
// Measured: 32768 tokens, 32 / 8 heads, window 4096, 4 sinks 1.89 to 1.99 ms (1.04 to 1.09 PFLOP/s); 16384, window 2048 0.53 ms; 8192, window
// 512 0.11 ms.
//
// Values of keys that no query of the block sees are not read: a partial block's rows in front of the windows, behind the sinks or
// past the length are copies of the nearest row that some query sees (masked for everyone).
#include "rr_attn_pipe.hpp"

#include <algorithm>
#include <type_traits>

namespace rr {

namespace {

struct WindowKernelArgs {
    Geom g;
    WindowArgs a;
    float scale_log2;
    float lazy_log2, lazy_sum;
    int m0, Nbq;                       // first query block, and how many
    int rows, share;                   // (KV group, head, query block) rows of the launch, and an XCD's run of them
};

// One half (64 keys) of a block whose rows `lo` .. `hi` and those below `sinks` (counted in the block) some query sees
__device__ __forceinline__ void issue_clamped(const Stager& st, const unsigned short* base, int n, int hf, unsigned dst, bool is_v, int sinks,
                                              int lo, int hi, int lane) {
    const unsigned short* block = base + (long long)n * 128 * st.ksl;
    const int r4 = lane >> 4, c = lane & 15;
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
        const int row = 4 * i + r4;                          // LDS row inside the wave's rows: decides the swizzle
        const int at = kTileKeys * hf + kRowsPerWave * st.wv + row;
        const int src_row = at < sinks ? at : max(min(at, hi), lo);
        const unsigned sw = is_v ? ((row & 7) << 1) : (row & 15);
        const unsigned off = 2u * ((unsigned)(src_row * st.ksl) + 8u * (c ^ sw));
        asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1"
                     :: "v"(off), "s"(block), "s"(dst + 4 * i * 256) : "memory");
    }
}

// kRagged: the queries begin or the keys end inside a block: clamped Q rows, predicated stores.
template <bool kRagged>
__global__ void __launch_bounds__(kThreads, 2)
k_window_mfma(WindowKernelArgs ka) {
    extern __shared__ __align__(16) unsigned char lds_generic[];
    lds_byte_t* lds = (lds_byte_t*)lds_generic;
    const float NEG_INF = -__builtin_huge_valf();
    const Geom& g = ka.g;
    const WindowArgs& a = ka.a;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);

    const int flat = ((int)blockIdx.x & 7) * ka.share + ((int)blockIdx.x >> 3);
    if (((int)blockIdx.x >> 3) >= ka.share || flat >= ka.rows) return;
    int id = flat;
    const int hl = id % g.G;
    id /= g.G;
    const int mq = id % ka.Nbq, grp = id / ka.Nbq;
    const int b = grp / g.Hkv, kv = grp - b * g.Hkv, h = kv * g.G + hl, m = ka.m0 + mq;

    Wave w;
    w.lds = lds;
    w.lane = lane; w.l32 = lane & 31; w.gsel = lane >> 5;
    w.sl2 = ka.scale_log2;
    w.lazy = ka.lazy_log2;
    w.lazy_sum = ka.lazy_sum;
    w.tight = true;
    w.init_addresses();
    const int l32 = w.l32, gsel = w.gsel;
    Stager st;
    st.Kp = reinterpret_cast<const unsigned short*>(a.K) + b * g.ksb + kv * g.ksh;
    st.Vp = reinterpret_cast<const unsigned short*>(a.V) + b * g.ksb + kv * g.ksh;
    st.ksl = g.ksl;
    st.lds0 = (unsigned)(uintptr_t)w.lds;
    st.wv = wv;
    st.init(lane);

    // ---- what the block's queries see ----
    int f = a.seq_first ? __builtin_amdgcn_readfirstlane(a.seq_first[m]) : 0;
    f = f < 0 ? 0 : (f > m ? m : f);
    const int s0 = 128 * f;                                  // the sequence's first position
    const int p_first = max(128 * m, g.q0), p_last = min(128 * m + 127, g.L - 1);
    const int W = a.window, s_end = min(s0 + min(a.sinks, g.L), g.L);          // sinks: s0 .. s_end - 1
    const int lo_first = max(s0, p_first - W + 1);           // first key of any window
    const int w_any = lo_first >> 7;                         // first block that some query's window reaches
    // (from the block's last position whether it exists or not: blocks a little further on are taken as partial ones)
    const int w_full = max(f, min(m, (128 * m + 128 - W + 127) >> 7 > 0 ? (128 * m + 128 - W + 127) >> 7 : 0));
    const int s_full = min(s_end >> 7, w_any);               // blocks f .. s_full - 1 hold nothing but sinks
    const int n_sink = max(0, s_full - f), cnt = n_sink + m - w_full;
    const bool sink_part = s_end > 128 * (f + n_sink) && f + n_sink < w_any;    // block f + n_sink: sinks end inside it
    auto block_at = [&](int it) {
        it = min(it, cnt - 1);
        return it < n_sink ? f + it : w_full + it - n_sink;
    };

    // ---- Q^T operand (rows that do not exist: a copy of the nearest real one) ----
    {
        const unsigned short* Qp = reinterpret_cast<const unsigned short*>(a.Q) + b * g.qsb + h * g.qsh;
        int row = 128 * m + 32 * wv + l32 - g.q0;
        if (kRagged) row = max(min(row, g.Lq - 1), 0);
#pragma unroll
        for (int kc = 0; kc < 8; ++kc) w.qf[kc] = *reinterpret_cast<const bf16x8*>(Qp + (long long)row * g.qsl + 16 * kc + 8 * gsel);
    }
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) w.acc[dt][r] = 0.f;
    w.mref = NEG_INF;
    w.lsum = 0.f;
    w.lfix = 0.f;                                            // (stays that: the sums are those of the probabilities before rounding)
    f32x16 sa, sb;
    bf16x8 pa[2], pb[2];

    if (cnt > 0) {
        // the loop of the block-sparse kernel (see there); past the last block it fetches that block once more
        int n_next = block_at(0);
        st.issue_k(n_next, 0, 0);
        wait_vm();
#pragma unroll
        for (int kc = 0; kc < 8; ++kc) asm volatile("" : "+a"(w.qf[kc]));      // complete here, not in the loop
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) { pa[c][e] = (__bf16)0.f; pb[c][e] = (__bf16)0.f; }
        int n_cur = n_next;
        auto tile = [&](auto half, bool fill, bool more, int nk, int nv) {
            constexpr int HF = decltype(half)::value;
            constexpr int KO = (HF ^ 1) * kTileBytes;
            constexpr int VO = HF * kTileBytes;
            phase<true, VO, KO, true>(w, sb, sa, pa, pb, !fill, st, st.k_src(nk, HF), st.k_dst(HF), st.v_src(nv, HF ^ 1), st.v_dst(HF ^ 1));
            phase<false, VO + 32 * 256, KO + 32 * 256, true>(w, sa, sb, pb, pa, more, st, nullptr, 0, nullptr, 0);
        };
        using std::integral_constant;
        for (int i = -1; i < cnt; ++i) {
            if (i >= 0) {
                __syncthreads();
                tile(integral_constant<int, 0>{}, false, true, n_next, n_cur);
                wait_vm();
            }
            __syncthreads();
            const int n2 = block_at(i + 2);
            tile(integral_constant<int, 1>{}, i < 0, i + 1 < cnt, n_next, n_next);
            if (i < 0) {
                mfma_settle_acc(w.acc);
#pragma unroll
                for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) w.acc[dt][r] = 0.f;
                mfma_settle_acc(w.acc);
            }
            wait_vm();
            n_cur = n_next;
            n_next = n2;
        }
        mfma_settle_acc(w.acc);
        mfma_settle_s(sa);
        mfma_settle_s(sb);
    }

    // ---- blocks that some queries see: masked key by key, nothing overlapped inside the wave ----
    const int pos = 128 * m + 32 * wv + l32, w_lo = 128 * m + 32 * wv, w_hi = w_lo + 31;       // of the lane's query, of the wave's
    auto partial_block = [&](int n) {
        const int k0 = 128 * n;
        const int lo = lo_first - k0, hi = min(127, g.L - 1 - k0), sinks = s_end - k0;         // rows of the block that some query sees
        __syncthreads();                                     // the buffers are free
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const int h0 = 64 * hf;                          // a half that no query sees stays out
            if (!(h0 < sinks || (h0 + 63 >= lo && h0 <= p_last - k0))) continue;
            // (no window reaches the block: the sinks' last row instead)
            const int first = lo > hi ? max(sinks - 1, 0) : max(lo, 0), last = lo > hi ? first : hi;
            issue_clamped(st, st.Kp, n, hf, st.k_dst(hf), false, sinks, first, last, lane);
            issue_clamped(st, st.Vp, n, hf, st.v_dst(hf), true, sinks, first, last, lane);
        }
        wait_vm();
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int key = k0 + 32 * j;
            if (key > w_hi || !(key + 31 > w_lo - W || key < s_end)) continue;
            f32x16& s = (j & 1) ? sb : sa;
            qk_step(w, j >> 1, j & 1, s);
            const bool whole = key + 31 <= w_lo && (key > w_hi - W || key + 31 < s_end);
            if (!whole) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int k = key + 8 * (r >> 2) + 4 * gsel + (r & 3);
                    s[r] = k <= pos && (k > pos - W || k < s_end) ? s[r] : NEG_INF;
                }
            }
            softmax_step<true>(w, s, pa);
            pv_step(w, j >> 1, j & 1, pa);
        }
    };
    // (one loop, so that the pass is there once: 12700 instructions so, 6400)
    const int in_front = sink_part ? 1 : 0, partial = in_front + w_full - w_any + 1;
    for (int i = 0; i < partial; ++i) partial_block(i < in_front ? f + n_sink : i + 1 < partial ? w_any + i - in_front : m);
    __syncthreads();

    // ---- normalise, write ----
    const float l = w.lsum + __shfl_xor(w.lsum, 32);
    const float inv = l > 0.f ? 1.0f / l : 0.f;
    unsigned char* ost = lds_generic + wv * (32 * kOutRowBytes);
    const long long wrow0 = (long long)w_lo - g.q0;          // row of Q and O of the wave's first query
    const int rows_q = kRagged ? (int)min(32ll, (long long)g.Lq - wrow0) : 32, rows_lo = kRagged ? (int)max(0ll, -wrow0) : 0;
    if (a.lse && gsel == 0 && l32 < rows_q && l32 >= rows_lo)
        a.lse[((long long)b * g.Hq + h) * g.Lq + wrow0 + l32] = l > 0.f ? w.mref * 0.6931471805599453f + logf(l) : NEG_INF;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int rg = 0; rg < 4; ++rg) {
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = w.acc[dt][4 * rg + e] * inv;
            const u32x2 o = {f32_to_bf16_bits(v[0]) | (f32_to_bf16_bits(v[1]) << 16), f32_to_bf16_bits(v[2]) | (f32_to_bf16_bits(v[3]) << 16)};
            *reinterpret_cast<u32x2*>(ost + l32 * kOutRowBytes + 2 * (32 * dt + 8 * rg + 4 * gsel)) = o;
        }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    unsigned short* Op = reinterpret_cast<unsigned short*>(a.O) + b * g.qsb + h * g.qsh + wrow0 * g.qsl;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int idx = lane + 64 * k, row = idx >> 4, ch = idx & 15;
        const u32x2 lo = *reinterpret_cast<const u32x2*>(ost + row * kOutRowBytes + 16 * ch);
        const u32x2 hi = *reinterpret_cast<const u32x2*>(ost + row * kOutRowBytes + 16 * ch + 8);
        const u32x4 o = {lo[0], lo[1], hi[0], hi[1]};
        if (row < rows_q && row >= rows_lo) *reinterpret_cast<u32x4*>(Op + (long long)row * g.qsl + 8 * ch) = o;
    }
}

}  // namespace

bool window_mfma_takes(const Geom& g, int dtype, const int32_t* seq_first, int B) {
    if (dtype != RR_BF16 || g.d != 128 || (seq_first && B != 128)) return false;
    // a tile's rows are addressed by 32-bit byte offsets from its first
    if (g.ksl > (1ll << 23)) return false;
    // A launch of few such rows ends when its longest does, and the generic kernel has four or eight times as many workgroups.  This
    // kernel / that one, us: 512 positions, window 200, 32 heads (128 rows) 22.1 / 15.4; 2048, window 512, 8 heads (128) 24.3 / 21.9; 200
    // of 24000, window 4096, 32 heads (64) 71 / 55, 500 (128 to 160) 73 / 87; 1024, 32 heads (256) 26.2 / 39.6.
    const long long rows = (long long)g.batch * g.Hq * ((g.L - 1) / 128 - g.q0 / 128 + 1);
    return rows > 128 && rows < (1ll << 23);
}

hipError_t launch_window_mfma(const Geom& g, const WindowArgs& a, hipStream_t st) {
    WindowKernelArgs ka;
    ka.g = g;
    ka.a = a;
    ka.scale_log2 = (float)(1.4426950408889634 / sqrt((double)g.d));
    ka.lazy_log2 = 8.0f;
    ka.lazy_sum = exp2f(ka.lazy_log2);
    ka.m0 = g.q0 / 128;
    ka.Nbq = (g.L - 1) / 128 - ka.m0 + 1;
    ka.rows = g.batch * g.Hq * ka.Nbq;
    ka.share = (ka.rows + 7) / 8;
    const bool ragged = g.L % 128 || g.q0 % 128;
    const void* kernel = ragged ? reinterpret_cast<const void*>(k_window_mfma<true>) : reinterpret_cast<const void*>(k_window_mfma<false>);
    const hipError_t e = allow_dynamic_lds(kernel, kLdsBytes);
    if (e != hipSuccess) return e;
    const dim3 grid(8u * (unsigned)ka.share);
    if (ragged) hipLaunchKernelGGL(k_window_mfma<true>, grid, dim3(kThreads), kLdsBytes, st, ka);
    else hipLaunchKernelGGL(k_window_mfma<false>, grid, dim3(kThreads), kLdsBytes, st, ka);
    return hipGetLastError();
}

}  // namespace rr
