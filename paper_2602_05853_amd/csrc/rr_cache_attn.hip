// Attention of a step (one new token, or a few) over a key-value cache in pages, and over the contiguous keys and values of a
// step with a sliding window: O_r = sum_j p_rj v_j, p_rj = exp(q_r k_j / sqrt(d)) / sum, over the keys that row r sees.
//
// What bounds it: the stream of the visible keys and values, each read once (2 d values per key and KV head against 4 d G T
// operations on them).  So a workgroup serves all G T rows of a KV head from the same keys (the rows are the columns of
// matrix tiles, rr_attn_frag.hpp), straight from memory to registers, the next keys requested before the softmax of the
// present ones; and the blocks of all sequences are dealt out evenly to one round of workgroups (rr_cache.hpp), each of which
// writes its parts' normalised outputs and log-sum-exps.  A second kernel joins the parts of every row.
// Arithmetic: fp32 throughout; bf16 scores are exact products summed in fp32, probabilities three exact bf16 terms.
//
// A tile of 16 keys lies in one page (pages are multiples of 16 positions), so an address is one page entry, read by a
// scalar load a step ahead, and the lane's row offsets.  Tiles without a page, or behind the end, are not read.
//
// Weights: the first kernel also keeps its scores (4 bytes per row and key against the 4 d and 8 d of a key's K and V), and a
// third adds exp(score - lse) over the rows of a KV head, in the order of the rows, to the positions' sums.
//
// Measured (bf16, 32 / 8 heads of 128): one token over 128K positions 96 us (5.6 TB/s) and 5.8 to join; 64 sequences of 200 to 16384,
// pages of 16, 442 + 9 + 27 us (the first at 4.9 TB/s); a step over a window of 8192 11.4 + 4.6 us.  Tried and not kept: the values of
// the next step requested with its keys (no change), three workgroups to a compute unit (128 us, spills), runs of shares to an XCD
// (no change, short steps 17.4 -> 19.7).
#include "rr_cache.hpp"
#include "rr_attn_frag.hpp"

#include <algorithm>
#include <type_traits>

namespace rr {

namespace {

constexpr int kCacheWorkgroups = 512;                   // two per compute unit, all resident
// Sequences that visit few blocks are not shared out: a workgroup to each (and KV head), one launch instead of two.  Shared / not, us,
// bf16, 32 / 8 heads: 1 sequence of 128 positions 12.1 / 9.6, 512 11.8 / 10.5, 1024 11.9 / 16.3; 16 sequences of 512 14.7 / 11.5, 640
// 20.0 / 13.8, 1024 20.8 / 19.0, 2048 29.6 / 32.3; 64 of 256 23.9 / 14.7, 1024 51.9 / 42.4, 2048 106 / 95 (but uneven ones of so many
// blocks would end when the longest does).
constexpr int kWholeBlocks = 4, kWholeBlocksOfMany = 8, kMany = 128;

__device__ __forceinline__ void store4(float* p, const f32x4& v) { *reinterpret_cast<f32x4*>(p) = v; }
__device__ __forceinline__ void store4(bf16_t* p, const f32x4& v) {
    const u32x2 o = {f32_to_bf16_bits(v[0]) | (f32_to_bf16_bits(v[1]) << 16),
                     f32_to_bf16_bits(v[2]) | (f32_to_bf16_bits(v[3]) << 16)};
    *reinterpret_cast<u32x2*>(p) = o;
}

// D: d where it fills the matrix tiles, so that a row's last channels need no check (which would wait for the keys in front of
// the work they are requested ahead of), or 0.
template <typename T, int NT, int D, int QT, int TL, int KW>
__global__ void __launch_bounds__(64 * KW, NT > 8 ? 1 : 2)
k_cache_attn(CacheArgs c) {
    using F = Frag<T, NT, TL>;
    constexpr int kThreads = 64 * KW, kQ = 16 * QT, kPitch = 16 * NT + 4;
    constexpr int kStep = 16 * TL * KW, kSteps = kUnit / kStep;      // keys of the workgroup at once, and trips to a block
    static_assert(kStep * kSteps == kUnit, "a block is whole steps");
    __shared__ __align__(16) float s_o[KW][kQ][kPitch];
    __shared__ float s_ref[KW][kQ], s_l[KW][kQ];
    __shared__ Shares<kThreads> s_shares;
    const float NEG_INF = -__builtin_huge_valf();
    const int d = D ? D : c.d;

    const int tid = threadIdx.x, lane = tid & 63, x = lane & 15, gq = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int R = c.G * c.T, pairs = c.Hkv * c.row_tiles;

    unsigned u, u_end;                                  // units (fewer than 2^31)
    Visit v;
    int b, pair, i_lo, upto = 0, base = 0;
    if (c.whole) {
        // a workgroup to a sequence and pair, which stores its rows itself (their units are numbered as if all sequences visited as
        // many blocks as any may)
        b = (int)blockIdx.x / pairs;
        pair = (int)blockIdx.x - b * pairs;
        i_lo = 0;
        v = visit(c, b);
        u = blockIdx.x * (unsigned)c.whole;
        u_end = u + (unsigned)v.n;
    } else {
        const int total = shares_scan(c, s_shares, upto);
        const Deal deal((unsigned)total * (unsigned)pairs, gridDim.x);
        if (blockIdx.x >= deal.W) return;
        u = deal.start(blockIdx.x);
        u_end = deal.start(blockIdx.x + 1);
        b = shares_find(c, s_shares, upto, (int)(u / (unsigned)pairs), &base, &v);
        const unsigned in_b = u - (unsigned)base * (unsigned)pairs;
        pair = (int)(in_b / (unsigned)v.n);
        i_lo = (int)(in_b - (unsigned)pair * (unsigned)v.n);
        // the join's: the workgroup that has a sequence's first unit says where the sequence begins
        if (tid == 0 && in_b == 0) c.front[b] = base;
        if (tid == 0 && blockIdx.x == 0) c.front[c.batch] = total;
    }

    // rows of a tile this lane reads, relative to its first key
    const long long k_off = (long long)x * c.ksl;
    long long v_off[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) v_off[r] = (long long)(4 * gq + r) * c.ksl;

    do {
        const int blocks = min(v.n - i_lo, (int)(u_end - u));
        const int kv = c.row_tiles == 1 ? pair : pair / c.row_tiles, rt = pair - kv * c.row_tiles;
        const int q_first = v.len - c.T, q_last = v.len - 1;

        // rows that do not exist repeat the last one and are not stored
        F qf[QT];
        int qpos[QT];
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const int rr = min(kQ * rt + 16 * t + x, R - 1), hl = c.T == 1 ? rr : rr / c.T, tk = rr - hl * c.T;
            qf[t].load(reinterpret_cast<const T*>(c.Q) + b * c.qsb + (long long)(kv * c.G + hl) * c.qsh + (long long)tk * c.qsl, d, gq);
            qpos[t] = q_first + tk;
        }
        const T* K = reinterpret_cast<const T*>(c.K) + (long long)kv * c.ksh;
        const T* V = reinterpret_cast<const T*>(c.V) + (long long)kv * c.ksh;
        const int steps = blocks * kSteps;
        auto first_key = [&](int st, int tl) { return v.block(i_lo + st / kSteps) * kUnit + (st % kSteps) * kStep + 16 * (TL * w + tl); };
        // page entries of a step, as loaded
        int entry[TL];
        auto request = [&](int st) {
#pragma unroll
            for (int tl = 0; tl < TL; ++tl) {
                const int key = first_key(st, tl);
                entry[tl] = c.table ? ((scalar_words_t)c.table)[(long long)b * c.width + page_of(c, min(key, q_last))] : 0;
            }
        };
        F kf[TL];
        int key0[TL], last[TL];                          // first key of a tile; the last of its keys that exists, -1: none does
        long long at[TL];                                // where the tile begins
        auto load_keys = [&](int st) {                   // the step's entries are in `entry`
#pragma unroll
            for (int tl = 0; tl < TL; ++tl) {
                key0[tl] = first_key(st, tl);
                const bool in = key0[tl] < v.len && (!c.table || (unsigned)entry[tl] < (unsigned)c.num_pages);
                last[tl] = in ? min(15, v.len - 1 - key0[tl]) : -1;
                at[tl] = c.table ? (long long)entry[tl] * c.psb + (long long)(key0[tl] - page_of(c, key0[tl]) * c.page) * c.ksl
                                 : (long long)b * c.psb + (long long)key0[tl] * c.ksl;
                if (last[tl] == 15) kf[tl].load(K + at[tl] + k_off, d, gq);
                else if (in) kf[tl].load(K + at[tl] + (long long)min(x, last[tl]) * c.ksl, d, gq);
                else kf[tl] = F{};
            }
        };
        auto load_values = [&](typename F::V& vf) {      // of the keys loaded last
#pragma unroll
            for (int tl = 0; tl < TL; ++tl)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    if (last[tl] == 15) F::load_v(vf, 4 * tl + r, V + at[tl] + v_off[r], d, x);
                    else if (last[tl] >= 0) F::load_v(vf, 4 * tl + r, V + at[tl] + (long long)min(4 * gq + r, last[tl]) * c.ksl, d, x);
                    else F::drop(vf, 4 * tl + r, true);
                }
        };
        f32x4 acc[QT][NT];
        float ref[QT], lsum[QT];
        auto walk = [&](auto careful) {
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                ref[t] = NEG_INF;
                lsum[t] = 0.f;
#pragma unroll
                for (int ch = 0; ch < NT; ++ch) acc[t][ch] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
            if (steps > 0) {
                request(0);
                load_keys(0);
                request(min(1, steps - 1));
            }
            for (int st = 0; st < steps; ++st) {
                typename F::V vf;
                load_values(vf);
                f32x4 s[QT][TL];
#pragma unroll
                for (int t = 0; t < QT; ++t)
#pragma unroll
                    for (int tl = 0; tl < TL; ++tl) s[t][tl] = f32x4{0.f, 0.f, 0.f, 0.f};
                F::template qk<QT>(s, kf, qf);
                int key_now[TL], last_now[TL];
#pragma unroll
                for (int tl = 0; tl < TL; ++tl) {
                    key_now[tl] = key0[tl];
                    last_now[tl] = last[tl];
                    const bool whole = last[tl] == 15 && key0[tl] + 15 <= q_first &&
                                       (key0[tl] > q_last - c.window || key0[tl] + 15 < c.sinks);
                    if (!whole) {
#pragma unroll
                        for (int t = 0; t < QT; ++t) {
                            f32x4 x4 = s[t][tl];
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                const int k = 4 * gq + r, key = key0[tl] + k;
                                const bool sees = k <= last[tl] && key <= qpos[t] && (key > qpos[t] - c.window || key < c.sinks);
                                x4[r] = sees ? x4[r] : NEG_INF;
                            }
                            s[t][tl] = x4;
                        }
                    }
                    if (c.scores) {
                        const int rows = min(R, kQ);
                        float* out = c.scores + (long long)(u + st / kSteps) * rows * kUnit + (st % kSteps) * kStep + 16 * (TL * w + tl) + 4 * gq;
#pragma unroll
                        for (int t = 0; t < QT; ++t)
                            if (16 * t + x < rows) *reinterpret_cast<f32x4*>(out + (16 * t + x) * kUnit) = s[t][tl];
                    }
                }
                // the next step's keys travel during the softmax and the second product, the entries behind them through
                // the next step (the careful walk has no registers for it)
                auto ahead = [&]() {
                    if (st + 1 < steps) {
                        load_keys(st + 1);
                                request(min(st + 2, steps - 1));
                    }
                };
                if (!decltype(careful)::value) ahead();
                float p[QT][4 * TL];
#pragma unroll
                for (int t = 0; t < QT; ++t) frag_softmax<TL, NT>(s[t], c.scale_log2, ref[t], lsum[t], acc[t], p[t]);
                if constexpr (decltype(careful)::value) {
                    // values of keys that no row sees are left out
#pragma unroll
                    for (int tl = 0; tl < TL; ++tl)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int k = 4 * gq + r, key = key_now[tl] + k;
                            F::drop(vf, 4 * tl + r, k > last_now[tl] || key > q_last || !(key > q_first - c.window || key < c.sinks));
                        }
                }
                F::template pv<QT, decltype(careful)::value>(acc, vf, p);
                if (decltype(careful)::value) ahead();
            }
        };
        walk(std::false_type{});
        if (has_nan(acc)) walk(std::true_type{});

        // the waves' shares, brought to one reference: the part's normalised output and log2 of its sum of exponentials
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            float l = lsum[t];
            l += __shfl_xor(l, 16);
            l += __shfl_xor(l, 32);
            if (gq == 0) { s_ref[w][16 * t + x] = ref[t]; s_l[w][16 * t + x] = l; }
            frag_store<F::kW, NT>(acc[t], &s_o[w][16 * t + x][0], gq);
        }
        __syncthreads();
        const long long slot = blockIdx.x + (long long)b * pairs + pair;
        for (int idx = tid; idx < kQ * 4 * NT; idx += kThreads) {
            const int q = idx / (4 * NT), ch = 4 * (idx - q * (4 * NT));
            if (kQ * rt + q >= R || ch >= d) continue;
            float top = NEG_INF;
#pragma unroll
            for (int i = 0; i < KW; ++i) top = fmaxf(top, s_ref[i][q]);
            float l = 0.f;
            f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < KW; ++i) {
                const float f = s_ref[i][q] == NEG_INF ? 0.f : __builtin_amdgcn_exp2f(s_ref[i][q] - top);
                l = fmaf(f, s_l[i][q], l);
                const f32x4 part = *reinterpret_cast<const f32x4*>(&s_o[i][q][ch]);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = fmaf(f, part[e], o[e]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = l > 0.f ? o[e] / l : 0.f;
            if (!c.whole) {
                *reinterpret_cast<f32x4*>(c.part_O + (slot * kQ + q) * d + ch) = o;
                if (ch == 0) c.part_lse[slot * kQ + q] = l > 0.f ? top + log2f(l) : NEG_INF;
            } else {
                const int rr = kQ * rt + q, hl = c.T == 1 ? rr : rr / c.T, tk = rr - hl * c.T, h = kv * c.G + hl;
                store4(reinterpret_cast<T*>(c.O) + b * c.qsb + h * c.qsh + tk * c.qsl + ch, o);
                if (ch == 0) {
                    const float l2 = top + log2f(l);
                    if (c.lse) c.lse[((long long)b * c.Hq + h) * c.T + tk] = l > 0.f ? l2 * 0.6931471805599453f : NEG_INF;
                    if (c.row_lse) c.row_lse[((long long)b * c.Hkv + kv) * R + rr] = l > 0.f ? l2 : -NEG_INF;
                }
            }
        }
        __syncthreads();                                 // the shares' places are free again

        u += (unsigned)blocks;
        i_lo += blocks;
        if (i_lo == v.n && u < u_end) {
            i_lo = 0;
            if (++pair == pairs) {
                pair = 0;
                b = shares_find(c, s_shares, upto, base + v.n, &base, &v);   // (units are left; empty sequences are passed over)
                if (tid == 0) c.front[b] = base;
            }
        }
    } while (u < u_end);
}

// One workgroup per query row: O = sum_p w_p O_p / sum_p w_p with w_p = 2^(lse_p - max), rounded once.
// A wave takes every KW-th part, eight requested at once, the first eight in front of everything that waits: one at a time, after the
// weights, their latencies were the kernel (64 parts 15.4 us, so 5.4).
template <typename T, int KW>
__global__ void __launch_bounds__(64 * KW)
k_cache_join(CacheArgs c, int row_tile, int workgroups) {
    constexpr int kThreads = 64 * KW, kAtOnce = 8;
    __shared__ float s_w[kCacheWorkgroups];
    __shared__ float s_red[KW], s_den[KW];
    __shared__ __align__(16) float s_o[KW][256];
    const float NEG_INF = -__builtin_huge_valf();
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int R = c.G * c.T, pairs = c.Hkv * c.row_tiles;
    const int row = blockIdx.x;                          // (b, kv, r)
    const int bk = row / R, r = row - bk * R, b = bk / c.Hkv, kv = bk - b * c.Hkv;
    const int rt = c.row_tiles == 1 ? 0 : r / row_tile, in_tile = r - rt * row_tile, pair = kv * c.row_tiles + rt;

    // (a scan of the lengths here as well would read batch lengths for each of batch rows: 20000 sequences, five of them with keys: 6731 us, so 224)
    const Visit v = visit(c, b);
    int parts = 0;
    long long first = 0;
    if (v.n > 0) {                                       // (else nobody has written its front)
        const Deal deal((unsigned)c.front[c.batch] * (unsigned)pairs, (unsigned)workgroups);
        const unsigned u = (unsigned)c.front[b] * (unsigned)pairs + (unsigned)pair * (unsigned)v.n;
        first = deal.owner(u);
        parts = (int)(deal.owner(u + (unsigned)v.n - 1) - (unsigned)first) + 1;
    }
    const long long slot = first + (long long)b * pairs + pair;
    const float* lse = c.part_lse + slot * row_tile + in_tile;
    const float* O = c.part_O + (slot * row_tile + in_tile) * c.d;

    // a lane has the channels 2 lane, 2 lane + 1, and the two 128 behind them
    const int ch = 2 * lane;
    float2 x[kAtOnce][2];
    auto request = [&](int p0) {
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            if (p0 + KW * i >= parts) break;             // (the same in every lane)
            const float* at = O + (long long)(p0 + KW * i) * row_tile * c.d;
            x[i][0] = *reinterpret_cast<const float2*>(at + (ch < c.d ? ch : 0));
            if (c.d > 128) x[i][1] = *reinterpret_cast<const float2*>(at + (128 + ch < c.d ? 128 + ch : 0));
        }
    };
    request(wv);
    float mx = NEG_INF;
    for (int p = tid; p < parts; p += kThreads) {
        const float l = lse[(long long)p * row_tile];
        s_w[p] = l;
        mx = fmaxf(mx, l);
    }
    mx = wave_max(mx);
    if (lane == 0) s_red[wv] = mx;
    __syncthreads();
    mx = s_red[0];
#pragma unroll
    for (int i = 1; i < KW; ++i) mx = fmaxf(mx, s_red[i]);

    float den = 0.f;
    float2 o[2] = {{0.f, 0.f}, {0.f, 0.f}};
    for (int p0 = wv; p0 < parts; p0 += KW * kAtOnce) {
        if (p0 != wv) request(p0);
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            if (p0 + KW * i >= parts) break;
            const float l = s_w[p0 + KW * i];
            if (l == NEG_INF) continue;                  // (whatever it holds)
            const float wp = __builtin_amdgcn_exp2f(l - mx);
            den += wp;
            o[0].x = fmaf(wp, x[i][0].x, o[0].x);
            o[0].y = fmaf(wp, x[i][0].y, o[0].y);
            if (c.d > 128) {
                o[1].x = fmaf(wp, x[i][1].x, o[1].x);
                o[1].y = fmaf(wp, x[i][1].y, o[1].y);
            }
        }
    }
    if (lane == 0) s_den[wv] = den;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        s_o[wv][128 * k + ch] = o[k].x;
        s_o[wv][128 * k + ch + 1] = o[k].y;
    }
    __syncthreads();
    den = 0.f;
#pragma unroll
    for (int i = 0; i < KW; ++i) den += s_den[i];
    const float inv = den > 0.f ? 1.0f / den : 0.f;
    const int hl = c.T == 1 ? r : r / c.T, tk = r - hl * c.T, h = kv * c.G + hl;
    if (4 * tid < c.d) {
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KW; ++i) sum += *reinterpret_cast<const f32x4*>(&s_o[i][4 * tid]);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] *= inv;
        store4(reinterpret_cast<T*>(c.O) + b * c.qsb + h * c.qsh + tk * c.qsl + 4 * tid, sum);
    }
    if (tid == 0) {
        const float l2 = mx + log2f(den);
        if (c.lse) c.lse[((long long)b * c.Hq + h) * c.T + tk] = den > 0.f ? l2 * 0.6931471805599453f : NEG_INF;
        if (c.row_lse) c.row_lse[row] = den > 0.f ? l2 : -NEG_INF;
    }
}

// weight[page][kv][slot] += sum over the KV head's rows of 2^(score - lse): a thread to four positions (of one page), eight
// blocks of a (sequence, KV head) to a trip, trips dealt out evenly.
__global__ void __launch_bounds__(256)
k_cache_weights(CacheArgs c, int row_tile) {
    __shared__ Shares<256> s_shares;
    const int R = c.G * c.T, rows = min(R, row_tile);
    int upto, base;
    const int total = shares_scan(c, s_shares, upto);
    const unsigned items = (unsigned)total * (unsigned)c.Hkv, each = (items + gridDim.x - 1) / gridDim.x;
    unsigned i = min(items, each * blockIdx.x);
    const unsigned end = min(items, i + each);
    if (i >= end) return;
    Visit v;
    int b = shares_find(c, s_shares, upto, (int)(i / (unsigned)c.Hkv), &base, &v);
    const unsigned in_b = i - (unsigned)base * (unsigned)c.Hkv;
    int kv = (int)(in_b / (unsigned)v.n), blk = (int)(in_b - (unsigned)kv * (unsigned)v.n);
    const int eighth = threadIdx.x >> 5, k = 4 * (threadIdx.x & 31);
    while (i < end) {
        const int n = min(v.n - blk, (int)(end - i));
        for (int j = eighth; j < n; j += 8) {
            const int pos = v.block(blk + j) * kUnit + k;
            if (pos >= v.len) continue;
            const int pg = page_of(c, pos), e = c.table[(long long)b * c.width + pg];
            if ((unsigned)e >= (unsigned)c.num_pages) continue;
            float* out = c.weight + ((long long)e * c.Hkv + kv) * c.page + (pos - pg * c.page);
            const f32x4 old = *reinterpret_cast<const f32x4*>(out);
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
            for (int rt = 0; rt < c.row_tiles; ++rt) {
                const int pair = kv * c.row_tiles + rt;
                const long long u = c.whole ? ((long long)b * c.Hkv * c.row_tiles + pair) * c.whole + blk + j
                                            : (long long)base * c.Hkv * c.row_tiles + (long long)pair * v.n + blk + j;
                const float* s = c.scores + u * rows * kUnit + k;
                const float* l = c.row_lse + ((long long)b * c.Hkv + kv) * R + rt * row_tile;
                const int here = min(rows, R - rt * row_tile);
#pragma unroll 4
                for (int q = 0; q < here; ++q) {
                    const f32x4 x = *reinterpret_cast<const f32x4*>(s + q * kUnit);
                    const float l2 = l[q];
#pragma unroll
                    for (int t = 0; t < 4; ++t) sum[t] += __builtin_amdgcn_exp2f(fmaf(x[t], c.scale_log2, -l2));
                }
            }
            // (slots behind the end belong to nobody yet: they keep what they hold)
            if (pos + 3 < v.len) {
                *reinterpret_cast<f32x4*>(out) = old + sum;
            } else {
                for (int t = 0; pos + t < v.len; ++t) out[t] = old[t] + sum[t];
            }
        }
        i += (unsigned)n;
        blk += n;
        if (blk == v.n && i < end) {
            blk = 0;
            if (++kv == c.Hkv) {
                kv = 0;
                b = shares_find(c, s_shares, upto, base + v.n, &base, &v);
            }
        }
    }
}

int row_tile_of(const CacheArgs& c, int dtype) { return dtype == RR_BF16 && c.d == 128 && c.G * c.T > 16 ? 32 : 16; }

}  // namespace

bool cache_attn_plan(const CacheArgs& c, int dtype, bool accumulate, CachePlan* p) {
    const long long R = (long long)c.G * c.T;
    if (R > (1 << 24)) return false;
    p->row_tile = row_tile_of(c, dtype);
    p->row_tiles = (int)((R + p->row_tile - 1) / p->row_tile);
    const long long pairs = (long long)c.Hkv * p->row_tiles, blocks = most_blocks(c.L, c.T, c.window, c.sinks);
    // units, and the indexes of pairs and rows, are 31 bits; a launch is fewer than 2^32 threads
    if (c.batch * pairs > 0x7fffff || c.batch * c.Hkv * R > 0xffffff || c.batch * pairs * blocks > 0x7fffffff - 4096) return false;
    const long long U = c.batch * blocks * pairs;
    p->workgroups = (int)std::max(1ll, std::min<long long>(kCacheWorkgroups, U));
    p->whole = blocks <= (c.batch * pairs < kMany ? kWholeBlocks : kWholeBlocksOfMany) ? (int)blocks : 0;
    if (p->whole) p->workgroups = (int)(c.batch * pairs);
    const long long slots = p->whole ? 0 : p->workgroups + c.batch * pairs;
    p->part_rows = (size_t)slots * p->row_tile;
    p->part_bytes = p->whole ? 0 : ((p->part_rows * (c.d + 1) + c.batch + 1) * sizeof(float) + 255) / 256 * 256;
    p->score_bytes = accumulate ? (size_t)U * (size_t)std::min<long long>(R, p->row_tile) * kUnit * sizeof(float) : 0;
    p->row_bytes = accumulate ? ((size_t)c.batch * c.Hkv * R * sizeof(float) + 255) / 256 * 256 : 0;
    return true;
}

hipError_t launch_cache_attn(const CacheArgs& c, int dtype, const CachePlan& plan, hipStream_t st) {
    auto launch = [&](auto kernel, int waves) -> hipError_t {
        hipLaunchKernelGGL(kernel, dim3((unsigned)plan.workgroups), dim3(64 * waves), 0, st, c);
        return hipGetLastError();
    };
    auto pick = [&](auto tiles, auto full) -> hipError_t {
        constexpr int N = decltype(tiles)::value, D = decltype(full)::value;
        if (dtype == RR_BF16) {
            if constexpr (D == 128)
                if (plan.row_tile == 32) return launch(k_cache_attn<bf16_t, N, D, 2, 2, 4>, 4);
            return launch(k_cache_attn<bf16_t, N, D, 1, 2, 4>, 4);
        }
        if constexpr (N > 8) return launch(k_cache_attn<float, N, D, 1, 1, 4>, 4);
        else return launch(k_cache_attn<float, N, D, 1, 1, 8>, 8);
    };
    using std::integral_constant;
    hipError_t e = hipErrorInvalidValue;
    switch ((c.d + 15) / 16) {
#define RR_CACHE_CASE(N) case N: e = c.d == 16 * N ? pick(integral_constant<int, N>{}, integral_constant<int, 16 * N>{}) \
                                             : pick(integral_constant<int, N>{}, integral_constant<int, 0>{}); break
        RR_CACHE_CASE(1); RR_CACHE_CASE(2); RR_CACHE_CASE(3); RR_CACHE_CASE(4);
        RR_CACHE_CASE(5); RR_CACHE_CASE(6); RR_CACHE_CASE(7); RR_CACHE_CASE(8);
        RR_CACHE_CASE(9); RR_CACHE_CASE(10); RR_CACHE_CASE(11); RR_CACHE_CASE(12);
        RR_CACHE_CASE(13); RR_CACHE_CASE(14); RR_CACHE_CASE(15); RR_CACHE_CASE(16);
#undef RR_CACHE_CASE
        default: break;
    }
    if (e != hipSuccess) return e;
    if (!plan.whole) {
        const dim3 rows((unsigned)(c.batch * c.Hkv * c.G * c.T));
        // (rows of few parts on four waves: 64 uneven sequences, 2048 rows of two or three parts)
        auto join = [&](auto kernel, int waves) {
            hipLaunchKernelGGL(kernel, rows, dim3(64 * waves), 0, st, c, plan.row_tile, plan.workgroups);
        };
        const bool many = plan.workgroups > 16ll * c.batch * c.Hkv * c.row_tiles;
        if (dtype == RR_BF16) many ? join(k_cache_join<bf16_t, 8>, 8) : join(k_cache_join<bf16_t, 4>, 4);
        else many ? join(k_cache_join<float, 8>, 8) : join(k_cache_join<float, 4>, 4);
        e = hipGetLastError();
    }
    if (e != hipSuccess || !c.scores) return e;
    const long long items = c.batch * most_blocks(c.L, c.T, c.window, c.sinks) * c.Hkv;
    hipLaunchKernelGGL(k_cache_weights, dim3((unsigned)std::min(2048ll, (items + 7) / 8)), dim3(256), 0, st, c, plan.row_tile);
    return hipGetLastError();
}

}  // namespace rr
