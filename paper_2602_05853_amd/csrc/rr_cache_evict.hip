// Eviction by accumulated weight: of the n positions of a (sequence, KV head) the first `sinks`, the last `recent` and the
// heaviest of the others are kept, `keep` in all (all where n <= keep), in their order, in the pages of another table.
//
// First launch, one workgroup to a (sequence, KV head): the weight of the last position that is kept by weight, found by
// its bits, eleven at a time from the top (weights mapped to unsigned numbers of the same order); heavier ones are kept, of equal
// ones as many as are left, the lower positions first; every wave then writes out the positions of its own run in order.  Caches
// of more positions than LDS holds keys for: the same in launches of a workgroup to 8192 positions.
// Last launch: the rows, 16 bytes of K and of V to a thread.  What bounds it: the copy.
// Measured (8 heads of 128, bf16): 131072 to 65536 positions 110 us of copy (4.9 TB/s) and 47 in the six launches in front; 16 sequences of
// 2049 to 2304 to 2048 47 and 12.
#include "rr_cache.hpp"

#include <algorithm>

namespace rr {

namespace {

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;
constexpr int kBins = 2048, kCopies = 4;                // of a histogram: lanes of equal index mod 4 share a copy
constexpr int kKeysInLds = 24576;                       // 96 KB beside the 32 KB of the histogram

// Unsigned numbers in the order of the weights; a number that is none counts as the heaviest, both zeros are one weight, and a
// position without a page comes last (0, which no weight maps to).
__device__ __forceinline__ unsigned weight_key(float w) {
    if (w != w) return 0xFFFFFFFFu;
    const unsigned u = __float_as_uint(w == 0.f ? 0.f : w);
    return (u >> 31) ? ~u : u | 0x80000000u;
}

// Exclusive sums over the workgroup's threads; *all = the sum.
__device__ __forceinline__ int scan_threads(int v, int* s_wave, int* all) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int upto = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int up = __shfl_up(upto, o);
        if (lane >= o) upto += up;
    }
    __syncthreads();                                    // (the sums of the call before have been read)
    if (lane == 63) s_wave[w] = upto;
    __syncthreads();
    int front = 0, sum = 0;
#pragma unroll
    for (int i = 0; i < kSelectWaves; ++i) {
        const int t = s_wave[i];
        front += i < w ? t : 0;
        sum += t;
    }
    *all = sum;
    return front + upto - v;
}

// The keys of all n <= kKeysInLds positions stay in LDS.
__global__ void __launch_bounds__(kSelectThreads)
k_evict_select(CacheArgs c, CacheEvictArgs a) {
    extern __shared__ __align__(16) unsigned lds[];
    unsigned* const s_hist = lds;                       // [kBins][kCopies]
    unsigned* const s_keys = lds + kBins * kCopies;
    __shared__ int s_wave[kSelectWaves];
    __shared__ int s_pick[2];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kv = blockIdx.x % c.Hkv, b = blockIdx.x / c.Hkv;
    const int n = length_of(c, b), keep = a.keep;
    int32_t* kept = a.kept + (long long)blockIdx.x * keep;
    if (n <= keep) {
        for (int i = tid; i < keep; i += kSelectThreads) kept[i] = i < n ? i : -1;
        return;
    }
    const int lo = a.sinks, hi = n - a.recent, want = keep - a.sinks - a.recent;    // `want` of the positions lo .. hi - 1
    const int32_t* table = c.table + (long long)b * c.width;
    // keys of four positions from a multiple of four on (they share a page), 0 for those that are not chosen from
    auto keys_at = [&](int pos) -> u32x4 {
        u32x4 k = {0u, 0u, 0u, 0u};
        if (pos >= hi || pos + 3 < lo) return k;
        const int pg = page_of(c, pos), e = table[pg];
        if ((unsigned)e >= (unsigned)c.num_pages) return k;
        const f32x4 v = *reinterpret_cast<const f32x4*>(c.weight + ((long long)e * c.Hkv + kv) * c.page + (pos - pg * c.page));
#pragma unroll
        for (int i = 0; i < 4; ++i) k[i] = weight_key(v[i]);
        return k;
    };
    // f(first position, keys) for the positions p0 + 4 i of a run, kAhead groups of four requested at once by a thread
    constexpr int kAhead = 4;
    auto sweep = [&](int from, int to, int first, int step, auto f) {
        // (all lanes of a wave take every trip, so that f may count over lanes; positions behind the end are in nobody's range)
        for (int p = from + 4 * first, trip = from; trip < to; p += 4 * step * kAhead, trip += 4 * step * kAhead) {
            u32x4 k[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                k[i] = p + 4 * step * i < to ? *reinterpret_cast<const u32x4*>(s_keys + p + 4 * step * i) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (trip + 4 * step * i < to) f(p + 4 * step * i < to ? p + 4 * step * i : n, k[i]);
        }
    };
    const int n4 = (n + 3) & ~3;
    for (int pos = 4 * tid; pos < n4; pos += 4 * kSelectThreads) *reinterpret_cast<u32x4*>(s_keys + pos) = keys_at(pos);
    __syncthreads();
    // the key of the want-th heaviest, found by its top 11 bits, the next 11 and the last 10; and how many with that key are kept
    unsigned prefix = 0u, mask = 0u;
    int left = want;
    if (want > 0) {
        for (int digit = 0; digit < 3; ++digit) {
            const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0;
            const unsigned bins = digit == 2 ? 1024u : 2048u;
            __syncthreads();
            for (int i = tid; i < kBins * kCopies / 4; i += kSelectThreads) reinterpret_cast<u32x4*>(s_hist)[i] = u32x4{0u, 0u, 0u, 0u};
            __syncthreads();
            sweep(0, n4, tid, kSelectThreads, [&](int pos, const u32x4& k) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (pos + i >= lo && pos + i < hi && (k[i] & mask) == prefix)
                        atomicAdd(&s_hist[((k[i] >> shift) & (bins - 1u)) * kCopies + (lane & (kCopies - 1))], 1u);
            });
            __syncthreads();
            // thread t: the bins 2047 - 2 t and 2046 - 2 t, so that threads go from the top down
            int h[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const u32x4 v = *reinterpret_cast<const u32x4*>(s_hist + (kBins - 1 - 2 * tid - i) * kCopies);
                h[i] = (int)(v[0] + v[1] + v[2] + v[3]);
            }
            int all;
            const int above = scan_threads(h[0] + h[1], s_wave, &all);
            if (above < left && left <= above + h[0]) { s_pick[0] = kBins - 1 - 2 * tid; s_pick[1] = left - above; }
            else if (above + h[0] < left && left <= above + h[0] + h[1]) { s_pick[0] = kBins - 2 - 2 * tid; s_pick[1] = left - above - h[0]; }
            __syncthreads();
            prefix |= (unsigned)s_pick[0] << shift;
            mask |= (bins - 1u) << shift;
            left = s_pick[1];
        }
    }
    // out in order: wave w has the positions of its own run, counts what it takes of it and then knows where its output begins
    const int run = ((n4 + 4 * kSelectThreads - 1) / (4 * kSelectThreads)) * 256;      // a multiple of four positions to a lane
    const int from = min(w * run, n4), to = min(from + run, n4);
    auto is_protected = [&](int pos) { return pos < n && (pos < lo || pos >= hi); };
    auto is_above = [&](int pos, unsigned k) { return is_protected(pos) || (want > 0 && pos >= lo && pos < hi && k > prefix); };
    auto is_equal = [&](int pos, unsigned k) { return want > 0 && pos >= lo && pos < hi && k == prefix; };
    int over = 0, same = 0;
    sweep(from, to, lane, 64, [&](int pos, const u32x4& k) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            over += is_above(pos + i, k[i]) ? 1 : 0;
            same += is_equal(pos + i, k[i]) ? 1 : 0;
        }
    });
    int all, same_front = scan_threads(same, s_wave, &all);
    same_front = __shfl(same_front, 0);                 // equal ones in front of the wave's run
    int same_here = same, over_here = over;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) { same_here += __shfl_xor(same_here, o); over_here += __shfl_xor(over_here, o); }
    const int equal_here = max(0, min(same_here, left - same_front));
    int out = scan_threads(lane == 0 ? over_here + equal_here : 0, s_wave, &all);
    out = __shfl(out, 0);
    int equal = same_front;
    // (a lane's four positions follow each other: what lies in front of one is counted over lower lanes and then over the four)
    auto in_front = [&](const bool (&on)[4], int* before) -> int {
        int all_of = 0;
        *before = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned long long set = __ballot(on[i]);
            *before += __builtin_amdgcn_mbcnt_hi((unsigned)(set >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)set, 0u));
            all_of += __popcll(set);
        }
        return all_of;
    };
    sweep(from, to, lane, 64, [&](int pos, const u32x4& k) {
        bool take[4], tie[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            take[i] = is_above(pos + i, k[i]);
            tie[i] = is_equal(pos + i, k[i]);
        }
        int before;
        const int ties = in_front(tie, &before);
        if (ties) {                                     // the same in every lane
            int rank = equal + before;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (tie[i]) take[i] = rank++ < left;
            equal += ties;
        }
        const int takes = in_front(take, &before);
        int at = out + before;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (take[i]) kept[at++] = pos + i;
        out += takes;
    });
}

// ---- longer sequences: the same with a workgroup to a chunk of a (sequence, KV head), the histograms in the workspace ----
// (One workgroup for all of 131072 positions took 157 us at best, these six launches 47.)

constexpr int kChunkThreads = 256, kChunkGroups = 8, kChunk = 4 * kChunkThreads * kChunkGroups;

struct EvictSpace {
    unsigned* hist;                     // [3][pairs][kBins]: digits of the keys that agree with what the digits before have picked
    unsigned* pick;                     // [3][pairs][2]: the key's leading digits, and how many of the keys that have them are kept
    int* count;                         // [pairs][chunks][2]: kept for sure (protected or heavier), equal to the last kept weight
    int pairs, chunks;
};

__global__ void __launch_bounds__(256)
k_evict_clear(u32x4* hist, int n) {
    const int i = (int)blockIdx.x * 256 + (int)threadIdx.x;
    if (i < n) hist[i] = u32x4{0u, 0u, 0u, 0u};
}

// What the digits up to `digits` - 1 have picked: the last of them from its histogram, by every workgroup for itself, the others as the
// stage before has left them.
__device__ __forceinline__ void picked(const EvictSpace& sp, int pair, int want, int digits, bool leave, int* s_wave, int* s_pick,
                                       unsigned* prefix, unsigned* mask, int* left) {
    constexpr int kPer = kBins / kChunkThreads;
    *prefix = 0u;
    *mask = digits == 0 ? 0u : digits == 1 ? 0xFFE00000u : digits == 2 ? 0xFFFFFC00u : 0xFFFFFFFFu;
    *left = want;
    if (digits == 0) return;
    if (digits > 1) {
        *prefix = sp.pick[((long long)(digits - 2) * sp.pairs + pair) * 2];
        *left = (int)sp.pick[((long long)(digits - 2) * sp.pairs + pair) * 2 + 1];
    }
    const unsigned* hist = sp.hist + ((long long)(digits - 1) * sp.pairs + pair) * kBins;
    const int top = kBins - 1 - kPer * (int)threadIdx.x;                // thread t: bins from the top down
    int h[kPer], sum = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) { h[i] = (int)hist[top - i]; sum += h[i]; }
    int upto = sum;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int up = __shfl_up(upto, o);
        if (lane >= o) upto += up;
    }
    if (lane == 63) s_wave[w] = upto;
    __syncthreads();
    int above = upto - sum;
#pragma unroll
    for (int i = 0; i < kChunkThreads / 64; ++i) above += i < w ? s_wave[i] : 0;
    if (above < *left && *left <= above + sum) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (above < *left && *left <= above + h[i]) { s_pick[0] = top - i; s_pick[1] = *left - above; }
            above += h[i];
        }
    }
    __syncthreads();
    *prefix |= (unsigned)s_pick[0] << (digits == 1 ? 21 : digits == 2 ? 10 : 0);
    *left = s_pick[1];
    if (leave && threadIdx.x == 0) {
        sp.pick[((long long)(digits - 1) * sp.pairs + pair) * 2] = *prefix;
        sp.pick[((long long)(digits - 1) * sp.pairs + pair) * 2 + 1] = (unsigned)*left;
    }
}

// kStage 0, 1, 2: the histogram of that digit; 3: the chunk's counts; 4: the kept positions.
template <int kStage>
__global__ void __launch_bounds__(kChunkThreads)
k_evict_chunks(CacheArgs c, CacheEvictArgs a, EvictSpace sp) {
    __shared__ unsigned s_hist[kStage < 3 ? kBins * kCopies : 1];
    __shared__ int s_wave[kChunkThreads / 64][2], s_scan[kChunkThreads / 64], s_pick[2], s_front[2];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int pair = blockIdx.y, kv = pair % c.Hkv, b = pair / c.Hkv;
    const int n = length_of(c, b), keep = a.keep, p0 = (int)blockIdx.x * kChunk;
    int32_t* kept = a.kept + (long long)pair * keep;
    if (n <= keep) {
        if (kStage == 4)
            for (long long i = (long long)blockIdx.x * kChunkThreads + tid; i < keep; i += (long long)gridDim.x * kChunkThreads)
                kept[i] = i < n ? (int)i : -1;
        return;
    }
    if (p0 >= n) return;
    const int lo = a.sinks, hi = n - a.recent, want = keep - a.sinks - a.recent;
    if (kStage < 3 && want == 0) return;
    unsigned prefix = 0u, mask = 0u;
    int left = 0;
    if (want > 0) {
        if (kStage < 4) {
            picked(sp, pair, want, kStage, blockIdx.x == 0, s_scan, s_pick, &prefix, &mask, &left);
        } else {
            prefix = sp.pick[(2ll * sp.pairs + pair) * 2];
            left = (int)sp.pick[(2ll * sp.pairs + pair) * 2 + 1];
        }
    }
    if (kStage < 3) {
        for (int i = tid; i < kBins * kCopies; i += kChunkThreads) s_hist[i] = 0u;
        __syncthreads();
    }
    // a thread's groups of four positions, each in one page: every page entry, then every weight (past the end: the last group's)
    const int32_t* table = c.table + (long long)b * c.width;
    int e[kChunkGroups];
    f32x4 v[kChunkGroups];
#pragma unroll
    for (int i = 0; i < kChunkGroups; ++i) e[i] = table[page_of(c, min(p0 + 4 * (tid + kChunkThreads * i), n - 1))];
#pragma unroll
    for (int i = 0; i < kChunkGroups; ++i) {
        const int pos = min(p0 + 4 * (tid + kChunkThreads * i), (n - 1) & ~3);
        const long long at = (unsigned)e[i] < (unsigned)c.num_pages ? e[i] : 0;
        v[i] = *reinterpret_cast<const f32x4*>(c.weight + (at * c.Hkv + kv) * c.page + (pos - page_of(c, pos) * c.page));
    }
    auto key = [&](int i, int r) { return (unsigned)e[i] < (unsigned)c.num_pages ? weight_key(v[i][r]) : 0u; };
    auto chosen_from = [&](int pos) { return pos >= lo && pos < hi; };
    if constexpr (kStage < 3) {
        constexpr int shift = kStage == 0 ? 21 : kStage == 1 ? 10 : 0;
        constexpr unsigned bins = kStage == 2 ? 1024u : 2048u;
#pragma unroll
        for (int i = 0; i < kChunkGroups; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const unsigned k = key(i, r);
                if (chosen_from(p0 + 4 * (tid + kChunkThreads * i) + r) && (k & mask) == prefix)
                    atomicAdd(&s_hist[((k >> shift) & (bins - 1u)) * kCopies + (lane & (kCopies - 1))], 1u);
            }
        __syncthreads();
        unsigned* hist = sp.hist + ((long long)kStage * sp.pairs + pair) * kBins;
        for (int i = tid; i < kBins; i += kChunkThreads) {
            unsigned sum = 0u;
#pragma unroll
            for (int q = 0; q < kCopies; ++q) sum += s_hist[i * kCopies + q];
            if (sum) atomicAdd(hist + i, sum);                          // whole numbers: any order gives the same
        }
    } else {
        // bit r + 4 i of a thread: position r of its group i is kept for sure, or has the last kept weight
        unsigned take = 0u, tie = 0u;
#pragma unroll
        for (int i = 0; i < kChunkGroups; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int pos = p0 + 4 * (tid + kChunkThreads * i) + r;
                const bool from = chosen_from(pos) && want > 0;
                if ((pos < n && (pos < lo || pos >= hi)) || (from && key(i, r) > prefix)) take |= 1u << (4 * i + r);
                else if (from && key(i, r) == prefix) tie |= 1u << (4 * i + r);
            }
        if constexpr (kStage == 3) {
            int over = __popc(take), same = __popc(tie);
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) { over += __shfl_xor(over, o); same += __shfl_xor(same, o); }
            if (lane == 0) { s_wave[w][0] = over; s_wave[w][1] = same; }
            __syncthreads();
            if (tid < 2) {
                int sum = 0;
#pragma unroll
                for (int i = 0; i < kChunkThreads / 64; ++i) sum += s_wave[i][tid];
                sp.count[((long long)pair * sp.chunks + blockIdx.x) * 2 + tid] = sum;
            }
        } else {
            // what the chunks in front keep: for sure, and of equal ones the first `left`
            if (w == 0) {
                int over = 0, same = 0;
                for (int i = lane; i < (int)blockIdx.x; i += 64) {
                    over += sp.count[((long long)pair * sp.chunks + i) * 2];
                    same += sp.count[((long long)pair * sp.chunks + i) * 2 + 1];
                }
#pragma unroll
                for (int o = 32; o > 0; o >>= 1) { over += __shfl_xor(over, o); same += __shfl_xor(same, o); }
                if (lane == 0) { s_front[0] = over + min(same, left); s_front[1] = same; }
            }
            __syncthreads();
            int out = s_front[0], equal = s_front[1];
            // group by group, every one a run of positions over the threads
            for (int i = 0; i < kChunkGroups; ++i) {
                const unsigned t4 = (tie >> (4 * i)) & 15u;
                unsigned k4 = (take >> (4 * i)) & 15u;
                auto in_front = [&](unsigned bits, int which, int* all) -> int {
                    int before = 0, mine = 0;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const unsigned long long set = __ballot((bits >> r) & 1u);
                        before += __builtin_amdgcn_mbcnt_hi((unsigned)(set >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)set, 0u));
                        mine += __popcll(set);
                    }
                    __syncthreads();
                    if (lane == 0) s_wave[w][which] = mine;
                    __syncthreads();
                    *all = 0;
#pragma unroll
                    for (int x = 0; x < kChunkThreads / 64; ++x) {
                        const int s = s_wave[x][which];
                        before += x < w ? s : 0;
                        *all += s;
                    }
                    return before;
                };
                int all;
                int rank = equal + in_front(t4, 1, &all);
                equal += all;
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if ((t4 >> r) & 1u) k4 |= rank++ < left ? 1u << r : 0u;
                int at = out + in_front(k4, 0, &all);
                out += all;
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if ((k4 >> r) & 1u) kept[at++] = p0 + 4 * (tid + kChunkThreads * i) + r;
            }
        }
    }
}

__global__ void __launch_bounds__(256)
k_evict_move(CacheArgs c, CacheEvictArgs a, u32x4* K, u32x4* V, int chunks, int log_piece) {
    const int kv = blockIdx.y % c.Hkv, b = blockIdx.y / c.Hkv;
    const int n = min(length_of(c, b), a.keep);
    if (blockIdx.x == 0 && kv == 0 && threadIdx.x == 0) a.to_length[b] = n;
    const int32_t* kept = a.kept + (long long)blockIdx.y * a.keep;
    const long long pieces = (long long)n * chunks;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < pieces; i += (long long)gridDim.x * 256) {
        const int r = (int)(i / chunks), ch = (int)(i - (long long)r * chunks);
        const int pos = kept[r];
        const int p0 = page_of(c, pos), p1 = page_of(c, r);
        const int e = c.table[(long long)b * c.width + p0], to = a.to[(long long)b * a.to_width + p1];
        if ((unsigned)e >= (unsigned)c.num_pages || (unsigned)to >= (unsigned)c.num_pages) continue;
        const int s0 = pos - p0 * c.page, s1 = r - p1 * c.page;
        const long long src = ((e * c.psb + kv * c.ksh + s0 * c.ksl) >> log_piece) + ch, dst = ((to * c.psb + kv * c.ksh + s1 * c.ksl) >> log_piece) + ch;
        const u32x4 k = K[src], v = V[src];
        K[dst] = k;
        V[dst] = v;
        if (ch == 0) c.weight[((long long)to * c.Hkv + kv) * c.page + s1] = c.weight[((long long)e * c.Hkv + kv) * c.page + s0];
    }
}

}  // namespace

size_t cache_evict_bytes(const CacheArgs& c) {
    if (c.L <= kKeysInLds) return 0;
    const size_t pairs = (size_t)c.batch * c.Hkv, chunks = ((size_t)c.L + kChunk - 1) / kChunk;
    return (3 * pairs * (kBins + 2) * sizeof(unsigned) + pairs * chunks * 2 * sizeof(int) + 255) / 256 * 256;
}

// expects batch * Hkv <= 65535, sinks + recent <= keep, keep positions within the new table, and cache_evict_bytes() of workspace
hipError_t launch_cache_evict(const CacheArgs& c, int dtype, const CacheEvictArgs& a, void* K, void* V, void* workspace, hipStream_t st) {
    const int pairs = c.batch * c.Hkv;
    hipError_t e;
    if (c.L <= kKeysInLds) {
        const size_t lds = sizeof(unsigned) * (kBins * kCopies + (size_t)(c.L + 3) / 4 * 4);
        e = allow_dynamic_lds(reinterpret_cast<const void*>(k_evict_select), lds);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(k_evict_select, dim3((unsigned)pairs), dim3(kSelectThreads), lds, st, c, a);
        e = hipGetLastError();
    } else {
        EvictSpace sp;
        sp.pairs = pairs;
        sp.chunks = (int)(((long long)c.L + kChunk - 1) / kChunk);
        sp.hist = reinterpret_cast<unsigned*>(workspace);
        sp.pick = sp.hist + 3ll * pairs * kBins;
        sp.count = reinterpret_cast<int*>(sp.pick + 6ll * pairs);
        const int pieces = 3 * pairs * kBins / 4;                       // (pairs <= 65535: below 2^27)
        hipLaunchKernelGGL(k_evict_clear, dim3((unsigned)((pieces + 255) / 256)), dim3(256), 0, st, reinterpret_cast<u32x4*>(sp.hist), pieces);
        e = hipGetLastError();
        auto stage = [&](auto kernel) {
            if (e != hipSuccess) return;
            hipLaunchKernelGGL(kernel, dim3((unsigned)sp.chunks, (unsigned)pairs), dim3(kChunkThreads), 0, st, c, a, sp);
            e = hipGetLastError();
        };
        stage(k_evict_chunks<0>);
        stage(k_evict_chunks<1>);
        stage(k_evict_chunks<2>);
        stage(k_evict_chunks<3>);
        stage(k_evict_chunks<4>);
    }
    if (e != hipSuccess) return e;
    const int log_piece = dtype == RR_BF16 ? 3 : 2, chunks = c.d >> log_piece;   // 16 bytes are 2^log_piece elements
    const long long n = (long long)std::min(c.L, a.keep) * chunks;
    const unsigned blocks = (unsigned)std::min<long long>((n + 255) / 256, 4096);
    hipLaunchKernelGGL(k_evict_move, dim3(blocks, (unsigned)(c.batch * c.Hkv)), dim3(256), 0, st, c, a, reinterpret_cast<u32x4*>(K),
                       reinterpret_cast<u32x4*>(V), chunks, log_piece);
    return hipGetLastError();
}

}  // namespace rr
