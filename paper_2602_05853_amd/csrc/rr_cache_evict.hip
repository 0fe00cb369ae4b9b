// Eviction by accumulated weight: of the n positions of a (sequence, KV head) the first `sinks`, the last `recent` and the
// heaviest of the others are kept, `keep` in all (all where n <= keep), in their order, in the pages of another table.
//
// First launch, one workgroup to a (sequence, KV head): the weight of the last position that is kept by weight, found by
// its bits, eleven at a time from the top (weights mapped to unsigned numbers of the same order); heavier ones are kept, of equal
// ones as many as are left, the lower positions first; every wave then writes out the positions of its own run in order.
// Second launch: the rows, 16 bytes of K and of V to a thread.  What bounds it: the copy.
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

// kInLds: the keys of all n <= kKeysInLds positions stay in LDS; otherwise every sweep reads the weights again.
template <bool kInLds>
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
        const int e = table[pos / c.page];
        if ((unsigned)e >= (unsigned)c.num_pages) return k;
        const f32x4 v = *reinterpret_cast<const f32x4*>(c.weight + ((long long)e * c.Hkv + kv) * c.page + pos % c.page);
#pragma unroll
        for (int i = 0; i < 4; ++i) k[i] = weight_key(v[i]);
        return k;
    };
    // f(first position, keys) for the positions p0 + 4 i of a run, kAhead groups of four requested at once by a thread
    constexpr int kAhead = 4;
    auto sweep = [&](int from, int to, int first, int step, auto f) {
        for (int p = from + 4 * first; p < to; p += 4 * step * kAhead) {
            u32x4 k[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int pos = p + 4 * step * i;
                if (kInLds) k[i] = pos < to ? *reinterpret_cast<const u32x4*>(s_keys + pos) : u32x4{0u, 0u, 0u, 0u};
                else k[i] = keys_at(pos < to ? pos : n);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (p + 4 * step * i < to) f(p + 4 * step * i, k[i]);
        }
    };
    const int n4 = (n + 3) & ~3;
    if (kInLds) {
        for (int pos = 4 * tid; pos < n4; pos += 4 * kSelectThreads) *reinterpret_cast<u32x4*>(s_keys + pos) = keys_at(pos);
        __syncthreads();
    }
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
    // (a thread's four positions follow each other, so ranks are sums over lanes and then over the four)
    for (int p = from; p < to; p += 256) {
        const int pos = p + 4 * lane;
        u32x4 k = {0u, 0u, 0u, 0u};
        if (pos < to) k = kInLds ? *reinterpret_cast<const u32x4*>(s_keys + pos) : keys_at(pos);
        int ties = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) ties += pos < to && is_equal(pos + i, k[i]) ? 1 : 0;
        int upto = ties;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int up = __shfl_up(upto, o);
            if (lane >= o) upto += up;
        }
        int rank = equal + upto - ties;
        bool take[4];
        int takes = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            take[i] = pos < to && is_above(pos + i, k[i]);
            if (pos < to && is_equal(pos + i, k[i])) take[i] = rank++ < left;
            takes += take[i] ? 1 : 0;
        }
        equal += __shfl(upto, 63);
        upto = takes;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int up = __shfl_up(upto, o);
            if (lane >= o) upto += up;
        }
        int at = out + upto - takes;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (take[i]) kept[at++] = pos + i;
        out += __shfl(upto, 63);
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
        const int e = c.table[(long long)b * c.width + pos / c.page], to = a.to[(long long)b * a.to_width + r / c.page];
        if ((unsigned)e >= (unsigned)c.num_pages || (unsigned)to >= (unsigned)c.num_pages) continue;
        const int s0 = pos % c.page, s1 = r % c.page;
        const long long src = ((e * c.psb + kv * c.ksh + s0 * c.ksl) >> log_piece) + ch, dst = ((to * c.psb + kv * c.ksh + s1 * c.ksl) >> log_piece) + ch;
        const u32x4 k = K[src], v = V[src];
        K[dst] = k;
        V[dst] = v;
        if (ch == 0) c.weight[((long long)to * c.Hkv + kv) * c.page + s1] = c.weight[((long long)e * c.Hkv + kv) * c.page + s0];
    }
}

}  // namespace

// expects batch * Hkv <= 65535, sinks + recent <= keep, and keep positions within the new table
hipError_t launch_cache_evict(const CacheArgs& c, int dtype, const CacheEvictArgs& a, void* K, void* V, hipStream_t st) {
    const bool in_lds = c.L <= kKeysInLds;
    const void* kernel = in_lds ? reinterpret_cast<const void*>(k_evict_select<true>) : reinterpret_cast<const void*>(k_evict_select<false>);
    const size_t lds = sizeof(unsigned) * (kBins * kCopies + (in_lds ? (size_t)(c.L + 3) / 4 * 4 : 0));
    hipError_t e = allow_dynamic_lds(kernel, lds);
    if (e != hipSuccess) return e;
    if (in_lds) hipLaunchKernelGGL(k_evict_select<true>, dim3((unsigned)(c.batch * c.Hkv)), dim3(kSelectThreads), lds, st, c, a);
    else hipLaunchKernelGGL(k_evict_select<false>, dim3((unsigned)(c.batch * c.Hkv)), dim3(kSelectThreads), lds, st, c, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int log_piece = dtype == RR_BF16 ? 3 : 2, chunks = c.d >> log_piece;   // 16 bytes are 2^log_piece elements
    const long long n = (long long)std::min(c.L, a.keep) * chunks;
    const unsigned blocks = (unsigned)std::min<long long>((n + 255) / 256, 4096);
    hipLaunchKernelGGL(k_evict_move, dim3(blocks, (unsigned)(c.batch * c.Hkv)), dim3(256), 0, st, c, a, reinterpret_cast<u32x4*>(K),
                       reinterpret_cast<u32x4*>(V), chunks, log_piece);
    return hipGetLastError();
}

}  // namespace rr
