// Eviction by accumulated weight: of the n positions of a (sequence, KV head) the first `sinks`, the last `recent` and the
// heaviest of the others are kept, `keep` in all (all where n <= keep), in their order, in the pages of another table.
//
// First launch, one workgroup to a (sequence, KV head): the weight of the last position that is kept by weight, found by
// its bits, eight at a time from the top (weights mapped to unsigned numbers of the same order); heavier ones are kept, of equal
// ones as many as are left, the lower positions first; positions are written out in order by a scan.
// Second launch: the rows, 16 bytes of K and of V to a thread.  What bounds it: the copy.
#include "rr_cache.hpp"

#include <algorithm>

namespace rr {

namespace {

constexpr int kSelectThreads = 1024;

// Unsigned numbers in the order of the weights; a number that is none counts as the heaviest, both zeros are one weight, and a
// position without a page comes last (0, which no weight maps to).
__device__ __forceinline__ unsigned weight_key(float w) {
    if (w != w) return 0xFFFFFFFFu;
    const unsigned u = __float_as_uint(w == 0.f ? 0.f : w);
    return (u >> 31) ? ~u : u | 0x80000000u;
}

__global__ void __launch_bounds__(kSelectThreads)
k_evict_select(CacheArgs c, CacheEvictArgs a) {
    __shared__ int s_hist[256];
    __shared__ int s_wave[kSelectThreads / 64][2];
    __shared__ int s_pick[2];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int kv = blockIdx.x % c.Hkv, b = blockIdx.x / c.Hkv;
    const int n = length_of(c, b), keep = a.keep;
    int32_t* kept = a.kept + (long long)blockIdx.x * keep;
    if (n <= keep) {
        for (int i = tid; i < keep; i += kSelectThreads) kept[i] = i < n ? i : -1;
        return;
    }
    const int lo = a.sinks, hi = n - a.recent, want = keep - a.sinks - a.recent;    // `want` of the positions lo .. hi - 1
    auto key_of = [&](int pos) -> unsigned {
        const int e = c.table[(long long)b * c.width + pos / c.page];
        if ((unsigned)e >= (unsigned)c.num_pages) return 0u;
        return weight_key(c.weight[((long long)e * c.Hkv + kv) * c.page + pos % c.page]);
    };
    // the top bits of the want-th heaviest so far, and how many of those that have them are wanted
    unsigned prefix = 0u, mask = 0u;
    int left = want;
    if (want > 0) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (tid < 256) s_hist[tid] = 0;
            __syncthreads();
            for (int pos = lo + tid; pos < hi; pos += kSelectThreads) {
                const unsigned k = key_of(pos);
                if ((k & mask) == prefix) atomicAdd(&s_hist[(k >> shift) & 255u], 1);
            }
            __syncthreads();
            if (w == 0) {                                               // lane l: the values 255 - 4 l .. 252 - 4 l, from the top
                int h[4], sum = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) { h[i] = s_hist[255 - 4 * lane - i]; sum += h[i]; }
                int upto = sum;
#pragma unroll
                for (int o = 1; o < 64; o <<= 1) {
                    const int up = __shfl_up(upto, o);
                    if (lane >= o) upto += up;
                }
                int above = upto - sum;
                if (above < left && left <= upto) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (above < left && left <= above + h[i]) { s_pick[0] = 255 - 4 * lane - i; s_pick[1] = left - above; }
                        above += h[i];
                    }
                }
            }
            __syncthreads();
            prefix |= (unsigned)s_pick[0] << shift;
            mask |= 255u << shift;
            left = s_pick[1];
        }
    }
    // out in order: every trip takes as many positions as there are threads
    int out = 0, equal = 0;                                             // kept, and equal ones met, so far
    for (int p0 = 0; p0 < n; p0 += kSelectThreads) {
        const int pos = p0 + tid;
        bool take = false, tie = false;
        if (pos < n) {
            if (pos < lo || pos >= hi) take = true;
            else if (want > 0) {
                const unsigned k = key_of(pos);
                take = k > prefix;
                tie = k == prefix;
            }
        }
        const unsigned long long below = (1ull << lane) - 1ull;
        const unsigned long long ties = __ballot(tie);
        if (lane == 0) s_wave[w][0] = __popcll(ties);
        __syncthreads();
        int tie_front = equal, tie_all = 0;
        for (int i = 0; i < kSelectThreads / 64; ++i) {
            const int t = s_wave[i][0];
            tie_front += i < w ? t : 0;
            tie_all += t;
        }
        take = take || (tie && tie_front + __popcll(ties & below) < left);
        const unsigned long long taken = __ballot(take);
        if (lane == 0) s_wave[w][1] = __popcll(taken);
        __syncthreads();
        int front = out, all = 0;
        for (int i = 0; i < kSelectThreads / 64; ++i) {
            const int t = s_wave[i][1];
            front += i < w ? t : 0;
            all += t;
        }
        if (take) kept[front + __popcll(taken & below)] = pos;
        out += all;
        equal += tie_all;
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
    hipLaunchKernelGGL(k_evict_select, dim3((unsigned)(c.batch * c.Hkv)), dim3(kSelectThreads), 0, st, c, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int log_piece = dtype == RR_BF16 ? 3 : 2, chunks = c.d >> log_piece;   // 16 bytes are 2^log_piece elements
    const long long n = (long long)std::min(c.L, a.keep) * chunks;
    const unsigned blocks = (unsigned)std::min<long long>((n + 255) / 256, 4096);
    hipLaunchKernelGGL(k_evict_move, dim3(blocks, (unsigned)(c.batch * c.Hkv)), dim3(256), 0, st, c, a, reinterpret_cast<u32x4*>(K),
                       reinterpret_cast<u32x4*>(V), chunks, log_piece);
    return hipGetLastError();
}

}  // namespace rr
