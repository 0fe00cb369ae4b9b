// What the kernels over a key-value cache share: which 128-key blocks a sequence's queries visit, how a launch's workgroups
// share the blocks of all sequences, and where a position lies.
#pragma once
#include "rr_common.hpp"

namespace rr {

namespace {

constexpr int kUnit = 128;                      // keys of a block

#if defined(__HIP_DEVICE_COMPILE__)
typedef const __attribute__((address_space(4))) int32_t* scalar_words_t;   // read with scalar loads
#else
typedef const int32_t* scalar_words_t;                                     // the host pass only parses the kernels
#endif

// position / page.  Pages are multiples of 16, so n = position / 16 < 2^27 is divided by p = page / 16: with l the bits of p - 1,
// s = 27 + l and M = ceil(2^s / p) <= 2^28, M p - 2^s < p <= 2^l, so n (M p - 2^s) < 2^s and n M / 2^s has the quotient as its
// whole part.  (A 32-bit division is some forty vector instructions.)
inline void set_page(CacheArgs* c, int page) {
    c->page = page;
    const unsigned p = (unsigned)page >> 4;
    int l = 0;
    while ((1u << l) < p) ++l;
    c->page_shift = 27 + l;
    c->page_mul = (unsigned)(((1ull << c->page_shift) + p - 1) / p);
}
__host__ __device__ inline int page_of(const CacheArgs& c, int pos) {
    return (int)(((unsigned long long)((unsigned)pos >> 4) * c.page_mul) >> c.page_shift);
}

// The blocks that a step at the end of `len` positions visits: 0 .. ns - 1, which hold sinks, then those from first_w to the end.
struct Visit {
    int len, ns, first_w, n;
    __host__ __device__ int block(int i) const { return i < ns ? i : first_w + i - ns; }
};
__host__ __device__ inline Visit visit_of(int len, int T, int window, int sinks) {
    Visit v;
    v.len = len;
    const long long lo = (long long)len - T - window + 1;           // first key of the earliest query's window
    v.first_w = lo > 0 ? (int)(lo / kUnit) : 0;
    const int ns = (int)(((long long)(sinks < len ? sinks : len) + kUnit - 1) / kUnit);
    v.ns = ns < v.first_w ? ns : v.first_w;
    v.n = len > 0 ? v.ns + (len - 1) / kUnit - v.first_w + 1 : 0;
    return v;
}
// The most blocks that any length up to L visits.  (Not those of L itself: a window of 128 that ends with a block is one block,
// one that ends inside a block is two.)
inline long long most_blocks(int L, int T, int window, int sinks) {
    const long long all = ((long long)L + kUnit - 1) / kUnit, near = (long long)window + T - 1;
    const long long some = ((long long)sinks + kUnit - 1) / kUnit + (near + 2 * kUnit - 2) / kUnit;
    return all < some ? all : some;
}

__device__ __forceinline__ int length_of(const CacheArgs& c, int b) {
    if (!c.length) return c.L;
    const int n = ((scalar_words_t)c.length)[b];
    return n < 0 ? 0 : (n > c.L ? c.L : n);
}
__device__ __forceinline__ Visit visit(const CacheArgs& c, int b) { return visit_of(length_of(c, b), c.T, c.window, c.sinks); }

// The units of a launch, in order: sequence by sequence, `pairs` (KV head and row tile) by pair, block by block.  The W
// workgroups take U / W or one more of them each, one after the other, whatever sequences they belong to, so all end together
// however uneven the lengths are; the part of a pair that a workgroup computes has slot w + (number of the pair), which is its own: from one
// part to the next at least one of the two grows.
// Every workgroup adds the lengths up for itself: up to 64 sequences a lane each, in every wave (no LDS, no barrier); more, thread t
// the sequences t per .. t per + per - 1, then a scan over threads.
template <int kThreads> struct Shares {
    int pre[kThreads + 1];                      // blocks of the sequences in front of thread t's
    int wave[kThreads / 64];
    int at;
};
__device__ __forceinline__ int blocks_of(const CacheArgs& c, int b) {
    int n = c.L;
    if (c.length) {
        n = c.length[b];
        n = n < 0 ? 0 : (n > c.L ? c.L : n);
    }
    return visit_of(n, c.T, c.window, c.sinks).n;
}
__device__ __forceinline__ int scan_lanes(int v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int up = __shfl_up(v, o);
        if (lane >= o) v += up;
    }
    return v;
}
// Blocks of all sequences; `upto`: of those up to the lane's (up to 64 sequences).
template <int kThreads>
__device__ __forceinline__ int shares_scan(const CacheArgs& c, Shares<kThreads>& s, int& upto) {
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    if (c.batch <= 64) {
        upto = scan_lanes(lane < c.batch ? blocks_of(c, lane) : 0);
        return __builtin_amdgcn_readlane(upto, 63);
    }
    const int per = (c.batch + kThreads - 1) / kThreads;
    int own = 0;
    for (int i = 0; i < per; ++i)
        if (tid * per + i < c.batch) own += blocks_of(c, tid * per + i);
    upto = scan_lanes(own);
    if (lane == 63) s.wave[w] = upto;
    __syncthreads();
    int front = 0;
#pragma unroll
    for (int i = 0; i < kThreads / 64; ++i) front += i < w ? s.wave[i] : 0;
    s.pre[tid] = front + upto - own;
    if (tid == kThreads - 1) s.pre[kThreads] = front + upto;
    __syncthreads();
    return s.pre[kThreads];
}
// The sequence that block `at` (0 <= at < the scan's total) of all sequences belongs to, its first block and its visit.
template <int kThreads>
__device__ __forceinline__ int shares_find(const CacheArgs& c, Shares<kThreads>& s, int upto, int at, int* base, Visit* v) {
    if (c.batch <= 64) {
        const int b = __popcll(__ballot(upto <= at));
        *base = b ? __builtin_amdgcn_readlane(upto, b - 1) : 0;
        *v = visit(c, b);
        return b;
    }
    const int tid = threadIdx.x;
    if (s.pre[tid] <= at && at < s.pre[tid + 1]) s.at = tid;
    __syncthreads();
    const int per = (c.batch + kThreads - 1) / kThreads;
    const int chunk = __builtin_amdgcn_readfirstlane(s.at);
    int b = chunk * per, front = __builtin_amdgcn_readfirstlane(s.pre[chunk]);
    *v = visit(c, b);
    while (at >= front + v->n) {
        front += v->n;
        *v = visit(c, ++b);
    }
    *base = front;
    __syncthreads();                            // s.at may be written again
    return b;
}
// How U units are dealt out to at most `workgroups`: to no more than take them in the same number of units each (fewer parts to
// join).  All of it in 32 bits: a division of 64 takes over a hundred instructions.
struct Deal {
    unsigned W, each, more;                     // the first `more` workgroups have one unit more than `each`
    __host__ __device__ Deal(unsigned U, unsigned workgroups) {
        const unsigned most = (U + workgroups - 1) / workgroups;
        W = most ? (U + most - 1) / most : 0;
        each = W ? U / W : 0;
        more = U - each * W;
    }
    __device__ __forceinline__ unsigned start(unsigned w) const { return each * w + (w < more ? w : more); }
    // the workgroup that has unit u
    __device__ __forceinline__ unsigned owner(unsigned u) const {
        const unsigned big = more * (each + 1);
        return u < big ? u / (each + 1) : more + (u - big) / each;
    }
};

}  // namespace

}  // namespace rr
