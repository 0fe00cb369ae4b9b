// New positions into their pages: token t of the count[b] new ones of sequence b goes to position length[b] - count[b] + t.
//
// What bounds it: the copy (each value read once and written once), and for a step's one token the launch.  A thread moves
// 16 bytes of K and of V; neighbours move neighbouring bytes of a row, rows follow each other within a head as in the pages.
// Measured: a prompt of 16384 positions, 8 heads of 128, with weights 17.6 us (5 TB/s); one position of 64 sequences 3.3 us.
#include "rr_cache.hpp"

#include <algorithm>

namespace rr {

namespace {

__global__ void __launch_bounds__(256)
k_cache_write(CacheArgs c, CacheWriteArgs a, u32x4* K, u32x4* V, int chunks, int log_piece) {
    // strides in 16-byte pieces; they and a row are whole pieces
    const long long n = (long long)c.T * chunks;                       // pieces of a (sequence, KV head)
    const int kv = blockIdx.y % c.Hkv, b = blockIdx.y / c.Hkv;
    int len = c.length[b], count = a.count ? a.count[b] : c.T;
    len = len < 0 ? 0 : (len > c.L ? c.L : len);
    count = count < 0 ? 0 : (count > c.T ? c.T : count);
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
        const int t = (int)(i / chunks), ch = (int)(i - (long long)t * chunks);
        if (t >= count) return;                                        // (t only grows)
        const int pos = len - count + t;
        if (pos < 0) continue;
        const int pg = page_of(c, pos), e = c.table[(long long)b * c.width + pg], slot = pos - pg * c.page;
        if ((unsigned)e >= (unsigned)c.num_pages) continue;
        const long long from = ((b * c.qsb + kv * c.qsh + t * c.qsl) >> log_piece) + ch;
        const long long to = ((e * c.psb + kv * c.ksh + slot * c.ksl) >> log_piece) + ch;
        const u32x4 k = reinterpret_cast<const u32x4*>(a.K)[from], v = reinterpret_cast<const u32x4*>(a.V)[from];
        K[to] = k;
        V[to] = v;
        if (c.weight && ch == 0)
            c.weight[((long long)e * c.Hkv + kv) * c.page + slot] = a.weight ? a.weight[((long long)b * c.Hkv + kv) * c.T + t] : 0.f;
    }
}

}  // namespace

// expects batch * Hkv <= 65535
hipError_t launch_cache_write(const CacheArgs& c, int dtype, const CacheWriteArgs& a, void* K, void* V, hipStream_t st) {
    const int log_piece = dtype == RR_BF16 ? 3 : 2, chunks = c.d >> log_piece;   // 16 bytes are 2^log_piece elements
    const long long n = (long long)c.T * chunks;
    const unsigned blocks = (unsigned)std::min<long long>((n + 255) / 256, 4096);
    hipLaunchKernelGGL(k_cache_write, dim3(blocks, (unsigned)(c.batch * c.Hkv)), dim3(256), 0, st, c, a, reinterpret_cast<u32x4*>(K),
                       reinterpret_cast<u32x4*>(V), chunks, log_piece);
    return hipGetLastError();
}

}  // namespace rr
