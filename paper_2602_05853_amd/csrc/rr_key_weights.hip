// Softmax weights that every key gets from the queries of a call: w_j = sum over the heads h of a KV group and the query rows i of
// exp(q_i k_j / sqrt(d) - lse_i) where j <= i's position; lse is what the attention of the same call has written.
//
// One product per (query, key) pair and no second one: half the operations of attention, and an exponential each.  A wave's keys
// stay in registers (rows of the matrix tiles), the queries (columns) pass by: they come to LDS 32 rows at a time, once for the
// workgroup's waves, in two stages; every lane adds up its own columns, which meet once, at the end of a tile of keys.
//
// Work split.  The stages of all tiles of keys, in order (a tile begins with the first stage that sees one of its keys, so the
// later the keys the fewer there are), are dealt out evenly to one round of workgroups; a workgroup whose share ends inside
// a tile leaves its sums in a slot, and a second kernel adds a tile's slots up in order.
// Measured (8192 tokens, 28 / 4 heads of 128, us): 271 to 280, 0.86 to 0.89 PFLOP/s (an exponential to every 256 operations: of 0.65 M
// cycles the vector units are busy 0.39 M, the matrix pipe 0.24 M); every wave reading the queries for itself 812 (they then come from L2 four times), a grid of tiles of keys and
// chunks of queries 309 to 454, by the order in which XCDs meet the early and the late keys.  Last 64 queries of 64K, 32 / 8 heads: 60.
#include "rr_attn_frag.hpp"

#include <algorithm>
#include <type_traits>

namespace rr {

namespace {

constexpr int kWaves = 4;
constexpr int kRows = 32;                                       // query rows to a stage
// Tiles of at most so many stages are not split, where they give the chip a workgroup to each compute unit, or are short.  (Split, the
// shares of at least two stages; us: 100 positions, 32 / 8 heads 21.7 whole, 14.6 split; fp32, 100 rows of 1000, 8 / 2 heads 44.4, 14.5;
// 32 rows of 2000, 32 / 8 heads 10.6, 15.0; 64 rows of 64K 60, 68.)
constexpr int kWholeStages = 16, kShortStages = 4, kManyTiles = 256;

// Pairs of 16-key tiles that a wave holds: 64 keys where they take 64 registers or fewer.
template <typename T, int NT> constexpr int pairs_of() {
    return std::is_same<T, bf16_t>::value ? (NT <= 8 ? 2 : 1) : (NT <= 4 ? 2 : 1);
}
int keys_of(int dtype, int d) {
    const int n = (d + 15) / 16;
    return 32 * kWaves * (dtype == RR_BF16 ? (n <= 8 ? 2 : 1) : (n <= 4 ? 2 : 1));
}

// The stages of a call.  Tile i of a (batch entry, KV head) holds the keys i keys .. of `tiles` such tiles; its stages are, head after
// head, those from skip(i) to per_head - 1, 32 rows each.
struct Stages {
    int G, tiles, per_head, per_tile, c0;                       // per_tile: stages that a tile's keys span; c0 = ceil(q0 / 32)
    long long per_pair;                                         // stages of all tiles of a (batch entry, KV head)
    int whole;                                                  // 1: a workgroup has one whole tile
    __host__ __device__ int skip(int i) const {
        const long long s = (long long)i * per_tile - c0;
        return s > 0 ? (int)s : 0;
    }
    __host__ __device__ long long of_tile(int i) const { return (long long)G * (per_head - skip(i)); }
    // stages of the tiles in front of tile i
    __host__ __device__ long long before(int i) const {
        const long long k = c0 / per_tile + 1;                  // the first tile that skips some
        long long skipped = 0;
        if (i > k) skipped = per_tile * ((k + i - 1) * (i - k) / 2) - c0 * (i - k);
        return G * ((long long)i * per_head - skipped);
    }
    // the tile that has stage u < per_pair
    __host__ __device__ int find(long long u) const {
        int lo = 0, hi = tiles - 1;
        while (lo < hi) {
            const int mid = lo + (hi - lo + 1) / 2;
            if (before(mid) <= u) lo = mid; else hi = mid - 1;
        }
        return lo;
    }
};

template <typename T, int NT, int PAIRS, int OCC>
__global__ void __launch_bounds__(64 * kWaves, OCC)
k_key_weights(Geom g, const T* Qp, const T* Kp, const float* lse, float* out, Stages sg, float scale_log2) {
    using F = Frag<T, NT, 2>;
    constexpr int kOwn = 32 * PAIRS, kKeys = kOwn * kWaves, kThreads = 64 * kWaves;
    constexpr int kPieces = 4 * (int)(sizeof(F::k) / 16);       // 16-byte pieces of a row that the fragments take, those past d included
    constexpr int kPitch = kPieces | 1;                         // odd: 16 rows' reads of one piece fall on all banks
    constexpr int kLoads = (kRows * kPieces + kThreads - 1) / kThreads;
    constexpr int kFull = 16 / (int)sizeof(T);                  // elements of a piece
    __shared__ u32x4 s_q[2][kRows * kPitch];
    __shared__ float s_l[2][kRows];
    const int tid = threadIdx.x, lane = tid & 63, x = lane & 15, gq = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const float INF = __builtin_huge_valf();

    long long u, u_end;
    if (sg.whole) {
        const int pair = (int)blockIdx.x / sg.tiles, i = (int)blockIdx.x - pair * sg.tiles;
        u = pair * sg.per_pair + sg.before(i);
        u_end = u + sg.of_tile(i);
    } else {
        const long long U = sg.per_pair * g.batch * g.Hkv;
        u = U * blockIdx.x / gridDim.x;
        u_end = U * (blockIdx.x + 1) / gridDim.x;
    }
    int pair = (int)(u / sg.per_pair), tile = sg.find(u - pair * sg.per_pair);
    while (u < u_end) {
        const int b = pair / g.Hkv, kv = pair - b * g.Hkv;
        const int key0 = tile * kKeys + kOwn * w;
        const int skip = sg.skip(tile), per = sg.per_head - skip;
        const int s_lo = (int)(u - pair * sg.per_pair - sg.before(tile));
        const int n = (int)min(u_end - u, sg.of_tile(tile) - s_lo);
        int hl = s_lo / per, at = s_lo - hl * per;              // the next stage to be requested
        int rows0 = 0;

        u32x4 piece[kLoads];
        float l = 0.f;
        auto request = [&]() {
            const int h = kv * g.G + hl, row0 = kRows * (skip + at);
            const T* Q = Qp + b * g.qsb + h * g.qsh;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int p = tid + kThreads * i, row = p / kPieces, c = kFull * (p % kPieces);
                // (channels past d are replaced when they are placed: nothing here waits)
                piece[i] = *reinterpret_cast<const u32x4*>(Q + (long long)min(row0 + row, g.Lq - 1) * g.qsl + (c < g.d ? c : 0));
            }
            if (tid < kRows) {
                l = lse[((long long)b * g.Hq + h) * g.Lq + min(row0 + tid, g.Lq - 1)];
                rows0 = row0;
            }
            if (++at == per) { at = 0; ++hl; }
        };
        auto place = [&](int buf) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int p = tid + kThreads * i, row = p / kPieces, c = p % kPieces;
                if (kRows * kPieces % kThreads == 0 || row < kRows)
                    s_q[buf][row * kPitch + c] = kFull * c < g.d ? piece[i] : u32x4{0u, 0u, 0u, 0u};
            }
            // log2 units; +inf: no such query, or one without a key
            if (tid < kRows) s_l[buf][tid] = rows0 + tid < g.Lq && l != -INF ? l * 1.4426950408889634f : INF;
        };
        int first = g.q0 + kRows * (skip + at), at_now = at;
        request();
        F kf[PAIRS][2];
        f32x4 sum[PAIRS][2];
#pragma unroll
        for (int i = 0; i < PAIRS; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                kf[i][e].load(Kp + b * g.ksb + kv * g.ksh + (long long)min(key0 + 32 * i + 16 * e + x, g.L - 1) * g.ksl, g.d, gq);
                sum[i][e] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
        place(0);
        // the keys are in their registers here: otherwise the loop's first products wait for them, and on later trips with the
        // same instructions for the queries just requested
#pragma unroll
        for (int i = 0; i < PAIRS; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (auto& k : kf[i][e].k) asm volatile("" : "+v"(k));
        for (int s = 0; s < n; ++s) {
            const int buf = s & 1;
            if (s + 1 < n) request();
            __syncthreads();                                    // the stage is in place, and the other buffer has been read
#pragma unroll 2
            for (int v = 0; v < kRows / 16; ++v) {
                F qf[1];
                const int row = 16 * v + x;
#pragma unroll
                for (int i = 0; i < (int)(sizeof(qf[0].k) / 16); ++i) {
                    const u32x4 q = s_q[buf][row * kPitch + 4 * i + gq];
                    qf[0].k[i] = __builtin_bit_cast(typename std::remove_reference<decltype(qf[0].k[0])>::type, q);
                }
                const float l2 = s_l[buf][row];
                f32x4 sc[PAIRS][1][2];
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) sc[i][0][e] = f32x4{0.f, 0.f, 0.f, 0.f};
                    F::template qk<1>(sc[i], kf[i], qf);
                }
                if (first + 16 * v >= key0 + kOwn - 1) {
#pragma unroll
                    for (int i = 0; i < PAIRS; ++i)
#pragma unroll
                        for (int e = 0; e < 2; ++e)
#pragma unroll
                            for (int r = 0; r < 4; ++r) sum[i][e][r] += __builtin_amdgcn_exp2f(fmaf(sc[i][0][e][r], scale_log2, -l2));
                } else {
#pragma unroll
                    for (int i = 0; i < PAIRS; ++i)
#pragma unroll
                        for (int e = 0; e < 2; ++e)
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                const float p = __builtin_amdgcn_exp2f(fmaf(sc[i][0][e][r], scale_log2, -l2));
                                sum[i][e][r] += key0 + 32 * i + 16 * e + 4 * gq + r <= first + row ? p : 0.f;
                            }
                }
            }
            if (++at_now == per) at_now = 0;
            first = g.q0 + kRows * (skip + at_now);
            if (s + 1 < n) place(buf ^ 1);
        }
        // a whole tile's sums are the answer; a part's go to its slot, [blockIdx.x + tiles in front][kKeys]
        const bool split = !sg.whole;
        float* mine = split ? out + ((long long)blockIdx.x + (long long)pair * sg.tiles + tile) * kKeys
                            : out + (long long)pair * g.L + (long long)tile * kKeys;
#pragma unroll
        for (int i = 0; i < PAIRS; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float v = sum[i][e][r];
#pragma unroll
                    for (int o = 1; o < 16; o <<= 1) v += __shfl_xor(v, o);
                    const int k = 32 * i + 16 * e + 4 * gq + r;
                    if (x == r && (split || key0 + k < g.L)) mine[kOwn * w + k] = v;
                }
        u += n;
        if (++tile == sg.tiles) { tile = 0; ++pair; }
        __syncthreads();                                        // the stages' buffers are free again
    }
}

// The slots of a tile, added up in order: a workgroup to a tile, a thread to a key.
__global__ void __launch_bounds__(256)
k_key_weights_join(const float* parts, float* out, Stages sg, int L, int keys, int pairs, int workgroups) {
    const int pair = (int)blockIdx.x / sg.tiles, tile = (int)blockIdx.x - pair * sg.tiles;
    const int key = tile * keys + (int)threadIdx.x;
    if ((int)threadIdx.x >= keys || key >= L) return;
    const long long U = sg.per_pair * pairs, u = pair * sg.per_pair + sg.before(tile), last = u + sg.of_tile(tile) - 1;
    const long long lo = ((u + 1) * workgroups - 1) / U, hi = ((last + 1) * workgroups - 1) / U;     // workgroups that had a share
    const float* p = parts + (lo + blockIdx.x) * keys + threadIdx.x;
    float v = 0.f;
#pragma unroll 4
    for (long long i = lo; i <= hi; ++i, p += keys) v += *p;
    out[(long long)pair * L + key] = v;
}

Stages stages_of(const Geom& g, int dtype) {
    Stages s;
    const int keys = keys_of(dtype, g.d);
    s.G = g.G;
    s.tiles = (g.L + keys - 1) / keys;
    s.per_head = (g.Lq + kRows - 1) / kRows;
    s.per_tile = keys / kRows;
    s.c0 = (g.q0 + kRows - 1) / kRows;
    s.per_pair = s.before(s.tiles);
    s.whole = (long long)g.G * s.per_head <= ((long long)g.batch * g.Hkv * s.tiles >= kManyTiles ? kWholeStages : kShortStages);
    return s;
}
// One round of workgroups, of at least two stages each and no more workgroups than finish as early
int workgroups_of(const Geom& g, const Stages& s, int occupancy) {
    const long long tiles = (long long)g.batch * g.Hkv * s.tiles, U = s.per_pair * g.batch * g.Hkv;
    if (s.whole) return (int)tiles;
    const long long each = std::max(2ll, (U + 256 * occupancy - 1) / (256 * occupancy));
    return (int)((U + each - 1) / each);
}
constexpr int kMostOccupancy = 3;

}  // namespace

size_t key_weights_bytes(const Geom& g, int dtype) {
    const Stages s = stages_of(g, dtype);
    if (s.whole) return 0;
    return ((size_t)workgroups_of(g, s, kMostOccupancy) + (size_t)g.batch * g.Hkv * s.tiles) * keys_of(dtype, g.d) * sizeof(float);
}

// expects batch * Hkv * tiles of keys, and a KV head's stages, within 31 bits, and key_weights_bytes() of workspace
hipError_t launch_key_weights(const Geom& g, int dtype, const void* Q, const void* K, const float* lse, float* out, void* workspace,
                              hipStream_t st) {
    const float scale_log2 = (float)(1.4426950408889634 / sqrt((double)g.d));
    const Stages s = stages_of(g, dtype);
    float* to = s.whole ? out : reinterpret_cast<float*>(workspace);
    int workgroups = 0;
    auto launch = [&](auto kernel, auto type, int occupancy) -> hipError_t {
        typedef decltype(type) T;
        workgroups = workgroups_of(g, s, occupancy);
        hipLaunchKernelGGL(kernel, dim3((unsigned)workgroups), dim3(64 * kWaves), 0, st, g, reinterpret_cast<const T*>(Q),
                           reinterpret_cast<const T*>(K), lse, to, s, scale_log2);
        return hipGetLastError();
    };
    auto pick = [&](auto tiles) -> hipError_t {
        constexpr int N = decltype(tiles)::value;
        constexpr int kBf16 = pairs_of<bf16_t, N>(), kF32 = pairs_of<float, N>();
        constexpr int kOccBf16 = N <= 8 ? kMostOccupancy : 2, kOccF32 = N <= 8 ? kMostOccupancy : 1;
        return dtype == RR_BF16 ? launch(k_key_weights<bf16_t, N, kBf16, kOccBf16>, bf16_t{}, kOccBf16)
                                : launch(k_key_weights<float, N, kF32, kOccF32>, float{}, kOccF32);
    };
    using std::integral_constant;
    hipError_t e = hipErrorInvalidValue;
    switch ((g.d + 15) / 16) {
#define RR_WEIGHTS_CASE(N) case N: e = pick(integral_constant<int, N>{}); break
        RR_WEIGHTS_CASE(1); RR_WEIGHTS_CASE(2); RR_WEIGHTS_CASE(3); RR_WEIGHTS_CASE(4);
        RR_WEIGHTS_CASE(5); RR_WEIGHTS_CASE(6); RR_WEIGHTS_CASE(7); RR_WEIGHTS_CASE(8);
        RR_WEIGHTS_CASE(9); RR_WEIGHTS_CASE(10); RR_WEIGHTS_CASE(11); RR_WEIGHTS_CASE(12);
        RR_WEIGHTS_CASE(13); RR_WEIGHTS_CASE(14); RR_WEIGHTS_CASE(15); RR_WEIGHTS_CASE(16);
#undef RR_WEIGHTS_CASE
        default: break;
    }
    if (e != hipSuccess || s.whole) return e;
    hipLaunchKernelGGL(k_key_weights_join, dim3((unsigned)(g.batch * g.Hkv * s.tiles)), dim3(256), 0, st, to, out, s, g.L,
                       keys_of(dtype, g.d), g.batch * g.Hkv, workgroups);
    return hipGetLastError();
}

}  // namespace rr
