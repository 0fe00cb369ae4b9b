// The pipeline of attention on 32 x 32 matrix tiles for bf16 rows of 128 channels (rr_attn_mfma.hip, where its design is
// described, and rr_window_mfma.hip): operand addressing, tile copies to LDS, one pipelined phase, and the plain steps.
#pragma once
#include "rr_common.hpp"

namespace rr {

namespace {

constexpr int kWaves = 4;                            // 32 queries each
constexpr int kThreads = 64 * kWaves;
constexpr int kTileKeys = 64;
constexpr int kRowsPerWave = kTileKeys / kWaves;     // tile rows each wave copies
constexpr int kCopies = kRowsPerWave / 4;            // copy instructions per wave and tile (4 rows each)
constexpr int kTileBytes = kTileKeys * 256;          // one 64 x 128 bf16 tile
constexpr int kLdsBytes = 4 * kTileBytes;            // K and V, two stages each
constexpr int kOutRowBytes = 264;                    // 128 bf16 + 8 bytes of padding
constexpr int kXchgFloats = 67;                      // per lane, of a wide workgroup's second group: O^T, reference, sums

typedef __attribute__((address_space(3))) void* lds_ptr_t;
typedef __attribute__((address_space(3))) unsigned char lds_byte_t;
typedef __attribute__((address_space(3))) int lds_int_t;
typedef __attribute__((address_space(3))) bf16x8 lds_bf16x8_t;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((address_space(3))) s16x4* lds_s16x4_ptr_t;

__device__ __forceinline__ int k_swz(int key, int chunk) { return key * 256 + ((chunk ^ (key & 15)) << 4); }
__device__ __forceinline__ int v_swz(int key, int chunk) { return key * 256 + ((chunk ^ ((key & 7) << 1)) << 4); }

#define SCHED_FENCE() __builtin_amdgcn_sched_barrier(0)

// The MFMAs are one-instruction asm statements so that the register class of every operand is
// fixed by hand: O^T and the Q^T operand live in the accumulation registers (only the matrix
// pipe touches them), S^T lands in ordinary vector registers because the softmax reads it with
// vector ALU instructions.  (Left to itself the compiler puts every MFMA result in accumulation
// registers and copies S^T out and back around each instruction.)
// The compiler does not see inside these statements and adds no wait states for them.  The code
// keeps the distances itself: inside the pipeline a result is only reused as the accumulator of
// the next MFMA of its chain (which the matrix pipe interlocks) or, for S^T, read by vector
// instructions a whole phase and a barrier later; wherever else vector instructions touch a
// result, a settle statement comes first.
#define RR_MFMA_TEXT "v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0"
__device__ __forceinline__ void mfma_pv(f32x16& acc, const bf16x8& vt, const bf16x8& pt) {
    asm volatile(RR_MFMA_TEXT : "+a"(acc) : "v"(vt), "v"(pt));
}
__device__ __forceinline__ void mfma_qk(f32x16& s, const bf16x8& k, const bf16x8& qt) {
    asm volatile(RR_MFMA_TEXT : "+v"(s) : "v"(k), "a"(qt));
}
__device__ __forceinline__ void mfma_qk_first(f32x16& s, const bf16x8& k, const bf16x8& qt) {
    asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(s) : "v"(k), "a"(qt));
}
// Idle issue cycles longer than the tail of the last MFMA, then the values pass through empty
// asm statements: whatever reads them afterwards depends on those statements and therefore
// cannot be scheduled in front of the idle cycles.
__device__ __forceinline__ void mfma_settle_s(f32x16& s) {
    asm volatile("s_nop 15\n\ts_nop 15\n\ts_nop 15" : "+v"(s));
}
__device__ __forceinline__ void mfma_settle_acc(f32x16 (&acc)[4]) {
    asm volatile("s_nop 15\n\ts_nop 15\n\ts_nop 15");
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) asm volatile("" : "+a"(acc[dt]));
}

// Per-wave state and operand addressing.
struct Wave {
    const lds_byte_t* lds;
    int lane, l32, gsel;
    float sl2;                         // log2(e) / sqrt(d)
    float lazy, lazy_sum;              // how far above the softmax reference a score may lie: in log2 units, and 2^ that
    bool tight;                        // a constant: no registers for two tiles of O^T outside their place, see move_reference
    bf16x8 qf[8];                      // Q^T operand: 16-wide d chunks
    f32x16 acc[4];                     // O^T: 32-row d tiles
    float mref;                        // softmax reference of the lane's query, log2 units
    float lsum;                        // this lane's part of the denominator: the sum of P as rounded
    float lfix;                        // what rounding took from it where that is known, for the log-sum-exp
    // Per-lane LDS byte addresses.  The XOR swizzle makes the chunk part of an address
    // base ^ (32 * kc) for K and base ^ (64 * dt) for V.
    unsigned ka0;                      // K: row lane%32, chunk gsel, swizzled
    unsigned va0;                      // V: keys 4 gsel + (lane%16)/4, d tile 0
    // ... and all of them, so that the hot loop forms no address: the chunk part is kaddr[kc] = ka0 ^ 32 kc,
    // vaddr[dt] = va0 ^ 64 dt; buffer, subtile and key-chunk selection ride in the instruction's immediate
    // offset (the loop is unrolled over the buffer parity for that).
    unsigned kaddr[8];
    unsigned vaddr[4];

    __device__ __forceinline__ void init_addresses() {
        const unsigned lds0 = (unsigned)(uintptr_t)lds;       // LDS addresses are 32 bits
        ka0 = lds0 + k_swz(l32, gsel);
        const int s16 = lane & 15, dhalf = (lane >> 4) & 1;
        const int key = 4 * gsel + (s16 >> 2);
        va0 = lds0 + 2 * kTileBytes + 8 * (s16 & 1) + v_swz(key, 2 * dhalf + ((s16 & 3) >> 1));
#pragma unroll
        for (int kc = 0; kc < 8; ++kc) kaddr[kc] = ka0 ^ (32u * kc);
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) vaddr[dt] = va0 ^ (64u * dt);
    }
    __device__ __forceinline__ unsigned ka(int kc) const { return ka0 ^ (32u * kc); }
    __device__ __forceinline__ unsigned va(int dt) const { return va0 ^ (64u * dt); }
    __device__ __forceinline__ bf16x8 kfrag_at(unsigned at, int buf, int t) const {
        return *(const lds_bf16x8_t*)(uintptr_t)(at + (unsigned)(buf * kTileBytes + t * 32 * 256));
    }
    // fragment reads of the pipeline: address register + compile-time byte offset
    template <int OFF>
    __device__ __forceinline__ bf16x8 kfrag_imm(int kc) const {
        return *(const lds_bf16x8_t*)(uintptr_t)(kaddr[kc] + (unsigned)OFF);
    }
    template <int OFF>
    __device__ __forceinline__ bf16x8 vfrag_imm(int u) const { return vfrag_at(vaddr[u >> 1] + (unsigned)OFF, 0, 0, u); }
    __device__ __forceinline__ bf16x8 kfrag(int buf, int t, int kc) const { return kfrag_at(ka(kc), buf, t); }
    // V^T operand (32 d rows x 16 keys) of d tile u >> 1 and 16-key chunk u & 1 of subtile t: two
    // transposing reads, keys {4g..4g+3} and {8+4g..8+4g+3} of the chunk (accumulator order).
    __device__ __forceinline__ bf16x8 vfrag(int buf, int t, int u) const { return vfrag_at(va(u >> 1), buf, t, u); }
    __device__ __forceinline__ bf16x8 vfrag_at(unsigned at, int buf, int t, int u) const {
        const unsigned p = at + (unsigned)(buf * kTileBytes + t * 32 * 256 + (u & 1) * 16 * 256);
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr_t)(uintptr_t)p);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr_t)(uintptr_t)(p + 8 * 256));
        typedef __attribute__((ext_vector_type(8))) short s16x8;
        const s16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(bf16x8, both);
    }
};

// S^T of one 32-key step, nothing overlapped (the diagonal block).
__device__ __forceinline__ void qk_step(const Wave& w, int buf, int t, f32x16& s) {
#pragma unroll
    for (int kc = 0; kc < 8; ++kc) {
        const bf16x8 kf = w.kfrag(buf, t, kc);
        if (kc == 0) mfma_qk_first(s, kf, w.qf[kc]);
        else mfma_qk(s, kf, w.qf[kc]);
    }
    mfma_settle_s(s);
}

// O^T += V^T P^T of one 32-key step, nothing overlapped.
__device__ __forceinline__ void pv_step(Wave& w, int buf, int t, const bf16x8 (&p)[2]) {
#pragma unroll
    for (int u = 0; u < 8; ++u) mfma_pv(w.acc[u >> 1], w.vfrag(buf, t, u), p[u & 1]);
    mfma_settle_acc(w.acc);
}

// P of a step's 16 scores against a reference: exp2, rounded; the sum of the rounded terms and of what rounding took.  (kExact,
// here and below: the sum of the terms before rounding, and nothing taken.)
template <bool kExact = false>
__device__ __forceinline__ void exp_all(const Wave& w, const f32x16& s, float ref, bf16x8 (&p)[2], float& psum, float& fix) {
    const float nb = -ref;
    bf16x2 ones;
    ones[0] = (__bf16)1.0f;
    ones[1] = (__bf16)1.0f;
    float sum = 0.f;
    psum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
        const float e0 = __builtin_amdgcn_exp2f(fmaf(s[r], w.sl2, nb));
        const float e1 = __builtin_amdgcn_exp2f(fmaf(s[r + 1], w.sl2, nb));
        sum += e0;
        sum += e1;
        bf16x2 pr;
        pr[0] = (__bf16)e0;
        pr[1] = (__bf16)e1;
        p[r >> 3][r & 7] = pr[0];
        p[r >> 3][(r & 7) + 1] = pr[1];
        psum = __builtin_amdgcn_fdot2_f32_bf16(pr, ones, psum, false);
    }
    if (kExact) psum = sum;
    fix = kExact ? 0.f : sum - psum;
}
__device__ __forceinline__ float max_of(const f32x16& s) {
    float mx = -__builtin_huge_valf();
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[r]);
    return mx;
}

// Moves the softmax reference of the lane's query up to the new maximum, rescales O^T and the
// denominator, and recomputes P of the step at hand.  Rare; entered by the whole wave.  (Where registers are short, each
// tile of O^T is back in place before the next is taken; without that the ragged and persistent forms spill 12 to 25
// registers: 32K tokens 3357 against 3296 us.  The plain form has room, and is 0.7 % faster without: 64K, 64 heads.)
template <bool kExact = false>
__device__ __forceinline__ void move_reference(Wave& w, const f32x16& s, bf16x8 (&p)[2], float& psum, float& fix, float mx) {
    mfma_settle_acc(w.acc);                             // O^T is about to be read by vector instructions
    float top = mx * w.sl2;
    top = fmaxf(top, __shfl_xor(top, 32));
    const float nref = fmaxf(w.mref, top);
    const float use = (nref == -__builtin_huge_valf()) ? 0.f : nref;
    const float alpha = __builtin_amdgcn_exp2f(w.mref - use);   // 0 while the reference is -inf
    w.mref = nref;
    w.lsum *= alpha;
    w.lfix *= alpha;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) {
#pragma unroll
        for (int r = 0; r < 16; ++r) w.acc[dt][r] *= alpha;
        if (w.tight) asm volatile("" : "+a"(w.acc[dt]));
    }
    exp_all<kExact>(w, s, use, p, psum, fix);
    mfma_settle_acc(w.acc);                             // ... and was written by them
}

// softmax of one 32-key step, nothing overlapped (the diagonal block)
template <bool kExact = false>
__device__ __forceinline__ void softmax_step(Wave& w, const f32x16& s, bf16x8 (&p)[2]) {
    float psum, fix;
    exp_all<kExact>(w, s, w.mref, p, psum, fix);
    const float mx = max_of(s);
    if (__any(mx * w.sl2 > w.mref + w.lazy)) move_reference<kExact>(w, s, p, psum, fix, mx);
    w.lsum += psum;
    w.lfix += fix;
}

// Global -> LDS copies of one 64 x 128 bf16 tile, kCopies instructions per wave (4 rows each), issued
// as asm statements: the compiler would otherwise make every later LDS read wait for them (it
// cannot tell that the reads go to the other buffer), which turns the prefetch into a blocking
// copy.  The kernel waits for them itself (wait_vm) before the barrier that hands a buffer over.
// Lane l lands in LDS slot (row l/16 of the group, physical chunk l%16) and therefore fetches
// logical chunk (l%16) ^ swizzle(row); the per-lane byte offsets of the wave's row groups are kept in
// registers, the tile origin is wave-uniform.
struct Stager {
    const unsigned short* Kp;
    const unsigned short* Vp;
    long long ksl;
    unsigned lds0;                     // LDS address of the buffers
    int wv;                            // wave index, uniform
    unsigned koff[kCopies];            // K: byte offset of this lane's 16 bytes in row group i
    unsigned voff[kCopies];            // V: same with the V swizzle

    __device__ __forceinline__ void init(int lane) {
        const int r4 = lane >> 4, c = lane & 15;
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const int row = 4 * i + r4;                    // row inside the wave's rows (16 | rows per wave: swizzle period)
            koff[i] = 2u * ((unsigned)(row * ksl) + 8u * (c ^ (row & 15)));
            voff[i] = 2u * ((unsigned)(row * ksl) + 8u * (c ^ ((row & 7) << 1)));
        }
    }
    // one of the copies of a tile: row group i of this wave's rows
    __device__ __forceinline__ void issue_one(const unsigned short* wave_src, unsigned wave_dst,
                                              const unsigned (&off)[kCopies], int i) const {
        asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1"
                     :: "v"(off[i]), "s"(wave_src), "s"(wave_dst + 4 * i * 256) : "memory");
    }
    // this wave's rows of half `hf` (64 keys) of key block n
    __device__ __forceinline__ const unsigned short* k_src(int n, int hf) const {
        return Kp + ((long long)n * 128 + kTileKeys * hf + kRowsPerWave * wv) * ksl;
    }
    __device__ __forceinline__ const unsigned short* v_src(int n, int hf) const {
        return Vp + ((long long)n * 128 + kTileKeys * hf + kRowsPerWave * wv) * ksl;
    }
    __device__ __forceinline__ unsigned k_dst(int buf) const { return lds0 + buf * kTileBytes + kRowsPerWave * wv * 256; }
    __device__ __forceinline__ unsigned v_dst(int buf) const { return lds0 + (2 + buf) * kTileBytes + kRowsPerWave * wv * 256; }
    // Half `hf` of a block whose last rows lie past the real length (`rows` real rows, 1 <= rows < 128): those LDS
    // rows get a copy of the last real row (finite, and masked by token causality wherever a real query meets
    // them).  Offsets are formed on the spot from the block origin: this path runs once per launch row at most.
    __device__ __forceinline__ void issue_partial(const unsigned short* base, int n, int hf, unsigned dst, bool is_v,
                                                  int rows, int lane) const {
        const unsigned short* block = base + (long long)n * 128 * ksl;
        const int r4 = lane >> 4, c = lane & 15;
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const int row = 4 * i + r4;                      // LDS row inside the wave's rows: decides the swizzle
            const int src_row = min(kTileKeys * hf + kRowsPerWave * wv + row, rows - 1);
            const unsigned sw = is_v ? ((row & 7) << 1) : (row & 15);
            const unsigned off = 2u * ((unsigned)(src_row * ksl) + 8u * (c ^ sw));
            asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1"
                         :: "v"(off), "s"(block), "s"(dst + 4 * i * 256) : "memory");
        }
    }
    __device__ __forceinline__ void issue_k(int n, int hf, int buf) const {
#pragma unroll
        for (int i = 0; i < kCopies; ++i) issue_one(k_src(n, hf), k_dst(buf), koff, i);
    }
    __device__ __forceinline__ void issue_v(int n, int hf, int buf) const {
#pragma unroll
        for (int i = 0; i < kCopies; ++i) issue_one(v_src(n, hf), v_dst(buf), voff, i);
    }
};

__device__ __forceinline__ void wait_vm() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// One pipeline phase: the MFMAs of PV(step j-1) [V^T fragments from LDS base vbase, operand pprev]
// and of QK(step j+1) [K fragments from kbase, result snext] interleaved with the exp2 / sum /
// max / bf16 rounding of step j [scores scur -> pcur], one element per MFMA slot, and (kFetch)
// with the wave's global -> LDS copies of the prefetched K and V tiles, one every other slot, so the
// copies never queue up in front of the arithmetic.  `valid` is false for the two fill phases at either end of a
// row, whose softmax is thrown away.
template <bool kFetch, int VOFF, int KOFF, bool kExact = false>
__device__ __forceinline__ void phase(Wave& w, const f32x16& scur, f32x16& snext,
                                      const bf16x8 (&pprev)[2], bf16x8 (&pcur)[2],
                                      bool valid, const Stager& st,
                                      const unsigned short* k_src, unsigned k_dst,
                                      const unsigned short* v_src, unsigned v_dst) {
    // The empty asm statements emit nothing.  Being ordered among themselves and with the MFMA
    // statements, they keep the compiler from sinking the softmax arithmetic out of the MFMA
    // shadow or hoisting all operand reads to the top.
    bf16x8 vf[2], kf[2];
    vf[0] = w.template vfrag_imm<VOFF>(0);
    kf[0] = w.template kfrag_imm<KOFF>(0);
    float psum = 0.f;
    const float nb = -w.mref;
    bf16x2 ones;
    ones[0] = (__bf16)1.0f;
    ones[1] = (__bf16)1.0f;
    // Softmax of step j, software pipelined over the MFMA slots so that no vector instruction waits for the
    // one in front of it: stage A (scale and shift of element k) runs at step k, B (its exp2) at step k + 1,
    // C (rounding the pair (2j, 2j+1) to bf16, which is what PV will use) at step 2j + 3, D (adding the pair to
    // the row sum) at step 2j + 4.
    constexpr int NE = 16;
    float tq[NE], ev[NE];
    auto step = [&](int sidx) {
        if (sidx >= 1 && sidx - 1 < NE) {                           // B
            ev[sidx - 1] = __builtin_amdgcn_exp2f(tq[sidx - 1]);
            asm volatile("" : "+v"(ev[sidx - 1]));
        }
        if (sidx < NE) {                                            // A
            tq[sidx] = fmaf(scur[sidx], w.sl2, nb);
            asm volatile("" : "+v"(tq[sidx]));
        }
        if (sidx >= 3 && (sidx & 1) && (sidx - 3) / 2 < NE / 2) {   // C
            const int er = sidx - 3;
            bf16x2 pr;
            pr[0] = (__bf16)ev[er];
            pr[1] = (__bf16)ev[er + 1];
            pcur[er >> 3][er & 7] = pr[0];
            pcur[er >> 3][(er & 7) + 1] = pr[1];
            asm volatile("" : "+v"(pcur[er >> 3]));
        }
        if (sidx >= 4 && !(sidx & 1) && (sidx - 4) / 2 < NE / 2) {  // D
            const int er = sidx - 4;
            if (kExact) {
                psum += ev[er];
                psum += ev[er + 1];
            } else {
                bf16x2 pr;
                pr[0] = pcur[er >> 3][er & 7];
                pr[1] = pcur[er >> 3][(er & 7) + 1];
                psum = __builtin_amdgcn_fdot2_f32_bf16(pr, ones, psum, false);   // sums what PV will use
            }
            asm volatile("" : "+v"(psum));
        }
    };
    // The scores of this step were completed by the last QK MFMA of the previous phase (an asm statement, so the
    // compiler adds no wait states for it); a vector instruction may read them 11 wait states after that MFMA
    // was issued.  The previous phase ends with a PV MFMA, which the matrix pipe accepts 8 wait states after
    // the QK one; the operand reads above and this statement add the rest whatever the compiler puts in
    // between.  The scores pass through the statement, so nothing that reads them can be scheduled in front.
    asm volatile("s_nop 2" : "+v"(const_cast<f32x16&>(scur)));
    // four steps run ahead of the first MFMA: they fill the softmax pipeline and cover the latency of the first
    // operand reads
    step(0);
    step(1);
    step(2);
    step(3);
    SCHED_FENCE();
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        // operand fragments of the next group are requested one group (2 MFMA slots) ahead
        if (u < 7) {
            vf[(u + 1) & 1] = w.template vfrag_imm<VOFF>(u + 1);
            kf[(u + 1) & 1] = w.template kfrag_imm<KOFF>(u + 1);
        }
#pragma unroll
        for (int sl = 0; sl < 2; ++sl) {
            // QK before PV: the phase then ends with a PV product, and the scores of the next step are complete
            // one MFMA earlier
            if (sl == 0) {
                if (u == 0) mfma_qk_first(snext, kf[0], w.qf[0]);
                else mfma_qk(snext, kf[u & 1], w.qf[u]);
                if (kFetch && (u & 1) == 0) st.issue_one(k_src, k_dst, st.koff, u >> 1);
                if (kFetch && (u & 1) == 1) st.issue_one(v_src, v_dst, st.voff, u >> 1);
            } else {
                mfma_pv(w.acc[u >> 1], vf[u & 1], pprev[u & 1]);
            }
            step(2 * u + sl + 4);
            SCHED_FENCE();
        }
    }
    // A score more than 2^8 (2^6) above the reference makes its term, hence the lane's sum of 16 terms,
    // exceed 2^8 (the first step of a row, whose reference is -inf, gives +inf): the sum is the
    // trigger, the maximum itself is only computed on the rare path.
    if (valid) {
        if (__any(!(psum <= w.lazy_sum))) {
            float fix;
            move_reference<kExact>(w, scur, pcur, psum, fix, max_of(scur));
            w.lfix += fix;
        }
        w.lsum += psum;
    }
}

}  // namespace

}  // namespace rr
