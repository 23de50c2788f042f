// The arithmetic of a tile for the shared latent 576/512, used by the verify and the prompt attention kernels: the scores of one
// tile and the product with V of the tile before, every instruction placed between two MFMAs by hand.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>
#include <utility>

#include "seer_device.h"
#include "seer_tile.h"

namespace seer {

namespace mla {
constexpr int kDqk = 576, kDv = 512;
constexpr int kMinPage = 32;                       // pages of 32 tokens or a larger power of two: a tile lies inside one page
constexpr int kTile = 32;
constexpr int kRowBytes = kDqk * 2;               // 1152
constexpr int kChunksPerRow = kRowBytes / 16;      // 72
constexpr int kStageBytes = kTile * kRowBytes;     // 36864
constexpr int kBlocks = kStageBytes / 1024;        // 36 one-KB wave loads per tile
constexpr int kWaves = 4;
constexpr int kRowsPerWg = 32 * kWaves;            // 128
constexpr int kStages = 3;                        // tile u (K operand), tile u-1 (V operand), one in flight
constexpr int kLoadsPerWave = kBlocks / kWaves;    // 9
constexpr int kKSteps = kDqk / 16;                 // 36
constexpr int kDTiles = kDv / 32;                  // 16
constexpr int kQRegSteps = 24;                     // contraction steps whose Q^T operand stays in registers
constexpr int kQLdsSteps = kKSteps - kQRegSteps;   // the remaining 12 are re-read from LDS every tile
static_assert(kBlocks % kWaves == 0, "every wave issues the same number of loads");

// Row r starts 1152 r bytes into the stage, i.e. at bank group (in 16-byte units) 8 (r & 1) of the 16
// that make up the 64 banks, so row parity supplies one bit of spread and the swizzle the other three.
__device__ __forceinline__ int swz(int row) { return (((row >> 1) & 1) << 2) | (((row >> 2) & 1) << 1) | ((row >> 3) & 1); }
}  // namespace mla

// LDS byte address of an object in LDS, for the address operands of the asm blocks below.
template <typename T>
__device__ __forceinline__ int lds_addr(T* p) {
    return static_cast<int>(reinterpret_cast<uintptr_t>((SEER_AS3 void*)(p)));
}

// Operand reads whose issue and completion are separated by hand (LDS returns in order, so
// "s_waitcnt lgkmcnt(N)" with N = the reads issued after a group means that group has arrived).
// The issuing block names the destination registers as outputs although they are only written
// when the read returns; the matching wait block takes them as read-write operands, so every use
// of the data is ordered after the wait.  They do not go through the builtins: the compiler puts a
// vmcnt(0) in front of those, because it cannot tell the reads apart from the direct-to-LDS loads
// still in flight.
//
// one read, one wait
#define SEER_MLA_READ128(dst, addr, OFF) \
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=&v"(dst) : "v"(addr), "n"(OFF))
#define SEER_MLA_READ_TR2(dst, addr_lo, addr_hi, OFF_LO, OFF_HI)                                           \
    asm volatile("ds_read_b64_tr_b16 %0, %2 offset:%4\n"                                                   \
                 "ds_read_b64_tr_b16 %1, %3 offset:%5"                                                     \
                 : "=&v"(dst[0]), "=&v"(dst[1])                                                            \
                 : "v"(addr_lo), "v"(addr_hi), "n"(OFF_LO), "n"(OFF_HI))
template <int N>
__device__ __forceinline__ void wait_lgkm() {
    static_assert(N >= 0 && N < 16, "lgkmcnt is a 4-bit counter");
    // (through the builtin: an instruction the compiler knows between two asm MFMAs on one accumulator keeps it from
    // padding them with a wait state of its own; vmcnt and expcnt fields at their maxima = no wait on those)
    __builtin_amdgcn_s_waitcnt(0xc07f | (N << 8));
}
#define SEER_MLA_FENCE() __builtin_amdgcn_sched_barrier(0)
// Keeps the computation of x at the place where it is written (see the D = 128 kernel).
#define SEER_MLA_PIN(x) asm volatile("" : "+v"(x))

// acc += A . B with the accumulator pinned to the AGPR half of the register file.  Written as asm
// because the compiler, left to choose, keeps part of the 256 accumulators in VGPRs and then
// spills the Q^T operands; with the accumulators forced into AGPRs everything else fits in VGPRs.
// The compiler does not see an MFMA here, so the code that later reads the accumulators with
// ordinary instructions (rescale, epilogue) first idles past the MFMA pipeline depth itself
// (mfma_drain).  Dependent MFMAs on one accumulator are interlocked by the hardware.
__device__ __forceinline__ void mfma_acc(f32x16& acc, u32x4 a, u32x4 b) {
    asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
}
// The score accumulator, pinned to VGPRs (all AGPRs hold O^T).
__device__ __forceinline__ void mfma_vgpr(f32x16& acc, u32x4 a, u32x4 b) {
    asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(acc) : "v"(a), "v"(b));
}
// ... starting from zero
__device__ __forceinline__ void mfma_vgpr_first(f32x16& acc, u32x4 a, u32x4 b) {
    asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(acc) : "v"(a), "v"(b));
}
__device__ __forceinline__ void mfma_drain() { asm volatile("s_nop 15\n\ts_nop 15" ::: "memory"); }

namespace mla {

template <typename F, int... I>
__device__ __forceinline__ void for_each_index(F&& f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>{}), ...);
}

// A wave issues in order, and an MFMA holds the matrix core for 32 cycles: whatever else a step has
// to issue (operand reads from LDS, the softmax arithmetic) only runs in the shadow of the MFMAs
// if it sits BETWEEN them, one MFMA at a time.  Both phases below are written that way: after
// every MFMA come the one or two LDS reads that feed an MFMA a fixed distance ahead, and a slice
// of vector-ALU work.

constexpr int kKAhead = 8;    // the K operand of score step kk is read kKAhead MFMAs before it is used
constexpr int kQAhead = 4;    // ... the parked Q^T operands kQAhead MFMAs before
constexpr int kVAhead = 6;    // the V^T operand of a P.V MFMA (two transposing reads) kVAhead MFMAs before
constexpr int kLoadFirst = 1, kLoadEvery = 4;   // load i of the next tile goes behind score MFMA kLoadFirst + i kLoadEvery
static_assert(kLoadFirst + (kLoadsPerWave - 1) * kLoadEvery < kKSteps, "all loads of a tile fit in one score phase");

// LDS reads outstanding behind the operand(s) of score step kk at the point where that step waits,
// from the order in which phase_a issues them
// (with V_AHEAD, the last kVAhead score steps are each followed by the two transposing reads of one of the first
// kVAhead P.V MFMAs of the phase that comes next)
constexpr int kVFirst = kKSteps - kVAhead;
constexpr int qk_wait_count(int kk, bool v_ahead) {
    int seq = 0, pos_k[kKSteps] = {}, pos_q[kKSteps] = {}, before[kKSteps] = {};
    for (int i = 0; i < kKAhead; ++i) pos_k[i] = seq++;
    for (int m = 0; m < kKSteps; ++m) {
        before[m] = seq;
        if (m + kKAhead < kKSteps) pos_k[m + kKAhead] = seq++;
        if (m + kQAhead >= kQRegSteps && m + kQAhead < kKSteps) pos_q[m + kQAhead] = seq++;
        if (v_ahead && m >= kVFirst) seq += 2;
    }
    int need = pos_k[kk];
    if (kk >= kQRegSteps && pos_q[kk] > need) need = pos_q[kk];
    return before[kk] - 1 - need;
}
static_assert(kQRegSteps >= kQAhead && qk_wait_count(0, false) == kKAhead - 1 && qk_wait_count(kKSteps - 1, false) == 0, "");
static_assert(qk_wait_count(kKSteps - 1, true) < 16, "lgkmcnt is a 4-bit counter");

// The V^T operand of P.V MFMA m (see phase_b) : two transposing reads into ring slot m % kVAhead.
template <int m>
__device__ __forceinline__ void v_read(u32x2 (&vr)[kVAhead][2], int a_even, int a_even8, int a_odd, int a_odd8) {
    constexpr int G2 = m >> 2, w = m & 3;
    constexpr int off_lo = G2 * 128 + (w >= 2 ? 16 : 0) * kRowBytes, off_hi = off_lo + 8 * kRowBytes;
    if constexpr (w & 1) SEER_MLA_READ_TR2(vr[m % kVAhead], a_odd, a_odd8, off_lo, off_hi);
    else SEER_MLA_READ_TR2(vr[m % kVAhead], a_even, a_even8, off_lo, off_hi);
}

// Phase A of a pipeline step: the scores of tile u (36 MFMAs into s_new) with, in their shadow, the
// probabilities of tile u-1 (s_old -> pk, l_run; the exponent reference m_use and the factor alpha of that
// tile were set during the phase B before).  ka: LDS addresses of this lane's K
// operand chunks for contraction steps 0..3 of the tile (steps 4g + j are 128 g bytes further);
// qt: LDS address of this lane's parked Q^T operands.  s_old must already carry -inf in masked slots.
// With DO_SM, the V^T operands of the first kVAhead P.V MFMAs of tile u-1 (addresses va) are requested behind the
// last score MFMAs, so that phase B starts without waiting for LDS.
// load(i): request load i of the next tile; extra(kk): other arithmetic for the shadow of score MFMA kk (no LDS traffic;
// it may write va before step kVFirst).
template <bool DO_QK, bool DO_SM, typename LOAD, typename EXTRA>
__device__ __forceinline__ void phase_a(const int (&ka)[4], int qt, const u32x4 (&qreg)[kQRegSteps], f32x16& s_new,
                                        f32x16& s_old, uint32_t (&pk)[8], float m_use, float& l_run, float alpha,
                                        float scale_log2, int (&va)[4], u32x2 (&vr)[kVAhead][2], LOAD&& load,
                                        EXTRA&& extra) {
    u32x4 kr[kKAhead], qr[kQAhead];
    if constexpr (DO_QK) {
        for_each_index([&](auto ic) __attribute__((always_inline)) {
            constexpr int I = decltype(ic)::value;
            (void)&kr, (void)&ka;   // (asm operands alone do not capture)
            SEER_MLA_READ128(kr[I], ka[I & 3], (I >> 2) * 128);
        }, std::make_integer_sequence<int, kKAhead>{});
    }
    float psum = 0.f, p_even = 0.f;
    if constexpr (!DO_QK && DO_SM) {
        for_each_index([&](auto ic) __attribute__((always_inline)) {
            (void)&vr, (void)&va;
            v_read<decltype(ic)::value>(vr, va[0], va[1], va[2], va[3]);
        }, std::make_integer_sequence<int, kVAhead>{});
    }
    // probability of slot i; two of them make one packed register
    auto element = [&](auto ic) __attribute__((always_inline)) {
        constexpr int i = decltype(ic)::value;
        if constexpr (DO_SM) {
            const float p = fast_exp2(fmaf(s_old[i], scale_log2, -m_use));
            if constexpr (i % 2 == 0) {
                p_even = p;
                SEER_MLA_PIN(p_even);
                // the sum takes the probabilities as the P.V product will see them, a pair per instruction,
                // one pair behind (not right after the packing that produces its operand)
                if constexpr (i >= 2) {
                    psum = add_bf16_pair(pk[(i >> 1) - 1], psum);
                    SEER_MLA_PIN(psum);
                }
            } else {
                pk[i >> 1] = cvt_pk_bf16(p_even, p);
                SEER_MLA_PIN(pk[i >> 1]);
            }
        }
    };
    SEER_MLA_FENCE();
    if constexpr (DO_QK) {
        for_each_index([&](auto ic) __attribute__((always_inline)) {
            constexpr int kk = decltype(ic)::value;
            (void)&kr, (void)&qr, (void)&ka, (void)&qt;   // (asm operands alone do not capture)
            wait_lgkm<qk_wait_count(kk, DO_SM)>();
            const u32x4 qv = kk < kQRegSteps ? qreg[kk < kQRegSteps ? kk : 0] : qr[kk % kQAhead];
            if constexpr (kk == 0) mfma_vgpr_first(s_new, kr[0], qv); else mfma_vgpr(s_new, kr[kk % kKAhead], qv);
            if constexpr (kk + kKAhead < kKSteps)
                SEER_MLA_READ128(kr[kk % kKAhead], ka[(kk + kKAhead) & 3], ((kk + kKAhead) >> 2) * 128);
            if constexpr (kk + kQAhead >= kQRegSteps && kk + kQAhead < kKSteps)
                SEER_MLA_READ128(qr[kk % kQAhead], qt, (kk + kQAhead - kQRegSteps) * 1024);
            if constexpr (DO_SM && kk >= kVFirst) {
                (void)&vr, (void)&va;
                v_read<kk - kVFirst>(vr, va[0], va[1], va[2], va[3]);
            }
            // one probability in the shadow of every second MFMA
            if constexpr (kk >= 2 && kk % 2 == 0 && (kk - 2) / 2 < 16) element(std::integral_constant<int, (kk - 2) / 2>{});
            // ... and one of this wave's loads of the next tile behind every kLoadEvery-th
            if constexpr (kk >= kLoadFirst && (kk - kLoadFirst) % kLoadEvery == 0 && (kk - kLoadFirst) / kLoadEvery < kLoadsPerWave)
                load(std::integral_constant<int, (kk - kLoadFirst) / kLoadEvery>{});
            extra(ic);
            SEER_MLA_FENCE();
        }, std::make_integer_sequence<int, kKSteps>{});
    } else {
        for_each_index(element, std::make_integer_sequence<int, 16>{});
    }
    if constexpr (DO_SM) {
        psum = add_bf16_pair(pk[7], psum);
        l_run = l_run * alpha + psum;
        SEER_MLA_PIN(l_run);
    }
}

// Phase B: O^T[d][row] += sum_token V[token][d] * P[row][token] for one tile (32 MFMAs), V = first 512
// dims of the latent through the transposing read.  MFMA m = 4 G2 + w works on the pair of d-tiles G2:
// w = 0, 1: even, odd d-tile, tokens 0..15;  w = 2, 3: even, odd d-tile, tokens 16..31.
// va = {a_even, a_even8, a_odd, a_odd8}: lane address for even / odd d-tiles; the token rows +8 and +24 differ
// from +0 and +16 in row bit 3, which the swizzle uses: they go through addresses of their own.
// The operands of MFMAs 0..kVAhead-1 are already on their way into vr (requested by phase A); shadow(m) is vector
// arithmetic to issue behind MFMA m (it must not touch LDS).
template <typename SHADOW>
__device__ __forceinline__ void phase_b(const int (&va)[4], u32x2 (&vr)[kVAhead][2], const uint32_t (&pk)[8],
                                        f32x16 (&acc)[kDTiles], SHADOW&& shadow) {
    const u32x4 pb0 = {pk[0], pk[1], pk[2], pk[3]};
    const u32x4 pb1 = {pk[4], pk[5], pk[6], pk[7]};
    for_each_index([&](auto ic) __attribute__((always_inline)) {
        constexpr int m = decltype(ic)::value;
        constexpr int left = kDTiles * 2 - 1 - m;                       // MFMAs after this one
        (void)&vr, (void)&va;                                           // (asm operands alone do not capture)
        wait_lgkm<2 * (left < kVAhead - 1 ? left : kVAhead - 1)>();
        const u32x4 v = {vr[m % kVAhead][0][0], vr[m % kVAhead][0][1], vr[m % kVAhead][1][0], vr[m % kVAhead][1][1]};
        mfma_acc(acc[(m >> 2) * 2 + (m & 1)], v, (m & 2) ? pb1 : pb0);
        if constexpr (m + kVAhead < kDTiles * 2) v_read<m + kVAhead>(vr, va[0], va[1], va[2], va[3]);
        shadow(ic);
        SEER_MLA_FENCE();
    }, std::make_integer_sequence<int, kDTiles * 2>{});
}

}  // namespace mla

}  // namespace seer
