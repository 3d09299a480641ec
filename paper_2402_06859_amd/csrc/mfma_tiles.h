// Operand tiles in LDS and the matrix instructions that read them: layouts, direct global-to-LDS loads, fragments and waits,
// shared by the matrix product kernels.
#pragma once
#include "device_common.h"

namespace rdcn {

namespace {

__device__ __forceinline__ int xcd_remap(int id, int n) {
    // Workgroups are dispatched round-robin over the 8 XCDs; give each XCD a
    // contiguous range of tiles so neighbouring tiles share its L2. The last
    // n % 8 workgroups keep their own index.
    const int full = n / 8 * 8;
    if (id >= full) return id;
    return (id % 8) * (n / 8) + id / 8;
}

// ---------------------------------------------------------------------------
// LDS layouts (one stage = one KB-deep slice of A and of B; KB = 64, or 32 in the deeper of the
// streamed blocks):
//  K-contiguous operand, ROWS x KB bf16: row r holds KB/8 chunks of 16 bytes; the
//    chunk of logical k-block kc sits in slot kc ^ kc_swz(r) (((r >> 1) & 7) for KB = 64).
//    Two rows share a 256-byte bank window, so 16 consecutive rows reading the same kc hit 16
//    distinct 16-byte bank groups (ds_read_b128 without conflicts).
//  K-strided operand, 64 k-rows x ROWS bf16 (rows contiguous along m): a k-row
//    holds ROWS/16 chunks of 32 bytes (16 m values); chunk c sits in slot
//    c ^ h(k). MFMA fragments are read with ds_read_b64_tr_b16, which transposes
//    within each 16-lane group: lane (g, j) reads the 4 m values 4(j%4)..+3 of
//    k-row 8g + j/4 (+4 for the second read) and receives the 8 k values of its
//    own m. h(k) spreads the 16 k-rows of one read over all bank groups.
// Loads go straight from global memory into LDS (global_load_lds, 16 bytes per
// lane, lane l writes bytes 16 l .. 16 l + 15 of a 1 KiB block), so the global
// address of each lane is chosen to land in the swizzled position.
// ---------------------------------------------------------------------------
#define LDS_AS __attribute__((address_space(3)))
typedef short s16x4_t __attribute__((ext_vector_type(4)));

// 16-byte direct global-to-LDS load: lane l's 16 bytes land at LDS byte address
// m0 + 16 l. Issued through asm so that the compiler adds no waits of its own:
// every consumer below waits explicitly (wait_vmcnt + s_barrier) for the stage
// it reads. M0 needs one wait state after it is written.
__device__ __forceinline__ void dma16(const void* gptr, uint32_t lds_base) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
                 :
                 : "v"(gptr), "s"(lds_base)
                 : "memory");
}

__device__ __forceinline__ uint32_t lds_addr(const bf16_t* p) { return (uint32_t)(uintptr_t)((LDS_AS const char*)p); }

// Slot XOR of row r of a K-contiguous operand stage of KB bf16 per row: KB = 64 (8 slots
// of 16 bytes, two rows per 256-byte bank window) or 32 (4 slots, four rows per window);
// 16 consecutive rows reading one slot hit 16 distinct 16-byte bank groups.
template <int KB>
__device__ __forceinline__ int kc_swz(int r) {
    return KB == 64 ? ((r >> 1) & 7) : ((r >> 2) & 3);
}

template <int ROWS>
__device__ __forceinline__ int kstr_swz(int k) {
    // ROWS = 128: 8 slots of 32 B per k-row; ROWS = 256: 16 slots, two 256 B windows per
    // k-row (the XOR spreads the k-rows of one read over all 8 slot positions of a window);
    // ROWS = 64: 4 slots, two k-rows per 256 B window
    return ROWS >= 128 ? (((k & 3) << 1) | ((k >> 3) & 1)) : ((((k >> 1) & 1) << 1) | ((k >> 3) & 1));
}

// 16 zero bytes in device memory: the source of the direct-to-LDS loads of K positions
// past a range, so a tail stage arrives in LDS already zero-padded.
__device__ __align__(16) const uint32_t kZero16[4] = {0u, 0u, 0u, 0u};

// Issue this thread's direct-to-LDS loads of one stage (KB deep) for one operand (NW waves).
// Rows past `rows` re-read the last row (K-strided: the 16-byte piece that holds it, so a row count that
// is no multiple of 8 needs a stride that is one; their results are discarded); K positions at
// or past kend read zeros. K-contiguous operands need kend - k0 to be a multiple of 8, or zeros behind kend
// up to one (then a 16-byte piece that straddles kend adds nothing).
// ROLLED keeps its addresses out of the registers and out of the prologue: for the 32 x 32 loop, whose
// accumulators and fragments need the registers and which loads one remainder per block with it, and for
// the streamed blocks, where one wave loads one partial stage with it and the hoisted addresses cost each
// launch (a request of 50 rows, unrolled -> rolled: 69.5 -> 68.1 us; with K remainders 69.9 -> 70.8). The
// other loops load their partial last stage, its re-reads and, without 32-bit offsets (under 8 rows),
// every stage with it: unrolled, the address arithmetic of its loads overlaps (the Feed head's training
// pass at batches 200 to 600, rolled -> unrolled: 420 -> 408 to 674 -> 661 us; requests of 1 to 7 rows
// at width 13824 or 10624: 74 -> 67 to 72 -> 70).
template <int ROWS, bool KS, int NW, int KB, bool ROLLED = false>
__device__ __forceinline__ void stage_load(const bf16_t* __restrict__ base, int64_t ld, int64_t rows, int64_t row0,
                                           int64_t k0, int64_t kend, bf16_t* lds, int wave, int lane) {
    constexpr int NI = ROWS * KB / (512 * NW);  // wave-instructions per thread (1 KiB each)
#pragma unroll(ROLLED ? 1 : NI)
    for (int j = 0; j < NI; ++j) {
        const int blk = wave * NI + j;  // 1 KiB block index within the stage
        int64_t gr, gk;
        if (!KS) {
            constexpr int CPR = KB / 8;    // 16-byte chunks per row
            constexpr int RPB = 64 / CPR;  // rows per 1 KiB block
            const int r = blk * RPB + lane / CPR;
            const int kc = (lane % CPR) ^ kc_swz<KB>(r);
            gr = row0 + r;
            gk = k0 + kc * 8;
            if (gr >= rows) gr = rows - 1;
            const void* src = gk < kend ? (const void*)(base + gr * ld + gk) : (const void*)kZero16;
            dma16(src, lds_addr(lds) + (uint32_t)__builtin_amdgcn_readfirstlane(blk) * 1024u);
        } else {
            constexpr int RPB = ROWS == 256 ? 2 : (ROWS == 128 ? 4 : 8);  // k-rows per 1 KiB block
            constexpr int QPR = 64 / RPB;             // 16-byte pieces per k-row
            const int kr = blk * RPB + lane / QPR;
            const int q = lane % QPR;
            const int c = (q >> 1) ^ kstr_swz<ROWS>(kr);
            gk = k0 + kr;
            gr = row0 + c * 16 + (q & 1) * 8;
            if (gr >= rows) gr = (rows - 1) & ~(int64_t)7;
            const void* src = gk < kend ? (const void*)(base + gk * ld + gr) : (const void*)kZero16;
            dma16(src, lds_addr(lds) + (uint32_t)__builtin_amdgcn_readfirstlane(blk) * 1024u);
        }
    }
}

// The same loads with the address split into a scalar base (wave-uniform, advanced by
// BK along K every step) and a loop-invariant per-lane 32-bit byte offset, computed
// once per block by stage_offsets: no address arithmetic between the barrier and the
// multiplies of a step.
__device__ __forceinline__ const void* uniform_ptr(const void* p) {
    const uint64_t v = (uint64_t)(uintptr_t)p;
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(v >> 32));
    return (const void*)(uintptr_t)(((uint64_t)hi << 32) | lo);
}

__device__ __forceinline__ void dma16_s(uint32_t voff, const void* sbase, uint32_t lds_base) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
                 :
                 : "v"(voff), "s"(sbase), "s"(lds_base)
                 : "memory");
}

// Per-lane byte offsets of stage_load's loads relative to element (row_base, k0) of a
// K-contiguous operand ([rows][ld]) or (k0, row_base) of a K-strided one ([K][ld]),
// with rows clamped as stage_load clamps them; row_base <= every clamped row.
template <int ROWS, bool KS, int NW, int KB>
__device__ __forceinline__ void stage_offsets(int64_t ld, int64_t rows, int64_t row0, int64_t row_base, int wave,
                                              int lane, uint32_t (&off)[ROWS * KB / (512 * NW)]) {
    constexpr int NI = ROWS * KB / (512 * NW);
#pragma unroll
    for (int j = 0; j < NI; ++j) {
        const int blk = wave * NI + j;
        if (!KS) {
            constexpr int CPR = KB / 8, RPB = 64 / CPR;
            const int r = blk * RPB + lane / CPR;
            const int kc = (lane % CPR) ^ kc_swz<KB>(r);
            int64_t gr = row0 + r;
            if (gr >= rows) gr = rows - 1;
            off[j] = (uint32_t)(((gr - row_base) * ld + kc * 8) * 2);
        } else {
            constexpr int RPB = ROWS == 256 ? 2 : (ROWS == 128 ? 4 : 8);
            constexpr int QPR = 64 / RPB;
            const int kr = blk * RPB + lane / QPR;
            const int q = lane % QPR;
            const int c = (q >> 1) ^ kstr_swz<ROWS>(kr);
            int64_t gr = row0 + c * 16 + (q & 1) * 8;
            if (gr >= rows) gr = (rows - 1) & ~(int64_t)7;
            off[j] = (uint32_t)((kr * ld + (gr - row_base)) * 2);
        }
    }
}

// MFMA fragment (16 rows x 32 k) of an operand tile at row offset rt, k offset ks.
template <int ROWS, bool KS, int KB>
__device__ __forceinline__ bf16x8_t load_frag(const bf16_t* lds, int rt, int ks, int lane) {
    const int i = lane & 15, g = lane >> 4;
    if (!KS) {
        const int r = rt + i;
        const int kc = ks / 8 + g;
        return __builtin_bit_cast(bf16x8_t, *(const u32x4_t*)(lds + r * KB + ((kc ^ kc_swz<KB>(r)) * 8)));
    } else {
        const int c = rt / 16;
        s16x4_t lo, hi;
        {
            const int kr = ks + 8 * g + (i >> 2);
            const int off = kr * ROWS + ((c ^ kstr_swz<ROWS>(kr)) * 16) + (i & 3) * 4;
            lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4_t*)(lds + off));
        }
        {
            const int kr = ks + 8 * g + 4 + (i >> 2);
            const int off = kr * ROWS + ((c ^ kstr_swz<ROWS>(kr)) * 16) + (i & 3) * 4;
            hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4_t*)(lds + off));
        }
        typedef short s16x8_t __attribute__((ext_vector_type(8)));
        const s16x8_t v = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
        return __builtin_bit_cast(bf16x8_t, v);
    }
}

typedef float f32x16_t __attribute__((ext_vector_type(16)));

__device__ __forceinline__ void wait_vmcnt(int n) {
    // s_waitcnt with vmcnt = n (n <= 63), expcnt and lgkmcnt left at their maxima
    switch (n) {
        case 0: __builtin_amdgcn_s_waitcnt(0 | (7 << 4) | (15 << 8)); break;
        case 2: __builtin_amdgcn_s_waitcnt(2 | (7 << 4) | (15 << 8)); break;
        case 4: __builtin_amdgcn_s_waitcnt(4 | (7 << 4) | (15 << 8)); break;
        case 6: __builtin_amdgcn_s_waitcnt(6 | (7 << 4) | (15 << 8)); break;
        case 8: __builtin_amdgcn_s_waitcnt(8 | (7 << 4) | (15 << 8)); break;
        case 12: __builtin_amdgcn_s_waitcnt(12 | (7 << 4) | (15 << 8)); break;
        case 16: __builtin_amdgcn_s_waitcnt(0 | (1 << 14) | (7 << 4) | (15 << 8)); break;
        default: __builtin_amdgcn_s_waitcnt(0 | (7 << 4) | (15 << 8)); break;
    }
}

__device__ __forceinline__ void wait_lgkm0() {
    // s_waitcnt lgkmcnt(0), vmcnt and expcnt left at their maxima
    __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4) | (0 << 8));
}

// The two MFMA shapes for bf16 or f16 operands (the same bit patterns either way: the
// LDS layout and fragment reads do not depend on the element type).
template <bool F16>
__device__ __forceinline__ f32x16_t mfma32x32x16(const bf16x8_t& b, const bf16x8_t& a, const f32x16_t& c) {
    if constexpr (F16)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, b), __builtin_bit_cast(half8_t, a),
                                                      c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(b, a, c, 0, 0, 0);
}
template <bool F16>
__device__ __forceinline__ f32x4_t mfma16x16x32(const bf16x8_t& b, const bf16x8_t& a, const f32x4_t& c) {
    if constexpr (F16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, b), __builtin_bit_cast(half8_t, a),
                                                      c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, a, c, 0, 0, 0);
}

// Fragments of 32 x 32 tiles (32 rows x 16 k, v_mfma_f32_32x32x16_bf16) by LDS byte address: lane
// l holds row l % 32 of the tile and the 8 k values 8 (l / 32) .. + 7 of the substep. K-strided
// operands use the transposing reads of load_frag, each 16-lane group G supplying row chunk
// G & 1 and k rows from 8 (G >> 1). Tile i of a wave and substep s differ from tile 0,
// substep 0 by an XOR of two address bits of the swizzled slot and by constants that go
// into the instruction's offset.
template <int ROWS, bool KS, int KB>
__device__ __forceinline__ uint32_t frag_base(const bf16_t* operand, int wrow, int lane) {
    if (!KS) {
        const int r = wrow + (lane & 31);
        return lds_addr(operand) + (uint32_t)(r * KB + (((lane >> 5) ^ kc_swz<KB>(r)) * 8)) * 2u;
    }
    const int i = lane & 15, G = lane >> 4, kr = 8 * (G >> 1) + (i >> 2), c = wrow / 16 + (G & 1);
    return lds_addr(operand) + (uint32_t)(kr * ROWS + ((c ^ kstr_swz<ROWS>(kr)) * 16) + (i & 3) * 4) * 2u;
}
template <int ROWS, bool KS, int KB>
__device__ __forceinline__ bf16x8_t frag_at(uint32_t base, uint32_t off, int i, int s) {
    if constexpr (!KS) {
        const uint32_t a = (base ^ (uint32_t)(s * 32)) + off + (uint32_t)(i * 32 * KB * 2);
        return __builtin_bit_cast(bf16x8_t, *(LDS_AS const u32x4_t*)a);
    } else {
        const uint32_t a = (base ^ (uint32_t)(i * 64)) + off + (uint32_t)(s * 16 * ROWS * 2);
        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4_t*)a);
        const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4_t*)(a + 4 * ROWS * 2));
        typedef short s16x8_t __attribute__((ext_vector_type(8)));
        const s16x8_t v = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
        return __builtin_bit_cast(bf16x8_t, v);
    }
}

}  // namespace

}  // namespace rdcn
