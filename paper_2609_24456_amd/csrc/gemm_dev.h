// The matrix product of the projection head (k_head.hip): C[m][n] = sum_k
// A[m][k] B[n][k] of two bf16 operands whose rows are contiguous in k, fp32
// accumulation on the matrix cores, 256 x 256 of C a workgroup.
//
// Eight wavefronts in two groups of four: group wm holds rows wm * 128 .. + 128
// of C, its wavefront wn columns wn * 64 .. + 64, as 8 x 4 tiles of
// v_mfma_f32_16x16x32_bf16 (128 accumulator registers a lane).  A step of 64 k
// is four phases, each a quarter of the wavefront's tile (16 instructions):
//     phase 0: rows half 0, columns half 0      1: half 0, half 1
//           2: half 1, half 0                   3: half 1, half 1
// A phase first reads from LDS what it needs anew (A half 0 / B half 1 / A half
// 1 / B half 0 of the next step: 8, 4, 8, 4 reads of 16 bytes a lane), starts
// the copy of one half of one operand (128 rows x 64 k) from memory into LDS
// for two steps on, then, after a barrier, multiplies.  Group 1 runs one
// barrier behind group 0, so on every SIMD one wavefront multiplies while the
// other reads.  LDS holds two steps (128 KB); a half is copied over as soon as
// both groups have read it, six phases before its next use, and is waited for
// with a count of the younger copies in flight, never by draining them.
//
// LDS rows are 128 bytes; the 16-byte piece c of row r lies at piece
// c ^ (r & 7), so the 16 rows that an MFMA operand reads at one k fall on
// different banks.  The copies go straight to LDS (lane l fills bytes 16 l of
// eight rows), so the permutation is made in the address that a lane reads.
// Rows beyond the operand and k beyond its end read as zeros: their lanes' byte
// offset lies outside the buffer descriptor's range.
//
// Who needs what is arranged as follows, P(t, p) being phase p of step t: the
// piece copied in P(t, p) overwrites one that was last read in the phase
// before; all reads of a phase are complete before its first barrier.  What a
// phase reads was waited for by every wavefront in the phase before it, ahead
// of that phase's first barrier.  Both hold for either group, since group 1's
// reads of a phase end at the barrier at which group 0 ends the same phase.
#pragma once

#include "common.h"

namespace conduit {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kGemmTile = 256;      // rows and columns of C a workgroup
constexpr int kGemmK = 64;          // k a step
constexpr int kGemmThreads = 512;
constexpr int kGemmLds = 131072;    // bytes: two steps of (256 + 256) rows x 128
constexpr int kGemmStep = 65536;    // bytes of one step
constexpr uint32_t kGemmOut = 0x80000000u;  // a byte offset outside every descriptor's range

struct GemmOperand {
    const uint16_t* p;  // bf16 bits, 16-byte aligned
    int64_t ld;         // elements from row to row, a multiple of 8, at most 2^21
};

// acc[mi][ni][i] = C[row0 + wm 128 + mi 16 + 4 (lane / 16) + i][col0 + wn 64 + ni 16 + lane % 16]
struct GemmAcc {
    f32x4_t c[8][4];
};

typedef __attribute__((address_space(3))) uint8_t lds_u8;

#define GEMM_READ8(r, a0, a1, off)                                                                      \
    asm volatile("ds_read_b128 %0, %8 offset:%10\n\tds_read_b128 %1, %9 offset:%10\n\t"                 \
                 "ds_read_b128 %2, %8 offset:%11\n\tds_read_b128 %3, %9 offset:%11\n\t"                 \
                 "ds_read_b128 %4, %8 offset:%12\n\tds_read_b128 %5, %9 offset:%12\n\t"                 \
                 "ds_read_b128 %6, %8 offset:%13\n\tds_read_b128 %7, %9 offset:%13\n\t"                 \
                 "s_waitcnt vmcnt(12) lgkmcnt(0)"                                                       \
                 : "=&v"(r[0][0]), "=&v"(r[0][1]), "=&v"(r[1][0]), "=&v"(r[1][1]), "=&v"(r[2][0]),      \
                   "=&v"(r[2][1]), "=&v"(r[3][0]), "=&v"(r[3][1])                                       \
                 : "v"(a0), "v"(a1), "n"(off), "n"((off) + 2048), "n"((off) + 4096), "n"((off) + 6144) \
                 : "memory")

#define GEMM_READ4(r, a0, a1, off)                                                              \
    asm volatile("ds_read_b128 %0, %4 offset:%6\n\tds_read_b128 %1, %5 offset:%6\n\t"           \
                 "ds_read_b128 %2, %4 offset:%7\n\tds_read_b128 %3, %5 offset:%7\n\t"           \
                 "s_waitcnt vmcnt(12) lgkmcnt(0)"                                               \
                 : "=&v"(r[0][0]), "=&v"(r[0][1]), "=&v"(r[1][0]), "=&v"(r[1][1])               \
                 : "v"(a0), "v"(a1), "n"(off), "n"((off) + 2048)                                \
                 : "memory")

__device__ __forceinline__ void gemm_barrier() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

template <int H, int G>
__device__ __forceinline__ void gemm_multiply(GemmAcc& acc, const u32x4_t (&a)[4][2], const u32x4_t (&b)[2][2]) {
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                acc.c[H * 4 + i][G * 2 + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    __builtin_bit_cast(bf16x8, a[i][k]), __builtin_bit_cast(bf16x8, b[j][k]), acc.c[H * 4 + i][G * 2 + j],
                    0, 0, 0);
            }
        }
    }
    __builtin_amdgcn_s_setprio(0);
}

// C of rows row0.. of A (of `rows` in all) and col0.. of B (of `cols`), over k
// in [64 step0, min(64 step1, K)); K and 64 step0 count elements of a row, K is
// a multiple of 8 or its operands hold zeros up to one.  `lds` holds kGemmLds
// bytes, free again for the caller when every wavefront has returned and met a
// barrier.
__device__ __forceinline__ void gemm_tile(const GemmOperand& A, int64_t row0, int64_t rows, const GemmOperand& B,
                                          int64_t col0, int64_t cols, int64_t K, int32_t step0, int32_t step1,
                                          uint8_t* lds, GemmAcc& acc) {
    const int lane = lane_id(), w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), wm = w / 4, wn = w % 4;
    const int piece = (lane % 8) ^ (lane / 8);
    __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint16_t*>(A.p + row0 * A.ld + (int64_t)step0 * kGemmK), 0, 0x7fffffff, 0x00027000);
    __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint16_t*>(B.p + col0 * B.ld + (int64_t)step0 * kGemmK), 0, 0x7fffffff, 0x00027000);
    // this lane's byte offsets within the operands' tiles: [half][issue]
    uint32_t va[2][2], vb[2][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = h * 64 + w * 8 + i * 128 + lane / 8;
            const int c = (w / 4) * 64 + h * 32 + (w % 4) * 8 + i * 128 + lane / 8;
            va[h][i] = row0 + r < rows ? (uint32_t)(r * A.ld * 2 + piece * 16) : kGemmOut;
            vb[h][i] = col0 + c < cols ? (uint32_t)(c * B.ld * 2 + piece * 16) : kGemmOut;
        }
    }
    const int32_t steps = step1 - step0;
    // k of this lane's piece in step t is valid below this many steps (of k) on
    const int64_t kleft = (K < (int64_t)step1 * kGemmK ? K : (int64_t)step1 * kGemmK) - (int64_t)step0 * kGemmK - piece * 8;
    const int32_t last = (int32_t)((kleft + kGemmK - 1) / kGemmK);  // steps in which the piece exists
    auto stage_a = [&](int h, int32_t t) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_u8*)lds + (t & 1) * kGemmStep + (h * 64 + w * 8 + i * 128) * 128,
                                                     16, t < last ? va[h][i] : kGemmOut, t * (kGemmK * 2), 0, 0);
    };
    auto stage_b = [&](int h, int32_t t) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rb, (lds_u8*)lds + (t & 1) * kGemmStep + 32768 + ((w / 4) * 64 + h * 32 + (w % 4) * 8 + i * 128) * 128, 16,
                t < last ? vb[h][i] : kGemmOut, t * (kGemmK * 2), 0, 0);
    };
    const uint32_t base = (uint32_t)(uintptr_t)(lds_u8*)lds;
    const uint32_t frag = (lane % 16) * 128 + (((lane / 16) ^ (lane & 7)) * 16);
    uint32_t a0 = base + wm * 16384 + frag, b0 = base + 32768 + wn * 8192 + frag;
    uint32_t a1 = base + wm * 16384 + (frag ^ 64), b1 = base + 32768 + wn * 8192 + (frag ^ 64);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) acc.c[i][j] = f32x4_t{0, 0, 0, 0};
    }
    u32x4_t a[4][2], bl[2][2], bh[2][2];
    stage_b(0, 0);
    stage_a(0, 0);
    stage_b(1, 0);
    stage_a(1, 0);
    stage_b(0, 1);
    stage_a(0, 1);
    stage_b(1, 1);
    stage_a(1, 1);
    asm volatile("s_waitcnt vmcnt(12)" ::: "memory");
    gemm_barrier();
    GEMM_READ4(bl, b0, b1, 0);
    if (wm == 1) gemm_barrier();  // group 1 runs one barrier behind
    for (int32_t t = 0; t < steps; ++t) {
        // (0, 0)
        stage_b(0, t + 2);
        GEMM_READ8(a, a0, a1, 0);
        gemm_barrier();
        gemm_multiply<0, 0>(acc, a, bl);
        gemm_barrier();
        // (0, 1)
        stage_a(0, t + 2);
        GEMM_READ4(bh, b0, b1, 4096);
        gemm_barrier();
        gemm_multiply<0, 1>(acc, a, bh);
        gemm_barrier();
        // (1, 0)
        stage_b(1, t + 2);
        GEMM_READ8(a, a0, a1, 8192);
        gemm_barrier();
        gemm_multiply<1, 0>(acc, a, bl);
        gemm_barrier();
        // (1, 1), and the next step's columns half 0
        const uint32_t next = (t & 1) ? 0u - kGemmStep : kGemmStep;
        a0 += next;
        a1 += next;
        b0 += next;
        b1 += next;
        stage_a(1, t + 2);
        GEMM_READ4(bl, b0, b1, 0);
        gemm_barrier();
        gemm_multiply<1, 1>(acc, a, bh);
        gemm_barrier();
    }
    if (wm == 0) gemm_barrier();
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the copies beyond the last step
    gemm_barrier();
}

}  // namespace conduit
