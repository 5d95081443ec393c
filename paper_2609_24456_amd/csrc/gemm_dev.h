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
//
// A transposed operand is copied as it stands, each half as 64 rows (k) of 128
// columns (256 bytes), and turned on the way out of LDS: ds_read_b64_tr_b16 lets
// 16 lanes read 4 rows of 16 columns, 8 bytes each, and hands lane c the four
// values of column c, so two of them make a lane's 8 k of an MFMA operand.  The
// four rows of one such read, and those of the next 16 lanes, lie on different
// banks: the 32-byte piece c of row k lies at piece c ^ (k % 4 + 4 (k / 8 % 2)).
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

#include <type_traits>

#include "common.h"

namespace conduit {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

constexpr int kGemmTile = 256;      // rows and columns of C a workgroup
constexpr int kGemmK = 64;          // k a step
constexpr int kGemmThreads = 512;
constexpr int kGemmLds = 131072;    // bytes: two steps of (256 + 256) rows x 128
constexpr int kGemmStep = 65536;    // bytes of one step
constexpr uint32_t kGemmOut = 0x80000000u;  // a byte offset outside every descriptor's range

// An operand stands in memory by rows of k, p[row * ld + k], or, in the
// transposed form (TA, TB below), by rows of rows: p[k * ld + row].
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

// 16 (8) reads that turn: for each of 4 (2) addresses k 0-3, 4-7, 32-35, 36-39 of
// the lane's group, the halves of the two steps' operands
#define GEMM_TURN16(r, a, off)                                                                             \
    asm volatile("ds_read_b64_tr_b16 %0, %16 offset:%20\n\tds_read_b64_tr_b16 %1, %16 offset:%21\n\t"      \
                 "ds_read_b64_tr_b16 %2, %16 offset:%22\n\tds_read_b64_tr_b16 %3, %16 offset:%23\n\t"      \
                 "ds_read_b64_tr_b16 %4, %17 offset:%20\n\tds_read_b64_tr_b16 %5, %17 offset:%21\n\t"      \
                 "ds_read_b64_tr_b16 %6, %17 offset:%22\n\tds_read_b64_tr_b16 %7, %17 offset:%23\n\t"      \
                 "ds_read_b64_tr_b16 %8, %18 offset:%20\n\tds_read_b64_tr_b16 %9, %18 offset:%21\n\t"      \
                 "ds_read_b64_tr_b16 %10, %18 offset:%22\n\tds_read_b64_tr_b16 %11, %18 offset:%23\n\t"    \
                 "ds_read_b64_tr_b16 %12, %19 offset:%20\n\tds_read_b64_tr_b16 %13, %19 offset:%21\n\t"    \
                 "ds_read_b64_tr_b16 %14, %19 offset:%22\n\tds_read_b64_tr_b16 %15, %19 offset:%23\n\t"    \
                 "s_waitcnt vmcnt(12) lgkmcnt(0)"                                                          \
                 : "=&v"(r[0][0].lo), "=&v"(r[0][0].hi), "=&v"(r[0][1].lo), "=&v"(r[0][1].hi),             \
                   "=&v"(r[1][0].lo), "=&v"(r[1][0].hi), "=&v"(r[1][1].lo), "=&v"(r[1][1].hi),             \
                   "=&v"(r[2][0].lo), "=&v"(r[2][0].hi), "=&v"(r[2][1].lo), "=&v"(r[2][1].hi),             \
                   "=&v"(r[3][0].lo), "=&v"(r[3][0].hi), "=&v"(r[3][1].lo), "=&v"(r[3][1].hi)              \
                 : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "n"(off), "n"((off) + 1024),                \
                   "n"((off) + 8192), "n"((off) + 9216)                                                    \
                 : "memory")

#define GEMM_TURN8(r, a, off)                                                                              \
    asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%10\n\tds_read_b64_tr_b16 %1, %8 offset:%11\n\t"        \
                 "ds_read_b64_tr_b16 %2, %8 offset:%12\n\tds_read_b64_tr_b16 %3, %8 offset:%13\n\t"        \
                 "ds_read_b64_tr_b16 %4, %9 offset:%10\n\tds_read_b64_tr_b16 %5, %9 offset:%11\n\t"        \
                 "ds_read_b64_tr_b16 %6, %9 offset:%12\n\tds_read_b64_tr_b16 %7, %9 offset:%13\n\t"        \
                 "s_waitcnt vmcnt(12) lgkmcnt(0)"                                                          \
                 : "=&v"(r[0][0].lo), "=&v"(r[0][0].hi), "=&v"(r[0][1].lo), "=&v"(r[0][1].hi),             \
                   "=&v"(r[1][0].lo), "=&v"(r[1][0].hi), "=&v"(r[1][1].lo), "=&v"(r[1][1].hi)              \
                 : "v"(a[0]), "v"(a[1]), "n"(off), "n"((off) + 1024), "n"((off) + 8192), "n"((off) + 9216) \
                 : "memory")

// a lane's 8 values of one MFMA operand, read whole or in two halves
struct GemmPair {
    u32x2_t lo, hi;
};
__device__ __forceinline__ bf16x8 gemm_operand(const u32x4_t& x) { return __builtin_bit_cast(bf16x8, x); }
__device__ __forceinline__ bf16x8 gemm_operand(const GemmPair& x) {
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(x.lo, x.hi, 0, 1, 2, 3));
}

__device__ __forceinline__ void gemm_barrier() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

template <int H, int G, typename FA, typename FB>
__device__ __forceinline__ void gemm_multiply(GemmAcc& acc, const FA (&a)[4][2], const FB (&b)[2][2]) {
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                acc.c[H * 4 + i][G * 2 + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    gemm_operand(a[i][k]), gemm_operand(b[j][k]), acc.c[H * 4 + i][G * 2 + j], 0, 0, 0);
            }
        }
    }
    __builtin_amdgcn_s_setprio(0);
}

// One operand's side of a tile: how its halves are copied and read.  A: rows
// wm * 128 + half * 64 .. + 64 of 256 for group wm; B: wn * 64 + half * 32 .. + 32
// for wavefront wn of a group.
template <bool B, bool TURN>
struct GemmSide {
    static constexpr int kSpan = B ? 32 : 64;  // consecutive rows of one wavefront's part of a half
    static constexpr uint32_t kBase = B ? 32768 : 0;
    const uint16_t* p;  // first row (or column), k = 0 of the first step
    int64_t ld;
    uint32_t off[2][2];  // this lane's byte offsets from p, per half and issue
    int32_t last[2];     // steps in which the lane's piece of an issue exists
    int32_t w;

    // place of row r (0..127) of half h among the tile's 256
    static __device__ __forceinline__ int row_of(int r, int h) { return r / kSpan * 2 * kSpan + h * kSpan + r % kSpan; }

    // rows row0 .. of `rows`; kleft: k from the first step on that exist
    __device__ __forceinline__ void init(const GemmOperand& o, int64_t row0, int64_t rows, int32_t step0, int64_t kleft) {
        const int lane = lane_id();
        w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        ld = o.ld;
        if constexpr (!TURN) {
            p = o.p + row0 * o.ld + (int64_t)step0 * kGemmK;
            const int piece = (lane % 8) ^ (lane / 8);
            last[0] = last[1] = (int32_t)((kleft - piece * 8 + kGemmK - 1) / kGemmK);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int r = row_of(w * 8 + i * 64 + lane / 8, h);
                    off[h][i] = row0 + r < rows ? (uint32_t)(r * o.ld * 2 + piece * 16) : kGemmOut;
                }
            }
        } else {
            p = o.p + (int64_t)step0 * kGemmK * o.ld + row0;
            const int turn = lane / 16 + 4 * (w / 2 % 2);
            const int r = (((lane % 16) / 2) ^ turn) * 16 + lane % 2 * 8;  // first of the lane's 8 rows in a half
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int k = (w + 8 * i) * 4 + lane / 16;
                last[i] = (int32_t)((kleft - k + kGemmK - 1) / kGemmK);
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    off[h][i] = row0 + row_of(r, h) < rows ? (uint32_t)(k * o.ld * 2 + row_of(r, h) * 2) : kGemmOut;
            }
        }
    }

    // start the copy of half h of step t
    __device__ __forceinline__ void stage(uint8_t* lds, int h, int32_t t) const {
        __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<uint16_t*>(TURN ? p + (int64_t)t * kGemmK * ld : p), 0, 0x7fffffff, 0x00027000);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t to = TURN ? h * 16384 + (w + 8 * i) * 1024 : row_of(w * 8 + i * 64, h) * 128;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_u8*)lds + (t & 1) * kGemmStep + kBase + to, 16,
                                                     t < last[i] ? off[h][i] : kGemmOut, TURN ? 0 : t * (kGemmK * 2), 0, 0);
        }
    }
};

// The tiles of a workgroup, one after the other: start() sets a tile and starts
// the copies of its first two steps, which then run under the caller's work on
// the tile before; run() multiplies.
//
// C of rows row0.. of A (of `rows` in all) and col0.. of B (of `cols`), over k in
// [64 step0, min(64 step1, K)); where an operand stands by rows of k, K is a
// multiple of 8 or the row holds zeros up to one; where it is transposed, rows
// (cols) is, or the rows hold as many more elements.  `lds`, kGemmLds bytes, is
// this object's alone.
template <bool TA, bool TB>
struct GemmTiles {
    GemmSide<false, TA> sa;
    GemmSide<true, TB> sb;
    int32_t steps;
    uint8_t* lds;

    __device__ __forceinline__ void start(const GemmOperand& A, int64_t row0, int64_t rows, const GemmOperand& B, int64_t col0,
                                          int64_t cols, int64_t K, int32_t step0, int32_t step1) {
        steps = step1 - step0;
        const int64_t kleft = (K < (int64_t)step1 * kGemmK ? K : (int64_t)step1 * kGemmK) - (int64_t)step0 * kGemmK;
        sa.init(A, row0, rows, step0, kleft);
        sb.init(B, col0, cols, step0, kleft);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            sb.stage(lds, 0, t);
            sa.stage(lds, 0, t);
            sb.stage(lds, 1, t);
            sa.stage(lds, 1, t);
        }
    }

    // (What the caller has loaded or stored since start() only makes the counted
    // waits stricter: the copies among themselves end in order.)
    __device__ __forceinline__ void run(GemmAcc& acc) {
        const int lane = lane_id(), w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), wm = w / 4, wn = w % 4;
        // what this lane reads: [two steps of 32 k], or per 16 rows
        const uint32_t base = (uint32_t)(uintptr_t)(lds_u8*)lds;
        uint32_t aa[TA ? 4 : 2], ab[2];
        const uint32_t frag = (lane % 16) * 128 + (((lane / 16) ^ (lane & 7)) * 16);
        const uint32_t trow = (lane / 16 * 8 + lane % 16 / 4) * 256 + lane % 4 * 8, turn = lane % 16 / 4 + 4 * (lane / 16 % 2);
        if constexpr (TA) {
#pragma unroll
            for (int i = 0; i < 4; ++i) aa[i] = base + trow + ((wm * 4 + i) ^ turn) * 32;
        } else {
            aa[0] = base + wm * 16384 + frag;
            aa[1] = base + wm * 16384 + (frag ^ 64);
        }
        if constexpr (TB) {
#pragma unroll
            for (int i = 0; i < 2; ++i) ab[i] = base + 32768 + trow + ((wn * 2 + i) ^ turn) * 32;
        } else {
            ab[0] = base + 32768 + wn * 8192 + frag;
            ab[1] = base + 32768 + wn * 8192 + (frag ^ 64);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
#pragma unroll
            for (int j = 0; j < 4; ++j) acc.c[i][j] = f32x4_t{0, 0, 0, 0};
        }
        typedef typename std::conditional<TA, GemmPair, u32x4_t>::type FA;
        typedef typename std::conditional<TB, GemmPair, u32x4_t>::type FB;
        FA a[4][2];
        FB bl[2][2], bh[2][2];
        // (macros: the offsets are the instructions' own)
#define GEMM_READ_A(h)                                     \
    do {                                                   \
        if constexpr (TA) GEMM_TURN16(a, aa, (h) * 16384); \
        else GEMM_READ8(a, aa[0], aa[1], (h) * 8192);      \
    } while (0)
#define GEMM_READ_B(r, h)                                  \
    do {                                                   \
        if constexpr (TB) GEMM_TURN8(r, ab, (h) * 16384);  \
        else GEMM_READ4(r, ab[0], ab[1], (h) * 4096);      \
    } while (0)
        asm volatile("s_waitcnt vmcnt(12)" ::: "memory");
        gemm_barrier();
        GEMM_READ_B(bl, 0);
        if (wm == 1) gemm_barrier();  // group 1 runs one barrier behind
        for (int32_t t = 0; t < steps; ++t) {
            // (0, 0)
            sb.stage(lds, 0, t + 2);
            GEMM_READ_A(0);
            gemm_barrier();
            gemm_multiply<0, 0>(acc, a, bl);
            gemm_barrier();
            // (0, 1)
            sa.stage(lds, 0, t + 2);
            GEMM_READ_B(bh, 1);
            gemm_barrier();
            gemm_multiply<0, 1>(acc, a, bh);
            gemm_barrier();
            // (1, 0)
            sb.stage(lds, 1, t + 2);
            GEMM_READ_A(1);
            gemm_barrier();
            gemm_multiply<1, 0>(acc, a, bl);
            gemm_barrier();
            // (1, 1), and the next step's columns half 0
            const uint32_t next = (t & 1) ? 0u - kGemmStep : kGemmStep;
#pragma unroll
            for (int i = 0; i < (TA ? 4 : 2); ++i) aa[i] += next;
#pragma unroll
            for (int i = 0; i < 2; ++i) ab[i] += next;
            sa.stage(lds, 1, t + 2);
            GEMM_READ_B(bl, 0);
            gemm_barrier();
            gemm_multiply<1, 1>(acc, a, bh);
            gemm_barrier();
        }
        if (wm == 0) gemm_barrier();
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the copies beyond the last step
        gemm_barrier();
#undef GEMM_READ_A
#undef GEMM_READ_B
    }
};

}  // namespace conduit
