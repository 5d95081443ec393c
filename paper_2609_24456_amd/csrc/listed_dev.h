// Launch arguments of the kernels on listed choices (k_top.hip, k_listed.hip).
#pragma once

#include "softmax_dev.h"

namespace conduit {

// Logits of more bytes are read and gradients written past the caches: half as much
// again as the last level holds (256 MB), since up to there the next reader finds part.
constexpr int64_t kPastBytes = 384 << 20;
constexpr int kMostListed = 128;      // choices a token
constexpr int kPartVectors = 32768;   // most vectors of a part of a row: its LDS grows with them

// how a call's rows are split: parts of `per` vectors
struct RowParts {
    int32_t parts, per;
};
RowParts top_parts(int64_t rows, int64_t V, bool bf16);
RowParts listed_parts(int64_t rows, int64_t V, bool bf16, bool whole_rows);
int64_t gradient_parts(int64_t V, bool bf16);  // wavefronts that a row's gradient takes where it has a launch of its own

// The K most probable choices of every token.
struct TopArgs {
    TokenShape shape;
    RowsView x;
    int64_t V;
    float c, inv_t, inv_lo;  // as in LogitsArgs
    bool once;               // the logits are read past the caches (rows_dev.h)
    const int32_t* tokens;   // NULL: no taken token
    const uint8_t* mask;
    RowsView ids, logps;
    int32_t K;
    float* logp;
    float* lse;
    float* entropy;
    uint32_t* err;
    // split rows: statistics and K keys of each part of a row
    int32_t parts;
    int32_t per;  // vectors a part, a multiple of 8
    Div31 by_parts;
    float* part;
    uint64_t* key;
    uint32_t* row_ticket;  // NULL: a second launch joins the parts
};

hipError_t launch_token_alternatives(const TopArgs& a, bool bf16, hipStream_t s);

// The row of a token as its listed choices and the others make it, for the
// gradient: dx_j = coef 2^(c (x_j - base)) for the others, and of a listed one
// by its own and the teacher's probability.
struct ListedRow {
    float base, coef;
    float top, log_s;   // log p = (x - top) / temperature - log_s
    float q_top, q_log; // log q = (y - q_top) / teacher's temperature - q_log
    float loss, over, w;
};

// who adds up the rows' parts in the loss: a launch over the tokens, the rows themselves (the last one's wavefront), or,
// of split rows, the gradient's launch
enum ListedSums : int32_t { SUM_LAUNCH, SUM_ROWS, SUM_NEXT };

struct ListedArgs {
    TokenShape shape;
    RowsView x, dx;
    int64_t V;
    float c, inv_t, inv_lo, lowest;
    bool once;  // as in TopArgs
    const uint8_t* mask;
    RowsView ids;
    int32_t K;
    uint32_t* err;
    // log-probabilities
    RowsView logps;
    float* rest;
    float* lse;
    // their gradient
    const float* lse_in;
    const float* rest_in;
    RowsView g;
    const float* h;
    // distillation
    RowsView teacher;
    float q_inv_t;
    bool reverse, with_rest, has_dx;
    bool past;  // the gradient is written past the caches (rows_dev.h)
    int32_t reduction;
    double scale;
    const float* weight;
    float* loss;
    float* stats;
    WorkspaceHead* head;
    uint32_t* row_count;
    double* partial;  // [kPolicyBlocks][2]
    int32_t sums;     // SUM_...
    bool counted;     // a launch before counts the tokens
    bool flat_mask;   // in one piece, at a multiple of 16 bytes
    // split rows
    int32_t parts, per;
    Div31 by_parts;
    float* part;           // [rows][parts][3]
    ListedRow* row;        // [rows]
    uint32_t* row_ticket;  // NULL: a second launch joins the parts
};

constexpr int64_t kCountedHere = 1024;  // most tokens that each row counts for itself
constexpr int64_t kCountedFlat = 2048;  // of a mask in one piece
constexpr int kDistillSums = 2;         // weighted and plain divergence

hipError_t launch_listed_logprobs(const ListedArgs& a, bool bf16, hipStream_t s);
hipError_t launch_listed_logprobs_backward(const ListedArgs& a, bool bf16, hipStream_t s);
hipError_t launch_distill_loss(const ListedArgs& a, bool bf16, hipStream_t s);

// ---------------------------------------------------------------------------
// device code of both
// ---------------------------------------------------------------------------
// Orders LDS accesses of a wavefront's lanes: what they wrote before is what
// they read after.
__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The first lane's value, in every lane.  Sums over lanes of products may be
// contracted to one's own product and the rounded other, and then differ from lane
// to lane in the last place: who writes a value must not depend on which lane it
// fell to.
__device__ __forceinline__ float uniform(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x)));
}

__device__ __forceinline__ uint64_t below_lane() { return (1ull << lane_id()) - 1; }

}  // namespace conduit
