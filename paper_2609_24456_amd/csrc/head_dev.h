// Launch arguments of the projection-head kernels (k_head.hip).
#pragma once

#include "gemm_dev.h"
#include "softmax_dev.h"

namespace conduit {

constexpr int kHeadSplits = 128;  // most parts of dX's sum over the choices
constexpr int kHeadTwo = 128;     // most tokens whose logits' gradient is kept in two halves

struct HeadArgs {
    TokenShape shape;
    int64_t N, V, H;  // B * T tokens, choices, hidden units
    RowsView x;       // hidden states, as given
    GemmOperand X, W; // rows the product reads: as given, or packed
    int64_t K;        // columns of X and W the product takes (H, or H rounded up to 8 where packed)
    uint16_t* x_pack; // NULL: X is read where it is
    uint16_t* w_pack; // NULL: W is read where it is
    const uint16_t* w_src;
    int64_t w_ld;
    const int32_t* tokens;
    const uint8_t* mask;
    float c, inv_t;
    uint32_t* err;
    // with a mask: the tokens that count
    int32_t* list;
    int32_t* place;
    const uint32_t* count;
    uint32_t* count_out;
    // forward
    float* part;   // [tiles of choices][N][3]
    float* taken;  // [N]
    float* logp;
    float* lse;
    float* entropy;
    // backward
    const float* lse_in;
    const float* entropy_in;
    const float* g;
    const float* h;
    RowsView dx;
    uint16_t* dw;
    int64_t dw_ld;
    uint16_t* d;     // [d_rows][d_ld]: the logits' gradient of a chunk
    int64_t d_ld;
    int64_t d_rows;  // N, or 2 N: after the live tokens' rows come the rows of what their rounding left
    float* dx_part;  // [splits][d_rows][h_ld]
    float* dx_sum;   // [N][h_ld]
    int64_t h_ld;
    int64_t chunk;   // choices a pass
    int32_t splits, cus;
};

hipError_t launch_head_logprobs(HeadArgs a, hipStream_t s);
hipError_t launch_head_backward(HeadArgs a, hipStream_t s);

}  // namespace conduit
