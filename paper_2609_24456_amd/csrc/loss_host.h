// Host side of the calls on token batches (losses.hip, listed.hip): argument
// checks and the layout of workspaces.
#pragma once

#include <cmath>
#include <initializer_list>
#include <string>

#include "loss_dev.h"

namespace conduit {

inline conduit_status bad(const char* msg) { return report_error(CONDUIT_EINVAL, msg); }

inline conduit_status launched(hipError_t e, const char* what) {
    if (e == hipSuccess) return CONDUIT_OK;
    return report_error(CONDUIT_EDEVICE, (std::string(what) + ": " + hipGetErrorString(e)).c_str());
}

#define CONDUIT_TRY(call)                        \
    do {                                         \
        const conduit_status st_ = (call);       \
        if (st_ != CONDUIT_OK) return st_;       \
    } while (0)

constexpr int64_t kMaxTokens = (1ll << 31) - 1;
constexpr int64_t kMaxWidth = 1ll << 28;
constexpr int64_t kMaxStride = 1ll << 40;
constexpr int64_t kMaxReach = 1ll << 56;  // elements from an array's first to past its last: every offset in bytes fits 64 bits
constexpr int64_t kSplitRows = kPolicyBlocks;  // row tickets of a workspace (fewer rows than this are split)

// rows (b, t) of `width` elements, b < B and t < T, end within kMaxReach (counts and strides of at most 2^63, not negative)
inline bool within_reach(int64_t B, int64_t stride_b, int64_t T, int64_t stride_t, int64_t width) {
    if (B <= 0 || T <= 0) return true;
    return (__int128)(B - 1) * stride_b + (__int128)(T - 1) * stride_t + width <= kMaxReach;
}

inline conduit_status check_batch(int64_t B, int64_t T, int64_t stride) {
    if (B < 0 || T < 0) return bad("the number of sequences and of tokens must be >= 0");
    if (B > kMaxTokens || T > kMaxTokens || (B > 0 && T > kMaxTokens / B)) return bad("the batch must hold fewer than 2^31 tokens");
    if (stride < T || stride > kMaxStride) return bad("stride must be at least T (and at most 2^40)");
    if (!within_reach(B, stride, 1, 0, T)) return bad("the per-token arrays must end within 2^56 elements of their start");
    return CONDUIT_OK;
}

inline int elem_size(int32_t dtype) { return dtype == CONDUIT_BF16 ? 2 : 4; }

inline bool misaligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

// where a [B, T] set of rows of any dtype lies; `out`: it is written, so no two rows may share an element
inline conduit_status check_rows_layout(const conduit_rows* r, int64_t B, int64_t T, bool out, const std::string& w) {
    if (r->width < 1 || r->width > kMaxWidth) return bad((w + ": width must be in [1, 2^28]").c_str());
    if (r->stride_b < 0 || r->stride_t < 0 || r->stride_b > kMaxStride || r->stride_t > kMaxStride)
        return bad((w + ": strides must be in [0, 2^40]").c_str());
    if (B == 0 || T == 0) return CONDUIT_OK;
    if (!within_reach(B, r->stride_b, T, r->stride_t, r->width))
        return bad((w + ": rows must end within 2^56 elements of their start").c_str());
    if (!r->data) return bad((w + ": NULL data").c_str());
    if (misaligned(r->data, elem_size(r->dtype))) return bad((w + ": data must be aligned to its elements").c_str());
    if (out) {
        const int64_t row = T > 1 ? (T - 1) * r->stride_t + r->width : r->width;
        const int64_t seq = B > 1 ? (B - 1) * r->stride_b + r->width : r->width;
        const bool in_order = (T <= 1 || r->stride_t >= r->width) && (B <= 1 || r->stride_b >= row);
        const bool across = (B <= 1 || r->stride_b >= r->width) && (T <= 1 || r->stride_t >= seq);
        if (!in_order && !across) return bad((w + ": rows must not overlap").c_str());
    }
    return CONDUIT_OK;
}

// a [B, T] set of rows of floats
inline conduit_status check_rows(const conduit_rows* r, int64_t B, int64_t T, bool out, const char* what) {
    const std::string w(what);
    if (!r) return bad((w + " must not be NULL").c_str());
    if (r->dtype != CONDUIT_F32 && r->dtype != CONDUIT_BF16) return bad((w + ": dtype must be F32 or BF16").c_str());
    return check_rows_layout(r, B, T, out, w);
}

inline int64_t rows_extent(const conduit_rows* r, int64_t B, int64_t T) {
    return ((B - 1) * r->stride_b + (T - 1) * r->stride_t + r->width) * elem_size(r->dtype);
}

inline bool apart(const void* a, int64_t na, const void* b, int64_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x + (uintptr_t)na <= y || y + (uintptr_t)nb <= x;
}

// the gradient's rows: the logits themselves, or apart from them
inline conduit_status check_gradient_rows(const conduit_rows* x, const conduit_rows* dx, int64_t B, int64_t T) {
    CONDUIT_TRY(check_rows(dx, B, T, true, "dlogits"));
    if (dx->dtype != x->dtype || dx->width != x->width) return bad("dlogits must have the logits' dtype and width");
    if (B == 0 || T == 0) return CONDUIT_OK;
    const bool same = dx->data == x->data && (T <= 1 || dx->stride_t == x->stride_t) && (B <= 1 || dx->stride_b == x->stride_b);
    if (!same && !apart(x->data, rows_extent(x, B, T), dx->data, rows_extent(dx, B, T)))
        return bad("dlogits must be the logits themselves or apart from them");
    return CONDUIT_OK;
}

// Two per-token arrays of 4-byte elements with the call's stride: they share no
// element.  (Columns of one wider array may lie between each other's rows.)
inline bool tokens_apart(const void* a, const void* b, int64_t B, int64_t T, int64_t stride) {
    const int64_t n = ((B - 1) * stride + T) * 4;
    if (apart(a, n, b, n)) return true;
    if (B <= 1) return false;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    const int64_t d = (int64_t)((x > y ? x - y : y - x) % (uintptr_t)(stride * 4));
    return d >= T * 4 && stride * 4 - d >= T * 4;
}

// every output apart from the other outputs, from every input `ins` that it is not itself, and from the tokens
inline conduit_status check_outputs(std::initializer_list<const void*> outs, std::initializer_list<const void*> ins,
                             const int32_t* tokens, int64_t B, int64_t T, int64_t stride) {
    for (const void* o : outs)
        if (o && misaligned(o, 4)) return bad("per-token arrays must be aligned to their elements");
    for (const void* i : ins)
        if (i && misaligned(i, 4)) return bad("per-token arrays must be aligned to their elements");
    if (misaligned(tokens, 4)) return bad("per-token arrays must be aligned to their elements");
    if (B == 0 || T == 0) return CONDUIT_OK;
    for (auto o = outs.begin(); o != outs.end(); ++o) {
        if (!*o) continue;
        for (auto p = outs.begin(); p != o; ++p)
            if (*p && !tokens_apart(*o, *p, B, T, stride)) return bad("outputs overlap");
        for (const void* i : ins)
            if (i && i != *o && !tokens_apart(*o, i, B, T, stride)) return bad("an output overlaps an input");
        if (tokens && !tokens_apart(*o, tokens, B, T, stride)) return bad("an output overlaps the tokens");
    }
    return CONDUIT_OK;
}

inline conduit_status check_temperature(double t) {
    const float c = (float)((double)kLog2e / t), inv = (float)(1.0 / t);
    if (!(t > 0.0) || !std::isfinite(t) || !std::isfinite(c) || !(c > 1e-30f) || !(inv > 1e-30f))
        return bad("temperature must be a positive number");
    return CONDUIT_OK;
}

// The lowest logit whose product with inv_lo, what rounding 1 / temperature left, is a float: the type's lowest, or one
// whose score is past the largest float by far (times 1 / temperature, which is at least 2^23 times inv_lo).
inline float lowest_score(float inv_lo) {
    constexpr float kMost = 3.4028235e38f;
    return std::fabs(inv_lo) < 1.0f ? -kMost : -0.5f * kMost / std::fabs(inv_lo);
}

inline conduit_status check_workspace(const void* ws, uint64_t bytes, uint64_t need) {
    if (!ws) return bad("NULL workspace");
    if (misaligned(ws, 256)) return bad("the workspace must be 256-byte aligned");
    if (bytes < need) return bad("the workspace is smaller than the call needs");
    return CONDUIT_OK;
}

// ---------------------------------------------------------------------------
// workspaces: [head][row tickets][row counts][what one call leaves for its own
// next launch].  The head and the tickets are zero between calls; the counts are
// written whole before they are read.
// ---------------------------------------------------------------------------
inline uint64_t up(uint64_t x) { return (x + 255) / 256 * 256; }

struct Layout {
    uint64_t row_ticket, row_count, rest, bytes;
};

inline Layout layout(int64_t B, uint64_t rest) {
    Layout l;
    l.row_ticket = sizeof(WorkspaceHead);
    l.row_count = l.row_ticket + 4 * kTicketStep * kSplitRows;
    l.rest = l.row_count + up(4 * (uint64_t)B);
    l.bytes = l.rest + up(rest);
    return l;
}

inline RowsView view(const conduit_rows* r) { return RowsView{r->data, r->stride_b, r->stride_t}; }

}  // namespace conduit
