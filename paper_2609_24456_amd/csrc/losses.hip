// Host side of the token log-probability and loss calls of include/conduit.h:
// argument checks, the layout of their workspaces, and the launches.
#include <cmath>
#include <initializer_list>
#include <string>

#include "head_dev.h"

using namespace conduit;

namespace {

conduit_status bad(const char* msg) { return report_error(CONDUIT_EINVAL, msg); }

conduit_status launched(hipError_t e, const char* what) {
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
bool within_reach(int64_t B, int64_t stride_b, int64_t T, int64_t stride_t, int64_t width) {
    if (B <= 0 || T <= 0) return true;
    return (__int128)(B - 1) * stride_b + (__int128)(T - 1) * stride_t + width <= kMaxReach;
}

conduit_status check_batch(int64_t B, int64_t T, int64_t stride) {
    if (B < 0 || T < 0) return bad("the number of sequences and of tokens must be >= 0");
    if (B > kMaxTokens || T > kMaxTokens || (B > 0 && T > kMaxTokens / B)) return bad("the batch must hold fewer than 2^31 tokens");
    if (stride < T || stride > kMaxStride) return bad("stride must be at least T (and at most 2^40)");
    if (!within_reach(B, stride, 1, 0, T)) return bad("the per-token arrays must end within 2^56 elements of their start");
    return CONDUIT_OK;
}

int elem_size(int32_t dtype) { return dtype == CONDUIT_F32 ? 4 : 2; }

bool misaligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

// a [B, T] set of rows; `out`: it is written, so no two rows may share an element
conduit_status check_rows(const conduit_rows* r, int64_t B, int64_t T, bool out, const char* what) {
    const std::string w(what);
    if (!r) return bad((w + " must not be NULL").c_str());
    if (r->dtype != CONDUIT_F32 && r->dtype != CONDUIT_BF16) return bad((w + ": dtype must be F32 or BF16").c_str());
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

int64_t rows_extent(const conduit_rows* r, int64_t B, int64_t T) {
    return ((B - 1) * r->stride_b + (T - 1) * r->stride_t + r->width) * elem_size(r->dtype);
}

bool apart(const void* a, int64_t na, const void* b, int64_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x + (uintptr_t)na <= y || y + (uintptr_t)nb <= x;
}

// the gradient's rows: the logits themselves, or apart from them
conduit_status check_gradient_rows(const conduit_rows* x, const conduit_rows* dx, int64_t B, int64_t T) {
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
bool tokens_apart(const void* a, const void* b, int64_t B, int64_t T, int64_t stride) {
    const int64_t n = ((B - 1) * stride + T) * 4;
    if (apart(a, n, b, n)) return true;
    if (B <= 1) return false;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    const int64_t d = (int64_t)((x > y ? x - y : y - x) % (uintptr_t)(stride * 4));
    return d >= T * 4 && stride * 4 - d >= T * 4;
}

// every output apart from the other outputs, from every input `ins` that it is not itself, and from the tokens
conduit_status check_outputs(std::initializer_list<const void*> outs, std::initializer_list<const void*> ins,
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

conduit_status check_temperature(double t) {
    const float c = (float)((double)kLog2e / t), inv = (float)(1.0 / t);
    if (!(t > 0.0) || !std::isfinite(t) || !std::isfinite(c) || !(c > 1e-30f) || !(inv > 1e-30f))
        return bad("temperature must be a positive number");
    return CONDUIT_OK;
}

conduit_status check_workspace(const void* ws, uint64_t bytes, uint64_t need) {
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
uint64_t up(uint64_t x) { return (x + 255) / 256 * 256; }

struct Layout {
    uint64_t row_ticket, row_count, rest, bytes;
};

Layout layout(int64_t B, uint64_t rest) {
    Layout l;
    l.row_ticket = sizeof(WorkspaceHead);
    l.row_count = l.row_ticket + 4 * kTicketStep * kSplitRows;
    l.rest = l.row_count + up(4 * (uint64_t)B);
    l.bytes = l.rest + up(rest);
    return l;
}

Layout policy_layout(int64_t B) { return layout(B, sizeof(double) * kPolicySums * kPolicyBlocks); }

// split rows: their parts' statistics, and what the rows' gradients need of them, behind the partial sums
Layout logits_layout(int64_t B, int64_t T, const conduit_rows* x) {
    const int64_t rows = B * T, parts = logits_parts(rows, x->width, x->dtype == CONDUIT_BF16);
    return layout(B, sizeof(double) * kPolicySums * kPolicyBlocks + (parts > 1 ? (uint64_t)rows * (12 * parts + sizeof(SplitRow)) : 0));
}

Layout preference_layout(int64_t P, int64_t T) {
    return layout(0, sizeof(double) * (4 * (uint64_t)P + 4 * (uint64_t)P * preference_parts(P, T)));
}

void place_workspace(PolicyArgs& p, void* ws, const Layout& l) {
    uint8_t* w = static_cast<uint8_t*>(ws);
    p.head = reinterpret_cast<WorkspaceHead*>(w);
    p.row_count = reinterpret_cast<uint32_t*>(w + l.row_count);
    p.partial = reinterpret_cast<double*>(w + l.rest);
}

void place_workspace(LogitsArgs& a, void* ws, const Layout& l) {
    uint8_t* w = static_cast<uint8_t*>(ws);
    const int64_t rows = a.shape.B * a.shape.T;
    a.row_ticket = reinterpret_cast<uint32_t*>(w + l.row_ticket);
    a.part = reinterpret_cast<float*>(w + l.rest + sizeof(double) * kPolicySums * kPolicyBlocks);
    a.split = reinterpret_cast<SplitRow*>(a.part + 3 * rows * a.parts);
}

conduit_status policy_terms(const conduit_policy_opts* o, PolicyTerms* t) {
    if (!o) return bad("NULL options");
    if (!(o->clip_low >= 0.0 && o->clip_low <= 1.0)) return bad("clip_low must be in [0, 1]");
    if (!(o->clip_high >= 0.0) || !std::isfinite(o->clip_high)) return bad("clip_high must be a number >= 0");
    if (!(o->dual_clip == 0.0 || o->dual_clip > 1.0) || !std::isfinite(o->dual_clip))
        return bad("dual_clip must be 0 (none) or greater than 1");
    if (!std::isfinite(o->kl_coef) || !std::isfinite(o->entropy_coef) || !std::isfinite(o->scale))
        return bad("kl_coef, entropy_coef and scale must be finite");
    if (o->reduction < CONDUIT_TOKEN_MEAN || o->reduction > CONDUIT_SUM) return bad("unknown reduction");
    *t = PolicyTerms{(float)(1.0 - o->clip_low), (float)(1.0 + o->clip_high), (float)o->dual_clip, (float)o->kl_coef,
                     (float)o->entropy_coef, o->reduction, o->scale};
    return CONDUIT_OK;
}

RowsView view(const conduit_rows* r) { return RowsView{r->data, r->stride_b, r->stride_t}; }

LogitsArgs logits_args(const conduit_rows* x, int64_t B, int64_t T, int64_t stride, const int32_t* tokens,
                       const uint8_t* mask, double temperature, uint32_t* err) {
    LogitsArgs a{};
    a.shape = make_shape(B, T, stride);
    a.x = view(x);
    a.V = x->width;
    a.c = (float)((double)1.4426950408889634074 / temperature);
    a.inv_t = (float)(1.0 / temperature);
    a.inv_lo = (float)(1.0 / temperature - (double)a.inv_t);
    a.tokens = tokens;
    a.mask = mask;
    a.err = err;
    a.parts = 1;
    return a;
}

// ---------------------------------------------------------------------------
// the projection head
// ---------------------------------------------------------------------------
// (byte offsets within 256 rows of an operand, rows of at most 2^21 elements, stay below 2^31)
constexpr int64_t kHeadMaxTokens = 1ll << 21, kHeadMaxChoices = 1ll << 22, kHeadMaxHidden = 1ll << 16;
constexpr int64_t kHeadMaxLd = 1ll << 21;
constexpr int64_t kHeadChunkBytes = 4ll << 30;  // of the logits' gradient
constexpr int64_t kHeadPartBytes = 4ll << 30;   // of the parts of the hidden states' gradient

int64_t ceil_to(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

// can the product's copies read these rows where they are (16-byte pieces, whole ones)
bool readable(const void* p, int64_t ld, int64_t width) {
    return !misaligned(p, 16) && ld % 8 == 0 && width % 8 == 0 && ld <= kHeadMaxLd;
}

bool one_after_another(const conduit_rows* r, int64_t B, int64_t T) {
    return B <= 1 || T <= 0 || r->stride_b == T * r->stride_t || T == 1;
}

int64_t row_step(const conduit_rows* r, int64_t T) { return T == 1 ? r->stride_b : r->stride_t; }

struct HeadLayout {
    bool pack_w, pack_x;  // pack_x: even without a mask
    int64_t K, ld, chunk, h_ld, d_rows;
    int32_t splits;
    uint64_t count, list, place, taken, part, x_pack, w_pack, d, dx_part, dx_sum, bytes;
};

// Everything but the chunk's arrays is sized for all B * T tokens counting; the
// hidden rows' copy is there whether or not a mask will ask for it.
HeadLayout head_layout(int64_t B, int64_t T, const conduit_rows* hidden, const conduit_rows* weight, int64_t V, bool backward) {
    HeadLayout l{};
    const int64_t N = B * T, H = hidden->width;
    l.pack_w = !readable(weight->data, weight->stride_t, H);
    l.pack_x = !readable(hidden->data, row_step(hidden, T), H) || !one_after_another(hidden, B, T);
    l.d_rows = N;
    if (backward && N <= kHeadTwo) {
        l.d_rows = 2 * N;
        l.pack_x = true;
    }
    l.ld = ceil_to(H, 8);
    l.K = l.ld;
    l.h_ld = ceil_to(H, 8);
    uint64_t at = layout(0, 0).bytes;
    auto take = [&](int64_t bytes) {
        const uint64_t p = at;
        at += up((uint64_t)bytes);
        return p;
    };
    l.count = take(4);
    l.list = take(4 * N);
    l.place = take(4 * N);
    l.x_pack = take(2 * l.d_rows * l.ld);
    l.w_pack = take(l.pack_w ? 2 * V * l.ld : 0);
    if (!backward) {
        l.taken = take(4 * N);
        l.part = take(12 * N * ((V + kGemmTile - 1) / kGemmTile));
    } else {
        const int64_t fit = N > 0 ? kHeadChunkBytes / (2 * N) / kGemmTile * kGemmTile : V;
        l.chunk = ceil_to(V < kHeadMaxLd ? V : kHeadMaxLd, kGemmTile);
        if (l.chunk > fit) l.chunk = fit > 4 * kGemmTile ? fit : 4 * kGemmTile;
        const int64_t most = N > 0 ? kHeadPartBytes / (4 * N * l.h_ld) : 1;
        l.splits = (int32_t)(most < 1 ? 1 : most < kHeadSplits ? most : kHeadSplits);
        l.d = take(2 * l.d_rows * l.chunk);
        l.dx_part = take(4 * l.d_rows * l.h_ld * l.splits);
        l.dx_sum = take(l.chunk < V ? 4 * N * l.h_ld : 0);
    }
    l.bytes = at;
    return l;
}

conduit_status check_head(const conduit_rows* hidden, const conduit_rows* weight, int64_t V, int64_t B, int64_t T) {
    CONDUIT_TRY(check_rows(hidden, B, T, false, "hidden"));
    CONDUIT_TRY(check_rows(weight, 1, V, false, "weight"));
    if (hidden->dtype != CONDUIT_BF16 || weight->dtype != CONDUIT_BF16) return bad("hidden and weight must be BF16");
    if (hidden->width != weight->width) return bad("hidden and weight must have the same width");
    if (hidden->width > kHeadMaxHidden) return bad("the hidden width must be at most 2^16");
    if (V < 1 || V > kHeadMaxChoices) return bad("the number of choices must be in [1, 2^22]");
    if (B * T > kHeadMaxTokens) return bad("the batch must hold at most 2^21 tokens");
    return CONDUIT_OK;
}

HeadArgs head_args(const conduit_rows* hidden, const conduit_rows* weight, int64_t V, int64_t B, int64_t T, int64_t stride,
                   const int32_t* tokens, const uint8_t* mask, double temperature, uint32_t* err, void* ws,
                   const HeadLayout& l) {
    uint8_t* w = static_cast<uint8_t*>(ws);
    auto u16 = [&](uint64_t at) { return reinterpret_cast<uint16_t*>(w + at); };
    HeadArgs a{};
    a.shape = make_shape(B, T, stride);
    a.N = B * T;
    a.V = V;
    a.H = hidden->width;
    a.x = view(hidden);
    a.K = l.K;
    a.d_rows = l.d_rows;
    a.tokens = tokens;
    a.mask = mask;
    a.c = (float)((double)1.4426950408889634074 / temperature);
    a.inv_t = (float)(1.0 / temperature);
    a.err = err;
    a.cus = device_cus();
    if (mask) {
        a.list = reinterpret_cast<int32_t*>(w + l.list);
        a.place = reinterpret_cast<int32_t*>(w + l.place);
        a.count_out = reinterpret_cast<uint32_t*>(w + l.count);
        a.count = a.count_out;
    }
    a.X = GemmOperand{static_cast<const uint16_t*>(hidden->data), row_step(hidden, T)};
    if (mask || l.pack_x) {
        a.x_pack = u16(l.x_pack);
        a.X = GemmOperand{a.x_pack, l.ld};
    }
    a.w_src = static_cast<const uint16_t*>(weight->data);
    a.w_ld = weight->stride_t;
    a.W = GemmOperand{a.w_src, a.w_ld};
    if (l.pack_w) {
        a.w_pack = u16(l.w_pack);
        a.W = GemmOperand{a.w_pack, l.ld};
    }
    return a;
}

}  // namespace

extern "C" {

conduit_status conduit_workspace_init(void* workspace, uint64_t bytes, void* stream) {
    if (!workspace || misaligned(workspace, 256)) return bad("the workspace must be 256-byte aligned and not NULL");
    if (bytes % 4) return bad("the workspace's size must be a multiple of 4");
    if (bytes == 0) return CONDUIT_OK;
    return launched(launch_fill_u32(static_cast<uint32_t*>(workspace), 0u, (int64_t)(bytes / 4), static_cast<hipStream_t>(stream)),
                    "workspace fill");
}

conduit_status conduit_token_logprobs_workspace(int64_t B, int64_t T, const conduit_rows* logits, uint64_t* bytes) {
    if (!bytes) return bad("NULL size pointer");
    CONDUIT_TRY(check_batch(B, T, T));
    CONDUIT_TRY(check_rows(logits, 0, 0, false, "logits"));
    *bytes = logits_layout(B, T, logits).bytes;
    return CONDUIT_OK;
}

conduit_status conduit_token_logprobs(const conduit_rows* logits, int64_t B, int64_t T, int64_t stride,
                                      const int32_t* tokens, const uint8_t* mask, double temperature, float* logp,
                                      float* lse, float* entropy, void* workspace, uint64_t workspace_bytes,
                                      void* stream) {
    CONDUIT_TRY(check_batch(B, T, stride));
    CONDUIT_TRY(check_rows(logits, B, T, false, "logits"));
    CONDUIT_TRY(check_temperature(temperature));
    if (B == 0 || T == 0) return CONDUIT_OK;
    if (!tokens) return bad("tokens must not be NULL");
    CONDUIT_TRY(check_outputs({logp, lse, entropy}, {}, tokens, B, T, stride));
    const Layout l = logits_layout(B, T, logits);
    CONDUIT_TRY(check_workspace(workspace, workspace_bytes, l.bytes));
    uint32_t* err = nullptr;
    CONDUIT_TRY(standalone_error_words(&err));
    const bool bf16 = logits->dtype == CONDUIT_BF16;
    LogitsArgs a = logits_args(logits, B, T, stride, tokens, mask, temperature, err);
    a.logp = logp;
    a.lse = lse;
    a.entropy = entropy;
    a.parts = logits_parts(B * T, a.V, bf16);
    place_workspace(a, workspace, l);
    return launched(launch_token_logprobs(a, bf16, static_cast<hipStream_t>(stream)), "token logprobs launch");
}

conduit_status conduit_token_logprobs_backward(const conduit_rows* logits, int64_t B, int64_t T, int64_t stride,
                                               const int32_t* tokens, const uint8_t* mask, double temperature,
                                               const float* lse, const float* entropy, const float* dlogp,
                                               const float* dentropy, const conduit_rows* dlogits, void* stream) {
    CONDUIT_TRY(check_batch(B, T, stride));
    CONDUIT_TRY(check_rows(logits, B, T, false, "logits"));
    CONDUIT_TRY(check_gradient_rows(logits, dlogits, B, T));
    CONDUIT_TRY(check_temperature(temperature));
    if (B == 0 || T == 0) return CONDUIT_OK;
    if (!tokens || !lse) return bad("tokens and lse must not be NULL");
    if (dentropy && !entropy) return bad("the gradient of the entropy needs the entropy");
    CONDUIT_TRY(check_outputs({}, {lse, entropy, dlogp, dentropy}, tokens, B, T, stride));
    uint32_t* err = nullptr;
    CONDUIT_TRY(standalone_error_words(&err));
    LogitsArgs a = logits_args(logits, B, T, stride, tokens, mask, temperature, err);
    a.dx = view(dlogits);
    a.lse_in = lse;
    a.entropy_in = entropy;
    a.g = dlogp;
    a.h = dentropy;
    return launched(launch_token_logprobs_backward(a, logits->dtype == CONDUIT_BF16, static_cast<hipStream_t>(stream)),
                    "token logprobs gradient launch");
}

void conduit_policy_opts_default(conduit_policy_opts* opts) {
    if (opts) *opts = conduit_policy_opts{0.2, 0.2, 0.0, 0.0, 0.0, 1.0, CONDUIT_TOKEN_MEAN, 0};
}

conduit_status conduit_policy_loss_workspace(int64_t B, int64_t T, uint64_t* bytes) {
    if (!bytes) return bad("NULL size pointer");
    CONDUIT_TRY(check_batch(B, T, T));
    *bytes = policy_layout(B).bytes;
    return CONDUIT_OK;
}

conduit_status conduit_policy_loss(const conduit_policy_opts* opts, int64_t B, int64_t T, int64_t stride,
                                   const float* logp, const float* old_logp, const float* ref_logp, const float* adv,
                                   const float* entropy, const uint8_t* mask, float* stats, float* dlogp,
                                   float* dentropy, void* workspace, uint64_t workspace_bytes, void* stream) {
    PolicyArgs p{};
    CONDUIT_TRY(policy_terms(opts, &p.o));
    CONDUIT_TRY(check_batch(B, T, stride));
    if (!stats || misaligned(stats, 4)) return bad("stats must not be NULL (and aligned)");
    if (B > 0 && T > 0 && (!logp || !adv)) return bad("logp and adv must not be NULL");
    CONDUIT_TRY(check_outputs({dlogp, dentropy}, {logp, old_logp, ref_logp, adv, entropy}, nullptr, B, T, stride));
    const Layout l = policy_layout(B);
    CONDUIT_TRY(check_workspace(workspace, workspace_bytes, l.bytes));
    uint32_t* err = nullptr;
    CONDUIT_TRY(standalone_error_words(&err));
    if (B == 0 || T == 0) B = T = stride = 0;
    p.shape = make_shape(B, T, stride);
    p.logp = logp;
    p.old_logp = old_logp ? old_logp : logp;
    p.ref_logp = ref_logp ? ref_logp : logp;
    p.adv = adv;
    p.entropy = entropy;
    p.mask = mask;
    p.stats = stats;
    p.dlogp = dlogp;
    p.dentropy = dentropy;
    place_workspace(p, workspace, l);
    return launched(launch_policy_loss(p, false, static_cast<hipStream_t>(stream)), "policy loss launch");
}

conduit_status conduit_policy_loss_logits_workspace(int64_t B, int64_t T, const conduit_rows* logits, uint64_t* bytes) {
    return conduit_token_logprobs_workspace(B, T, logits, bytes);
}

conduit_status conduit_policy_loss_logits(const conduit_policy_opts* opts, const conduit_rows* logits, int64_t B,
                                          int64_t T, int64_t stride, const int32_t* tokens, const float* old_logp,
                                          const float* ref_logp, const float* adv, const uint8_t* mask,
                                          double temperature, float* logp, float* entropy, float* stats,
                                          const conduit_rows* dlogits, void* workspace, uint64_t workspace_bytes,
                                          void* stream) {
    PolicyArgs p{};
    CONDUIT_TRY(policy_terms(opts, &p.o));
    CONDUIT_TRY(check_batch(B, T, stride));
    CONDUIT_TRY(check_rows(logits, B, T, false, "logits"));
    CONDUIT_TRY(check_gradient_rows(logits, dlogits, B, T));
    CONDUIT_TRY(check_temperature(temperature));
    if (!stats || misaligned(stats, 4)) return bad("stats must not be NULL (and aligned)");
    const bool empty = B == 0 || T == 0;
    if (!empty && (!tokens || !adv || !logp || !entropy)) return bad("tokens, adv, logp and entropy must not be NULL");
    // (not in place here: the statistics are summed up after logp and entropy are written)
    for (const float* o : {(const float*)logp, (const float*)entropy})
        for (const float* i : {old_logp, ref_logp, adv})
            if (!empty && o && o == i) return bad("logp and entropy must be apart from the inputs");
    CONDUIT_TRY(check_outputs({logp, entropy}, {old_logp, ref_logp, adv}, tokens, B, T, stride));
    const Layout l = logits_layout(B, T, logits);
    CONDUIT_TRY(check_workspace(workspace, workspace_bytes, l.bytes));
    uint32_t* err = nullptr;
    CONDUIT_TRY(standalone_error_words(&err));
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (empty) {
        p.shape = make_shape(0, 0, 0);
        p.stats = stats;
        place_workspace(p, workspace, l);
        return launched(launch_policy_loss(p, false, s), "policy loss launch");
    }
    const bool bf16 = logits->dtype == CONDUIT_BF16;
    LogitsArgs a = logits_args(logits, B, T, stride, tokens, mask, temperature, err);
    a.dx = view(dlogits);
    a.logp = logp;
    a.entropy = entropy;
    a.parts = logits_parts(B * T, a.V, bf16);
    place_workspace(a, workspace, l);
    p.shape = a.shape;
    p.logp = logp;
    p.old_logp = old_logp ? old_logp : logp;
    p.ref_logp = ref_logp ? ref_logp : logp;
    p.adv = adv;
    p.entropy = entropy;
    p.mask = mask;
    p.tokens = tokens;
    p.V = a.V;
    p.stats = stats;
    place_workspace(p, workspace, l);
    return launched(launch_policy_loss_logits(a, p, bf16, s), "policy loss launch");
}

void conduit_preference_opts_default(conduit_preference_opts* opts) {
    if (opts) *opts = conduit_preference_opts{0.1, 0.0, 1.0, CONDUIT_PREFERENCE_SIGMOID, 0};
}

conduit_status conduit_preference_loss_workspace(int64_t P, int64_t T, uint64_t* bytes) {
    if (!bytes) return bad("NULL size pointer");
    if (P < 0) return bad("the number of pairs must be >= 0");
    if (P > kMaxTokens / 2) return bad("the batch must hold fewer than 2^31 tokens");
    CONDUIT_TRY(check_batch(2 * P, T, T));
    *bytes = preference_layout(P, T).bytes;
    return CONDUIT_OK;
}

conduit_status conduit_preference_loss(const conduit_preference_opts* opts, int64_t P, int64_t T, int64_t stride,
                                       const float* logp, const float* ref_logp, const uint8_t* mask, float* loss,
                                       float* chosen, float* rejected, float* stats, float* dlogp, void* workspace,
                                       uint64_t workspace_bytes, void* stream) {
    if (!opts) return bad("NULL options");
    if (!(opts->beta > 0.0) || !std::isfinite(opts->beta)) return bad("beta must be a positive number");
    if (!(opts->label_smoothing >= 0.0 && opts->label_smoothing < 1.0)) return bad("label_smoothing must be in [0, 1)");
    if (!std::isfinite(opts->scale)) return bad("scale must be finite");
    if (opts->loss < CONDUIT_PREFERENCE_SIGMOID || opts->loss > CONDUIT_PREFERENCE_SQUARED) return bad("unknown preference loss");
    if (P < 0) return bad("the number of pairs must be >= 0");
    if (P > kMaxTokens / 2) return bad("the batch must hold fewer than 2^31 tokens");
    CONDUIT_TRY(check_batch(2 * P, T, stride));
    if (!stats || misaligned(stats, 4)) return bad("stats must not be NULL (and aligned)");
    if (P > 0 && (!loss || (T > 0 && !logp))) return bad("logp and loss must not be NULL");
    for (const float* o : {loss, chosen, rejected})
        if (o && misaligned(o, 4)) return bad("loss, chosen and rejected must be aligned to their elements");
    CONDUIT_TRY(check_outputs({dlogp}, {logp, ref_logp}, nullptr, 2 * P, T, stride));
    const Layout l = preference_layout(P, T);
    CONDUIT_TRY(check_workspace(workspace, workspace_bytes, l.bytes));
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (P == 0) return launched(launch_fill_u32(reinterpret_cast<uint32_t*>(stats), 0u, 4, s), "preference loss launch");
    PreferenceArgs a{};
    a.P = P;
    a.T = T;
    a.stride = stride;
    a.beta = opts->beta;
    a.smoothing = opts->label_smoothing;
    a.scale = opts->scale;
    a.squared = opts->loss == CONDUIT_PREFERENCE_SQUARED;
    a.length_norm = opts->length_norm != 0;
    a.logp = logp;
    a.ref = ref_logp;
    a.mask = mask;
    a.loss = loss;
    a.chosen = chosen;
    a.rejected = rejected;
    a.stats = stats;
    a.dlogp = dlogp;
    a.parts = preference_parts(P, T);
    uint8_t* w = static_cast<uint8_t*>(workspace);
    a.head = reinterpret_cast<WorkspaceHead*>(w);
    a.pair = reinterpret_cast<double*>(w + l.rest);
    a.partial = a.pair + 4 * P;
    return launched(launch_preference_loss(a, s), "preference loss launch");
}

conduit_status conduit_head_logprobs_workspace(int64_t B, int64_t T, const conduit_rows* hidden, const conduit_rows* weight,
                                               int64_t V, uint64_t* bytes) {
    if (!bytes) return bad("NULL size pointer");
    CONDUIT_TRY(check_batch(B, T, T));
    CONDUIT_TRY(check_head(hidden, weight, V, B, T));
    *bytes = head_layout(B, T, hidden, weight, V, false).bytes;
    return CONDUIT_OK;
}

conduit_status conduit_head_logprobs(const conduit_rows* hidden, const conduit_rows* weight, int64_t V, int64_t B, int64_t T,
                                     int64_t stride, const int32_t* tokens, const uint8_t* mask, double temperature,
                                     float* logp, float* lse, float* entropy, void* workspace, uint64_t workspace_bytes,
                                     void* stream) {
    CONDUIT_TRY(check_batch(B, T, stride));
    CONDUIT_TRY(check_head(hidden, weight, V, B, T));
    CONDUIT_TRY(check_temperature(temperature));
    if (B == 0 || T == 0) return CONDUIT_OK;
    if (!tokens) return bad("tokens must not be NULL");
    CONDUIT_TRY(check_outputs({logp, lse, entropy}, {}, tokens, B, T, stride));
    const HeadLayout l = head_layout(B, T, hidden, weight, V, false);
    CONDUIT_TRY(check_workspace(workspace, workspace_bytes, l.bytes));
    uint32_t* err = nullptr;
    CONDUIT_TRY(standalone_error_words(&err));
    HeadArgs a = head_args(hidden, weight, V, B, T, stride, tokens, mask, temperature, err, workspace, l);
    uint8_t* w = static_cast<uint8_t*>(workspace);
    a.taken = reinterpret_cast<float*>(w + l.taken);
    a.part = reinterpret_cast<float*>(w + l.part);
    a.logp = logp;
    a.lse = lse;
    a.entropy = entropy;
    return launched(launch_head_logprobs(a, static_cast<hipStream_t>(stream)), "head logprobs launch");
}

conduit_status conduit_head_logprobs_backward_workspace(int64_t B, int64_t T, const conduit_rows* hidden,
                                                        const conduit_rows* weight, int64_t V, uint64_t* bytes) {
    if (!bytes) return bad("NULL size pointer");
    CONDUIT_TRY(check_batch(B, T, T));
    CONDUIT_TRY(check_head(hidden, weight, V, B, T));
    *bytes = head_layout(B, T, hidden, weight, V, true).bytes;
    return CONDUIT_OK;
}

conduit_status conduit_head_logprobs_backward(const conduit_rows* hidden, const conduit_rows* weight, int64_t V, int64_t B,
                                              int64_t T, int64_t stride, const int32_t* tokens, const uint8_t* mask,
                                              double temperature, const float* lse, const float* entropy, const float* dlogp,
                                              const float* dentropy, const conduit_rows* dhidden, const conduit_rows* dweight,
                                              void* workspace, uint64_t workspace_bytes, void* stream) {
    CONDUIT_TRY(check_batch(B, T, stride));
    CONDUIT_TRY(check_head(hidden, weight, V, B, T));
    CONDUIT_TRY(check_rows(dhidden, B, T, true, "dhidden"));
    CONDUIT_TRY(check_rows(dweight, 1, V, true, "dweight"));
    if (dhidden->dtype != CONDUIT_BF16 || dweight->dtype != CONDUIT_BF16) return bad("dhidden and dweight must be BF16");
    if (dhidden->width != hidden->width || dweight->width != hidden->width)
        return bad("dhidden and dweight must have the hidden width");
    CONDUIT_TRY(check_temperature(temperature));
    const bool empty = B == 0 || T == 0;
    if (!empty) {
        if (!tokens || !lse) return bad("tokens and lse must not be NULL");
        if (dentropy && !entropy) return bad("the gradient of the entropy needs the entropy");
        CONDUIT_TRY(check_outputs({}, {lse, entropy, dlogp, dentropy}, tokens, B, T, stride));
        if (!apart(dhidden->data, rows_extent(dhidden, B, T), hidden->data, rows_extent(hidden, B, T)) ||
            !apart(dhidden->data, rows_extent(dhidden, B, T), weight->data, rows_extent(weight, 1, V)) ||
            !apart(dweight->data, rows_extent(dweight, 1, V), hidden->data, rows_extent(hidden, B, T)) ||
            !apart(dhidden->data, rows_extent(dhidden, B, T), dweight->data, rows_extent(dweight, 1, V)))
            return bad("dhidden and dweight must be apart from each other and from the inputs");
    }
    if (!apart(dweight->data, rows_extent(dweight, 1, V), weight->data, rows_extent(weight, 1, V)))
        return bad("dhidden and dweight must be apart from each other and from the inputs");
    const HeadLayout l = head_layout(B, T, hidden, weight, V, true);
    CONDUIT_TRY(check_workspace(workspace, workspace_bytes, l.bytes));
    uint32_t* err = nullptr;
    CONDUIT_TRY(standalone_error_words(&err));
    HeadArgs a = head_args(hidden, weight, V, empty ? 0 : B, empty ? 0 : T, empty ? 0 : stride, tokens, mask, temperature, err,
                           workspace, l);
    uint8_t* w = static_cast<uint8_t*>(workspace);
    a.lse_in = lse;
    a.entropy_in = entropy;
    a.g = dlogp;
    a.h = dentropy;
    a.dx = view(dhidden);
    a.dw = static_cast<uint16_t*>(dweight->data);
    a.dw_ld = dweight->stride_t;
    a.chunk = l.chunk;
    a.splits = l.splits;
    a.d = reinterpret_cast<uint16_t*>(w + l.d);
    a.d_ld = l.chunk;
    a.dx_part = reinterpret_cast<float*>(w + l.dx_part);
    a.dx_sum = reinterpret_cast<float*>(w + l.dx_sum);
    a.h_ld = l.h_ld;
    return launched(launch_head_backward(a, static_cast<hipStream_t>(stream)), "head gradient launch");
}

}  // extern "C"
