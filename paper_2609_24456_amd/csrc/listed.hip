// Host side of the calls on listed choices of include/conduit.h: argument checks,
// the layout of their workspaces, and the launches.
#include "listed_dev.h"
#include "loss_host.h"

using namespace conduit;

namespace {

// [B, T] rows of K listed values of one dtype
conduit_status check_listed(const conduit_rows* r, int64_t B, int64_t T, int32_t dtype, bool out, const char* what) {
    const std::string w(what);
    if (!r) return bad((w + " must not be NULL").c_str());
    if (r->dtype != dtype) return bad((w + (dtype == CONDUIT_I32 ? ": dtype must be I32" : ": dtype must be F32")).c_str());
    if (r->width < 1 || r->width > kMostListed) return bad((w + ": width must be in [1, 128]").c_str());
    return check_rows_layout(r, B, T, out, w);
}

// the values beside the choices' numbers
conduit_status check_values(const conduit_rows* r, const conduit_rows* ids, int64_t B, int64_t T, bool out, const char* what) {
    CONDUIT_TRY(check_listed(r, B, T, CONDUIT_F32, out, what));
    if (r->width != ids->width) return bad((std::string(what) + " must have as many values a token as ids").c_str());
    return CONDUIT_OK;
}

// a written set of rows is apart from other rows, and from per-token arrays of `size` bytes an element
conduit_status check_apart(const conduit_rows* o, const char* what, std::initializer_list<const conduit_rows*> rows,
                           std::initializer_list<const void*> tokens, const uint8_t* mask, int64_t B, int64_t T, int64_t stride) {
    const std::string w(what);
    const int64_t n = rows_extent(o, B, T), each = (B - 1) * stride + T;
    for (const conduit_rows* r : rows)
        if (r && !apart(o->data, n, r->data, rows_extent(r, B, T))) return bad((w + " must be apart from the call's other arrays").c_str());
    for (const void* t : tokens)
        if (t && !apart(o->data, n, t, 4 * each)) return bad((w + " must be apart from the call's other arrays").c_str());
    if (mask && !apart(o->data, n, mask, each)) return bad((w + " must be apart from the call's other arrays").c_str());
    return CONDUIT_OK;
}

// per-token outputs apart from rows that are read and from the mask
conduit_status check_outputs_apart(std::initializer_list<const void*> outs, std::initializer_list<const conduit_rows*> rows,
                                   const uint8_t* mask, int64_t B, int64_t T, int64_t stride) {
    const int64_t each = (B - 1) * stride + T;
    for (const void* o : outs) {
        if (!o) continue;
        for (const conduit_rows* r : rows)
            if (!apart(o, 4 * each, r->data, rows_extent(r, B, T))) return bad("an output overlaps an input");
        if (mask && !apart(o, 4 * each, mask, each)) return bad("an output overlaps the mask");
    }
    return CONDUIT_OK;
}

// One launch takes fewer than 2^31 parts of rows (the range of the division that finds a part's row).  Checked before
// anything is enqueued: a call that has begun leaves the workspace's counters for its last launch to clear.
conduit_status check_parts(int64_t B, int64_t T, int64_t parts) {
    if (B * T * parts >= 1ll << 31) return bad("the rows of the batch must take fewer than 2^31 parts in all");
    return CONDUIT_OK;
}

conduit_status check_K(int64_t K) {
    if (K < 1 || K > kMostListed) return bad("the number of choices a token must be in [1, 128]");
    return CONDUIT_OK;
}

// ---------------------------------------------------------------------------
// workspaces
// ---------------------------------------------------------------------------
struct ListedLayout {
    RowParts split;
    Layout l;
    uint64_t part, more;  // offsets: statistics of the parts; their keys, or the rows' records
};

ListedLayout top_layout(int64_t B, int64_t T, const conduit_rows* x, int64_t K) {
    ListedLayout o;
    const int64_t rows = B * T;
    o.split = top_parts(rows, x->width, x->dtype == CONDUIT_BF16);
    const uint64_t n = o.split.parts > 1 ? (uint64_t)rows * o.split.parts : 0;
    o.l = layout(B, up(12 * n) + 8 * n * (uint64_t)K);
    o.part = o.l.rest;
    o.more = o.part + up(12 * n);
    return o;
}

ListedLayout listed_layout(int64_t B, int64_t T, const conduit_rows* x, bool whole_rows) {
    ListedLayout o;
    const int64_t rows = B * T;
    o.split = listed_parts(rows, x->width, x->dtype == CONDUIT_BF16, whole_rows);
    const uint64_t n = o.split.parts > 1 ? (uint64_t)rows * o.split.parts : 0, sums = up(sizeof(double) * kDistillSums * kPolicyBlocks);
    o.l = layout(B, sums + up(12 * n) + (n > 0 ? sizeof(ListedRow) * (uint64_t)rows : 0));
    o.part = o.l.rest + sums;
    o.more = o.part + up(12 * n);
    return o;
}

// Distillation without a gradient scans its rows, with one it holds them: the workspace is of the larger.
ListedLayout distill_layout(int64_t B, int64_t T, const conduit_rows* x, bool has_dx) {
    ListedLayout o = listed_layout(B, T, x, has_dx), other = listed_layout(B, T, x, !has_dx);
    if (other.l.bytes > o.l.bytes) o.l.bytes = other.l.bytes;
    return o;
}

// arguments that every call has
template <typename Args>
void common_args(Args& a, const conduit_rows* x, int64_t B, int64_t T, int64_t stride, const conduit_rows* ids, const uint8_t* mask,
                 double temperature, uint32_t* err) {
    a.shape = make_shape(B, T, stride);
    a.x = view(x);
    a.V = x->width;
    // (by the rows' bytes, whatever lies between them)
    a.once = (double)(B * T) * (double)x->width * elem_size(x->dtype) > (double)kPastBytes;
    a.c = (float)((double)1.4426950408889634074 / temperature);
    a.inv_t = (float)(1.0 / temperature);
    a.inv_lo = (float)(1.0 / temperature - (double)a.inv_t);
    a.mask = mask;
    a.ids = view(ids);
    a.K = (int32_t)ids->width;
    a.err = err;
}

void set_gradient(ListedArgs& a, const conduit_rows* dx) {
    a.dx = view(dx);
    a.has_dx = true;
    a.past = a.once;
}

template <typename Args>
void place_parts(Args& a, uint8_t* w, const ListedLayout& o) {
    a.parts = o.split.parts;
    a.per = o.split.per;
    a.by_parts = make_div31((uint32_t)o.split.parts);
    a.part = reinterpret_cast<float*>(w + o.part);
    // (a ticket a row is there for this many)
    a.row_ticket = a.shape.B * a.shape.T <= kSplitRows ? reinterpret_cast<uint32_t*>(w + o.l.row_ticket) : nullptr;
}

conduit_status workspace_size(int64_t B, int64_t T, const conduit_rows* logits, int64_t K, uint64_t* bytes) {
    if (!bytes) return bad("NULL size pointer");
    CONDUIT_TRY(check_batch(B, T, T));
    CONDUIT_TRY(check_rows(logits, 0, 0, false, "logits"));
    return check_K(K);
}

}  // namespace

extern "C" {

conduit_status conduit_token_alternatives_workspace(int64_t B, int64_t T, const conduit_rows* logits, int64_t K, uint64_t* bytes) {
    CONDUIT_TRY(workspace_size(B, T, logits, K, bytes));
    *bytes = top_layout(B, T, logits, K).l.bytes;
    return CONDUIT_OK;
}

conduit_status conduit_token_alternatives(const conduit_rows* logits, int64_t B, int64_t T, int64_t stride, const int32_t* tokens,
                                          const uint8_t* mask, double temperature, const conduit_rows* ids,
                                          const conduit_rows* logps, float* logp, float* lse, float* entropy, void* workspace,
                                          uint64_t workspace_bytes, void* stream) {
    CONDUIT_TRY(check_batch(B, T, stride));
    CONDUIT_TRY(check_rows(logits, B, T, false, "logits"));
    CONDUIT_TRY(check_listed(ids, B, T, CONDUIT_I32, true, "ids"));
    CONDUIT_TRY(check_values(logps, ids, B, T, true, "logps"));
    CONDUIT_TRY(check_temperature(temperature));
    if (B == 0 || T == 0) return CONDUIT_OK;
    if (logp && !tokens) return bad("logp needs the tokens");
    CONDUIT_TRY(check_outputs({logp, lse, entropy}, {}, tokens, B, T, stride));
    CONDUIT_TRY(check_apart(ids, "ids", {logits, logps}, {tokens, logp, lse, entropy}, mask, B, T, stride));
    CONDUIT_TRY(check_apart(logps, "logps", {logits}, {tokens, logp, lse, entropy}, mask, B, T, stride));
    CONDUIT_TRY(check_outputs_apart({logp, lse, entropy}, {logits}, mask, B, T, stride));
    const ListedLayout l = top_layout(B, T, logits, ids->width);
    CONDUIT_TRY(check_parts(B, T, l.split.parts));
    CONDUIT_TRY(check_workspace(workspace, workspace_bytes, l.l.bytes));
    uint32_t* err = nullptr;
    CONDUIT_TRY(standalone_error_words(&err));
    TopArgs a{};
    common_args(a, logits, B, T, stride, ids, mask, temperature, err);
    a.tokens = tokens;
    a.logps = view(logps);
    a.logp = logp;
    a.lse = lse;
    a.entropy = entropy;
    uint8_t* w = static_cast<uint8_t*>(workspace);
    place_parts(a, w, l);
    a.key = reinterpret_cast<uint64_t*>(w + l.more);
    return launched(launch_token_alternatives(a, logits->dtype == CONDUIT_BF16, static_cast<hipStream_t>(stream)),
                    "token alternatives launch");
}

conduit_status conduit_listed_logprobs_workspace(int64_t B, int64_t T, const conduit_rows* logits, int64_t K, uint64_t* bytes) {
    CONDUIT_TRY(workspace_size(B, T, logits, K, bytes));
    *bytes = listed_layout(B, T, logits, false).l.bytes;
    return CONDUIT_OK;
}

conduit_status conduit_listed_logprobs(const conduit_rows* logits, int64_t B, int64_t T, int64_t stride, const conduit_rows* ids,
                                       const uint8_t* mask, double temperature, const conduit_rows* logps, float* rest, float* lse,
                                       void* workspace, uint64_t workspace_bytes, void* stream) {
    CONDUIT_TRY(check_batch(B, T, stride));
    CONDUIT_TRY(check_rows(logits, B, T, false, "logits"));
    CONDUIT_TRY(check_listed(ids, B, T, CONDUIT_I32, false, "ids"));
    CONDUIT_TRY(check_values(logps, ids, B, T, true, "logps"));
    CONDUIT_TRY(check_temperature(temperature));
    if (B == 0 || T == 0) return CONDUIT_OK;
    CONDUIT_TRY(check_outputs({rest, lse}, {}, nullptr, B, T, stride));
    CONDUIT_TRY(check_apart(logps, "logps", {logits, ids}, {rest, lse}, mask, B, T, stride));
    CONDUIT_TRY(check_outputs_apart({rest, lse}, {logits, ids}, mask, B, T, stride));
    const ListedLayout l = listed_layout(B, T, logits, false);
    CONDUIT_TRY(check_parts(B, T, l.split.parts));
    CONDUIT_TRY(check_workspace(workspace, workspace_bytes, l.l.bytes));
    uint32_t* err = nullptr;
    CONDUIT_TRY(standalone_error_words(&err));
    ListedArgs a{};
    common_args(a, logits, B, T, stride, ids, mask, temperature, err);
    a.logps = view(logps);
    a.rest = rest;
    a.lse = lse;
    place_parts(a, static_cast<uint8_t*>(workspace), l);
    return launched(launch_listed_logprobs(a, logits->dtype == CONDUIT_BF16, static_cast<hipStream_t>(stream)), "listed logprobs launch");
}

conduit_status conduit_listed_logprobs_backward(const conduit_rows* logits, int64_t B, int64_t T, int64_t stride,
                                                const conduit_rows* ids, const uint8_t* mask, double temperature, const float* lse,
                                                const float* rest, const conduit_rows* dlogps, const float* drest,
                                                const conduit_rows* dlogits, void* stream) {
    CONDUIT_TRY(check_batch(B, T, stride));
    CONDUIT_TRY(check_rows(logits, B, T, false, "logits"));
    CONDUIT_TRY(check_listed(ids, B, T, CONDUIT_I32, false, "ids"));
    CONDUIT_TRY(check_values(dlogps, ids, B, T, false, "dlogps"));
    CONDUIT_TRY(check_gradient_rows(logits, dlogits, B, T));
    CONDUIT_TRY(check_temperature(temperature));
    if (B == 0 || T == 0) return CONDUIT_OK;
    if (!lse) return bad("lse must not be NULL");
    if (drest && !rest) return bad("the gradient of the rest needs the rest");
    CONDUIT_TRY(check_outputs({}, {lse, rest, drest}, nullptr, B, T, stride));
    CONDUIT_TRY(check_apart(dlogits, "dlogits", {ids, dlogps}, {lse, rest, drest}, mask, B, T, stride));
    CONDUIT_TRY(check_parts(B, T, gradient_parts(logits->width, logits->dtype == CONDUIT_BF16)));
    uint32_t* err = nullptr;
    CONDUIT_TRY(standalone_error_words(&err));
    ListedArgs a{};
    common_args(a, logits, B, T, stride, ids, mask, temperature, err);
    a.lowest = lowest_score(a.inv_lo);
    a.lse_in = lse;
    a.rest_in = rest;
    a.g = view(dlogps);
    a.h = drest;
    set_gradient(a, dlogits);
    return launched(launch_listed_logprobs_backward(a, logits->dtype == CONDUIT_BF16, static_cast<hipStream_t>(stream)),
                    "listed logprobs gradient launch");
}

void conduit_distill_opts_default(conduit_distill_opts* opts) {
    if (opts) *opts = conduit_distill_opts{1.0, 1.0, CONDUIT_DISTILL_FORWARD, CONDUIT_TOKEN_MEAN, 0, 0};
}

conduit_status conduit_distill_loss_workspace(int64_t B, int64_t T, const conduit_rows* logits, int64_t K, uint64_t* bytes) {
    CONDUIT_TRY(workspace_size(B, T, logits, K, bytes));
    *bytes = distill_layout(B, T, logits, true).l.bytes;
    return CONDUIT_OK;
}

conduit_status conduit_distill_loss(const conduit_distill_opts* opts, const conduit_rows* logits, int64_t B, int64_t T, int64_t stride,
                                    const conduit_rows* ids, const conduit_rows* teacher, const float* weight, const uint8_t* mask,
                                    double temperature, float* loss, float* stats, const conduit_rows* dlogits, void* workspace,
                                    uint64_t workspace_bytes, void* stream) {
    if (!opts) return bad("NULL options");
    if (opts->loss < CONDUIT_DISTILL_FORWARD || opts->loss > CONDUIT_DISTILL_REVERSE) return bad("unknown divergence");
    if (opts->reduction < CONDUIT_TOKEN_MEAN || opts->reduction > CONDUIT_SUM) return bad("unknown reduction");
    const bool reverse = opts->loss == CONDUIT_DISTILL_REVERSE, with_rest = opts->rest != 0;
    if (reverse && !with_rest) return bad("the reverse divergence needs the rest: the student's probability outside the list");
    CONDUIT_TRY(check_temperature(opts->teacher_temperature));
    if (with_rest && opts->teacher_temperature != 1.0) return bad("with the rest the teacher's log-probabilities are taken as they are: teacher_temperature 1");
    if (!std::isfinite(opts->scale)) return bad("scale must be finite");
    CONDUIT_TRY(check_batch(B, T, stride));
    CONDUIT_TRY(check_rows(logits, B, T, false, "logits"));
    CONDUIT_TRY(check_listed(ids, B, T, CONDUIT_I32, false, "ids"));
    CONDUIT_TRY(check_values(teacher, ids, B, T, false, "teacher"));
    if (dlogits) CONDUIT_TRY(check_gradient_rows(logits, dlogits, B, T));
    CONDUIT_TRY(check_temperature(temperature));
    if (!stats || misaligned(stats, 4)) return bad("stats must not be NULL (and aligned)");
    const bool empty = B == 0 || T == 0;
    if (!empty) {
        if (!loss) return bad("loss must not be NULL");
        CONDUIT_TRY(check_outputs({loss}, {weight}, nullptr, B, T, stride));
        if (loss == weight) return bad("loss must be apart from the inputs");  // (the statistics are summed up after it is written)
        CONDUIT_TRY(check_outputs_apart({loss}, {logits, ids, teacher}, mask, B, T, stride));
        if (dlogits) CONDUIT_TRY(check_apart(dlogits, "dlogits", {ids, teacher}, {weight, loss}, mask, B, T, stride));
        // (the statistics are three values on their own)
        const int64_t each = (B - 1) * stride + T;
        for (const conduit_rows* r : {logits, ids, teacher, dlogits})
            if (r && !apart(stats, 12, r->data, rows_extent(r, B, T))) return bad("stats must be apart from the call's other arrays");
        for (const void* t : {static_cast<const void*>(weight), static_cast<const void*>(loss)})
            if (t && !apart(stats, 12, t, 4 * each)) return bad("stats must be apart from the call's other arrays");
        if (mask && !apart(stats, 12, mask, each)) return bad("stats must be apart from the call's other arrays");
    }
    const ListedLayout l = distill_layout(B, T, logits, dlogits != nullptr);
    CONDUIT_TRY(check_parts(B, T, l.split.parts));
    if (dlogits && l.split.parts > 1) CONDUIT_TRY(check_parts(B, T, gradient_parts(logits->width, logits->dtype == CONDUIT_BF16)));
    CONDUIT_TRY(check_workspace(workspace, workspace_bytes, l.l.bytes));
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (empty) return launched(launch_fill_u32(reinterpret_cast<uint32_t*>(stats), 0u, 3, s), "distillation launch");
    uint32_t* err = nullptr;
    CONDUIT_TRY(standalone_error_words(&err));
    ListedArgs a{};
    common_args(a, logits, B, T, stride, ids, mask, temperature, err);
    a.teacher = view(teacher);
    a.q_inv_t = (float)(1.0 / opts->teacher_temperature);
    a.reverse = reverse;
    a.with_rest = with_rest;
    a.reduction = opts->reduction;
    a.scale = opts->scale;
    a.weight = weight;
    a.loss = loss;
    a.stats = stats;
    if (dlogits) set_gradient(a, dlogits);
    uint8_t* w = static_cast<uint8_t*>(workspace);
    a.head = reinterpret_cast<WorkspaceHead*>(w);
    a.row_count = reinterpret_cast<uint32_t*>(w + l.l.row_count);
    a.partial = reinterpret_cast<double*>(w + l.l.rest);
    place_parts(a, w, l);
    // (the mean over sequences needs each one's tokens, which a launch over the tokens does not count)
    const bool sequences = opts->reduction == CONDUIT_SEQUENCE_MEAN;
    a.flat_mask = mask && !sequences && (stride == T || B == 1) && !misaligned(mask, 16);
    a.counted = mask && B * T > (sequences ? kPolicyBlocks : a.flat_mask ? kCountedFlat : kCountedHere);
    a.sums = B * T > kPolicyBlocks ? SUM_LAUNCH : a.parts > 1 && a.has_dx ? SUM_NEXT : SUM_ROWS;
    a.row = reinterpret_cast<ListedRow*>(w + l.more);
    return launched(launch_distill_loss(a, logits->dtype == CONDUIT_BF16, s), "distillation launch");
}

}  // extern "C"
