// Device code and launch arguments shared by the loss kernels (k_logits.hip,
// k_policy.hip, k_preference.hip, k_head.hip): per-token arrays, the policy
// loss of one token, reductions in a fixed order.
#pragma once

#include "common.h"

namespace conduit {

// Every per-token array of a call is [B, T] with rows `stride` elements apart.
struct TokenShape {
    int64_t B, T, stride;
    Div31 by_T;  // of n = b * T + t
    __device__ __forceinline__ int64_t at(uint32_t n) const {
        const uint32_t b = div31(n, by_T);
        return (int64_t)b * stride + (n - b * (uint32_t)T);
    }
};

inline TokenShape make_shape(int64_t B, int64_t T, int64_t stride) {
    return TokenShape{B, T, stride, make_div31((uint32_t)(T > 0 ? T : 1))};
}

// [B, T] rows of `width` elements: row (b, t) starts at b * stride_b + t * stride_t
struct RowsView {
    void* data;
    int64_t stride_b, stride_t;
    __device__ __forceinline__ int64_t at(uint32_t n, const TokenShape& s) const {
        const uint32_t b = div31(n, s.by_T);
        return (int64_t)b * stride_b + (int64_t)(n - b * (uint32_t)s.T) * stride_t;
    }
};

// The options of the policy loss as the kernels take them.
struct PolicyTerms {
    float lo, hi;    // 1 - clip_low, 1 + clip_high
    float dual;      // 0: no dual clip
    float kl, ent;
    int32_t reduction;
    double scale;
};

// Head of a workspace: counters that every call finds and leaves at zero.
constexpr int kTicketGroups = 32;
constexpr uint32_t kTicketStep = 32;  // words from a ticket to the next: a cache line each
struct WorkspaceHead {
    uint64_t counts;  // tokens that count, and from bit 32 on rows (sequences) with at least one
    uint32_t ticket;
    uint32_t pad[61];
    struct {
        uint32_t ticket;
        uint32_t pad[kTicketStep - 1];
    } group[kTicketGroups];
};
static_assert(sizeof(WorkspaceHead) == 256 + 128 * kTicketGroups, "workspace head");

constexpr int kPolicySums = 6;     // weighted loss, KL and entropy; clipped, log ratio and ratio
constexpr int kPolicyBlocks = 512; // most workgroups that a sum over the tokens is spread over

struct PolicyArgs {
    TokenShape shape;
    PolicyTerms o;
    const float* logp;
    const float* old_logp;  // (absent: logp)
    const float* ref_logp;  // (absent: logp)
    const float* adv;
    const float* entropy;
    bool has_entropy;
    const uint8_t* mask;
    const int32_t* tokens;  // with V: tokens outside [0, V) add nothing (NULL: every token is valid)
    int64_t V;
    float* stats;
    float* dlogp;
    float* dentropy;
    WorkspaceHead* head;
    uint32_t* row_count;  // [B] counted tokens, with the mean over rows
    double* partial;      // [kPolicyBlocks][kPolicySums]
};

// What the gradient of a row split into parts needs from the join of its parts:
// dx = e^(d) gp + ..., as GradCoef in k_logits.hip, at d = c (x - base), and the
// taken token's own.  Nothing of it grows with the logits, as lse would.
struct SplitRow {
    float base, gp, hp, off, taken;
};

struct LogitsArgs {
    TokenShape shape;
    RowsView x, dx;
    int64_t V;
    float c;      // log2(e) / temperature
    float inv_t;  // 1 / temperature
    float inv_lo; // what its rounding left
    const int32_t* tokens;
    const uint8_t* mask;
    float* logp;
    float* lse;
    float* entropy;
    const float* lse_in;
    const float* entropy_in;
    const float* g;  // gradient of logp
    const float* h;  // gradient of the entropy
    uint32_t* err;
    // split rows: (maximum, sum, weighted sum) of each part of a row, and a ticket a row
    float* part;
    uint32_t* row_ticket;
    int32_t parts;
    SplitRow* split;  // by token number, from the split loss to its gradient launch
};

hipError_t launch_token_count(const PolicyArgs& a, hipStream_t s);
hipError_t launch_policy_loss(const PolicyArgs& a, bool counted, hipStream_t s);
hipError_t launch_token_logprobs(const LogitsArgs& a, bool bf16, hipStream_t s);
hipError_t launch_token_logprobs_backward(const LogitsArgs& a, bool bf16, hipStream_t s);
hipError_t launch_policy_loss_logits(const LogitsArgs& a, const PolicyArgs& p, bool bf16, hipStream_t s);
int logits_parts(int64_t rows, int64_t V, bool bf16);

struct PreferenceArgs {
    int64_t P, T, stride;
    double beta, smoothing, scale;
    int32_t squared, length_norm;
    const float* logp;
    const float* ref;
    const uint8_t* mask;
    float* loss;
    float* chosen;
    float* rejected;
    float* stats;
    float* dlogp;
    WorkspaceHead* head;
    double* pair;     // [P][4]: loss, u, margin > 0, tokens
    double* partial;  // [2 P][parts][2]: sum, tokens
    int32_t parts;
};

hipError_t launch_preference_loss(const PreferenceArgs& a, hipStream_t s);
int preference_parts(int64_t P, int64_t T);

// ---------------------------------------------------------------------------
// launches of a workgroup for each of many rows
// ---------------------------------------------------------------------------
// A launch takes fewer than 2^32 threads in a dimension, so many workgroups are
// spread over two; the last of them may have nothing to do.
inline dim3 grid_of(int64_t blocks, int threads) {
    constexpr int64_t kAcross = 1 << 20;
    if (blocks * threads < 1ll << 32) return dim3((unsigned)blocks);
    return dim3((unsigned)kAcross, (unsigned)((blocks + kAcross - 1) / kAcross));
}
__device__ __forceinline__ uint32_t block_number() { return blockIdx.y * gridDim.x + blockIdx.x; }

// ---------------------------------------------------------------------------
// constants and small functions
// ---------------------------------------------------------------------------
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_fast(float x) { return __builtin_amdgcn_logf(x); }

// exp(x) in a few instructions: 2^t for t = x log2(e) rounded, times 1 + ln2 r for
// what the rounding of t (and of log2(e)) left out, so that the error does not
// grow with x
__device__ __forceinline__ float exp_fast(float x) {
    const float t = x * kLog2e, r = fmaf(x, kLog2e, -t) + x * 1.9259629911e-8f;  // (the last: log2(e) - kLog2e)
    const float e = exp2_fast(t);
    return fabsf(t) < 128.0f ? fmaf(e, r * kLn2, e) : e;  // (beyond: 0 or infinity, which times r may be no number)
}

// k = exp(x) - 1 - x (x^2 / 2 at small x) and em1 = exp(x) - 1: the series up to
// x^9 below |x| = 1/2 (the first term left out is x^8 * 2 / 10! of the whole,
// under 3e-9), where the difference would cancel.  Both are infinity at infinity.
__device__ __forceinline__ void exp_remainder(float x, float* k, float* em1) {
    float p = 1.0f / 362880.0f;
    p = fmaf(p, x, 1.0f / 40320.0f);
    p = fmaf(p, x, 1.0f / 5040.0f);
    p = fmaf(p, x, 1.0f / 720.0f);
    p = fmaf(p, x, 1.0f / 120.0f);
    p = fmaf(p, x, 1.0f / 24.0f);
    p = fmaf(p, x, 1.0f / 6.0f);
    p = fmaf(p, x, 0.5f);
    p = p * x * x;
    const float e = exp_fast(x) - 1.0f;
    const bool small = fabsf(x) < 0.5f;
    *k = small ? p : x < INFINITY ? e - x : e;
    *em1 = small ? p + x : e;
}

// exp(x) - 1
__device__ __forceinline__ float expm1_fast(float x) {
    float k, em1;
    exp_remainder(x, &k, &em1);
    return em1;
}

// ---------------------------------------------------------------------------
// the policy loss of one token
// ---------------------------------------------------------------------------
struct TokenLoss {
    float term, kl, ratio, log_ratio;
    float slope;  // derivative of term + kl_coef * kl with respect to logp
    float held;   // 1 if the clip or the dual clip decides
};

// r = exp(logp - old); term = max(-A r, -A clip(r, lo, hi)), and where A < 0
// at most -A dual; kl = exp(ref - logp) - (ref - logp) - 1.  A NaN stays one
// (no fmax, which would drop it); an advantage of 0 has no term however large
// the ratio.  Equal log-probabilities, -inf among them, have ratio 1 and kl 0,
// so an absent old or reference policy is passed as logp itself.  Without
// branches: the lanes of a wavefront hold tokens of every kind.
__device__ __forceinline__ TokenLoss policy_token(const PolicyTerms& o, float logp, float old, float ref, float adv) {
    TokenLoss r;
    r.log_ratio = logp == old ? 0.0f : logp - old;
    r.ratio = exp_fast(r.log_ratio);
    const float plain = adv == 0.0f ? 0.0f : -adv * r.ratio;
    const float kept = r.ratio < o.lo ? o.lo : r.ratio > o.hi ? o.hi : r.ratio;
    const float bound = -adv * kept, ceiling = -adv * o.dual;
    const bool held = bound > plain;
    const float term = held ? bound : plain;
    const bool dual = (o.dual > 0.0f) & (adv < 0.0f) & (term > ceiling);
    r.term = dual ? ceiling : term;
    r.held = held | dual ? 1.0f : 0.0f;
    const float x = ref == logp ? 0.0f : ref - logp;
    float em1;
    exp_remainder(x, &r.kl, &em1);
    r.slope = held | dual ? 0.0f : plain;
    r.slope = o.kl != 0.0f ? fmaf(-o.kl, em1, r.slope) : r.slope;
    return r;
}

// weight of a token: of the mean over tokens, of the mean over rows of each
// row's mean, or 1
__device__ __forceinline__ double token_weight(const PolicyTerms& o, uint32_t tokens, uint32_t rows, uint32_t row) {
    if (o.reduction == CONDUIT_SUM) return 1.0;
    if (o.reduction == CONDUIT_TOKEN_MEAN) return 1.0 / (double)(tokens > 0 ? tokens : 1);
    return 1.0 / ((double)(rows > 0 ? rows : 1) * (double)(row > 0 ? row : 1));
}

// A few tokens of one weight, and a lane's sums.
struct TokenSums {
    double v[kPolicySums] = {0, 0, 0, 0, 0, 0};
    __device__ __forceinline__ void add(bool on, const TokenLoss& t, float entropy) {
        v[0] += on ? t.term : 0.0f;
        v[1] += on ? t.kl : 0.0f;
        v[2] += on ? entropy : 0.0f;
        v[3] += on ? t.held : 0.0f;
        v[4] += on ? t.log_ratio : 0.0f;
        v[5] += on ? t.ratio : 0.0f;
    }
};

struct PolicySums {
    double v[kPolicySums] = {0, 0, 0, 0, 0, 0};
    __device__ __forceinline__ void add(double w, const TokenSums& t) {
#pragma unroll
        for (int i = 0; i < kPolicySums; ++i) v[i] += i < 3 ? w * t.v[i] : t.v[i];
    }
};

// ---------------------------------------------------------------------------
// reductions in a fixed order
// ---------------------------------------------------------------------------
// The two sides of one step of a butterfly, in every lane: its own value and the
// lane's 1 or 2 away, or mirrored in its 8 or 16 (DPP moves), then, by swaps of
// rows, those of the even and the odd row of 16 and of the two halves.
template <typename T>
struct Sides {
    T a, b;
};

template <int STEP>
__device__ __forceinline__ Sides<uint32_t> sides(uint32_t x) {
    constexpr int kCtrl[4] = {0xB1, 0x4E, 0x141, 0x140};  // quad_perm 1032, quad_perm 2301, row_half_mirror, row_mirror
    if constexpr (STEP < 4) {
        return {x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, kCtrl[STEP], 0xf, 0xf, true)};
    } else {
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        const u32x2 r = STEP == 4 ? __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(x, x, false, false))
                                  : __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(x, x, false, false));
        return {r.x, r.y};
    }
}

template <int STEP>
__device__ __forceinline__ Sides<float> sides(float x) {
    const Sides<uint32_t> r = sides<STEP>(__builtin_bit_cast(uint32_t, x));
    return {__builtin_bit_cast(float, r.a), __builtin_bit_cast(float, r.b)};
}

template <int STEP>
__device__ __forceinline__ Sides<double> sides(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const Sides<uint32_t> lo = sides<STEP>((uint32_t)u), hi = sides<STEP>((uint32_t)(u >> 32));
    return {__builtin_bit_cast(double, (uint64_t)lo.a | (uint64_t)hi.a << 32),
            __builtin_bit_cast(double, (uint64_t)lo.b | (uint64_t)hi.b << 32)};
}

template <int STEP, typename T, typename Op>
__device__ __forceinline__ T reduce_step(T x, Op op) {
    const Sides<T> r = sides<STEP>(x);
    return op(r.a, r.b);
}

// reduction over groups of LANES lanes, the same value in every lane of a group
template <int LANES, typename T, typename Op>
__device__ __forceinline__ T lanes_reduce(T x, Op op) {
    if constexpr (LANES > 1) x = reduce_step<0>(x, op);
    if constexpr (LANES > 2) x = reduce_step<1>(x, op);
    if constexpr (LANES > 4) x = reduce_step<2>(x, op);
    if constexpr (LANES > 8) x = reduce_step<3>(x, op);
    if constexpr (LANES > 16) x = reduce_step<4>(x, op);
    if constexpr (LANES > 32) x = reduce_step<5>(x, op);
    return x;
}

template <int LANES, typename T>
__device__ __forceinline__ T lanes_sum(T x) {
    return lanes_reduce<LANES>(x, [](T a, T b) { return a + b; });
}

__device__ __forceinline__ double wave_sum(double x) { return lanes_sum<kWave>(x); }

// sums of N doubles over a workgroup of NT threads, in every thread (every
// thread takes part; `lds` holds N * NT / 64 doubles and may be reused after
// the next barrier)
template <int NT, int N>
__device__ __forceinline__ void block_sum(double (&x)[N], double* lds) {
    constexpr int W = NT / kWave;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = wave_sum(x[i]);
    if constexpr (W == 1) return;
    const int w = threadIdx.x / kWave;
    if (lane_id() == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) lds[i * W + w] = x[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = lanes_sum<W>(lds[i * W + lane_id() % W]);
    __syncthreads();
}

// Last arrival of a launch's workgroups: true in every thread of the one that
// drew the last ticket.  What the first wavefront stored with store_agent before
// is at the device's point of coherence by then (its stores are waited for
// before the ticket is drawn), where load_agent reads it, so no fence, and with
// it no write-back of the L2 under the outputs, is needed.  An atomic on one word
// takes 13 ns after the one before it (512 workgroups: 7 us), so more than 32
// workgroups draw from 32 words, and the last of each from the common one.  The
// tickets are left at 0.
__device__ __forceinline__ void store_agent(double* p, double v) {
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ double load_agent(const double* p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ bool draw_last(uint32_t* ticket, uint32_t total) {
    const bool last = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == total - 1;
    if (last) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return last;
}

// one lane's draw of a workgroup's (or a row's) ticket `k` of `total`
__device__ __forceinline__ bool draw_ticket(WorkspaceHead* head, uint32_t k, uint32_t total) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the stores before it are acknowledged
    uint32_t words = total;
    if (total > kTicketGroups) {
        const uint32_t g = k % kTicketGroups;
        if (!draw_last(&head->group[g].ticket, (total - g + kTicketGroups - 1) / kTicketGroups)) return false;
        words = kTicketGroups;
    }
    return draw_last(&head->ticket, words);
}

__device__ __forceinline__ bool last_block(WorkspaceHead* head, uint32_t block, uint32_t total) {
    __shared__ bool s_last;
    if (threadIdx.x == 0) s_last = draw_ticket(head, block, total);
    __syncthreads();
    return s_last;
}

// The 8 statistics from the sums over every token.
__device__ __forceinline__ void write_policy_stats(const PolicyTerms& o, const double* v, uint32_t tokens, float* stats) {
    const double n = tokens > 0 ? (double)tokens : 1.0;
    double loss = v[0];
    if (o.kl != 0.0f) loss += (double)o.kl * v[1];
    if (o.ent != 0.0f) loss -= (double)o.ent * v[2];
    stats[0] = (float)(o.scale * loss);
    stats[1] = (float)v[0];
    stats[2] = (float)v[1];
    stats[3] = (float)v[2];
    stats[4] = (float)(v[3] / n);
    stats[5] = (float)(-v[4] / n);
    stats[6] = (float)(v[5] / n);
    stats[7] = (float)tokens;
}

// this lane's share (every step-th from `first`) of the sums in n slots
__device__ __forceinline__ void sum_slots(const double* slots, uint32_t first, uint32_t step, uint32_t n, double (&t)[kPolicySums]) {
#pragma unroll
    for (int i = 0; i < kPolicySums; ++i) t[i] = 0.0;
    for (uint32_t k = first; k < n; k += step) {
        double p[kPolicySums];
#pragma unroll
        for (int i = 0; i < kPolicySums; ++i) p[i] = load_agent(slots + (int64_t)k * kPolicySums + i);
#pragma unroll
        for (int i = 0; i < kPolicySums; ++i) t[i] += p[i];
    }
}

// Batches of few rows (at most kPolicyBlocks): the row's own workgroup or
// wavefront leaves its sums in slot n, and the last row's first wavefront adds
// the slots up, in a fixed order.  Called by that first wavefront of every row,
// lane 0 holding the row's values (`on`: it counts).
__device__ __forceinline__ void finish_row(const PolicyArgs& a, uint32_t n, bool on, const TokenLoss& t, double w, float entropy) {
    const uint32_t rows = (uint32_t)(a.shape.B * a.shape.T);
    const uint32_t tokens = a.mask ? (uint32_t)a.head->counts : rows;
    const int lane = threadIdx.x % kWave;
    bool last = false;
    if (lane == 0) {
        TokenSums one;
        one.add(on, t, entropy);
        PolicySums s;
        s.add(w, one);
#pragma unroll
        for (int i = 0; i < kPolicySums; ++i) store_agent(a.partial + (int64_t)n * kPolicySums + i, s.v[i]);
        last = draw_ticket(a.head, n, rows);
    }
    if (!__builtin_amdgcn_readfirstlane((int)last)) return;
    double v[kPolicySums];
    sum_slots(a.partial, lane, kWave, rows, v);
#pragma unroll
    for (int i = 0; i < kPolicySums; ++i) v[i] = wave_sum(v[i]);
    if (lane == 0) {
        write_policy_stats(a.o, v, tokens, a.stats);
        a.head->counts = 0;  // for the next call
    }
}

// All sums are in 64 bits (the partial sums of terms of both signs may be far
// larger than their total, and past the largest float): lane i of the first
// wavefront adds the wavefronts' i-th sums and stores them in the workgroup's
// slot; the last workgroup adds the slots up, in a fixed order, writes the
// statistics and clears the counters.
template <int NT>
__device__ __forceinline__ void finish_policy(const PolicyArgs& a, const PolicySums& s, uint32_t tokens, bool counted,
                                              double* lds) {
    constexpr int W = NT / kWave;
    double v[kPolicySums];
#pragma unroll
    for (int i = 0; i < kPolicySums; ++i) v[i] = wave_sum(s.v[i]);
    if (lane_id() == 0) {
#pragma unroll
        for (int i = 0; i < kPolicySums; ++i) lds[i * W + threadIdx.x / kWave] = v[i];
    }
    __syncthreads();
    double mine = 0.0;
    if (threadIdx.x < kPolicySums) {
#pragma unroll
        for (int k = 0; k < W; ++k) mine += lds[threadIdx.x * W + k];
    }
    if (gridDim.x == 1) {
        __syncthreads();
        if (threadIdx.x < kPolicySums) lds[threadIdx.x] = mine;
        __syncthreads();
        if (threadIdx.x == 0) write_policy_stats(a.o, lds, tokens, a.stats);
    } else {
        if (threadIdx.x < kPolicySums) store_agent(a.partial + (int64_t)blockIdx.x * kPolicySums + threadIdx.x, mine);
        if (!last_block(a.head, blockIdx.x, gridDim.x)) return;
        double t[kPolicySums];
        sum_slots(a.partial, threadIdx.x, NT, gridDim.x, t);
        block_sum<NT, kPolicySums>(t, lds);
        if (threadIdx.x == 0) write_policy_stats(a.o, t, tokens, a.stats);
    }
    if (counted && threadIdx.x == 0) a.head->counts = 0;  // for the next call
}

}  // namespace conduit
