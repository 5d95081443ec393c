// Softmax statistics of rows of scores, in parts that can be joined
// (k_logits.hip, k_head.hip, k_top.hip, k_listed.hip).  The scores are c x, c = log2(e) / temperature.
#pragma once

#include "loss_dev.h"

namespace conduit {

constexpr float kNone = -INFINITY;
constexpr float kFloor = -1024.0f;  // 2^d is 0 below; keeps 0 * d from being NaN at d = -inf

// Running statistics of a part of a row: m = max x, s = sum 2^d, u = sum 2^d d
// with d = c (x - m).
struct Stat {
    float m, s, u;
};

__device__ __forceinline__ Stat no_stat() { return Stat{kNone, 0.0f, 0.0f}; }

__device__ __forceinline__ Stat join(const Stat& a, const Stat& b, float c) {
    Stat r;
    r.m = a.m > b.m ? a.m : b.m;
    // equal maxima, -inf ones among them, have no distance
    const float da = a.m == r.m ? 0.0f : (a.m - r.m) * c, db = b.m == r.m ? 0.0f : (b.m - r.m) * c;
    const float ea = exp2_fast(da), eb = exp2_fast(db);
    const float sa = a.s * ea, sb = b.s * eb;
    r.s = sa + sb;
    r.u = fmaf(a.u, ea, sa * fmaxf(da, kFloor)) + fmaf(b.u, eb, sb * fmaxf(db, kFloor));
    return r;
}

template <int N>
__device__ __forceinline__ float top_of(const float (&x)[N], float top) {
#pragma unroll
    for (int i = 0; i < N; ++i) top = fmaxf(top, x[i]);
    return top;
}

// the running maximum becomes at least `top`
__device__ __forceinline__ void raise(Stat& st, float top, float c) {
    if (top > st.m) {
        const float d = (st.m - top) * c, e = exp2_fast(d);
        st.u = fmaf(st.s, fmaxf(d, kFloor), st.u) * e;
        st.s *= e;
        st.m = top;
    }
}

// elements that are no larger than the running maximum
template <int N>
__device__ __forceinline__ void add(Stat& st, const float (&x)[N], float c) {
    const float base = st.m == kNone ? 0.0f : st.m;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float d = (x[i] - base) * c, e = exp2_fast(d);
        st.s += e;
        st.u = fmaf(e, fmaxf(d, kFloor), st.u);
    }
}

template <int N>
__device__ __forceinline__ void accumulate(Stat& st, const float (&x)[N], float c) {
    raise(st, top_of(x, kNone), c);
    add(st, x, c);
}

// joined over groups of LANES lanes, in every lane: their largest maximum first,
// then one rescaling a lane and plain sums
template <int LANES>
__device__ __forceinline__ Stat join_lanes(const Stat& a, float c) {
    Stat r;
    r.m = lanes_reduce<LANES>(a.m, [](float x, float y) { return x > y ? x : y; });
    const float d = a.m == r.m ? 0.0f : (a.m - r.m) * c, e = exp2_fast(d), s = a.s * e;
    r.s = lanes_sum<LANES>(s);
    r.u = lanes_sum<LANES>(fmaf(a.u, e, s * fmaxf(d, kFloor)));
    return r;
}

// log p of a score, by the log-normaliser given.  The scores are far from 0 where log p
// need not be, so a rounded 1 / temperature would cost |z| 2^-25 of p: its rest goes
// along, from the score `lowest` on (below, -infinity among them, p is 0 whatever the
// rest, which times the score could be no number, or the other infinity).
struct LogP {
    float inv_t, inv_lo, lowest, lse;
    __device__ __forceinline__ float of(float x) const { return fmaf(x, inv_t, fmaf(fmaxf(x, lowest), inv_lo, -lse)); }
};

// what a row's statistics say
struct RowValues {
    float base;     // m, or 0 in a row without weight
    float inv_s;    // 1 / S, 0 in a row without weight
    float log2_s;
    float lse, entropy, logp, one_minus_p;
};

// log p of a score that is `d` from the largest (0 or below).  In powers of two it may be
// past the largest float where log p is not: choices at the type's lowest value.
__device__ __forceinline__ float log_p_from(float d, float c, float inv_t, float log2_s) {
    const float r = (d * c - log2_s) * kLn2;
    return r == kNone ? fmaf(d, inv_t, -log2_s * kLn2) : r;
}

// max x / temperature + log_s.  inv_lo: what the rounding of 1 / temperature to inv_t
// left, which at a large maximum is as much as the rounding of lse itself (0: not
// counted).  Where its share is past the largest float the score is by far, and lse is
// the score's infinity, whatever the share's sign.
__device__ __forceinline__ float log_normaliser(float m, float log_s, float inv_t, float inv_lo) {
    const float lo = fmaf(m, inv_lo, log_s);
    return fabsf(lo) == INFINITY ? m * inv_t : fmaf(m, inv_t, lo);
}

__device__ __forceinline__ RowValues row_values(const Stat& st, float xa, float c, float inv_t, float inv_lo) {
    RowValues r;
    if (st.s == 0.0f) {
        r.base = r.inv_s = r.log2_s = r.entropy = r.one_minus_p = 0.0f;
        r.lse = r.logp = kNone;
        return r;
    }
    r.base = st.m;
    r.inv_s = 1.0f / st.s;
    r.log2_s = log2_fast(st.s);
    r.lse = log_normaliser(st.m, r.log2_s * kLn2, inv_t, inv_lo);
    r.entropy = (r.log2_s - st.u * r.inv_s) * kLn2;
    r.logp = log_p_from(xa - st.m, c, inv_t, r.log2_s);
    r.one_minus_p = -expm1_fast(r.logp);
    return r;
}

}  // namespace conduit
