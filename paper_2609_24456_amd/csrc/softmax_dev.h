// Softmax statistics of rows of scores, in parts that can be joined
// (k_logits.hip, k_head.hip).  The scores are c x, c = log2(e) / temperature.
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

// what a row's statistics say
struct RowValues {
    float base;     // m, or 0 in a row without weight
    float inv_s;    // 1 / S, 0 in a row without weight
    float log2_s;
    float lse, entropy, logp, one_minus_p;
};

// inv_lo: what the rounding of 1 / temperature to inv_t left, which at a large
// maximum is as much as the rounding of lse itself (0: not counted)
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
    r.lse = fmaf(st.m, inv_t, fmaf(st.m, inv_lo, r.log2_s * kLn2));
    r.entropy = (r.log2_s - st.u * r.inv_s) * kLn2;
    r.logp = ((xa - st.m) * c - r.log2_s) * kLn2;
    r.one_minus_p = -expm1_fast(r.logp);
    return r;
}

}  // namespace conduit
