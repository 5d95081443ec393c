// The preference loss over P pairs of sequences and its gradient
// (conduit_preference_loss).  Rows 0..P-1 are the chosen answers, P..2P-1 the
// rejected ones.
//
//   d_i = sum over the row's counted tokens of logp - ref  [/ their number]
//   u   = beta (d_chosen - d_rejected)
//   sigmoid: -(1 - e) log s(u) - e log s(-u);  squared: (u / beta - 1 / (2 beta))^2
//   loss = scale * mean over the pairs
//
// The gradient is the same number at every counted token of a row, of opposite
// sign in the two rows, so the second pass over a row reads only its mask.  It
// waits for both rows' sums: one workgroup takes a pair by itself, or, where
// there are too few pairs to fill the GPU, one launch adds up parts of rows and
// a second joins a pair's parts and writes the gradient of one part each.
// 9 bytes are read and 4 written a token, but latency bounds the sizes that occur:
// 128 pairs of 2,048 tokens 6.7 us, 2 pairs of 65,537 (two launches) 9.6.
#include "loss_dev.h"

namespace conduit {

namespace {

constexpr int kPairThreads = 512;
constexpr int kPartTokens = 4096;  // tokens of one part of a row

struct RowSum {
    double v[2] = {0, 0};  // sum, tokens
};

// this thread's share of tokens [t0, t1) of row b
__device__ __forceinline__ RowSum row_sum(const PreferenceArgs& a, int64_t b, int64_t t0, int64_t t1) {
    RowSum r;
    const float* lp = a.logp + b * a.stride;
    const float* rf = a.ref ? a.ref + b * a.stride : nullptr;
    const uint8_t* mk = a.mask ? a.mask + b * a.stride : nullptr;
    for (int64_t t = t0 + 4 * (int64_t)threadIdx.x; t < t1; t += 4 * kPairThreads) {
        if (t + 4 <= t1) {
            float x[4], y[4] = {0, 0, 0, 0};
            uint32_t m = 0x01010101u;
            __builtin_memcpy(x, lp + t, 16);
            if (rf) __builtin_memcpy(y, rf + t, 16);
            if (mk) __builtin_memcpy(&m, mk + t, 4);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (m >> (8 * i) & 255u) {
                    r.v[0] += (double)x[i] - (double)y[i];
                    r.v[1] += 1.0;
                }
        } else {
            for (int64_t k = t; k < t1; ++k)
                if (!mk || mk[k]) {
                    r.v[0] += (double)lp[k] - (rf ? (double)rf[k] : 0.0);
                    r.v[1] += 1.0;
                }
        }
    }
    return r;
}

__device__ __forceinline__ void write_gradient(const PreferenceArgs& a, int64_t b, int64_t t0, int64_t t1, float q) {
    float* out = a.dlogp + b * a.stride;
    const uint8_t* mk = a.mask ? a.mask + b * a.stride : nullptr;
    for (int64_t t = t0 + 4 * (int64_t)threadIdx.x; t < t1; t += 4 * kPairThreads) {
        if (t + 4 <= t1) {
            uint32_t m = 0x01010101u;
            if (mk) __builtin_memcpy(&m, mk + t, 4);
            float g[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) g[i] = m >> (8 * i) & 255u ? q : 0.0f;
            __builtin_memcpy(out + t, g, 16);
        } else {
            for (int64_t k = t; k < t1; ++k) out[k] = !mk || mk[k] ? q : 0.0f;
        }
    }
}

struct Pair {
    double loss, u, chosen, rejected, tokens;
    double q_chosen, q_rejected;  // gradient at the rows' tokens
};

__device__ __forceinline__ Pair pair_loss(const PreferenceArgs& a, const double (&s)[4]) {
    Pair p;
    const double nc = a.length_norm && s[1] > 0 ? s[1] : 1.0, nr = a.length_norm && s[3] > 0 ? s[3] : 1.0;
    const double beta = a.beta, dc = s[0] / nc, dr = s[2] / nr;
    p.chosen = beta * dc;
    p.rejected = beta * dr;
    p.u = beta * (dc - dr);
    double q;
    if (a.squared) {
        const double off = dc - dr - 0.5 / beta;
        p.loss = off * off;
        q = 2.0 * off;
    } else {
        // with t = exp(-|u|): -log s(u) = max(-u, 0) + log(1 + t), s(u) = 1 / (1 + t) for u > 0, else t / (1 + t)
        const double e = a.smoothing, t = exp(-fabs(p.u)), z = log1p(t), low = t / (1.0 + t), high = 1.0 / (1.0 + t);
        p.loss = (1.0 - e) * ((p.u < 0 ? -p.u : 0.0) + z);
        if (e > 0.0) p.loss += e * ((p.u > 0 ? p.u : 0.0) + z);
        q = beta * (p.u > 0 ? e * high - (1.0 - e) * low : e * low - (1.0 - e) * high);
    }
    p.tokens = s[1] + s[3];
    const double each = a.scale * q / (double)a.P;
    p.q_chosen = each / nc;
    p.q_rejected = -each / nr;
    return p;
}

__device__ __forceinline__ void write_pair(const PreferenceArgs& a, int64_t p, const Pair& r) {
    a.loss[p] = (float)r.loss;
    if (a.chosen) a.chosen[p] = (float)r.chosen;
    if (a.rejected) a.rejected[p] = (float)r.rejected;
    store_agent(a.pair + 4 * p, r.loss);
    store_agent(a.pair + 4 * p + 1, r.u);
    store_agent(a.pair + 4 * p + 2, r.u > 0 ? 1.0 : 0.0);
    store_agent(a.pair + 4 * p + 3, r.tokens);
}

// the last workgroup's means over the pairs
__device__ __forceinline__ void write_means(const PreferenceArgs& a, double* lds) {
    double t[4] = {0, 0, 0, 0};
    for (int64_t p = threadIdx.x; p < a.P; p += kPairThreads) {
#pragma unroll
        for (int i = 0; i < 4; ++i) t[i] += load_agent(a.pair + 4 * p + i);
    }
    block_sum<kPairThreads, 4>(t, lds);
    if (threadIdx.x == 0) {
        const double n = (double)a.P;
        a.stats[0] = (float)(a.scale * t[0] / n);
        a.stats[1] = (float)(t[2] / n);
        a.stats[2] = (float)(t[1] / n);
        a.stats[3] = (float)t[3];
    }
}

__global__ __launch_bounds__(kPairThreads) void k_preference(PreferenceArgs a) {
    __shared__ double lds[4 * kPairThreads / kWave];
    const int64_t p = block_number();
    if (p >= a.P) return;
    const RowSum c = row_sum(a, p, 0, a.T), r = row_sum(a, a.P + p, 0, a.T);
    double s[4] = {c.v[0], c.v[1], r.v[0], r.v[1]};
    block_sum<kPairThreads, 4>(s, lds);
    const Pair x = pair_loss(a, s);
    if (threadIdx.x == 0) write_pair(a, p, x);
    if (a.dlogp) {
        write_gradient(a, p, 0, a.T, (float)x.q_chosen);
        write_gradient(a, a.P + p, 0, a.T, (float)x.q_rejected);
    }
    if (last_block(a.head, (uint32_t)p, (uint32_t)a.P)) write_means(a, lds);
}

// parts of rows: grid (parts, 2 P)
__global__ __launch_bounds__(kPairThreads) void k_preference_sums(PreferenceArgs a) {
    __shared__ double lds[2 * kPairThreads / kWave];
    const int64_t b = blockIdx.y, t0 = (int64_t)blockIdx.x * kPartTokens;
    RowSum r = row_sum(a, b, t0, t0 + kPartTokens < a.T ? t0 + kPartTokens : a.T);
    block_sum<kPairThreads, 2>(r.v, lds);
    if (threadIdx.x == 0) {
        a.partial[2 * (b * a.parts + blockIdx.x)] = r.v[0];
        a.partial[2 * (b * a.parts + blockIdx.x) + 1] = r.v[1];
    }
}

__global__ __launch_bounds__(kPairThreads) void k_preference_join(PreferenceArgs a) {
    __shared__ double lds[4 * kPairThreads / kWave];
    const int64_t b = blockIdx.y, p = b < a.P ? b : b - a.P, t0 = (int64_t)blockIdx.x * kPartTokens;
    double s[4] = {0, 0, 0, 0};
    for (int k = threadIdx.x; k < a.parts; k += kPairThreads) {
        const double* c = a.partial + 2 * (p * a.parts + k);
        const double* r = a.partial + 2 * ((a.P + p) * a.parts + k);
        s[0] += c[0];
        s[1] += c[1];
        s[2] += r[0];
        s[3] += r[1];
    }
    block_sum<kPairThreads, 4>(s, lds);
    const Pair x = pair_loss(a, s);
    if (a.dlogp)
        write_gradient(a, b, t0, t0 + kPartTokens < a.T ? t0 + kPartTokens : a.T,
                       (float)(b < a.P ? x.q_chosen : x.q_rejected));
    if (blockIdx.x == 0 && b < a.P) {  // one workgroup a pair
        if (threadIdx.x == 0) write_pair(a, p, x);
        if (last_block(a.head, (uint32_t)p, (uint32_t)a.P)) write_means(a, lds);
    }
}

}  // namespace

// Parts of a row, 1: a workgroup takes a pair by itself.  Rows are split where
// the pairs alone would leave half of the compute units without one.
int preference_parts(int64_t P, int64_t T) {
    if (2 * P > device_cus() || T <= kPartTokens) return 1;
    return (int)((T + kPartTokens - 1) / kPartTokens);
}

hipError_t launch_preference_loss(const PreferenceArgs& a, hipStream_t s) {
    if (a.parts <= 1) {
        hipLaunchKernelGGL(k_preference, grid_of(a.P, kPairThreads), dim3(kPairThreads), 0, s, a);
        return hipGetLastError();
    }
    const dim3 grid((unsigned)a.parts, (unsigned)(2 * a.P));
    hipLaunchKernelGGL(k_preference_sums, grid, dim3(kPairThreads), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_preference_join, grid, dim3(kPairThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace conduit
