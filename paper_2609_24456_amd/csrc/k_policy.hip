// The clipped policy loss with a KL term over a [B, T] batch of tokens, and its
// gradient with respect to the log-probabilities (conduit_policy_loss).
//
// Per token (policy_token): r = exp(logp - old), the pessimistic one of -A r and
// -A clip(r), with a ceiling of -A dual for A < 0, plus kl_coef times
// exp(x) - 1 - x at x = ref - logp, minus entropy_coef times the entropy; the
// loss is the weighted sum over the tokens that the mask counts.  The weight
// needs the number of those tokens (of the whole batch, or of the row and the
// number of rows with any), so a batch with a mask takes a count first, which
// reads one byte a token; up to kSmallChunks chunks one workgroup counts and
// sums by itself, in one launch.
//
// Bytes bound it: 20 read and 8 written a token beside the mask.  Sums run in
// fp64 and are joined in a fixed order (finish_policy), so a call's results do
// not depend on the order in which workgroups end.
#include "loss_dev.h"

namespace conduit {

namespace {

constexpr int kPolicyThreads = 256;
constexpr int kSmallThreads = 512;
constexpr int kChunk = 4;             // tokens a lane takes at once
constexpr int kSmallChunks = 4096;    // most chunks, and most rows, that one workgroup takes by itself
constexpr int kCountBytes = 16 * kWave;  // mask bytes a wavefront counts at once

struct Chunks {
    int64_t T;
    uint32_t total;   // chunks of the batch
    uint32_t per_row;
    Div31 by_row;
};

__device__ __forceinline__ void load4(const float* p, int n, float (&v)[kChunk]) {
    if (n == kChunk) {
        __builtin_memcpy(v, p, 16);
    } else {
#pragma unroll
        for (int i = 0; i < kChunk; ++i) v[i] = i < n ? p[i] : 0.0f;
    }
}

__device__ __forceinline__ void store4(float* p, int n, const float (&v)[kChunk]) {
    if (n == kChunk) {
        __builtin_memcpy(p, v, 16);
    } else {
#pragma unroll
        for (int i = 0; i < kChunk; ++i)
            if (i < n) p[i] = v[i];
    }
}

__device__ __forceinline__ uint32_t load_mask4(const uint8_t* p, int n) {
    uint32_t m = 0;
    if (n == kChunk) {
        __builtin_memcpy(&m, p, 4);
    } else {
#pragma unroll
        for (int i = 0; i < kChunk; ++i)
            if (i < n) m |= (uint32_t)p[i] << (8 * i);
    }
    return m;
}

// number of non-zero bytes
__device__ __forceinline__ uint32_t count_bytes(uint32_t x) {
    return __builtin_popcount((((x & 0x7f7f7f7fu) + 0x7f7f7f7fu) | x) & 0x80808080u);
}

__device__ __forceinline__ void policy_chunk(const PolicyArgs& a, int64_t at, uint32_t mask, int n, double w,
                                             PolicySums& sums) {
    float lp[kChunk], old[kChunk], ref[kChunk], adv[kChunk], ent[kChunk], g[kChunk], h[kChunk];
    load4(a.logp + at, n, lp);
    load4(a.adv + at, n, adv);
    if (a.old_logp) load4(a.old_logp + at, n, old);
    if (a.ref_logp) load4(a.ref_logp + at, n, ref);
    if (a.entropy) load4(a.entropy + at, n, ent);
    const float wf = (float)(w * a.o.scale), we = -a.o.ent * wf;
#pragma unroll
    for (int i = 0; i < kChunk; ++i) {
        g[i] = h[i] = 0.0f;
        bool on = i < n && (mask >> (8 * i) & 255u) != 0;
        if (on && a.tokens) {
            const int32_t tok = a.tokens[at + i];
            on = tok >= 0 && tok < a.V;
        }
        if (!on) continue;
        const TokenLoss t = policy_token(a.o, lp[i], a.old_logp != nullptr, a.old_logp ? old[i] : 0.0f,
                                         a.ref_logp != nullptr, a.ref_logp ? ref[i] : 0.0f, adv[i]);
        sums.add(w, t, a.entropy ? ent[i] : 0.0f);
        g[i] = wf * t.slope;
        h[i] = we;
    }
    if (a.dlogp) store4(a.dlogp + at, n, g);
    if (a.dentropy) store4(a.dentropy + at, n, h);
}

template <int NT, bool SMALL>
__global__ __launch_bounds__(NT) void k_policy_loss(PolicyArgs a, Chunks ch, bool counted) {
    __shared__ double lds[kPolicySums * NT / kWave];
    __shared__ uint32_t s_count[SMALL ? kSmallChunks : 1];
    uint32_t tokens = (uint32_t)(a.shape.B * a.shape.T), rows = (uint32_t)a.shape.B;
    const uint32_t first = blockIdx.x * NT + threadIdx.x, step = gridDim.x * NT;
    auto place = [&](uint32_t c, uint32_t* b, int64_t* at, int* n) {
        *b = div31(c, ch.by_row);
        const int64_t t = (int64_t)(c - *b * ch.per_row) * kChunk;
        *at = (int64_t)*b * a.shape.stride + t;
        *n = ch.T - t < kChunk ? (int)(ch.T - t) : kChunk;
    };
    if (SMALL && a.mask) {
        for (uint32_t b = threadIdx.x; b < (uint32_t)a.shape.B; b += NT) s_count[b] = 0;
        __syncthreads();
        for (uint32_t c = first; c < ch.total; c += step) {
            uint32_t b;
            int64_t at;
            int n;
            place(c, &b, &at, &n);
            const uint32_t k = count_bytes(load_mask4(a.mask + at, n));
            if (k) atomicAdd(&s_count[b], k);
        }
        __syncthreads();
        double t[2] = {0, 0};
        for (uint32_t b = threadIdx.x; b < (uint32_t)a.shape.B; b += NT) {
            t[0] += s_count[b];
            t[1] += s_count[b] != 0;
        }
        block_sum<NT, 2>(t, lds);
        tokens = (uint32_t)t[0];
        rows = (uint32_t)t[1];
    } else if (counted) {
        tokens = a.head->tokens;
        rows = a.head->rows;
    }
    PolicySums sums;
    const double flat = token_weight(a.o, tokens, rows, (uint32_t)a.shape.T);
    for (uint32_t c = first; c < ch.total; c += step) {
        uint32_t b;
        int64_t at;
        int n;
        place(c, &b, &at, &n);
        const uint32_t mask = a.mask ? load_mask4(a.mask + at, n) : 0x01010101u;
        double w = flat;
        if (a.o.reduction == CONDUIT_SEQUENCE_MEAN && a.mask)
            w = token_weight(a.o, tokens, rows, SMALL ? s_count[b] : a.row_count[b]);
        policy_chunk(a, at, mask, n, w, sums);
    }
    finish_policy<NT>(a, sums, tokens, counted, lds);
}

// non-zero mask bytes of [t0, t0 + 16) below T
__device__ __forceinline__ uint32_t count16(const uint8_t* row, int64_t t0, int64_t T) {
    if (t0 + 16 <= T) {
        uint32_t v[4];
        __builtin_memcpy(v, row + t0, 16);
        return count_bytes(v[0]) + count_bytes(v[1]) + count_bytes(v[2]) + count_bytes(v[3]);
    }
    uint32_t k = 0;
    for (int64_t t = t0; t < T; ++t) k += row[t] != 0;
    return k;
}

// Counted tokens of the batch: wavefronts take parts of kCountBytes mask bytes
// of a row.  Whole numbers, so the order of the additions is free.
__global__ __launch_bounds__(kPolicyThreads) void k_token_count(PolicyArgs a, uint32_t items, uint32_t per_row,
                                                                Div31 by_row) {
    __shared__ double lds[kPolicyThreads / kWave];
    const uint32_t waves = gridDim.x * (kPolicyThreads / kWave);
    double tokens[1] = {0};
    for (uint32_t i = blockIdx.x * (kPolicyThreads / kWave) + threadIdx.x / kWave; i < items; i += waves) {
        const uint32_t b = div31(i, by_row);
        const int64_t t0 = (int64_t)(i - b * per_row) * kCountBytes + lane_id() * 16;
        tokens[0] += count16(a.mask + (int64_t)b * a.shape.stride, t0, a.shape.T);
    }
    block_sum<kPolicyThreads, 1>(tokens, lds);
    if (threadIdx.x == 0 && tokens[0] > 0) atomicAdd(&a.head->tokens, (uint32_t)tokens[0]);
}

// Counted tokens of every row, of the batch, and the rows with any: NT threads a
// row, kRows rows a workgroup at once.
template <int NT, int kRows>
__global__ __launch_bounds__(NT * kRows) void k_row_count(PolicyArgs a) {
    constexpr int kAll = NT * kRows;
    __shared__ double lds[2 * kAll / kWave];
    double sums[2] = {0, 0};
    const int tid = threadIdx.x % NT;
    for (int64_t first = (int64_t)blockIdx.x * kRows; first < a.shape.B; first += (int64_t)gridDim.x * kRows) {
        const int64_t b = first + threadIdx.x / NT;
        double k[1] = {0};
        if (b < a.shape.B) {
            const uint8_t* row = a.mask + b * a.shape.stride;
            for (int64_t t0 = 16 * (int64_t)tid; t0 < a.shape.T; t0 += 16 * NT) k[0] += count16(row, t0, a.shape.T);
        }
        if constexpr (kRows > 1) k[0] = wave_sum(k[0]);  // NT = 64: a wavefront a row
        else block_sum<NT, 1>(k, lds);
        if (tid == 0 && b < a.shape.B) {
            a.row_count[b] = (uint32_t)k[0];
            sums[0] += k[0];
            sums[1] += k[0] > 0;
        }
    }
    block_sum<kAll, 2>(sums, lds);
    if (threadIdx.x == 0 && sums[0] > 0) {
        atomicAdd(&a.head->tokens, (uint32_t)sums[0]);
        atomicAdd(&a.head->rows, (uint32_t)sums[1]);
    }
}

}  // namespace

// A row of up to 1,024 tokens takes a wavefront, up to 16,384 a workgroup of 256
// lanes, a longer one 1,024 lanes: 16 bytes a lane and round.
hipError_t launch_token_count(const PolicyArgs& a, hipStream_t s) {
    auto grid = [](int64_t want) { return dim3((unsigned)(want < kPolicyBlocks ? want : kPolicyBlocks)); };
    const int64_t B = a.shape.B, T = a.shape.T;
    if (a.o.reduction == CONDUIT_SEQUENCE_MEAN) {
        if (T <= kCountBytes) hipLaunchKernelGGL((k_row_count<64, 4>), grid((B + 3) / 4), dim3(256), 0, s, a);
        else if (T <= 16 * kCountBytes) hipLaunchKernelGGL((k_row_count<256, 1>), grid(B), dim3(256), 0, s, a);
        else hipLaunchKernelGGL((k_row_count<1024, 1>), grid(B), dim3(1024), 0, s, a);
        return hipGetLastError();
    }
    const uint32_t per_row = (uint32_t)((T + kCountBytes - 1) / kCountBytes);
    const int64_t items = B * per_row;
    hipLaunchKernelGGL(k_token_count, grid((items + kPolicyThreads / kWave - 1) / (kPolicyThreads / kWave)),
                       dim3(kPolicyThreads), 0, s, a, (uint32_t)items, per_row, make_div31(per_row));
    return hipGetLastError();
}

// counted: the counts stand in the workspace already (and are cleared here)
hipError_t launch_policy_loss(const PolicyArgs& args, bool counted, hipStream_t s) {
    PolicyArgs a = args;
    // rows that follow each other without a gap are one, unless each has its own weight
    if (a.shape.stride == a.shape.T && (a.o.reduction != CONDUIT_SEQUENCE_MEAN || !a.mask))
        a.shape = make_shape(1, a.shape.B * a.shape.T, a.shape.B * a.shape.T);
    Chunks ch;
    ch.T = a.shape.T;
    ch.per_row = (uint32_t)((a.shape.T + kChunk - 1) / kChunk);
    ch.total = (uint32_t)a.shape.B * ch.per_row;
    ch.by_row = make_div31(ch.per_row > 0 ? ch.per_row : 1);
    if (!counted && ch.total <= (uint32_t)kSmallChunks) {
        hipLaunchKernelGGL((k_policy_loss<kSmallThreads, true>), dim3(1), dim3(kSmallThreads), 0, s, a, ch, false);
        return hipGetLastError();
    }
    if (!counted && a.mask) {
        const hipError_t e = launch_token_count(a, s);
        if (e != hipSuccess) return e;
        counted = true;
    }
    const uint32_t want = (ch.total + kPolicyThreads - 1) / kPolicyThreads;
    const uint32_t grid = want < (uint32_t)kPolicyBlocks ? want : (uint32_t)kPolicyBlocks;
    hipLaunchKernelGGL((k_policy_loss<kPolicyThreads, false>), dim3(grid), dim3(kPolicyThreads), 0, s, a, ch, counted);
    return hipGetLastError();
}

}  // namespace conduit
