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
// not depend on the order in which workgroups end.  8 x 333 tokens: 6.6 us, the
// host's call; 256 x 4,096 masked: 17.1 us (18 MB would take 3.7), traced alone
// 4.6 for the count and 13.2 for the tokens, the tickets and the last
// workgroup's sums (with lanes added up in fp32 12.2).
#include "loss_dev.h"

namespace conduit {

namespace {

constexpr int kPolicyThreads = 512;
constexpr int kSmallThreads = 1024;
constexpr int kChunk = 4;             // tokens a lane takes at once
constexpr int kSmallChunks = 2048;    // most chunks, and most rows, that one workgroup takes by itself
constexpr int kCountThreads = 1024;
constexpr int kCountBlocks = 64;      // few: each ends in an atomic on one word

struct Chunks {
    int64_t T;
    uint32_t total;   // chunks of the batch
    uint32_t per_row;
    Div31 by_row;
};

__device__ __forceinline__ void store4(float* p, int n, const float (&v)[kChunk]) {
    if (n == kChunk) {
        __builtin_memcpy(p, v, 16);
    } else {
#pragma unroll
        for (int i = 0; i < kChunk; ++i)
            if (i < n) p[i] = v[i];
    }
}

__device__ __forceinline__ uint32_t mask_tail(const uint8_t* p, int n) {
    uint32_t m = 0;
    for (int i = 0; i < n; ++i) m |= (uint32_t)p[i] << (8 * i);
    return m;
}

// number of non-zero bytes
__device__ __forceinline__ uint32_t count_bytes(uint32_t x) {
    return __builtin_popcount((((x & 0x7f7f7f7fu) + 0x7f7f7f7fu) | x) & 0x80808080u);
}

// a chunk's inputs, loaded ahead of what they wait for
struct ChunkData {
    float lp[kChunk], old[kChunk], ref[kChunk], adv[kChunk], ent[kChunk];
    uint32_t mask;
    int n;
    int64_t at;
    uint32_t row;
};

__device__ __forceinline__ ChunkData load_chunk(const PolicyArgs& a, const Chunks& ch, uint32_t c) {
    ChunkData d;
    d.row = div31(c, ch.by_row);
    const int64_t t = (int64_t)(c - d.row * ch.per_row) * kChunk;
    d.at = (int64_t)d.row * a.shape.stride + t;
    d.n = ch.T - t < kChunk ? (int)(ch.T - t) : kChunk;
    // one branch around all loads: a branch at each would wait for each
    if (d.n == kChunk) {
        d.mask = 0x01010101u;
        if (a.mask) __builtin_memcpy(&d.mask, a.mask + d.at, 4);
        __builtin_memcpy(d.lp, a.logp + d.at, 16);
        __builtin_memcpy(d.adv, a.adv + d.at, 16);
        __builtin_memcpy(d.old, a.old_logp + d.at, 16);
        __builtin_memcpy(d.ref, a.ref_logp + d.at, 16);
        __builtin_memcpy(d.ent, a.entropy + d.at, 16);
    } else {
        d.mask = a.mask ? mask_tail(a.mask + d.at, d.n) : 0x01010101u;
#pragma unroll
        for (int i = 0; i < kChunk; ++i) {
            const int64_t k = d.at + (i < d.n ? i : 0);
            d.lp[i] = a.logp[k];
            d.adv[i] = a.adv[k];
            d.old[i] = a.old_logp[k];
            d.ref[i] = a.ref_logp[k];
            d.ent[i] = a.entropy[k];
        }
    }
    return d;
}

__device__ __forceinline__ ChunkData load_chunk_mask(const PolicyArgs& a, const Chunks& ch, uint32_t c) {
    ChunkData d;
    d.row = div31(c, ch.by_row);
    const int64_t t = (int64_t)(c - d.row * ch.per_row) * kChunk;
    d.n = ch.T - t < kChunk ? (int)(ch.T - t) : kChunk;
    const uint8_t* p = a.mask + (int64_t)d.row * a.shape.stride + t;
    if (d.n == kChunk) __builtin_memcpy(&d.mask, p, 4);
    else d.mask = mask_tail(p, d.n);
    return d;
}

__device__ __forceinline__ void policy_chunk(const PolicyArgs& a, const ChunkData& d, double w, PolicySums& sums) {
    const float wf = (float)(w * a.o.scale), we = -a.o.ent * wf;
    float g[kChunk], h[kChunk];
    TokenSums few;
    int32_t tok[kChunk];
    if (a.tokens) {
#pragma unroll
        for (int i = 0; i < kChunk; ++i) tok[i] = i < d.n ? a.tokens[d.at + i] : -1;
    }
#pragma unroll
    for (int i = 0; i < kChunk; ++i) {
        bool on = (i < d.n) & ((d.mask >> (8 * i) & 255u) != 0);
        if (a.tokens) on = on & (tok[i] >= 0) & (tok[i] < a.V);
        const TokenLoss t = policy_token(a.o, d.lp[i], d.old[i], d.ref[i], d.adv[i]);
        few.add(on, t, a.has_entropy ? d.ent[i] : 0.0f);
        g[i] = on ? wf * t.slope : 0.0f;
        h[i] = on ? we : 0.0f;
    }
    sums.add(w, few);
    if (a.dlogp) store4(a.dlogp + d.at, d.n, g);
    if (a.dentropy) store4(a.dentropy + d.at, d.n, h);
}

template <int NT, bool SMALL>
__global__ __launch_bounds__(NT) void k_policy_loss(PolicyArgs a, Chunks ch, bool counted) {
    __shared__ double lds[kPolicySums * NT / kWave];
    __shared__ uint32_t s_count[SMALL ? kSmallChunks : 1];
    uint32_t tokens = (uint32_t)(a.shape.B * a.shape.T), rows = (uint32_t)a.shape.B;
    const uint32_t first = blockIdx.x * NT + threadIdx.x, step = gridDim.x * NT;
    ChunkData d;
    if (first < ch.total) d = load_chunk(a, ch, first);
    if (SMALL && a.mask) {
        const bool by_row = a.o.reduction == CONDUIT_SEQUENCE_MEAN;
        if (by_row) {
            for (uint32_t b = threadIdx.x; b < (uint32_t)a.shape.B; b += NT) s_count[b] = 0;
            __syncthreads();
        }
        double t[2] = {0, 0};
        for (uint32_t c = first; c < ch.total; c += step) {
            const ChunkData o = c == first ? d : load_chunk_mask(a, ch, c);
            const uint32_t k = count_bytes(o.n == kChunk ? o.mask : o.mask & ((1u << (8 * o.n)) - 1u));
            t[0] += k;
            if (by_row && k && atomicAdd(&s_count[o.row], k) == 0) t[1] += 1.0;
        }
        block_sum<NT, 2>(t, lds);  // (its barriers also end the counting)
        tokens = (uint32_t)t[0];
        rows = (uint32_t)t[1];
    } else if (counted) {
        const uint64_t counts = a.head->counts;
        tokens = (uint32_t)counts;
        rows = (uint32_t)(counts >> 32);
    }
    PolicySums sums;
    const double flat = token_weight(a.o, tokens, rows, (uint32_t)a.shape.T);
    for (uint32_t c = first; c < ch.total; c += step) {
        if (c != first) d = load_chunk(a, ch, c);
        double w = flat;
        if (a.o.reduction == CONDUIT_SEQUENCE_MEAN && a.mask)
            w = token_weight(a.o, tokens, rows, SMALL ? s_count[d.row] : a.row_count[d.row]);
        policy_chunk(a, d, w, sums);
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

// Counted tokens of every row, of the batch, and the rows with any.  LANES lanes
// take a row (a wavefront, or the workgroup); rows that follow each other
// without a gap and have no weight of their own are one row, cut into parts.
// Whole numbers, so the order of the additions is free.
template <int LANES>
__global__ __launch_bounds__(kCountThreads) void k_count(PolicyArgs a, int64_t rows, int64_t T, int64_t stride, int64_t last_T) {
    __shared__ double lds[2 * kCountThreads / kWave];
    constexpr int kRows = kCountThreads / LANES;
    double sums[2] = {0, 0};
    const int tid = threadIdx.x % LANES;
    const bool each = a.o.reduction == CONDUIT_SEQUENCE_MEAN;
    for (int64_t r0 = (int64_t)blockIdx.x * kRows; r0 < rows; r0 += (int64_t)gridDim.x * kRows) {
        const int64_t b = r0 + threadIdx.x / LANES, end = b == rows - 1 ? last_T : T;
        uint32_t k = 0;
        if (b < rows) {
            const uint8_t* row = a.mask + b * stride;
#pragma unroll 4
            for (int64_t t0 = 16 * (int64_t)tid; t0 < end; t0 += 16 * LANES) k += count16(row, t0, end);
        }
        if (!each) {
            sums[0] += k;
            continue;
        }
        double n[1] = {(double)k};
        if constexpr (LANES == kWave) n[0] = wave_sum(n[0]);
        else block_sum<kCountThreads, 1>(n, lds);
        if (tid == 0 && b < rows) {
            a.row_count[b] = (uint32_t)n[0];
            sums[0] += n[0];
            sums[1] += n[0] > 0;
        }
    }
    block_sum<kCountThreads, 2>(sums, lds);
    if (threadIdx.x == 0 && sums[0] > 0)
        atomicAdd(reinterpret_cast<unsigned long long*>(&a.head->counts),
                  (unsigned long long)sums[0] | (unsigned long long)sums[1] << 32);
}

}  // namespace

// A row of up to 16,384 tokens takes a wavefront, a longer one a workgroup; with
// one weight for all tokens, contiguous rows are taken as parts of 16,384.
hipError_t launch_token_count(const PolicyArgs& a, hipStream_t s) {
    constexpr int64_t kPart = 16 * kCountThreads;
    int64_t rows = a.shape.B, T = a.shape.T, stride = a.shape.stride, last = a.shape.T;
    if (a.o.reduction != CONDUIT_SEQUENCE_MEAN && (stride == T || rows == 1)) {
        const int64_t n = rows * T;
        T = stride = n < kPart ? n : kPart;
        rows = (n + T - 1) / T;
        last = n - (rows - 1) * T;
    } else if (T <= kPart) {
        const int64_t want = (rows + kCountThreads / kWave - 1) / (kCountThreads / kWave);
        hipLaunchKernelGGL((k_count<kWave>), dim3((unsigned)(want < kCountBlocks ? want : kCountBlocks)), dim3(kCountThreads), 0, s,
                           a, rows, T, stride, last);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((k_count<kCountThreads>), dim3((unsigned)(rows < kCountBlocks ? rows : kCountBlocks)), dim3(kCountThreads),
                       0, s, a, rows, T, stride, last);
    return hipGetLastError();
}

// counted: the counts stand in the workspace already (and are cleared here)
hipError_t launch_policy_loss(const PolicyArgs& args, bool counted, hipStream_t s) {
    PolicyArgs a = args;
    a.has_entropy = a.entropy != nullptr;
    if (!a.entropy) a.entropy = a.logp;  // (read, not used)
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
