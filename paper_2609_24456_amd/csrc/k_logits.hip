// Log-probabilities of the taken tokens from logits, their gradient, and the
// policy loss from logits to the logits' gradient in one pass over them
// (conduit_token_logprobs, _backward, conduit_policy_loss_logits).
//
// With d_j = c (x_j - max x), c = log2(e) / temperature, S = sum_j 2^d_j and
// U = sum_j 2^d_j d_j, in fp32:
//     lse = max x / temperature + ln2 log2 S,   logp = ln2 (d_a - log2 S),
//     entropy = ln2 (log2 S - U / S),           p_j = 2^d_j / S,
//     dx_j = (g ([j = a] - p_j) - h p_j (log p_j + entropy)) / temperature
// for gradients g of logp and h of the entropy.  The maximum goes before the
// scale: d_j then has two roundings of its own size however large the logits
// are, and a row at the type's lowest value is as good as any other.  A choice
// at -inf has no weight; a row of nothing else has logp = lse = -inf, entropy 0
// and gradient 0.
//
// Each lane keeps its own running maximum, sum and weighted sum over the
// elements it loads (rescaled when the maximum grows), and the lanes are joined
// once a row, so a row costs one pass and one barrier.  The loss kernel keeps
// the row's vectors in registers between the two uses, so that its logits cross
// HBM once in each direction.
#include <type_traits>

#include "softmax_dev.h"

namespace conduit {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

enum LogitsMode { LOGPROBS, LOSS };

template <bool BF16>
struct Elem;
template <>
struct Elem<true> {
    using T = uint16_t;
    static constexpr int kPer = 8;
    static __device__ __forceinline__ float one(T x) { return __builtin_bit_cast(float, (uint32_t)x << 16); }
    static __device__ __forceinline__ void unpack(u32x4 v, float (&x)[kPer]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __builtin_bit_cast(float, v[i] << 16);
            x[2 * i + 1] = __builtin_bit_cast(float, v[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ T round(float x) { return __builtin_bit_cast(T, (__bf16)x); }
    static __device__ __forceinline__ u32x4 pack(const float (&x)[kPer]) {
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (uint32_t)round(x[2 * i]) | (uint32_t)round(x[2 * i + 1]) << 16;
        return v;
    }
};
template <>
struct Elem<false> {
    using T = float;
    static constexpr int kPer = 4;
    static __device__ __forceinline__ float one(T x) { return x; }
    static __device__ __forceinline__ void unpack(u32x4 v, float (&x)[kPer]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w = v[i];  // (a value: bit_cast of a vector's element as an lvalue reads element 0)
            x[i] = __builtin_bit_cast(float, w);
        }
    }
    static __device__ __forceinline__ T round(float x) { return x; }
    static __device__ __forceinline__ u32x4 pack(const float (&x)[kPer]) {
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_bit_cast(uint32_t, x[i]);
        return v;
    }
};

// 16-byte accesses at the elements' own alignment (rows of any width start anywhere)
template <typename T>
__device__ __forceinline__ u32x4 load16(const T* p) {
    u32x4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}
template <typename T>
__device__ __forceinline__ void store16(T* p, u32x4 v) {
    __builtin_memcpy(p, &v, 16);
}

// keeps a vector packed: without it the unpacked halves of one use would be kept
// in registers for the next
__device__ __forceinline__ u32x4 again(u32x4 v) {
    asm volatile("" : "+v"(v));
    return v;
}

// K vectors of a lane
template <bool BF16, int K>
__device__ __forceinline__ void accumulate_tile(Stat& st, const u32x4 (&v)[K], float c) {
    using E = Elem<BF16>;
    float top = kNone;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float f[E::kPer];
        E::unpack(v[k], f);
        top = top_of(f, top);
    }
    raise(st, top, c);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float f[E::kPer];
        E::unpack(again(v[k]), f);
        add(st, f, c);
    }
}

// joined over WAVES wavefronts of a workgroup, in every thread
template <int WAVES>
__device__ __forceinline__ Stat join_block(Stat s, Stat* lds, float c) {
    s = join_lanes<kWave>(s, c);
    if constexpr (WAVES == 1) return s;
    if (lane_id() == 0) lds[threadIdx.x / kWave] = s;
    __syncthreads();
    Stat r = lds[lane_id() % WAVES];
    return join_lanes<WAVES>(r, c);
}

// the gradient of one logit: d = c (x - base)
struct GradCoef {
    float gp;    // -g / (temperature S)
    float hp;    // -h / (temperature S)
    float off;   // entropy - ln2 log2 S
};

template <bool ENT>
__device__ __forceinline__ float logit_gradient(const GradCoef& k, float x, float c, float base) {
    const float d = (x - base) * c, e = exp2_fast(d);
    if constexpr (!ENT) return k.gp * e;
    return e * fmaf(k.hp, fmaf(fmaxf(d, kFloor), kLn2, k.off), k.gp);
}

// the loss's part of a row: gradients of its log-probability and entropy
struct RowGrad {
    float g = 0.0f, h = 0.0f;
};

__device__ __forceinline__ GradCoef grad_coef(const LogitsArgs& a, const RowGrad& g, const RowValues& r) {
    return GradCoef{-g.g * a.inv_t * r.inv_s, -g.h * a.inv_t * r.inv_s, r.entropy - kLn2 * r.log2_s};
}

// the taken token's own, at logit xa
template <bool ENT>
__device__ __forceinline__ float taken_gradient(const LogitsArgs& a, const RowGrad& g, const RowValues& r, const GradCoef& k, float xa) {
    const float d = a.inv_t * (g.g * r.one_minus_p);
    if constexpr (!ENT) return d;
    return d + logit_gradient<true>(GradCoef{0.0f, k.hp, k.off}, xa, a.c, r.base);
}

// what the loss of a row needs beside its log-probability, loaded ahead of it
struct RowData {
    float old, ref, adv;
    double w;
    bool has_old, has_ref;
};

__device__ __forceinline__ RowData row_data(const PolicyArgs& p, int64_t at, uint32_t b) {
    RowData d;
    // (an absent policy's is logp itself, which the call has yet to write)
    d.has_old = p.old_logp != p.logp;
    d.has_ref = p.ref_logp != p.logp;
    d.old = p.old_logp[at];
    d.ref = p.ref_logp[at];
    d.adv = p.adv[at];
    uint32_t tokens = (uint32_t)(p.shape.B * p.shape.T), rows = (uint32_t)p.shape.B, row = (uint32_t)p.shape.T;
    if (p.mask) {
        const uint64_t counts = p.head->counts;
        tokens = (uint32_t)counts;
        rows = (uint32_t)(counts >> 32);
        if (p.o.reduction == CONDUIT_SEQUENCE_MEAN) row = p.row_count[b];
    }
    d.w = token_weight(p.o, tokens, rows, row);
    return d;
}

__device__ __forceinline__ RowGrad row_loss(const PolicyArgs& p, const RowData& d, float logp, TokenLoss* out) {
    const TokenLoss t = policy_token(p.o, logp, d.has_old ? d.old : logp, d.has_ref ? d.ref : logp, d.adv);
    const float wf = (float)(d.w * p.o.scale);
    if (out) *out = t;
    return RowGrad{wf * t.slope, -p.o.ent * wf};
}

__device__ __forceinline__ bool token_ok(const LogitsArgs& a, int32_t tok) {
    if (tok >= 0 && tok < a.V) return true;
    flag_error(a.err, ERR_TOKEN);
    return false;
}

// ---------------------------------------------------------------------------
// short rows: LANES lanes a row, up to E elements a lane.  Latency bounds it: 16,384
// rows of 18 with the loss and its gradient 7.45 us (an empty launch is 2.3, the
// bytes 0.6).
// ---------------------------------------------------------------------------
constexpr int kShortThreads = 256;
constexpr int kShortElems = 8;

template <bool BF16, int MODE, int LANES>
__global__ __launch_bounds__(kShortThreads) void k_rows_short(LogitsArgs a, PolicyArgs p, bool counted) {
    using E = Elem<BF16>;
    using T = typename E::T;
    constexpr int kRows = kShortThreads / LANES;
    __shared__ double lds[MODE == LOSS ? kPolicySums * kShortThreads / kWave : 1];
    const int l = threadIdx.x % LANES;
    const uint32_t n_rows = (uint32_t)(a.shape.B * a.shape.T);
    PolicySums sums;
    for (uint32_t n = blockIdx.x * kRows + threadIdx.x / LANES; n < n_rows; n += gridDim.x * kRows) {
        const int64_t at = a.shape.at(n);
        const bool on = !a.mask || a.mask[at];
        const int32_t tok = on ? a.tokens[at] : 0;
        const bool ok = on && (l != 0 ? tok >= 0 && tok < a.V : token_ok(a, tok));
        const T* x = static_cast<const T*>(a.x.data) + a.x.at(n, a.shape);
        float v[kShortElems];
        RowValues r;
        RowData rd;
        if (ok) {
            if constexpr (MODE == LOSS) rd = row_data(p, at, div31(n, a.shape.by_T));
            float xa = 0.0f;  // the taken one's, in the lane that holds it
#pragma unroll
            for (int i = 0; i < kShortElems; ++i) {
                v[i] = l + i * LANES < a.V ? E::one(x[l + i * LANES]) : kNone;
                if (l + i * LANES == tok) xa = v[i];
            }
            Stat st = no_stat();
            accumulate(st, v, a.c);
            // (a plain sum over the lanes: the others hold 0)
            r = row_values(join_lanes<LANES>(st, a.c), lanes_sum<LANES>(xa), a.c, a.inv_t, a.inv_lo);
        }
        if (l == 0) {
            if (a.logp) a.logp[at] = ok ? r.logp : 0.0f;
            if (a.lse) a.lse[at] = ok ? r.lse : 0.0f;
            if (a.entropy) a.entropy[at] = ok ? r.entropy : 0.0f;
        }
        if constexpr (MODE == LOSS) {
            T* dx = static_cast<T*>(a.dx.data) + a.dx.at(n, a.shape);
            RowGrad rg;
            if (ok) {
                TokenLoss t;
                rg = row_loss(p, rd, r.logp, &t);
                if (l == 0) {
                    TokenSums one;
                    one.add(true, t, r.entropy);
                    sums.add(rd.w, one);
                }
            }
            const GradCoef k{ok ? -rg.g * a.inv_t * r.inv_s : 0.0f, ok ? -rg.h * a.inv_t * r.inv_s : 0.0f,
                             ok ? r.entropy - kLn2 * r.log2_s : 0.0f};
#pragma unroll
            for (int i = 0; i < kShortElems; ++i) {
                const int j = l + i * LANES;
                if (j >= a.V) break;
                float d = 0.0f;
                if (ok && r.inv_s != 0.0f) {
                    if (j == tok)
                        d = rg.h != 0.0f ? taken_gradient<true>(a, rg, r, k, v[i]) : taken_gradient<false>(a, rg, r, k, v[i]);
                    else if (rg.h != 0.0f)
                        d = logit_gradient<true>(k, v[i], a.c, r.base);
                    else
                        d = logit_gradient<false>(k, v[i], a.c, r.base);
                }
                dx[j] = E::round(d);
            }
        }
    }
    if constexpr (MODE == LOSS)
        finish_policy<kShortThreads>(p, sums, p.mask ? (uint32_t)p.head->counts : n_rows, counted, lds);
}

// ---------------------------------------------------------------------------
// longer rows: WAVES wavefronts a row, K vectors a lane in registers
// ---------------------------------------------------------------------------
// HBM bounds it.  Log-probabilities only: 256 lanes a row, several rows a compute
// unit, so that one row's join runs under another's loads (8,176 rows of 32,001
// fp32: 77 us, 5.3 TB/s, where a reduction over 4 GiB reads 6.0 and a copy moves
// 4.7; 1,024 lanes a row: 111).  The loss holds a whole row of up
// to 256 KB in 1,024 lanes' registers and writes its gradient from there (8,192
// rows of 128,000 bf16, 36% of them live: 545 us for 2.9 GB, 5.2 TB/s).
template <bool BF16, int MODE, int WAVES, int K>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * kWave) void k_rows(LogitsArgs a, PolicyArgs p, bool few_rows) {
    using E = Elem<BF16>;
    using T = typename E::T;
    constexpr int kPer = E::kPer;
    constexpr int NT = WAVES * kWave;
    constexpr int kTile = NT * K;  // vectors
    __shared__ Stat lds[WAVES];
    uint32_t n = block_number();
    if constexpr (WAVES == 1) n = n * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    if (n >= (uint32_t)(a.shape.B * a.shape.T)) return;
    const uint32_t tid = threadIdx.x % NT;
    const int64_t at = a.shape.at(n);
    const T* x = static_cast<const T*>(a.x.data) + a.x.at(n, a.shape);
    const uint32_t V = (uint32_t)a.V, nv = V / kPer, tail = V % kPer;
    const int32_t tok = a.tokens[at];  // (beside the mask's load, not after it)
    const bool on = !a.mask || a.mask[at];
    const bool ok = on && (tid != 0 ? tok >= 0 && tok < a.V : token_ok(a, tok));
    T* dx = MODE == LOSS ? static_cast<T*>(a.dx.data) + a.dx.at(n, a.shape) : nullptr;
    if (!ok) {
        if (tid == 0) {
            if (a.logp) a.logp[at] = 0.0f;
            if (a.lse) a.lse[at] = 0.0f;
            if (a.entropy) a.entropy[at] = 0.0f;
        }
        if constexpr (MODE == LOSS) {
            if (few_rows && tid < kWave) finish_row(p, n, false, TokenLoss{}, 0.0f, 0.0f);
            for (uint32_t i = tid; i < nv; i += NT) store16(dx + (size_t)i * kPer, u32x4{0, 0, 0, 0});
            if (tid < tail) dx[nv * kPer + tid] = E::round(0.0f);
        }
        return;
    }
    RowData rd;
    if constexpr (MODE == LOSS) rd = row_data(p, at, div31(n, a.shape.by_T));
    const float xa = E::one(x[tok]);
    const float xt = tid < tail ? E::one(x[nv * kPer + tid]) : kNone;
    Stat st = no_stat();
    u32x4 v[K];
    const u32x4 none = BF16 ? u32x4{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u}
                            : u32x4{0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u};
    // from the last tile to the first, which then stays in registers
    for (int32_t base = nv > 0 ? (int32_t)((nv - 1) / kTile * kTile) : 0; base >= 0; base -= kTile) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const uint32_t i = base + k * NT + tid;
            v[k] = i < nv ? load16(x + (size_t)i * kPer) : none;
        }
        accumulate_tile<BF16>(st, v, a.c);
    }
    {
        const float f[1] = {xt};
        accumulate(st, f, a.c);
    }
    const RowValues r = row_values(join_block<WAVES>(st, lds, a.c), xa, a.c, a.inv_t, a.inv_lo);
    if (tid == 0) {
        if (a.logp) a.logp[at] = r.logp;
        if (a.lse) a.lse[at] = r.lse;
        if (a.entropy) a.entropy[at] = r.entropy;
    }
    if constexpr (MODE == LOSS) {
        TokenLoss loss;
        const RowGrad rg = row_loss(p, rd, r.logp, &loss);
        if (few_rows && tid < kWave) finish_row(p, n, true, loss, rd.w, r.entropy);
        const GradCoef k = grad_coef(a, rg, r);
        const bool empty = r.inv_s == 0.0f;
        auto write = [&](auto ent) {
            constexpr bool ENT = decltype(ent)::value;
            auto vector = [&](uint32_t i, u32x4 raw) {
                float f[kPer];
                E::unpack(raw, f);
#pragma unroll
                for (int j = 0; j < kPer; ++j) f[j] = empty ? 0.0f : logit_gradient<ENT>(k, f[j], a.c, r.base);
                store16(dx + (size_t)i * kPer, E::pack(f));
            };
#pragma unroll
            for (int q = 0; q < K; ++q) {
                const uint32_t i = q * NT + tid;
                if (i < nv) vector(i, again(v[q]));
            }
            for (uint32_t i = kTile + tid; i < nv; i += NT) vector(i, load16(x + (size_t)i * kPer));
            if (tid < tail) dx[nv * kPer + tid] = E::round(empty ? 0.0f : logit_gradient<ENT>(k, xt, a.c, r.base));
            // the taken token's own, by the lane that wrote its vector
            const uint32_t i = (uint32_t)tok / kPer;
            if (i < nv ? tid == i % NT : tid == (uint32_t)tok - nv * kPer) {
                dx[tok] = E::round(empty ? 0.0f : taken_gradient<ENT>(a, rg, r, k, xa));
            }
        };
        if (rg.h != 0.0f) write(std::true_type{});
        else write(std::false_type{});
    }
}

// ---------------------------------------------------------------------------
// few long rows: parts of rows, joined by the last workgroup of each row.  Latency
// bounds it: 64 rows of 128,000 bf16 8.4 us; with the loss and the gradient's launch
// 18.4 (16.4 MB read once and written once would take 6.7), one row 10.6.
// ---------------------------------------------------------------------------
constexpr int kPartThreads = 256;
constexpr int kPartK = 8;

template <bool BF16, int MODE>
__global__ __launch_bounds__(kPartThreads) void k_rows_parts(LogitsArgs a, PolicyArgs p) {
    using E = Elem<BF16>;
    using T = typename E::T;
    constexpr int kPer = E::kPer;
    __shared__ Stat lds[kPartThreads / kWave];
    __shared__ bool s_last;
    const uint32_t n = blockIdx.y, part = blockIdx.x, tid = threadIdx.x;
    const int64_t at = a.shape.at(n);
    const T* x = static_cast<const T*>(a.x.data) + a.x.at(n, a.shape);
    const uint32_t V = (uint32_t)a.V, nv = V / kPer, tail = V % kPer;
    const int32_t tok = a.tokens[at];
    const bool on = !a.mask || a.mask[at];
    const uint32_t per = (nv + a.parts - 1) / a.parts, lo = part * per, hi = lo + per < nv ? lo + per : nv;
    const u32x4 none = BF16 ? u32x4{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u}
                            : u32x4{0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u};
    Stat st = no_stat();
    float xa = 0.0f;
    bool ok = on;
    for (uint32_t base = lo; ok && base < hi; base += kPartThreads * kPartK) {
        u32x4 v[kPartK];
#pragma unroll
        for (int k = 0; k < kPartK; ++k) {
            const uint32_t i = base + k * kPartThreads + tid;
            v[k] = i < hi ? load16(x + (size_t)i * kPer) : none;
        }
        if (base == lo) {  // the token's own loads run beside the first of the row's
            ok = tid != 0 || part != 0 ? tok >= 0 && tok < a.V : token_ok(a, tok);
            if (ok) xa = E::one(x[tok]);
        }
        accumulate_tile<BF16>(st, v, a.c);
    }
    if (!ok) {
        if (part == 0 && tid == 0) {
            if (a.logp) a.logp[at] = 0.0f;
            if (a.lse) a.lse[at] = 0.0f;
            if (a.entropy) a.entropy[at] = 0.0f;
        }
        if constexpr (MODE == LOSS) {
            if (part == 0 && tid < (uint32_t)kWave) finish_row(p, n, false, TokenLoss{}, 0.0f, 0.0f);
        }
        return;
    }
    if (part == 0 && tid < tail) {
        const float f[1] = {E::one(x[nv * kPer + tid])};
        accumulate(st, f, a.c);
    }
    st = join_block<kPartThreads / kWave>(st, lds, a.c);
    float* mine = a.part + 3 * ((int64_t)n * a.parts + part);
    if (tid == 0) {
        __hip_atomic_store(mine, st.m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(mine + 1, st.s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(mine + 2, st.u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // acknowledged before the ticket is drawn
        s_last = draw_last(a.row_ticket + n * kTicketStep, (uint32_t)a.parts);
    }
    __syncthreads();
    if (!s_last || tid >= (uint32_t)kWave) return;
    Stat all = no_stat();
    for (int k = tid; k < a.parts; k += kWave) {
        const float* q = a.part + 3 * ((int64_t)n * a.parts + k);
        Stat o;
        o.m = __hip_atomic_load(q, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        o.s = __hip_atomic_load(q + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        o.u = __hip_atomic_load(q + 2, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        all = join(all, o, a.c);
    }
    const RowValues r = row_values(join_lanes<kWave>(all, a.c), xa, a.c, a.inv_t, a.inv_lo);
    if (tid == 0) {
        if (a.logp) a.logp[at] = r.logp;
        if (a.lse) a.lse[at] = r.lse;
        if (a.entropy) a.entropy[at] = r.entropy;
    }
    if constexpr (MODE == LOSS) {
        const RowData rd = row_data(p, at, div31(n, a.shape.by_T));
        TokenLoss loss;
        const RowGrad rg = row_loss(p, rd, r.logp, &loss);
        if (tid == 0) {
            const GradCoef k = grad_coef(a, rg, r);
            const float taken = rg.h != 0.0f ? taken_gradient<true>(a, rg, r, k, xa) : taken_gradient<false>(a, rg, r, k, xa);
            a.split[n] = r.inv_s == 0.0f ? SplitRow{0.0f, 0.0f, 0.0f, 0.0f, 0.0f} : SplitRow{r.base, k.gp, k.hp, k.off, taken};
        }
        finish_row(p, n, true, loss, rd.w, r.entropy);
    }
}

// ---------------------------------------------------------------------------
// the gradient of the logits from the row's saved log-normaliser, or, SPLIT, from
// what the loss of split rows left for it: wavefronts take parts of kGradK
// vectors a lane of a row.  HBM bounds it: 2,048 rows of 50,001 fp32 with
// entropies 115 us, 5.0 TB/s, a large copy's rate (4.9).
// ---------------------------------------------------------------------------
constexpr int kGradThreads = 256;
constexpr int kGradK = 4;

// by the log-normaliser given
struct FromLse {
    float inv_t, inv_lo, lse, entropy;
    RowGrad g;
    // The scores are far from 0 where log p_j need not be, so a rounded 1 / temperature would cost |z_j| 2^-25 of p_j:
    // its rest goes along (of the lowest finite value for a choice at -inf: the rest may be 0).
    __device__ __forceinline__ float log_p(float f) const {
        return fmaf(f, inv_t, fmaf(fmaxf(f, -3.4028235e38f), inv_lo, -lse));
    }
    __device__ __forceinline__ bool with_entropy() const { return g.h != 0.0f; }
    template <bool ENT>
    __device__ __forceinline__ float of(float f, float gj) const {
        const float q = log_p(f), e = exp2_fast(q * kLog2e);  // log p_j, p_j
        if constexpr (!ENT) return -gj * inv_t * e;
        return -inv_t * e * fmaf(g.h, fmaxf(q, kFloor) + entropy, gj);
    }
    template <bool ENT>
    __device__ __forceinline__ float other(float f) const { return of<ENT>(f, g.g); }
    template <bool ENT>
    __device__ __forceinline__ float taken(float f) const {
        const float d = inv_t * (g.g * -expm1_fast(log_p(f)));
        if constexpr (!ENT) return d;
        return d + of<true>(f, 0.0f);
    }
};

// by the row's statistics, as k_rows does
struct FromStats {
    float c;
    SplitRow r;
    __device__ __forceinline__ bool with_entropy() const { return r.hp != 0.0f; }
    template <bool ENT>
    __device__ __forceinline__ float other(float f) const { return logit_gradient<ENT>(GradCoef{r.gp, r.hp, r.off}, f, c, r.base); }
    template <bool ENT>
    __device__ __forceinline__ float taken(float) const { return r.taken; }
};

template <bool BF16, bool SPLIT>
__global__ __launch_bounds__(kGradThreads) void k_rows_gradient(LogitsArgs a, uint32_t items, uint32_t per_row, Div31 by_row) {
    using E = Elem<BF16>;
    using T = typename E::T;
    constexpr int kPer = E::kPer;
    const uint32_t item = block_number() * (kGradThreads / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    if (item >= items) return;
    const uint32_t n = div31(item, by_row), part = item - n * per_row, lane = lane_id();
    const int64_t at = a.shape.at(n);
    const T* x = static_cast<const T*>(a.x.data) + a.x.at(n, a.shape);
    T* dx = static_cast<T*>(a.dx.data) + a.dx.at(n, a.shape);
    const uint32_t V = (uint32_t)a.V, nv = V / kPer, tail = V % kPer;
    const bool on = !a.mask || a.mask[at];
    const int32_t tok = on ? a.tokens[at] : 0;
    const bool ok = on && (lane != 0 || part != 0 ? tok >= 0 && tok < a.V : token_ok(a, tok));
    const uint32_t base = part * kGradK * kWave + lane;
    const bool mine = part == 0 && lane < tail;  // the elements after the last vector
    typename std::conditional<SPLIT, FromStats, FromLse>::type grad;
    bool weight = ok;
    if constexpr (SPLIT) {
        grad.c = a.c;
        if (ok) grad.r = a.split[n];
    } else {
        grad.inv_t = a.inv_t;
        grad.inv_lo = a.inv_lo;
        grad.lse = ok ? a.lse_in[at] : 0.0f;
        grad.g.g = ok && a.g ? a.g[at] : 0.0f;
        grad.g.h = ok && a.h ? a.h[at] : 0.0f;
        grad.entropy = ok && a.entropy_in ? a.entropy_in[at] : 0.0f;
        weight = ok && grad.lse != kNone;
    }
    if (!weight) {  // nothing counts, or a row without weight
#pragma unroll
        for (int k = 0; k < kGradK; ++k) {
            const uint32_t i = base + k * kWave;
            if (i < nv) store16(dx + (size_t)i * kPer, u32x4{0, 0, 0, 0});
        }
        if (mine) dx[nv * kPer + lane] = E::round(0.0f);
        return;
    }
    u32x4 v[kGradK];
#pragma unroll
    for (int k = 0; k < kGradK; ++k) {
        const uint32_t i = base + k * kWave;
        v[k] = i < nv ? load16(x + (size_t)i * kPer) : u32x4{0, 0, 0, 0};
    }
    const float xt = mine ? E::one(x[nv * kPer + lane]) : 0.0f;
    const float xa = SPLIT ? 0.0f : E::one(x[tok]);
    auto write = [&](auto ent) {
        constexpr bool ENT = decltype(ent)::value;
#pragma unroll
        for (int k = 0; k < kGradK; ++k) {
            const uint32_t i = base + k * kWave;
            float f[kPer];
            E::unpack(v[k], f);
#pragma unroll
            for (int j = 0; j < kPer; ++j) f[j] = grad.template other<ENT>(f[j]);
            if (i < nv) store16(dx + (size_t)i * kPer, E::pack(f));
        }
        if (mine) dx[nv * kPer + lane] = E::round(grad.template other<ENT>(xt));
        // the taken token's own, by the lane that wrote its vector
        const uint32_t i = (uint32_t)tok / kPer;
        const bool holds = i < nv ? i / (kGradK * kWave) == part && i % kWave == lane
                                  : part == 0 && (uint32_t)tok - nv * kPer == lane;
        if (holds) dx[tok] = E::round(grad.template taken<ENT>(xa));
    };
    if (grad.with_entropy()) write(std::true_type{});
    else write(std::false_type{});
}

template <bool BF16, bool SPLIT>
hipError_t launch_gradient(const LogitsArgs& a, hipStream_t s) {
    const int64_t nv = a.V / Elem<BF16>::kPer;
    const int64_t per_row = nv > 0 ? (nv + kGradK * kWave - 1) / (kGradK * kWave) : 1;
    const int64_t rows = a.shape.B * a.shape.T;
    // one launch takes fewer than 2^31 parts (the division's range)
    const int64_t items = rows * per_row;
    if (items >= 1ll << 31) return hipErrorInvalidValue;
    const dim3 grid = grid_of((items + kGradThreads / kWave - 1) / (kGradThreads / kWave), kGradThreads);
    hipLaunchKernelGGL((k_rows_gradient<BF16, SPLIT>), grid, dim3(kGradThreads), 0, s, a, (uint32_t)items, (uint32_t)per_row,
                       make_div31((uint32_t)per_row));
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// which kernel a row's width takes
// ---------------------------------------------------------------------------
template <bool BF16, int MODE>
hipError_t launch_short(const LogitsArgs& a, const PolicyArgs& p, bool counted, hipStream_t s) {
    const int64_t rows = a.shape.B * a.shape.T;
    auto go = [&](auto lanes) {
        constexpr int LANES = decltype(lanes)::value;
        const int64_t want = (rows + kShortThreads / LANES - 1) / (kShortThreads / LANES);
        const int64_t cap = MODE == LOSS ? kPolicyBlocks : 16LL * device_cus();
        hipLaunchKernelGGL((k_rows_short<BF16, MODE, LANES>), dim3((unsigned)(want < cap ? want : cap)),
                           dim3(kShortThreads), 0, s, a, p, counted);
        return hipGetLastError();
    };
    if (a.V <= 4 * kShortElems) return go(std::integral_constant<int, 4>{});
    if (a.V <= 8 * kShortElems) return go(std::integral_constant<int, 8>{});
    if (a.V <= 16 * kShortElems) return go(std::integral_constant<int, 16>{});
    if (a.V <= 32 * kShortElems) return go(std::integral_constant<int, 32>{});
    return go(std::integral_constant<int, 64>{});
}

constexpr int64_t kShortWidth = 64 * kShortElems;

template <bool BF16, int MODE>
hipError_t launch_long(const LogitsArgs& a, const PolicyArgs& p, bool few_rows, hipStream_t s) {
    const int64_t rows = a.shape.B * a.shape.T, nv = a.V / Elem<BF16>::kPer;
    const dim3 grid = grid_of(rows, 256);
    if (nv <= 8 * kWave) {
        hipLaunchKernelGGL((k_rows<BF16, MODE, 1, 8>), grid_of((rows + 3) / 4, 256), dim3(256), 0, s, a, p, few_rows);
    } else if constexpr (MODE == LOGPROBS) {  // nothing stays: any width goes by in tiles of 8 vectors a lane
        hipLaunchKernelGGL((k_rows<BF16, LOGPROBS, 4, 8>), grid, dim3(256), 0, s, a, p, few_rows);
    } else if (nv <= 4096) {
        hipLaunchKernelGGL((k_rows<BF16, LOSS, 4, 16>), grid, dim3(256), 0, s, a, p, few_rows);
    } else {
        hipLaunchKernelGGL((k_rows<BF16, LOSS, 16, 16>), grid_of(rows, 1024), dim3(1024), 0, s, a, p, few_rows);
    }
    return hipGetLastError();
}

template <bool BF16, int MODE>
hipError_t launch_parts(const LogitsArgs& a, const PolicyArgs& p, hipStream_t s) {
    hipLaunchKernelGGL((k_rows_parts<BF16, MODE>), dim3((unsigned)a.parts, (unsigned)(a.shape.B * a.shape.T)),
                       dim3(kPartThreads), 0, s, a, p);
    return hipGetLastError();
}

template <bool BF16>
hipError_t logprobs(const LogitsArgs& a, hipStream_t s) {
    if (a.V <= kShortWidth) return launch_short<BF16, LOGPROBS>(a, PolicyArgs{}, false, s);
    if (a.parts > 1) return launch_parts<BF16, LOGPROBS>(a, PolicyArgs{}, s);
    return launch_long<BF16, LOGPROBS>(a, PolicyArgs{}, false, s);
}

// Split rows (fewer than the GPU has compute units) and up to kPolicyBlocks
// whole ones sum the statistics up as they go; more rows leave them to a launch
// over the tokens (its 9 us against as many tickets, 13 ns each).
template <bool BF16>
hipError_t loss_logits(const LogitsArgs& a, const PolicyArgs& p, hipStream_t s) {
    hipError_t e = hipSuccess;
    if (p.mask) e = launch_token_count(p, s);  // the tokens' weight needs their number
    if (e != hipSuccess) return e;
    if (a.V <= kShortWidth) return launch_short<BF16, LOSS>(a, p, p.mask != nullptr, s);
    if (a.parts > 1) {
        e = launch_parts<BF16, LOSS>(a, p, s);
        if (e == hipSuccess) e = launch_gradient<BF16, true>(a, s);
        return e;
    }
    const bool few = a.shape.B * a.shape.T <= kPolicyBlocks;
    e = launch_long<BF16, LOSS>(a, p, few, s);
    if (e != hipSuccess || few) return e;
    return launch_policy_loss(p, p.mask != nullptr, s);
}

}  // namespace

// Parts of a row: rows are split where the rows alone would leave compute units
// without a workgroup, into parts of at least four vectors a lane: 64 rows of
// 128,000 bf16 7.1 us (whole, a workgroup each: 14.0), 16 rows 5.7, one row 5.4.
int logits_parts(int64_t rows, int64_t V, bool bf16) {
    const int64_t cus = device_cus(), nv = V / (bf16 ? 8 : 4);
    if (V <= kShortWidth || rows >= cus || rows > kPolicyBlocks || rows <= 0) return 1;
    const int64_t want = (2 * cus + rows - 1) / rows, most = nv / (4 * kPartThreads);
    const int64_t parts = want < most ? want : most;
    return parts > 1 ? (int)parts : 1;
}

hipError_t launch_token_logprobs(const LogitsArgs& a, bool bf16, hipStream_t s) {
    return bf16 ? logprobs<true>(a, s) : logprobs<false>(a, s);
}

hipError_t launch_token_logprobs_backward(const LogitsArgs& a, bool bf16, hipStream_t s) {
    return bf16 ? launch_gradient<true, false>(a, s) : launch_gradient<false, false>(a, s);
}

hipError_t launch_policy_loss_logits(const LogitsArgs& a, const PolicyArgs& p, bool bf16, hipStream_t s) {
    return bf16 ? loss_logits<true>(a, p, s) : loss_logits<false>(a, p, s);
}

}  // namespace conduit
