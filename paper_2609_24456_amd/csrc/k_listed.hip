// Log-probabilities of a few listed choices of every token and of all others
// together, their gradient, and the divergence of a student from a teacher whose
// probabilities are known at the listed choices, logits to their gradient in one
// call (conduit_listed_logprobs, _backward, conduit_distill_loss).
//
// The pass over a row sums the others only: the listed choices are marked in a
// bit map in LDS and count as -infinity there.  What is left to the others is
// often far smaller than what the listed ones hold, and would be lost in the
// difference of two sums.  With m, s the others' maximum and sum, and M, S the
// whole row's, in powers of two as in k_logits.hip:
//     log p_k = (x_k - M) / temperature - log S,   log p_rest = (m - M) / temperature + log s - log S.
// The divergence goes by u = log q - log p of each listed choice, and of the rest
// where it counts as one more:
//     forward  sum q log (q / p) = sum q (exp(-u) - 1 + u) + sum q - sum p
//     reverse  sum p log (p / q) = sum p (exp u - 1 - u) + sum p - sum q
// whose terms have one sign, so that a small divergence is not a difference of
// large sums.  The gradient of a listed choice goes by its own u, that of any
// other is 2^(c (x - m)) times one number of the row.
//
// Duplicates of a choice are found by the bit map (a bit that is set already),
// and only then looked for in the list.
#include <type_traits>

#include "listed_dev.h"
#include "rows_dev.h"

namespace conduit {

namespace {

enum ListedMode { SCORES, DISTILL, DIVERGENCE };  // (DIVERGENCE: distillation without the gradient)

constexpr int kListedThreads = 256;
constexpr int kShortElems = 8;                        // elements a lane of a short row
constexpr int64_t kShortRow = kShortElems * kWave;
constexpr int kFewLanes = 16, kFewElems = 4;          // of rows that share a wavefront

// ---------------------------------------------------------------------------
// sums over the choices that are not listed
// ---------------------------------------------------------------------------
struct Mass {
    float m, s;
};

__device__ __forceinline__ Mass no_mass() { return Mass{kNone, 0.0f}; }

template <int N>
__device__ __forceinline__ void add_mass(Mass& t, const float (&x)[N], float c) {
    const float base = t.m == kNone ? 0.0f : t.m;
#pragma unroll
    for (int i = 0; i < N; ++i) t.s += exp2_fast((x[i] - base) * c);
}

__device__ __forceinline__ void raise_mass(Mass& t, float top, float c) {
    if (top > t.m) {
        t.s *= exp2_fast((t.m - top) * c);
        t.m = top;
    }
}

template <int N>
__device__ __forceinline__ void accumulate_mass(Mass& t, const float (&x)[N], float c) {
    raise_mass(t, top_of(x, kNone), c);
    add_mass(t, x, c);
}

template <bool BF16, int K>
__device__ __forceinline__ void accumulate_mass_tile(Mass& t, const u32x4 (&v)[K], float c) {
    using E = Elem<BF16>;
    float top = kNone;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float f[E::kPer];
        E::unpack(v[k], f);
        top = top_of(f, top);
    }
    raise_mass(t, top, c);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float f[E::kPer];
        E::unpack(again(v[k]), f);
        add_mass(t, f, c);
    }
}

// joined over groups of LANES lanes that are alike, or over all of them, in every lane
template <int LANES>
__device__ __forceinline__ Mass join_mass(const Mass& a, float c) {
    Mass r;
    r.m = lanes_reduce<LANES>(a.m, [](float x, float y) { return x > y ? x : y; });
    r.s = lanes_sum<LANES>(a.s * exp2_fast(a.m == r.m ? 0.0f : (a.m - r.m) * c));
    return Mass{uniform(r.m), uniform(r.s)};
}

// ---------------------------------------------------------------------------
// A row's list is worked on by LANES lanes: a wavefront, or a part of one, whose
// other parts have rows of their own.
// ---------------------------------------------------------------------------
template <int LANES>
__device__ __forceinline__ uint32_t group_lane() { return lane_id() % LANES; }

// the first lane's value, in every lane
template <int LANES>
__device__ __forceinline__ float group_first(float x) {
    if constexpr (LANES == kWave) return uniform(x);
    else return __shfl(x, 0, LANES);
}

template <int LANES>
__device__ __forceinline__ bool group_any(bool x) {
    const uint64_t all = __ballot(x);
    if constexpr (LANES == kWave) return all != 0;
    else return (all >> lane_id() / LANES * LANES & ((1ull << LANES) - 1)) != 0;
}

template <int LANES>
__device__ __forceinline__ Mass join_group(const Mass& a, float c) {
    Mass r;
    r.m = lanes_reduce<LANES>(a.m, [](float x, float y) { return x > y ? x : y; });
    r.s = lanes_sum<LANES>(a.s * exp2_fast(a.m == r.m ? 0.0f : (a.m - r.m) * c));
    return Mass{group_first<LANES>(r.m), group_first<LANES>(r.s)};
}

// ---------------------------------------------------------------------------
// the listed choices of a token: two a lane
// ---------------------------------------------------------------------------
constexpr int kLists = kMostListed / kWave;

struct Listed {
    int32_t id[kLists];
    float y[kLists];     // the teacher's value, or the gradient
    float x[kLists];     // the score
    bool on[kLists];     // a choice of the row
    bool first[kLists];  // the first of its number in the list
};

template <int LANES = kWave>
__device__ __forceinline__ void load_ids(const ListedArgs& a, uint32_t n, Listed& e) {
    const int32_t* ids = static_cast<const int32_t*>(a.ids.data) + a.ids.at(n, a.shape);
#pragma unroll
    for (int i = 0; i < kLists; ++i) {
        const int32_t k = i * LANES + group_lane<LANES>();
        e.id[i] = k < a.K ? ids[k] : -1;
    }
}

template <int LANES = kWave>
__device__ __forceinline__ void load_values(const ListedArgs& a, const RowsView& rows, uint32_t n, Listed& e) {
    const float* y = static_cast<const float*>(rows.data) + rows.at(n, a.shape);
#pragma unroll
    for (int i = 0; i < kLists; ++i) {
        const int32_t k = i * LANES + group_lane<LANES>();
        e.y[i] = k < a.K ? y[k] : 0.0f;
    }
}

// which of them are choices at all: a teacher's of value -infinity is as if not listed
template <bool VALUES>
__device__ __forceinline__ void check_ids(const ListedArgs& a, Listed& e, bool flags) {
#pragma unroll
    for (int i = 0; i < kLists; ++i) {
        e.on[i] = e.id[i] >= 0 && e.id[i] < a.V && !(VALUES && e.y[i] == kNone);
        e.first[i] = e.on[i];
        if (flags && e.id[i] >= a.V) flag_error(a.err, ERR_TOKEN);
    }
}

template <bool BF16>
__device__ __forceinline__ void load_scores(const typename Elem<BF16>::T* x, Listed& e) {
#pragma unroll
    for (int i = 0; i < kLists; ++i) e.x[i] = e.on[i] ? Elem<BF16>::one(x[e.id[i]]) : kNone;
}

// Those of a number that the list has before are not the first.  sum: the values of
// equal numbers are added up at the first, in the list's order.
template <bool SUM, int LANES = kWave>
__device__ void find_first(Listed& e, int32_t K) {
    float y[kLists];
#pragma unroll
    for (int i = 0; i < kLists; ++i) y[i] = e.y[i];
    for (int32_t j = 0; j < K; ++j) {
        const int i = j / LANES, from = j % LANES;
        const int32_t id = __shfl(i == 0 ? e.id[0] : e.id[1], from, LANES);
        const float v = __shfl(i == 0 ? y[0] : y[1], from, LANES);
        if (!__shfl((int)(i == 0 ? e.on[0] : e.on[1]), from, LANES)) continue;
#pragma unroll
        for (int k = 0; k < kLists; ++k) {
            const int32_t mine = k * LANES + group_lane<LANES>();
            if (!e.on[k] || e.id[k] != id || mine == j) continue;
            if (mine > j) e.first[k] = false;
            else if (SUM) e.y[k] += v;
        }
    }
}

// Marks the listed choices of one or more lanes' elements; true if a number is
// there twice.  place(id, &word, &bit): false if the choice is not among them.
template <int LANES = kWave, typename Place>
__device__ __forceinline__ bool mark(const Listed& e, Place place) {
    bool twice = false;
#pragma unroll
    for (int i = 0; i < kLists; ++i) {
        uint32_t* word;
        uint32_t bit;
        if (e.on[i] && place((uint32_t)e.id[i], &word, &bit)) twice |= (atomicOr(word, bit) & bit) != 0;
    }
    return group_any<LANES>(twice);
}

// elements of a vector whose bits are set, at -infinity
template <bool BF16>
__device__ __forceinline__ u32x4 without(u32x4 v, uint32_t bits) {
    constexpr uint32_t kLow = BF16 ? 0xff80u : 0xff800000u;
#pragma unroll
    for (int j = 0; j < Elem<BF16>::kPer; ++j) {
        if (!(bits >> j & 1)) continue;
        if constexpr (BF16) v[j / 2] = j % 2 ? (v[j / 2] & 0xffffu) | kLow << 16 : (v[j / 2] & 0xffff0000u) | kLow;
        else v[j] = kLow;
    }
    return v;
}

// the elements of a vector whose bits are not set
template <bool BF16, bool PAST>
__device__ __forceinline__ void store_others(typename Elem<BF16>::T* p, const float (&f)[Elem<BF16>::kPer], uint32_t bits) {
    if (bits == 0) return put16<PAST>(p, Elem<BF16>::pack(f));
#pragma unroll
    for (int j = 0; j < Elem<BF16>::kPer; ++j)
        if (!(bits >> j & 1)) p[j] = Elem<BF16>::round(f[j]);
}

// ---------------------------------------------------------------------------
// a row from the others' sum and its listed choices, by LANES lanes
// ---------------------------------------------------------------------------
template <int LANES>
__device__ __forceinline__ float top_of_lanes(float x) {
    return lanes_reduce<LANES>(x, [](float p, float q) { return p > q ? p : q; });
}

// a (exp s - 1 - s) for s = log(b / a): b - a - a s, which at small s cancels
__device__ __forceinline__ float curve(float a, float b, float s) {
    float k, em1;
    exp_remainder(s, &k, &em1);
    if (fabsf(s) < 0.5f) return a * k;
    return a == 0.0f ? b : (b - a) - a * s;
}

// b - a = a (exp s - 1)
__device__ __forceinline__ float apart_by(float a, float b, float s) {
    float k, em1;
    exp_remainder(s, &k, &em1);
    return fabsf(s) < 0.5f ? a * em1 : b - a;
}

// what a row's sums say
struct RowMass {
    float top, log_s;    // M (0 in a row without weight), log S
    float share, rest;   // 2^(c (m - M)) / S, log p_rest
    bool weight, some;   // anything but -infinity in the row, among the others
    __device__ __forceinline__ float logp(float x, float inv_t) const { return fmaf(x - top, inv_t, -log_s); }
};

template <int LANES = kWave>
__device__ __forceinline__ RowMass row_mass(const Listed& e, const Mass& others, float c, float inv_t) {
    RowMass r;
    float top = kNone;
#pragma unroll
    for (int i = 0; i < kLists; ++i) top = fmaxf(top, e.first[i] ? e.x[i] : kNone);
    top = top_of_lanes<LANES>(fmaxf(top, others.m));
    r.top = top != kNone ? top : 0.0f;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kLists; ++i) sum += e.first[i] ? exp2_fast((e.x[i] - r.top) * c) : 0.0f;
    const float d = others.m == top ? 0.0f : others.m - top, k = exp2_fast(d * c);
    const float S = fmaf(others.s, k, group_first<LANES>(lanes_sum<LANES>(sum)));
    r.weight = !(S == 0.0f);  // (a row of NaN alone has no largest score either)
    const float log2_s = r.weight ? log2_fast(S) : 0.0f;
    r.log_s = log2_s * kLn2;
    r.some = !(others.s == 0.0f);
    r.share = r.weight ? k / S : 0.0f;
    r.rest = r.some ? fmaf(d, inv_t, (log2_fast(others.s) - log2_s) * kLn2) : kNone;
    return r;
}

// the teacher's side of a row
struct Teacher {
    float top, log;  // log q = (y - top) / temperature - log: the largest goes first, as for the scores
    double left;     // what its listed probabilities leave (with_rest)
    bool any;
};

template <int LANES = kWave>
__device__ __forceinline__ Teacher teacher_row(const ListedArgs& a, const Listed& e) {
    Teacher t{0.0f, 0.0f, 0.0, false};
    bool any = false;
#pragma unroll
    for (int i = 0; i < kLists; ++i) any |= e.first[i];
    t.any = group_any<LANES>(any);
    if (a.with_rest) {
        // in 64 bits: what is left of 1 may be far smaller than the sum's own rounding in 32
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < kLists; ++i) sum += e.first[i] ? exp((double)e.y[i]) : 0.0;
        t.left = 1.0 - lanes_sum<LANES>(sum);
        return t;
    }
    float top = kNone;
#pragma unroll
    for (int i = 0; i < kLists; ++i) top = fmaxf(top, e.first[i] ? e.y[i] : kNone);
    t.top = t.any ? top_of_lanes<LANES>(top) : 0.0f;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kLists; ++i) sum += e.first[i] ? exp2_fast((e.y[i] - t.top) * (a.q_inv_t * kLog2e)) : 0.0f;
    t.log = t.any ? log2_fast(group_first<LANES>(lanes_sum<LANES>(sum))) * kLn2 : 0.0f;
    return t;
}

constexpr double kLeastRest = 1.0 / 8388608.0;  // 2^-23: what 32-bit log-probabilities say of a rest at best

// The forward divergence of a row in which a log-probability is past the largest float (choices at the type's lowest
// value, small temperatures): its product with the teacher's probability need not be.  What is left out of it, sum q log
// q, is nothing beside it.
template <int LANES>
__device__ __forceinline__ float far_divergence(const ListedArgs& a, const Listed& e, const Mass& others, const RowMass& r,
                                                const Teacher& t, float q_rest) {
    float loss = 0.0f;
#pragma unroll
    for (int i = 0; i < kLists; ++i) {
        const float q = e.first[i] ? exp_fast((e.y[i] - t.top) * a.q_inv_t - t.log) : 0.0f;
        if (q != 0.0f) loss = e.x[i] == kNone ? INFINITY : fmaf(q * a.inv_t, r.top - e.x[i], loss);
    }
    loss = group_first<LANES>(lanes_sum<LANES>(loss));
    return r.some && q_rest != 0.0f ? fmaf(q_rest * a.inv_t, r.top - others.m, loss) : loss;
}

// The divergence of a row and what its gradient needs; w: the token's weight.
template <int LANES = kWave>
__device__ __forceinline__ ListedRow distill_row(const ListedArgs& a, const Listed& e, const Mass& others, const RowMass& r,
                                                 const Teacher& t, float w) {
    ListedRow o{};
    o.top = r.top;
    o.log_s = r.log_s;
    o.q_top = t.top;
    o.q_log = t.log;
    o.base = others.m == kNone ? 0.0f : others.m;
    o.w = w * a.inv_t;
    if (!a.with_rest && !t.any) {  // the teacher says nothing
        o.w = 0.0f;
        return o;
    }
    if (!r.weight) {
        o.loss = INFINITY;
        o.w = 0.0f;
        return o;
    }
    float loss = 0.0f;
#pragma unroll
    for (int i = 0; i < kLists; ++i) {
        if (!e.first[i]) continue;
        const float lq = (e.y[i] - t.top) * a.q_inv_t - t.log, lp = r.logp(e.x[i], a.inv_t);
        const float q = exp_fast(lq), p = exp_fast(lp), u = lq - lp;
        loss += a.reverse ? curve(p, q, u) : curve(q, p, -u);
    }
    loss = group_first<LANES>(lanes_sum<LANES>(loss));
    const float p_rest = r.some ? exp_fast(r.rest) : 0.0f;
    if (!a.with_rest) {
        o.loss = loss + p_rest;
        if (o.loss == INFINITY) o.loss = far_divergence<LANES>(a, e, others, r, t, 0.0f);
        o.coef = r.some && o.w != 0.0f ? o.w * r.share : 0.0f;  // (a share that is no number counts for nothing at weight 0)
        return o;
    }
    const double kept = r.some ? (t.left > kLeastRest ? t.left : kLeastRest) : 0.0;
    o.over = (float)(kept - t.left);
    const float q_rest = (float)kept, away = r.some ? log2_fast(q_rest) * kLn2 - r.rest : 0.0f;
    if (a.reverse) {
        o.loss = loss + (r.some ? curve(p_rest, q_rest, away) : 0.0f) - o.over;
        // (others without weight have none of the gradient however far away they are: 0 times infinity)
        o.coef = r.some && o.w != 0.0f && r.share != 0.0f ? -o.w * (r.share * (away + o.loss)) : 0.0f;
    } else {
        o.loss = loss + (r.some ? curve(q_rest, p_rest, -away) : 0.0f) + o.over;
        if (o.loss == INFINITY) o.loss = far_divergence<LANES>(a, e, others, r, t, q_rest);
        // (1 + over) share - q_rest / s
        float k, em1;
        exp_remainder(away, &k, &em1);
        const float d = fabsf(away) < 0.5f ? r.share * (o.over - em1) : fmaf(1.0f + o.over, r.share, -q_rest / others.s);
        o.coef = r.some && o.w != 0.0f ? o.w * d : 0.0f;
    }
    return o;
}

// the gradient of a listed choice of score x and teacher's value y
__device__ __forceinline__ float listed_gradient(const ListedArgs& a, const ListedRow& o, float x, float y) {
    if (o.w == 0.0f) return 0.0f;
    const float lq = (y - o.q_top) * a.q_inv_t - o.q_log, lp = fmaf(x - o.top, a.inv_t, -o.log_s);
    const float q = exp_fast(lq), p = exp_fast(lp), u = lq - lp;
    if (a.reverse) return p == 0.0f ? 0.0f : -o.w * p * (u + o.loss);
    return o.w * fmaf(p, o.over, apart_by(q, p, -u));
}

template <int LANES = kWave>
__device__ __forceinline__ void write_scores(const ListedArgs& a, uint32_t n, int64_t at, const Listed& e, const Mass& others) {
    const RowMass r = row_mass<LANES>(e, others, a.c, a.inv_t);
    float* out = static_cast<float*>(a.logps.data) + a.logps.at(n, a.shape);
#pragma unroll
    for (int i = 0; i < kLists; ++i) {
        const int32_t k = i * LANES + group_lane<LANES>();
        if (k < a.K) out[k] = e.on[i] ? r.logp(e.x[i], a.inv_t) : kNone;
    }
    if (group_lane<LANES>() != 0) return;
    if (a.rest) a.rest[at] = r.rest;
    if (a.lse) a.lse[at] = r.weight ? log_normaliser(r.top, r.log_s, a.inv_t, a.inv_lo) : kNone;
}

// per-token outputs of a token that does not count, by LANES lanes
template <int MODE, int LANES = kWave>
__device__ __forceinline__ void write_nothing(const ListedArgs& a, uint32_t n, int64_t at) {
    if constexpr (MODE == SCORES) {
        float* out = static_cast<float*>(a.logps.data) + a.logps.at(n, a.shape);
        for (int32_t k = group_lane<LANES>(); k < a.K; k += LANES) out[k] = 0.0f;
        if (group_lane<LANES>() == 0 && a.rest) a.rest[at] = 0.0f;
        if (group_lane<LANES>() == 0 && a.lse) a.lse[at] = 0.0f;
    } else {
        if (group_lane<LANES>() == 0) a.loss[at] = 0.0f;
    }
}

// ---------------------------------------------------------------------------
// the loss's sums
// ---------------------------------------------------------------------------
// Tokens that count, by a wavefront: of a small batch from the mask itself, else from
// the launch before.  A mask in one piece goes by in 16 bytes a lane, one round of
// loads for 2,048 tokens, any other by bytes.  (The launch takes 4.6 us and a gap; 2,048
// rows of 50,001 bf16 59.8 us with the counting, 57 without; of 8,192 tokens it costs
// the rows more than the launch.)
struct Counts {
    uint32_t tokens, rows;  // that count, and sequences with one (for the mean over these)
};

__device__ __forceinline__ Counts counted_tokens(const ListedArgs& a) {
    const uint32_t n_rows = (uint32_t)(a.shape.B * a.shape.T);
    if (!a.mask) return Counts{n_rows, (uint32_t)a.shape.B};
    if (a.counted) return Counts{(uint32_t)a.head->counts, (uint32_t)(a.head->counts >> 32)};
    if (a.flat_mask) {
        constexpr uint32_t kAtOnce = 2;
        const uint32_t whole = n_rows / 16, rest = n_rows % 16;
        uint32_t mine = lane_id() < rest && a.mask[whole * 16 + lane_id()] ? 1 : 0;
#pragma unroll 1
        for (uint32_t base = 0; base < whole; base += kAtOnce * kWave) {
            u32x4 m[kAtOnce];
#pragma unroll
            for (uint32_t i = 0; i < kAtOnce; ++i) {
                const uint32_t k = base + i * kWave + lane_id();
                m[i] = k < whole ? load16(a.mask + (size_t)k * 16) : u32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (uint32_t i = 0; i < kAtOnce; ++i) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t x = m[i][q];
                    mine += __builtin_popcount((((x & 0x7f7f7f7fu) + 0x7f7f7f7fu) | x) & 0x80808080u);  // bytes that are not 0
                }
            }
        }
        return Counts{(uint32_t)__builtin_amdgcn_readfirstlane(lanes_sum<kWave>(mine)), 0};
    }
    Counts c{0, 0};
    uint32_t last = ~0u;  // the sequence of the last token that counts
    for (uint32_t base = 0; base < n_rows; base += 8 * kWave) {
        uint8_t on[8];
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            const uint32_t n = base + i * kWave + lane_id();
            on[i] = n < n_rows ? a.mask[a.shape.at(n)] : 0;
        }
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            const uint64_t m = __ballot(on[i] != 0);
            c.tokens += __builtin_popcountll(m);
            if (a.reduction != CONDUIT_SEQUENCE_MEAN || m == 0) continue;
            // the first of its sequence: the one before it that counts is of another
            const uint32_t b = div31(base + i * kWave + lane_id(), a.shape.by_T);
            const uint64_t before = m & below_lane();
            const uint32_t other = __shfl(b, before ? 63 - __builtin_clzll(before) : 0, kWave);
            c.rows += __builtin_popcountll(__ballot(on[i] && b != (before ? other : last)));
            last = __shfl(b, 63 - __builtin_clzll(m), kWave);
        }
    }
    return c;
}

// Tokens of a sequence that count, by a wavefront.
__device__ __forceinline__ uint32_t sequence_tokens(const ListedArgs& a, uint32_t b) {
    if (!a.mask) return (uint32_t)a.shape.T;
    if (a.counted) return a.row_count[b];
    const uint8_t* mask = a.mask + (int64_t)b * a.shape.stride;
    uint32_t tokens = 0;
    for (uint32_t base = 0; base < (uint32_t)a.shape.T; base += 8 * kWave) {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            const uint32_t t = base + i * kWave + lane_id();
            tokens += __builtin_popcountll(__ballot(t < (uint32_t)a.shape.T && mask[t]));
        }
    }
    return tokens;
}

// The token's part in the loss.  (a.counted or by a whole wavefront: see the two above)
__device__ __forceinline__ double token_part(const ListedArgs& a, uint32_t n, int64_t at, const Counts& c) {
    PolicyTerms o{};
    o.reduction = a.reduction;
    const uint32_t row = a.reduction == CONDUIT_SEQUENCE_MEAN ? sequence_tokens(a, div31(n, a.shape.by_T)) : 1;
    const double w = token_weight(o, c.tokens, c.rows, row);
    return a.weight ? w * (double)a.weight[at] : w;
}

__device__ __forceinline__ void write_distill_stats(const ListedArgs& a, const double (&v)[kDistillSums], uint32_t tokens) {
    a.stats[0] = (float)(a.scale * v[0]);
    a.stats[1] = (float)(v[1] / (double)(tokens > 0 ? tokens : 1));
    a.stats[2] = (float)tokens;
    if (a.counted) a.head->counts = 0;  // for the next call
}

// `slots` contributions, each left by one wavefront (or workgroup), added up by
// the wavefront of the last: as finish_row does for the policy loss
__device__ __forceinline__ void finish_distill(const ListedArgs& a, uint32_t slot, uint32_t slots, double w_loss, double loss, uint32_t tokens) {
    bool last = false;
    if (lane_id() == 0) {
        store_agent(a.partial + (int64_t)slot * kDistillSums, w_loss);
        store_agent(a.partial + (int64_t)slot * kDistillSums + 1, loss);
        last = draw_ticket(a.head, slot, slots);
    }
    if (!__builtin_amdgcn_readfirstlane((int)last)) return;
    double v[kDistillSums] = {0.0, 0.0};
    for (uint32_t k = lane_id(); k < slots; k += kWave) {
#pragma unroll
        for (int i = 0; i < kDistillSums; ++i) v[i] += load_agent(a.partial + (int64_t)k * kDistillSums + i);
    }
#pragma unroll
    for (int i = 0; i < kDistillSums; ++i) v[i] = wave_sum(v[i]);
    if (lane_id() == 0) write_distill_stats(a, v, tokens);
}

// a row's contribution, by its first wavefront
__device__ __forceinline__ void finish_token(const ListedArgs& a, uint32_t n, double part, float loss, uint32_t tokens) {
    const double w_loss = part == 0.0 ? 0.0 : part * (double)loss;
    if (a.sums == SUM_ROWS) finish_distill(a, n, (uint32_t)(a.shape.B * a.shape.T), w_loss, (double)loss, tokens);
    if (a.sums == SUM_NEXT && lane_id() == 0) {  // (nothing waits for it here: no tickets)
        a.partial[(int64_t)n * kDistillSums] = w_loss;
        a.partial[(int64_t)n * kDistillSums + 1] = (double)loss;
    }
}

// what SUM_NEXT left, by one wavefront of the next launch
__device__ __forceinline__ void sum_rows(const ListedArgs& a) {
    const uint32_t rows = (uint32_t)(a.shape.B * a.shape.T), tokens = counted_tokens(a).tokens;
    double v[kDistillSums] = {0.0, 0.0};
    for (uint32_t k = lane_id(); k < rows; k += kWave) {
#pragma unroll
        for (int i = 0; i < kDistillSums; ++i) v[i] += a.partial[(int64_t)k * kDistillSums + i];
    }
#pragma unroll
    for (int i = 0; i < kDistillSums; ++i) v[i] = wave_sum(v[i]);
    if (lane_id() == 0) write_distill_stats(a, v, tokens);
}

// sums over the tokens of a batch of many rows
constexpr int kSumThreads = 256;

__global__ __launch_bounds__(kSumThreads) void k_distill_sum(ListedArgs a) {
    __shared__ double lds[kDistillSums * kSumThreads / kWave];
    double v[kDistillSums] = {0.0, 0.0};
    const uint32_t n_rows = (uint32_t)(a.shape.B * a.shape.T);
    const Counts counts = counted_tokens(a);
    for (uint32_t n = blockIdx.x * kSumThreads + threadIdx.x; n < n_rows; n += gridDim.x * kSumThreads) {
        const int64_t at = a.shape.at(n);
        if (a.mask && !a.mask[at]) continue;
        const double part = token_part(a, n, at, counts), loss = (double)a.loss[at];
        v[0] += part == 0.0 ? 0.0 : part * loss;
        v[1] += loss;
    }
    block_sum<kSumThreads, kDistillSums>(v, lds);
    if (threadIdx.x < kWave) finish_distill(a, blockIdx.x, gridDim.x, v[0], v[1], counts.tokens);
}

// ---------------------------------------------------------------------------
// short rows: LANES lanes each, up to E elements a lane
// ---------------------------------------------------------------------------
// The list's part of a row bounds it, not the row (fp32, K = 8 of 300, distillation:
// 65,536 rows 82 us; 244 rows of 257, 43% of them live: 7.8, of which a launch is 2.3).
// So many rows of up to 64 choices with short lists share a wavefront, 16 lanes each
// (65,536 rows of 18, K = 8: 23 us, a wavefront each 77; scores of 5 choices 8.6 against
// 29).  The loss's workgroups are few, since each draws a ticket; a large batch has
// them of 1,024 threads (256: 103 us for the 77).  Five wavefronts a SIMD (96
// registers) cover each other; four take 2 to 4% longer.
template <bool BF16, int MODE, int NT, int LANES, int E>
__global__ __launch_bounds__(NT, MODE == DISTILL ? 5 : 1) void k_listed_short(ListedArgs a) {
    using T = typename Elem<BF16>::T;
    constexpr int kRows = NT / LANES;
    static_assert(E <= 32 && kRows <= kWave, "a word of bits a lane");
    __shared__ uint32_t s_bits[kRows][LANES];
    __shared__ double s_sum[kDistillSums][kRows];
    const uint32_t w = LANES == kWave ? __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) : threadIdx.x / LANES, l = group_lane<LANES>();
    const uint32_t n_rows = (uint32_t)(a.shape.B * a.shape.T), V = (uint32_t)a.V;
    uint32_t* bits = s_bits[w];
    double sums[kDistillSums] = {0.0, 0.0};
    const Counts counts = MODE == DISTILL ? counted_tokens(a) : Counts{};
    for (uint32_t n = block_number() * kRows + w; n < n_rows; n += gridDim.x * gridDim.y * kRows) {
        const int64_t at = a.shape.at(n);
        const T* x = static_cast<const T*>(a.x.data) + a.x.at(n, a.shape);
        T* dx = MODE == DISTILL && a.has_dx ? static_cast<T*>(a.dx.data) + a.dx.at(n, a.shape) : nullptr;
        if (a.mask && !a.mask[at]) {
            write_nothing<MODE, LANES>(a, n, at);
            if (MODE == DISTILL && a.has_dx) {
                for (uint32_t j = l; j < V; j += LANES) dx[j] = Elem<BF16>::round(0.0f);
            }
            continue;
        }
        Listed e;
        load_ids<LANES>(a, n, e);
        if constexpr (MODE == DISTILL) load_values<LANES>(a, a.teacher, n, e);
        float v[E];
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = l + i * LANES < V ? Elem<BF16>::one(x[l + i * LANES]) : kNone;
        check_ids<MODE == DISTILL>(a, e, true);
        load_scores<BF16>(x, e);
        wave_fence();  // (the last row's bits are read)
        bits[l] = 0;
        wave_fence();
        const bool twice = mark<LANES>(e, [&](uint32_t id, uint32_t** word, uint32_t* bit) {
            *word = bits + id % LANES;
            *bit = 1u << id / LANES;
            return true;
        });
        if (twice) find_first<false, LANES>(e, a.K);
        wave_fence();
        const uint32_t marked = bits[l];
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = marked >> i & 1 ? kNone : v[i];
        Mass others = no_mass();
        accumulate_mass(others, v, a.c);
        others = join_group<LANES>(others, a.c);
        if constexpr (MODE == SCORES) {
            write_scores<LANES>(a, n, at, e, others);
        } else {
            const double part = token_part(a, n, at, counts);
            const ListedRow o = distill_row<LANES>(a, e, others, row_mass<LANES>(e, others, a.c, a.inv_t), teacher_row<LANES>(a, e), (float)(part * a.scale));
            if (l == 0) a.loss[at] = o.loss;
            sums[0] += part == 0.0 ? 0.0 : part * (double)o.loss;
            sums[1] += (double)o.loss;
            if (a.has_dx) {
                const bool none = o.coef == 0.0f;  // whatever the scores are
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const uint32_t j = l + i * LANES;
                    if (j < V && !(marked >> i & 1))
                        dx[j] = Elem<BF16>::round(none ? 0.0f : o.coef * exp2_fast((v[i] - o.base) * a.c));
                }
#pragma unroll
                for (int i = 0; i < kLists; ++i)
                    if (e.first[i]) dx[e.id[i]] = Elem<BF16>::round(listed_gradient(a, o, e.x[i], e.y[i]));
            }
        }
    }
    if constexpr (MODE == DISTILL) {
        if (l == 0) {
            s_sum[0][w] = sums[0];
            s_sum[1][w] = sums[1];
        }
        __syncthreads();
        if (threadIdx.x >= kWave) return;
        const double v0 = lanes_sum<kRows>(s_sum[0][lane_id() % kRows]), v1 = lanes_sum<kRows>(s_sum[1][lane_id() % kRows]);
        finish_distill(a, blockIdx.x, gridDim.x, v0, v1, counts.tokens);
    }
}

// ---------------------------------------------------------------------------
// longer rows, or parts of them, whose gradient is not written here: a workgroup
// each
// ---------------------------------------------------------------------------
// HBM bounds it (4,088 rows of 50,001 fp32, K = 32: 131 us, 6.2 TB/s; 36% of them live
// 56, 5.3), few rows are bound by latency (64 of 128,000 bf16 in parts, K = 5: 8.0 us on
// logits in the caches, of which a launch is 2.3 and the loads 2).  The list, the
// token's weight and the teacher's side are the first wavefront's, under the row's
// loads; a number met twice is noted with a part's sums, so that the join looks for
// duplicates (110 ns an entry) only then.
constexpr int kScanVectors = 8;  // vectors a lane and tile

// a row's list with its scores, and the teacher's side of it, by one wavefront
struct RowList {
    Listed e;
    Teacher t;
    double part;      // the token's weight
    uint32_t tokens;  // that count
    bool twice;   // a number may be there more than once
};

// what does not wait for the row; check: entries that are no choices are flagged
template <int MODE>
__device__ __forceinline__ void load_list(const ListedArgs& a, uint32_t n, bool check, RowList& r) {
    load_ids(a, n, r.e);
    if constexpr (MODE == DISTILL) load_values(a, a.teacher, n, r.e);
    check_ids<MODE == DISTILL>(a, r.e, check);
}

// the token's weight, behind the row's loads
template <int MODE>
__device__ __forceinline__ void load_weight(const ListedArgs& a, uint32_t n, int64_t at, RowList& r) {
    if constexpr (MODE == DISTILL) {
        const Counts counts = counted_tokens(a);
        r.tokens = counts.tokens;
        r.part = token_part(a, n, at, counts);
    }
}

// the row from its others' sum, by one wavefront
template <bool BF16, int MODE>
__device__ __forceinline__ void finish_listed(const ListedArgs& a, uint32_t n, int64_t at, const Mass& others, RowList& r) {
    if (r.twice) {
        find_first<false>(r.e, a.K);
        if constexpr (MODE == DISTILL) r.t = teacher_row(a, r.e);
    }
    if constexpr (MODE == SCORES) {
        write_scores(a, n, at, r.e, others);
    } else {
        const ListedRow o = distill_row(a, r.e, others, row_mass(r.e, others, a.c, a.inv_t), r.t, (float)(r.part * a.scale));
        if (lane_id() == 0) a.loss[at] = o.loss;
        if (lane_id() == 0 && a.has_dx) a.row[n] = o;
        finish_token(a, n, r.part, o.loss, r.tokens);
    }
}

// A row's parts leave their others' maximum and sum, and whether they met a number
// twice (0 or 1: a choice is in one part alone).
constexpr int kPartWords = 3;

// the join of a row's parts, by one wavefront
template <bool BF16, int MODE>
__device__ __forceinline__ void join_listed(const ListedArgs& a, uint32_t n, int64_t at, RowList& r) {
    Mass all = no_mass();
    bool twice = false;
    for (int32_t p = lane_id(); p < a.parts; p += kWave) {
        const float* q = a.part + kPartWords * ((int64_t)n * a.parts + p);
        const float m = __hip_atomic_load(q, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const float s = __hip_atomic_load(q + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        twice |= __hip_atomic_load(q + 2, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != 0.0f;
        const float top = m > all.m ? m : all.m;
        all.s = all.s * exp2_fast(all.m == top ? 0.0f : (all.m - top) * a.c) + s * exp2_fast(m == top ? 0.0f : (m - top) * a.c);
        all.m = top;
    }
    r.twice = __ballot(twice) != 0;
    finish_listed<BF16, MODE>(a, n, at, join_mass<kWave>(all, a.c), r);
}

template <bool BF16, int MODE, bool ONCE>
__global__ __launch_bounds__(kListedThreads) void k_listed_scan(ListedArgs a) {
    using E = Elem<BF16>;
    using T = typename E::T;
    constexpr int kPer = E::kPer;
    constexpr int kWords = kScanVectors * kPer / 32;  // of bits, a lane and tile
    constexpr uint32_t kTile = kListedThreads * kScanVectors;
    extern __shared__ uint32_t s_bits[];  // [tiles][kListedThreads][kWords]
    __shared__ uint32_t s_tail;
    __shared__ Mass s_mass[kListedThreads / kWave];
    const uint32_t item = block_number(), tid = threadIdx.x;
    if (item >= (uint32_t)(a.shape.B * a.shape.T) * (uint32_t)a.parts) return;
    const uint32_t n = div31(item, a.by_parts), part = item - n * (uint32_t)a.parts;
    const int64_t at = a.shape.at(n);
    if (a.mask && !a.mask[at]) {
        if (part == 0 && tid < kWave) {
            write_nothing<MODE>(a, n, at);
            if constexpr (MODE == DISTILL) finish_token(a, n, 0.0, 0.0f, counted_tokens(a).tokens);
        }
        return;
    }
    const T* x = static_cast<const T*>(a.x.data) + a.x.at(n, a.shape);
    const RowVectors<BF16, 4> row(x, (uint32_t)a.V);
    const T* vx = x + row.head;  // the vectors
    const uint32_t nv = row.count;
    const uint32_t lo = part * (uint32_t)a.per < nv ? part * (uint32_t)a.per : nv, hi = lo + a.per < nv ? lo + a.per : nv;
    RowList r{};
    if (tid < kWave) load_list<MODE>(a, n, part == 0, r);  // (ahead of the row's loads)
    u32x4 v[kScanVectors];
    auto load = [&](uint32_t base) {
#pragma unroll
        for (int k = 0; k < kScanVectors; ++k) {
            const uint32_t i = base + k * kListedThreads + tid;
            v[k] = i < hi ? read16<ONCE>(vx + (size_t)i * kPer) : no_vector<BF16>();
        }
    };
    load(lo);
    const uint32_t tiles = (hi - lo + kTile - 1) / kTile;
    for (uint32_t i = tid; i < tiles * kListedThreads * kWords; i += kListedThreads) s_bits[i] = 0;
    if (tid == 0) s_tail = 0;
    __syncthreads();
    if (tid < kWave) {
        load_scores<BF16>(x, r.e);
        load_weight<MODE>(a, n, at, r);
        r.twice = mark(r.e, [&](uint32_t id, uint32_t** word, uint32_t* bit) {
            uint32_t i, j;
            row.find(id, &i, &j);
            if (i >= nv) {
                *word = &s_tail;
                *bit = 1u << j;
                return part == 0;
            }
            if (i < lo || i >= hi) return false;
            const uint32_t q = i - lo, tile = q / kTile, slot = q % kTile / kListedThreads, at_bit = slot * kPer + j;
            *word = s_bits + (tile * kListedThreads + q % kListedThreads) * kWords + at_bit / 32;
            *bit = 1u << at_bit % 32;
            return true;
        });
        if constexpr (MODE == DISTILL) r.t = teacher_row(a, r.e);
    }
    __syncthreads();
    Mass others = no_mass();
    if (part == 0 && tid < row.beside()) {
        const float f[1] = {s_tail >> tid & 1 ? kNone : E::one(x[row.beside_at(tid)])};
        accumulate_mass(others, f, a.c);
    }
    for (uint32_t tile = 0; tile < tiles; ++tile) {
        if (tile > 0) load(lo + tile * kTile);
        uint32_t bits[kWords], any = 0;
#pragma unroll
        for (int i = 0; i < kWords; ++i) any |= bits[i] = s_bits[(tile * kListedThreads + tid) * kWords + i];
        if (any) {
#pragma unroll
            for (int k = 0; k < kScanVectors; ++k) v[k] = without<BF16>(v[k], bits[k * kPer / 32] >> k * kPer % 32 & ((1u << kPer) - 1));
        }
        accumulate_mass_tile<BF16>(others, v, a.c);
    }
    others = join_mass<kWave>(others, a.c);
    if (lane_id() == 0) s_mass[tid / kWave] = others;
    __syncthreads();
    if (tid >= kWave) return;
    others = join_mass<kListedThreads / kWave>(s_mass[lane_id() % (kListedThreads / kWave)], a.c);
    if (a.parts == 1) return finish_listed<BF16, MODE>(a, n, at, others, r);
    bool last = false;
    if (lane_id() == 0) {
        float* mine = a.part + kPartWords * (int64_t)item;
        __hip_atomic_store(mine, others.m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(mine + 1, others.s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(mine + 2, r.twice ? 1.0f : 0.0f, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // acknowledged before the ticket is drawn
        if (a.row_ticket) last = draw_last(a.row_ticket + n * kTicketStep, (uint32_t)a.parts);
    }
    if (__builtin_amdgcn_readfirstlane((int)last)) join_listed<BF16, MODE>(a, n, at, r);
}

// the join of many split rows, by a launch of its own: a wavefront a row
template <bool BF16, int MODE>
__global__ __launch_bounds__(kListedThreads) void k_listed_join(ListedArgs a) {
    const uint32_t n = block_number() * (kListedThreads / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    if (n >= (uint32_t)(a.shape.B * a.shape.T)) return;
    const int64_t at = a.shape.at(n);
    if (a.mask && !a.mask[at]) return;
    RowList r{};
    load_list<MODE>(a, n, false, r);
    load_weight<MODE>(a, n, at, r);
    load_scores<BF16>(static_cast<const typename Elem<BF16>::T*>(a.x.data) + a.x.at(n, a.shape), r.e);
    if constexpr (MODE == DISTILL) r.t = teacher_row(a, r.e);
    join_listed<BF16, MODE>(a, n, at, r);
}

// ---------------------------------------------------------------------------
// rows that fit the registers of WAVES wavefronts, K vectors a lane
// ---------------------------------------------------------------------------
// A row crosses memory once in each direction.  HBM bounds it where the rows are
// wide or fp32 (4,088 rows of 32,001 fp32, 36% of them live: 134 us, 5.3 TB/s; 8,192 of
// 128,000 bf16: 557, 5.1; a large copy reaches 4.7-4.9, a fill 6.9), the steps of a row
// one after the other where they are not: load, sum, join, the list's part, store.  A
// lane takes up to 16 vectors, so that a row has few wavefronts to join and a compute
// unit several rows at different steps, and what a lane's vectors have beyond the row
// is left out (read and written, V x rows bf16, before rows started at boundaries:
// 5,001 x 16,384 on one wavefront 91 us, on four 166-235; 10,001 x 8,192 on two 90, on
// four 109; 50,001 x 2,048 on eight 110, on sixteen 137; fp32, with half the work in a
// vector, is better on sixteen of 8 vectors: 32,001 x 4,088 147, on eight of 16 156).
// The list is loaded ahead of the row and its scores behind it.  Up to 1,024 vectors
// the scores alone go this way too: a row's steps hide under those of three others
// (65,536 rows of 2,100 bf16, K = 5: 79 us, a workgroup a row 327), and rows from 513
// choices on are better loaded in vectors (2,000 bf16: 70, by elements 198; distilled
// 194 against 608).
constexpr int kRowVectors = 16 * 1024;  // of a workgroup of 1,024

template <int WAVES>
__device__ __forceinline__ void row_sync() {
    if constexpr (WAVES == 1) wave_fence();
    else __syncthreads();
}

template <bool BF16, int MODE, int WAVES, int K, bool PAST>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * kWave) void k_listed_rows(ListedArgs a) {
    using E = Elem<BF16>;
    using T = typename E::T;
    constexpr int kPer = E::kPer;
    constexpr int NT = WAVES * kWave;
    constexpr int kWords = K * kPer / 32;
    constexpr int kRows = WAVES == 1 ? 256 / kWave : 1;  // of a workgroup
    __shared__ uint32_t s_bits[kRows][NT][kWords];
    __shared__ uint32_t s_beside[kRows][2];
    __shared__ Mass s_mass[WAVES];
    __shared__ ListedRow s_row;
    static_assert(MODE == DISTILL || WAVES == 1);
    constexpr int LIST = MODE == SCORES ? SCORES : DISTILL;
    const uint32_t w = WAVES == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) : 0;
    const uint32_t n = block_number() * kRows + w, tid = threadIdx.x % NT;
    if (n >= (uint32_t)(a.shape.B * a.shape.T)) return;
    const int64_t at = a.shape.at(n);
    const T* x = static_cast<const T*>(a.x.data) + a.x.at(n, a.shape);
    T* dx = MODE == DISTILL ? static_cast<T*>(a.dx.data) + a.dx.at(n, a.shape) : nullptr;
    using Vectors = RowVectors<BF16, MODE == DISTILL ? 64 : 4>;
    static_assert(Vectors::kMostBeside <= kWave);
    const Vectors row(MODE == DISTILL ? dx : x, (uint32_t)a.V);
    const T* vx = x + row.head;  // the vectors
    T* vdx = MODE == DISTILL ? dx + row.head : nullptr;
    const uint32_t nv = row.count, beside = row.beside();
    if (a.mask && !a.mask[at]) {
        if constexpr (MODE == DISTILL) {
            for (uint32_t i = tid; i < nv; i += NT) put16<PAST>(vdx + (size_t)i * kPer, u32x4{0, 0, 0, 0});
            if (tid < beside) dx[row.beside_at(tid)] = E::round(0.0f);
        }
        if (tid < kWave) {
            write_nothing<LIST>(a, n, at);
            if constexpr (LIST == DISTILL) finish_token(a, n, 0.0, 0.0f, counted_tokens(a).tokens);
        }
        return;
    }
    // the list first: its scores' addresses wait for it under the row's loads
    RowList r{};
    if (tid < kWave) load_list<LIST>(a, n, true, r);
    // vectors k of all lanes are beyond the row from some k on: nothing is done for them
    u32x4 v[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const uint32_t i = k * NT + tid;
        v[k] = no_vector<BF16>();
        if (k * NT < nv && i < nv) v[k] = load16(vx + (size_t)i * kPer);
    }
    float xt = tid < beside ? E::one(x[row.beside_at(tid)]) : kNone;
    if (tid < kWave) {
        load_scores<BF16>(x, r.e);
        load_weight<LIST>(a, n, at, r);
    }
#pragma unroll
    for (int i = 0; i < kWords; ++i) s_bits[w][tid][i] = 0;
    if (tid < 2) s_beside[w][tid] = 0;
    row_sync<WAVES>();
    if (tid < kWave) {
        r.twice = mark(r.e, [&](uint32_t id, uint32_t** word, uint32_t* bit) {
            uint32_t i, j;
            row.find(id, &i, &j);
            const uint32_t at_bit = i / NT * kPer + j;
            *word = i < nv ? &s_bits[w][i % NT][at_bit / 32] : &s_beside[w][j / 32];
            *bit = 1u << (i < nv ? at_bit : j) % 32;
            return true;
        });
        if (r.twice) find_first<false>(r.e, a.K);
    }
    row_sync<WAVES>();
    if (LIST == DISTILL && tid < kWave) r.t = teacher_row(a, r.e);
    uint32_t bits[kWords], any = 0;
#pragma unroll
    for (int i = 0; i < kWords; ++i) any |= bits[i] = s_bits[w][tid][i];
    auto listed = [&](int k) { return bits[k * kPer / 32] >> k * kPer % 32 & ((1u << kPer) - 1); };
    if (any) {
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (listed(k)) v[k] = without<BF16>(v[k], listed(k));
    }
    const bool listed_beside = tid < beside && (s_beside[w][tid / 32] >> tid % 32 & 1);
    if (listed_beside) xt = kNone;
    Mass others = no_mass();
    {
        float top = xt;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (k * NT < nv) {
                float f[kPer];
                E::unpack(v[k], f);
                top = top_of(f, top);
            }
        }
        others.m = top;
        const float f[1] = {xt};
        add_mass(others, f, a.c);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (k * NT < nv) {
                float f[kPer];
                E::unpack(again(v[k]), f);
                add_mass(others, f, a.c);
            }
        }
    }
    others = join_mass<kWave>(others, a.c);
    if constexpr (WAVES > 1) {
        if (lane_id() == 0) s_mass[tid / kWave] = others;
        __syncthreads();
        others = join_mass<WAVES>(s_mass[lane_id() % WAVES], a.c);
    }
    if constexpr (MODE == SCORES) {
        write_scores(a, n, at, r.e, others);
        return;
    }
    ListedRow o{};
    if (tid < kWave) {
        o = distill_row(a, r.e, others, row_mass(r.e, others, a.c, a.inv_t), r.t, (float)(r.part * a.scale));
        if (tid == 0) {
            if constexpr (WAVES > 1) s_row = o;
            a.loss[at] = o.loss;
        }
#pragma unroll
        for (int i = 0; i < kLists; ++i)
            if (MODE == DISTILL && r.e.first[i]) dx[r.e.id[i]] = E::round(listed_gradient(a, o, r.e.x[i], r.e.y[i]));
    }
    if constexpr (MODE == DIVERGENCE) return finish_token(a, n, r.part, o.loss, r.tokens);
    if constexpr (WAVES > 1) {
        __syncthreads();
        o.coef = s_row.coef;
        o.base = s_row.base;
    }
    const float coef = uniform(o.coef), base = uniform(o.base);
    if (coef == 0.0f) {  // whatever the scores are
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = no_vector<BF16>();
        xt = kNone;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const uint32_t i = k * NT + tid;
        if (k * NT >= nv || i >= nv) continue;
        float f[kPer];
        E::unpack(again(v[k]), f);
#pragma unroll
        for (int j = 0; j < kPer; ++j) f[j] = coef * exp2_fast((f[j] - base) * a.c);
        store_others<BF16, PAST>(vdx + (size_t)i * kPer, f, listed(k));
    }
    if (tid < beside && !listed_beside) dx[row.beside_at(tid)] = E::round(coef * exp2_fast((xt - base) * a.c));
    if (tid < kWave) finish_token(a, n, r.part, o.loss, r.tokens);
}

// ---------------------------------------------------------------------------
// the gradient of given gradients of the log-probabilities, or, SPLIT, of the
// divergence of split rows from what their join left: wavefronts take parts of
// kGradK vectors a lane of a row
// ---------------------------------------------------------------------------
// HBM bounds it (2,048 rows of 50,001 fp32, 42% of them live, K = 32: 116 us, 4.8 TB/s).
// Each wavefront loads the list again and marks what is in its part of the row, in 1 KB
// of LDS a workgroup: no barrier.
constexpr int kGradK = 4;

template <bool BF16, bool SPLIT, bool PAST>
__global__ __launch_bounds__(kListedThreads) void k_listed_gradient(ListedArgs a, uint32_t items, uint32_t per_row, Div31 by_row) {
    using E = Elem<BF16>;
    using T = typename E::T;
    constexpr int kPer = E::kPer;
    constexpr uint32_t kWindow = kGradK * kWave;
    static_assert(kGradK * kPer <= 32, "a word of bits a lane");
    __shared__ uint32_t s_bits[kListedThreads / kWave][kWave + 2];  // (the last two: beside the vectors)
    const uint32_t w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = lane_id();
    const uint32_t item = block_number() * (kListedThreads / kWave) + w;
    if (SPLIT && a.sums == SUM_NEXT && item == 0) sum_rows(a);
    if (item >= items) return;
    const uint32_t n = div31(item, by_row), part = item - n * per_row;
    const int64_t at = a.shape.at(n);
    const T* x = static_cast<const T*>(a.x.data) + a.x.at(n, a.shape);
    T* dx = static_cast<T*>(a.dx.data) + a.dx.at(n, a.shape);
    const RowVectors<BF16, 64> row(dx, (uint32_t)a.V);
    const T* vx = x + row.head;  // the vectors
    T* vdx = dx + row.head;
    const uint32_t nv = row.count;
    const uint32_t first = part * kWindow, base = first + lane;
    const bool mine = part == 0 && lane < row.beside();  // the elements beside the vectors
    bool weight = !a.mask || a.mask[at];
    float lse = 0.0f;
    if constexpr (!SPLIT) {
        lse = weight ? a.lse_in[at] : 0.0f;
        weight = weight && lse != kNone;
    }
    if (!weight) {  // nothing counts, or a row without weight
#pragma unroll
        for (int k = 0; k < kGradK; ++k) {
            const uint32_t i = base + k * kWave;
            if (i < nv) put16<PAST>(vdx + (size_t)i * kPer, u32x4{0, 0, 0, 0});
        }
        if (mine) dx[row.beside_at(lane)] = E::round(0.0f);
        return;
    }
    u32x4 v[kGradK];
#pragma unroll
    for (int k = 0; k < kGradK; ++k) {
        const uint32_t i = base + k * kWave;
        v[k] = i < nv ? load16(vx + (size_t)i * kPer) : u32x4{0, 0, 0, 0};
    }
    const float xt = mine ? E::one(x[row.beside_at(lane)]) : 0.0f;
    Listed e;
    load_ids(a, n, e);
    load_values(a, SPLIT ? a.teacher : a.g, n, e);
    check_ids<SPLIT>(a, e, !SPLIT && part == 0);
    ListedRow o{};
    float sum = 0.0f, h = 0.0f, rest = 0.0f;  // of the gradients; of log p_rest; log p_rest
    if constexpr (SPLIT) {
        o = a.row[n];
    } else {
#pragma unroll
        for (int i = 0; i < kLists; ++i) sum += e.on[i] ? e.y[i] : 0.0f;
        sum = uniform(lanes_sum<kWave>(sum));
        if (a.h) {
            rest = a.rest_in[at];
            h = rest == kNone ? 0.0f : a.h[at];  // (no others: their log-probability stays -infinity)
        }
    }
    // the listed choices of this part of the row
    uint32_t* bits = s_bits[w];
    bits[lane] = 0;
    if (lane < 2) bits[kWave + lane] = 0;
    wave_fence();
#pragma unroll
    for (int i = 0; i < kLists; ++i) {
        uint32_t k, j;
        row.find((uint32_t)e.id[i], &k, &j);
        e.on[i] = e.on[i] && (k < nv ? k - first < kWindow : part == 0);
        e.first[i] = e.on[i];
    }
    load_scores<BF16>(x, e);
    const bool twice = mark(e, [&](uint32_t id, uint32_t** word, uint32_t* bit) {
        uint32_t k, j;
        row.find(id, &k, &j);
        *word = bits + (k < nv ? k % kWave : kWave + j / 32);
        *bit = 1u << (k < nv ? (k - first) / kWave * kPer + j : j % 32);
        return true;
    });
    if (twice) find_first<!SPLIT>(e, a.K);
    wave_fence();
    const uint32_t marked = bits[lane], marked_beside = bits[kWave + lane / 32] >> lane % 32 & 1;
    const LogP by{a.inv_t, a.inv_lo, a.lowest, lse};
    // of any other choice: coef times its share of the rest (with h), or its probability
    float coef, shift = 0.0f;
    if constexpr (SPLIT) {
        coef = o.coef;
    } else if (h == 0.0f) {
        coef = -sum * a.inv_t;
    } else {
        shift = rest;
        coef = -fmaf(sum, exp_fast(rest), h * expm1_fast(rest)) * a.inv_t;
    }
    // (held: the log-probability of a choice, or of one among the others, is 0 at most, which the rounding of a large lse
    // or rest would pass: 2^-24 of it, 64 at 1e9.  NaN stays.)
    auto log_p = [&](float f, float less, auto held) {
        const float q = by.of(f) - less;
        return held && q > 0.0f ? 0.0f : q;
    };
    auto write = [&](auto held) {
        auto other = [&](float f) {
            if (coef == 0.0f) return 0.0f;
            if constexpr (SPLIT) return coef * exp2_fast((f - o.base) * a.c);
            return coef * exp2_fast(log_p(f, shift, held) * kLog2e);
        };
#pragma unroll
        for (int k = 0; k < kGradK; ++k) {
            const uint32_t i = base + k * kWave;
            float f[kPer];
            E::unpack(v[k], f);
#pragma unroll
            for (int j = 0; j < kPer; ++j) f[j] = other(f[j]);
            if (i < nv) store_others<BF16, PAST>(vdx + (size_t)i * kPer, f, marked >> k * kPer & ((1u << kPer) - 1));
        }
        if (mine && !marked_beside) dx[row.beside_at(lane)] = E::round(other(xt));
#pragma unroll
        for (int i = 0; i < kLists; ++i) {
            if (!e.first[i]) continue;
            float d;
            if constexpr (SPLIT) d = listed_gradient(a, o, e.x[i], e.y[i]);
            else d = (e.y[i] - (sum + h) * exp_fast(log_p(e.x[i], 0.0f, held))) * a.inv_t;
            dx[e.id[i]] = E::round(d);
        }
    };
    constexpr float kHeld = 65536.0f;  // (off by 2^-8 at most below; held always, 65,536 rows of 18 choices take 7 to 10% longer)
    if (SPLIT || fabsf(lse) + fabsf(shift) < kHeld) write(std::false_type{});
    else write(std::true_type{});
}

template <bool BF16, bool SPLIT>
hipError_t launch_gradient(const ListedArgs& a, hipStream_t s) {
    const int64_t per_row = gradient_parts(a.V, BF16);
    const int64_t items = a.shape.B * a.shape.T * per_row;  // fewer than 2^31 (the caller's check)
    auto go = [&](auto past) {
        hipLaunchKernelGGL((k_listed_gradient<BF16, SPLIT, decltype(past)::value>),
                           grid_of((items + kListedThreads / kWave - 1) / (kListedThreads / kWave), kListedThreads), dim3(kListedThreads), 0,
                           s, a, (uint32_t)items, (uint32_t)per_row, make_div31((uint32_t)per_row));
    };
    if (a.past) go(std::true_type{});
    else go(std::false_type{});
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// which kernel a row's width takes
// ---------------------------------------------------------------------------
template <bool BF16, int MODE>
hipError_t launch_short(const ListedArgs& a, hipStream_t s) {
    const int64_t rows = a.shape.B * a.shape.T;
    auto go = [&](auto threads, auto lanes, auto elems) {
        constexpr int NT = decltype(threads)::value, LANES = decltype(lanes)::value, E = decltype(elems)::value, kRows = NT / LANES;
        const int64_t want = (rows + kRows - 1) / kRows;
        // (the loss's workgroups each leave a sum)
        const dim3 grid = MODE == DISTILL ? dim3((unsigned)(want < kPolicyBlocks ? want : kPolicyBlocks)) : grid_of(want, NT);
        hipLaunchKernelGGL((k_listed_short<BF16, MODE, NT, LANES, E>), grid, dim3(NT), 0, s, a);
        return hipGetLastError();
    };
    using Small = std::integral_constant<int, kListedThreads>;
    using Large = std::integral_constant<int, 1024>;
    using Part = std::integral_constant<int, kFewLanes>;
    using Wave = std::integral_constant<int, kWave>;
    using Few = std::integral_constant<int, kFewElems>;
    using Elems = std::integral_constant<int, kShortElems>;
    // (a sequence's tokens are counted by whole wavefronts where no launch has counted them, up to kPolicyBlocks rows)
    const bool few = rows > kPolicyBlocks && a.V <= kFewElems * kFewLanes && a.K <= kLists * kFewLanes;
    if constexpr (MODE == DISTILL) {
        if (rows > (few ? 32 : 8) * kPolicyBlocks) return few ? go(Large{}, Part{}, Few{}) : go(Large{}, Wave{}, Elems{});
    }
    return few ? go(Small{}, Part{}, Few{}) : go(Small{}, Wave{}, Elems{});
}

template <bool BF16, int MODE>
hipError_t launch_scan(const ListedArgs& a, hipStream_t s) {
    constexpr int kPer = Elem<BF16>::kPer;
    const int64_t rows = a.shape.B * a.shape.T, items = rows * a.parts;  // fewer than 2^31 (the caller's check)
    constexpr int kTile = kListedThreads * kScanVectors;
    const unsigned lds = (a.per + kTile - 1) / kTile * (kTile * kPer / 8);
    // (with a gradient to come the rows are read again)
    if (a.once && !a.has_dx) hipLaunchKernelGGL((k_listed_scan<BF16, MODE, true>), grid_of(items, kListedThreads), dim3(kListedThreads), lds, s, a);
    else hipLaunchKernelGGL((k_listed_scan<BF16, MODE, false>), grid_of(items, kListedThreads), dim3(kListedThreads), lds, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.parts == 1 || a.row_ticket) return e;
    constexpr int kRows = kListedThreads / kWave;
    hipLaunchKernelGGL((k_listed_join<BF16, MODE>), grid_of((rows + kRows - 1) / kRows, kListedThreads), dim3(kListedThreads), 0, s, a);
    return hipGetLastError();
}

template <bool BF16, int MODE, int WAVES, int K>
hipError_t launch_rows(const ListedArgs& a, hipStream_t s) {
    constexpr int kRows = WAVES == 1 ? 4 : 1, kThreads = WAVES * kRows * kWave;
    const dim3 grid = grid_of((a.shape.B * a.shape.T + kRows - 1) / kRows, kThreads);
    if (MODE == DISTILL && a.past) hipLaunchKernelGGL((k_listed_rows<BF16, MODE, WAVES, K, MODE == DISTILL>), grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((k_listed_rows<BF16, MODE, WAVES, K, false>), grid, dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

template <bool BF16>
hipError_t listed_logprobs(const ListedArgs& a, hipStream_t s) {
    if (a.V <= kShortRow) return launch_short<BF16, SCORES>(a, s);
    if (a.V / Elem<BF16>::kPer <= 16 * kWave) return launch_rows<BF16, SCORES, 1, 16>(a, s);
    return launch_scan<BF16, SCORES>(a, s);
}

template <bool BF16>
hipError_t distill(const ListedArgs& a, hipStream_t s) {
    const int64_t rows = a.shape.B * a.shape.T, nv = a.V / Elem<BF16>::kPer;
    hipError_t e = hipSuccess;
    if (a.counted) {  // the tokens' weight needs their number
        PolicyArgs p{};
        p.shape = a.shape;
        p.o.reduction = a.reduction;
        p.mask = a.mask;
        p.head = a.head;
        p.row_count = a.row_count;
        e = launch_token_count(p, s);
        if (e != hipSuccess) return e;
    }
    if (a.V <= kShortRow) return launch_short<BF16, DISTILL>(a, s);
    if (a.parts == 1 && nv <= 16 * kWave) {
        e = a.has_dx ? launch_rows<BF16, DISTILL, 1, 16>(a, s) : launch_rows<BF16, DIVERGENCE, 1, 16>(a, s);
    } else if (a.parts > 1 || !a.has_dx) {
        e = launch_scan<BF16, DISTILL>(a, s);
        if (e == hipSuccess && a.has_dx) e = launch_gradient<BF16, true>(a, s);
    } else if (nv <= 16 * 2 * kWave) {
        e = launch_rows<BF16, DISTILL, 2, 16>(a, s);
    } else if (nv <= 16 * 4 * kWave) {
        e = launch_rows<BF16, DISTILL, 4, 16>(a, s);
    } else if (nv <= 16 * 8 * kWave) {
        e = launch_rows<BF16, DISTILL, BF16 ? 8 : 16, BF16 ? 16 : 8>(a, s);
    } else {
        e = launch_rows<BF16, DISTILL, 16, 16>(a, s);
    }
    if (e != hipSuccess || a.sums != SUM_LAUNCH) return e;
    const int64_t want = (rows + kSumThreads - 1) / kSumThreads;
    hipLaunchKernelGGL(k_distill_sum, dim3((unsigned)(want < kPolicyBlocks ? want : kPolicyBlocks)), dim3(kSumThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace

// Parts of a row: rows are split where the rows alone would leave compute units
// without a workgroup, into parts of at least four vectors a lane, or where a row
// is wider than one workgroup takes (whole_rows: than its registers hold).
RowParts listed_parts(int64_t rows, int64_t V, bool bf16, bool whole_rows) {
    const int64_t cus = device_cus(), nv = V / (bf16 ? 8 : 4), least = whole_rows && nv > kRowVectors ? kListedThreads * kScanVectors : kPartVectors;
    if (V <= kShortRow || rows <= 0) return RowParts{1, (int32_t)nv};
    int64_t parts = (nv + least - 1) / least;
    if (rows < cus) {
        const int64_t want = (2 * cus + rows - 1) / rows, most = nv / (4 * kListedThreads);
        const int64_t split = want < most ? want : most;
        if (split > parts) parts = split;
    }
    return RowParts{(int32_t)parts, (int32_t)((nv + parts - 1) / parts)};
}

int64_t gradient_parts(int64_t V, bool bf16) {
    const int64_t nv = V / (bf16 ? 8 : 4);
    return nv > 0 ? (nv + kGradK * kWave - 1) / (kGradK * kWave) : 1;
}

hipError_t launch_listed_logprobs(const ListedArgs& a, bool bf16, hipStream_t s) {
    return bf16 ? listed_logprobs<true>(a, s) : listed_logprobs<false>(a, s);
}

hipError_t launch_listed_logprobs_backward(const ListedArgs& a, bool bf16, hipStream_t s) {
    return bf16 ? launch_gradient<true, false>(a, s) : launch_gradient<false, false>(a, s);
}

hipError_t launch_distill_loss(const ListedArgs& a, bool bf16, hipStream_t s) {
    return bf16 ? distill<true>(a, s) : distill<false>(a, s);
}

}  // namespace conduit
