// The K most probable choices of every token with their log-probabilities,
// beside the taken token's, the log-normaliser and the entropy
// (conduit_token_alternatives).
//
// A choice's rank goes by its key: the score's bits in the order of the numbers
// (-0 as 0), then its number counted from the end, so that no two keys are equal
// and the lowest number comes first among equal scores.  Of a row cut into any
// pieces the K-th largest of the pieces' maxima is at most the K-th largest
// score: at least K scores reach it.  With the lanes' running maxima as the
// pieces, which the softmax keeps anyway, few more than K do (256 lanes, K = 64:
// 74 of scores in random places), and these are ranked by counting, each, the
// larger ones.
//
// Where the row does not fit the registers of a wavefront, the pass also leaves
// the maximum of every group of 8 vectors (128 bytes, a cache line) in LDS: only
// groups that reach the bound are read again.
//
// Rows whose scores are equal in many places, or that hold their largest ones in
// few lanes, may have more candidates than the lists take.  Then the K-th
// largest maximum of a group is found exactly.  Fewer than K groups are above
// it, and of those that reach it the first K are enough; among their elements
// the K-th largest key is found bit by bit.
#include <type_traits>

#include "listed_dev.h"
#include "rows_dev.h"

namespace conduit {

namespace {

constexpr int kTopThreads = 256;
constexpr int kTopVectors = 8;   // vectors a lane and tile
constexpr int kGroup = 8;        // vectors a group
constexpr int kMostCandidates = 512;
constexpr int kMostGroups = 512;
constexpr int kShortCandidates = 256;
constexpr int kShortElems = 8;       // elements a lane of a short row
constexpr int64_t kShortRow = kShortElems * kWave;
static_assert(2 * kMostListed <= kMostGroups && kMostListed <= kShortCandidates, "the exact selection fits the lists");
static_assert(kPartVectors % kGroup == 0, "whole groups");

// a score's place among the numbers, at least that of -infinity: 0x007fffff
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);  // (-0 becomes 0)
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_score(uint32_t k) {
    return __builtin_bit_cast(float, k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
__device__ __forceinline__ uint64_t choice_key(float x, uint32_t j) { return (uint64_t)order_key(x) << 32 | (uint32_t)~j; }

// A bound that at least `need` keys reach, and at most `spare` more unless keys are
// equal: bit by bit from the highest in which the largest key `hi` and the least `lo`
// differ.  reach(t): how many reach t (uniform); at least `need` reach lo.
template <typename Reach>
__device__ __forceinline__ uint32_t bound_between(uint32_t hi, uint32_t lo, uint32_t need, uint32_t spare, Reach reach) {
    if (hi == lo) return lo;
    int bit = 31 - __builtin_clz(hi ^ lo);
    uint32_t t = hi >> bit >> 1 << bit << 1;  // what they have in common: all reach it
    for (; bit >= 0; --bit) {
        const uint32_t trial = t | 1u << bit, n = reach(trial);
        if (n < need) continue;
        t = trial;
        if (n <= need + spare) break;
    }
    return t;
}

__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
    return __builtin_amdgcn_readfirstlane(lanes_reduce<kWave>(x, [](uint32_t p, uint32_t q) { return p > q ? p : q; }));
}

// of a wavefront's N keys a lane (need: at most 64 N)
template <int N>
__device__ __forceinline__ uint32_t key_bound(const uint32_t (&key)[N], uint32_t need, uint32_t spare) {
    uint32_t hi = key[0], lo = key[0];
#pragma unroll
    for (int i = 1; i < N; ++i) {
        hi = key[i] > hi ? key[i] : hi;
        lo = key[i] < lo ? key[i] : lo;
    }
    return bound_between(wave_max(hi), ~wave_max(~lo), need, spare, [&](uint32_t least) {
        uint32_t n = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) n += __builtin_popcountll(__ballot(key[i] >= least));
        return n;
    });
}

// a row whose log-normaliser is no number (a NaN or +infinity among its scores) has no ranking
__device__ __forceinline__ bool no_ranking(const Stat& s) { return !(s.s == s.s); }

struct TopRow {
    int32_t* ids;
    float* logps;
    __device__ __forceinline__ TopRow(const TopArgs& a, uint32_t n)
        : ids(static_cast<int32_t*>(a.ids.data) + a.ids.at(n, a.shape)),
          logps(static_cast<float*>(a.logps.data) + a.logps.at(n, a.shape)) {}
};

__device__ __forceinline__ void write_values(const TopArgs& a, int64_t at, float logp, float lse, float entropy) {
    if (a.logp) a.logp[at] = logp;
    if (a.lse) a.lse[at] = lse;
    if (a.entropy) a.entropy[at] = entropy;
}

// K entries of one kind, by NT threads
template <int NT>
__device__ __forceinline__ void fill_row(const TopArgs& a, const TopRow& o, uint32_t tid, int32_t from, int32_t id, float logp) {
    for (int32_t k = from + (int32_t)tid; k < a.K; k += NT) {
        o.ids[k] = id;
        o.logps[k] = logp;
    }
}

// a token that does not count
template <int NT>
__device__ __forceinline__ void write_nothing(const TopArgs& a, uint32_t n, int64_t at, uint32_t tid) {
    if (tid == 0) write_values(a, at, 0.0f, 0.0f, 0.0f);
    fill_row<NT>(a, TopRow(a, n), tid, 0, 0, 0.0f);
}

// the candidates' ranks, f(rank, key) for the first K of them
template <int NT, typename F>
__device__ __forceinline__ void rank(const uint64_t* cand, uint32_t n, int32_t K, uint32_t tid, F f) {
    for (uint32_t c = tid; c < n; c += NT) {
        const uint64_t key = cand[c];
        uint32_t r = 0;
#pragma unroll 8
        for (uint32_t j = 0; j < n; ++j) r += cand[j] > key;
        if (r < (uint32_t)K) f(r, key);
    }
}

// the row's K choices from its candidates, by NT threads
template <int NT>
__device__ __forceinline__ void write_ranked(const TopArgs& a, uint32_t row, const uint64_t* cand, uint32_t n, const RowValues& r,
                                             uint32_t tid) {
    const TopRow o(a, row);
    const bool weight = r.inv_s != 0.0f;
    const float base = uniform(r.base), log2_s = uniform(r.log2_s);
    rank<NT>(cand, n, a.K, tid, [&](uint32_t k, uint64_t key) {
        o.ids[k] = (int32_t)~(uint32_t)key;
        o.logps[k] = weight ? log_p_from(key_score((uint32_t)(key >> 32)) - base, a.c, a.inv_t, log2_s) : kNone;
    });
    if (n < (uint32_t)a.K) fill_row<NT>(a, o, tid, (int32_t)n, -1, kNone);  // fewer choices than K
}

// does the token count, with its taken token (flagged where that is outside the vocabulary)
__device__ __forceinline__ bool counts(const TopArgs& a, int64_t at, bool flags, int32_t* tok) {
    *tok = 0;
    if (a.mask && !a.mask[at]) return false;
    if (!a.tokens) return true;
    *tok = a.tokens[at];
    if (*tok >= 0 && *tok < a.V) return true;
    if (flags) flag_error(a.err, ERR_TOKEN);
    return false;
}

// ---------------------------------------------------------------------------
// a lane's statistics over tiles of vectors
// ---------------------------------------------------------------------------
// The sums go by d' = c x - B in one rounding, with B the rounded c max x: what it
// is off by is a factor of the whole sum, which stat() takes out.  (That leaves 7.5
// cycles of a fp32 element and 9.5 of a bf16 one, 4 of them of the exponential, of
// 9.5 and 11.5.)  A choice at -infinity would give 0 times -infinity: a tile whose
// weighted sum is no number is summed again with the exponents held, and so are
// those after it.
//   The rounding of B is at most half its last place, 1/2 below kFar: a factor of at
// most sqrt 2.  It grows with B, from 2^31 on past the exponents' range, so from kFar
// on (large scores, choices forbidden by a large finite value, small temperatures)
// a wavefront's sums go by c (x - max x) as in softmax_dev.h, with nothing to take out.
// (4,096 rows of 128,000 bf16 with half of the choices at -1e9, K = 64: 190 us, of
// ordinary scores 180; fp32 rows and narrower ones take the same time either way.)
constexpr float kFar = 0x1p24f;

struct TileStat {
    Stat st = no_stat();
    float B = 0.0f;
    bool held = false, far = false;  // uniform (far: c max x was beyond kFar)

    // as Stat has them, which go by c (x - max x)
    __device__ __forceinline__ Stat stat(float c) const {
        if (far || st.m == kNone) return st;
        const float d = fmaf(st.m, c, -B), e = exp2_fast(-d);
        return Stat{st.m, st.s * e, fmaf(-d, st.s, st.u) * e};
    }

    template <bool BF16, bool HELD, int STRIDE, int N>
    __device__ __forceinline__ void sum(const u32x4 (&v)[N], float c, uint32_t left) {
        using E = Elem<BF16>;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if (HELD && k * STRIDE >= left) continue;  // nothing but padding
            float f[E::kPer];
            E::unpack(again(v[k]), f);
#pragma unroll
            for (int j = 0; j < E::kPer; ++j) {
                const float d = fmaf(f[j], c, -B), e = exp2_fast(d);
                st.s += e;
                st.u = fmaf(e, HELD ? fmaxf(d, kFloor) : d, st.u);
            }
        }
    }

    // top: the largest of the lane's vectors, STRIDE apart; left: the row's vectors from the tile on
    template <bool BF16, int STRIDE, int N>
    __device__ __forceinline__ void add_tile(const u32x4 (&v)[N], float top, float c, uint32_t left) {
        const float b = top * c;
        if (!far && __ballot(top > st.m && !(fabsf(b) < kFar)) != 0) {
            st = stat(c);
            far = true;
        }
        if (far) {
            raise(st, top, c);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                float f[Elem<BF16>::kPer];
                Elem<BF16>::unpack(again(v[k]), f);
                conduit::add(st, f, c);
            }
            return;
        }
        if (top > st.m) {
            const float d = fminf(B - b, 0.0f), e = exp2_fast(d);
            st.u = fmaf(st.s, fmaxf(d, kFloor), st.u) * e;
            st.s *= e;
            st.m = top;
            B = b;
        }
        if (left >= N * STRIDE && !held) {
            const Stat before = st;
            sum<BF16, false, STRIDE>(v, c, left);
            if (__ballot(!(st.u == st.u)) == 0) return;
            st = before;
            held = true;
        }
        sum<BF16, true, STRIDE>(v, c, left);
    }
};

// ---------------------------------------------------------------------------
// the shortest rows: LANES lanes each, up to kFewElems elements a lane
// ---------------------------------------------------------------------------
// Every choice is ranked against all others, with the row's keys in LDS.  Latency
// bounds it (16,384 rows of 18 fp32, K = 5: 4.7 us; on a wavefront a row 13.3; of 64: 9.9
// against 15.8, but of 100 on 32 lanes 19.7 against 16.1).
constexpr int kFewElems = 4;

template <bool BF16, int LANES>
__global__ __launch_bounds__(kTopThreads) void k_top_few(TopArgs a) {
    using E = Elem<BF16>;
    using T = typename E::T;
    constexpr int kRows = kTopThreads / LANES, kMost = LANES * kFewElems;
    __shared__ __align__(16) uint64_t s_key[kRows][kMost + 2];  // (2: rows' banks apart)
    const uint32_t l = threadIdx.x % LANES, g = threadIdx.x / LANES, n = block_number() * kRows + g;
    if (n >= (uint32_t)(a.shape.B * a.shape.T)) return;
    const int64_t at = a.shape.at(n);
    int32_t tok;
    if (!counts(a, at, l == 0, &tok)) return write_nothing<LANES>(a, n, at, l);
    const T* x = static_cast<const T*>(a.x.data) + a.x.at(n, a.shape);
    float v[kFewElems], xa = 0.0f;
#pragma unroll
    for (int i = 0; i < kFewElems; ++i) {
        const int32_t j = l + i * LANES;
        v[i] = j < a.V ? E::one(x[j]) : kNone;
        if (j == tok) xa = v[i];  // (the others hold 0)
    }
    uint64_t key[kFewElems];  // 0 beyond the row
#pragma unroll
    for (int i = 0; i < kFewElems; ++i) {
        const uint32_t j = l + i * LANES;
        key[i] = j < a.V ? choice_key(v[i], j) : 0;
        s_key[g][j] = key[i];
    }
    Stat st = no_stat();
    accumulate(st, v, a.c);
    st = join_lanes<LANES>(st, a.c);
    const RowValues r = row_values(st, lanes_sum<LANES>(xa), a.c, a.inv_t, a.inv_lo);
    if (l == 0) write_values(a, at, r.logp, r.lse, r.entropy);
    const TopRow o(a, n);
    if (no_ranking(st)) return fill_row<LANES>(a, o, l, 0, -1, __builtin_nanf(""));
    wave_fence();
    uint32_t rank[kFewElems] = {};
    for (uint32_t m = 0; m < a.V; m += 2) {
        const uint64_t p = s_key[g][m], q = s_key[g][m + 1];
#pragma unroll
        for (int i = 0; i < kFewElems; ++i) rank[i] += (uint32_t)(p > key[i]) + (uint32_t)(q > key[i]);
    }
#pragma unroll
    for (int i = 0; i < kFewElems; ++i) {
        if (key[i] == 0 || rank[i] >= (uint32_t)a.K) continue;
        o.ids[rank[i]] = l + i * LANES;
        o.logps[rank[i]] = r.inv_s != 0.0f ? log_p_from(v[i] - r.base, a.c, a.inv_t, r.log2_s) : kNone;
    }
    if (a.V < a.K) fill_row<LANES>(a, o, l, (int32_t)a.V, -1, kNone);
}

// ---------------------------------------------------------------------------
// short rows: a wavefront each, E elements a lane
// ---------------------------------------------------------------------------
template <bool BF16>
__global__ __launch_bounds__(kTopThreads) void k_top_short(TopArgs a) {
    using T = typename Elem<BF16>::T;
    constexpr int E = kShortElems;
    __shared__ uint64_t s_cand[kTopThreads / kWave][kShortCandidates];
    const uint32_t w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), l = lane_id();
    const uint32_t n = block_number() * (kTopThreads / kWave) + w;
    if (n >= (uint32_t)(a.shape.B * a.shape.T)) return;
    uint64_t* cand = s_cand[w];
    const int64_t at = a.shape.at(n);
    int32_t tok;
    if (!counts(a, at, l == 0, &tok)) return write_nothing<kWave>(a, n, at, l);
    const T* x = static_cast<const T*>(a.x.data) + a.x.at(n, a.shape);
    float v[E];
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = l + i * kWave < a.V ? Elem<BF16>::one(x[l + i * kWave]) : kNone;
    const float xa = Elem<BF16>::one(x[tok]);
    Stat st = no_stat();
    accumulate(st, v, a.c);
    const float mine = st.m;
    st = join_lanes<kWave>(st, a.c);
    const RowValues r = row_values(st, xa, a.c, a.inv_t, a.inv_lo);
    if (l == 0) write_values(a, at, r.logp, r.lse, r.entropy);
    if (no_ranking(st)) return fill_row<kWave>(a, TopRow(a, n), l, 0, -1, __builtin_nanf(""));
    uint32_t key[E];  // 0 beyond the row
#pragma unroll
    for (int i = 0; i < E; ++i) key[i] = l + i * kWave < a.V ? order_key(v[i]) : 0;
    uint32_t bound = 1;
    if (a.K < kWave && a.V > kWave) {
        const uint32_t top[1] = {order_key(mine)};
        bound = key_bound(top, (uint32_t)a.K, (uint32_t)a.K / 4);
    }
    auto reach = [&](uint32_t least) {
        uint32_t n = 0;
#pragma unroll
        for (int i = 0; i < E; ++i) n += __builtin_popcountll(__ballot(key[i] >= least));
        return n;
    };
    uint32_t some = reach(bound), ties = kShortCandidates;  // (all that reach the bound)
    if (some > (uint32_t)a.K + (uint32_t)a.K / 2 + 16) {  // ranking takes the square of their number
        bound = key_bound(key, (uint32_t)a.K, (uint32_t)a.K / 4);
        some = reach(bound);
    }
    if (some > kShortCandidates) {
        bound = key_bound(key, (uint32_t)a.K, 0);
        ties = (uint32_t)a.K - reach(bound + 1);  // (exactly K reach it, or the K-th largest is it)
    }
    // an element's number grows with i and then with the lane: ties are met in order
    uint32_t found = 0, equal = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const uint64_t same = __ballot(key[i] == bound);
        const bool take = key[i] > bound || (key[i] == bound && equal + __builtin_popcountll(same & below_lane()) < ties);
        const uint64_t taken = __ballot(take);
        if (take) cand[found + __builtin_popcountll(taken & below_lane())] = (uint64_t)key[i] << 32 | (uint32_t)~(l + i * kWave);
        found += __builtin_popcountll(taken);
        equal += __builtin_popcountll(same);
    }
    wave_fence();
    write_ranked<kWave>(a, n, cand, found, r, l);
}

// ---------------------------------------------------------------------------
// rows of up to kWaveElems elements a lane, in vectors: a wavefront each
// ---------------------------------------------------------------------------
// Four pieces a lane give the bound; where few pieces hold the largest scores, so
// that too many reach it, it is found among the scores themselves.  Equal ones beyond
// the list's room are counted from the row's start.  The counting bounds it, not the
// memory (16,384 rows, K = 20: 1,000 bf16 25 us, by elements in the order of the
// lanes 43; 2,100 fp32 41, a workgroup a row 70; 4,000 bf16 47 against 73; K = 100
// of 4,000 fp32 100).
constexpr int kWaveElems = 64;  // a lane
constexpr uint32_t kLeastKey = 0x007fffffu;  // -infinity's

template <bool BF16>
__global__ __launch_bounds__(kTopThreads) void k_top_wave(TopArgs a) {
    using E = Elem<BF16>;
    using T = typename E::T;
    constexpr int kPer = E::kPer, kWaveVectors = kWaveElems / kPer;
    __shared__ uint64_t s_cand[kTopThreads / kWave][kShortCandidates];
    const uint32_t w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), l = lane_id();
    const uint32_t n = block_number() * (kTopThreads / kWave) + w;
    if (n >= (uint32_t)(a.shape.B * a.shape.T)) return;
    uint64_t* cand = s_cand[w];
    const int64_t at = a.shape.at(n);
    int32_t tok;
    if (!counts(a, at, l == 0, &tok)) return write_nothing<kWave>(a, n, at, l);
    const T* x = static_cast<const T*>(a.x.data) + a.x.at(n, a.shape);
    const uint32_t V = (uint32_t)a.V, nv = V / kPer, tail = V % kPer, K = (uint32_t)a.K;
    u32x4 v[kWaveVectors];
#pragma unroll
    for (int k = 0; k < kWaveVectors; ++k) {
        v[k] = no_vector<BF16>();
        if (k * kWave < nv && k * kWave + l < nv) v[k] = load16(x + (size_t)(k * kWave + l) * kPer);
    }
    const float xt = l < tail ? E::one(x[nv * kPer + l]) : kNone, xa = E::one(x[tok]);
    // four pieces of the row a lane, by their largest
    float top[4] = {xt, kNone, kNone, kNone}, most = kNone;
#pragma unroll
    for (int k = 0; k < kWaveVectors; ++k) {
        if (k * kWave < nv) {
            float f[kPer];
            E::unpack(v[k], f);
            const float mine = top_of(f, kNone);
            top[k % 4] = fmaxf(top[k % 4], mine);
            most = fmaxf(most, mine);
        }
    }
    TileStat ts;
    ts.add_tile<BF16, kWave>(v, most, a.c, nv);
    Stat st = ts.stat(a.c);
    {
        const float f[1] = {xt};
        accumulate(st, f, a.c);
    }
    st = join_lanes<kWave>(st, a.c);
    const RowValues r = row_values(st, xa, a.c, a.inv_t, a.inv_lo);
    if (l == 0) write_values(a, at, r.logp, r.lse, r.entropy);
    if (no_ranking(st)) return fill_row<kWave>(a, TopRow(a, n), l, 0, -1, __builtin_nanf(""));
    // f(k, j, score) for the lane's elements, j of vector k (and j = 0 of the tail, k = kWaveVectors); all lanes together
    auto each = [&](auto f) {
#pragma unroll
        for (int k = 0; k < kWaveVectors; ++k) {
            if (k * kWave < nv) {
                float e[kPer];
                E::unpack(again(v[k]), e);
#pragma unroll
                for (int j = 0; j < kPer; ++j) f(k, j, e[j]);
            }
        }
        f(kWaveVectors, 0, xt);
    };
    auto reach = [&](uint32_t least) {  // (padding is at -infinity, which all reach)
        const float score = key_score(least > kLeastKey ? least : kLeastKey);
        uint32_t some = 0;
        each([&](int, int, float e) { some += __builtin_popcountll(__ballot(e >= score)); });
        return some;
    };
    uint32_t key[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) key[i] = order_key(top[i]);
    const uint32_t hi = __builtin_amdgcn_readfirstlane(order_key(st.m));
    uint32_t bound = key_bound(key, K, K / 4), ties = ~0u;  // (all that reach the bound)
#pragma unroll 1
    for (int round = 0;; ++round) {
        if (round > 0) bound = bound_between(hi, kLeastKey, K, round == 1 ? K / 4 : 0, reach);
        // (ranking takes the square of their number)
        if (reach(bound) <= (round == 0 ? K + K / 2 + 32 : kShortCandidates)) break;
        if (round < 2) continue;
        if (bound < kLeastKey) bound = kLeastKey;
        ties = K - reach(bound + 1);  // (the K-th largest is it)
        break;
    }
    const float score = key_score(bound > kLeastKey ? bound : kLeastKey);
    auto place = [&](int k, int j) { return k < kWaveVectors ? (k * kWave + l) * kPer + j : nv * kPer + l; };
    uint32_t found = 0;
    auto take = [&](bool mine, uint32_t number, float e) {
        const uint64_t taken = __ballot(mine);
        if (mine) cand[found + __builtin_popcountll(taken & below_lane())] = choice_key(e, number);
        found += __builtin_popcountll(taken);
    };
    if (ties == ~0u) {
        each([&](int k, int j, float e) {
            const bool mine = e >= score && (k < kWaveVectors ? k * kWave + l < nv : l < tail);
            if (__ballot(mine) != 0) take(mine, place(k, j), e);
        });
    } else {
        // of the equal ones the first: by vector, then lane, then element
        uint32_t equal = 0;
#pragma unroll 1
        for (uint32_t k = 0; k * kWave < nv + kWave; ++k) {
            const bool last = k * kWave >= nv;  // the tail
            const uint32_t base = last ? nv * kPer + l : (k * kWave + l) * kPer, many = last ? 1 : kPer;
            const bool here = last ? l < tail : k * kWave + l < nv;
            float e[kPer];
            uint32_t same = 0;
            for (uint32_t j = 0; j < kPer; ++j) {
                e[j] = here && j < many ? E::one(x[base + j]) : kNone;
                same += here && j < many && e[j] == score;
            }
            uint32_t upto = same;
#pragma unroll
            for (int d = 1; d < kWave; d *= 2) {
                const uint32_t o = __shfl_up(upto, d, kWave);
                upto += l >= (uint32_t)d ? o : 0;
            }
            uint32_t before = equal + upto - same;
            for (uint32_t j = 0; j < kPer; ++j) {
                const bool valid = here && j < many, is = valid && e[j] == score;
                take(valid && (e[j] > score || (is && before < ties)), base + j, e[j]);
                before += is;
            }
            equal += __shfl(upto, kWave - 1, kWave);
        }
    }
    wave_fence();
    write_ranked<kWave>(a, n, cand, found, r, l);
}

// ---------------------------------------------------------------------------
// longer rows, or parts of them: a workgroup each
// ---------------------------------------------------------------------------
// HBM bounds it, and the exponentials nearly as much in bf16 (4,096 rows of 128,000
// bf16, K = 64: 195 us, 5.4 TB/s, where a reduction that only reads reaches 6.0; in the
// caches' order 202, by the sums of softmax_dev.h 219).  Few rows are bound by latency: 64 rows of
// 128,000 bf16 in parts, K = 20: 14 us, of which the loads take 3, the part's
// selection 3 and the join's 4.  Five or six workgroups a compute unit (80
// registers) cover each other's loads; eight cost spills, workgroups of 512 lanes
// have their selections at the same time (masked rows: 98 against 115).
struct TopShared {
    uint64_t cand[kMostCandidates];
    uint32_t list[kMostGroups];
    uint32_t top[kTopThreads];
    Stat stat[kTopThreads / kWave];
    uint32_t sum[2][kTopThreads / kWave];
    uint32_t groups, found;
    bool last;
};

// sum over the workgroup, in every thread; `turn` alternates from call to call
__device__ __forceinline__ uint32_t block_count(TopShared& s, uint32_t mine, int turn) {
    mine = lanes_sum<kWave>(mine);
    if (lane_id() == 0) s.sum[turn][threadIdx.x / kWave] = mine;
    __syncthreads();
    uint32_t r = 0;
#pragma unroll
    for (int i = 0; i < kTopThreads / kWave; ++i) r += s.sum[turn][i];
    return r;
}

// The K-th largest of all keys, which `each(f)` gives f one after the other, is
// found bit by bit, and those that reach it become the candidates: K of them, or
// all if there are fewer.  Every thread takes part.
template <typename Each>
__device__ __forceinline__ uint32_t exact_candidates(TopShared& s, int32_t K, Each each) {
    uint64_t t = 0;
    for (int bit = 63; bit >= 0; --bit) {
        const uint64_t trial = t | 1ull << bit;
        uint32_t mine = 0;
        each([&](uint64_t key) { mine += key >= trial; });
        if (block_count(s, mine, bit & 1) >= (uint32_t)K) t = trial;
    }
    if (threadIdx.x == 0) s.found = 0;
    __syncthreads();
    each([&](uint64_t key) {
        if (key != 0 && key >= t) s.cand[atomicAdd(&s.found, 1u)] = key;
    });
    __syncthreads();
    return s.found;
}

// The statistics joined over the workgroup, and the bound that K of the lanes' largest
// keys reach, in every thread; the lists are empty.
__device__ __forceinline__ Stat block_stat(TopShared& s, Stat st, uint32_t key, float c, int32_t K, uint32_t* bound) {
    const uint32_t tid = threadIdx.x, lane = lane_id();
    s.top[tid] = key;
    if (tid == 0) s.groups = s.found = 0;
    st = join_lanes<kWave>(st, c);
    if (lane == 0) s.stat[tid / kWave] = st;
    __syncthreads();
    uint32_t top[kTopThreads / kWave];
#pragma unroll
    for (int i = 0; i < kTopThreads / kWave; ++i) top[i] = s.top[i * kWave + lane];
    *bound = key_bound(top, (uint32_t)K, (uint32_t)K / 4);
    return join_lanes<kTopThreads / kWave>(s.stat[lane % (kTopThreads / kWave)], c);
}

// Joins a row's parts: their statistics, and the K largest of their K keys each.
// By a whole workgroup.
__device__ void join_top(const TopArgs& a, uint32_t n, int64_t at, float xa, TopShared& s) {
    const uint32_t tid = threadIdx.x;
    // the best of every part come first, then the second best, ...: the lanes' largest are spread over the first ranks
    const uint64_t* keys = a.key + (int64_t)n * a.parts * a.K;
    const uint32_t total = (uint32_t)a.parts * (uint32_t)a.K;
    auto each = [&](auto f) {
        for (uint32_t e = tid; e < total; e += kTopThreads) {
            const uint32_t r = div31(e, a.by_parts), p = e - r * (uint32_t)a.parts;
            f(__hip_atomic_load(keys + (int64_t)p * a.K + r, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
        }
    };
    uint32_t mine = 0;
    uint64_t first = 0;
    each([&](uint64_t key) {
        const uint32_t k = (uint32_t)(key >> 32);
        mine = k > mine ? k : mine;
        first = key;
    });
    Stat st = no_stat();
    for (int32_t p = tid; p < a.parts; p += kTopThreads) {
        const float* q = a.part + 3 * ((int64_t)n * a.parts + p);
        Stat o;
        o.m = __hip_atomic_load(q, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        o.s = __hip_atomic_load(q + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        o.u = __hip_atomic_load(q + 2, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        st = join(st, o, a.c);
    }
    uint32_t bound = 0, found = total;
    if (total <= kTopThreads) {  // all are candidates
        st = join_lanes<kWave>(st, a.c);
        if (lane_id() == 0) s.stat[tid / kWave] = st;
        s.cand[tid] = first;
        __syncthreads();
        st = join_lanes<kTopThreads / kWave>(s.stat[lane_id() % (kTopThreads / kWave)], a.c);
    } else {
        st = block_stat(s, st, mine, a.c, a.K, &bound);
    }
    const RowValues r = row_values(st, xa, a.c, a.inv_t, a.inv_lo);
    if (tid == 0) write_values(a, at, r.logp, r.lse, r.entropy);
    if (no_ranking(st)) return fill_row<kTopThreads>(a, TopRow(a, n), tid, 0, -1, __builtin_nanf(""));
    if (total > kTopThreads) {
        each([&](uint64_t key) {
            if (key == 0 || (uint32_t)(key >> 32) < bound) return;
            const uint32_t k = atomicAdd(&s.found, 1u);
            if (k < kMostCandidates) s.cand[k] = key;
        });
        __syncthreads();
        found = s.found;
        if (found > kMostCandidates) found = exact_candidates(s, a.K, each);
    }
    write_ranked<kTopThreads>(a, n, s.cand, found, r, tid);
}

template <bool BF16, bool ONCE>
__global__ __launch_bounds__(kTopThreads, 6) void k_top_rows(TopArgs a) {
    using E = Elem<BF16>;
    using T = typename E::T;
    constexpr int kPer = E::kPer;
    extern __shared__ float s_group[];  // the groups' maxima
    __shared__ TopShared s;
    const uint32_t item = block_number(), tid = threadIdx.x;
    if (item >= (uint32_t)(a.shape.B * a.shape.T) * (uint32_t)a.parts) return;
    const uint32_t n = div31(item, a.by_parts), part = item - n * (uint32_t)a.parts;
    const int64_t at = a.shape.at(n);
    int32_t tok;
    if (!counts(a, at, part == 0 && tid == 0, &tok)) {
        if (part == 0) write_nothing<kTopThreads>(a, n, at, tid);
        return;
    }
    const T* x = static_cast<const T*>(a.x.data) + a.x.at(n, a.shape);
    const RowVectors<BF16, 4> row(x, (uint32_t)a.V);
    const T* vx = x + row.head;  // the vectors
    const uint32_t nv = row.count;
    const uint32_t lo = part * (uint32_t)a.per < nv ? part * (uint32_t)a.per : nv, hi = lo + a.per < nv ? lo + a.per : nv;
    const uint32_t groups = (hi - lo + kGroup - 1) / kGroup;
    const bool last_one = part == 0 && tid < row.beside();  // the elements beside the vectors
    const float xt = last_one ? E::one(x[row.beside_at(tid)]) : kNone;
    const float xa = E::one(x[tok]);
    TileStat ts;
    for (uint32_t base = lo; base < hi; base += kTopThreads * kTopVectors) {
        u32x4 v[kTopVectors];
#pragma unroll
        for (int k = 0; k < kTopVectors; ++k) {
            const uint32_t i = base + k * kTopThreads + tid;
            v[k] = i < hi ? read16<ONCE>(vx + (size_t)i * kPer) : no_vector<BF16>();
        }
        float top = kNone;
#pragma unroll
        for (int k = 0; k < kTopVectors; ++k) {
            const uint32_t i = base + k * kTopThreads + tid;
            float f[kPer];
            if (base + k * kTopThreads >= hi) continue;
            E::unpack(v[k], f);
            const float mine = top_of(f, kNone);
            top = fmaxf(top, mine);
            const float group = lanes_reduce<kGroup>(mine, [](float p, float q) { return fmaxf(p, q); });
            if (tid % kGroup == 0 && i < hi) s_group[(i - lo) / kGroup] = group;
        }
        ts.add_tile<BF16, kTopThreads>(v, top, a.c, hi - base);
    }
    Stat st = ts.stat(a.c);
    {
        const float f[1] = {xt};
        accumulate(st, f, a.c);
    }
    uint32_t bound;
    st = block_stat(s, st, order_key(st.m), a.c, a.K, &bound);
    const RowValues r = row_values(st, xa, a.c, a.inv_t, a.inv_lo);
    uint32_t found = 0;
    if (!no_ranking(st)) {
        for (uint32_t g = tid; g < groups; g += kTopThreads) {
            if (order_key(s_group[g]) < bound) continue;
            const uint32_t k = atomicAdd(&s.groups, 1u);
            if (k < kMostGroups) s.list[k] = g;
        }
        __syncthreads();
        uint32_t listed = s.groups;
        auto each = [&](auto f) {
            for (uint32_t q = tid / kGroup; q < listed; q += kTopThreads / kGroup) {
                const uint32_t i = lo + s.list[q] * kGroup + tid % kGroup;
                if (i >= hi) continue;
                float e[kPer];
                E::unpack(load16(vx + (size_t)i * kPer), e);
#pragma unroll
                for (int j = 0; j < kPer; ++j) f(choice_key(e[j], row.head + i * kPer + j));
            }
            if (last_one) f(choice_key(xt, row.beside_at(tid)));
        };
        if (listed <= kMostGroups) {
            each([&](uint64_t key) {
                if ((uint32_t)(key >> 32) < bound) return;
                const uint32_t k = atomicAdd(&s.found, 1u);
                if (k < kMostCandidates) s.cand[k] = key;
            });
            __syncthreads();
            found = s.found;
        }
        if (listed > kMostGroups || found > kMostCandidates) {
            uint32_t t = 0;  // the K-th largest maximum (0: fewer groups)
            for (int bit = 31; bit >= 0; --bit) {
                const uint32_t trial = t | 1u << bit;
                uint32_t k = 0;
                for (uint32_t g = tid; g < groups; g += kTopThreads) k += order_key(s_group[g]) >= trial;
                if (block_count(s, k, bit & 1) >= (uint32_t)a.K) t = trial;
            }
            __syncthreads();
            if (tid < kWave) {
                uint32_t k = 0, equal = 0;
                for (uint32_t base = 0; base < groups; base += kWave) {
                    const uint32_t g = base + tid, key = g < groups ? order_key(s_group[g]) : 0;
                    const uint64_t same = __ballot(g < groups && key == t);
                    const bool take = g < groups && (key > t || (key == t && equal + __builtin_popcountll(same & below_lane()) < (uint32_t)a.K));
                    const uint64_t taken = __ballot(take);
                    if (take) s.list[k + __builtin_popcountll(taken & below_lane())] = g;
                    k += __builtin_popcountll(taken);
                    equal += __builtin_popcountll(same);
                }
                if (tid == 0) s.groups = k;
            }
            __syncthreads();
            listed = s.groups;
            found = exact_candidates(s, a.K, each);
        }
    }
    if (a.parts == 1) {
        if (tid == 0) write_values(a, at, r.logp, r.lse, r.entropy);
        if (no_ranking(st)) return fill_row<kTopThreads>(a, TopRow(a, n), tid, 0, -1, __builtin_nanf(""));
        return write_ranked<kTopThreads>(a, n, s.cand, found, r, tid);
    }
    // a part: its K keys in order (0: there are fewer) and its statistics, for the join
    uint64_t* key = a.key + (int64_t)item * a.K;
    rank<kTopThreads>(s.cand, found, a.K, tid, [&](uint32_t k, uint64_t v) {
        __hip_atomic_store(key + k, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    });
    for (uint32_t k = found + tid; k < (uint32_t)a.K; k += kTopThreads) __hip_atomic_store(key + k, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (tid == 0) {
        float* mine = a.part + 3 * (int64_t)item;
        __hip_atomic_store(mine, st.m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(mine + 1, st.s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(mine + 2, st.u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (!a.row_ticket) return;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // every wavefront's stores are acknowledged before the ticket is drawn
    __syncthreads();
    if (tid == 0) s.last = draw_last(a.row_ticket + n * kTicketStep, (uint32_t)a.parts);
    __syncthreads();
    if (s.last) join_top(a, n, at, xa, s);
}

// the join of many split rows, by a launch of its own
template <bool BF16>
__global__ __launch_bounds__(kTopThreads) void k_top_join(TopArgs a) {
    __shared__ TopShared s;
    const uint32_t n = block_number();
    if (n >= (uint32_t)(a.shape.B * a.shape.T)) return;
    const int64_t at = a.shape.at(n);
    int32_t tok;
    if (!counts(a, at, false, &tok)) return;
    using E = Elem<BF16>;
    join_top(a, n, at, E::one((static_cast<const typename E::T*>(a.x.data) + a.x.at(n, a.shape))[tok]), s);
}

template <bool BF16>
hipError_t alternatives(const TopArgs& a, hipStream_t s) {
    const int64_t rows = a.shape.B * a.shape.T;
    constexpr int kRows = kTopThreads / kWave;
    auto few = [&](auto lanes) {
        constexpr int LANES = decltype(lanes)::value, kFewRows = kTopThreads / LANES;
        hipLaunchKernelGGL((k_top_few<BF16, LANES>), grid_of((rows + kFewRows - 1) / kFewRows, kTopThreads), dim3(kTopThreads), 0, s, a);
        return hipGetLastError();
    };
    if (a.V <= 4 * kFewElems) return few(std::integral_constant<int, 4>{});
    if (a.V <= 8 * kFewElems) return few(std::integral_constant<int, 8>{});
    if (a.V <= 16 * kFewElems) return few(std::integral_constant<int, 16>{});
    const dim3 each = grid_of((rows + kRows - 1) / kRows, kTopThreads);
    if (a.V <= kShortRow) {
        hipLaunchKernelGGL((k_top_short<BF16>), each, dim3(kTopThreads), 0, s, a);
        return hipGetLastError();
    }
    if (a.V / Elem<BF16>::kPer * Elem<BF16>::kPer <= kWaveElems * kWave) {
        hipLaunchKernelGGL((k_top_wave<BF16>), each, dim3(kTopThreads), 0, s, a);
        return hipGetLastError();
    }
    const int64_t items = rows * a.parts;  // fewer than 2^31 (the caller's check)
    auto go = [&](auto once) {
        hipLaunchKernelGGL((k_top_rows<BF16, decltype(once)::value>), grid_of(items, kTopThreads), dim3(kTopThreads),
                           sizeof(float) * (a.per / kGroup), s, a);
    };
    if (a.once) go(std::true_type{});
    else go(std::false_type{});
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.parts == 1 || a.row_ticket) return e;
    hipLaunchKernelGGL((k_top_join<BF16>), grid_of(rows, kTopThreads), dim3(kTopThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace

// Parts of a row: as in k_logits.hip, or where a row is wider than the groups'
// maxima of one workgroup; whole groups each.
RowParts top_parts(int64_t rows, int64_t V, bool bf16) {
    const int64_t cus = device_cus(), nv = V / (bf16 ? 8 : 4);
    if (V <= kShortRow || rows <= 0) return RowParts{1, (int32_t)nv};
    int64_t parts = (nv + kPartVectors - 1) / kPartVectors;
    if (rows < cus) {
        const int64_t want = (2 * cus + rows - 1) / rows, most = nv / (4 * kTopThreads);
        const int64_t split = want < most ? want : most;
        if (split > parts) parts = split;
    }
    const int64_t per = ((nv + parts - 1) / parts + kGroup - 1) / kGroup * kGroup;
    return RowParts{(int32_t)((nv + per - 1) / per), (int32_t)per};
}

hipError_t launch_token_alternatives(const TopArgs& a, bool bf16, hipStream_t s) {
    return bf16 ? alternatives<true>(a, s) : alternatives<false>(a, s);
}

}  // namespace conduit
