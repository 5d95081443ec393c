// Log-probabilities of the taken tokens from the last hidden states X and the
// output projection W, and the gradients of both, without the [tokens, V] logits
// ever being in memory whole (conduit_head_logprobs, _backward).
//
// Forward: logits z = X W^T / temperature are produced 256 x 256 at a time on
// the matrix cores (gemm_dev.h); each tile leaves every token's maximum, sum and
// weighted sum over its 256 choices (as in k_logits.hip) and, where the taken
// token is among them, its score.  A second launch joins a token's tiles.  The
// tile holds choices as rows and tokens as columns of the product, so that a
// lane has 32 choices of one token and most of the reduction is its own.
//
// Backward: the tiles are produced again, turned into the logits' gradient
//     d = (g ([j = token] - p_j) - h p_j (log p_j + entropy)) / temperature
// and rounded once to bf16, the type of W and X: over many tokens its error, of
// random sign from element to element, is no more than that of the gradients' own
// rounding.  Up to kHeadTwo tokens, whose few large elements would not average
// out, what the rounding left is kept too, as another bf16 row of d beside a
// second copy of the token's hidden states: 16 bits of each element.  (10 tokens,
// 7,925 choices, 1,088 units: error 0.0027 of the gradients with one row, 0.0017
// with two, the outputs' own rounding; 16 bits cost 8 us of 81.  128,000 choices, 4,096 units:
// 16 tokens 693 us and 745, 128 tokens 865 and 1,003; beyond, 0.0024 with one.)
// Then
//     dX = d W  (split along the choices, parts joined in a fixed order),
//     dW = d^T X
// by the same product, which turns W, X and d as it reads them.  Batches whose d would pass
// kHeadChunkBytes run in chunks of choices; dX accumulates over them in fp32.
//
// The matrix cores bound both, at the clock that the card's power leaves them: 8,192
// tokens (masked), 128,000 choices, 4,096 units in 2.55 ms, 1,220 TFLOP/s of the live
// tokens' products; a bare library product of such sizes reaches 1,410-1,530.  The
// three products of the gradients (4,096 tokens, 2,048 units): 2.37 ms, 1,150 TFLOP/s.
//
// Tokens that the mask leaves out take no part: a first launch lists the others
// in order, and the hidden rows are packed by that list.  Their number stays on
// the device: grids are sized for all tokens, workgroups beyond return at once.
#include <type_traits>

#include "gemm_dev.h"
#include "head_dev.h"

namespace conduit {

namespace {

constexpr int kListThreads = 1024;
constexpr int kHeadXcds = 8;
constexpr int kHeadGroup = 8;  // column tiles that neighbours in a launch share

__device__ __forceinline__ int64_t live_tokens(const HeadArgs& a) { return a.count ? (int64_t)*a.count : a.N; }

// rows of the logits' gradient, for n live tokens
__device__ __forceinline__ bool two_halves(const HeadArgs& a) { return a.d_rows > a.N; }
__device__ __forceinline__ int64_t gradient_rows(const HeadArgs& a, int64_t n) { return two_halves(a) ? 2 * n : n; }

// The tokens that count, in order: list[k] = token, place[token] = k or -1, and
// their number.  One workgroup; a lane takes 16 tokens a round.
__global__ __launch_bounds__(kListThreads) void k_head_list(HeadArgs a) {
    __shared__ uint32_t s_wave[kListThreads / kWave + 1];
    constexpr int kPer = 16;
    uint32_t done = 0;
    for (int64_t base = 0; base < a.N; base += kListThreads * kPer) {
        const int64_t n0 = base + (int64_t)threadIdx.x * kPer;
        uint32_t on = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int64_t n = n0 + i;
            if (n >= a.N) break;
            const int64_t at = a.shape.at((uint32_t)n);
            if (!a.mask[at]) continue;
            const int32_t tok = a.tokens[at];
            if (tok >= 0 && tok < a.V) on |= 1u << i;
            else flag_error(a.err, ERR_TOKEN);
        }
        const uint32_t mine = __builtin_popcount(on);
        uint32_t incl = mine;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const uint32_t up = __shfl_up(incl, d, kWave);
            if (lane_id() >= d) incl += up;
        }
        if (lane_id() == kWave - 1) s_wave[threadIdx.x / kWave] = incl;
        __syncthreads();
        if (threadIdx.x == 0) {
            uint32_t sum = 0;
            for (int w = 0; w < kListThreads / kWave; ++w) {
                const uint32_t c = s_wave[w];
                s_wave[w] = sum;
                sum += c;
            }
            s_wave[kListThreads / kWave] = sum;
        }
        __syncthreads();
        uint32_t k = done + s_wave[threadIdx.x / kWave] + incl - mine;
        done += s_wave[kListThreads / kWave];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (n0 + i >= a.N) break;
            const bool counts = on >> i & 1;
            a.place[n0 + i] = counts ? (int32_t)k : -1;
            if (counts) a.list[k++] = (int32_t)(n0 + i);
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) *a.count_out = done;
}

// dst[k][0..ld) = src row of the k-th token, zeros beyond `width`; with `rows`
// given, plain rows (the projection's) instead of tokens.  The tokens' rows twice
// where d has two halves.
__global__ __launch_bounds__(256) void k_head_pack(HeadArgs a, const uint16_t* src, int64_t src_ld, int64_t width, uint16_t* dst,
                                                   int64_t ld, int64_t rows, bool tokens) {
    const int64_t n = tokens ? live_tokens(a) : rows, n_rows = tokens ? gradient_rows(a, n) : n;
    for (int64_t k = blockIdx.x; k < n_rows; k += gridDim.x) {
        const int64_t r = k < n ? k : k - n;
        const uint16_t* x = src + (tokens ? a.x.at((uint32_t)(a.list ? a.list[r] : r), a.shape) : r * src_ld);
        uint16_t* y = dst + k * ld;
        for (int64_t c = 8 * (int64_t)threadIdx.x; c < ld; c += 8 * 256) {
            u32x4_t v = {0, 0, 0, 0};
            if (c + 8 <= width) {
                __builtin_memcpy(&v, x + c, 16);
            } else {
                uint16_t e[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) e[i] = c + i < width ? x[c + i] : (uint16_t)0;
                __builtin_memcpy(&v, e, 16);
            }
            *reinterpret_cast<u32x4_t*>(y + c) = v;
        }
    }
}

// ---------------------------------------------------------------------------
// which tile of C a workgroup takes
// ---------------------------------------------------------------------------
// A launch has a workgroup for every compute unit (LDS holds one), and workgroup
// b, on die b % 8 (of 8, with an L2 each), takes the places b, b + gridDim, ...
// A die has an eighth of the row tiles, and walks them kHeadGroup column tiles at
// a time, so that the 32 workgroups it runs at once share 4 row tiles and 8
// column tiles.
struct TileWalk {
    int32_t row_tiles, col_tiles, lo, n, place, end;
    int32_t row, col;

    __device__ __forceinline__ TileWalk(int64_t rows, int64_t cols)
        : row_tiles((int32_t)rows), col_tiles((int32_t)cols), row(0), col(0) {
        const int32_t x = blockIdx.x % kHeadXcds;
        lo = (int32_t)(rows * x / kHeadXcds);
        n = (int32_t)(rows * (x + 1) / kHeadXcds) - lo;
        place = blockIdx.x / kHeadXcds;
        end = n * col_tiles;
    }
    // the next tile of this workgroup into row, col; false: there is none
    __device__ __forceinline__ bool next() {
        if (place >= end) return false;
        const int32_t g = place / (n * kHeadGroup), r = place - g * n * kHeadGroup, c0 = g * kHeadGroup;
        const int32_t width = col_tiles - c0 < kHeadGroup ? col_tiles - c0 : kHeadGroup;
        row = lo + r / width;
        col = c0 + r % width;
        place += gridDim.x / kHeadXcds;
        return true;
    }
};

// workgroups: one a compute unit (and no more than places), a multiple of the dies
unsigned tile_grid(int64_t row_tiles, int64_t col_tiles, int32_t cus) {
    const int64_t places = (row_tiles + kHeadXcds - 1) / kHeadXcds * col_tiles, each = cus / kHeadXcds > 0 ? cus / kHeadXcds : 1;
    return (unsigned)(kHeadXcds * (places < each ? places : each));
}

__device__ __forceinline__ int64_t tiles(int64_t n) { return (n + kGemmTile - 1) / kGemmTile; }

// joined over the four lanes 16 apart
template <int STEP>
__device__ __forceinline__ Stat join_step(const Stat& s, float c) {
    const Sides<float> m = sides<STEP>(s.m), t = sides<STEP>(s.s), u = sides<STEP>(s.u);
    return join(Stat{m.a, t.a, u.a}, Stat{m.b, t.b, u.b}, c);
}
__device__ __forceinline__ Stat join_quarters(const Stat& s, float c) { return join_step<5>(join_step<4>(s, c), c); }

// ---------------------------------------------------------------------------
// forward: the statistics of a tile
// ---------------------------------------------------------------------------
// The statistics of ROWS x 16 choices of one token in four lanes 16 apart: lane
// group q holds choices 16 i + 4 q + j as x[i][j].  `first` is the first choice
// of this lane's; the taken token's score is left in `taken` where it is here.
template <int ROWS>
__device__ __forceinline__ Stat score_stat(f32x4_t (&x)[ROWS], int64_t first, int64_t V, int32_t tok, float c, float* taken) {
    if (V - first < 16 * ROWS) {  // the last tile: choices beyond have no weight
        const int32_t end = (int32_t)(V - first);
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[i][j] = i * 16 + j < end ? x[i][j] : kNone;
        }
    }
    const int64_t from = (int64_t)tok - first;
    if (from >= 0 && from < 16 * ROWS) {  // in few tiles
        const int32_t at = (int32_t)from;
        float xt = 0.0f;
        bool here = false;
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                xt = i * 16 + j == at ? x[i][j] : xt;
                here |= i * 16 + j == at;
            }
        }
        if (here) *taken = xt;
    }
    float top = kNone;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) top = fmaxf(top, x[i][j]);
    }
    Stat st = no_stat();
    raise(st, top, c);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const float v[4] = {x[i][0], x[i][1], x[i][2], x[i][3]};
        add(st, v, c);
    }
    return join_quarters(st, c);
}

__global__ __launch_bounds__(kGemmThreads) void k_head_stats(HeadArgs a) {
    __shared__ __align__(1024) uint8_t lds[kGemmLds];
    __shared__ Stat stat[2][kGemmTile];
    const int64_t n = live_tokens(a);
    const int lane = lane_id(), w = threadIdx.x / kWave, wm = w / 4, wn = w % 4, q = lane / 16, col = lane % 16;
    const int32_t steps = (int32_t)((a.K + kGemmK - 1) / kGemmK);
    TileWalk walk(tiles(a.V), tiles(n));
    GemmTiles<false, false> gemm;
    gemm.lds = lds;
    bool more = walk.next();
    if (more) gemm.start(a.W, (int64_t)walk.row * kGemmTile, a.V, a.X, (int64_t)walk.col * kGemmTile, n, a.K, 0, steps);
    while (more) {
        const int64_t row = walk.row, v0 = row * kGemmTile, n0 = (int64_t)walk.col * kGemmTile;
        int32_t tok[4];  // ahead of the product, which hides the loads
#pragma unroll
        for (int ni = 0; ni < 4; ++ni) {
            const int64_t k = n0 + wn * 64 + ni * 16 + col;
            tok[ni] = k < n ? a.tokens[a.shape.at((uint32_t)(a.list ? a.list[k] : k))] : -1;
        }
        GemmAcc acc;
        gemm.run(acc);
#pragma unroll
        for (int ni = 0; ni < 4; ++ni) asm volatile("" : "+v"(tok[ni]));  // waited for before the next copies start
        more = walk.next();
        if (more) gemm.start(a.W, (int64_t)walk.row * kGemmTile, a.V, a.X, (int64_t)walk.col * kGemmTile, n, a.K, 0, steps);
#pragma unroll
        for (int ni = 0; ni < 4; ++ni) {
            const int64_t k = n0 + wn * 64 + ni * 16 + col;
            f32x4_t x[8];
#pragma unroll
            for (int mi = 0; mi < 8; ++mi) x[mi] = acc.c[mi][ni];
            const Stat st = score_stat<8>(x, v0 + wm * 128 + 4 * q, a.V, tok[ni], a.c, a.taken + k);
            if (q == 0) stat[wm][wn * 64 + ni * 16 + col] = st;
        }
        lds_barrier();
        if (threadIdx.x < kGemmTile && n0 + threadIdx.x < n) {
            const Stat st = join(stat[0][threadIdx.x], stat[1][threadIdx.x], a.c);
            float* p = a.part + (row * a.N + n0 + threadIdx.x) * 3;
            p[0] = st.m;
            p[1] = st.s;
            p[2] = st.u;
        }
        // (run() meets barriers before stat is written again)
    }
}

// The same for at most 16 tokens, which W's bytes bound: a wavefront takes 64
// choices and reads its rows of W straight into registers, a set of kFewSteps x
// 32 hidden units ahead of the one it multiplies, without LDS or barriers.  The
// hidden states come out of the caches, a quarter as many bytes again: with 32
// tokens they would be half, and the tiles of 256 are as fast (16 tokens of 2,048
// units, 128,000 choices: 119 us, 4.4 TB/s, against 150; 32 tokens 147 against 138).
constexpr int kFewThreads = 256;
constexpr int kFewTokens = 16;
constexpr int kFewSteps = 4;
constexpr int kFewHidden = 2048;

// acc[i][j]: the product of row 16 i + 4 q + j from w on (of `rows` that exist) and token lane % 16
__device__ __forceinline__ void few_scores(const HeadArgs& a, const uint16_t* w, int64_t rows, int64_t n, f32x4_t (&acc)[4]) {
    const int lane = lane_id(), q = lane / 16, col = lane % 16;
    __amdgpu_buffer_rsrc_t rw =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(w), 0, 0x7fffffff, 0x00027000);
    __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(a.X.p), 0, 0x7fffffff, 0x00027000);
    uint32_t vw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) vw[i] = i * 16 + col < rows ? (uint32_t)((i * 16 + col) * a.W.ld * 2 + q * 16) : kGemmOut;
    const uint32_t vx = col < n ? (uint32_t)(col * a.X.ld * 2 + q * 16) : kGemmOut;
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = f32x4_t{0, 0, 0, 0};
    u32x4_t fw[2][kFewSteps][4], fx[2][kFewSteps];
    const int32_t sets = (int32_t)((a.K + 32 * kFewSteps - 1) / (32 * kFewSteps));
    auto load = [&](int32_t set, u32x4_t (&x)[kFewSteps][4], u32x4_t (&y)[kFewSteps]) {
#pragma unroll
        for (int t = 0; t < kFewSteps; ++t) {
            const int32_t k0 = (set * kFewSteps + t) * 32;
            const bool in = k0 + q * 8 < a.K;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                x[t][i] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rw, in ? vw[i] : kGemmOut, k0 * 2, 0));
            y[t] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rx, in ? vx : kGemmOut, k0 * 2, 0));
        }
    };
    auto multiply = [&](const u32x4_t (&x)[kFewSteps][4], const u32x4_t (&y)[kFewSteps]) {
#pragma unroll
        for (int t = 0; t < kFewSteps; ++t) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x[t][i]), __builtin_bit_cast(bf16x8, y[t]),
                                                                 acc[i], 0, 0, 0);
        }
    };
    load(0, fw[0], fx[0]);
    for (int32_t set = 0; set < sets; set += 2) {
        load(set + 1, fw[1], fx[1]);  // (beyond the last: zeros)
        multiply(fw[0], fx[0]);
        load(set + 2, fw[0], fx[0]);
        multiply(fw[1], fx[1]);
    }
}

__global__ __launch_bounds__(kFewThreads) void k_head_stats_few(HeadArgs a) {
    __shared__ Stat stat[kFewThreads / kWave][kFewTokens];
    const int64_t n = live_tokens(a);
    if (n == 0) return;
    const int lane = lane_id(), w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), q = lane / 16, col = lane % 16;
    const int64_t v0 = (int64_t)blockIdx.x * kGemmTile + w * 64;
    const int32_t tok = col < n ? a.tokens[a.shape.at((uint32_t)(a.list ? a.list[col] : col))] : -1;
    f32x4_t acc[4];
    few_scores(a, a.W.p + v0 * a.W.ld, a.V - v0, n, acc);
    const Stat mine = score_stat<4>(acc, v0 + 4 * q, a.V, tok, a.c, a.taken + col);
    if (q == 0) stat[w][col] = mine;
    __syncthreads();
    if (threadIdx.x < kFewTokens && threadIdx.x < n) {
        Stat st = stat[0][threadIdx.x];
#pragma unroll
        for (int i = 1; i < kFewThreads / kWave; ++i) st = join(st, stat[i][threadIdx.x], a.c);
        float* p = a.part + ((int64_t)blockIdx.x * a.N + threadIdx.x) * 3;
        p[0] = st.m;
        p[1] = st.s;
        p[2] = st.u;
    }
}

// a token's tiles joined, by LANES lanes (16, or a workgroup)
template <int LANES>
__global__ __launch_bounds__(256) void k_head_join(HeadArgs a) {
    __shared__ Stat lds[256 / kWave];
    const int64_t t = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    const int l = threadIdx.x % LANES;
    if (t >= a.N) return;
    const int64_t at = a.shape.at((uint32_t)t);
    int64_t k = t;
    bool ok = true;
    if (a.place) {
        k = a.place[t];
        ok = k >= 0;
    } else {
        const int32_t tok = a.tokens[at];
        ok = tok >= 0 && tok < a.V;
        if (!ok && l == 0) flag_error(a.err, ERR_TOKEN);
    }
    if (!ok) {
        if (l == 0) {
            if (a.logp) a.logp[at] = 0.0f;
            if (a.lse) a.lse[at] = 0.0f;
            if (a.entropy) a.entropy[at] = 0.0f;
        }
        return;
    }
    Stat st = no_stat();
    const int32_t n_tiles = (int32_t)tiles(a.V);
#pragma unroll 4
    for (int32_t r = l; r < n_tiles; r += LANES) {
        const float* p = a.part + ((int64_t)r * a.N + k) * 3;
        st = join(st, Stat{p[0], p[1], p[2]}, a.c);
    }
    if constexpr (LANES == 16) {
        st = join_lanes<16>(st, a.c);
    } else {
        st = join_lanes<kWave>(st, a.c);
        if (lane_id() == 0) lds[threadIdx.x / kWave] = st;
        __syncthreads();
        st = join_lanes<256 / kWave>(lds[lane_id() % (256 / kWave)], a.c);
    }
    const RowValues r = row_values(st, a.taken[k], a.c, a.inv_t, 0.0f);
    if (l == 0) {
        if (a.logp) a.logp[at] = r.logp;
        if (a.lse) a.lse[at] = r.lse;
        if (a.entropy) a.entropy[at] = r.entropy;
    }
}

// ---------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------
// one logit's gradient from its product x; l2 = log2(e) lse, g and h over the temperature
__device__ __forceinline__ float score_gradient(const HeadArgs& a, float x, float l2, float g, float h, float entropy) {
    const float d = fmaf(x, a.c, -l2), p = exp2_fast(d);  // log2 p, p
    return -p * (a.h ? fmaf(h, fmaf(fmaxf(d, kFloor), kLn2, entropy), g) : g);
}

// the taken token's own: g (1 - p) without the cancellation of a probability near 1
__device__ __forceinline__ float taken_gradient(const HeadArgs& a, float x, float lse, float g, float h, float entropy) {
    const float lp = fmaf(x, a.inv_t, -lse);
    const float d = -g * expm1_fast(lp);
    return a.h ? d - h * exp2_fast(lp * kLog2e) * (fmaxf(lp, kFloor) + entropy) : d;
}

// what the rounding to bf16 leaves (infinities and NaN stand in the first half)
__device__ __forceinline__ float second_half(float x) {
    const float rest = x - (float)(__bf16)x;
    return fabsf(rest) < 1e38f ? rest : 0.0f;
}

// the logits' gradient of a tile of choices [v_base, v_base + v_count) of W, into
// d [token][choice - v_base]
__global__ __launch_bounds__(kGemmThreads) void k_head_gradient(HeadArgs a, int64_t v_base, int64_t v_count) {
    __shared__ __align__(1024) uint8_t lds[kGemmLds];
    const int64_t n = live_tokens(a);
    const int lane = lane_id(), w = threadIdx.x / kWave, wm = w / 4, wn = w % 4, q = lane / 16, col = lane % 16;
    const int32_t steps = (int32_t)((a.K + kGemmK - 1) / kGemmK);
    const bool two = two_halves(a);
    const GemmOperand W{a.W.p + v_base * a.W.ld, a.W.ld};
    TileWalk walk(tiles(v_count), tiles(n));
    GemmTiles<false, false> gemm;
    gemm.lds = lds;
    bool more = walk.next();
    if (more) gemm.start(W, (int64_t)walk.row * kGemmTile, v_count, a.X, (int64_t)walk.col * kGemmTile, n, a.K, 0, steps);
    while (more) {
        const int64_t v0 = (int64_t)walk.row * kGemmTile, n0 = (int64_t)walk.col * kGemmTile;
        int32_t tok[4];
        float g[4], h[4], lse[4], entropy[4];  // g and h over the temperature
#pragma unroll
        for (int ni = 0; ni < 4; ++ni) {
            const int64_t k = n0 + wn * 64 + ni * 16 + col;
            tok[ni] = -1;
            g[ni] = h[ni] = lse[ni] = entropy[ni] = 0.0f;
            if (k < n) {
                const int64_t at = a.shape.at((uint32_t)(a.list ? a.list[k] : k));
                const int32_t t = a.tokens[at];
                const bool ok = t >= 0 && t < a.V;  // (without a mask there is no list that leaves others out)
                if (!ok && v_base == 0 && walk.row == 0 && wm == 0 && q == 0) flag_error(a.err, ERR_TOKEN);
                tok[ni] = t;
                lse[ni] = a.lse_in[at];
                if (ok && a.g) g[ni] = a.g[at] * a.inv_t;
                if (ok && a.h) h[ni] = a.h[at] * a.inv_t;
                if (ok && a.h) entropy[ni] = a.entropy_in[at];
            }
        }
        GemmAcc acc;
        gemm.run(acc);
#pragma unroll
        for (int ni = 0; ni < 4; ++ni)  // waited for before the next copies start
            asm volatile("" : "+v"(tok[ni]), "+v"(g[ni]), "+v"(h[ni]), "+v"(lse[ni]), "+v"(entropy[ni]));
        more = walk.next();
        if (more) gemm.start(W, (int64_t)walk.row * kGemmTile, v_count, a.X, (int64_t)walk.col * kGemmTile, n, a.K, 0, steps);
        const int64_t first = v0 + wm * 128 + 4 * q;  // of this lane's choices in the chunk
#pragma unroll
        for (int ni = 0; ni < 4; ++ni) {
            const int64_t k = n0 + wn * 64 + ni * 16 + col;
            // the taken token's place among this lane's choices
            const int64_t from = tok[ni] - (v_base + first);
            const bool near = from >= 0 && from < 128 && from % 16 < 4;
            const bool live = (g[ni] != 0.0f || h[ni] != 0.0f) && lse[ni] != kNone;
            const float l2 = lse[ni] * kLog2e;
            float x[8][4];
#pragma unroll
            for (int mi = 0; mi < 8; ++mi) {
#pragma unroll
                for (int i = 0; i < 4; ++i) x[mi][i] = score_gradient(a, acc.c[mi][ni][i], l2, g[ni], h[ni], entropy[ni]);
            }
            if (near) {  // in few tiles
#pragma unroll
                for (int mi = 0; mi < 8; ++mi) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (from != mi * 16 + i) continue;
                        x[mi][i] = taken_gradient(a, acc.c[mi][ni][i], lse[ni], g[ni], h[ni], entropy[ni]);
                    }
                }
            }
            if (!live || first + 128 > v_count) {  // nothing from this token, or the last tile: zeros beyond
#pragma unroll
                for (int mi = 0; mi < 8; ++mi) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[mi][i] = live && first + mi * 16 + i < v_count ? x[mi][i] : 0.0f;
                }
            }
            // 16 bytes a lane: of rows mi and mi + 1, lanes of q = 0, 2 take the first's choices 0-7 and 8-15, q = 1, 3 the second's
            auto write = [&](int64_t row) {
                uint16_t* out = a.d + row * a.d_ld + v0 + wm * 128 + (q & 1) * 16 + (q / 2) * 8;
#pragma unroll
                for (int mi = 0; mi < 8; mi += 2) {
                    uint32_t e[2][2];
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            e[m][i] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x[mi + m][2 * i]) |
                                      (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x[mi + m][2 * i + 1]) << 16;
                    }
                    const u32x2_t s0 = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_permlane16_swap(e[0][0], e[1][0], false, false));
                    const u32x2_t s1 = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_permlane16_swap(e[0][1], e[1][1], false, false));
                    if (k < n) *reinterpret_cast<u32x4_t*>(out + mi * 16) = u32x4_t{s0.x, s1.x, s0.y, s1.y};
                }
            };
            write(k);
            if (two) {
#pragma unroll
                for (int mi = 0; mi < 8; ++mi) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[mi][i] = second_half(x[mi][i]);
                }
                write(n + k);
            }
        }
    }
}

// The same for at most 16 tokens, as in k_head_stats_few: 64 choices a wavefront.
__global__ __launch_bounds__(kFewThreads) void k_head_gradient_few(HeadArgs a, int64_t v_base, int64_t v_count) {
    static_assert(kFewTokens <= kHeadTwo);
    const int64_t n = live_tokens(a);
    if (n == 0) return;
    const int lane = lane_id(), w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), q = lane / 16, col = lane % 16;
    const int64_t v0 = (int64_t)blockIdx.x * kGemmTile + w * 64, first = v0 + 4 * q;
    int32_t tok = -1;
    float g = 0.0f, h = 0.0f, lse = 0.0f, entropy = 0.0f;
    if (col < n) {
        const int64_t at = a.shape.at((uint32_t)(a.list ? a.list[col] : col));
        tok = a.tokens[at];
        const bool ok = tok >= 0 && tok < a.V;
        if (!ok && v_base == 0 && v0 == 0 && q == 0) flag_error(a.err, ERR_TOKEN);
        lse = a.lse_in[at];
        if (ok && a.g) g = a.g[at] * a.inv_t;
        if (ok && a.h) h = a.h[at] * a.inv_t;
        if (ok && a.h) entropy = a.entropy_in[at];
    }
    f32x4_t acc[4];
    few_scores(a, a.W.p + (v_base + v0) * a.W.ld, v_count - v0, n, acc);
    if (col >= n) return;
    const int64_t from = tok - (v_base + first);  // the taken token's place among this lane's choices
    const bool live = (g != 0.0f || h != 0.0f) && lse != kNone;
    const float l2 = lse * kLog2e;
    uint16_t* out = a.d + col * a.d_ld + first;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint16_t e[2][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = 16 * i + j;
            float x = score_gradient(a, acc[i][j], l2, g, h, entropy);
            if (from == c) x = taken_gradient(a, acc[i][j], lse, g, h, entropy);
            x = live && first + c < v_count ? x : 0.0f;
            e[0][j] = __builtin_bit_cast(uint16_t, (__bf16)x);
            e[1][j] = __builtin_bit_cast(uint16_t, (__bf16)second_half(x));
        }
        __builtin_memcpy(out + 16 * i, e[0], 8);
        __builtin_memcpy(out + n * a.d_ld + 16 * i, e[1], 8);
    }
}

// Parts along k (of 8 steps at least) that a product of n_tiles tiles is split
// into: as many as fill a number of rounds of the compute units, for the number
// for which rounds times the length of a part, and 8 steps' time for a tile's
// start and its sums, is least.
__device__ __forceinline__ int32_t splits(int64_t n_tiles, int32_t steps, int32_t cus, int32_t most) {
    if (n_tiles <= 0) return 1;
    int32_t best = 1;
    float cost = (float)((n_tiles + cus - 1) / cus) * ((float)steps + 8.0f);
    if (most > steps / 8) most = steps / 8;
    for (int32_t rounds = 1; rounds <= 8; ++rounds) {
        int64_t s = (int64_t)rounds * cus / n_tiles;
        if (s > most) s = most;
        if (s < 1) continue;
        const float c = (float)((n_tiles * s + cus - 1) / cus) * ((float)steps / (float)s + 8.0f);
        if (c < cost) {
            cost = c;
            best = (int32_t)s;
        }
    }
    return best;
}

// part s of dX^T tiles: rows = hidden units, columns = tokens, k = choices (W as it stands is transposed here)
__global__ __launch_bounds__(kGemmThreads) void k_head_dhidden(HeadArgs a, int64_t v_base, int64_t v_count) {
    __shared__ __align__(1024) uint8_t lds[kGemmLds];
    const int64_t n = gradient_rows(a, live_tokens(a));
    const int32_t row_tiles = (int32_t)tiles(a.H), col_tiles = (int32_t)tiles(n), steps = (int32_t)((v_count + kGemmK - 1) / kGemmK);
    const int32_t S = splits((int64_t)row_tiles * col_tiles, steps, a.cus, a.splits);
    const GemmOperand W{a.W.p + v_base * a.W.ld, a.W.ld}, D{a.d, a.d_ld};
    const int lane = lane_id(), w = threadIdx.x / kWave, wm = w / 4, wn = w % 4, q = lane / 16, col = lane % 16;
    TileWalk walk((int64_t)row_tiles * S, col_tiles);
    GemmTiles<true, false> gemm;
    gemm.lds = lds;
    auto start = [&] {
        const int32_t s = walk.row / row_tiles;
        gemm.start(W, (int64_t)(walk.row % row_tiles) * kGemmTile, a.K, D, (int64_t)walk.col * kGemmTile, n, v_count,
                   (int32_t)((int64_t)steps * s / S), (int32_t)((int64_t)steps * (s + 1) / S));
    };
    bool more = walk.next();
    if (more) start();
    while (more) {
        const int64_t h0 = (int64_t)(walk.row % row_tiles) * kGemmTile, n0 = (int64_t)walk.col * kGemmTile;
        float* part = a.dx_part + (int64_t)(walk.row / row_tiles) * a.d_rows * a.h_ld;
        GemmAcc acc;
        gemm.run(acc);
        more = walk.next();
        if (more) start();
#pragma unroll
        for (int ni = 0; ni < 4; ++ni) {
            const int64_t k = n0 + wn * 64 + ni * 16 + col;
            if (k >= n) continue;
#pragma unroll
            for (int mi = 0; mi < 8; ++mi) {
                const int64_t h = h0 + wm * 128 + mi * 16 + 4 * q;
                if (h < a.h_ld) *reinterpret_cast<f32x4_t*>(part + k * a.h_ld + h) = acc.c[mi][ni];
            }
        }
    }
}

// the parts of dX of this chunk of choices (and, beyond the first, of those
// before) in a fixed order; after the last chunk bf16 rows, zeros where nothing
// counts.  GROUPS wavefronts share the parts of the same units, one after the
// other's; blockIdx.y takes the units' next 1,024 / GROUPS.  (10 tokens of 1,088
// units: four 7.6 us, one 14.3; 128 of 1,024: 15.0 and 16.4; 200 of 2,048: 15.5 and 13.6.)
template <int GROUPS>
__global__ __launch_bounds__(256) void k_head_dhidden_join(HeadArgs a, int64_t v_count, bool first, bool last) {
    constexpr int kLanes = 256 / GROUPS;
    __shared__ f32x4_t s_sum[GROUPS][kLanes];
    const int64_t t = blockIdx.x;
    const int64_t k = a.place ? a.place[t] : t;
    const int64_t n = live_tokens(a);
    const int32_t steps = (int32_t)((v_count + kGemmK - 1) / kGemmK);
    const int32_t S = splits(tiles(a.H) * tiles(gradient_rows(a, n)), steps, a.cus, a.splits);
    const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
    const int32_t s0 = S * group / GROUPS, s1 = S * (group + 1) / GROUPS;
    uint16_t* out = static_cast<uint16_t*>(a.dx.data) + a.dx.at((uint32_t)t, a.shape);
    for (int64_t h0 = 4 * kLanes * (int64_t)blockIdx.y; h0 < a.h_ld; h0 += 4 * kLanes * (int64_t)gridDim.y) {
        const int64_t h = h0 + 4 * lane;
        f32x4_t sum = {0, 0, 0, 0};
        f32x4_t* total = reinterpret_cast<f32x4_t*>(a.dx_sum + k * a.h_ld + h);
        if (k >= 0 && h < a.h_ld) {
            if (!first && group == 0) sum = *total;
            const int64_t step = a.d_rows * a.h_ld;
            auto add = [&](const float* part) {
                int32_t s = s0;
                for (; s + 8 <= s1; s += 8) {  // eight under way at once, added in their order
                    f32x4_t x[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const f32x4_t*>(part + (s + i) * step);
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum += x[i];
                }
                for (; s < s1; ++s) sum += *reinterpret_cast<const f32x4_t*>(part + s * step);
            };
            if (two_halves(a)) add(a.dx_part + (n + k) * a.h_ld + h);
            add(a.dx_part + k * a.h_ld + h);
        }
        if constexpr (GROUPS > 1) {
            s_sum[group][lane] = sum;
            __syncthreads();
            if (group == 0) {
#pragma unroll
                for (int i = 1; i < GROUPS; ++i) sum += s_sum[i][lane];
            }
            __syncthreads();
        }
        if (group != 0 || h >= a.h_ld) continue;
        if (!last && k >= 0) *total = sum;
        if (last) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (h + i < a.H) out[h + i] = __builtin_bit_cast(uint16_t, (__bf16)sum[i]);
        }
    }
}

__global__ __launch_bounds__(256) void k_head_zero(HeadArgs a) {
    for (int64_t v = blockIdx.x; v < a.V; v += gridDim.x)
        for (int64_t h = threadIdx.x; h < a.H; h += 256) a.dw[v * a.dw_ld + h] = 0;
}

// dW of a chunk: rows = hidden units, columns = choices, k = tokens (X and d as they stand are transposed here)
__global__ __launch_bounds__(kGemmThreads) void k_head_dweight(HeadArgs a, int64_t v_base, int64_t v_count) {
    __shared__ __align__(1024) uint8_t lds[kGemmLds];
    const int64_t n = gradient_rows(a, live_tokens(a));
    const int lane = lane_id(), w = threadIdx.x / kWave, wm = w / 4, wn = w % 4, q = lane / 16, col = lane % 16;
    const GemmOperand D{a.d, a.d_ld};
    const int32_t steps = (int32_t)((n + kGemmK - 1) / kGemmK);
    TileWalk walk(tiles(v_count), tiles(a.H));  // (column tiles are many here: they take the rows' part in the walk)
    GemmTiles<true, true> gemm;
    gemm.lds = lds;
    auto start = [&] {
        gemm.start(a.X, (int64_t)walk.col * kGemmTile, a.K, D, (int64_t)walk.row * kGemmTile, (v_count + 7) / 8 * 8, n, 0, steps);
    };
    bool more = walk.next();
    if (more) start();
    while (more) {
        const int64_t h0 = (int64_t)walk.col * kGemmTile, v0 = (int64_t)walk.row * kGemmTile;
        GemmAcc acc;
        gemm.run(acc);
        more = walk.next();
        if (more) start();
#pragma unroll
        for (int ni = 0; ni < 4; ++ni) {
            const int64_t v = v0 + wn * 64 + ni * 16 + col;
            uint16_t* out = a.dw + (v_base + v) * a.dw_ld;
#pragma unroll
            for (int mi = 0; mi < 8; mi += 2) {
                uint32_t e[2][2];  // as in k_head_gradient
#pragma unroll
                for (int m = 0; m < 2; ++m) {
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        e[m][i] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)acc.c[mi + m][ni][2 * i]) |
                                  (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)acc.c[mi + m][ni][2 * i + 1]) << 16;
                }
                const u32x2_t s0 = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_permlane16_swap(e[0][0], e[1][0], false, false));
                const u32x2_t s1 = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_permlane16_swap(e[0][1], e[1][1], false, false));
                const u32x4_t x = {s0.x, s1.x, s0.y, s1.y};
                const int64_t h = h0 + wm * 128 + (mi + (q & 1)) * 16 + (q / 2) * 8;
                if (v >= v_count) continue;
                if (h + 8 <= a.H) {
                    __builtin_memcpy(out + h, &x, 16);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (h + i < a.H) out[h + i] = (uint16_t)(x[i / 2] >> (i % 2 * 16));
                }
            }
        }
    }
}

}  // namespace

#define HEAD_LAUNCH(kernel, grid, threads, ...)                                 \
    do {                                                                        \
        hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, s, __VA_ARGS__);     \
        const hipError_t e_ = hipGetLastError();                                \
        if (e_ != hipSuccess) return e_;                                        \
    } while (0)

namespace {

// the list of tokens that count, and operands whose rows the product can read
hipError_t prepare_operands(HeadArgs& a, hipStream_t s) {
    if (a.mask) HEAD_LAUNCH(k_head_list, dim3(1), kListThreads, a);
    if (a.x_pack) {
        HEAD_LAUNCH(k_head_pack, dim3((unsigned)(a.d_rows < 65536 ? a.d_rows : 65536)), 256, a, static_cast<const uint16_t*>(a.x.data), 0,
                    a.H, a.x_pack, a.X.ld, 0, true);
    }
    if (a.w_pack) {
        HEAD_LAUNCH(k_head_pack, dim3((unsigned)(a.V < 65536 ? a.V : 65536)), 256, a, a.w_src, a.w_ld, a.H, a.w_pack, a.W.ld, a.V,
                    false);
    }
    return hipSuccess;
}

int64_t host_tiles(int64_t n) { return (n + kGemmTile - 1) / kGemmTile; }

// At most 16 tokens, by rows of W in registers or by tiles: long rows of more
// choices than one round of tiles are as fast or faster by tiles (16 tokens, 4,096
// units: scores over 128,000 choices 214 us by tiles and 249 by rows, 70,000 210 and
// 212, 32,000 90 and 76; of 8,192 units and 128,000 choices 411 and 406; the logits'
// gradient 256 and 290, 107 and 106 over 32,000, 106 and 79 of 2,048 units and 64,000).
bool few_tokens(const HeadArgs& a, int64_t choices) {
    return a.N <= kFewTokens && (a.K <= kFewHidden || host_tiles(choices) <= a.cus);
}

}  // namespace

hipError_t launch_head_logprobs(HeadArgs a, hipStream_t s) {
    hipError_t e = prepare_operands(a, s);
    if (e != hipSuccess) return e;
    if (few_tokens(a, a.V)) HEAD_LAUNCH(k_head_stats_few, dim3((unsigned)host_tiles(a.V)), kFewThreads, a);
    else HEAD_LAUNCH(k_head_stats, dim3(tile_grid(host_tiles(a.V), host_tiles(a.N), a.cus)), kGemmThreads, a);
    // few tokens: a workgroup each
    if (a.N <= 4 * a.cus) HEAD_LAUNCH(k_head_join<256>, dim3((unsigned)a.N), 256, a);
    else HEAD_LAUNCH(k_head_join<16>, dim3((unsigned)((a.N + 15) / 16)), 256, a);
    return hipSuccess;
}

hipError_t launch_head_backward(HeadArgs a, hipStream_t s) {
    if (a.N == 0) {  // no tokens: the projection's gradient is 0
        HEAD_LAUNCH(k_head_zero, dim3((unsigned)(a.V < 65536 ? a.V : 65536)), 256, a);
        return hipSuccess;
    }
    hipError_t e = prepare_operands(a, s);
    if (e != hipSuccess) return e;
    for (int64_t v = 0; v < a.V; v += a.chunk) {
        const int64_t count = a.V - v < a.chunk ? a.V - v : a.chunk;
        const bool first = v == 0, last = v + count == a.V;
        if (few_tokens(a, count)) HEAD_LAUNCH(k_head_gradient_few, dim3((unsigned)host_tiles(count)), kFewThreads, a, v, count);
        else HEAD_LAUNCH(k_head_gradient, dim3(tile_grid(host_tiles(count), host_tiles(a.N), a.cus)), kGemmThreads, a, v, count);
        HEAD_LAUNCH(k_head_dhidden, dim3(tile_grid(host_tiles(a.H) * a.splits, host_tiles(a.N), a.cus)), kGemmThreads, a, v, count);
        if (a.N <= kHeadTwo)  // few tokens' sums are of many parts
            HEAD_LAUNCH(k_head_dhidden_join<4>, dim3((unsigned)a.N, (unsigned)((a.h_ld + 255) / 256)), 256, a, count, first, last);
        else
            HEAD_LAUNCH(k_head_dhidden_join<1>, dim3((unsigned)a.N), 256, a, count, first, last);
        HEAD_LAUNCH(k_head_dweight, dim3(tile_grid(host_tiles(count), host_tiles(a.H), a.cus)), kGemmThreads, a, v, count);
    }
    return hipSuccess;
}

}  // namespace conduit
