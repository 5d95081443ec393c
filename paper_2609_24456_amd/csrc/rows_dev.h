// Rows of float or bf16 scores in 16-byte vectors (k_logits.hip, k_top.hip,
// k_listed.hip).
#pragma once

#include "softmax_dev.h"

namespace conduit {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

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
// ONCE: past the caches' order, at a higher rate, for rows that these do not hold: of
// 1,488 rows of 128,000 bf16 the best 64 in 84 us, else 91; 32 given choices of 4,088 x
// 50,001 fp32 130, else 139
template <bool ONCE, typename T>
__device__ __forceinline__ u32x4 read16(const T* p) {
    typedef u32x4 __attribute__((aligned(2))) any;
    if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const any*>(p));
    else return load16(p);
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

// A row of V elements as vectors from an ALIGN-byte boundary on, and the elements beside
// them: fewer than ALIGN bytes of them before, fewer than kPer after.
//   4, to be read: 16-byte accesses that start at an odd bf16 element take longer (the
// best 64 of 1,488 rows of 127,999: 106 us, from the boundary on 83; rows of odd widths
// start at one every other time).
//   64, to be written: see put16.
template <bool BF16, int ALIGN>
struct RowVectors {
    static constexpr int kPer = Elem<BF16>::kPer, kSize = 16 / kPer;
    static constexpr int kMostBeside = ALIGN / kSize - 1 + kPer - 1;
    uint32_t head;   // elements before the vectors
    uint32_t count;  // vectors
    uint32_t rest;   // elements after them
    __device__ __forceinline__ RowVectors(const void* row, uint32_t V) {
        head = (uint32_t)(-reinterpret_cast<uintptr_t>(row) % ALIGN) / kSize;
        head = head < V ? head : V;
        count = (V - head) / kPer;
        rest = (V - head) % kPer;
    }
    // the elements beside the vectors: those after them, then those before
    __device__ __forceinline__ uint32_t beside() const { return rest + head; }
    __device__ __forceinline__ uint32_t beside_at(uint32_t t) const { return t < rest ? head + count * kPer + t : t - rest; }
    // where element `id` is: vector i (count: beside them) and its place j
    __device__ __forceinline__ void find(uint32_t id, uint32_t* i, uint32_t* j) const {
        const uint32_t k = id - head;
        *i = id < head ? count : k / kPer;
        *j = id < head ? rest + id : k % kPer;
    }
};

// A vector of a gradient, at a multiple of 16 bytes.  PAST: past the caches, at a higher
// rate, for gradients that these do not hold until they are read: 8,192 x 128,000 bf16,
// 36% of them live, 557 us, else 594; then read and written once more 1,280 and 1,337;
// but 2,048 x 50,001, which the caches hold, 148 and 126.  Rows that do not start at a
// 64-byte boundary lose by it (4,088 x 32,001 fp32, 36% live: from a boundary on 135, from
// the first element on 149, in the caches' order 141).
template <bool PAST, typename T>
__device__ __forceinline__ void put16(T* p, u32x4 v) {
    if constexpr (PAST) __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p));
    else *reinterpret_cast<u32x4*>(p) = v;
}

// a vector of scores at -inf
template <bool BF16>
__device__ __forceinline__ u32x4 no_vector() {
    constexpr uint32_t w = BF16 ? 0xff80ff80u : 0xff800000u;
    return u32x4{w, w, w, w};
}

}  // namespace conduit
