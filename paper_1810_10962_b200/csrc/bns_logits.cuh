// What the kernels that walk rows of logits share: 2^(c z - reference) of 16-byte vectors, maxima, sums over a block.
#pragma once

#include "bns_elements.cuh"

namespace bns {

constexpr float kLn2 = 0.6931471805599453f;
constexpr double kLn2Exact = 0.693147180559945309;
constexpr float kFar = 0x1p29f;       // beyond it the rounding of max c, 2^-24 of it, is too much for an exponent
constexpr float kNear = 0x1p28f;      // beside a maximum within it, what lies below -kFar is 0

// Values whose maximum, times c, is beyond kFar add nothing but the maximum.
__device__ __forceinline__ float reference(float m) { return fabsf(m) <= kFar ? m : __int_as_float(0x7f800000); }

// ---- arithmetic on 16-byte vectors of logits.  The kernels issue some nine instructions an element where memory leaves
// time for twelve, so pairs go through packed fp32 arithmetic, and bf16 maxima are taken on the stored pairs.
template <typename T>
struct TopOf;
template <>
struct TopOf<F32> {
    float v;
    __device__ __forceinline__ TopOf() : v(-__builtin_huge_valf()) {}
    __device__ __forceinline__ void add(const uint4& raw) {
        const float* f = reinterpret_cast<const float*>(&raw);
        v = fmaxf(v, fmaxf(fmaxf(f[0], f[1]), fmaxf(f[2], f[3])));
    }
    __device__ __forceinline__ float get() const { return v; }
};
template <>
struct TopOf<BF16> {
    __nv_bfloat162 v;
    __device__ __forceinline__ TopOf() { *reinterpret_cast<unsigned*>(&v) = 0xff80ff80u; }
    __device__ __forceinline__ void add(const uint4& raw) {
        const __nv_bfloat162* w = reinterpret_cast<const __nv_bfloat162*>(&raw);
        v = __hmax2(v, __hmax2(__hmax2(w[0], w[1]), __hmax2(w[2], w[3])));
    }
    __device__ __forceinline__ float get() const { return fmaxf(__low2float(v), __high2float(v)); }
};

// 2^(c value - ref) of a vector's pairs.
template <typename T>
__device__ __forceinline__ void exp_pairs(const uint4& raw, pair_t c, pair_t minus_ref, pair_t (&e)[8 / sizeof(typename T::storage)]) {
    constexpr int V = 16 / sizeof(typename T::storage);
    Vec<T, V> x;
    x.raw = raw;
#pragma unroll
    for (int q = 0; q < V / 2; ++q) {
        float lo, hi;
        split_pair(fma2(vec_pair<T, V>(x, q), c, minus_ref), lo, hi);
        e[q] = make_pair(exp2_fast(lo), exp2_fast(hi));
    }
}
__device__ __forceinline__ pair_t twice(float v) { return make_pair(v, v); }
__device__ __forceinline__ float both(pair_t v) {
    float lo, hi;
    split_pair(v, lo, hi);
    return lo + hi;
}

// A value of all threads of the block, joined in warp order; `fold` is shared memory for a value of each warp.
template <typename Join>
__device__ __forceinline__ float block_of(float v, float* fold, Join&& join_two) {
    const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = join_two(v, __shfl_xor_sync(0xffffffffu, v, o));
    __syncthreads();
    if (lane == 0) fold[threadIdx.x >> 5] = v;
    __syncthreads();
    v = fold[0];
    for (int w = 1; w < warps; ++w) v = join_two(v, fold[w]);
    __syncthreads();
    return v;
}

}  // namespace bns
