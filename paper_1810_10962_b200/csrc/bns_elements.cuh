// What every kernel file of the library uses: programmatic dependent launch, element types, vectors of
// up to 16 bytes, packed fp32 pairs, 2^x.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace bns {

// Programmatic dependent launch: wait until the preceding kernel of the stream has completed and
// its writes are visible (a no-op when the launch did not ask for early scheduling).
__device__ __forceinline__ void grid_dependency_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// Allow the next kernel of the stream to be scheduled once every block of this one got here.
__device__ __forceinline__ void grid_dependency_launch() { asm volatile("griddepcontrol.launch_dependents;"); }

// ------------------------------------------------------------------------------------ element types
struct F32 {
    using storage = float;
};
struct BF16 {
    using storage = unsigned short;
};

template <typename T>
__device__ __forceinline__ float to_float(typename T::storage v);
template <>
__device__ __forceinline__ float to_float<F32>(float v) {
    return v;
}
template <>
__device__ __forceinline__ float to_float<BF16>(unsigned short v) {
    return __uint_as_float(static_cast<unsigned>(v) << 16);
}
template <typename T>
__device__ __forceinline__ typename T::storage from_float(float v);
template <>
__device__ __forceinline__ float from_float<F32>(float v) {
    return v;
}
template <>
__device__ __forceinline__ unsigned short from_float<BF16>(float v) {
    return __bfloat16_as_ushort(__float2bfloat16_rn(v));  // round to nearest even
}

template <int BYTES>
struct RawWord;
template <>
struct RawWord<2> {
    using type = unsigned short;
};
template <>
struct RawWord<4> {
    using type = unsigned;
};
template <>
struct RawWord<8> {
    using type = uint2;
};
template <>
struct RawWord<16> {
    using type = uint4;
};

// V consecutive elements moved as one machine word of 2..16 bytes.
template <typename T, int V>
struct Vec {
    using S = typename T::storage;
    using raw_t = typename RawWord<sizeof(S) * V>::type;
    raw_t raw;
    __device__ __forceinline__ void load(const S* p) { raw = *reinterpret_cast<const raw_t*>(p); }
    __device__ __forceinline__ void store(S* p) const { *reinterpret_cast<raw_t*>(p) = raw; }
    __device__ __forceinline__ float get(int j) const { return to_float<T>(reinterpret_cast<const S*>(&raw)[j]); }
    __device__ __forceinline__ void set(int j, float v) { reinterpret_cast<S*>(&raw)[j] = from_float<T>(v); }
    // whole-vector conversion; the bf16 case works on 32-bit pairs (one shift or mask per element on the
    // way in, one cvt.rn.bf16x2.f32 per pair on the way out)
    __device__ __forceinline__ void unpack(float (&f)[V]) const {
        if constexpr (sizeof(S) == 2 && V >= 2) {
            const unsigned* w = reinterpret_cast<const unsigned*>(&raw);
#pragma unroll
            for (int q = 0; q < V / 2; ++q) {
                f[2 * q] = __uint_as_float(w[q] << 16);
                f[2 * q + 1] = __uint_as_float(w[q] & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) f[j] = get(j);
        }
    }
    __device__ __forceinline__ void pack(const float (&f)[V]) {
        if constexpr (sizeof(S) == 2 && V >= 2) {
            unsigned* w = reinterpret_cast<unsigned*>(&raw);
#pragma unroll
            for (int q = 0; q < V / 2; ++q) {
                __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * q], f[2 * q + 1]);  // low half = first argument
                w[q] = *reinterpret_cast<unsigned*>(&h);
            }
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) set(j, f[j]);
        }
    }
};

// Two fp32 values in one 64-bit register pair, for the packed fp32x2 arithmetic of sm_100 (each half is
// an ordinary round-to-nearest fp32 operation, so results equal the scalar ones bit for bit).
using pair_t = unsigned long long;
__device__ __forceinline__ pair_t make_pair(float lo, float hi) {
    pair_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void split_pair(pair_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ pair_t add2(pair_t a, pair_t b) {
    pair_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ pair_t mul2(pair_t a, pair_t b) {
    pair_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ pair_t fma2(pair_t a, pair_t b, pair_t c) {
    pair_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}

// Elements 2q and 2q+1 of a vector as a pair, and back (bf16: one 32-bit word holds both).
template <typename T, int V>
__device__ __forceinline__ pair_t vec_pair(const Vec<T, V>& v, int q) {
    if constexpr (sizeof(typename T::storage) == 2) {
        const unsigned w = reinterpret_cast<const unsigned*>(&v.raw)[q];
        return make_pair(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    } else {
        const float* f = reinterpret_cast<const float*>(&v.raw);
        return make_pair(f[2 * q], f[2 * q + 1]);
    }
}
template <typename T, int V>
__device__ __forceinline__ void set_vec_pair(Vec<T, V>& v, int q, pair_t p) {
    float lo, hi;
    split_pair(p, lo, hi);
    if constexpr (sizeof(typename T::storage) == 2) {
        __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);  // low half = first argument
        reinterpret_cast<unsigned*>(&v.raw)[q] = *reinterpret_cast<unsigned*>(&h);
    } else {
        float* f = reinterpret_cast<float*>(&v.raw);
        f[2 * q] = lo;
        f[2 * q + 1] = hi;
    }
}

__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));   // 2 ulp, 2^-126 and below give 0
    return r;
}

__device__ __forceinline__ unsigned smem_address(const void* p) { return static_cast<unsigned>(__cvta_generic_to_shared(p)); }

}  // namespace bns
