// Divergence of a student's logits from a teacher's top logits, and its gradient.
//
//   p = softmax over the row's entries of teacher / tau;  q = softmax over the vocabulary of z / tau
//   loss = tau^2 sum_k p_k (log p_k - log q_{i_k});   dz_v = dloss tau (q_v [row has entries] - sum over k with i_k = v of p_k)
//
// Bound by HBM: the logits are read once (forward), or read once and the gradient written once.  A block owns a row;
// the pass that writes the gradient reads the row again, out of L2 (148 SMs hold a few rows of some 100 KB each).
// The statistics are one pass with a running maximum and sum a thread, joined in a fixed order.
//
// All exponentials are 2^x: with c = log2(e) / tau, exp(z / tau - max) = 2^(z c - max c) is one multiply-add.
#pragma once

#include "bns_elements.cuh"

namespace bns {

constexpr int kDistillThreads = 512;
constexpr int kDistillMaxEntries = 1024;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));   // 2 ulp, 2^-126 and below give 0
    return r;
}

// Maximum m of a set of values times c (rounded once: it is only the reference) and sum of 2^(value c - m).
struct TopSum {
    float m, s;
};
__device__ __forceinline__ TopSum top_of(float value, float c) {
    const float m = value * c;
    return {m, m == __int_as_float(0xff800000) ? 0.f : exp2_fast(fmaf(value, c, -m))};
}
// Joins two; a side without values (m = -inf, s = 0) changes nothing.  NaN travels in s.
__device__ __forceinline__ TopSum join(TopSum a, TopSum b) {
    const float m = fmaxf(a.m, b.m);
    const float ref = m == __int_as_float(0xff800000) ? 0.f : m;
    return {m, a.s * exp2_fast(a.m - ref) + b.s * exp2_fast(b.m - ref)};
}

struct Distill {
    const void* z;
    const void* teacher;
    const void* index;
    const float* dloss;
    const float* lse_in;  // backward only
    float* loss;
    float* lse;
    void* dz;
    int64_t z_stride, dz_stride;
    int64_t rows;
    int V, K;
    int index64, teacher_bf16;
    float tau, c;         // c = log2(e) / tau
};

struct DistillForward {};   // loss and log-sum
struct DistillBackward {};  // gradient, from the log-sum of the forward call
struct DistillStep {};      // both in one launch

template <typename T, typename WHAT>
__global__ void __launch_bounds__(kDistillThreads) distill_kernel(const Distill a) {
    using S = typename T::storage;
    constexpr int V = 16 / sizeof(S);
    constexpr bool kLoss = !__is_same(WHAT, DistillBackward), kGrad = !__is_same(WHAT, DistillForward);
    constexpr int kWarpsHere = kDistillThreads / 32;
    __shared__ float p[kDistillMaxEntries];
    __shared__ int place[kDistillMaxEntries];
    __shared__ TopSum fold[kWarpsHere];
    __shared__ float fold2[kWarpsHere];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const float inf = __int_as_float(0x7f800000);
    grid_dependency_wait();
    grid_dependency_launch();
    const int64_t row = blockIdx.x;
    const S* z = static_cast<const S*>(a.z) + row * a.z_stride;

    // the teacher's distribution: places outside the vocabulary (or negative: no entry) carry nothing
    TopSum t{-inf, 0.f};
    for (int k = tid; k < a.K; k += kDistillThreads) {
        const int64_t e = row * a.K + k;
        const int64_t i = a.index64 ? static_cast<const long long*>(a.index)[e] : static_cast<const int*>(a.index)[e];
        const bool there = i >= 0 && i < a.V;
        const float v = a.teacher_bf16 ? to_float<BF16>(static_cast<const unsigned short*>(a.teacher)[e])
                                       : static_cast<const float*>(a.teacher)[e];
        place[k] = there ? static_cast<int>(i) : -1;
        p[k] = there ? v : -inf;
        if (there) t = join(t, top_of(v, a.c));
    }
    auto block_join = [&](TopSum v) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const TopSum w{__shfl_xor_sync(0xffffffffu, v.m, o), __shfl_xor_sync(0xffffffffu, v.s, o)};
            v = join(v, w);
        }
        __syncthreads();
        if (lane == 0) fold[warp] = v;
        __syncthreads();
        v = lane < kWarpsHere ? fold[lane] : TopSum{-inf, 0.f};
#pragma unroll
        for (int o = kWarpsHere / 2; o > 0; o >>= 1) {
            const TopSum w{__shfl_xor_sync(0xffffffffu, v.m, o), __shfl_xor_sync(0xffffffffu, v.s, o)};
            v = join(v, w);
        }
        return TopSum{__shfl_sync(0xffffffffu, v.m, 0), __shfl_sync(0xffffffffu, v.s, 0)};
    };
    const TopSum teacher = block_join(t);
    const bool any = teacher.s != 0.f;            // false: no entry, or all at -inf

    // head: elements before the row's first 16-byte boundary; then whole vectors; then the tail
    const int head = min(a.V, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(z) & 15)) & 15) / static_cast<int>(sizeof(S)));
    const int vectors = (a.V - head) / V, tail = head + vectors * V;
    const S* body = z + head;

    TopSum st{-inf, 0.f};
    if constexpr (kLoss) {
        auto take = [&](float v) { st = join(st, top_of(v, a.c)); };
        if (tid < head) take(to_float<T>(z[tid]));
        if (tid < a.V - tail) take(to_float<T>(z[tail + tid]));
        for (int v = tid; v < vectors; v += kDistillThreads) {
            Vec<T, V> x;
            float f[V];
            x.load(body + static_cast<int64_t>(v) * V);
            x.unpack(f);
            float m = f[0];
#pragma unroll
            for (int j = 1; j < V; ++j) m = fmaxf(m, f[j]);
            m = fmaxf(m * a.c, st.m);
            const float ref = m == -inf ? 0.f : m;
            float s = st.s * exp2_fast(st.m - ref);
#pragma unroll
            for (int j = 0; j < V; ++j) s += exp2_fast(fmaf(f[j], a.c, -ref));
            st = TopSum{m, s};
        }
        st = block_join(st);
    }
    // q_v = 2^(z_v c - shift) scale
    float shift, scale;
    if constexpr (kLoss) {
        shift = st.m == -inf ? 0.f : st.m;
        scale = 1.f / st.s;
        if (tid == 0 && a.lse) a.lse[row] = (st.m + log2f(st.s)) * kLn2;
    } else {
        // lse tau c = shift + rest, with the same c as in z c, so that only z - lse tau feels its rounding; rest goes
        // into the factor
        const double exponent = static_cast<double>(a.lse_in[row]) * a.tau * a.c;
        shift = static_cast<float>(exponent);
        scale = exp2_fast(static_cast<float>(shift - exponent));
    }
    // p_k, and the loss
    float loss = 0.f, between = 0.f;               // between: log-sum of the student minus the teacher's
    if constexpr (kLoss) between = ((st.m - teacher.m) + (log2f(st.s) - log2f(teacher.s))) * kLn2;
    for (int k = tid; k < a.K; k += kDistillThreads) {
        float pk = 0.f;
        if (place[k] >= 0 && any) {
            const float v = p[k];
            pk = v == -inf ? 0.f : exp2_fast(fmaf(v, a.c, -teacher.m)) / teacher.s;
            if constexpr (kLoss) {
                if (pk != 0.f) loss = fmaf(pk, (v - to_float<T>(z[place[k]])) / a.tau + between, loss);
            }
        }
        p[k] = pk;
    }
    if constexpr (kLoss) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) loss += __shfl_xor_sync(0xffffffffu, loss, o);
        if (lane == 0) fold2[warp] = loss;
        __syncthreads();
        if (tid == 0) {
            float sum = 0.f;
            for (int w = 0; w < kWarpsHere; ++w) sum += fold2[w];
            a.loss[row] = a.tau * a.tau * sum;
        }
    } else {
        __syncthreads();
    }
    if constexpr (kGrad) {
        S* dz = static_cast<S*>(a.dz) + row * a.dz_stride;
        const float g = a.dloss[row] * a.tau;
        const float factor = any ? g * scale : 0.f;
        auto q = [&](float v) { return any ? exp2_fast(fmaf(v, a.c, -shift)) * factor : 0.f; };
        if (tid < head) dz[tid] = from_float<T>(q(to_float<T>(z[tid])));
        if (tid < a.V - tail) dz[tail + tid] = from_float<T>(q(to_float<T>(z[tail + tid])));
        const bool same_phase = ((reinterpret_cast<uintptr_t>(dz) ^ reinterpret_cast<uintptr_t>(z)) & 15) == 0;
        for (int v = tid; v < vectors; v += kDistillThreads) {
            Vec<T, V> x;
            float f[V];
            x.load(body + static_cast<int64_t>(v) * V);
            x.unpack(f);
#pragma unroll
            for (int j = 0; j < V; ++j) f[j] = q(f[j]);
            S* to = dz + head + static_cast<int64_t>(v) * V;
            if (same_phase) {
                x.pack(f);
                x.store(to);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) to[j] = from_float<T>(f[j]);
            }
        }
        __syncthreads();   // the entries' places have their q: now q minus the teacher's share (every repetition of a
                           // place writes the same value, the sum over all of them in the list's order)
        for (int k = tid; k < a.K; k += kDistillThreads) {
            const int i = place[k];
            if (i < 0 || !any) continue;
            float share = 0.f;
            for (int j = 0; j < a.K; ++j)
                if (place[j] == i) share += p[j];
            dz[i] = from_float<T>(q(to_float<T>(z[i])) - g * share);
        }
    }
}

}  // namespace bns
