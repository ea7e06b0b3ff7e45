// Global norm over many gradients, and clipping by it.
//
//   norm = sqrt(sum over all elements of all tensors of g^2);  factor = 1 where norm <= max_norm, else max_norm / norm
//   out = g factor
//
// Bound by HBM: the norm reads every element once, clipping reads it again (what fits of it out of L2, hence back to front)
// and writes it (3.7 GB of bf16: the norm 0.53 ms, 7.0 TB/s; clipping 1.69 ms in all).  The list travels in the kernels'
// arguments, so nothing is copied to the device and a captured graph holds all it needs.  All tensors are taken as one line
// of 16-byte vectors, whatever their sizes, which the blocks take chunk by chunk; elements outside whole vectors go with a
// place of their own in front of each tensor's vectors.
//
// Squares are added in fp32 over a batch of vectors, batches and everything above in 64 bits.  A batch whose sum leaves the
// range in which fp32 squares are exact enough is done again in 64 bits.
#pragma once

#include "bns_elements.cuh"

namespace bns {

constexpr int kClipThreads = 256;
constexpr int kClipDepth = 8;            // vectors in flight per thread
constexpr int kClipBlocks = 3;           // per SM: 80 registers, which clipping needs (four an SM: 3.8 TB/s in fp32 for 6.2)

template <int N>
struct ClipList {
    int64_t first[N + 1];                // places in the line, and its length
    const void* in[N];
    void* out[N];
    int64_t elements[N];                 // times two, plus one for bf16
    int count, chunk;                    // tensors; places that a block takes at a time
    int in_place;                        // all of them
};

// Where a tensor's whole vectors begin and how many there are.
template <typename T>
struct ClipSpan {
    int head;
    int64_t vectors, n;
    __device__ __forceinline__ ClipSpan(const void* p, int64_t elements) : n(elements) {
        constexpr int V = 16 / sizeof(typename T::storage);
        const int to_word = static_cast<int>((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / static_cast<int>(sizeof(typename T::storage));
        head = n < to_word ? static_cast<int>(n) : to_word;
        vectors = (n - head) / V;
    }
    // thread t's element outside whole vectors, or -1: at most 2 V - 2 of them
    __device__ __forceinline__ int64_t loose(int t) const {
        constexpr int V = 16 / sizeof(typename T::storage);
        const int64_t tail = head + vectors * V;
        return t < head ? t : t >= 16 && t < 32 && tail + t - 16 < n ? tail + t - 16 : -1;
    }
};

// Calls visit(tensor, from, to: its places) for the tensors of chunk c of the line.
template <int N, typename Visit>
__device__ __forceinline__ void visit_chunk(const ClipList<N>& list, int64_t c, Visit&& visit) {
    const int64_t begin = c * list.chunk, end = min(begin + list.chunk, list.first[list.count]);
    int low = 0, high = list.count;                      // the last tensor that begins at or before `begin` is in [low, high)
    while (high - low > 1) {
        const int middle = (low + high) / 2;
        if (list.first[middle] <= begin)
            low = middle;
        else
            high = middle;
    }
    int64_t first = list.first[low];
    for (int e = low; e < list.count && first < end; ++e) {
        const int64_t last = list.first[e + 1];
        visit(e, max(begin, first) - first, min(end, last) - first);
        first = last;
    }
}
template <int N>
__host__ __device__ __forceinline__ int64_t chunks_of(const ClipList<N>& list) { return (list.first[list.count] + list.chunk - 1) / list.chunk; }

template <typename T>
__device__ __forceinline__ double squares_of(const void* data, int64_t elements, int64_t from, int64_t to) {
    using S = typename T::storage;
    constexpr int V = 16 / sizeof(S);
    const S* p = static_cast<const S*>(data);
    const ClipSpan<T> span(data, elements);
    double total = 0.;
    if (from == 0) {
        const int64_t i = span.loose(threadIdx.x);
        if (i >= 0) {
            const double f = to_float<T>(p[i]);
            total = f * f;
        }
    }
    const int64_t begin = from > 0 ? from - 1 : 0;
    const uint4* body = reinterpret_cast<const uint4*>(p + span.head) + begin;
    const int count = static_cast<int>(to - 1 - begin);
    for (int v0 = threadIdx.x; v0 < count; v0 += kClipThreads * kClipDepth) {
        Vec<T, V> x[kClipDepth];
#pragma unroll
        for (int i = 0; i < kClipDepth; ++i) {
            x[i].raw = make_uint4(0, 0, 0, 0);
            if (v0 + i * kClipThreads < count) x[i].raw = body[v0 + i * kClipThreads];
        }
        pair_t sum[2] = {};
#pragma unroll
        for (int i = 0; i < kClipDepth; ++i)
#pragma unroll
            for (int q = 0; q < V / 2; ++q) {
                const pair_t f = vec_pair<T, V>(x[i], q);
                sum[q & 1] = fma2(f, f, sum[q & 1]);
            }
        float lo, hi;
        split_pair(add2(sum[0], sum[1]), lo, hi);
        const float s = lo + hi;
        if (s > 0x1p-80f && s < 0x1p120f) {          // squares below 2^-126 are not whole, but then they do not count
            total += s;
            continue;
        }
        unsigned bits = 0;
#pragma unroll
        for (int i = 0; i < kClipDepth; ++i) bits |= x[i].raw.x | x[i].raw.y | x[i].raw.z | x[i].raw.w;
        if (bits & (sizeof(S) == 2 ? 0x7fff7fffu : 0x7fffffffu)) {      // not all zeros
#pragma unroll 1
            for (int i = 0; i < kClipDepth; ++i) {
                const int v = v0 + i * kClipThreads;
                if (v >= count) break;
                const S* f = reinterpret_cast<const S*>(body + v);
#pragma unroll 1
                for (int j = 0; j < V; ++j) {
                    const double d = to_float<T>(f[j]);
                    total += d * d;
                }
            }
        }
    }
    return total;
}

// The sum over the block's threads, for thread 0.
__device__ __forceinline__ double block_sum(double v, double* fold) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) fold[threadIdx.x >> 5] = v;
    __syncthreads();
    if (threadIdx.x < 32) {
        v = threadIdx.x < kClipThreads / 32 ? fold[threadIdx.x] : 0.;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    }
    return v;
}

template <int N>
__global__ void __launch_bounds__(kClipThreads, kClipBlocks) clip_squares_kernel(const __grid_constant__ ClipList<N> list, double* partial) {
    __shared__ double fold[kClipThreads / 32];
    grid_dependency_wait();
    grid_dependency_launch();
    double total = 0.;
    const int64_t chunks = chunks_of(list);
    for (int64_t c = blockIdx.x; c < chunks; c += gridDim.x)
        visit_chunk(list, c, [&](int e, int64_t from, int64_t to) {
            const int64_t elements = list.elements[e];
            if (elements & 1)
                total += squares_of<BF16>(list.in[e], elements >> 1, from, to);
            else
                total += squares_of<F32>(list.in[e], elements >> 1, from, to);
        });
    total = block_sum(total, fold);
    if (threadIdx.x == 0) partial[blockIdx.x] = total;
}

// The norm from the blocks' sums, in the same order by every block that asks; all its threads get the sum.
__device__ __forceinline__ double sum_partials(const double* partial, int count, double* fold) {
    if (count == 1) return partial[0];
    double v = 0.;
    for (int i = threadIdx.x; i < count; i += kClipThreads) v += partial[i];
    v = block_sum(v, fold);
    __syncthreads();
    if (threadIdx.x == 0) fold[0] = v;
    __syncthreads();
    return fold[0];
}

// The norm, and the sum of all squares for whom it may concern.
__global__ void __launch_bounds__(kClipThreads) clip_norm_kernel(const double* partial, int count, double* total, float* norm) {
    __shared__ double fold[kClipThreads / 32];
    grid_dependency_wait();
    grid_dependency_launch();
    const double sum = sum_partials(partial, count, fold);
    if (threadIdx.x == 0) {
        *total = sum;
        *norm = static_cast<float>(sqrt(sum));
    }
}

template <typename T>
__device__ __forceinline__ void scale_span(const void* data, void* out, int64_t elements, int64_t from, int64_t to, float factor) {
    using S = typename T::storage;
    constexpr int V = 16 / sizeof(S);
    const S* p = static_cast<const S*>(data);
    S* o = static_cast<S*>(out);
    const ClipSpan<T> span(data, elements);
    if (from == 0) {
        const int64_t i = span.loose(threadIdx.x);
        if (i >= 0) o[i] = from_float<T>(to_float<T>(p[i]) * factor);
    }
    const int64_t begin = from > 0 ? from - 1 : 0;
    const uint4* body = reinterpret_cast<const uint4*>(p + span.head) + begin;
    S* to_body = o + span.head + begin * V;
    const int count = static_cast<int>(to - 1 - begin);
    if (reinterpret_cast<uintptr_t>(to_body) & 15) {       // at another phase than the gradient: element by element
        for (int v = threadIdx.x; v < count; v += kClipThreads) {
            Vec<T, V> x;
            x.raw = body[v];
#pragma unroll
            for (int j = 0; j < V; ++j) to_body[static_cast<int64_t>(v) * V + j] = from_float<T>(x.get(j) * factor);
        }
        return;
    }
    const pair_t by = make_pair(factor, factor);
    for (int v0 = threadIdx.x; v0 < count; v0 += kClipThreads * kClipDepth) {
        Vec<T, V> x[kClipDepth];
#pragma unroll
        for (int i = 0; i < kClipDepth; ++i)
            if (v0 + i * kClipThreads < count) x[i].raw = body[v0 + i * kClipThreads];
#pragma unroll
        for (int i = 0; i < kClipDepth; ++i) {
            if (v0 + i * kClipThreads >= count) continue;
            Vec<T, V> y;
#pragma unroll
            for (int q = 0; q < V / 2; ++q) set_vec_pair<T, V>(y, q, mul2(vec_pair<T, V>(x[i], q), by));
            __stcs(reinterpret_cast<uint4*>(to_body) + v0 + i * kClipThreads, y.raw);
        }
    }
}

// The block's chunk with a factor that fp32 has no normal number for, in 64 bits.
template <typename T>
__device__ __forceinline__ void scale_span_exactly(const void* data, void* out, int64_t elements, int64_t from, int64_t to, double factor) {
    constexpr int V = 16 / sizeof(typename T::storage);
    const typename T::storage* p = static_cast<const typename T::storage*>(data);
    typename T::storage* o = static_cast<typename T::storage*>(out);
    const ClipSpan<T> span(data, elements);
    auto scale = [&](int64_t i) { o[i] = from_float<T>(static_cast<float>(to_float<T>(p[i]) * factor)); };
    if (from == 0 && span.loose(threadIdx.x) >= 0) scale(span.loose(threadIdx.x));
    const int64_t begin = span.head + (from > 0 ? from - 1 : 0) * V, end = span.head + (to - 1) * V;
    for (int64_t i = begin + threadIdx.x; i < end; i += kClipThreads) scale(i);
}
template <int N>
__device__ __noinline__ void scale_exactly(const ClipList<N>& list, double factor) {
    visit_chunk(list, gridDim.x - 1 - blockIdx.x, [&](int e, int64_t from, int64_t to) {
        if (list.elements[e] & 1)
            scale_span_exactly<BF16>(list.in[e], list.out[e], list.elements[e] >> 1, from, to, factor);
        else
            scale_span_exactly<F32>(list.in[e], list.out[e], list.elements[e] >> 1, from, to, factor);
    });
}

// A block takes one chunk: blocks that walk down several drift apart, and reads and writes then go all over the memory (3.7 GB
// of bf16: 4.8 TB/s read + written for 6.5).  Every block finds the norm itself from the blocks' sums, or from their total where
// there are many blocks.  The line is taken back to front, since what the norm read last may still be in L2.
template <int N>
__global__ void __launch_bounds__(kClipThreads, kClipBlocks) clip_scale_kernel(const __grid_constant__ ClipList<N> list, const double* partial, int count, float max_norm, float* norm) {
    __shared__ double fold[kClipThreads / 32];
    grid_dependency_wait();
    grid_dependency_launch();
    const double exact = sqrt(sum_partials(partial, count, fold));
    const float rounded = static_cast<float>(exact);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = rounded;
    const double quotient = max_norm / exact;
    const float factor = rounded <= max_norm ? 1.f : static_cast<float>(quotient);
    const bool small = factor < 0x1p-126f && quotient > 0.;
    if (factor == 1.f && list.in_place) return;
    if (small) {
        scale_exactly(list, quotient);
        return;
    }
    visit_chunk(list, gridDim.x - 1 - blockIdx.x, [&](int e, int64_t from, int64_t to) {
        const void* in = list.in[e];
        void* out = list.out[e];
        if (factor == 1.f && in == out) return;
        const int64_t elements = list.elements[e];
        if (elements & 1)
            scale_span<BF16>(in, out, elements >> 1, from, to, factor);
        else
            scale_span<F32>(in, out, elements >> 1, from, to, factor);
    });
}

}  // namespace bns
