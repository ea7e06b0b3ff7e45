// Divergence of a student's logits from a teacher's top logits, and its gradient.
//
//   p = softmax over the row's entries of teacher / tau;  q = softmax over the vocabulary of z / tau
//   loss = tau^2 sum_k p_k (log p_k - log q_{i_k});   dz_v = dloss tau (q_v [row has entries] - sum over k with i_k = v of p_k)
//
// Bound by HBM: the logits have to be read once (forward), or read once and the gradient written once.  A row is walked by
// the blocks of a cluster, each on its part: a pass with a running maximum and sum, an exchange over the cluster through
// distributed shared memory, and for the gradient a second pass that finds part of the row in L2.  What a row needs
// besides its logits (entries, the logits at their places, its weight) is asked for before the first pass, so that its
// latencies, some 8 us in a row when each is waited for in turn, lie under the stream.
//
// Eight 16-byte loads in flight a thread and 1024 threads an SM: with four loads and 2048 threads the rows in flight
// (592 of 256 KB at 131072 bf16 values) leave nothing of a row in L2 (4096 rows: 416 us against 509).
// Measured and not kept: rows held on the chip between the passes, in registers and shared memory of one block per SM or
// of a cluster (4096 x 131072: 480 and 620 us; the phases of a row no longer overlap those of others).
//
// All exponentials are 2^x: with c = log2(e) / tau, exp(z / tau - max) = 2^(z c - max c) is one multiply-add.
#pragma once

#include <cfloat>
#include <type_traits>

#include "bns_async.cuh"

namespace bns {

constexpr int kDistillMaxEntries = 1024;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kFar = 0x1p29f;       // beyond it the rounding of max c, 2^-24 of it, is too much for an exponent
constexpr float kNear = 0x1p28f;      // beside a maximum within it, what lies below -kFar is 0

// Maximum m of a set of values times c (rounded once: it is only the reference) and sum of 2^(value c - m).  Values whose
// maximum is beyond kFar (masks such as -1e10, or the type's lowest value) add nothing but the maximum: a row whose own
// maximum is beyond kNear is done again, of differences.
struct TopSum {
    float m, s;
};
__device__ __forceinline__ float reference(float m) { return fabsf(m) <= kFar ? m : __int_as_float(0x7f800000); }
__device__ __forceinline__ TopSum top_of(float value, float c) {
    const float m = value * c;
    return {m, exp2_fast(fmaf(value, c, -reference(m)))};
}
// Joins two; a side without values (m = -inf, s = 0) changes nothing.  NaN travels in s.
__device__ __forceinline__ TopSum join(TopSum a, TopSum b) {
    const float m = fmaxf(a.m, b.m);
    const float ref = m == __int_as_float(0xff800000) ? 0.f : m;
    return {m, a.s * exp2_fast(a.m - ref) + b.s * exp2_fast(b.m - ref)};
}

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
template <typename T>
__device__ __forceinline__ void add_exps(const uint4& raw, pair_t c, pair_t minus_ref, pair_t& sum) {
    constexpr int P = 8 / sizeof(typename T::storage);
    pair_t e[P];
    exp_pairs<T>(raw, c, minus_ref, e);
#pragma unroll
    for (int q = 0; q < P; ++q) sum = add2(sum, e[q]);
}
// Writes 2^(c value - shift) factor; `vectors`: the place is 16-byte aligned.
template <typename T, bool VECTORS>
__device__ __forceinline__ void write_exps(typename T::storage* to, const uint4& raw, pair_t c, pair_t minus_shift, pair_t factor) {
    constexpr int V = 16 / sizeof(typename T::storage), P = V / 2;
    pair_t e[P];
    exp_pairs<T>(raw, c, minus_shift, e);
    Vec<T, V> o;
#pragma unroll
    for (int q = 0; q < P; ++q) set_vec_pair<T, V>(o, q, mul2(e[q], factor));
    if constexpr (VECTORS) {
        __stcs(reinterpret_cast<uint4*>(to), o.raw);
    } else {
        const typename T::storage* f = reinterpret_cast<const typename T::storage*>(&o.raw);
#pragma unroll
        for (int j = 0; j < V; ++j) to[j] = f[j];
    }
}
__device__ __forceinline__ pair_t twice(float v) { return make_pair(v, v); }
__device__ __forceinline__ float both(pair_t v) {
    float lo, hi;
    split_pair(v, lo, hi);
    return lo + hi;
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
    int parts, per;       // blocks a row is split over, vectors of each
};

struct DistillForward {};   // loss and log-sum
struct DistillBackward {};  // gradient, from the log-sum of the forward call
struct DistillStep {};      // both in one launch

constexpr int kDistillThreads = 512, kDistillSmall = 128;      // of a block; the second for short rows
constexpr int kDistillParts = 8;                                    // most blocks a row is split over
constexpr int kDistillOwn = 2;                                      // entries that a thread looks after
static_assert(kDistillThreads * kDistillOwn == kDistillMaxEntries);
constexpr int kDistillDepth = 8;                                    // vectors in flight per thread

// The student's maximum and sum as the forward call's log-sum tells them: lse tau c = m + rest with the same c as in
// z c, so that only z - lse tau feels its rounding; 2^rest stands in for the sum.
__device__ __forceinline__ TopSum student_of(const Distill& a, float lse) {
    const double exponent = static_cast<double>(lse) * a.tau * a.c;
    const float m = static_cast<float>(exponent);
    return {m, exp2_fast(static_cast<float>(exponent - m))};
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

// Both pairs of all lanes joined: the maximum first, so that each sum is scaled once.
__device__ __forceinline__ void warp_join(TopSum& a, TopSum& b) {
    float ma = a.m, mb = b.m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        ma = fmaxf(ma, __shfl_xor_sync(0xffffffffu, ma, o));
        mb = fmaxf(mb, __shfl_xor_sync(0xffffffffu, mb, o));
    }
    const float inf = __int_as_float(0x7f800000);
    a.s *= exp2_fast(a.m - (ma == -inf ? 0.f : ma));
    b.s *= exp2_fast(b.m - (mb == -inf ? 0.f : mb));
    a.m = ma;
    b.m = mb;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
        b.s += __shfl_xor_sync(0xffffffffu, b.s, o);
    }
}

// The teacher's probability at place i: the sum over all entries there, in the list's order.
__device__ __forceinline__ float share_of(const int* place, const float* p, int K, int i) {
    float share = 0.f;
    for (int j = 0; j < K; j += 4) {
        const int4 at = *reinterpret_cast<const int4*>(place + j);
        const float4 pj = *reinterpret_cast<const float4*>(p + j);
        share += at.x == i ? pj.x : 0.f;
        share += at.y == i ? pj.y : 0.f;
        share += at.z == i ? pj.z : 0.f;
        share += at.w == i ? pj.w : 0.f;
    }
    return share;
}

// A row whose largest logit, or largest teacher's value, times c is beyond kNear (all of them masked with -1e10 or with the
// type's lowest value, say): everything is taken of differences, which the fast form has no time for.  Runs after the fast
// form has written what it made of the row, and replaces that: there nothing is kept in registers for later, and its
// loops are left rolled (4096 x 131072: 419 us; 416 without it, 430 unrolled, 450 as a function that is called).  Every block looks at the whole row and writes its own columns.  A row of -inf alone
// has no answer: it stays.
template <typename T, bool LOSS, bool GRAD>
__device__ __forceinline__ void distill_far_row(const Distill& a, const int* place, float* p, float* fold) {
    using S = typename T::storage;
    constexpr int V = 16 / sizeof(S);
    int block, tid;      // read again, so that nothing derived from them is kept across the fast form's loops
    asm volatile("mov.u32 %0, %%ctaid.x;" : "=r"(block));
    asm volatile("mov.u32 %0, %%tid.x;" : "=r"(tid));
    const int64_t row = block / a.parts;
    const int part = block - static_cast<int>(row) * a.parts, threads = blockDim.x;
    const S* z = static_cast<const S*>(a.z) + row * a.z_stride;
    const float inf = __int_as_float(0x7f800000);
    auto larger = [](float x, float y) { return fmaxf(x, y); };
    auto plus = [](float x, float y) { return x + y; };
    float base = 0.f, sum = 1.f;
    if constexpr (LOSS) {
        float top = -inf;
#pragma unroll 1
        for (int v = tid; v < a.V; v += threads) top = fmaxf(top, to_float<T>(z[v]));
        base = block_of(top, fold, larger);
        if (base == -inf) return;
        float mine = 0.f;
#pragma unroll 1
        for (int v = tid; v < a.V; v += threads) mine += exp2_fast((to_float<T>(z[v]) - base) * a.c);
        sum = block_of(mine, fold, plus);
    } else {
        base = a.lse_in[row] * a.tau;
    }
    auto entry = [&](int k) {
        const int64_t e = row * a.K + k;
        return a.teacher_bf16 ? to_float<BF16>(static_cast<const unsigned short*>(a.teacher)[e])
                              : static_cast<const float*>(a.teacher)[e];
    };
    float most = -inf, total = 0.f;
#pragma unroll 1
    for (int k = tid; k < a.K; k += threads)
        if (place[k] >= 0) most = fmaxf(most, entry(k));
    most = block_of(most, fold, larger);
    const bool any = most != -inf;
#pragma unroll 1
    for (int k = tid; k < a.K; k += threads)
        if (place[k] >= 0 && any) total += exp2_fast((entry(k) - most) * a.c);
    total = block_of(total, fold, plus);
    float loss = 0.f;
#pragma unroll 1
    for (int k = tid; k < (a.K + 3) / 4 * 4; k += threads) {
        float pk = 0.f;
        if (k < a.K && place[k] >= 0 && any) {
            const float v = (entry(k) - most) * a.c;
            pk = exp2_fast(v) / total;
            if (LOSS && pk != 0.f)
                loss = fmaf(pk, (v + log2f(sum) - log2f(total)) * kLn2 + (base - to_float<T>(z[place[k]])) / a.tau, loss);
        }
        p[k] = pk;
    }
    if constexpr (LOSS) {
        loss = block_of(loss, fold, plus);
        if (tid == 0 && part == 0) {
            a.loss[row] = a.tau * a.tau * loss;
            if (a.lse) a.lse[row] = base / a.tau + log2f(sum) * kLn2;
        }
    }
    if constexpr (GRAD) {
        S* dz = static_cast<S*>(a.dz) + row * a.dz_stride;
        const float g = a.dloss[row] * a.tau, factor = g / sum;
        const int head = min(a.V, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(z) & 15)) & 15) / static_cast<int>(sizeof(S)));
        const int vectors = (a.V - head) / V, begin = min(vectors, part * a.per), end = min(vectors, begin + a.per);
        const int first = part == 0 ? 0 : head + begin * V, last = part == a.parts - 1 ? a.V : head + end * V;
        auto q = [&](float v) {
            const float e = (v - base) * a.c;
            return exp2_fast(e > 0.f ? 0.f : e) * factor;      // above 0 only by the rounding of a given log-sum
        };
#pragma unroll 1
        for (int v = first + tid; v < last; v += threads) dz[v] = from_float<T>(any ? q(to_float<T>(z[v])) : 0.f);
        __syncthreads();
#pragma unroll 1
        for (int k = tid; k < a.K; k += threads) {
            const int i = place[k];
            if (i >= first && i < last && any) dz[i] = from_float<T>(q(to_float<T>(z[i])) - g * share_of(place, p, a.K, i));
        }
    }
}

// Part blockIdx % parts of row blockIdx / parts: `per` vectors, and the loose elements at either end of the row.
template <typename T, typename WHAT, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) distill_kernel(const Distill a) {
    using S = typename T::storage;
    constexpr int V = 16 / sizeof(S), kWarps = THREADS / 32, kMost = THREADS * kDistillOwn;
    constexpr bool kLoss = !__is_same(WHAT, DistillBackward), kGrad = !__is_same(WHAT, DistillForward);
    __shared__ __align__(16) float p[kMost];      // filled up to a multiple of four with no entries
    __shared__ __align__(16) int place[kMost];
    __shared__ TopSum fold[2][kWarps];                  // teacher, student
    __shared__ TopSum of_part[kDistillParts];
    __shared__ float sums[kWarps];
    __shared__ bool far;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const float inf = __int_as_float(0x7f800000);
    // Another block's shared memory may be written once that block runs: all of the cluster arrive here, and wait for one
    // another after the row's pass, which hides it
    if (kLoss && a.parts > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
    grid_dependency_wait();
    grid_dependency_launch();
    const int64_t row = blockIdx.x / a.parts;
    const int part = blockIdx.x - static_cast<int>(row) * a.parts;
    const S* z = static_cast<const S*>(a.z) + row * a.z_stride;

    // asked for first: the entries (places outside the vocabulary, or negative ones, are none), the row's scalars, loose elements
    int64_t own_index[kDistillOwn];
    float own_value[kDistillOwn], own_z[kDistillOwn];
#pragma unroll
    for (int o = 0; o < kDistillOwn; ++o) {
        const int k = tid + o * THREADS;
        own_index[o] = -1;
        own_value[o] = -inf;
        if (k < a.K) {
            const int64_t e = row * a.K + k;
            own_index[o] = a.index64 ? static_cast<const long long*>(a.index)[e] : static_cast<const int*>(a.index)[e];
            own_value[o] = a.teacher_bf16 ? to_float<BF16>(static_cast<const unsigned short*>(a.teacher)[e])
                                          : static_cast<const float*>(a.teacher)[e];
        }
    }
    float g = 0.f, lse = 0.f;
    if constexpr (kGrad) g = a.dloss[row] * a.tau;
    if constexpr (!kLoss) lse = a.lse_in[row];
    const int head = min(a.V, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(z) & 15)) & 15) / static_cast<int>(sizeof(S)));
    const int vectors = (a.V - head) / V, tail = head + vectors * V;
    const int begin = min(vectors, part * a.per), end = min(vectors, begin + a.per);
    // elements outside whole vectors: those before them belong to the first part, those after them to the last
    const int loose = part == 0 && tid < head ? tid : part == a.parts - 1 && tid >= 32 && tid - 32 < a.V - tail ? tail + tid - 32 : -1;
    const float loose_z = loose >= 0 ? to_float<T>(z[loose]) : -inf;
    const uint4* body = reinterpret_cast<const uint4*>(z + head);
    uint4 x[kDistillDepth];
    auto fetch = [&](int v0) {
#pragma unroll
        for (int i = 0; i < kDistillDepth; ++i)
            if (v0 + i * THREADS < end) x[i] = body[v0 + i * THREADS];
    };
    fetch(begin + tid);
    TopSum teacher{-inf, 0.f}, st{-inf, 0.f};
#pragma unroll
    for (int o = 0; o < kDistillOwn; ++o) {
        const int k = tid + o * THREADS;
        if (own_index[o] < 0 || own_index[o] >= a.V) {
            own_index[o] = -1;
            own_value[o] = -inf;
        } else {
            TopSum t = top_of(own_value[o], a.c);
            if (own_value[o] != -inf) t.m = fmaxf(t.m, -FLT_MAX);      // the type's lowest value is not -inf
            teacher = join(teacher, t);
        }
        own_z[o] = own_index[o] >= 0 ? to_float<T>(z[own_index[o]]) : 0.f;
        if (k < (a.K + 3) / 4 * 4) place[k] = static_cast<int>(own_index[o]);
    }

    if constexpr (kLoss) {
        if (loose >= 0) st = top_of(loose_z, a.c);
        for (int v0 = begin + tid; v0 < end; v0 += THREADS * kDistillDepth) {
            if (v0 != begin + tid) fetch(v0);
            TopOf<T> top;
#pragma unroll
            for (int i = 0; i < kDistillDepth; ++i)
                if (v0 + i * THREADS < end) top.add(x[i]);
            const float m = fmaxf(top.get() * a.c, st.m);
            const float ref = reference(m);
            pair_t sum = make_pair(st.s * exp2_fast(st.m - ref), 0.f);
#pragma unroll
            for (int i = 0; i < kDistillDepth; ++i)
                if (v0 + i * THREADS < end) add_exps<T>(x[i], twice(a.c), twice(-ref), sum);
            st = TopSum{m, both(sum)};
        }
    }
    // one exchange for both: every warp joins all warps' pairs, in the same order
    warp_join(teacher, st);
    if (lane == 0) {
        fold[0][warp] = teacher;
        fold[1][warp] = st;
    }
    __syncthreads();
    teacher = lane < kWarps ? fold[0][lane] : TopSum{-inf, 0.f};
    st = lane < kWarps ? fold[1][lane] : TopSum{-inf, 0.f};
    warp_join(teacher, st);
    if constexpr (kLoss) {
        if (a.parts > 1) {      // every block of the cluster gets every block's pair, and joins them in the same order
            asm volatile("barrier.cluster.wait;" ::: "memory");      // all of them run
            if (tid < a.parts) {
                unsigned to;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(smem_address(&of_part[part])), "r"(tid));
                asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(st.m), "f"(st.s) : "memory");
            }
            asm volatile("barrier.cluster.arrive.release;" ::: "memory");
            asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
            st = of_part[0];
            for (int q = 1; q < a.parts; ++q) st = join(st, of_part[q]);
        }
    } else {
        st = student_of(a, lse);
    }
    const bool any = teacher.s != 0.f;             // false: no entry, or all at -inf

    // the log-sum of a backward call tells -inf (nothing to do again) from far down
    if (tid == 0) far = (!(fabsf(st.m) <= kNear) && (kLoss || lse != -inf)) || (fabsf(teacher.m) > kNear && teacher.m != -inf);
    if (kLoss && tid == 0 && part == 0 && a.lse) a.lse[row] = (st.m + log2f(st.s)) * kLn2;

    // p_k, and the loss of differences to the two maxima: log p_k - log q_k in units of ln 2
    float loss = 0.f;
    const float between = kLoss ? log2f(st.s) - log2f(teacher.s) : 0.f;
#pragma unroll
    for (int o = 0; o < kDistillOwn; ++o) {
        const int k = tid + o * THREADS;
        const float v = fmaf(own_value[o], a.c, -teacher.m);
        const float pk = any && own_value[o] != -inf ? exp2_fast(v) / teacher.s : 0.f;
        if (kLoss && pk != 0.f) loss = fmaf(pk, (v - fmaf(own_z[o], a.c, -st.m)) + between, loss);
        if (k < (a.K + 3) / 4 * 4) p[k] = pk;
    }
    if constexpr (kLoss) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) loss += __shfl_xor_sync(0xffffffffu, loss, o);
        if (lane == 0) sums[warp] = loss;
    }
    if constexpr (kGrad) {
        // q_v g = 2^(z_v c - shift) factor
        const float shift = st.m == -inf ? 0.f : st.m, factor = g / st.s;
        S* dz = static_cast<S*>(a.dz) + row * a.dz_stride;
        if (loose >= 0) dz[loose] = from_float<T>(any ? exp2_fast(fmaf(loose_z, a.c, -shift)) * factor : 0.f);
        auto write = [&](auto aligned) {
            for (int v0 = begin + tid; v0 < end; v0 += THREADS * kDistillDepth) {
                if (kLoss || v0 != begin + tid) fetch(v0);
                S* to = dz + head + static_cast<int64_t>(v0) * V;
#pragma unroll
                for (int i = 0; i < kDistillDepth; ++i)
                    if (v0 + i * THREADS < end)
                        write_exps<T, aligned.value>(to + i * THREADS * V, x[i], twice(a.c), twice(-shift), twice(factor));
            }
        };
        if (!any)
            for (int v = begin * V + tid; v < end * V; v += THREADS) dz[head + v] = from_float<T>(0.f);
        else if (((reinterpret_cast<uintptr_t>(dz) ^ reinterpret_cast<uintptr_t>(z)) & 15) == 0)
            write(std::true_type{});
        else
            write(std::false_type{});
        __syncthreads();     // the places of the entries in this part have their q: now q minus the teacher's share, the sum
                             // over all entries there in the list's order, the same for every repetition of a place
        const int first = part == 0 ? 0 : head + begin * V, last = part == a.parts - 1 ? a.V : head + end * V;
#pragma unroll
        for (int o = 0; o < kDistillOwn; ++o) {
            const int i = static_cast<int>(own_index[o]);
            if (i < first || i >= last || !any) continue;
            const float share = share_of(place, p, a.K, i);
            dz[i] = from_float<T>(exp2_fast(fmaf(own_z[o], a.c, -shift)) * factor - g * share);
        }
    } else {
        __syncthreads();
    }
    if (kLoss && tid == 0 && part == 0) {
        float sum = 0.f;
        for (int w = 0; w < kWarps; ++w) sum += sums[w];
        a.loss[row] = a.tau * a.tau * kLn2 * sum;
    }
    if (far) {
        __syncthreads();     // what this replaces is written
        distill_far_row<T, kLoss, kGrad>(a, place, p, sums);
    }
}

}  // namespace bns
