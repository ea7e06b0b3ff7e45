// Log probabilities of given tokens with the distribution's entropy and its top alternatives, and the logits' gradient.
//
//   q = softmax of z / tau;  logp = log q_token;  H = - sum_v q_v log q_v;  alternatives: the K largest (z_v, lowest v first)
//   dz_v = (dlogp ([v = token] - q_v) - dH q_v (log q_v + H)) / tau
//
// Bound by HBM: forward reads the logits once (4096 x 131072 bf16: 168 us, 6.4 TB/s), backward reads them and writes the gradient
// (317 us, 6.8 TB/s).  With c = log2(e) / tau and a reference m, the largest z c so far, a pass keeps
//   s = sum 2^(z c - m)  and  t = sum 2^(z c - m) (z c - m);  then  log2 q_v = z_v c - m - log2 s,  H = ln 2 (log2 s - t / s)
// t is a sum of terms of one sign, and a change of the reference by d scales both by 2^d after t has got d s.
// Small blocks (128 or 256 threads, 1024 an SM) with eight 16-byte loads in flight a thread: a row's reductions lie under the
// streams of other rows (blocks of 512: 182 us).
//
// Alternatives without a second pass: a thread keeps the largest value of each of its segments (up to eight) beside the
// sums, which the running maximum needs anyway.  K threads' largest values bound the K-th largest of the row from below,
// so only segments that reach that bound are read again (K of some 1000 segments, a few per cent of the row, out of L2);
// what reaches it, some K values, is ordered by comparing all with all.  20 of them: 201 us at the size above; each thread
// looking through its own segments took 291, as it waits for them one after another.
#pragma once

#include "bns_logits.cuh"

namespace bns {

constexpr int kLogpThreads = 256, kLogpSmall = 128, kLogpLarge = 512;     // of a block
constexpr int kLogpParts = 8;                           // most blocks a row is split over
constexpr int kLogpDepth = 8;                           // vectors in flight per thread
constexpr int kLogpMaxTop = 64;
constexpr int kLogpSegments = 8;                        // of a thread
constexpr int kLogpFound = 1024;                        // values that reach the bound, before the slow way is taken
constexpr int kLogpQueue = 512;                         // segments that reach it, likewise
constexpr int kLogpLooks = 4;                           // vectors of queued segments in flight per thread
constexpr float kLogpFloor = -0x1p60f;                  // stands in for anything lower: 2^(floor c - m) = 0, and 0 times it is 0
static_assert(kLogpParts * kLogpMaxTop <= kLogpFound);

struct LogProbs {
    const void* z;
    const void* token;
    const float *lse_in, *entropy_in, *dlogp, *dentropy;   // backward; dentropy may be NULL
    float *logp, *entropy, *lse, *top;
    int* index;
    void* dz;
    int64_t z_stride, dz_stride, rows;
    int V, K, token64;
    float tau, c;
    int parts, per;       // blocks of a row, vectors of each
    int walkers, walk;    // backward: the same where each block walks over all of its row
};

// Largest log-sum that the gradient takes q from.  It is rounded once, so q is off by half its step: 2^-17 just below 256 in fp32, 2^-13
// below 4096 for bf16 (2^-21 at ordinary log-sums of 8 to 16), beside the sum's own error.
template <typename T>
constexpr float kLogpKept = sizeof(typename T::storage) == 2 ? 0x1p12f : 0x1p8f;

// m, s and t of a set of values; m = -inf: none that counts.
struct Stats {
    float m, s, t;
};
// 2^d and d for a side whose reference moves up by -d; no reference yet: nothing to scale.
__device__ __forceinline__ void move_reference(Stats& a, float m) {
    const float d = a.m == m ? 0.f : fmaxf(a.m - m, -0x1p30f), f = exp2_fast(d);
    a.t = f * fmaf(d, a.s, a.t);
    a.s *= f;
    a.m = m;
}
// All lanes' sums joined: the maximum first, so that each is scaled once.
__device__ __forceinline__ void warp_join(Stats& a) {
    float m = a.m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    move_reference(a, m);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
        a.t += __shfl_xor_sync(0xffffffffu, a.t, o);
    }
}

// Whole numbers in the order of the values, both zeros alike; 0 is below -inf.
__device__ __forceinline__ unsigned order_key(float v) {
    const unsigned u = __float_as_uint(v + 0.f);
    return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float of_key(unsigned k) { return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xffffffffu)); }

// Not below the floor; NaN stays.
template <typename T>
__device__ __forceinline__ void raise_to_floor(uint4& raw) {
    if constexpr (sizeof(typename T::storage) == 2) {
        __nv_bfloat162* w = reinterpret_cast<__nv_bfloat162*>(&raw);
        const __nv_bfloat162 floor = __float2bfloat162_rn(kLogpFloor);
#pragma unroll
        for (int q = 0; q < 4; ++q) w[q] = __hmax2_nan(w[q], floor);
    } else {
        float* f = reinterpret_cast<float*>(&raw);
#pragma unroll
        for (int q = 0; q < 4; ++q) asm("max.NaN.f32 %0, %0, %1;" : "+f"(f[q]) : "f"(kLogpFloor));
    }
}

template <typename T>
__device__ __forceinline__ void add_stats(uint4 raw, pair_t c, pair_t minus_ref, pair_t& sum, pair_t& weighted) {
    constexpr int V = 16 / sizeof(typename T::storage);
    raise_to_floor<T>(raw);
    Vec<T, V> x;
    x.raw = raw;
#pragma unroll
    for (int q = 0; q < V / 2; ++q) {
        const pair_t u = fma2(vec_pair<T, V>(x, q), c, minus_ref);
        float lo, hi;
        split_pair(u, lo, hi);
        const pair_t e = make_pair(exp2_fast(lo), exp2_fast(hi));
        sum = add2(sum, e);
        weighted = fma2(e, u, weighted);
    }
}

template <typename T>
__device__ __forceinline__ bool any_nan(const uint4& raw) {
    constexpr int V = 16 / sizeof(typename T::storage);
    Vec<T, V> x;
    x.raw = raw;
    bool nan = false;
#pragma unroll
    for (int j = 0; j < V; ++j) nan |= x.get(j) != x.get(j);
    return nan;
}

// What a row's values are turned into log q with.
struct LogQ {
    float tau, c, m, log_s, base, lse;
    bool far;            // of differences to the largest value
    __device__ __forceinline__ float operator()(float v) const {
        if (far) return (v - base) / tau - log_s * kLn2;
        if (v < 0.f && !(v * c >= -kFar)) return v / tau - lse;     // a mask beside ordinary values: v c may leave fp32's range
        return (fmaf(v, c, -m) - log_s) * kLn2;
    }
};

// A value and its place as one number: the larger value, then the lower place, is the larger number.
using ranked_t = unsigned long long;
__device__ __forceinline__ ranked_t ranked(unsigned key, int at) { return static_cast<ranked_t>(key) << 32 | (0xffffffffu - static_cast<unsigned>(at)); }
__device__ __forceinline__ unsigned key_of(ranked_t r) { return static_cast<unsigned>(r >> 32); }
__device__ __forceinline__ int place_of(ranked_t r) { return static_cast<int>(0xffffffffu - static_cast<unsigned>(r)); }

struct Found {
    ranked_t value[kLogpFound];
    int count;
};

// put(rank, value) gets the K largest of `count` different numbers.
template <typename Put>
__device__ __forceinline__ void rank_found(const ranked_t* value, int count, int K, Put&& put) {
    for (int i = threadIdx.x; i < count; i += blockDim.x) {
        const ranked_t mine = value[i];
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < count; ++j) rank += value[j] > mine;
        if (rank < K) put(rank, mine);
    }
}

// Whole numbers of the values, NaN below all of them.
template <typename T>
__device__ __forceinline__ unsigned key_at(const typename T::storage* z, int v) {
    const float x = to_float<T>(z[v]);
    return x == x ? order_key(x) : 0u;
}

// The K-th largest number of the places [first, last) itself, for parts where more than kLogpFound values lie above `bound`, K
// of them or more: by halving, a walk over the part each time.  `found` gets the fewer than K numbers above it.
template <typename T>
__device__ __noinline__ unsigned find_bound(const typename T::storage* z, int first, int last, unsigned bound, int K, Found& found) {
    const int tid = threadIdx.x, threads = blockDim.x;
    auto reached = [&](unsigned key) {      // how many values reach it
        __syncthreads();
        if (tid == 0) found.count = 0;
        __syncthreads();
        int n = 0;
        for (int v = first + tid; v < last; v += threads) n += key_at<T>(z, v) >= key;
        n = __reduce_add_sync(0xffffffffu, n);
        if ((tid & 31) == 0 && n) atomicAdd(&found.count, n);
        __syncthreads();
        return found.count;
    };
    unsigned low = bound + 1, high = 0xffffffffu;
    while (low < high) {
        const unsigned middle = high - (high - low) / 2;
        if (reached(middle) >= K)
            low = middle;
        else
            high = middle - 1;
    }
    __syncthreads();
    if (tid == 0) found.count = 0;
    __syncthreads();
    for (int v = first + tid; v < last; v += threads) {
        const unsigned k = key_at<T>(z, v);
        if (k > low) found.value[atomicAdd(&found.count, 1)] = ranked(k, v);
    }
    __syncthreads();
    return low;
}

// Adds to `found`, up to K, the first places of [first, last) whose value is at the bound.
template <typename T>
__device__ __noinline__ void find_equals(const typename T::storage* z, int first, int last, unsigned bound, int K, Found& found, int* fold) {
    const int tid = threadIdx.x, threads = blockDim.x, lane = tid & 31, warp = tid >> 5, warps = threads >> 5;
    int have = found.count;
    for (int v0 = first; v0 < last && have < K; v0 += threads) {
        const int v = v0 + tid;
        const bool here = v < last && key_at<T>(z, v) == bound;
        const unsigned votes = __ballot_sync(0xffffffffu, here);
        __syncthreads();
        if (lane == 0) fold[warp] = __popc(votes);
        __syncthreads();
        int before = have + __popc(votes & ((1u << lane) - 1)), all = 0;
        for (int w = 0; w < warps; ++w) {
            before += w < warp ? fold[w] : 0;
            all += fold[w];
        }
        if (here && before < K) found.value[before] = ranked(bound, v);
        have = min(K, have + all);
    }
    __syncthreads();
    if (tid == 0) found.count = have;
    __syncthreads();
}

// Largest value of a row and sums over it of 2^d and 2^d d, d = (value - largest) c, by one block; for rows that the fast
// forms have no exponent for.  A row of -inf alone has a largest value of -inf, and NaN for sums.
template <typename T>
__device__ __noinline__ void sums_of_differences(const typename T::storage* z, int V, float c, float* fold, float& top, float& s, float& t) {
    using S = typename T::storage;
    constexpr int kVec = 16 / sizeof(S);
    auto larger = [](float p, float q) { return fmaxf(p, q); };
    auto plus = [](float p, float q) { return p + q; };
    const int head = min(V, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(z) & 15)) & 15) / static_cast<int>(sizeof(S)));
    const int vectors = (V - head) / kVec, tail = head + vectors * kVec, tid = threadIdx.x, threads = blockDim.x;
    const uint4* body = reinterpret_cast<const uint4*>(z + head);
    const int loose = tid < head ? tid : tid >= 32 && tid - 32 < V - tail ? tail + tid - 32 : -1;
    TopOf<T> mine;
#pragma unroll 4
    for (int v = tid; v < vectors; v += threads) mine.add(body[v]);
    top = block_of(fmaxf(mine.get(), loose >= 0 ? to_float<T>(z[loose]) : -__builtin_huge_valf()), fold, larger);
    s = t = 0.f;
    auto add = [&](float value) {
        const float d = (value - top) * c, e = exp2_fast(d);
        s += e;
        if (e != 0.f) t = fmaf(e, d, t);
    };
    if (loose >= 0) add(to_float<T>(z[loose]));
#pragma unroll 2
    for (int v = tid; v < vectors; v += threads) {
        Vec<T, kVec> x;
        x.raw = body[v];
#pragma unroll
        for (int j = 0; j < kVec; ++j) add(x.get(j));
    }
    s = block_of(s, fold, plus);
    t = block_of(t, fold, plus);
}

// What a block has in shared memory for the alternatives.
template <int THREADS>
struct TopShared {
    float segment[kLogpSegments][THREADS];                  // each thread's largest values
    Found found;
    ranked_t merged[kLogpParts * kLogpMaxTop];              // first block: every part's first ones
    unsigned key_range[2][THREADS / 32];
    int queue[kLogpQueue], queued;
    int fold[THREADS / 32];
};
template <int THREADS>
__device__ __forceinline__ TopShared<THREADS>& top_shared() {
    extern __shared__ __align__(16) char dynamic[];
    return *reinterpret_cast<TopShared<THREADS>*>(dynamic);
}

// A row's place in memory: elements in front of whole vectors, the part's vectors, the thread's element outside them or -1.  Those
// before the vectors belong to the first part, those after them to the last.
template <typename T>
struct RowPart {
    int head, begin, end, loose;
    __device__ __forceinline__ RowPart(const void* z, const LogProbs& a, int part) {
        using S = typename T::storage;
        constexpr int V = 16 / sizeof(S);
        const int tid = threadIdx.x;
        head = min(a.V, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(z) & 15)) & 15) / static_cast<int>(sizeof(S)));
        const int vectors = (a.V - head) / V;
        const int tail = head + vectors * V;
        begin = min(vectors, part * a.per);
        end = min(vectors, begin + a.per);
        loose = part == 0 && tid < head ? tid : part == a.parts - 1 && tid >= 32 && tid - 32 < a.V - tail ? tail + tid - 32 : -1;
    }
};
// Batches of vectors that make up a segment, so that a thread has kLogpSegments at the most.
template <int THREADS>
__device__ __forceinline__ int segment_batches(const LogProbs& a) {
    constexpr int kBatch = THREADS * kLogpDepth;
    return ((a.per + kBatch - 1) / kBatch + kLogpSegments - 1) / kLogpSegments;
}

// The K largest values of a row and their places.  `loose_z` and `mine` are the thread's element outside vectors and its largest
// one; everything else is found again, so that the pass over the row has its registers.
template <typename T, int THREADS>
__device__ __forceinline__ void alternatives(const LogProbs& a, int64_t row, int part, float loose_z, float mine, LogQ log_q) {
    using S = typename T::storage;
    constexpr int V = 16 / sizeof(S), kWarps = THREADS / 32, kBatch = THREADS * kLogpDepth;
    TopShared<THREADS>& sh = top_shared<THREADS>();
    Found& found = sh.found;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const float inf = __int_as_float(0x7f800000);
    const S* z = static_cast<const S*>(a.z) + row * a.z_stride;
    const RowPart<T> at_row(z, a, part);
    const int head = at_row.head, begin = at_row.begin, end = at_row.end, loose = at_row.loose, group = segment_batches<THREADS>(a);
    const uint4* body = reinterpret_cast<const uint4*>(z + head);
    // The largest bound that K threads' values reach, or a little lower, bit by bit below what all values have in common;
    // keys of bf16 values differ in their upper half.
    const bool has = loose >= 0 || begin + tid < end;
    const unsigned own_key = has ? order_key(mine) : 0u;
    constexpr int kLowest = sizeof(S) == 2 ? 16 : 0;
    const unsigned warp_most = __reduce_max_sync(0xffffffffu, own_key), warp_least = __reduce_min_sync(0xffffffffu, own_key);
    if (lane == 0) sh.key_range[0][warp] = warp_most, sh.key_range[1][warp] = warp_least;
    if (tid == 0) found.count = sh.queued = 0;
    __syncthreads();
    const unsigned most = __reduce_max_sync(0xffffffffu, sh.key_range[0][lane % kWarps]);
    const unsigned least = __reduce_min_sync(0xffffffffu, sh.key_range[1][lane % kWarps]);
    const int highest = 31 - __clz(most ^ least);          // -1: all the same
    const unsigned common = highest == 31 ? 0u : most & ~((2u << (highest & 31)) - 1u);
    unsigned bound = highest < 0 ? most : common;
    const int enough = a.K + a.K / 4 + 4;
#pragma unroll 1
    for (int bit = highest; bit >= kLowest; --bit) {
        const unsigned candidate = bound | (1u << bit);
        const int reach = __syncthreads_count(own_key >= candidate);
        if (reach >= a.K) bound = candidate;
        if (reach >= a.K && reach <= enough) break;
    }
    const int first = part == 0 ? 0 : head + begin * V, last = part == a.parts - 1 ? a.V : head + end * V;
    const int deep = max(1, min(kLogpDepth, (end - begin + THREADS - 1) / THREADS)), per_segment = deep * group, shift = 32 - __clz(per_segment - 1);
    auto look = [&](float v, int at) {
        const unsigned k = order_key(v);
        if (v == v && k >= bound) {
            const int to = atomicAdd(&found.count, 1);
            if (to < kLogpFound) found.value[to] = ranked(k, at);
        }
    };
    // Once as a rule.  Where there is no room for all that reach the bound (equal logits all over a row, a vocabulary masked
    // with one value but for a few places) the exact bound is taken, values above it are looked for in the same way, and
    // those at it place by place.
#pragma unroll 1
    for (bool exactly = false;; exactly = true) {
        // segments that reach the bound are queued, and all threads share their vectors
        if (has && own_key >= bound) {
            if (loose >= 0) look(loose_z, loose);
            for (int g = 0; begin + tid + g * group * kBatch < end; ++g)
                if (order_key(sh.segment[g][tid]) >= bound) {
                    const int to = atomicAdd(&sh.queued, 1);
                    if (to < kLogpQueue) sh.queue[to] = tid + g * group * kBatch;
                }
        }
        __syncthreads();
        const int looks = sh.queued > kLogpQueue ? 0 : sh.queued << shift;
        for (int w0 = tid; w0 < looks; w0 += THREADS * kLogpLooks) {
            int at[kLogpLooks];
            uint4 x[kLogpLooks];
#pragma unroll
            for (int i = 0; i < kLogpLooks; ++i) {
                const int w = w0 + i * THREADS, k = w & ((1 << shift) - 1);
                at[i] = w < looks && k < per_segment ? begin + sh.queue[w >> shift] + k * THREADS : end;
                if (at[i] < end) x[i] = body[at[i]];
            }
#pragma unroll
            for (int i = 0; i < kLogpLooks; ++i) {
                if (at[i] >= end) continue;
                Vec<T, V> y;
                y.raw = x[i];
                TopOf<T> top;
                top.add(y.raw);
                if (order_key(top.get()) < bound) continue;
#pragma unroll
                for (int j = 0; j < V; ++j) look(y.get(j), head + at[i] * V + j);
            }
        }
        __syncthreads();
        const bool room = found.count <= kLogpFound && sh.queued <= kLogpQueue;
        if (room && !exactly) break;
        if (exactly) {
            --bound;             // what lies above it has been looked for
            if (!room) bound = find_bound<T>(z, first, last, bound, a.K, found);
            if (bound && found.count < a.K) find_equals<T>(z, first, last, bound, a.K, found, sh.fold);
            break;
        }
        bound = highest < 0 ? most : common;
#pragma unroll 1
        for (int bit = highest; bit >= kLowest; --bit)
            if (__syncthreads_count(own_key >= (bound | (1u << bit))) >= a.K) bound |= 1u << bit;
        if (kLowest && bound && !(bound >> 31)) bound |= 0xffffu;      // of values below zero the lower half is ones
        ++bound;
        __syncthreads();
        if (tid == 0) found.count = sh.queued = 0;
        __syncthreads();
    }
    const int count = found.count;
    auto write = [&](int rank, ranked_t value) {
        a.top[row * a.K + rank] = log_q(of_key(key_of(value)));
        a.index[row * a.K + rank] = place_of(value);
    };
    auto nothing = [&](int rank) {
        a.top[row * a.K + rank] = -inf;
        a.index[row * a.K + rank] = -1;
    };
    if (a.parts == 1) {
        rank_found(found.value, count, a.K, write);
        for (int k = count + tid; k < a.K; k += THREADS) nothing(k);
    } else {
        // every part's K first go to the first block, which orders them; what is not there has key 0
        auto send = [&](int rank, ranked_t value) {
            unsigned to;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(smem_address(&sh.merged[part * a.K + rank])), "r"(0));
            asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(to), "l"(value) : "memory");
        };
        rank_found(found.value, count, a.K, send);
        for (int k = count + tid; k < a.K; k += THREADS) send(k, ranked(0u, k + part * a.K));
        asm volatile("barrier.cluster.arrive.release;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
        if (part == 0)
            rank_found(sh.merged, a.parts * a.K, a.K, [&](int rank, ranked_t value) {
                if (key_of(value))
                    write(rank, value);
                else
                    nothing(rank);
            });
    }
}

// Part blockIdx % parts of row blockIdx / parts: `per` vectors, and the loose elements at either end of the row.
template <typename T, bool TOP, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) logp_forward_kernel(const __grid_constant__ LogProbs a) {
    using S = typename T::storage;
    constexpr int kWarps = THREADS / 32;
    __shared__ Stats fold[kWarps];
    __shared__ Stats of_part[kLogpParts];
    __shared__ float sums[kWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const float inf = __int_as_float(0x7f800000);
    // Another block's shared memory may be written once that block runs: all of the cluster arrive here, and wait for one
    // another after the row's pass, which hides it
    if (a.parts > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
    grid_dependency_wait();
    grid_dependency_launch();
    const int64_t row = blockIdx.x / a.parts;
    const int part = blockIdx.x - static_cast<int>(row) * a.parts;
    const S* z = static_cast<const S*>(a.z) + row * a.z_stride;
    int64_t token = -1;
    if (tid == 0 && part == 0) token = a.token64 ? static_cast<const long long*>(a.token)[row] : static_cast<const int*>(a.token)[row];
    const RowPart<T> at_row(z, a, part);
    const int head = at_row.head, begin = at_row.begin, end = at_row.end, loose = at_row.loose;
    const float loose_z = loose >= 0 ? to_float<T>(z[loose]) : -inf;
    const uint4* body = reinterpret_cast<const uint4*>(z + head);
    uint4 x[kLogpDepth];
    auto fetch = [&](int v0) {
#pragma unroll
        for (int i = 0; i < kLogpDepth; ++i)
            if (v0 + i * THREADS < end) x[i] = body[v0 + i * THREADS];
    };
    fetch(begin + tid);
    float token_z = 0.f;
    const bool given = token >= 0 && token < a.V;
    if (given) token_z = to_float<T>(z[token]);

    Stats st{-inf, 0.f, 0.f};
    if (loose >= 0) {
        const float m = loose_z * a.c;
        if (fabsf(m) <= kFar) {
            const float u = fmaf(loose_z, a.c, -m), e = exp2_fast(u);      // what rounding m has left
            st = Stats{m, e, e * u};
        } else {
            st = Stats{m == m ? m : -inf, m == m ? 0.f : m, 0.f};
        }
    }
    constexpr int kBatch = THREADS * kLogpDepth;
    const int group = segment_batches<THREADS>(a);
    float mine = loose_z == loose_z ? loose_z : -inf;   // the thread's largest
    float of_segment = -inf;
    int segments = 0, left = group;
    for (int v0 = begin + tid; v0 < end; v0 += kBatch) {
        if (v0 != begin + tid) fetch(v0);
        TopOf<T> top;
#pragma unroll
        for (int i = 0; i < kLogpDepth; ++i)
            if (v0 + i * THREADS < end) top.add(x[i]);
        const float largest = top.get();
        const float m = fmaxf(largest * a.c, st.m);
        if (fabsf(m) <= kFar) {
            move_reference(st, m);
            pair_t sum = make_pair(st.s, 0.f), weighted = make_pair(st.t, 0.f);
#pragma unroll
            for (int i = 0; i < kLogpDepth; ++i)
                if (v0 + i * THREADS < end) add_stats<T>(x[i], twice(a.c), twice(-m), sum, weighted);
            st.s = both(sum);
            st.t = both(weighted);
        } else {                                       // nothing here counts beside an ordinary maximum, but NaN does
            bool nan = false;
#pragma unroll
            for (int i = 0; i < kLogpDepth; ++i)
                if (v0 + i * THREADS < end) nan |= any_nan<T>(x[i]);
            st = Stats{m, nan ? __int_as_float(0x7fffffff) : st.s, 0.f};
        }
        if constexpr (TOP) {
            of_segment = fmaxf(of_segment, largest);
            mine = fmaxf(mine, largest);
            if (--left == 0 || v0 + kBatch >= end) {
                top_shared<THREADS>().segment[segments++][tid] = of_segment;
                of_segment = -inf;
                left = group;
            }
        }
    }
    warp_join(st);
    if (lane == 0) fold[warp] = st;
    __syncthreads();
    st = lane < kWarps ? fold[lane] : Stats{-inf, 0.f, 0.f};
    warp_join(st);
    if (a.parts > 1) {      // every block of the cluster gets every block's sums, and joins them in the same order
        asm volatile("barrier.cluster.wait;" ::: "memory");      // all of them run
        if (tid < a.parts) {
            unsigned to;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(smem_address(&of_part[part])), "r"(tid));
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(st.m) : "memory");
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to + 4), "f"(st.s) : "memory");
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to + 8), "f"(st.t) : "memory");
        }
        asm volatile("barrier.cluster.arrive.release;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
        st = lane < a.parts ? of_part[lane] : Stats{-inf, 0.f, 0.f};
        warp_join(st);
    }

    const float log_s = log2f(st.s);
    float lse = static_cast<float>((static_cast<double>(st.m) + log_s) * kLn2Exact), entropy = (log_s - st.t / st.s) * kLn2;
    LogQ log_q{a.tau, a.c, st.m, log_s, 0.f, lse, false};
    if (!(fabsf(st.m) <= kNear)) {
        // The largest value times c is too large for the fast form (a row masked with -1e10 or the type's lowest value
        // throughout, say): everything of differences.  Every block looks at the whole row.
        float top, s, t;
        sums_of_differences<T>(z, a.V, a.c, sums, top, s, t);
        if (top != -inf || st.s != st.s) {
            log_q = LogQ{a.tau, a.c, 0.f, log2f(s), top, 0.f, true};
            lse = top / a.tau + log_q.log_s * kLn2;
            entropy = (log_q.log_s - t / s) * kLn2;
        } else {                                       // nothing is left of the row
            log_q = LogQ{1.f, 1.f, 0.f, 0.f, 0.f, 0.f, false};   // -inf of all that is there
            lse = -inf;
            entropy = 0.f;
        }
    }
    if (tid == 0 && part == 0) {
        a.logp[row] = given ? log_q(token_z) : 0.f;
        a.lse[row] = lse;
        if (a.entropy) a.entropy[row] = entropy;
    }

    if constexpr (TOP) alternatives<T, THREADS>(a, row, part, loose_z, mine, log_q);
}

// Gradients of the elements outside vectors and of the vectors [begin, end) of a row whose log-sum's rounding is too much for q: largest value and
// sum once more, of differences.
template <typename T>
__device__ __noinline__ void gradient_of_differences(const LogProbs& a, const typename T::storage* z, typename T::storage* dz, int head, int begin, int end,
                                                     int loose, int token, float g, float h, float entropy, float lse, float* fold) {
    using S = typename T::storage;
    constexpr int V = 16 / sizeof(S);
    float base, s, t;
    sums_of_differences<T>(z, a.V, a.c, fold, base, s, t);
    const float log_s = log2f(s);
    const bool empty = lse == -__builtin_huge_valf() && base == lse;       // a log-sum of -inf may also be one that has left fp32's range
    auto value = [&](float v) {
        if (empty) return 0.f;
        const float u = (v - base) * a.c - log_s, e = exp2_fast(u);
        return e == 0.f ? 0.f : -e * (g + h * fmaf(u, kLn2, entropy));
    };
    auto at_token = [&](float v) { return empty ? 0.f : value(v) + g; };
    const uint4* body = reinterpret_cast<const uint4*>(z + head);
    const int threads = blockDim.x;
    const bool in_body = token >= head + begin * V && token < head + end * V;
    const bool mine = in_body && ((token - head) / V - begin) % threads == threadIdx.x;
    const float token_z = mine ? to_float<T>(z[token]) : 0.f;
    if (loose >= 0) dz[loose] = from_float<T>(loose == token ? at_token(to_float<T>(z[loose])) : value(to_float<T>(z[loose])));
    const bool words = ((reinterpret_cast<uintptr_t>(dz) ^ reinterpret_cast<uintptr_t>(z)) & 15) == 0;
    for (int v0 = begin + threadIdx.x; v0 < end; v0 += threads * kLogpDepth) {
        uint4 x[kLogpDepth];
#pragma unroll
        for (int i = 0; i < kLogpDepth; ++i)
            if (v0 + i * threads < end) x[i] = body[v0 + i * threads];
#pragma unroll
        for (int i = 0; i < kLogpDepth; ++i) {
            const int v = v0 + i * threads;
            if (v >= end) continue;
            Vec<T, V> y, o;
            y.raw = x[i];
#pragma unroll
            for (int j = 0; j < V; ++j) o.set(j, value(y.get(j)));
            S* to = dz + head + static_cast<int64_t>(v) * V;
            if (words) {
                __stcs(reinterpret_cast<uint4*>(to), o.raw);
            } else {
                const S* f = reinterpret_cast<const S*>(&o.raw);
#pragma unroll
                for (int j = 0; j < V; ++j) to[j] = f[j];
            }
        }
    }
    if (mine) dz[token] = from_float<T>(at_token(token_z));
}

// The gradient: q_v = 2^(z_v c - m) / rest from the forward call's log-sum, so every element by itself:
//   dz_v = 2^u (k0 + k1 u) with u = z_v c - m,  and dlogp / tau more at the token.
template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) logp_backward_kernel(const LogProbs a) {
    using S = typename T::storage;
    constexpr int V = 16 / sizeof(S);
    __shared__ float fold[THREADS / 32];
    const int tid = threadIdx.x;
    grid_dependency_wait();
    grid_dependency_launch();
    // last row first: what the forward call read last may still be in L2
    const int64_t block = blockIdx.x / a.parts, row = a.rows - 1 - block;
    const int part = blockIdx.x - static_cast<int>(block) * a.parts;
    const S* z = static_cast<const S*>(a.z) + row * a.z_stride;
    S* dz = static_cast<S*>(a.dz) + row * a.dz_stride;
    const RowPart<T> at_row(z, a, part);
    const int head = at_row.head, begin = at_row.begin, end = at_row.end, loose = at_row.loose;
    const float loose_z = loose >= 0 ? to_float<T>(z[loose]) : 0.f;
    const uint4* body = reinterpret_cast<const uint4*>(z + head);
    uint4 x[kLogpDepth];
    auto fetch = [&](int v0) {
#pragma unroll
        for (int i = 0; i < kLogpDepth; ++i)
            if (v0 + i * THREADS < end) x[i] = body[v0 + i * THREADS];
    };
    fetch(begin + tid);
    const int64_t given = a.token64 ? static_cast<const long long*>(a.token)[row] : static_cast<const int*>(a.token)[row];
    const int token = given >= 0 && given < a.V ? static_cast<int>(given) : -1;
    const float g = token >= 0 ? a.dlogp[row] / a.tau : 0.f, h = a.dentropy ? a.dentropy[row] / a.tau : 0.f;
    const float lse = a.lse_in[row], entropy = a.dentropy ? a.entropy_in[row] : 0.f;
    // The forward call's m + log2 s again, which was found with the same rounded c as z c here: times log2(e) itself, since with tau c in its
    // place c's rounding would move every q of the row by up to 2^-24 lse.
    const double exponent = static_cast<double>(lse) * (1. / kLn2Exact);
    const float m = static_cast<float>(exponent), rest = static_cast<float>(exponent - m);
    // log q = ln 2 (u - rest)
    const float scale = exp2_fast(-rest), k0 = -(g + h * (entropy - rest * kLn2)) * scale, k1 = -h * kLn2 * scale;
    if (!(fabsf(lse) <= kLogpKept<T>)) {
        // Each block walks over all of the row for the sum, so only as many of them work on it as run at the same time
        // (2048 x 131072 fp32, all rows like this: eight 3.37 ms, one 0.93; rows within kLogpKept 0.32).
        if (part < a.walkers) {
            LogProbs walk = a;
            walk.parts = a.walkers;
            walk.per = a.walk;
            const RowPart<T> share(z, walk, part);
            gradient_of_differences<T>(a, z, dz, head, share.begin, share.end, share.loose, token, g, h, entropy, lse, fold);
        }
        return;
    }
    auto value = [&](float v) {
        const float u = fmaf(v < kLogpFloor ? kLogpFloor : v, a.c, -m);
        return exp2_fast(u) * fmaf(k1, u, k0);
    };
    // the token's element has its thread add what is due there
    auto at_token = [&](float v) { return value(v) + g; };
    const bool in_body = token >= head + begin * V && token < head + end * V;
    const bool mine = in_body && ((token - head) / V - begin) % THREADS == tid;
    const float token_z = mine ? to_float<T>(z[token]) : 0.f;
    if (loose >= 0) dz[loose] = from_float<T>(loose == token ? at_token(loose_z) : value(loose_z));
    const bool words = ((reinterpret_cast<uintptr_t>(dz) ^ reinterpret_cast<uintptr_t>(z)) & 15) == 0;
    for (int v0 = begin + tid; v0 < end; v0 += THREADS * kLogpDepth) {
        if (v0 != begin + tid) fetch(v0);
#pragma unroll
        for (int i = 0; i < kLogpDepth; ++i) {
            const int v = v0 + i * THREADS;
            if (v >= end) continue;
            Vec<T, V> o;
            raise_to_floor<T>(x[i]);
            Vec<T, V> y;
            y.raw = x[i];
#pragma unroll
            for (int q = 0; q < V / 2; ++q) {
                const pair_t u = fma2(vec_pair<T, V>(y, q), twice(a.c), twice(-m));
                float lo, hi;
                split_pair(u, lo, hi);
                set_vec_pair<T, V>(o, q, mul2(make_pair(exp2_fast(lo), exp2_fast(hi)), fma2(u, twice(k1), twice(k0))));
            }
            S* to = dz + head + static_cast<int64_t>(v) * V;
            if (words) {
                __stcs(reinterpret_cast<uint4*>(to), o.raw);
            } else {
                const S* f = reinterpret_cast<const S*>(&o.raw);
#pragma unroll
                for (int j = 0; j < V; ++j) to[j] = f[j];
            }
        }
    }
    if (mine) dz[token] = from_float<T>(at_token(token_z));
}

}  // namespace bns
