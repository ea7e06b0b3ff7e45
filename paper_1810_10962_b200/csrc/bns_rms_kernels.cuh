// Root-mean-square norm of the rows of a [rows, D] tensor with the residual's addition, and its gradient.
//
//   s = x + residual (fp32, not rounded before it is normalised); h = s in the tensor's type
//   rstd = 1 / sqrt(mean(s^2) + eps);  y = s rstd w
//   8-bit output: a = max |y| over a group of columns, scale = a / 448 (1 where a = 0), q = e4m3(y / scale)
//   gradient at the stored h: c = mean(w dy h rstd);  dx = rstd (w dy - h rstd c) + dh;  dw = sum over rows of dy h rstd
//
// Bound by HBM: a row is read once and lives in registers (EPT elements a thread), so every tensor crosses the
// memory system once.  A block owns a row at a time and walks down the rows with a grid stride; the next row's loads are
// issued before this row's sums are joined, so that loads stay in flight across the block's barriers.  The weights are read
// from L1 for every row (they would cost as many registers as the row).  The gradient keeps its columns' sums over the rows in
// registers and leaves them once, one row of partial sums per block.
#pragma once

#include "bns_elements.cuh"

namespace bns {

constexpr int kRmsMaxThreads = 1024;
constexpr int kRmsGroup = 128;        // columns of a scale in the grouped 8-bit form

struct RmsNone {};                    // output forms of the forward kernel
struct RmsRowScale {};
struct RmsGroupScale {};

// Sum and maximum over the block in one exchange; every thread gets both.  `turn` alternates between two buffers,
// so that one barrier per row is enough.  Warps' partial results are combined in warp order by everybody.
struct BlockExchange {
    float sum[2][32];
    float top[2][32];
};

// The larger magnitude, NaN winning.
__device__ __forceinline__ float max_or_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)));
    return r;
}

// Elementwise arithmetic on a thread's vector, two elements an instruction where it has them.
template <int V>
__device__ __forceinline__ void add_to(float (&a)[V], const float (&b)[V]) {
    if constexpr (V == 1) {
        a[0] += b[0];
    } else {
#pragma unroll
        for (int j = 0; j < V; j += 2) split_pair(add2(make_pair(a[j], a[j + 1]), make_pair(b[j], b[j + 1])), a[j], a[j + 1]);
    }
}
template <int V>
__device__ __forceinline__ void multiply_by(float (&a)[V], const float (&b)[V]) {
    if constexpr (V == 1) {
        a[0] *= b[0];
    } else {
#pragma unroll
        for (int j = 0; j < V; j += 2) split_pair(mul2(make_pair(a[j], a[j + 1]), make_pair(b[j], b[j + 1])), a[j], a[j + 1]);
    }
}
template <int V>
__device__ __forceinline__ void multiply_by(float (&a)[V], float b) {
    if constexpr (V == 1) {
        a[0] *= b;
    } else {
#pragma unroll
        for (int j = 0; j < V; j += 2) split_pair(mul2(make_pair(a[j], a[j + 1]), make_pair(b, b)), a[j], a[j + 1]);
    }
}
// acc += a b: two partial sums where V allows it
template <int V>
__device__ __forceinline__ void add_products(float (&acc)[2], const float (&a)[V], const float (&b)[V]) {
    if constexpr (V == 1) {
        acc[0] = fmaf(a[0], b[0], acc[0]);
    } else {
#pragma unroll
        for (int j = 0; j < V; j += 2)
            split_pair(fma2(make_pair(a[j], a[j + 1]), make_pair(b[j], b[j + 1]), make_pair(acc[0], acc[1])), acc[0], acc[1]);
    }
}
template <int V>
__device__ __forceinline__ float top_of_vector(const float (&a)[V]) {
    float m = fabsf(a[0]);
#pragma unroll
    for (int j = 1; j < V; ++j) m = max_or_nan(m, a[j]);
    return m;
}

template <bool TOP>
__device__ __forceinline__ void block_exchange(float& sum, float& top, BlockExchange& ex, int turn) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if constexpr (TOP) top = max_or_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
    }
    const int warps = blockDim.x >> 5;
    if (warps == 1) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) {
        ex.sum[turn][warp] = sum;
        if constexpr (TOP) ex.top[turn][warp] = top;
    }
    __syncthreads();
    sum = lane < warps ? ex.sum[turn][lane] : 0.f;
    if constexpr (TOP) top = lane < warps ? ex.top[turn][lane] : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if constexpr (TOP) top = max_or_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
    }
}

__device__ __forceinline__ unsigned short e4m3_pair(float lo, float hi) {
    unsigned short r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

template <int V>
__device__ __forceinline__ void store_e4m3(uint8_t* p, const float (&f)[V]) {
    if constexpr (V == 1) {
        *p = static_cast<uint8_t>(e4m3_pair(f[0], 0.f));
    } else {
        typename RawWord<V>::type raw;
        unsigned short* half = reinterpret_cast<unsigned short*>(&raw);
#pragma unroll
        for (int j = 0; j < V / 2; ++j) half[j] = e4m3_pair(f[2 * j], f[2 * j + 1]);
        *reinterpret_cast<typename RawWord<V>::type*>(p) = raw;
    }
}

// What multiplies s w to give y / scale, from the largest |s w| of the group.  y = s rstd w, so rstd cancels in
// y / scale = s w 448 / max|s w|: the 8-bit values carry no rounding of rstd or of the scale.  A group of zeros has
// scale 1; infinities and NaN give NaN, as the formula does.  `lift` keeps 448 / max finite for groups below 2^-100, and what
// the reciprocal makes of those above 2^100 from the numbers that it takes for 0.
struct Quant {
    float a, lift, factor;
    __device__ __forceinline__ Quant(float top, float rstd) {
        const float inf = __int_as_float(0x7f800000);
        a = top * rstd;
        lift = top < 0x1p-100f ? 0x1p100f : top > 0x1p100f ? 0x1p-100f : 1.f;
        float inverse;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inverse) : "f"(top * lift));   // 1 ulp
        factor = a == 0.f ? 0.f : top < inf && a < inf ? 448.f * inverse : __int_as_float(0x7fffffff);
    }
    __device__ __forceinline__ float scale() const { return a == 0.f ? 1.f : a * (1.f / 448.f); }
    template <int V>
    __device__ __forceinline__ void apply(float (&sw)[V]) const {
        if (lift != 1.f) multiply_by<V>(sw, lift);
        multiply_by<V>(sw, factor);
    }
};

struct RmsForward {
    const void* x;
    const void* residual;  // or NULL
    const float* weight;
    void* y;               // the tensor's type, or e4m3
    float* scales;         // [rows] or [rows][ceil(D / 128)]
    void* h;               // or NULL
    float* rstd;
    int64_t rows, x_stride, residual_stride;
    int D;
    float eps, inv_D;
};

// Vectors of V elements that a thread holds.
template <int V, int EPT>
constexpr int kRmsVectors = EPT / V < 1 ? 1 : EPT / V < 8 ? EPT / V : 8;

// A thread's vectors t, t + blockDim, ... of a row.
template <typename T, int V, int NV>
struct RowPiece {
    Vec<T, V> v[NV];
    __device__ __forceinline__ void load(const typename T::storage* row, int vectors) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = threadIdx.x + i * blockDim.x;
            if (at < vectors) v[i].raw = __ldcs(reinterpret_cast<const typename Vec<T, V>::raw_t*>(row + static_cast<int64_t>(at) * V));
        }
    }
};

// V weights, in 16-byte words where WORDS says that they begin at one.
template <int V, bool WORDS>
__device__ __forceinline__ void load_weights(const float* weight, int at, float (&w)[V]) {
    if constexpr (WORDS && V >= 4) {
#pragma unroll
        for (int j = 0; j < V; j += 4) {
            const float4 q = __ldg(reinterpret_cast<const float4*>(weight + at * V + j));
            w[j] = q.x;
            w[j + 1] = q.y;
            w[j + 2] = q.z;
            w[j + 3] = q.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) w[j] = __ldg(weight + at * V + j);
    }
}

// Rows whose stride is no multiple of a vector begin at any phase.  The blocks of a launch are a multiple of V then, so
// that a block meets one phase only: the whole vectors of its rows begin at column `head`, its threads keep the same columns
// in every row, and the up to 2 V - 2 columns outside whole vectors are the first threads' extra ones.
template <typename S, int V, bool LOOSE>
struct RowPhase {
    int head = 0, vectors, extra = -1;   // extra: this thread's column outside whole vectors
    __device__ __forceinline__ RowPhase(const void* first_row, int D) {
        if constexpr (LOOSE) {
            head = min(D, static_cast<int>(((16 - (reinterpret_cast<uintptr_t>(first_row) & 15)) & 15) / sizeof(S)));
            vectors = (D - head) / V;
            const int t = threadIdx.x, tail = head + vectors * V;
            extra = t < head ? t : t >= 16 && t < 32 && tail + t - 16 < D ? tail + t - 16 : -1;
        } else {
            vectors = D / V;
        }
    }
};

template <typename T, int V, int EPT, bool LOOSE, typename OUT>
__global__ void __launch_bounds__(kRmsMaxThreads) rms_forward_kernel(const RmsForward a) {
    using S = typename T::storage;
    constexpr int NV = kRmsVectors<V, EPT>;
    constexpr bool kRow = __is_same(OUT, RmsRowScale), kGroup = __is_same(OUT, RmsGroupScale);
    static_assert(!(LOOSE && kGroup), "groups of columns begin at whole vectors");
    __shared__ BlockExchange ex;
    extern __shared__ float segment[];    // grouped form with V < 4: largest |s w| of every 32 V columns
    const int B = blockDim.x;
    const RowPhase<S, V, LOOSE> at(static_cast<const S*>(a.x) + blockIdx.x * a.x_stride, a.D);
    const int vectors = at.vectors;
    grid_dependency_wait();
    grid_dependency_launch();

    // at a phase the weights have no vectors: a thread keeps its own
    float kept[LOOSE ? NV : 1][V], extra_w = 0.f;
    if constexpr (LOOSE) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = threadIdx.x + i * B;
            if (v < vectors) load_weights<V, false>(a.weight + at.head, v, kept[i]);
        }
        if (at.extra >= 0) extra_w = a.weight[at.extra];
    }
    auto weights = [&](int i, float (&w)[V]) {
        if constexpr (LOOSE) {
#pragma unroll
            for (int j = 0; j < V; ++j) w[j] = kept[i][j];
        } else {
            load_weights<V, true>(a.weight, threadIdx.x + i * B, w);
        }
    };
    RowPiece<T, V, NV> vx, vr;
    float next_extra = 0.f;
    auto fetch = [&](int64_t row) {
        const S* x = static_cast<const S*>(a.x) + row * a.x_stride;
        const S* r = static_cast<const S*>(a.residual) + (a.residual ? row * a.residual_stride : 0);
        vx.load(x + at.head, vectors);
        if (a.residual) vr.load(r + at.head, vectors);
        if (LOOSE && at.extra >= 0) next_extra = to_float<T>(x[at.extra]) + (a.residual ? to_float<T>(r[at.extra]) : 0.f);
    };
    int turn = 0;
    if (blockIdx.x < a.rows) fetch(blockIdx.x);
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        float s[NV][V], squares[2] = {0.f, 0.f}, top = 0.f;
        const float extra = next_extra;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            vx.v[i].unpack(s[i]);
            if (a.residual) {
                float f[V];
                vr.v[i].unpack(f);
                add_to<V>(s[i], f);
            }
        }
        if (row + gridDim.x < a.rows) fetch(row + gridDim.x);
        S* h = static_cast<S*>(a.h) + row * a.D;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = threadIdx.x + i * B;
            if (v < vectors) {
                if (a.h) {
                    Vec<T, V> o;
                    o.pack(s[i]);
                    o.store(h + at.head + static_cast<int64_t>(v) * V);
                }
                if constexpr (kRow) {
                    float w[V];
                    weights(i, w);
                    multiply_by<V>(w, s[i]);
                    top = max_or_nan(top, top_of_vector<V>(w));
                }
                add_products<V>(squares, s[i], s[i]);
            }
        }
        float sum = squares[0] + squares[1];
        if (LOOSE && at.extra >= 0) {
            if (a.h) h[at.extra] = from_float<T>(extra);
            sum = fmaf(extra, extra, sum);
            if constexpr (kRow) top = max_or_nan(top, extra * extra_w);
        }
        // s w of vector i, zeros past the row's end
        auto product = [&](int i, float (&p)[V]) {
            if (threadIdx.x + i * B < vectors) {
                weights(i, p);
                multiply_by<V>(p, s[i]);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) p[j] = 0.f;
            }
        };
        if constexpr (kGroup && V < 4) {
            // a warp's 32 V columns lie inside one group: their maximum goes through shared memory
            __syncthreads();   // the previous row's readers are done
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float p[V];
                product(i, p);
                float m = top_of_vector<V>(p);
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) m = max_or_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
                if ((threadIdx.x & 31) == 0) segment[(threadIdx.x + i * B) >> 5] = m;
            }
            __syncthreads();
        }
        block_exchange<kRow>(sum, top, ex, turn);
        const float rstd = rsqrtf(fmaf(sum, a.inv_D, a.eps));   // 2 ulp
        if (threadIdx.x == 0) a.rstd[row] = rstd;
        if constexpr (!kRow && !kGroup) {
            S* y = static_cast<S*>(a.y) + row * a.D;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int v = threadIdx.x + i * B;
                if (v >= vectors) continue;
                float f[V];
                weights(i, f);
                multiply_by<V>(s[i], rstd);
                multiply_by<V>(f, s[i]);
                Vec<T, V> o;
                o.pack(f);
                o.store(y + at.head + static_cast<int64_t>(v) * V);
            }
            if (LOOSE && at.extra >= 0) y[at.extra] = from_float<T>(extra * rstd * extra_w);
        } else {
            const int groups = (a.D + kRmsGroup - 1) / kRmsGroup;
            uint8_t* q = static_cast<uint8_t*>(a.y) + row * a.D;
            const Quant of_row(top, rstd);
            if (kRow && threadIdx.x == 0) a.scales[row] = of_row.scale();
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int v = threadIdx.x + i * B;
                float p[V];
                product(i, p);
                if constexpr (kRow) {
                    of_row.template apply<V>(p);
                } else {
                    float m = 0.f;
                    if constexpr (V >= 4) {
                        m = top_of_vector<V>(p);
#pragma unroll
                        for (int o = kRmsGroup / V / 2; o > 0; o >>= 1) m = max_or_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
                    } else {
                        constexpr int kSegments = kRmsGroup / (32 * V);
                        const int first = (v >> 5) / kSegments * kSegments;
#pragma unroll
                        for (int k = 0; k < kSegments; ++k)
                            if (first + k < (vectors + 31) >> 5) m = max_or_nan(m, segment[first + k]);
                    }
                    const Quant quant(m, rstd);
                    if (v < vectors && v % (kRmsGroup / V) == 0) a.scales[row * groups + v / (kRmsGroup / V)] = quant.scale();
                    quant.template apply<V>(p);
                }
                if (v < vectors) store_e4m3<V>(q + at.head + static_cast<int64_t>(v) * V, p);
            }
            if (LOOSE && at.extra >= 0) {
                float p[1] = {extra * extra_w};
                of_row.template apply<1>(p);
                store_e4m3<1>(q + at.extra, p);
            }
        }
    }
}

// Rows wider than a block's registers: the same arithmetic in two walks over the row, the second mostly out of L2.
template <typename T, int V, typename OUT>
__global__ void __launch_bounds__(kRmsMaxThreads) rms_forward_wide_kernel(const RmsForward a) {
    using S = typename T::storage;
    constexpr bool kRow = __is_same(OUT, RmsRowScale), kGroup = __is_same(OUT, RmsGroupScale);
    __shared__ BlockExchange ex;
    grid_dependency_wait();
    grid_dependency_launch();
    const int B = blockDim.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = B >> 5;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const S* x = static_cast<const S*>(a.x) + row * a.x_stride;
        const S* r = static_cast<const S*>(a.residual) + (a.residual ? row * a.residual_stride : 0);
        auto element = [&](int i) { return to_float<T>(x[i]) + (a.residual ? to_float<T>(r[i]) : 0.f); };
        float sum = 0.f, top = 0.f;
        const int vectors = a.D / V;
        for (int v = threadIdx.x; v < vectors; v += B) {
            Vec<T, V> vx;
            float s[V];
            vx.load(x + static_cast<int64_t>(v) * V);
            vx.unpack(s);
            if (a.residual) {
                Vec<T, V> vr;
                float f[V];
                vr.load(r + static_cast<int64_t>(v) * V);
                vr.unpack(f);
#pragma unroll
                for (int j = 0; j < V; ++j) s[j] += f[j];
            }
            if (a.h) {
                Vec<T, V> o;
                o.pack(s);
                o.store(static_cast<S*>(a.h) + row * a.D + static_cast<int64_t>(v) * V);
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                sum = fmaf(s[j], s[j], sum);
                if constexpr (kRow) top = max_or_nan(top, fabsf(s[j] * a.weight[v * V + j]));
            }
        }
        block_exchange<kRow>(sum, top, ex, turn);
        const float rstd = rsqrtf(fmaf(sum, a.inv_D, a.eps));   // 2 ulp
        if (threadIdx.x == 0) a.rstd[row] = rstd;
        if constexpr (kGroup) {
            // a warp per group, four columns a lane
            const int groups = (a.D + kRmsGroup - 1) / kRmsGroup;
            for (int g = warp; g < groups; g += warps) {
                float p[4], m = 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int i = g * kRmsGroup + j * 32 + lane;
                    p[j] = i < a.D ? element(i) * a.weight[i] : 0.f;
                    m = max_or_nan(m, fabsf(p[j]));
                }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) m = max_or_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
                const Quant quant(m, rstd);
                if (lane == 0) a.scales[row * groups + g] = quant.scale();
                quant.template apply<4>(p);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int i = g * kRmsGroup + j * 32 + lane;
                    if (i < a.D)
                        static_cast<uint8_t*>(a.y)[row * a.D + i] = static_cast<uint8_t>(e4m3_pair(p[j], 0.f));
                }
            }
        } else {
            const Quant quant(top, rstd);
            if constexpr (kRow) {
                if (threadIdx.x == 0) a.scales[row] = quant.scale();
            }
            for (int v = threadIdx.x; v < vectors; v += B) {
                float f[V];
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float s = element(v * V + j), w = a.weight[v * V + j];
                    f[j] = kRow ? s * w : s * rstd * w;
                }
                if constexpr (kRow) {
                    quant.template apply<V>(f);
                    store_e4m3<V>(static_cast<uint8_t*>(a.y) + row * a.D + static_cast<int64_t>(v) * V, f);
                } else {
                    Vec<T, V> o;
                    o.pack(f);
                    o.store(static_cast<S*>(a.y) + row * a.D + static_cast<int64_t>(v) * V);
                }
            }
        }
    }
}

struct RmsBackward {
    const void *dy, *h, *dh;  // dh or NULL
    const float *weight, *rstd;
    void* dx;
    float* partial;           // [blocks][D]: a block's sums for dweight
    int64_t rows, dy_stride, h_stride, dh_stride;
    int D;
    float inv_D;
};

template <typename T, int V, int EPT, bool LOOSE>
__global__ void __launch_bounds__(kRmsMaxThreads) rms_backward_kernel(const RmsBackward a) {
    using S = typename T::storage;
    constexpr int NV = kRmsVectors<V, EPT>;
    __shared__ BlockExchange ex;
    const int B = blockDim.x;
    // last row first: its h is what the forward kernel wrote last and may still be in L2 (1 % where it directly follows)
    auto row_of = [&](int64_t step) { return a.rows - 1 - step; };
    const RowPhase<S, V, LOOSE> at(static_cast<const S*>(a.h) + row_of(blockIdx.x) * a.h_stride, a.D);
    const int vectors = at.vectors;
    grid_dependency_wait();
    grid_dependency_launch();
    float dw[NV][V], extra_dw = 0.f, extra_w = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) dw[i][j] = 0.f;
    if (LOOSE && at.extra >= 0) extra_w = a.weight[at.extra];
    // two-byte rows have the registers for dh a row ahead as well
    constexpr bool kAhead = sizeof(S) == 2 && EPT == 8;
    RowPiece<T, V, NV> vy, vh, vd, ahead;
    float next_rstd = 0.f, next_extra_y = 0.f, next_extra_h = 0.f;
    auto fetch = [&](int64_t row) {
        const S* dy = static_cast<const S*>(a.dy) + row * a.dy_stride;
        const S* h = static_cast<const S*>(a.h) + row * a.h_stride;
        vy.load(dy + at.head, vectors);
        vh.load(h + at.head, vectors);
        if (LOOSE && at.extra >= 0) {
            next_extra_y = to_float<T>(dy[at.extra]);
            next_extra_h = to_float<T>(h[at.extra]);
        }
        if (kAhead && a.dh) ahead.load(static_cast<const S*>(a.dh) + row * a.dh_stride + at.head, vectors);
        next_rstd = a.rstd[row];
    };
    int turn = 0;
    if (blockIdx.x < a.rows) fetch(row_of(blockIdx.x));
    for (int64_t step = blockIdx.x; step < a.rows; step += gridDim.x, turn ^= 1) {
        const int64_t row = row_of(step);
        const float rstd = next_rstd, extra_y = next_extra_y * extra_w, extra_xhat = next_extra_h * rstd;
        const S* dh = static_cast<const S*>(a.dh) + (a.dh ? row * a.dh_stride : 0);
        if (kAhead)
            vd = ahead;
        else if (a.dh)
            vd.load(dh + at.head, vectors);
        float inner[2] = {0.f, 0.f}, xhat[NV][V], wdy[NV][V];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = threadIdx.x + i * B;
            if (v < vectors) {
                float w[V];
                load_weights<V, !LOOSE>(a.weight + at.head, v, w);
                vy.v[i].unpack(wdy[i]);
                vh.v[i].unpack(xhat[i]);
                multiply_by<V>(xhat[i], rstd);
                if constexpr (V == 1) {
                    dw[i][0] = fmaf(wdy[i][0], xhat[i][0], dw[i][0]);
                } else {
#pragma unroll
                    for (int j = 0; j < V; j += 2)
                        split_pair(fma2(make_pair(wdy[i][j], wdy[i][j + 1]), make_pair(xhat[i][j], xhat[i][j + 1]),
                                        make_pair(dw[i][j], dw[i][j + 1])), dw[i][j], dw[i][j + 1]);
                }
                multiply_by<V>(wdy[i], w);
                add_products<V>(inner, wdy[i], xhat[i]);
            }
        }
        float sum = inner[0] + inner[1], none = 0.f;
        if (LOOSE && at.extra >= 0) {
            extra_dw = fmaf(next_extra_y, extra_xhat, extra_dw);
            sum = fmaf(extra_y, extra_xhat, sum);
        }
        if (step + gridDim.x < a.rows) fetch(row_of(step + gridDim.x));
        block_exchange<false>(sum, none, ex, turn);
        const float c = sum * a.inv_D;
        S* dx = static_cast<S*>(a.dx) + row * a.D;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = threadIdx.x + i * B;
            if (v >= vectors) continue;
            multiply_by<V>(xhat[i], -c);
            add_to<V>(wdy[i], xhat[i]);
            multiply_by<V>(wdy[i], rstd);
            if (a.dh) {
                float fd[V];
                vd.v[i].unpack(fd);
                add_to<V>(wdy[i], fd);
            }
            Vec<T, V> o;
            o.pack(wdy[i]);
            o.store(dx + at.head + static_cast<int64_t>(v) * V);
        }
        if (LOOSE && at.extra >= 0) {
            float f = rstd * fmaf(-extra_xhat, c, extra_y);
            if (a.dh) f += to_float<T>(dh[at.extra]);
            dx[at.extra] = from_float<T>(f);
        }
    }
    float* p = a.partial + static_cast<int64_t>(blockIdx.x) * a.D;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = threadIdx.x + i * B;
        if (v >= vectors) continue;
#pragma unroll
        for (int j = 0; j < V; ++j) p[at.head + v * V + j] = dw[i][j];
    }
    if (LOOSE && at.extra >= 0) p[at.extra] = extra_dw;
}

// Rows wider than a block's registers.  The block's sums for dweight stay in its own row of `partial`, which only
// the thread that owns the column touches.
template <typename T>
__global__ void __launch_bounds__(kRmsMaxThreads) rms_backward_wide_kernel(const RmsBackward a) {
    using S = typename T::storage;
    __shared__ BlockExchange ex;
    grid_dependency_wait();
    grid_dependency_launch();
    const int B = blockDim.x;
    float* p = a.partial + static_cast<int64_t>(blockIdx.x) * a.D;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const S* dy = static_cast<const S*>(a.dy) + row * a.dy_stride;
        const S* h = static_cast<const S*>(a.h) + row * a.h_stride;
        const S* dh = static_cast<const S*>(a.dh) + (a.dh ? row * a.dh_stride : 0);
        const float rstd = a.rstd[row];
        const bool first = row == blockIdx.x;
        float sum = 0.f, none = 0.f;
        for (int i = threadIdx.x; i < a.D; i += B) {
            const float fy = to_float<T>(dy[i]), xhat = to_float<T>(h[i]) * rstd;
            p[i] = fmaf(fy, xhat, first ? 0.f : p[i]);
            sum = fmaf(a.weight[i] * fy, xhat, sum);
        }
        block_exchange<false>(sum, none, ex, turn);
        const float c = sum * a.inv_D;
        for (int i = threadIdx.x; i < a.D; i += B) {
            const float fy = to_float<T>(dy[i]), xhat = to_float<T>(h[i]) * rstd;
            float f = rstd * fmaf(-xhat, c, a.weight[i] * fy);
            if (a.dh) f += to_float<T>(dh[i]);
            static_cast<S*>(a.dx)[row * a.D + i] = from_float<T>(f);
        }
    }
}

// dweight: 32 columns a block, 32 threads a column over the blocks' sums, joined in a fixed order.
__global__ void __launch_bounds__(1024) rms_dweight_kernel(const float* partial, int blocks, int D, float* dweight) {
    __shared__ float fold[32][33];
    grid_dependency_wait();
    grid_dependency_launch();
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5, column = blockIdx.x * 32 + lane;
    float sum = 0.f;
    if (column < D) {
#pragma unroll 8
        for (int b = part; b < blocks; b += 32) sum += partial[static_cast<int64_t>(b) * D + column];
    }
    fold[part][lane] = sum;
    __syncthreads();
    sum = fold[lane][part];     // now a warp has a column
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0 && blockIdx.x * 32 + part < D) dweight[blockIdx.x * 32 + part] = sum;
}

}  // namespace bns
