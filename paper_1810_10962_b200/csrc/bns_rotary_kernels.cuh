// Root-mean-square norm of every head of queries and keys, with the rotation by position in the same pass, and its gradient.
//
//   rstd = 1 / sqrt(mean(x^2) + eps);  n = x rstd;  y = R_p (n w): pairs (a, b) of the first `rotary` elements become
//   (a cos - b sin, b cos + a sin) with the angles of position p, the others stay
//   gradient: d = R_p^T dy;  dw = sum over positions and heads of d n;  dx = rstd (w d - n mean(w d n))
//
// Bound by HBM: a head is read once, written once.  A thread holds one vector of a pair's first elements and the matching
// vector of its second elements, so a rotation needs no neighbour; 1 to 32 lanes share a head (eight for 128 bf16 elements)
// and join their sums by shuffles.  A warp takes one position and several of its heads, so that position, angles and weights
// are fetched once for all of them.  rstd is not kept: the gradient has x at hand and takes both sums in one exchange.
#pragma once

#include "bns_elements.cuh"

namespace bns {

constexpr int kRotaryWarps = 8;      // of a block

struct HeadRows {
    const void* x;
    const void* dy;                  // backward, dense like y
    const float* weight;
    void* y;                         // or dx: dense [batch][length][heads][D]
    int64_t batch_stride, position_stride, head_stride;
    int heads, chunks;               // blocks along the heads
};

struct HeadNorm {
    HeadRows q, k;
    const float *cos, *sin;          // [positions][R / 2]
    const void* position;            // [batch][length]
    float* partial;                  // backward: [blocks of q and k][D]
    int64_t tokens;
    int length, D, R, positions, position64, interleaved, batched;
    float eps, inv_D;
};

// A thread's share of a head: NU units of two vectors.
template <typename T, int V, int NU>
struct HeadPiece {
    using S = typename T::storage;
    int first[NU], second[NU], angle[NU];   // columns of the vectors (-1: none), first pair (-1: not turned)
    __device__ __forceinline__ HeadPiece(const HeadNorm& a, int lane, int lanes) {
        const int turned = a.R / 2 / V;
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int u = lane + i * lanes;
            if (u < turned) {
                first[i] = a.interleaved ? 2 * u * V : u * V;
                second[i] = a.interleaved ? first[i] + V : a.R / 2 + u * V;
                angle[i] = u * V;
            } else {
                const int at = a.R + 2 * (u - turned) * V;
                first[i] = at < a.D ? at : -1;
                second[i] = at + V < a.D ? at + V : -1;
                angle[i] = -1;
            }
        }
    }
};

template <typename T, int V>
struct HeadUnit {
    using S = typename T::storage;
    Vec<T, V> a, b;
    __device__ __forceinline__ void load(const S* row, int first, int second) {
        if (first >= 0) a.raw = __ldcs(reinterpret_cast<const typename Vec<T, V>::raw_t*>(row + first));
        if (second >= 0) b.raw = __ldcs(reinterpret_cast<const typename Vec<T, V>::raw_t*>(row + second));
    }
    // elements that are not there are 0
    __device__ __forceinline__ void unpack(int first, int second, float (&f)[2 * V]) const {
        float lo[V], hi[V];
        a.unpack(lo);
        b.unpack(hi);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            f[j] = first >= 0 ? lo[j] : 0.f;
            f[V + j] = second >= 0 ? hi[j] : 0.f;
        }
    }
    __device__ __forceinline__ void store(S* row, int first, int second, const float (&f)[2 * V]) {
        float lo[V], hi[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            lo[j] = f[j];
            hi[j] = f[V + j];
        }
        a.pack(lo);
        b.pack(hi);
        if (first >= 0) a.store(row + first);
        if (second >= 0) b.store(row + second);
    }
};

// V floats, in words where their place allows it.
template <int V>
__device__ __forceinline__ void load_floats(const float* p, float (&f)[V], bool words) {
    if (V >= 4 && words) {
#pragma unroll
        for (int j = 0; j + 4 <= V; j += 4) {
            const float4 q = __ldg(reinterpret_cast<const float4*>(p + j));
            f[j] = q.x;
            f[j + 1] = q.y;
            f[j + 2] = q.z;
            f[j + 3] = q.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = __ldg(p + j);
    }
}

// Turns the pairs of a unit: (f_j, f_{V+j}), or neighbours.  `sign` = -1 turns back.
template <int V>
__device__ __forceinline__ void turn(float (&f)[2 * V], const float (&c)[V], const float (&s)[V], bool interleaved, float sign) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const float si = s[j] * sign;
        if (interleaved) {
            const float x = f[2 * j], y = f[2 * j + 1];
            f[2 * j] = fmaf(x, c[j], -y * si);
            f[2 * j + 1] = fmaf(y, c[j], x * si);
        } else {
            const float x = f[j], y = f[V + j];
            f[j] = fmaf(x, c[j], -y * si);
            f[V + j] = fmaf(y, c[j], x * si);
        }
    }
}

__device__ __forceinline__ int64_t position_of(const HeadNorm& a, int64_t token) {
    return a.position64 ? static_cast<const long long*>(a.position)[token] : static_cast<const int*>(a.position)[token];
}
__device__ __forceinline__ int64_t offset_of(const HeadNorm& a, const HeadRows& r, int64_t token) {
    if (!a.batched) return token * r.position_stride;
    const int64_t b = token / a.length;
    return b * r.batch_stride + (token - b * a.length) * r.position_stride;
}

template <int NU, int V>
__device__ __forceinline__ void load_angles(const HeadNorm& a, int64_t p, const int (&angle)[NU], float (&c)[NU][V], float (&s)[NU][V], bool words) {
#pragma unroll
    for (int i = 0; i < NU; ++i) {
        if (angle[i] >= 0) {
            load_floats<V>(a.cos + p * (a.R / 2) + angle[i], c[i], words);
            load_floats<V>(a.sin + p * (a.R / 2) + angle[i], s[i], words);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                c[i][j] = 1.f;
                s[i][j] = 0.f;
            }
        }
    }
}
template <int NU, int V>
__device__ __forceinline__ void load_head_weights(const float* w, const int (&first)[NU], const int (&second)[NU], float (&f)[NU][2 * V], bool words) {
#pragma unroll
    for (int i = 0; i < NU; ++i) {
        float lo[V] = {}, hi[V] = {};
        if (first[i] >= 0) load_floats<V>(w + first[i], lo, words);
        if (second[i] >= 0) load_floats<V>(w + second[i], hi, words);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            f[i][j] = lo[j];
            f[i][V + j] = hi[j];
        }
    }
}

// A warp: one position, heads chunk * slots * UH + slot + slots * i of queries (blockIdx.y < q.chunks) or keys.
template <typename T, int V, int NU, int UH>
__global__ void __launch_bounds__(kRotaryWarps * 32) head_norm_forward_kernel(const __grid_constant__ HeadNorm a, int lanes, int words) {
    using S = typename T::storage;
    grid_dependency_wait();
    grid_dependency_launch();
    const int64_t token = static_cast<int64_t>(blockIdx.x) * kRotaryWarps + (threadIdx.x >> 5);
    if (token >= a.tokens) return;
    const bool of_q = static_cast<int>(blockIdx.y) < a.q.chunks;
    const HeadRows& r = of_q ? a.q : a.k;
    const int chunk = of_q ? blockIdx.y : blockIdx.y - a.q.chunks;
    const int lane = threadIdx.x & (lanes - 1), slot = (threadIdx.x & 31) / lanes, slots = 32 / lanes;
    const int64_t p = position_of(a, token);
    const HeadPiece<T, V, NU> at(a, lane, lanes);
    const S* x = static_cast<const S*>(r.x) + offset_of(a, r, token);
    S* y = static_cast<S*>(r.y) + token * r.heads * a.D;
    const int head0 = chunk * slots * UH + slot;
    HeadUnit<T, V> in[UH][NU];
#pragma unroll
    for (int h = 0; h < UH; ++h)
#pragma unroll
        for (int i = 0; i < NU; ++i)
            if (head0 + h * slots < r.heads) in[h][i].load(x + (head0 + h * slots) * r.head_stride, at.first[i], at.second[i]);
    const bool known = p >= 0 && p < a.positions;
    float c[NU][V], s[NU][V], w[NU][2 * V];
    load_angles<NU, V>(a, known ? p : 0, at.angle, c, s, words & 1);
    load_head_weights<NU, V>(r.weight, at.first, at.second, w, words & 2);
#pragma unroll
    for (int h = 0; h < UH; ++h) {
        float f[NU][2 * V], squares = 0.f;
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            in[h][i].unpack(at.first[i], at.second[i], f[i]);
#pragma unroll
            for (int j = 0; j < 2 * V; ++j) squares = fmaf(f[i][j], f[i][j], squares);
        }
        for (int o = lanes / 2; o > 0; o >>= 1) squares += __shfl_xor_sync(0xffffffffu, squares, o);
        const float rstd = rsqrtf(fmaf(squares, a.inv_D, a.eps));   // 2 ulp
        if (head0 + h * slots >= r.heads) continue;
        S* to = y + static_cast<int64_t>(head0 + h * slots) * a.D;
#pragma unroll
        for (int i = 0; i < NU; ++i) {
#pragma unroll
            for (int j = 0; j < 2 * V; ++j) f[i][j] = known ? f[i][j] * rstd * w[i][j] : 0.f;
            if (at.angle[i] >= 0 && known) turn<V>(f[i], c[i], s[i], a.interleaved, 1.f);
            in[h][i].store(to, at.first[i], at.second[i], f[i]);
        }
    }
}

// The same walk with a grid stride over the positions; a block leaves its sums for the weight in a row of `partial`.
template <typename T, int V, int NU, int UH>
__global__ void __launch_bounds__(kRotaryWarps * 32) head_norm_backward_kernel(const __grid_constant__ HeadNorm a, int lanes, int words) {
    using S = typename T::storage;
    extern __shared__ float sums[];          // [warps][D]
    grid_dependency_wait();
    grid_dependency_launch();
    const bool of_q = static_cast<int>(blockIdx.y) < a.q.chunks;
    const HeadRows& r = of_q ? a.q : a.k;
    const int chunk = of_q ? blockIdx.y : blockIdx.y - a.q.chunks;
    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & (lanes - 1), slot = (threadIdx.x & 31) / lanes, slots = 32 / lanes;
    const HeadPiece<T, V, NU> at(a, lane, lanes);
    const int head0 = chunk * slots * UH + slot;
    float dw[NU][2 * V] = {}, w[NU][2 * V];
    load_head_weights<NU, V>(r.weight, at.first, at.second, w, words & 2);
    for (int64_t token = static_cast<int64_t>(blockIdx.x) * kRotaryWarps + warp; token < a.tokens; token += static_cast<int64_t>(gridDim.x) * kRotaryWarps) {
        const int64_t p = position_of(a, token);
        const S* x = static_cast<const S*>(r.x) + offset_of(a, r, token);
        const int64_t dense = token * r.heads * a.D;
        const S* dy = static_cast<const S*>(r.dy) + dense;
        S* dx = static_cast<S*>(r.y) + dense;
        HeadUnit<T, V> in[UH][NU], up[UH][NU];
#pragma unroll
        for (int h = 0; h < UH; ++h)
#pragma unroll
            for (int i = 0; i < NU; ++i)
                if (head0 + h * slots < r.heads) {
                    in[h][i].load(x + (head0 + h * slots) * r.head_stride, at.first[i], at.second[i]);
                    up[h][i].load(dy + static_cast<int64_t>(head0 + h * slots) * a.D, at.first[i], at.second[i]);
                }
        const bool known = p >= 0 && p < a.positions;
        float c[NU][V], s[NU][V];
        load_angles<NU, V>(a, known ? p : 0, at.angle, c, s, words & 1);
#pragma unroll
        for (int h = 0; h < UH; ++h) {
            const bool there = head0 + h * slots < r.heads;
            float f[NU][2 * V], d[NU][2 * V], squares = 0.f, inner = 0.f;
#pragma unroll
            for (int i = 0; i < NU; ++i) {
                in[h][i].unpack(at.first[i], at.second[i], f[i]);
                up[h][i].unpack(at.first[i], at.second[i], d[i]);
                if (at.angle[i] >= 0) turn<V>(d[i], c[i], s[i], a.interleaved, -1.f);
#pragma unroll
                for (int j = 0; j < 2 * V; ++j) {
                    squares = fmaf(f[i][j], f[i][j], squares);
                    inner = fmaf(f[i][j] * w[i][j], d[i][j], inner);
                }
            }
            for (int o = lanes / 2; o > 0; o >>= 1) {
                squares += __shfl_xor_sync(0xffffffffu, squares, o);
                inner += __shfl_xor_sync(0xffffffffu, inner, o);
            }
            if (!there) continue;
            const float rstd = rsqrtf(fmaf(squares, a.inv_D, a.eps)), mean = inner * rstd * a.inv_D;
            S* to = dx + static_cast<int64_t>(head0 + h * slots) * a.D;
#pragma unroll
            for (int i = 0; i < NU; ++i) {
#pragma unroll
                for (int j = 0; j < 2 * V; ++j) {
                    const float n = f[i][j] * rstd;
                    if (known) dw[i][j] = fmaf(d[i][j], n, dw[i][j]);
                    d[i][j] = known ? rstd * fmaf(-n, mean, w[i][j] * d[i][j]) : 0.f;
                }
                in[h][i].store(to, at.first[i], at.second[i], d[i]);
            }
        }
    }
    // the slots of a warp, then the warps of the block, in order
    float* mine = sums + warp * a.D;
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
        for (int j = 0; j < 2 * V; ++j) {
            float v = dw[i][j];
            for (int o = 16; o >= lanes; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
            const int column = j < V ? at.first[i] : at.second[i];
            if (slot == 0 && column >= 0) mine[column + j % V] = v;
        }
    __syncthreads();
    float* to = a.partial + (static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x) * a.D;
    for (int i = threadIdx.x; i < a.D; i += blockDim.x) {
        float v = 0.f;
        for (int k = 0; k < kRotaryWarps; ++k) v += sums[k * a.D + i];
        to[i] = v;
    }
}

// Gradients of both weights (blockIdx.y): 32 columns a block, 32 threads a column over the blocks' sums, joined in a fixed order.
__global__ void __launch_bounds__(1024) head_weight_kernel(const float* partial, int q_rows, int k_rows, int D, float* dq_weight, float* dk_weight) {
    __shared__ float fold[32][33];
    grid_dependency_wait();
    grid_dependency_launch();
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5, column = blockIdx.x * 32 + lane;
    const int first = blockIdx.y ? q_rows : 0, rows = blockIdx.y ? k_rows : q_rows;
    float* out = blockIdx.y ? dk_weight : dq_weight;
    float sum = 0.f;
    if (column < D) {
#pragma unroll 8
        for (int b = part; b < rows; b += 32) sum += partial[static_cast<int64_t>(first + b) * D + column];
    }
    fold[part][lane] = sum;
    __syncthreads();
    sum = fold[lane][part];     // now a warp has a column
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0 && blockIdx.x * 32 + part < D) out[blockIdx.x * 32 + part] = sum;
}

}  // namespace bns
