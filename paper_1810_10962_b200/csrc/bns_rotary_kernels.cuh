// Root-mean-square norm of every head of queries and keys, with the rotation by position in the same pass, and its gradient.
//
//   rstd = 1 / sqrt(mean(x^2) + eps);  n = x rstd;  y = R_p (n w): pairs (a, b) of the first `rotary` elements become
//   (a cos - b sin, b cos + a sin) with the angles of position p, the others stay
//   gradient: d = R_p^T dy;  dw = sum over positions and heads of d n;  dx = rstd (w d - n mean(w d n))
//
// Bound by HBM: a head is read once, written once.  A thread holds one vector of a pair's first elements and the matching
// vector of its second elements, so a rotation needs no neighbour; 1 to 32 lanes share a head (eight for 128 bf16 elements)
// and join their sums by shuffles.  A warp takes one position and makes rounds over its heads, so that position, angles and
// weights are fetched once and multiplied into one factor for an element and one for its partner; the next rounds' loads are
// in flight meanwhile, and all arithmetic goes two elements an instruction.  rstd is not kept: the gradient has x at hand and
// takes both sums in one exchange.
//
// 8192 positions of 32 + 8 heads of 128 bf16: forward 30 us (5.6 TB/s; four heads a warp without rounds, scalar arithmetic and
// factors 45), gradient 54 us (4.7 TB/s).  The gradient is held back by its registers: angles, weights, the weight's sums and
// two heads' elements leave 16 warps an SM.  Of what was tried against that, each against 58 us at the time, smaller vectors
// (63), the sums in shared memory (58) and copies ahead through shared memory (54, but 145 instead of 114 where neighbours are
// paired and 107 instead of 89 in fp32) did not pay.
#pragma once

#include "bns_elements.cuh"

namespace bns {

constexpr int kRotaryWarps = 4;      // of a block

struct HeadRows {
    const void* x;
    const void* dy;                  // backward, dense like y
    const float* weight;
    void* y;                         // or dx: dense [batch][length][heads][D]
    int64_t batch_stride, position_stride, head_stride;
    int heads, rounds, chunks;       // rounds of a warp, warps along the heads
    int blocks;                      // backward: of each chunk
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

// The V pairs of values of a unit: (2 q, 2 q + 1) of its first vector, then of its second one; single elements are one pair.
template <typename T, int V>
struct HeadUnit {
    using S = typename T::storage;
    using raw_t = typename Vec<T, V>::raw_t;
    Vec<T, V> a, b;
    __device__ __forceinline__ HeadUnit() { a.raw = b.raw = raw_t{}; }      // what is never loaded is 0
    __device__ __forceinline__ void load(const S* row, int first, int second) {
        if (first >= 0) a.raw = __ldcs(reinterpret_cast<const raw_t*>(row + first));
        if (second >= 0) b.raw = __ldcs(reinterpret_cast<const raw_t*>(row + second));
    }
    __device__ __forceinline__ void unpack(pair_t (&p)[V]) const {
        if constexpr (V == 1) {
            p[0] = make_pair(a.get(0), b.get(0));
        } else {
#pragma unroll
            for (int q = 0; q < V / 2; ++q) {
                p[q] = vec_pair<T, V>(a, q);
                p[V / 2 + q] = vec_pair<T, V>(b, q);
            }
        }
    }
    static __device__ __forceinline__ void zero(S* row, int first, int second) {
        if (first >= 0) *reinterpret_cast<raw_t*>(row + first) = raw_t{};
        if (second >= 0) *reinterpret_cast<raw_t*>(row + second) = raw_t{};
    }
    static __device__ __forceinline__ void store(S* row, int first, int second, const pair_t (&p)[V]) {
        Vec<T, V> a, b;
        if constexpr (V == 1) {
            float lo, hi;
            split_pair(p[0], lo, hi);
            a.set(0, lo);
            b.set(0, hi);
        } else {
#pragma unroll
            for (int q = 0; q < V / 2; ++q) {
                set_vec_pair<T, V>(a, q, p[q]);
                set_vec_pair<T, V>(b, q, p[V / 2 + q]);
            }
        }
        if (first >= 0) a.store(row + first);
        if (second >= 0) b.store(row + second);
    }
};

// What a rotation adds to pair q: the pair of the other vector, or its own two values exchanged.
template <int V, bool INTERLEAVED>
__device__ __forceinline__ pair_t partner(const pair_t (&p)[V], int q) {
    if constexpr (INTERLEAVED || V == 1) {
        float lo, hi;
        split_pair(p[q], lo, hi);
        return make_pair(hi, lo);
    } else {
        return p[(q + V / 2) % V];
    }
}

__device__ __forceinline__ float sum_of(pair_t p) {
    float lo, hi;
    split_pair(p, lo, hi);
    return lo + hi;
}

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

__device__ __forceinline__ int64_t position_of(const HeadNorm& a, int64_t token) {
    return a.position64 ? static_cast<const long long*>(a.position)[token] : static_cast<const int*>(a.position)[token];
}
__device__ __forceinline__ int64_t offset_of(const HeadNorm& a, const HeadRows& r, int64_t token) {
    if (!a.batched) return token * r.position_stride;
    const int64_t b = token / a.length;
    return b * r.batch_stride + (token - b * a.length) * r.position_stride;
}

// Pair by pair the factors of a value itself (cos) and of its partner (sin with the partner's sign, SIGN = -1: turning back).
template <int NU, int V, bool INTERLEAVED>
__device__ __forceinline__ void load_angles(const HeadNorm& a, int64_t p, const int (&angle)[NU], pair_t (&own)[NU][V], pair_t (&other)[NU][V], float sign, bool words) {
#pragma unroll
    for (int i = 0; i < NU; ++i) {
        float c[V], s[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            c[j] = 1.f;
            s[j] = 0.f;
        }
        if (angle[i] >= 0) {
            load_floats<V>(a.cos + p * (a.R / 2) + angle[i], c, words);
            load_floats<V>(a.sin + p * (a.R / 2) + angle[i], s, words);
        }
#pragma unroll
        for (int q = 0; q < V; ++q) {
            if constexpr (INTERLEAVED || V == 1) {
                own[i][q] = make_pair(c[q], c[q]);
                other[i][q] = make_pair(-sign * s[q], sign * s[q]);
            } else {
                const int j = 2 * q % V;
                own[i][q] = make_pair(c[j], c[j + 1]);
                other[i][q] = 2 * q < V ? make_pair(-sign * s[j], -sign * s[j + 1]) : make_pair(sign * s[j], sign * s[j + 1]);
            }
        }
    }
}
template <int NU, int V>
__device__ __forceinline__ void load_head_weights(const float* w, const int (&first)[NU], const int (&second)[NU], pair_t (&p)[NU][V], bool words) {
#pragma unroll
    for (int i = 0; i < NU; ++i) {
        float f[2][V] = {};
        if (first[i] >= 0) load_floats<V>(w + first[i], f[0], words);
        if (second[i] >= 0) load_floats<V>(w + second[i], f[1], words);
#pragma unroll
        for (int q = 0; q < V; ++q) p[i][q] = make_pair(f[2 * q / V][2 * q % V], f[(2 * q + 1) / V][(2 * q + 1) % V]);
    }
}

// A warp's rounds over its heads: round i takes heads first + i * slots, of this lane's slot.
struct HeadRounds {
    int first, count, own;       // rounds of the warp, of the slot
    __device__ __forceinline__ HeadRounds(const HeadRows& r, int chunk, int slot, int slots) {
        first = chunk * r.rounds * slots + slot;
        count = min(r.rounds, (r.heads - first + slot + slots - 1) / slots);
        own = min(count, (r.heads - first + slots - 1) / slots);
    }
};

// A warp: one position, some rounds of queries (blockIdx.y < q.chunks) or keys, DEPTH of them in flight.
template <typename T, int V, int NU, int DEPTH, bool INTERLEAVED>
__global__ void __launch_bounds__(kRotaryWarps * 32, NU == 1 ? 6 : 1) head_norm_forward_kernel(const __grid_constant__ HeadNorm a, int lanes, int words) {
    using S = typename T::storage;
    grid_dependency_wait();
    grid_dependency_launch();
    const int64_t token = static_cast<int64_t>(blockIdx.x) * kRotaryWarps + (threadIdx.x >> 5);
    if (token >= a.tokens) return;
    const bool of_q = static_cast<int>(blockIdx.y) < a.q.chunks;
    const HeadRows& r = of_q ? a.q : a.k;
    const int lane = threadIdx.x & (lanes - 1), slot = (threadIdx.x & 31) / lanes, slots = 32 / lanes;
    const int64_t p = position_of(a, token);
    const HeadPiece<T, V, NU> at(a, lane, lanes);
    const HeadRounds rounds(r, of_q ? blockIdx.y : blockIdx.y - a.q.chunks, slot, slots);
    S* y = static_cast<S*>(r.y) + (token * r.heads + rounds.first) * a.D;
    const int64_t y_step = static_cast<int64_t>(slots) * a.D;
    if (p < 0 || p >= a.positions) {         // padding
        for (int round = 0; round < rounds.own; ++round, y += y_step)
#pragma unroll
            for (int i = 0; i < NU; ++i) HeadUnit<T, V>::zero(y, at.first[i], at.second[i]);
        return;
    }
    const S* x = static_cast<const S*>(r.x) + offset_of(a, r, token) + rounds.first * r.head_stride;
    const int64_t x_step = slots * r.head_stride;
    HeadUnit<T, V> ring[DEPTH][NU];
    int ahead = 0;
    auto fetch = [&](HeadUnit<T, V> (&to)[NU]) {
        if (ahead++ < rounds.own) {
#pragma unroll
            for (int i = 0; i < NU; ++i) to[i].load(x, at.first[i], at.second[i]);
            x += x_step;
        }
    };
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) fetch(ring[d]);
    // of a value itself and of its partner: cos and sin times the weights that these have
    pair_t own[NU][V], other[NU][V], w[NU][V];
    load_angles<NU, V, INTERLEAVED>(a, p, at.angle, own, other, 1.f, words & 1);
    load_head_weights<NU, V>(r.weight, at.first, at.second, w, words & 2);
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
        for (int q = 0; q < V; ++q) {
            own[i][q] = mul2(own[i][q], w[i][q]);
            other[i][q] = mul2(other[i][q], partner<V, INTERLEAVED>(w[i], q));
        }
    for (int round0 = 0; round0 < rounds.count; round0 += DEPTH) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            if (round0 + d >= rounds.count) break;
            pair_t f[NU][V], squares = 0;
#pragma unroll
            for (int i = 0; i < NU; ++i) {
                ring[d][i].unpack(f[i]);
#pragma unroll
                for (int q = 0; q < V; ++q) squares = fma2(f[i][q], f[i][q], squares);
            }
            fetch(ring[d]);
            float sum = sum_of(squares);
            for (int o = lanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            const float rstd = rsqrtf(fmaf(sum, a.inv_D, a.eps));   // 2 ulp
            const pair_t by = make_pair(rstd, rstd);
#pragma unroll
            for (int i = 0; i < NU; ++i) {
                pair_t out[V];
#pragma unroll
                for (int q = 0; q < V; ++q) f[i][q] = mul2(f[i][q], by);
                if (at.angle[i] >= 0) {
#pragma unroll
                    for (int q = 0; q < V; ++q) out[q] = fma2(f[i][q], own[i][q], mul2(partner<V, INTERLEAVED>(f[i], q), other[i][q]));
                } else {
#pragma unroll
                    for (int q = 0; q < V; ++q) out[q] = mul2(f[i][q], own[i][q]);
                }
                if (round0 + d < rounds.own) HeadUnit<T, V>::store(y, at.first[i], at.second[i], out);
            }
            y += y_step;
        }
    }
}

// The same rounds with a grid stride over the positions; a block leaves its sums for the weight in a row of `partial`.
template <typename T, int V, int NU, int DEPTH, bool INTERLEAVED>
__global__ void __launch_bounds__(kRotaryWarps * 32, NU == 1 ? 4 : 1) head_norm_backward_kernel(const __grid_constant__ HeadNorm a, int lanes, int words) {
    using S = typename T::storage;
    extern __shared__ float sums[];          // [warps][D]
    grid_dependency_wait();
    grid_dependency_launch();
    // queries' and keys' chunks have blocks in proportion to their rounds
    const int of_queries = a.q.chunks * a.q.blocks, block = blockIdx.x;
    const HeadRows& r = block < of_queries ? a.q : a.k;
    const int mine_of = block < of_queries ? block : block - of_queries, chunk = mine_of / r.blocks;
    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & (lanes - 1), slot = (threadIdx.x & 31) / lanes, slots = 32 / lanes;
    const HeadPiece<T, V, NU> at(a, lane, lanes);
    const HeadRounds rounds(r, chunk, slot, slots);
    pair_t dw[NU][V] = {}, w[NU][V];
    load_head_weights<NU, V>(r.weight, at.first, at.second, w, words & 2);
    const int64_t step = static_cast<int64_t>(r.blocks) * kRotaryWarps, x_step = slots * r.head_stride, y_step = static_cast<int64_t>(slots) * a.D;
    int64_t token = static_cast<int64_t>(mine_of - chunk * r.blocks) * kRotaryWarps + warp;
    int64_t next = token < a.tokens ? position_of(a, token) : 0;
    for (; token < a.tokens; token += step) {
        const int64_t p = next, dense = (token * r.heads + rounds.first) * a.D;
        if (token + step < a.tokens) next = position_of(a, token + step);
        S* dx = static_cast<S*>(r.y) + dense;
        if (p < 0 || p >= a.positions) {         // padding
            for (int round = 0; round < rounds.own; ++round, dx += y_step)
#pragma unroll
                for (int i = 0; i < NU; ++i) HeadUnit<T, V>::zero(dx, at.first[i], at.second[i]);
            continue;
        }
        const S* x = static_cast<const S*>(r.x) + offset_of(a, r, token) + rounds.first * r.head_stride;
        const S* dy = static_cast<const S*>(r.dy) + dense;
        HeadUnit<T, V> ring[DEPTH][2][NU];
        int ahead = 0;
        auto fetch = [&](HeadUnit<T, V> (&to)[2][NU]) {
            if (ahead++ < rounds.own) {
#pragma unroll
                for (int i = 0; i < NU; ++i) {
                    to[0][i].load(x, at.first[i], at.second[i]);
                    to[1][i].load(dy, at.first[i], at.second[i]);
                }
                x += x_step;
                dy += y_step;
            }
        };
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) fetch(ring[d]);
        pair_t own[NU][V], other[NU][V];
        load_angles<NU, V, INTERLEAVED>(a, p, at.angle, own, other, -1.f, words & 1);
        for (int round0 = 0; round0 < rounds.count; round0 += DEPTH) {
#pragma unroll
            for (int h = 0; h < DEPTH; ++h) {
                if (round0 + h >= rounds.count) break;
                pair_t f[NU][V], d[NU][V], squares = 0, inner = 0;
#pragma unroll
                for (int i = 0; i < NU; ++i) {
                    pair_t g[V];
                    ring[h][0][i].unpack(f[i]);
                    ring[h][1][i].unpack(g);
#pragma unroll
                    for (int q = 0; q < V; ++q) {
                        d[i][q] = g[q];
                        if (at.angle[i] >= 0) d[i][q] = fma2(g[q], own[i][q], mul2(partner<V, INTERLEAVED>(g, q), other[i][q]));
                        squares = fma2(f[i][q], f[i][q], squares);
                        inner = fma2(mul2(f[i][q], w[i][q]), d[i][q], inner);
                    }
                }
                fetch(ring[h]);
                float sum = sum_of(squares), sum_inner = sum_of(inner);
                for (int o = lanes / 2; o > 0; o >>= 1) {
                    sum += __shfl_xor_sync(0xffffffffu, sum, o);
                    sum_inner += __shfl_xor_sync(0xffffffffu, sum_inner, o);
                }
                if (round0 + h < rounds.own) {
                    const float rstd = rsqrtf(fmaf(sum, a.inv_D, a.eps)), mean = sum_inner * rstd * a.inv_D;
                    const pair_t by = make_pair(rstd, rstd), less = make_pair(-mean, -mean);
#pragma unroll
                    for (int i = 0; i < NU; ++i) {
#pragma unroll
                        for (int q = 0; q < V; ++q) {
                            const pair_t n = mul2(f[i][q], by);
                            dw[i][q] = fma2(d[i][q], n, dw[i][q]);
                            d[i][q] = mul2(by, fma2(n, less, mul2(w[i][q], d[i][q])));
                        }
                        HeadUnit<T, V>::store(dx, at.first[i], at.second[i], d[i]);
                    }
                }
                dx += y_step;
            }
        }
    }
    // the slots of a warp, then the warps of the block, in order
    float* mine = sums + warp * a.D;
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
        for (int j = 0; j < 2 * V; ++j) {
            float lo, hi;
            split_pair(dw[i][j / 2], lo, hi);
            float v = j % 2 ? hi : lo;
            for (int o = 16; o >= lanes; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
            const int column = j < V ? at.first[i] : at.second[i];
            if (slot == 0 && column >= 0) mine[column + j % V] = v;
        }
    __syncthreads();
    float* to = a.partial + static_cast<int64_t>(blockIdx.x) * a.D;
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
