// The linear head's loss and gradient for few rows of x in fp32, on the fp32 pipes.
//
//   z = x W^T;  (maximum, sum of exponentials) of every row;  G_tv = dloss_t (exp(z_tv - lse_t) - [v = y_t])
//   dx = G W;  dW = G^T x
//
// An element of W takes part in T products a pass.  For the tensor cores W would first be laid out as fp16 terms, which moves
// some 12 more bytes an element and pass, for tiles of 128 rows that are mostly empty; up to 32 rows (forward) and 16
// (backward) the fp32 pipes are through sooner.
//
//   logits    a warp takes R rows of W; its lanes stride along the width, with x in shared memory and R T sums in
//             registers, joined over the lanes by halves (the lanes end up with different sums).  Four rows of W share
//             what is read of x: 16 bytes a lane take the time of 16 multiply-adds
//   products  a thread takes C columns of x, W, dx and dW; x and dx's sums stay in registers while it walks down rows of W
//             (each read once, each row of dW written once); G comes through shared memory (from L1 the products took
//             1.5 times as long at 16 rows).  Blocks leave partial sums of dx, which a third kernel joins in order
//
// 32768 x 1024: forward 34 us for one row (134 MB at 3.9 TB/s), 40 for 4, 62 for 16, 87 for 32, where it is bound by the
// multiply-adds and shared memory (tensor cores: 115 to 122); forward and backward 115, 130 and 210 us for 1, 4 and 16
// rows (tensor cores: 309; at 32 rows 316 against 309, so that this is not done).
#pragma once

#include "bns_head_kernels.cuh"

namespace bns {

constexpr int kFewRows = 32, kFewRowsBackward = 16;      // at most
constexpr size_t kFewSharedMost = size_t{216} << 10;     // of x
constexpr int kFewProductThreads = 256, kFewTile = 32;   // of the products: threads, rows of W whose G is in shared memory
constexpr int kFewLane = 4;                              // columns of a lane, or of a thread of the products

template <int ROWS>
struct FewShape {
    static constexpr int kThreads = ROWS > 16 ? 256 : 512;        // 128 sums a thread take twice the registers
    static constexpr int kR = ROWS <= 2 ? 8 : 4;
};

struct HeadFew {
    const float* x;
    const float* w;
    const void* target;
    const float* lse;      // gradient
    const float* dloss;
    float2* partial;       // [blocks][T] maximum (base 2) and sum
    float* target_logit;
    unsigned* status;      // cleared here, or (gradient) written
    float* G;              // [V][ROWS]
    float* sums;           // [chunks][T][D]
    float* dx;
    float* dw;
    int64_t x_stride, w_stride;
    int target64, T, V, D;
    int pitch;             // of x in shared memory: whole chunks where W's rows are not made of words
    int chunks, per;       // products: rows of W a block
    int groups;            // products: blocks across the width
};

// Sums over the warp's lanes of N values each: lane l ends with those of index l N / 32 ... (N >= 32), or of index l N / 32.
template <int N, int O>
__device__ __forceinline__ void few_sum(float* v, int lane) {
    if constexpr (O > 0) {
        if constexpr (N > 1) {
            constexpr int H = N / 2;
            const bool upper = lane & O;
#pragma unroll
            for (int i = 0; i < H; ++i) {
                const float send = upper ? v[i] : v[i + H], keep = upper ? v[i + H] : v[i];
                v[i] = keep + __shfl_xor_sync(0xffffffffu, send, O);
            }
            few_sum<H, O / 2>(v, lane);
        } else {
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], O);
            few_sum<1, O / 2>(v, lane);
        }
    }
}

// WORDS: a lane's four columns are one 16-byte word; else they lie 32 apart.
template <int ROWS, bool WORDS, bool GRAD>
__global__ void __launch_bounds__(FewShape<ROWS>::kThreads, 1) head_few_logits_kernel(const HeadFew a) {
    using Form = FewShape<ROWS>;
    constexpr int R = Form::kR, N = R * ROWS, PER = N > 32 ? N / 32 : 1, SAME = N < 32 ? 32 / N : 1, kWarps = Form::kThreads / 32;
    extern __shared__ __align__(16) float few_x[];
    __shared__ float2 fold[kWarps][N];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const float inf = __int_as_float(0x7f800000);
    grid_dependency_wait();
    grid_dependency_launch();
    if (!GRAD && blockIdx.x == 0 && tid == 0) *a.status = 0;
    for (int t = 0; t < ROWS; ++t)
        for (int d = tid; d < a.pitch; d += Form::kThreads)
            few_x[t * a.pitch + d] = t < a.T && d < a.D ? a.x[t * a.x_stride + d] : 0.f;
    // what this lane's sums belong to
    const int first = lane * N / 32;
    int64_t y[PER];
    float lse[PER], weight[PER];
    float2 st[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int t = (first + i) % ROWS;
        y[i] = t < a.T ? head::load_index(a.target, t, a.target64) : -1;
        st[i] = make_float2(-inf, 0.f);
        if constexpr (GRAD) {
            const bool counts = y[i] >= 0 && y[i] < a.V;
            lse[i] = counts ? a.lse[t] : 0.f;
            weight[i] = counts ? a.dloss[t] : 0.f;
        }
    }
    if (GRAD && blockIdx.x == 0 && warp == 0) {       // a warp's lanes have all of the targets
        bool past = false;
#pragma unroll
        for (int i = 0; i < PER; ++i) past |= y[i] >= a.V;
        past = __any_sync(0xffffffffu, past);
        if (lane == 0) *a.status = past ? BNS_FLAG_BAD_TARGET : 0;
    }
    __syncthreads();
    const int step = gridDim.x * kWarps * R, chunks = (a.D + 32 * kFewLane - 1) / (32 * kFewLane);
    const int own = WORDS ? lane * kFewLane : lane;
    float now[R][kFewLane], next[R][kFewLane];
    auto fetch = [&](float(&to)[R][kFewLane], int v0, int c) {
        const int d = c * 32 * kFewLane + own;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float* from = a.w + (v0 + r) * a.w_stride + d;
            const bool row = v0 + r < a.V;
            if constexpr (WORDS) {
                const float4 v = row && d < a.D ? *reinterpret_cast<const float4*>(from) : make_float4(0.f, 0.f, 0.f, 0.f);
                to[r][0] = v.x, to[r][1] = v.y, to[r][2] = v.z, to[r][3] = v.w;
            } else {
#pragma unroll
                for (int j = 0; j < kFewLane; ++j) to[r][j] = row && d + 32 * j < a.D ? from[32 * j] : 0.f;
            }
        }
    };
    int v0 = (warp * gridDim.x + blockIdx.x) * R;      // few rows of W are spread over the SMs first
    if (v0 < a.V) fetch(now, v0, 0);
    for (; v0 < a.V; v0 += step) {
        float z[N];
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = 0.f;
        for (int c = 0; c < chunks; ++c) {
            if (c + 1 < chunks)
                fetch(next, v0, c + 1);
            else if (v0 + step < a.V)
                fetch(next, v0 + step, 0);
            const int d = c * 32 * kFewLane + own;
            if (d < a.pitch) {
#pragma unroll
                for (int t = 0; t < ROWS; ++t) {
                    float x[kFewLane];
                    const float* from = few_x + t * a.pitch + d;
                    if constexpr (WORDS) {
                        const float4 v = *reinterpret_cast<const float4*>(from);
                        x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
                    } else {
#pragma unroll
                        for (int j = 0; j < kFewLane; ++j) x[j] = from[32 * j];
                    }
#pragma unroll
                    for (int r = 0; r < R; ++r)
#pragma unroll
                        for (int j = 0; j < kFewLane; ++j) z[r * ROWS + t] = fmaf(now[r][j], x[j], z[r * ROWS + t]);
                }
            }
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int j = 0; j < kFewLane; ++j) now[r][j] = next[r][j];
        }
        few_sum<N, 16>(z, lane);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int v = v0 + (first + i) / ROWS, t = (first + i) % ROWS;
            if (v >= a.V) continue;
            if constexpr (GRAD) {
                // a row that does not count has weight 0, and may hold anything
                const float q = exp2_fast((z[i] - lse[i]) * kHeadLog2e) - (v == y[i] ? 1.f : 0.f);
                a.G[static_cast<int64_t>(v) * ROWS + t] = y[i] >= 0 && y[i] < a.V ? weight[i] * q : 0.f;
            } else {
                // the reference is the rounded product z log2(e), the exponents are differences to just that number: its
                // rounding, some 4e-4 at a logit of 3e4, is in the sum and so cancels when a target's logit is compared with it
                const float m = fmaxf(st[i].x, z[i] * kHeadLog2e), ref = m == -inf ? 0.f : m;
                st[i] = make_float2(m, st[i].y * exp2_fast(st[i].x - ref) + exp2_fast(fmaf(z[i], kHeadLog2e, -ref)));
                if (v == y[i] && t < a.T) a.target_logit[t] = z[i];
            }
        }
    }
    if constexpr (!GRAD) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (lane % SAME == 0) fold[warp][first + i] = st[i];
        __syncthreads();
        if (tid < a.T) {
            float m = -inf, s = 0.f;
            for (int w0 = 0; w0 < kWarps; ++w0)
                for (int r = 0; r < R; ++r) m = fmaxf(m, fold[w0][r * ROWS + tid].x);
            const float ref = m == -inf ? 0.f : m;
            for (int w0 = 0; w0 < kWarps; ++w0)
                for (int r = 0; r < R; ++r) {
                    const float2 p = fold[w0][r * ROWS + tid];
                    s += p.y * exp2_fast(p.x - ref);
                }
            a.partial[static_cast<int64_t>(blockIdx.x) * a.T + tid] = make_float2(m, s);
        }
    }
}

// WORDS: a thread's columns are one word; else they lie a block's threads apart.
template <int ROWS, bool WORDS>
__global__ void __launch_bounds__(kFewProductThreads, ROWS <= 8 ? 2 : 1) head_few_products_kernel(const HeadFew a) {
    constexpr int C = kFewLane, U = 4;      // columns, rows of W in flight
    grid_dependency_wait();
    grid_dependency_launch();
    const int chunk = blockIdx.x / a.groups, group = blockIdx.x - chunk * a.groups, threads = blockDim.x;
    const int d = group * threads * C + static_cast<int>(threadIdx.x) * (WORDS ? C : 1), apart = WORDS ? 1 : threads;
    const int begin = chunk * a.per, end = min(a.V, begin + a.per);
    float x[ROWS][C], dx[ROWS][C];
#pragma unroll
    for (int t = 0; t < ROWS; ++t)
#pragma unroll
        for (int j = 0; j < C; ++j) {
            x[t][j] = t < a.T && d + j * apart < a.D ? a.x[t * a.x_stride + d + j * apart] : 0.f;
            dx[t][j] = 0.f;
        }
    auto get = [&](const float* from, float(&to)[C]) {
        if constexpr (WORDS) {
            if (d >= a.D) return;
            Vec<F32, C> v;
            v.load(from + d);
            v.unpack(to);
        } else {
#pragma unroll
            for (int j = 0; j < C; ++j)
                if (d + j * threads < a.D) to[j] = from[d + j * threads];
        }
    };
    auto put = [&](float* to, const float(&from)[C]) {
        if constexpr (WORDS) {
            if (d >= a.D) return;
            Vec<F32, C> v;
            v.pack(from);
            v.store(to + d);
        } else {
#pragma unroll
            for (int j = 0; j < C; ++j)
                if (d + j * threads < a.D) to[d + j * threads] = from[j];
        }
    };
    float now[U][C] = {}, next[U][C] = {};
    auto fetch = [&](float(&to)[U][C], int v0) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (v0 + u < end) get(a.w + (v0 + u) * a.w_stride, to[u]);
    };
    fetch(now, begin);
    // G by tiles of rows of W through shared memory, the next tile's copies under this one's products
    __shared__ __align__(16) float tile[2][kFewTile * ROWS];
    constexpr int P = ROWS >= 4 ? 4 : ROWS;      // values a copy
    auto ask = [&](int v0, int turn) {
        const int count = min(kFewTile, end - v0) * ROWS;
        for (int at = threadIdx.x * P; at < count; at += blockDim.x * P)
            asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem_address(&tile[turn][at])),
                         "l"(a.G + static_cast<int64_t>(v0) * ROWS + at), "n"(P * 4)
                         : "memory");
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    ask(begin, 0);
    int turn = 1;
    for (int v0 = begin; v0 < end; v0 += U) {
        const int at = (v0 - begin) % kFewTile;
        if (at == 0) {
            turn ^= 1;
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            __syncthreads();        // this tile is there, and nobody reads the other
            ask(v0 + kFewTile, turn ^ 1);
        }
        fetch(next, v0 + U);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (v0 + u >= end) break;
            const float* g = tile[turn] + (at + u) * ROWS;
            float o[C] = {};
            constexpr int GV = ROWS >= 4 ? 4 : ROWS;
#pragma unroll
            for (int t0 = 0; t0 < ROWS; t0 += GV) {
                Vec<F32, GV> gv;
                gv.load(g + t0);
#pragma unroll
                for (int q = 0; q < GV; ++q)
#pragma unroll
                    for (int j = 0; j < C; ++j) {
                        dx[t0 + q][j] = fmaf(gv.get(q), now[u][j], dx[t0 + q][j]);
                        o[j] = fmaf(gv.get(q), x[t0 + q][j], o[j]);
                    }
            }
            put(a.dw + static_cast<int64_t>(v0 + u) * a.D, o);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < C; ++j) now[u][j] = next[u][j];
    }
    float* sums = a.sums + static_cast<int64_t>(chunk) * a.T * a.D;
#pragma unroll
    for (int t = 0; t < ROWS; ++t)
        if (t < a.T) put(sums + static_cast<int64_t>(t) * a.D, dx[t]);
}

// dx from the blocks' sums, in their order: 32 elements a block, eight warps on a part of the sums each.
__global__ void __launch_bounds__(256) head_few_join_kernel(const HeadFew a) {
    __shared__ float fold[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    grid_dependency_wait();
    grid_dependency_launch();
    const int64_t total = static_cast<int64_t>(a.T) * a.D, i = blockIdx.x * int64_t{32} + lane;
    float s = 0.f;
    if (i < total) {
#pragma unroll 8
        for (int c = warp; c < a.chunks; c += 8) s += a.sums[c * total + i];
    }
    fold[warp][lane] = s;
    __syncthreads();
    if (warp || i >= total) return;
    s = 0.f;
#pragma unroll
    for (int q = 0; q < 8; ++q) s += fold[q][lane];
    a.dx[i] = s;
}

}  // namespace bns
