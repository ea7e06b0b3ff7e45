// Linear head + softmax cross entropy over a large vocabulary, without keeping the logits.
//
//   z = x W^T;  lse_t = log sum_v exp z_tv;  loss_t = lse_t - z_{t, y_t}
//   G_tv = dloss_t (exp(z_tv - lse_t) - [v = y_t]);  dx = G W;  dW = G^T x
//
// Three matrix products on the tensor cores (2 T V D operations each, the logits twice: once per direction), all
// run by one persistent kernel with different operand layouts and epilogues:
//   LSE   z tile -> per row maximum and sum of exponentials of the tile's columns, and the target's logit
//   GRAD  z tile -> G tile, bf16, into a buffer that holds one piece of the vocabulary
//   OUT   dx and dW tiles -> the gradient in the tensor's type, or fp32 partial sums
//
// One CTA per SM; a tile is 128 x 256 with its fp32 accumulator in tensor memory (two of them, so that the epilogue of
// one tile runs under the products of the next).  Warp 0 feeds a ring of shared-memory stages by TMA (64 elements of
// K a stage, 128-byte swizzle), warp 1 issues tcgen05.mma, warps 4-7 read the accumulator back.  Operands are bf16; either
// may be stored with K or with its other dimension contiguous (G^T, and W and x as the right-hand sides of the
// gradients), so no tensor is transposed.  fp32 tensors are split into three bf16 terms (8 + 8 + 8 bits) and the six
// products that matter in fp32 are added up in the same accumulator, smallest first.
//
// Every wait is bounded: one that runs out is counted, and the block ends without touching memory further.
#pragma once

#include <cuda.h>

#include "bns.h"
#include "bns_elements.cuh"

namespace bns {

constexpr int kHeadM = 128, kHeadN = 256, kHeadK = 64;   // tile, and K per stage
constexpr int kHeadStages = 4;
constexpr int kHeadThreads = 256;
constexpr unsigned kHeadStageA = kHeadM * kHeadK * 2, kHeadStageB = kHeadN * kHeadK * 2;
constexpr unsigned kHeadSmem = kHeadStages * (kHeadStageA + kHeadStageB) + 1024;
constexpr int kHeadRaster = 16;        // row tiles that are swept together, so that their operand stays in L2
constexpr unsigned kHeadPolls = 1u << 22;
constexpr float kHeadLog2e = 1.4426950408889634f, kHeadLn2 = 0.6931471805599453f;

// Bounded waits that ran out since the library was loaded.
__device__ unsigned g_head_timeouts;

// ------------------------------------------------------------------------------------ PTX wrappers
namespace head {

__device__ __forceinline__ unsigned smem(const void* p) { return static_cast<unsigned>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void barrier_init(unsigned bar, unsigned arrivals) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(arrivals) : "memory");
}
__device__ __forceinline__ void barrier_expect(unsigned bar, unsigned bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void barrier_arrive(unsigned bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool barrier_try(unsigned bar, unsigned parity) {
    unsigned done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    return done != 0;
}
// False once this wait, or another one of the block, has run out.
__device__ __forceinline__ bool wait(unsigned bar, unsigned parity, volatile int* gave_up) {
    for (unsigned i = 0; i < kHeadPolls; ++i) {
        if (barrier_try(bar, parity)) return true;
        if ((i & 255) == 255 && *gave_up) return false;
    }
    *gave_up = 1;
    atomicAdd(&g_head_timeouts, 1u);
    return false;
}
__device__ __forceinline__ void tma_load(unsigned dst, const CUtensorMap* map, int x, int y, unsigned bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void commit(unsigned bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void mma(unsigned d, uint64_t a, uint64_t b, unsigned idesc, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(static_cast<unsigned>(accumulate))
        : "memory");
}
__device__ __forceinline__ void load32(unsigned address, float (&f)[32]) {
    __syncwarp();
    unsigned* r = reinterpret_cast<unsigned*>(f);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
          "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
          "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(address));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Shared-memory matrix descriptor, 128-byte swizzle.  K contiguous: rows of 128 bytes, groups of eight rows 1024
// bytes apart.  Other dimension contiguous: 64 elements of it by eight of K are 1024 bytes, the next eight of K
// follow, the next 64 elements are one TMA box (64 x 64, 8192 bytes) away.
template <bool K_CONTIGUOUS>
__device__ __forceinline__ uint64_t descriptor(unsigned address) {
    constexpr uint64_t lead = K_CONTIGUOUS ? 1 : 8192 >> 4, stride = 1024 >> 4;
    return static_cast<uint64_t>((address & 0x3ffff) >> 4) | (lead << 16) | (stride << 32) | (uint64_t{1} << 46) |
           (uint64_t{2} << 61);
}
// What 16 elements of K add to the descriptor's address field.
template <bool K_CONTIGUOUS>
__device__ __forceinline__ constexpr uint64_t descriptor_step() {
    return K_CONTIGUOUS ? 32 >> 4 : 2048 >> 4;
}

__device__ __forceinline__ int64_t load_index(const void* p, int64_t i, int is64) {
    return is64 ? static_cast<const long long*>(p)[i] : static_cast<const int*>(p)[i];
}

}  // namespace head

// ------------------------------------------------------------------------------------ the product
struct HeadGemm {
    int M, N;                    // rows and columns of the product that exist
    int tiles_m, tiles_n, splits;
    int k_blocks, pairs;         // stages of K per pair of terms; 1 pair, or 6 for fp32 tensors
    int a_pitch, b_pitch;        // elements from one bf16 term of a row to the next
    // LSE and GRAD
    const void* target;          // [M]
    int target64;
    int first;                   // vocabulary index of column 0
    int V;
    float2* partial;             // LSE: [tiles_n][M] maximum (base 2) and sum
    float* target_logit;         // LSE: [M]
    unsigned* status;            // LSE: cleared here, set by the kernel that joins the partial sums
    const float *lse, *dloss;    // GRAD: [M]
    unsigned short* G;           // GRAD: [M][terms][pitch]
    int64_t G_stride;
    int G_pitch, terms;
    // OUT
    void* out;                   // the tensor's type
    int64_t out_stride;
    float* sums;                 // [splits][M][N] fp32, or NULL: `out` is written directly
    int add;                     // add what `sums` holds
    int last;                    // with sums: write `out` (one split only)
};

enum { kHeadLse = 0, kHeadGrad = 1, kHeadOut = 2 };

// Which terms a pair multiplies, smallest products first (the single pair of bf16 tensors is the last one).
__device__ __forceinline__ void head_pair(int pair, int pairs, int& a, int& b) {
    const int p = pair + 6 - pairs;
    a = (0x201100 >> (4 * (5 - p))) & 15;
    b = (0x021010 >> (4 * (5 - p))) & 15;
}

struct HeadTile {
    int m, n, split, k0, k1;
    __device__ __forceinline__ HeadTile(const HeadGemm& g, int id) {
        const int per = g.tiles_m * g.tiles_n;
        split = id / per;
        const int r = id - split * per;
        const int band = r / (kHeadRaster * g.tiles_n), first = band * kHeadRaster;
        const int rows = min(kHeadRaster, g.tiles_m - first), q = r - first * g.tiles_n;
        m = first + q % rows;
        n = q / rows;
        const int total = g.k_blocks * g.pairs;
        k0 = static_cast<int>(static_cast<int64_t>(total) * split / g.splits);
        k1 = static_cast<int>(static_cast<int64_t>(total) * (split + 1) / g.splits);
    }
};

template <int KIND, bool A_K, bool B_K, typename T>
__global__ void __launch_bounds__(kHeadThreads, 1)
    head_gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const HeadGemm g) {
    extern __shared__ unsigned char raw[];
    __shared__ __align__(8) uint64_t bars[2 * kHeadStages + 5];
    __shared__ unsigned tmem_base;
    __shared__ int gave_up;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned ring = (head::smem(raw) + 1023) & ~1023u;
    const unsigned full = head::smem(bars), empty = full + 8 * kHeadStages, ready = empty + 8 * kHeadStages,
                   drained = ready + 16, flush = drained + 16;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kHeadStages; ++s) {
            head::barrier_init(full + 8 * s, 1);
            head::barrier_init(empty + 8 * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            head::barrier_init(ready + 8 * b, 1);
            head::barrier_init(drained + 8 * b, 128);
        }
        head::barrier_init(flush, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        gave_up = 0;
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_b) : "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(head::smem(&tmem_base)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    head::fence_before();
    __syncthreads();
    head::fence_after();
    const unsigned tmem = tmem_base;
    grid_dependency_wait();
    grid_dependency_launch();

    const int tiles = g.tiles_m * g.tiles_n * g.splits;
    int issued = 0;   // stages that thread 0 has asked TMA to fill
    if (warp == 0) {
        if (lane == 0) {
            int it = 0;
            bool ok = true;
            for (int id = blockIdx.x; ok && id < tiles; id += gridDim.x) {
                const HeadTile t(g, id);
                for (int k = t.k0; k < t.k1; ++k, ++it) {
                    const int s = it % kHeadStages;
                    if (it >= kHeadStages && !(ok = head::wait(empty + 8 * s, (it / kHeadStages - 1) & 1, &gave_up))) break;
                    const unsigned bar = full + 8 * s, sa = ring + s * (kHeadStageA + kHeadStageB), sb = sa + kHeadStageA;
                    head::barrier_expect(bar, kHeadStageA + kHeadStageB);
                    int ta, tb;
                    const int pair = k / g.k_blocks, kk = (k - pair * g.k_blocks) * kHeadK;
                    head_pair(pair, g.pairs, ta, tb);
                    if constexpr (A_K) {
                        head::tma_load(sa, &map_a, ta * g.a_pitch + kk, t.m * kHeadM, bar);
                    } else {
#pragma unroll
                        for (int q = 0; q < kHeadM / 64; ++q)
                            head::tma_load(sa + q * 8192, &map_a, ta * g.a_pitch + t.m * kHeadM + q * 64, kk, bar);
                    }
                    if constexpr (B_K) {
                        head::tma_load(sb, &map_b, tb * g.b_pitch + kk, t.n * kHeadN, bar);
                    } else {
#pragma unroll
                        for (int q = 0; q < kHeadN / 64; ++q)
                            head::tma_load(sb + q * 8192, &map_b, tb * g.b_pitch + t.n * kHeadN + q * 64, kk, bar);
                    }
                }
            }
            issued = it;
        }
    } else if (warp == 1) {
        if (lane == 0) {
            constexpr unsigned idesc = (1u << 4) | (1u << 7) | (1u << 10) | (A_K ? 0u : 1u << 15) | (B_K ? 0u : 1u << 16) |
                                       ((kHeadN >> 3) << 17) | ((kHeadM >> 4) << 24);
            int it = 0, n = 0;
            bool ok = true;
            for (int id = blockIdx.x; ok && id < tiles; id += gridDim.x, ++n) {
                const HeadTile t(g, id);
                const int buffer = n & 1;
                if (n >= 2 && !(ok = head::wait(drained + 8 * buffer, (n / 2 - 1) & 1, &gave_up))) break;
                head::fence_after();
                const unsigned d = tmem + buffer * kHeadN;
                for (int k = t.k0; k < t.k1; ++k, ++it) {
                    const int s = it % kHeadStages;
                    if (!(ok = head::wait(full + 8 * s, (it / kHeadStages) & 1, &gave_up))) break;
                    head::fence_after();
                    const unsigned sa = ring + s * (kHeadStageA + kHeadStageB);
                    const uint64_t da = head::descriptor<A_K>(sa), db = head::descriptor<B_K>(sa + kHeadStageA);
#pragma unroll
                    for (int q = 0; q < kHeadK / 16; ++q)
                        head::mma(d, da + q * head::descriptor_step<A_K>(), db + q * head::descriptor_step<B_K>(), idesc,
                                  k > t.k0 || q > 0);
                    head::commit(empty + 8 * s);
                }
                if (!ok) break;
                head::commit(ready + 8 * buffer);
            }
        }
    } else if (warp >= 4) {
        using S = typename T::storage;
        const int slot = warp & 3;
        if (KIND == kHeadLse && blockIdx.x == 0 && threadIdx.x == 128 && g.status) *g.status = 0;
        int n = 0;
        for (int id = blockIdx.x; id < tiles; id += gridDim.x, ++n) {
            const HeadTile t(g, id);
            const int buffer = n & 1;
            if (!__all_sync(0xffffffffu, head::wait(ready + 8 * buffer, (n / 2) & 1, &gave_up))) break;
            head::fence_after();
            const unsigned src = tmem + buffer * kHeadN + (static_cast<unsigned>(slot * 32) << 16);
            const int row = t.m * kHeadM + slot * 32 + lane, column0 = t.n * kHeadN;
            const bool in = row < g.M;
            const int columns = min(kHeadN, g.N - column0);     // that exist
            if constexpr (KIND == kHeadLse) {
                const float inf = __int_as_float(0x7f800000);
                const int64_t y = in ? head::load_index(g.target, row, g.target64) : -1;
                const int64_t mine = y - g.first - column0;     // the target's place in this tile, if it is in it
                float m = -inf, s = 0.f;
                for (int c = 0; c < columns; c += 32) {
                    float f[32];
                    head::load32(src + c, f);
                    if (columns - c < 32) {
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (c + j >= columns) f[j] = -inf;
                    }
                    float top = f[0];
#pragma unroll
                    for (int j = 1; j < 32; ++j) top = fmaxf(top, f[j]);
                    top = fmaxf(top * kHeadLog2e, m);
                    const float ref = top == -inf ? 0.f : top;
                    s *= head::exp2_fast(m - ref);
#pragma unroll
                    for (int j = 0; j < 32; ++j) s += head::exp2_fast(fmaf(f[j], kHeadLog2e, -ref));
                    m = top;
                    if (mine >= c && mine < c + 32 && mine < columns) {
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (mine == c + j) g.target_logit[row] = f[j];
                    }
                }
                if (in) g.partial[static_cast<int64_t>(t.n) * g.M + row] = make_float2(m, s);
            } else if constexpr (KIND == kHeadGrad) {
                const int64_t y = in ? head::load_index(g.target, row, g.target64) : -1;
                const int64_t mine = y - g.first - column0;
                const bool counts = y >= 0 && y < g.V;
                const float lse = counts ? g.lse[row] : 0.f, scale = counts ? g.dloss[row] : 0.f;
                // lse log2(e) = shift + rest, log2(e) being the same fp32 number as in z log2(e), so that only the
                // difference z - lse feels its rounding; rest goes into the factor
                const float shift = lse * kHeadLog2e;
                const float factor = scale * head::exp2_fast(-fmaf(lse, kHeadLog2e, -shift));
                const int padded = (columns + kHeadK - 1) / kHeadK * kHeadK;   // zeros up to whole stages of K
                for (int c = 0; c < padded; c += 32) {
                    float f[32];
                    head::load32(src + c, f);
                    if (in) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            f[j] = counts && c + j < columns ? head::exp2_fast(fmaf(f[j], kHeadLog2e, -shift)) * factor : 0.f;
                            if (mine == c + j && c + j < columns) f[j] -= scale;
                        }
                        unsigned short* to = g.G + row * g.G_stride + column0 + c;
                        for (int term = 0; term < g.terms; ++term) {
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                Vec<BF16, 8> o;
                                float e[8];
#pragma unroll
                                for (int j = 0; j < 8; ++j) e[j] = f[q * 8 + j];
                                o.pack(e);
                                o.store(to + term * static_cast<int64_t>(g.G_pitch) + q * 8);
                                o.unpack(e);
#pragma unroll
                                for (int j = 0; j < 8; ++j) f[q * 8 + j] -= e[j];   // what the term leaves for the next
                            }
                        }
                    }
                }
            } else {
                for (int c = 0; c < columns; c += 32) {
                    float f[32];
                    head::load32(src + c, f);
                    const int left = columns - c;
                    float* p = g.sums + (static_cast<int64_t>(t.split) * g.M + row) * g.N + column0 + c;
                    if (in && g.sums) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            if (j < left) {
                                if (g.add) f[j] += p[j];
                                if (!g.last) p[j] = f[j];
                            }
                        }
                    }
                    if (in && (!g.sums || g.last)) {
                        S* to = static_cast<S*>(g.out) + row * g.out_stride + column0 + c;
                        constexpr int V = 16 / sizeof(S);
                        if (left >= 32 && (reinterpret_cast<uintptr_t>(to) & 15) == 0) {
#pragma unroll
                            for (int q = 0; q < 32 / V; ++q) {
                                Vec<T, V> o;
                                float e[V];
#pragma unroll
                                for (int j = 0; j < V; ++j) e[j] = f[q * V + j];
                                o.pack(e);
                                o.store(to + q * V);
                            }
                        } else {
#pragma unroll
                            for (int j = 0; j < 32; ++j)
                                if (j < left) to[j] = from_float<T>(f[j]);
                        }
                    }
                }
            }
            head::fence_before();
            head::barrier_arrive(drained + 8 * buffer);
        }
    }
    __syncthreads();
    if (gave_up) {
        // a block that gave up leaves only when its copies have landed and its products have ended
        if (threadIdx.x == 0)
            for (int i = max(0, issued - kHeadStages); i < issued; ++i)
                for (unsigned n = 0; n < kHeadPolls && !head::barrier_try(full + 8 * (i % kHeadStages), (i / kHeadStages) & 1); ++n) {
                }
        if (threadIdx.x == 32) {
            head::commit(flush);
            for (unsigned n = 0; n < kHeadPolls && !head::barrier_try(flush, 0); ++n) {
            }
        }
        __syncthreads();
    }
    if (warp == 2) {
        head::fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
}

// ------------------------------------------------------------------------------------ around the products
// Rows into bf16 terms: the first is the value rounded, the next what that leaves, and so on; each term's row is padded
// with zeros to `pitch` elements.  One term lays out bf16 rows whose stride TMA cannot take.
template <typename T>
__global__ void __launch_bounds__(256) head_terms_kernel(const void* src, int64_t stride, int rows, int D, int terms, int pitch,
                                                         unsigned short* dst) {
    grid_dependency_wait();
    grid_dependency_launch();
    const int64_t total = static_cast<int64_t>(rows) * pitch;
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < total; i += gridDim.x * 256ll) {
        const int64_t row = i / pitch;
        const int column = static_cast<int>(i - row * pitch);
        float v = column < D ? to_float<T>(static_cast<const typename T::storage*>(src)[row * stride + column]) : 0.f;
        for (int t = 0; t < terms; ++t) {
            const unsigned short b = from_float<BF16>(v);
            dst[(row * terms + t) * pitch + column] = b;
            v -= to_float<BF16>(b);
        }
    }
}

// Joins the tiles' maxima and sums of a row: 32 rows a block, eight threads a row, in a fixed order.
__global__ void __launch_bounds__(256) head_join_kernel(const float2* partial, int tiles, int rows, const float* target_logit,
                                                        const void* target, int target64, int V, float* loss, float* lse,
                                                        unsigned* status) {
    __shared__ float2 fold[8][32];
    grid_dependency_wait();
    grid_dependency_launch();
    const float inf = __int_as_float(0x7f800000);
    const int row = blockIdx.x * 32 + (threadIdx.x & 31), part = threadIdx.x >> 5;
    auto join = [&](float2 a, float2 b) {
        const float m = fmaxf(a.x, b.x), ref = m == -inf ? 0.f : m;
        return make_float2(m, a.y * head::exp2_fast(a.x - ref) + b.y * head::exp2_fast(b.x - ref));
    };
    float2 v = make_float2(-inf, 0.f);
    if (row < rows)
        for (int t = part; t < tiles; t += 8) v = join(v, partial[static_cast<int64_t>(t) * rows + row]);
    fold[part][threadIdx.x & 31] = v;
    __syncthreads();
    if (part || row >= rows) return;
    for (int q = 1; q < 8; ++q) v = join(v, fold[q][threadIdx.x]);
    const float rest = log2f(v.y);
    lse[row] = (v.x + rest) * kHeadLn2;
    const int64_t y = head::load_index(target, row, target64);
    // the difference to the largest first: where the model is sure, lse and the target's logit are nearly equal
    loss[row] = y >= 0 && y < V ? (fmaf(-target_logit[row], kHeadLog2e, v.x) + rest) * kHeadLn2 : 0.f;
    if (y >= V) atomicOr(status, BNS_FLAG_BAD_TARGET);
}

// Adds up the splits of a product, in order, and rounds once.
template <typename T>
__global__ void __launch_bounds__(256) head_sum_kernel(const float* sums, int splits, int rows, int columns, void* out,
                                                       int64_t stride) {
    grid_dependency_wait();
    grid_dependency_launch();
    const int64_t total = static_cast<int64_t>(rows) * columns;
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < total; i += gridDim.x * 256ll) {
        float v = 0.f;
        for (int s = 0; s < splits; ++s) v += sums[s * total + i];
        const int64_t row = i / columns;
        static_cast<typename T::storage*>(out)[row * stride + (i - row * columns)] = from_float<T>(v);
    }
}

}  // namespace bns
