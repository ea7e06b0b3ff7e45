// Linear head + softmax cross entropy over a large vocabulary, without keeping the logits.
//
//   z = x W^T;  lse_t = log sum_v exp z_tv;  loss_t = lse_t - z_{t, y_t}
//   G_tv = dloss_t (exp(z_tv - lse_t) - [v = y_t]);  dx = G W;  dW = G^T x
//
// Three matrix products on the tensor cores (2 T V D operations each, the logits twice: once per direction), all
// run by one persistent kernel with different operand layouts and epilogues:
//   LSE   z tile -> per row maximum and sum of exponentials of the tile's columns, and the target's logit
//   GRAD  z tile -> G tile, bf16, into a buffer that holds one piece of the vocabulary, a tile's 256 columns together
//         (with whole rows of G instead, whose 64 KB strides put each row of a box of G^T in another page, the product
//         G^T x ran at two thirds of the tensor cores' cycles instead of four fifths)
//   OUT   dx and dW tiles -> the gradient in the tensor's type, or fp32 partial sums
// bf16 tensors have a G of bf16: both operands of a product have one type, and a second term for the rest would double the time of dx
// and dW.  It costs bits: dx and dW are 0.0019 of their norm from 64 bits at 4096 x 131072 x 4096, where their own rounding alone
// makes 0.0017; 0.0020 at 24 rows.
//
// A CTA pair (two SMs) owns a 256 x 256 tile: each CTA keeps 128 rows of it in its tensor memory and half of either
// operand's stage in its shared memory, so that a stage's bytes per product are half of what two single CTAs would
// move.  Products with at most 128 rows run the same kernel with single CTAs (128 x 256).  Warp 0 feeds a ring of stages
// by TMA (64 elements of K, 128-byte swizzle), warp 1 of the first CTA issues tcgen05.mma, warps 4-11 read the
// accumulator back, 128 columns of a row a thread; the accumulator is double buffered.  Operands are bf16; either may be
// stored with K or with its other dimension contiguous (G^T, and W and x as the right-hand sides of the gradients),
// so no tensor is transposed.  fp32 tensors are split into two fp16 terms (11 + 11 bits): scaled by a power of two that
// brings the tensor's largest value to 2^13, high = fp16(v), low = fp16((v - high) 2^11), so that the low term keeps its bits
// down to 2^-38 of the largest value; the products high low and low high are added up first and scaled by 2^-11, then
// high high (the fourth is below 2^-22 of the result).  Three bf16 terms need six products for the same accuracy.
//
// The tensor core truncates as it accumulates: after n steps of 16 a sum has lost some n 2^-25 of itself, always towards
// zero.  Where the result is an fp32 number (the logits, everything of fp32 tensors) the sum is therefore
// taken in segments of K, which the epilogue's threads add up in registers, rounding to nearest: 512 elements for bf16
// (256 cost 9 % of the time, 307 -> 334 us at 2048 x 50257 x 2048, for half of an error of 3e-7), 128 where a CTA works
// alone (few rows, whose errors do not average out: at 4 x 3187 x 1120 the loss is 3e-7 off instead of 8e-7; 24 x 32768 x
// 1024 takes 25 us either way, 128 x 50000 x 4096 96 instead of 90), 256 for the high terms of fp32 (at 512 the loss is
// 1e-6 off, at 256 4e-7), 4096 for products with a low term, which count 2^-11.
// The gradient takes its logits in the segments of the statistics, so that it meets the very numbers that the log-sum was made
// of: with one sum over a width of 4096 a logit of 60 is 5e-4 lower, and a row that is sure of its target got a gradient of that
// size at it (4096 x 131072 x 4096, forward and backward: 13.6 ms instead of 13.4).
//
// Every wait is bounded: one that runs out is counted, and the block ends without touching memory further.
#pragma once

#include <cuda.h>
#include <cuda_fp16.h>

#include "bns.h"
#include "bns_async.cuh"

namespace bns {

constexpr int kHeadM = 128, kHeadN = 256, kHeadK = 64;   // rows of a CTA, columns of a tile, K per stage
constexpr int kHeadSegment = 8, kHeadSegmentFew = 2, kHeadSegmentHigh = 4, kHeadSegmentLow = 64;   // stages of K per segment
constexpr int kHeadThreads = 384;

// Narrow tiles of the products with the logits, for few rows and few columns: 64 columns, and half of A's stage.
constexpr int kHeadNarrow = 64, kHeadNarrowRows = 64;

// Ring of a CTA that works alone (CTAS = 1) or as half of a pair (2) on tiles of N columns.
template <int CTAS, int N>
struct HeadRing {
    static constexpr bool kNarrow = N == kHeadNarrow;
    static constexpr int kStages = kNarrow ? 10 : CTAS == 2 ? 6 : 4;
    static constexpr int kRows = kNarrow ? kHeadNarrowRows : kHeadM;   // of A's stage; the products read 128 all the same, what
                                                                       // lies there ends in rows that do not exist
    static constexpr int kColumns = N / CTAS;            // of B in this CTA's stage
    static constexpr unsigned kStageA = kRows * kHeadK * 2, kStageB = kColumns * kHeadK * 2, kStage = kStageA + kStageB;
    static constexpr unsigned kStaging = 8 * 32 * 128;   // 32 rows of 32 fp32 values for each warp of the epilogue
    static constexpr unsigned kSmem = kStages * kStage + kStaging + 1024;
};
// Row tiles that are swept together, so that their operand stays in L2 (2048 x 50257 x 2048 forward 314 us, 326 with four, 314 with 64;
// 4096 x 131072 x 4096 forward and backward 13.7 ms, 14.3 and 14.7).
constexpr int kHeadRaster = 16;
constexpr float kHeadLow = 2048.f;                       // what the low fp16 term is stored times
constexpr float kHeadTop = 8192.f;                       // where an fp32 tensor's largest value is brought to, at the least
constexpr float kHeadLog2e = 1.4426950408889634f, kHeadLn2 = 0.6931471805599453f;

// ------------------------------------------------------------------------------------ PTX wrappers
namespace head {

// The same shared-memory place in the pair's first CTA.
template <int CTAS>
__device__ __forceinline__ unsigned in_first(unsigned address) {
    if constexpr (CTAS == 1) return address;
    unsigned r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(address));
    return r;
}
template <int CTAS>
__device__ __forceinline__ void arrive_in_first(unsigned bar) {
    if constexpr (CTAS == 1)
        asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
    else
        // release at the block's scope only: at the cluster's it would wait for the epilogue's stores to reach L2, and what
        // is handed over is tensor memory, ordered by the tcgen05 fence before
        asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(in_first<CTAS>(bar)) : "memory");
}
// `bar` lies in the pair's first CTA, the data goes to this one.
template <int CTAS>
__device__ __forceinline__ void tma_load(unsigned dst, const CUtensorMap* map, int x, int y, unsigned bar) {
    if constexpr (CTAS == 1)
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(bar)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], "
            "[%4];" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(bar)
            : "memory");
}
template <int CTAS>
__device__ __forceinline__ void tma_load(unsigned dst, const CUtensorMap* map, int x, int y, int z, unsigned bar) {
    if constexpr (CTAS == 1)
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
                dst),
            "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], "
            "[%1, {%2, %3, %4}], [%5];" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
            : "memory");
}
template <int CTAS>
__device__ __forceinline__ void tma_load(unsigned dst, const CUtensorMap* map, int x, int y, int z, int w, unsigned bar) {
    if constexpr (CTAS == 1)
        asm volatile(
            "cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(
                dst),
            "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], "
            "[%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
            : "memory");
}
// Arrives on `bar` (in both CTAs of a pair) when the products issued so far have ended.
template <int CTAS>
__device__ __forceinline__ void commit(unsigned bar) {
    if constexpr (CTAS == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    else
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
            "h"(static_cast<unsigned short>(3))
            : "memory");
}
// Boxes from shared to global memory, in groups that a thread waits for.
__device__ __forceinline__ void tma_store(const CUtensorMap* map, unsigned src, int x, int y) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(src)
                 : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
__device__ __forceinline__ void tma_store(const CUtensorMap* map, unsigned src, int x, int y, int z) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(x), "r"(y),
                 "r"(z), "r"(src)
                 : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// At most `LEFT` of the thread's groups have still to read their shared memory.
template <int LEFT>
__device__ __forceinline__ void wait_stores_read() {
    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(LEFT) : "memory");
}
__device__ __forceinline__ void wait_stores() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
template <int CTAS>
__device__ __forceinline__ void mma(unsigned d, uint64_t a, uint64_t b, unsigned idesc, bool accumulate) {
    if constexpr (CTAS == 1)
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.u32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(static_cast<unsigned>(accumulate))
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.u32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(static_cast<unsigned>(accumulate))
            : "memory");
}
template <int CTAS>
__device__ __forceinline__ void tensor_memory_alloc(unsigned where) {
    if constexpr (CTAS == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(where) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(where) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
}
template <int CTAS>
__device__ __forceinline__ void tensor_memory_free(unsigned base) {
    if constexpr (CTAS == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(base));
    else
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(base));
}
// Barrier over the CTAs of a pair (or the block).
template <int CTAS>
__device__ __forceinline__ void sync_all() {
    if constexpr (CTAS == 1) {
        __syncthreads();
    } else {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
}
__device__ __forceinline__ void load32(unsigned address, float (&f)[32]) {
    __syncwarp();
    unsigned* r = reinterpret_cast<unsigned*>(f);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
          "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
          "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(address)
        : "memory");
}
__device__ __forceinline__ void load16(unsigned address, float (&f)[16]) {
    __syncwarp();
    unsigned* r = reinterpret_cast<unsigned*>(f);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(address)
        : "memory");
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
    int k_blocks, pairs;         // stages of K per pair of terms; 1 pair, or 3 for fp32 tensors
    int a_pitch, b_pitch;        // elements from one term of a row to the next
    int b_chunks;                // B with its other dimension contiguous: its map counts that in chunks of 64, one load a stage
    // LSE and GRAD
    const void* target;          // [M]
    int target64;
    int first;                   // vocabulary index of column 0
    int V;
    float2* partial;             // LSE: [2 tiles_n][M] maximum (base 2) and sum of half a tile's columns
    float* target_logit;         // LSE: [M]
    unsigned* status;            // LSE: cleared here, set by the kernel that joins the partial sums; GRAD with find_unit: written
    const float *lse, *dloss;    // GRAD: [M]
    float* unit;                 // GRAD: G holds the gradient divided by this; OUT: multiplied in again
    int find_unit;               // GRAD: every warp of the epilogue finds it itself, block 0 leaves it there
    const float *a_scale, *b_scale;   // fp32: what the terms of x (LSE, GRAD) and of B have been multiplied by
    // OUT
    void* out;                   // the tensor's type
    int64_t out_stride;
    int out_boxes;               // OUT: rows of `out` are whole 16-byte words, so it is written by TMA
    float* sums;                 // [splits][M][N] fp32, or NULL: `out` is written directly
    int add;                     // add what `sums` holds
    int last;                    // with sums: write `out` (one split only)
    // dW, after the last piece: two idle warps of each block add up dx's parts
    const float* join_sums;
    void* join_out;
    int join_parts;
    int64_t join_total;          // elements of a part
};

enum { kHeadLse = 0, kHeadGrad = 1, kHeadOut = 2 };

// Which terms a pair multiplies: low high, high low, high high (the single pair of bf16 tensors is the last one).
__device__ __forceinline__ void head_pair(int pair, int pairs, int& a, int& b) {
    const int p = pair + 3 - pairs;
    a = p == 0;
    b = p == 1;
}
// Where a segment that begins at k ends.  In fp32 those of the low terms end before the high ones begin.
template <bool FP32, int CTAS>
__device__ __forceinline__ int head_segment_end(const HeadGemm& g, int k, int k1) {
    if constexpr (!FP32) return min(k + (CTAS == 1 ? kHeadSegmentFew : kHeadSegment), k1);
    const int low = 2 * g.k_blocks;
    return min(k < low ? min(k + kHeadSegmentLow, low) : k + kHeadSegmentHigh, k1);
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
        k0 = 0;
        k1 = g.k_blocks * g.pairs;
        if (g.splits > 1) {
            const int64_t total = k1;
            k0 = static_cast<int>(total * split / g.splits);
            k1 = static_cast<int>(total * (split + 1) / g.splits);
        }
    }
};

// The largest |dloss| of the rows that count, over a warp's share of them: G is kept in units of it (1 if that is zero).
// With one weight for all rows, as a mean has, the largest entry of a row of G is then p - 1 itself; its rounding to
// bf16 does not carry that of the weight, which would be the same in every row and add up.  `flags` takes what the status word
// says of the targets.
__device__ __forceinline__ float head_unit(const void* target, int target64, const float* dloss, int rows, int V, int first, int step,
                                           unsigned& flags) {
    float top = 0.f;
    bool past = false;
#pragma unroll 4
    for (int t = first; t < rows; t += step) {
        const int64_t y = head::load_index(target, t, target64);
        const float g = fabsf(dloss[t]);
        if (y >= 0 && y < V && g < __int_as_float(0x7f800000)) top = fmaxf(top, g);
        past |= y >= V;
    }
    __syncwarp();
    flags = __any_sync(0xffffffffu, past) ? BNS_FLAG_BAD_TARGET : 0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    return top;
}

// Adds up the parts of a product in a fixed order and rounds once: vectors of V elements, BATCH of them at a time.  LANES lanes
// share a vector, each with every LANES-th part: many parts come with few elements, and one lane would wait for each
// of them in turn.  Warp `warp` of `warps`.
template <typename T, int V, int LANES, int BATCH>
__device__ __forceinline__ void head_join_parts(const HeadGemm& g, int warp, int warps, int lane) {
    constexpr int kPer = 32 / LANES;                         // vectors of a warp
    const int64_t vectors = g.join_total / V, stride = static_cast<int64_t>(warps) * kPer;
    const int mine = lane % LANES;
    for (int64_t base = static_cast<int64_t>(warp) * kPer; base < vectors; base += stride * BATCH) {
        const int64_t i0 = base + lane / LANES;
        float v[BATCH][V] = {};
#pragma unroll 4
        for (int s = mine; s < g.join_parts; s += LANES) {
            Vec<F32, V> x[BATCH];
#pragma unroll
            for (int b = 0; b < BATCH; ++b)
                if (i0 + b * stride < vectors) x[b].load(g.join_sums + s * g.join_total + (i0 + b * stride) * V);
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                if (i0 + b * stride < vectors) {
                    float f[V];
                    x[b].unpack(f);
#pragma unroll
                    for (int j = 0; j < V; ++j) v[b][j] += f[j];
                }
            }
        }
        __syncwarp();
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1)
#pragma unroll
            for (int b = 0; b < BATCH; ++b)
#pragma unroll
                for (int j = 0; j < V; ++j) v[b][j] += __shfl_xor_sync(0xffffffffu, v[b][j], o);
        if (mine == 0) {
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                if (i0 + b * stride < vectors) {
                    Vec<T, V> o;
                    o.pack(v[b]);
                    o.store(static_cast<typename T::storage*>(g.join_out) + (i0 + b * stride) * V);
                }
            }
        }
    }
}

// A value (scaled already) as two fp16 numbers.
__device__ __forceinline__ void split_half(float v, unsigned short& high, unsigned short& low) {
    const __half h = __float2half_rn(v);
    high = __half_as_ushort(h);
    low = __half_as_ushort(__float2half_rn((v - __half2float(h)) * kHeadLow));
}
__device__ __forceinline__ uint2 pack_halves(const unsigned short (&h)[4]) {
    return make_uint2(h[0] | static_cast<unsigned>(h[1]) << 16, h[2] | static_cast<unsigned>(h[3]) << 16);
}

// What a thread of the epilogue does with its half of a tile's columns of a row, 32 at a time.
template <int KIND, typename T, int N>
struct HeadEpilogue {
    using S = typename T::storage;
    static constexpr bool kFp32 = sizeof(S) == 4;
    static constexpr int kHalf = N / 2;
    const HeadGemm& g;
    const HeadTile& t;
    int row, column0, columns;   // first column, and how many of the half exist
    bool in;
    // LSE and GRAD
    int mine = -1;               // the target's place in the half
    bool counts = false;
    float unscale = 1.f, c;      // LSE and GRAD: logits = unscale accumulator; c = log2(e) unscale
    float m, s;                  // LSE
    float shift, factor, one;    // GRAD
    int half, lane;
    float4* stage;               // the warp's 32 x 128 bytes
    const CUtensorMap* map;      // of G, or of the output
    int& turn;                   // of the two buffers
    // where the lane's four columns of the warp's row lane / 8 go, the step to four rows below, and rows that exist
    int rows_left;
    float* sums_at = nullptr;
    S* out_at = nullptr;
    int64_t sums_step = 0, out_step = 0;

    __device__ __forceinline__ HeadEpilogue(const HeadGemm& g_, const HeadTile& t_, int row_, int half_, float4* stage_, const CUtensorMap* map_, int& turn_, float unit)
        : g(g_), t(t_), row(row_), column0(t_.n * N + half_ * kHalf), in(row_ < g_.M), half(half_),
          lane(threadIdx.x & 31), stage(stage_), map(map_), turn(turn_) {
        const int64_t first = row - lane + (lane >> 3);
        rows_left = static_cast<int>(g.M - first);
        columns = min(kHalf, g.N - column0);
        if constexpr (KIND != kHeadOut) {
            const int64_t y = in ? head::load_index(g.target, row, g.target64) : -1;
            counts = y >= 0 && y < g.V;
            const int64_t place = y - g.first - column0;
            if (counts && place >= 0 && place < columns) mine = static_cast<int>(place);
            if constexpr (kFp32) unscale = 1.f / *g.a_scale / *g.b_scale;      // powers of two
            c = kHeadLog2e * unscale;
        }
        if constexpr (KIND == kHeadLse) {
            m = __int_as_float(0xff800000);
            s = 0.f;
        } else if constexpr (KIND == kHeadGrad) {
            const float lse = counts ? g.lse[row] : 0.f;
            one = counts ? g.dloss[row] / unit * (kFp32 ? kHeadTop : 1.f) : 0.f;
            // lse log2(e) = shift + rest, log2(e) being the same fp32 number as in z log2(e), so that only the
            // difference z - lse feels its rounding; rest goes into the factor
            shift = lse * kHeadLog2e;
            factor = one * exp2_fast(-fmaf(lse, kHeadLog2e, -shift));
        } else {
            factor = unit;
            if constexpr (kFp32) factor *= 1.f / *g.b_scale / kHeadTop;
            const int at = column0 + 4 * (lane & 7);
            if (g.sums) sums_at = g.sums + (t.split * static_cast<int64_t>(g.M) + first) * g.N + at;
            sums_step = 4 * static_cast<int64_t>(g.N);
            out_at = static_cast<S*>(g.out) + first * g.out_stride + at;
            out_step = 4 * g.out_stride;
        }
    }
    // Columns that the accumulator has to be read for: G is written up to whole stages of K, zeros where nothing is.
    __device__ __forceinline__ int extent() const {
        if constexpr (KIND == kHeadGrad) return min(kHalf, (g.N + kHeadK - 1) / kHeadK * kHeadK - column0);
        return columns;
    }
    __device__ __forceinline__ void chunk(int at, float* f) {
        if constexpr (KIND == kHeadLse) {
            const float inf = __int_as_float(0x7f800000);
            if (columns - at < 32) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (at + j >= columns) f[j] = -inf;
            }
            float top = f[0];
#pragma unroll
            for (int j = 1; j < 32; ++j) top = fmaxf(top, f[j]);
            top = fmaxf(top * c, m);
            const float ref = top == -inf ? 0.f : top;
            s *= exp2_fast(m - ref);
#pragma unroll
            for (int j = 0; j < 32; ++j) s += exp2_fast(fmaf(f[j], c, -ref));
            m = top;
            if (mine >= at && mine < at + 32) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (mine == at + j) g.target_logit[row] = f[j] * unscale;
            }
        } else if constexpr (KIND == kHeadGrad) {
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                f[j] = counts && at + j < columns ? exp2_fast(fmaf(f[j], c, -shift)) * factor : 0.f;
                if (mine == at + j) f[j] -= one;
            }
            if constexpr (kFp32) {
                unsigned high[16], low[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    unsigned short h0, h1, l0, l1;
                    split_half(f[2 * j], h0, l0);
                    split_half(f[2 * j + 1], h1, l1);
                    high[j] = h0 | static_cast<unsigned>(h1) << 16;
                    low[j] = l0 | static_cast<unsigned>(l1) << 16;
                }
                send(high, column0 % kHeadN + at, column0 / kHeadN);
                send(low, kHeadN + column0 % kHeadN + at, column0 / kHeadN);
            } else {
                unsigned w[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) w[j] = pack_pair(f[2 * j], f[2 * j + 1]);
                send(w, column0 % kHeadN + at, column0 / kHeadN);
            }
        } else {
            const int left = columns - at - 4 * (lane & 7);
            const bool whole = g.N % 4 == 0;     // rows of sums and of the output begin at whole vectors
            S* to = out_at + at;
            if (g.out_boxes) {
#pragma unroll
                for (int j = 0; j < 32; j += 2) split_pair(mul2(make_pair(f[j], f[j + 1]), make_pair(factor, factor)), f[j], f[j + 1]);
                if constexpr (kFp32) {
                    send_floats(f, column0 + at);
                } else {
                    unsigned w[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) w[j] = pack_pair(f[2 * j], f[2 * j + 1]);
                    send(w, column0 + at, -1);
                }
                return;
            }
            float* sums = sums_at + at;
            spread(f, [&](int, float (&v)[4]) {
                if (left > 0) {
                    scale(v);
                    if (g.sums) put_or_add(sums, v, left, whole);
                    if (!g.sums || g.last) {
                        if (whole) {
                            Vec<T, 4> o;
                            o.pack(v);
                            o.store(to);
                        } else {
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                if (j < left) to[j] = from_float<T>(v[j]);
                        }
                    }
                }
                sums += sums_step;
                to += out_step;
            });
        }
    }
    __device__ __forceinline__ static unsigned pack_pair(float lo, float hi) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const unsigned*>(&h);
    }
    // The warp's 32 rows x 32 columns of 16 bits, a row a lane, into shared memory (64-byte rows, 64-byte swizzle) and out
    // by TMA, which drops rows and columns past the tensor's end.  Two buffers; z < 0: the map has two dimensions.  A warp
    // none of whose rows exist leaves both buffers alone: it would commit no group, and the wait for all groups but the last
    // frees the other buffer only while every turn commits one.
    __device__ __forceinline__ void send(const unsigned (&w)[16], int x, int z) {
        if (row - lane >= g.M) return;
        if (lane == 0) head::wait_stores_read<1>();
        __syncwarp();
        const unsigned buffer = smem_address(stage) + turn * 2048;
        turn ^= 1;
#pragma unroll
        for (int u = 0; u < 4; ++u)
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(buffer + lane * 64 + ((u ^ ((lane >> 1) & 3)) << 4)),
                         "r"(w[4 * u]), "r"(w[4 * u + 1]), "r"(w[4 * u + 2]), "r"(w[4 * u + 3])
                         : "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
            if (z < 0)
                head::tma_store(map, buffer, x, row);
            else
                head::tma_store(map, buffer, x, row, z);
        }
    }
    // The same for fp32: 128-byte rows, 128-byte swizzle, one buffer.
    __device__ __forceinline__ void send_floats(const float* f, int x) {
        if (row - lane >= g.M) return;
        if (lane == 0) head::wait_stores_read<0>();
        __syncwarp();
        const unsigned buffer = smem_address(stage);
#pragma unroll
        for (int u = 0; u < 8; ++u)
            asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(buffer + lane * 128 + ((u ^ (lane & 7)) << 4)), "f"(f[4 * u]),
                         "f"(f[4 * u + 1]), "f"(f[4 * u + 2]), "f"(f[4 * u + 3])
                         : "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) head::tma_store(map, buffer, x, row);
    }
    __device__ __forceinline__ void scale(float (&v)[4]) const {
        const pair_t by = make_pair(factor, factor);
        split_pair(mul2(make_pair(v[0], v[1]), by), v[0], v[1]);
        split_pair(mul2(make_pair(v[2], v[3]), by), v[2], v[3]);
    }
    // Adds what is there, and writes the sum back unless it is the last.
    __device__ __forceinline__ void put_or_add(float* p, float (&v)[4], int left, bool whole) const {
        if (whole) {
            float4* q = reinterpret_cast<float4*>(p);
            if (g.add) {
                const float4 old = *q;
                v[0] += old.x;
                v[1] += old.y;
                v[2] += old.z;
                v[3] += old.w;
            }
            if (!g.last) *q = make_float4(v[0], v[1], v[2], v[3]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (j >= left) continue;
                if (g.add) v[j] += p[j];
                if (!g.last) p[j] = v[j];
            }
        }
    }
    // Turns the warp's 32 rows x 32 columns, a row a lane, through shared memory into eight lanes a row: put(i, v) gets
    // columns 4 (lane % 8) .. + 3 of the warp's row 4 i + lane / 8, so that a store covers 64 or 128 contiguous bytes of a
    // row.  For sums and for outputs that TMA cannot write.
    template <typename Put>
    __device__ __forceinline__ void spread(const float* f, Put&& put) const {
        __syncwarp();
#pragma unroll
        for (int u = 0; u < 8; ++u)
            stage[lane * 8 + (u ^ (lane & 7))] = make_float4(f[4 * u], f[4 * u + 1], f[4 * u + 2], f[4 * u + 3]);
        __syncwarp();
        float4 q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = 4 * i + (lane >> 3);
            q[i] = stage[r * 8 + ((lane & 7) ^ (r & 7))];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (4 * i >= rows_left) break;
            float v[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
            put(i, v);
        }
    }
    __device__ __forceinline__ void finish() {
        if constexpr (KIND == kHeadLse) {
            if (in) g.partial[static_cast<int64_t>(t.n * 2 + half) * g.M + row] = make_float2(m, s);
        }
    }
};

template <int KIND, bool A_K, bool B_K, typename T, int CTAS, int N>
__global__ void __launch_bounds__(kHeadThreads, 1)
    head_gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                     const __grid_constant__ CUtensorMap map_c, const HeadGemm g) {
    using Ring = HeadRing<CTAS, N>;
    constexpr int kStages = Ring::kStages;
    constexpr bool kFp32 = sizeof(typename T::storage) == 4, kSegments = KIND != kHeadOut || kFp32;
    extern __shared__ unsigned char raw[];
    __shared__ __align__(8) uint64_t bars[2 * kStages + 5];
    __shared__ unsigned tmem_base;
    __shared__ volatile int gave_up;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = CTAS == 1 ? 0 : static_cast<int>(blockIdx.x & 1);      // in the pair
    const int worker = blockIdx.x / CTAS, workers = gridDim.x / CTAS;
    const unsigned head_raw = smem_address(raw), ring = (head_raw + 1023) & ~1023u;
    const unsigned full = smem_address(bars), empty = full + 8 * kStages, ready = empty + 8 * kStages, drained = ready + 16,
                   flush = drained + 16;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            barrier_init(full + 8 * s, 1);
            barrier_init(empty + 8 * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            barrier_init(ready + 8 * b, 1);
            barrier_init(drained + 8 * b, 8 * CTAS);
        }
        barrier_init(flush, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        gave_up = 0;
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_b) : "memory");
    }
    if (warp == 2) head::tensor_memory_alloc<CTAS>(smem_address(&tmem_base));
    head::fence_before();
    __syncthreads();
    if constexpr (CTAS == 2) head::sync_all<CTAS>();      // the other CTA's barriers exist
    head::fence_after();
    const unsigned tmem = tmem_base;
    grid_dependency_wait();
    grid_dependency_launch();

    const int tiles = g.tiles_m * g.tiles_n * g.splits;
    // The ring's place of this thread: stage, and parity of its barriers' current phase.  Neither loop divides: at some 500
    // cycles a stage a few dozen of them in the loop that feeds the ring show.
    int s = 0;
    unsigned phase = 0;
    auto advance = [&]() {
        if (++s == kStages) {
            s = 0;
            phase ^= 1;
        }
    };
    if (warp < 4) {
        if (warp == 0 && lane == 0) {
            const unsigned full_first = head::in_first<CTAS>(full);
            const int k_end = g.k_blocks * kHeadK;
            bool ok = true;
            for (int id = worker; ok && id < tiles; id += workers) {
                const HeadTile t(g, id);
                const int row = (t.m * CTAS + rank) * kHeadM, column = t.n * N + rank * Ring::kColumns;
                int pair = g.pairs > 1 ? t.k0 / g.k_blocks : 0, kk = (t.k0 - pair * g.k_blocks) * kHeadK, ta, tb;
                head_pair(pair, g.pairs, ta, tb);
                for (int k = t.k0; k < t.k1; ++k) {
                    if (!(ok = wait_bounded(empty + 8 * s, phase ^ 1, &gave_up))) break;     // passes at once on the first round
                    const unsigned bar = full_first + 8 * s, sa = ring + s * Ring::kStage, sb = sa + Ring::kStageA;
                    if (rank == 0) barrier_expect(full + 8 * s, CTAS * Ring::kStage);
                    if constexpr (KIND == kHeadOut) {       // A is G, in blocks of 256 columns
                        if constexpr (A_K)
                            head::tma_load<CTAS>(sa, &map_a, ta * kHeadN + kk % kHeadN, row, kk / kHeadN, bar);
                        else
                            head::tma_load<CTAS>(sa, &map_a, 0, kk, (ta * kHeadN + row % kHeadN) / 64, row / kHeadN, bar);
                    } else {
                        head::tma_load<CTAS>(sa, &map_a, ta * g.a_pitch + kk, row, bar);
                    }
                    if constexpr (B_K) {
                        head::tma_load<CTAS>(sb, &map_b, tb * g.b_pitch + kk, column, bar);
                    } else if (g.b_chunks) {
                        head::tma_load<CTAS>(sb, &map_b, 0, kk, (tb * g.b_pitch + column) / 64, bar);
                    } else {
#pragma unroll
                        for (int q = 0; q < Ring::kColumns / 64; ++q)
                            head::tma_load<CTAS>(sb + q * 8192, &map_b, tb * g.b_pitch + column + q * 64, kk, bar);
                    }
                    advance();
                    kk += kHeadK;
                    if (kk == k_end) {
                        kk = 0;
                        head_pair(++pair, g.pairs, ta, tb);
                    }
                }
            }
            // the products have read every stage: nothing arrives here any more once the block ends
            for (int i = 0; ok && i < kStages; ++i) {
                ok = wait_bounded(empty + 8 * s, phase ^ 1, &gave_up);
                if (ok) advance();
            }
        } else if (warp == 1 && lane == 0 && rank == 0) {
            constexpr unsigned idesc = (1u << 4) | (kFp32 ? 0u : (1u << 7) | (1u << 10)) | (A_K ? 0u : 1u << 15) | (B_K ? 0u : 1u << 16) |
                                       ((N >> 3) << 17) | ((CTAS * kHeadM >> 4) << 24);
            int n = 0;
            bool ok = true;
            for (int id = worker; ok && id < tiles; id += workers) {
                const HeadTile t(g, id);
                for (int k = t.k0, end; ok && k < t.k1; k = end, ++n) {
                    const int buffer = n & 1;
                    end = kSegments ? head_segment_end<kFp32, CTAS>(g, k, t.k1) : t.k1;
                    if (n >= 2 && !(ok = wait_bounded(drained + 8 * buffer, (n / 2 - 1) & 1, &gave_up))) break;
                    head::fence_after();
                    const unsigned d = tmem + buffer * N;
                    for (int kk = k; kk < end; ++kk) {
                        if (!(ok = wait_bounded(full + 8 * s, phase, &gave_up))) break;
                        head::fence_after();
                        const unsigned sa = ring + s * Ring::kStage;
                        const uint64_t da = head::descriptor<A_K>(sa), db = head::descriptor<B_K>(sa + Ring::kStageA);
#pragma unroll
                        for (int q = 0; q < kHeadK / 16; ++q)
                            head::mma<CTAS>(d, da + q * head::descriptor_step<A_K>(), db + q * head::descriptor_step<B_K>(), idesc,
                                            kk > k || q > 0);
                        head::commit<CTAS>(empty + 8 * s);
                        advance();
                    }
                    if (!ok) break;
                    head::commit<CTAS>(ready + 8 * buffer);
                }
            }
        }
        if constexpr (KIND == kHeadOut && !A_K) {
            if (warp >= 2 && g.join_parts) {
                const int at = blockIdx.x * 2 + warp - 2, of = gridDim.x * 2;
                const bool whole = g.join_total % 4 == 0;       // a part begins at a 16-byte boundary
                // eight lanes a vector where there are fewer vectors than two a lane (24 x 1024, 37 parts: dW's kernel 28 -> 18 us)
                if (g.join_parts >= 8 && g.join_total < static_cast<int64_t>(of) * 32 * 2 * (whole ? 4 : 1)) {
                    if (whole)
                        head_join_parts<T, 4, 8, 1>(g, at, of, lane);
                    else
                        head_join_parts<T, 1, 8, 1>(g, at, of, lane);
                } else if (whole) {
                    head_join_parts<T, 4, 1, 4>(g, at, of, lane);
                } else {
                    head_join_parts<T, 1, 1, 4>(g, at, of, lane);
                }
            }
        }
        __syncwarp();
    } else {
        const int slot = warp & 3, half = (warp - 4) >> 2;
        float4* stage = reinterpret_cast<float4*>(raw + (ring - head_raw) + kStages * Ring::kStage) + (warp - 4) * 256;
        if (KIND == kHeadLse && blockIdx.x == 0 && threadIdx.x == 128 && g.status) *g.status = 0;
        float unit = 1.f;
        if (KIND == kHeadGrad && g.find_unit) {
            unsigned flags;
            unit = head_unit(g.target, g.target64, g.dloss, g.M, g.V, lane, 32, flags);
            unit = unit > 0.f ? unit : 1.f;
            if (blockIdx.x == 0 && threadIdx.x == 128) {
                *g.unit = unit;
                *g.status = flags;
            }
        } else if (KIND != kHeadLse) {
            unit = *g.unit;
        }
        int n = 0, turn = 0;
        bool ok = true;
        for (int id = worker; ok && id < tiles; id += workers) {
            const HeadTile t(g, id);
            // The splits are made for a full piece of the vocabulary, whose parts have four stages at the least.  A last piece with
            // fewer stages than splits leaves some without any: no product is made for those, and the sums have all of theirs
            if (KIND == kHeadOut && t.k0 == t.k1) continue;
            HeadEpilogue<KIND, T, N> e(g, t, (t.m * CTAS + rank) * kHeadM + slot * 32 + lane, half, stage, &map_c, turn, unit);
            const unsigned lanes = tmem + (static_cast<unsigned>(slot * 32) << 16) + half * (N / 2);
            auto wait_ready = [&]() {
                ok = __all_sync(0xffffffffu, wait_bounded(ready + 8 * (n & 1), (n / 2) & 1, &gave_up));
                head::fence_after();
                return ok;
            };
            auto give_back = [&]() {
                head::fence_before();
                __syncwarp();
                if (lane == 0) head::arrive_in_first<CTAS>(drained + 8 * (n & 1));
                ++n;
            };
            if constexpr (kSegments) {
                float acc[N / 2];
#pragma unroll
                for (int j = 0; j < N / 2; ++j) acc[j] = 0.f;
                for (int k = t.k0; k < t.k1; k = head_segment_end<kFp32, CTAS>(g, k, t.k1)) {
                    if (!wait_ready()) break;
                    const float weight = kFp32 && k < 2 * g.k_blocks ? 1.f / kHeadLow : 1.f;
#pragma unroll
                    for (int c = 0; c < N / 2; c += 16) {
                        float f[16];
                        head::load16(lanes + (n & 1) * N + c, f);
#pragma unroll
                        for (int j = 0; j < 16; ++j) acc[c + j] = fmaf(f[j], weight, acc[c + j]);
                    }
                    give_back();
                }
                if (!ok) break;
                const int extent = e.extent();
#pragma unroll
                for (int c = 0; c < N / 2; c += 32)
                    if (c < extent) e.chunk(c, acc + c);
                e.finish();
            } else {
                if (!wait_ready()) break;
                const int extent = e.extent();
                for (int c = 0; c < extent; c += 32) {
                    float f[32];
                    head::load32(lanes + (n & 1) * N + c, f);
                    e.chunk(c, f);
                }
                e.finish();
                give_back();
            }
        }
        if (KIND != kHeadLse && lane == 0) head::wait_stores();
    }
    __syncthreads();
    if (gave_up) {
        // a block that gave up leaves only when its copies have landed and its products have ended
        if (threadIdx.x == 0 && rank == 0)
            for (int q = 0; q < kStages; ++q)     // the last fill of stage q; one that was never filled passes
                for (unsigned n = 0; n < kPolls && !barrier_try(full + 8 * q, q < s ? phase : phase ^ 1); ++n) {
                }
        if (threadIdx.x == 32 && rank == 0) {
            head::commit<CTAS>(flush);
            for (unsigned n = 0; n < kPolls && !barrier_try(flush, 0); ++n) {
            }
        }
        __syncthreads();
    }
    if constexpr (CTAS == 2) head::sync_all<CTAS>();
    if (warp == 2) {
        head::fence_after();
        head::tensor_memory_free<CTAS>(tmem);
    }
}

// ------------------------------------------------------------------------------------ around the products
__global__ void __launch_bounds__(1024) head_unit_kernel(const void* target, int target64, const float* dloss, int rows, int V,
                                                         float* unit, unsigned* status) {
    __shared__ float fold[32];
    grid_dependency_wait();
    grid_dependency_launch();
    unsigned flags;
    const float top = head_unit(target, target64, dloss, rows, V, threadIdx.x, 1024, flags);
    if ((threadIdx.x & 31) == 0) fold[threadIdx.x >> 5] = top;
    const bool past = __syncthreads_or(flags);
    if (threadIdx.x == 0) {
        *status = past ? BNS_FLAG_BAD_TARGET : 0;
        float all = 0.f;
        for (int w = 0; w < 32; ++w) all = fmaxf(all, fold[w]);
        *unit = all > 0.f ? all : 1.f;
    }
}

// bf16 rows whose stride TMA cannot take, laid out with rows of `pitch` elements, padded with zeros.
struct HeadCopy {
    static constexpr int kTerms = 1;
    using From = BF16;
    __device__ __forceinline__ static void put(const float (&v)[8], float, unsigned short* to, int) {
        Vec<BF16, 8> o;
        o.pack(v);
        o.store(to);
    }
};
// fp32 rows as two fp16 terms, each padded with zeros to `pitch` elements.
struct HeadSplit {
    static constexpr int kTerms = 2;
    using From = F32;
    __device__ __forceinline__ static void put(const float (&v)[8], float scale, unsigned short* to, int pitch) {
        unsigned short high[2][4], low[2][4];
#pragma unroll
        for (int j = 0; j < 8; ++j) split_half(v[j] * scale, high[j / 4][j % 4], low[j / 4][j % 4]);
        const uint2 h0 = pack_halves(high[0]), h1 = pack_halves(high[1]), l0 = pack_halves(low[0]), l1 = pack_halves(low[1]);
        *reinterpret_cast<uint4*>(to) = make_uint4(h0.x, h0.y, h1.x, h1.y);
        *reinterpret_cast<uint4*>(to + pitch) = make_uint4(l0.x, l0.y, l1.x, l1.y);
    }
};

// Eight columns of a row (zeros past its end), in 16-byte words where its stride allows it.
template <typename T>
__device__ __forceinline__ void load_eight(const typename T::storage* row, int first, int D, bool words, float (&v)[8]) {
    constexpr int kWord = 16 / sizeof(typename T::storage);
    if (words && first + 8 <= D) {
#pragma unroll
        for (int j = 0; j < 8; j += kWord) {
            Vec<T, kWord> x;
            float f[kWord];
            x.load(row + first + j);
            x.unpack(f);
#pragma unroll
            for (int i = 0; i < kWord; ++i) v[j + i] = f[i];
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = first + j < D ? to_float<T>(row[first + j]) : 0.f;
    }
}

// The largest finite magnitude of a matrix, as the bits of a float, into *top (which starts at 0).
__global__ void __launch_bounds__(256) head_top_kernel(const float* src, int64_t stride, int rows, int D, unsigned* top) {
    grid_dependency_wait();
    grid_dependency_launch();
    const int first = (blockIdx.x * 32 + (threadIdx.x & 31)) * 8;
    unsigned most = 0;
    if (first < D) {
        for (int64_t row = blockIdx.y * 8 + (threadIdx.x >> 5); row < rows; row += gridDim.y * 8) {
            float v[8];
            load_eight<F32>(src + row * stride, first, D, stride % 4 == 0, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const unsigned bits = __float_as_uint(fabsf(v[j]));
                if (bits < 0x7f800000u) most = max(most, bits);
            }
        }
    }
    most = __reduce_max_sync(0xffffffffu, most);
    if ((threadIdx.x & 31) == 0 && most) atomicMax(top, most);
}

// The power of two that brings a tensor whose largest value has these bits to [2^13, 2^14).
__device__ __forceinline__ float head_scale(unsigned top) {
    const int exponent = top ? static_cast<int>(top >> 23) : 127;    // biased
    return __uint_as_float(static_cast<unsigned>(min(254, 127 + 13 + 127 - exponent)) << 23);
}

// Eight columns a thread.  For fp32 the scale is made of *top and left in *scale.
template <typename FORM>
__global__ void __launch_bounds__(256) head_terms_kernel(const void* src, int64_t stride, int rows, int D, int pitch,
                                                         unsigned short* dst, const unsigned* top, float* scale) {
    using T = typename FORM::From;
    grid_dependency_wait();
    grid_dependency_launch();
    float by = 1.f;
    if constexpr (FORM::kTerms > 1) {
        by = head_scale(*top);
        if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *scale = by;
    }
    const int units = pitch / 8, unit = blockIdx.x * 32 + (threadIdx.x & 31);
    if (unit >= units) return;
    const bool words = stride % (16 / static_cast<int>(sizeof(typename T::storage))) == 0;
    for (int64_t row = blockIdx.y * 8 + (threadIdx.x >> 5); row < rows; row += gridDim.y * 8) {
        float v[8];
        load_eight<T>(static_cast<const typename T::storage*>(src) + row * stride, unit * 8, D, words, v);
        FORM::put(v, by, dst + row * FORM::kTerms * pitch + unit * 8, pitch);
    }
}

// Joins the half tiles' maxima and sums of a row: 32 rows a block, 32 threads a row, in a fixed order.
__global__ void __launch_bounds__(1024) head_join_kernel(const float2* partial, int strips, int rows, const float* target_logit,
                                                         const void* target, int target64, int V, float* loss, float* lse,
                                                         unsigned* status) {
    __shared__ float2 fold[32][33];
    grid_dependency_wait();
    grid_dependency_launch();
    const float inf = __int_as_float(0x7f800000);
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
    int row = blockIdx.x * 32 + lane;
    auto join = [&](float2 a, float2 b) {
        const float m = fmaxf(a.x, b.x), ref = m == -inf ? 0.f : m;
        return make_float2(m, a.y * exp2_fast(a.x - ref) + b.y * exp2_fast(b.x - ref));
    };
    float2 v = make_float2(-inf, 0.f);
    if (row < rows) {
        for (int t0 = part; t0 < strips; t0 += 128) {
            float2 x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                x[i] = t0 + i * 32 < strips ? partial[static_cast<int64_t>(t0 + i * 32) * rows + row] : make_float2(-inf, 0.f);
            v = join(v, join(join(x[0], x[1]), join(x[2], x[3])));
        }
    }
    fold[part][lane] = v;
    __syncthreads();
    v = fold[lane][part];       // now a warp has a row
    row = blockIdx.x * 32 + part;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        v = join(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o)));
    if (lane || row >= rows) return;
    const float rest = log2f(v.y);
    lse[row] = (v.x + rest) * kHeadLn2;
    const int64_t y = head::load_index(target, row, target64);
    // the difference to the largest first: where the model is sure, lse and the target's logit are nearly equal
    loss[row] = y >= 0 && y < V ? (fmaf(-target_logit[row], kHeadLog2e, v.x) + rest) * kHeadLn2 : 0.f;
    if (y >= V) atomicOr(status, BNS_FLAG_BAD_TARGET);
}

}  // namespace bns
