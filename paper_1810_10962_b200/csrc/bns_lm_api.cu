// Host side of the language-model operators declared in include/bns.h: residual add + root-mean-square norm,
// linear head + cross entropy, top-k distillation.  Checks, plans, workspace layout and launches; nothing here allocates
// device memory or synchronises the host.
#include <algorithm>
#include <atomic>

#include "bns_distill_kernels.cuh"
#include "bns_head_few_kernels.cuh"
#include "bns_head_kernels.cuh"
#include "bns_lm_host.h"
#include "bns_rms_kernels.cuh"

namespace {

using namespace bns;

// ------------------------------------------------------------------------------------ root-mean-square norm
bns_status check_rows(const bns_rows* sh) {
    if (!sh) return BNS_ERR_NULL;
    if (sh->rows < 0 || sh->columns <= 0) return BNS_ERR_SHAPE;
    if (!known(sh->dtype)) return BNS_ERR_DTYPE;
    return BNS_OK;
}

struct RmsPlan {
    int V;
    bool loose;      // rows at any phase
    unsigned threads;
    int elements;    // of a row that a thread holds: 8 or 16; 0 = the row does not fit the block's registers
    unsigned grid;
};

// Both kernels are compiled for 64 registers a thread, so 1024 threads an SM.  Eight elements a thread leave room for
// the next row's loads of fp32 tensors and for the gradient's column sums; sixteen of bf16 fit the forward kernel, whose
// reductions then have half as many threads (8192 x 8192 to 8 bits: 80 us against 86).  Rows at any phase in vectors: 1531 x 2050
// fp32, forward and backward, 28.5 us against 40 element by element.
RmsPlan plan_rms(int rows, int columns, int dtype, VectorRule::Kind kind, bool eight) {
    RmsPlan pl;
    const int full = 16 / elem_bytes(dtype);
    pl.loose = kind == VectorRule::kPhase;
    if (pl.loose && columns > kRmsMaxThreads * 8) kind = VectorRule::kElements;   // phases come with eight elements a thread
    pl.loose = kind == VectorRule::kPhase;
    pl.V = kind == VectorRule::kElements ? 1 : full;
    const int vectors = divide_up(columns, pl.V);
    for (pl.elements = eight || pl.V == 1 || pl.loose ? 8 : 16; pl.elements <= 16; pl.elements *= 2) {
        const int threads = divide_up(divide_up(vectors, std::max(1, pl.elements / pl.V)), 32) * 32;
        pl.threads = static_cast<unsigned>(threads);
        if (threads <= kRmsMaxThreads || pl.V == 1) break;
    }
    if (pl.threads > kRmsMaxThreads) {
        pl.elements = 0;
        pl.threads = kRmsMaxThreads;
    }
    const int blocks_per_sm = std::max(1, std::min(32, kRmsMaxThreads / static_cast<int>(pl.threads)));
    int64_t grid = static_cast<int64_t>(sm_count()) * blocks_per_sm;
    grid -= grid % full;             // a block meets one phase
    pl.grid = static_cast<unsigned>(std::min<int64_t>(rows, grid));
    return pl;
}

// V is a vector's elements, or 1.
#define BNS_LM_BY_TYPE_V(dtype, V_, CALL)                   \
    do {                                                    \
        if ((dtype) == BNS_F32) {                           \
            using T = F32;                                  \
            if ((V_) == 1) {                                \
                constexpr int V = 1;                        \
                CALL;                                       \
            } else {                                        \
                constexpr int V = 4;                        \
                CALL;                                       \
            }                                               \
        } else {                                            \
            using T = BF16;                                 \
            if ((V_) == 1) {                                \
                constexpr int V = 1;                        \
                CALL;                                       \
            } else {                                        \
                constexpr int V = 8;                        \
                CALL;                                       \
            }                                               \
        }                                                   \
    } while (0)

template <typename OUT>
bns_status rms_forward(const bns_rows* sh, const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                       const float* weight, float eps, void* y, float* scales, void* h, float* rstd, void* cuda_stream) {
    constexpr bool quantized = !__is_same(OUT, RmsNone);
    if (sh->rows == 0) return BNS_OK;
    if (!x || !weight || !y || !rstd || (quantized && !scales)) return BNS_ERR_NULL;
    if (!(eps > 0.f) || x_stride < sh->columns || (residual && residual_stride < sh->columns)) return BNS_ERR_SHAPE;
    const size_t eb = elem_bytes(sh->dtype);
    if (!aligned(x, eb) || !aligned(residual, eb) || !aligned(h, eb) || !aligned(weight, 4) || !aligned(rstd, 4) ||
        !aligned(scales, 4) || !(quantized || aligned(y, eb)))
        return BNS_ERR_ALIGN;
    constexpr bool grouped = __is_same(OUT, RmsGroupScale);
    VectorRule rule(sh->columns, static_cast<int>(eb));
    rule.tensor(x, x_stride);
    rule.tensor(residual, residual_stride);
    rule.tensor(h, sh->columns);
    if (quantized)
        rule.bytes(y);
    else
        rule.tensor(y, sh->columns);
    if (!aligned(weight, 16) && rule.kind == VectorRule::kAligned) rule.kind = VectorRule::kPhase;   // keeps its weights
    if (grouped && rule.kind == VectorRule::kPhase) rule.kind = VectorRule::kElements;   // groups begin at whole vectors
    const RmsPlan pl = plan_rms(sh->rows, sh->columns, sh->dtype, rule.kind, sh->dtype == BNS_F32);
    const RmsForward a{x, residual, weight, y, scales, h, rstd, sh->rows, x_stride, residual_stride, sh->columns, eps,
                       1.f / static_cast<float>(sh->columns)};
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const Shape shape{pl.grid, pl.threads};
    const size_t smem = grouped && pl.V == 1 ? pl.threads / 32 * 8 * sizeof(float) : 0;
    BNS_LM_BY_TYPE_V(sh->dtype, pl.V, {
        if (pl.elements == 0) {
            launch(BNS_KERNEL_RMS_FORWARD, rms_forward_wide_kernel<T, V, OUT>, shape, 0, stream, a);
        } else if constexpr (V == 1) {
            launch(BNS_KERNEL_RMS_FORWARD, rms_forward_kernel<T, 1, 8, false, OUT>, shape, smem, stream, a);
        } else {
            if constexpr (!grouped) {
                if (pl.loose) {
                    launch(BNS_KERNEL_RMS_FORWARD, rms_forward_kernel<T, V, 8, true, OUT>, shape, 0, stream, a);
                    return last_error();
                }
            }
            if (pl.elements == 8)
                launch(BNS_KERNEL_RMS_FORWARD, rms_forward_kernel<T, V, 8, false, OUT>, shape, 0, stream, a);
            else
                launch(BNS_KERNEL_RMS_FORWARD, rms_forward_kernel<T, V, 16, false, OUT>, shape, 0, stream, a);
        }
    });
    return last_error();
}

template <typename T, int V>
void rms_backward(const RmsPlan& pl, const Shape& grid, const RmsBackward& a, cudaStream_t stream) {
    if (pl.elements == 0) {
        launch(BNS_KERNEL_RMS_BACKWARD, rms_backward_wide_kernel<T>, grid, 0, stream, a);
    } else if constexpr (V == 1) {
        launch(BNS_KERNEL_RMS_BACKWARD, rms_backward_kernel<T, 1, 8, false>, grid, 0, stream, a);
    } else {
        if (pl.loose)
            launch(BNS_KERNEL_RMS_BACKWARD, rms_backward_kernel<T, V, 8, true>, grid, 0, stream, a);
        else if (pl.elements == 8)
            launch(BNS_KERNEL_RMS_BACKWARD, rms_backward_kernel<T, V, 8, false>, grid, 0, stream, a);
        else
            launch(BNS_KERNEL_RMS_BACKWARD, rms_backward_kernel<T, V, 16, false>, grid, 0, stream, a);
    }
}

// Blocks of the gradient kernel, at the most: each leaves a row of partial sums.
int rms_backward_blocks(int rows) { return std::min(rows, sm_count() * 32); }

// ------------------------------------------------------------------------------------ head
// Aimed at for G of a piece, and for a piece's operand in fp16 terms.  Four times as much buys nothing (4096 x 131072 x 4096 bf16
// 13.8 ms against 13.7, 1021 x 32003 x 1000 fp32 798 us against 796), a quarter costs 4 and 14 %.
constexpr size_t kHeadPieceBytes = size_t{256} << 20;
constexpr int kHeadPieceLeast = 4096;

// What the kernels leave for one another besides arrays.
struct HeadScalars {
    float unit;                      // G is kept in units of this
    float x_scale, w_scale;          // fp32: what the terms of x and of the piece of w have been multiplied by
    unsigned x_top, w_top;           // their largest magnitudes
};

struct HeadProblem {
    int T, V, D, dtype;
    bool f32, copy_x, copy_w;       // operands laid out anew in the workspace
    int terms, pairs;
    int pitch;                      // of a copied row's term
    int piece, pieces;              // columns of the vocabulary at a time
    int G_pitch;
    int splits;                     // of dx along the vocabulary
    int few;                        // rows of the kernels for few rows, or 0; with them, of the products:
    bool few_words;                 // W's rows are made of 16-byte words
    int few_threads, few_groups, few_chunks, few_per;
    size_t off_scalars, off_x, off_w, off_G, off_partial, off_logit, off_sums, total;
};

bns_status check_head(const bns_head* sh) {
    if (!sh) return BNS_ERR_NULL;
    if (sh->rows < 0 || sh->vocabulary <= 0 || sh->width <= 0 || sh->rows > 1 << 24 || sh->vocabulary > 1 << 28 ||
        sh->width > 1 << 20 || sh->x_stride < sh->width || sh->w_stride < sh->width)
        return BNS_ERR_SHAPE;
    if (!known(sh->dtype)) return BNS_ERR_DTYPE;
    return BNS_OK;
}

// CTAs that work on a tile of a product with M rows, and columns of a tile of the products with the logits.  Narrow tiles pay
// while one round of them covers the vocabulary (5 x 2564 x 3160 forward: 32 -> 25 us); beyond that they read x too
// often, and a product of 64 columns takes as long as one of 256 (24 x 32768 x 1024 forward: 24 -> 37 us).
int head_ctas(int M) { return M <= kHeadM ? 1 : 2; }
int head_columns(int rows, int vocabulary) {
    return rows <= kHeadNarrowRows && vocabulary <= kHeadNarrow * sm_count() ? kHeadNarrow : kHeadN;
}

bool tma_rows(int64_t stride) { return stride % 8 == 0 && stride < int64_t{1} << 38; }

// Parts that dx's sum over the vocabulary is taken in.  With few rows it has few tiles and a long sum: the parts fill the
// SMs.  With many the last round of tiles leaves SMs idle: parts even the rounds out (4096 x 4096: 256 tiles on 74 pairs
// are 4 rounds, in halves 3.5).  Each part costs a write and a read of fp32 sums.
int split_head(const HeadProblem& p) {
    const int ctas = head_ctas(p.T);
    const int64_t workers = sm_count() / ctas;
    const int64_t tiles = static_cast<int64_t>(divide_up(p.T, kHeadM * ctas)) * divide_up(p.D, kHeadN);
    const int64_t steps = static_cast<int64_t>(divide_up(p.piece, kHeadK)) * p.pairs;
    const double step_us = 0.32 * p.pieces, sums_us = static_cast<double>(p.T) * p.D * 8 / 5e6;   // of all pieces; of a part
    int best = 1;
    double least = 1e300;
    for (int s = 1; s <= 64 && (s == 1 || steps / s >= 4); ++s) {
        const double cost = static_cast<double>(divide_up(tiles * s, workers)) * static_cast<double>(divide_up<int64_t>(steps, s)) * step_us +
                            (s > 1 ? s * sums_us * p.pieces + 3.0 : 0.0);
        if (cost < least) {
            least = cost;
            best = s;
        }
    }
    return best;
}

int few_pitch(int width, bool words) { return words ? width : divide_up(width, 32 * kFewLane) * 32 * kFewLane; }

// Rows that the few rows' kernels are compiled for, or 0 where the tensor cores do the products: fp32 only (bf16 needs no new
// layout for the tensor cores: 32768 x 1024 with one row 24 us forward, 64 on the fp32 pipes), while x fits shared memory.
int few_rows(const bns_head* sh, bool words, bool backward) {
    if (sh->dtype != BNS_F32 || sh->rows == 0 || sh->rows > (backward ? kFewRowsBackward : kFewRows)) return 0;
    int rows = 1;
    while (rows < sh->rows) rows *= 2;
    return static_cast<size_t>(rows) * few_pitch(sh->width, words) * sizeof(float) <= kFewSharedMost ? rows : 0;
}

HeadProblem plan_head(const bns_head* sh, bool backward) {
    HeadProblem p{};
    p.few_words = sh->width % kFewLane == 0 && sh->w_stride % kFewLane == 0;
    p.few = few_rows(sh, p.few_words, backward);
    p.T = sh->rows;
    p.V = sh->vocabulary;
    p.D = sh->width;
    p.dtype = sh->dtype;
    p.f32 = sh->dtype == BNS_F32;
    p.copy_x = p.f32 || !tma_rows(sh->x_stride);
    p.copy_w = p.f32 || !tma_rows(sh->w_stride);
    p.terms = p.f32 ? 2 : 1;
    p.pairs = p.f32 ? 3 : 1;
    p.pitch = divide_up(p.D, kHeadK) * kHeadK;
    if (p.T == 0) {                 // the status word is all that is written
        p.total = kHeaderBytes;
        return p;
    }
    size_t column = 0;              // workspace bytes per column of the vocabulary
    if (p.copy_w) column = static_cast<size_t>(p.terms) * p.pitch * 2;
    if (backward) column = std::max(column, static_cast<size_t>(p.T) * p.terms * 2);
    if (p.few) {
        size_t at = kHeaderBytes;
        auto take = [&](size_t bytes) {
            const size_t here = at;
            at = align_up(at + bytes);
            return here;
        };
        p.few_threads = std::min(kFewProductThreads, divide_up(divide_up(p.D, kFewLane), 32) * 32);
        p.few_groups = divide_up(p.D, p.few_threads * kFewLane);
        const int blocks = sm_count() * 2 * (kFewProductThreads / p.few_threads);
        p.few_per = std::max(8, divide_up(p.V, std::max(1, blocks / p.few_groups)));
        p.few_chunks = divide_up(p.V, p.few_per);
        if (backward) {
            p.off_G = take(static_cast<size_t>(p.V) * p.few * 4);
            p.off_sums = take(static_cast<size_t>(p.few_chunks) * p.T * p.D * 4);
        } else {
            p.off_partial = take(static_cast<size_t>(sm_count()) * p.T * sizeof(float2));
            p.off_logit = take(static_cast<size_t>(p.T) * 4);
        }
        p.total = at;
        return p;
    }
    int64_t piece = p.V;
    if (column) piece = std::max<int64_t>(kHeadPieceLeast, static_cast<int64_t>(kHeadPieceBytes / column) / kHeadN * kHeadN);
    if (g_head_piece > 0 && (p.copy_w || backward)) piece = std::min<int64_t>(piece, g_head_piece);
    p.pieces = static_cast<int>(divide_up<int64_t>(p.V, piece));
    // equal pieces of whole tiles
    p.piece = static_cast<int>(std::min<int64_t>(p.V, divide_up(divide_up(p.V, p.pieces), kHeadN) * static_cast<int64_t>(kHeadN)));
    p.pieces = divide_up(p.V, p.piece);
    p.splits = 1;
    p.G_pitch = divide_up(p.piece, kHeadN) * kHeadN;
    if (backward) p.splits = split_head(p);
    size_t at = kHeaderBytes;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at = align_up(at + bytes);
        return here;
    };
    const size_t T = p.T;
    p.off_scalars = take(sizeof(HeadScalars));
    if (p.copy_x) p.off_x = take(T * p.terms * p.pitch * 2);
    if (p.copy_w) p.off_w = take(static_cast<size_t>(p.piece) * p.terms * p.pitch * 2);
    if (backward) {
        p.off_G = take(T * p.terms * p.G_pitch * 2);
        if (p.splits > 1 || p.pieces > 1) p.off_sums = take(T * p.splits * p.D * 4);
    } else {
        p.off_partial = take(2 * T * (divide_up(p.V, head_columns(p.T, p.V)) + p.pieces) * sizeof(float2));
        p.off_logit = take(T * 4);
    }
    p.total = at;
    return p;
}

// Tensor map; operands are 16-bit values in boxes of 64 (128 bytes, swizzled) by box[1] by ...
bool encode_map(CUtensorMap* map, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box,
                CUtensorMapDataType type = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B) {
    using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static std::atomic<void*> entry{nullptr};
    void* fn = entry.load(std::memory_order_relaxed);
    if (!fn) {
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess || !fn)
            return false;
        entry.store(fn, std::memory_order_relaxed);
    }
    const cuuint32_t steps[4] = {1, 1, 1, 1};
    return reinterpret_cast<Encode>(fn)(map, type, static_cast<cuuint32_t>(rank), const_cast<void*>(base), dims, strides, box, steps,
                                        CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                                        CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A matrix operand: rows of `terms` terms (one of bf16, or two of fp16), `pitch` elements apart.  With `blocks`, blocks of 256 columns (of each term) of
// all rows after one another.
struct Operand {
    const void* base;
    int64_t stride;     // elements from one row to the next
    int rows, columns;  // that exist; with several terms a term's padding exists too
    int terms, pitch;
    int blocks = 0;

    cuuint64_t wide() const { return static_cast<cuuint64_t>(terms > 1 ? terms * static_cast<int64_t>(pitch) : columns); }
    // Rows are read in whole chunks of 64 elements only where no chunk passes the row's end.
    bool chunks() const { return wide() % 64 == 0; }

    // K contiguous: `box_rows` rows of 64 elements of K.
    bool map_k(CUtensorMap* m, unsigned box_rows) const {
        const cuuint64_t dims[3] = {wide(), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(blocks)};
        const cuuint64_t strides[2] = {static_cast<cuuint64_t>(stride) * 2, static_cast<cuuint64_t>(stride) * 2 * rows};
        const cuuint32_t box[3] = {kHeadK, box_rows, 1};
        return encode_map(m, base, blocks ? 3 : 2, dims, strides, box);
    }
    // The other dimension contiguous: 64 rows (of K) of `columns` elements, 64 at a time one after another in shared
    // memory; where that can be one box, it is (a box for each 64 cost 5 % of the products' time).
    bool map_mn(CUtensorMap* m, unsigned box_columns) const {
        const cuuint64_t row_bytes = static_cast<cuuint64_t>(stride) * 2;
        const cuuint64_t dims[4] = {64, static_cast<cuuint64_t>(rows), wide() / 64, static_cast<cuuint64_t>(blocks)};
        const cuuint64_t strides[3] = {row_bytes, 128, row_bytes * rows};
        const cuuint32_t box[4] = {64, kHeadK, box_columns / 64, 1};
        if (chunks()) return encode_map(m, base, blocks ? 4 : 3, dims, strides, box);
        const cuuint64_t flat[2] = {wide(), static_cast<cuuint64_t>(rows)};
        return encode_map(m, base, 2, flat, strides, box);
    }
    // To be written by the epilogue: 32 x 32 values a box.
    bool map_out(CUtensorMap* m, bool floats) const {
        const cuuint64_t row_bytes = static_cast<cuuint64_t>(stride) * (floats ? 4 : 2);
        const cuuint64_t dims[3] = {wide(), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(blocks)};
        const cuuint64_t strides[2] = {row_bytes, row_bytes * rows};
        const cuuint32_t box[3] = {32, 32, 1};
        return encode_map(m, base, blocks ? 3 : 2, dims, strides, box,
                          floats ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
                          floats ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B);
    }
};

template <int KIND, bool A_K, bool B_K, typename T, int CTAS, int N>
bns_status head_gemm_on(int kind, const CUtensorMap& ma, const CUtensorMap& mb, const CUtensorMap& mc, const HeadGemm& g, cudaStream_t stream) {
    static std::atomic<bool> raised[kMaxDevices];
    int device = -1;
    if (cudaGetDevice(&device) != cudaSuccess || device < 0 || device >= kMaxDevices) return BNS_ERR_CUDA;
    auto kernel = head_gemm_kernel<KIND, A_K, B_K, T, CTAS, N>;
    constexpr unsigned smem = HeadRing<CTAS, N>::kSmem;
    if (!raised[device].load(std::memory_order_relaxed)) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) {
            cudaGetLastError();
            return BNS_ERR_CUDA;
        }
        raised[device].store(true, std::memory_order_relaxed);
    }
    const int64_t tiles = static_cast<int64_t>(g.tiles_m) * g.tiles_n * g.splits;
    if (tiles >= int64_t{1} << 30) return BNS_ERR_SHAPE;
    const int64_t workers = sm_count() / CTAS;
    launch(kind, kernel, Shape{static_cast<unsigned>(g.join_parts ? workers : std::min(tiles, workers)) * CTAS, kHeadThreads, CTAS}, smem,
           stream, ma, mb, mc, g);
    return last_error();
}

// CTA pairs with 256 x 256 tiles; single CTAs where the product has no more rows than one of them holds.  The products with
// the logits may have narrow tiles.
template <int KIND, bool A_K, bool B_K, typename T>
bns_status head_gemm(int kind, const Operand& a, const Operand& b, const Operand& c, HeadGemm g, int K, cudaStream_t stream) {
    const int ctas = head_ctas(g.M), columns = KIND == kHeadOut ? kHeadN : head_columns(g.M, g.V);
    const unsigned box_rows = columns == kHeadNarrow ? kHeadNarrowRows : kHeadM, box_columns = static_cast<unsigned>(columns / ctas);
    CUtensorMap ma, mb, mc{};
    if (!(A_K ? a.map_k(&ma, box_rows) : a.map_mn(&ma, box_rows))) return BNS_ERR_CUDA;
    if (!(B_K ? b.map_k(&mb, box_columns) : b.map_mn(&mb, box_columns))) return BNS_ERR_CUDA;
    g.b_chunks = !B_K && b.chunks();
    if (KIND == kHeadGrad && !c.map_out(&mc, false)) return BNS_ERR_CUDA;
    if (KIND == kHeadOut) {
        constexpr bool floats = sizeof(typename T::storage) == 4;
        g.out_boxes = !g.sums && c.stride % (floats ? 4 : 8) == 0;
        if (g.out_boxes && !c.map_out(&mc, floats)) return BNS_ERR_CUDA;
    }
    g.tiles_m = divide_up(g.M, kHeadM * ctas);
    g.tiles_n = divide_up(g.N, columns);
    g.k_blocks = divide_up(K, kHeadK);
    g.pairs = a.terms > 1 ? 3 : 1;
    g.a_pitch = a.pitch;
    g.b_pitch = b.pitch;
    if constexpr (KIND != kHeadOut)
        if (columns == kHeadNarrow) return head_gemm_on<KIND, A_K, B_K, T, 1, kHeadNarrow>(kind, ma, mb, mc, g, stream);
    return ctas == 2 ? head_gemm_on<KIND, A_K, B_K, T, 2, kHeadN>(kind, ma, mb, mc, g, stream)
                     : head_gemm_on<KIND, A_K, B_K, T, 1, kHeadN>(kind, ma, mb, mc, g, stream);
}

// Rows laid out in the workspace: bf16 as they are, fp32 as two fp16 terms scaled by the largest value.
bns_status lay_out(const HeadProblem& p, const void* src, int64_t stride, int rows, void* dst, unsigned* top, float* scale, cudaStream_t stream) {
    const unsigned across = static_cast<unsigned>(divide_up(p.pitch / 8, 32)), down = static_cast<unsigned>(std::min(divide_up(rows, 8), 65535));
    unsigned short* to = static_cast<unsigned short*>(dst);
    if (!p.f32) {
        launch(BNS_KERNEL_HEAD_VECTOR, head_terms_kernel<HeadCopy>, Shape{across, 256, 1, down}, 0, stream, src, stride, rows, p.D, p.pitch,
               to, static_cast<const unsigned*>(nullptr), static_cast<float*>(nullptr));
        return last_error();
    }
    if (cudaMemsetAsync(top, 0, sizeof(unsigned), stream) != cudaSuccess) return BNS_ERR_CUDA;
    const unsigned few = std::max(1u, std::min(down, static_cast<unsigned>(sm_count()) * 8 / across));
    launch(BNS_KERNEL_HEAD_VECTOR, head_top_kernel, Shape{across, 256, 1, few}, 0, stream, static_cast<const float*>(src), stride, rows,
           p.D, top);
    launch(BNS_KERNEL_HEAD_VECTOR, head_terms_kernel<HeadSplit>, Shape{across, 256, 1, down}, 0, stream, src, stride, rows, p.D, p.pitch,
           to, static_cast<const unsigned*>(top), scale);
    return last_error();
}

// x as an operand; a copy is laid out here.
bns_status rows_of_x(const HeadProblem& p, const bns_head* sh, const void* x, char* ws, cudaStream_t stream, Operand& o) {
    o = Operand{x, sh->x_stride, p.T, p.D, 1, 0};
    if (!p.copy_x) return BNS_OK;
    o = Operand{ws + p.off_x, static_cast<int64_t>(p.terms) * p.pitch, p.T, p.pitch, p.terms, p.pitch};
    HeadScalars* s = reinterpret_cast<HeadScalars*>(ws + p.off_scalars);
    return lay_out(p, x, sh->x_stride, p.T, ws + p.off_x, &s->x_top, &s->x_scale, stream);
}

// Rows [first, first + count) of w.
bns_status rows_of_w(const HeadProblem& p, const bns_head* sh, const void* w, int first, int count, char* ws, cudaStream_t stream, Operand& o) {
    const char* from = static_cast<const char*>(w) + static_cast<int64_t>(first) * sh->w_stride * elem_bytes(p.dtype);
    o = Operand{from, sh->w_stride, count, p.D, 1, 0};
    if (!p.copy_w) return BNS_OK;
    o = Operand{ws + p.off_w, static_cast<int64_t>(p.terms) * p.pitch, count, p.pitch, p.terms, p.pitch};
    HeadScalars* s = reinterpret_cast<HeadScalars*>(ws + p.off_scalars);
    return lay_out(p, from, sh->w_stride, count, ws + p.off_w, &s->w_top, &s->w_scale, stream);
}

// The few rows' kernels: the logits' statistics, or the gradients.
template <int ROWS, bool WORDS, bool GRAD>
bns_status few_logits(const HeadFew& a, cudaStream_t stream) {
    static std::atomic<bool> raised[kMaxDevices];
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess || device < 0 || device >= kMaxDevices) return BNS_ERR_CUDA;
    auto kernel = head_few_logits_kernel<ROWS, WORDS, GRAD>;
    if (!raised[device].load(std::memory_order_relaxed)) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kFewSharedMost)) != cudaSuccess) {
            cudaGetLastError();
            return BNS_ERR_CUDA;
        }
        raised[device].store(true, std::memory_order_relaxed);
    }
    launch(GRAD ? BNS_KERNEL_HEAD_GRADIENT : BNS_KERNEL_HEAD_LOGITS, kernel,
           Shape{static_cast<unsigned>(sm_count()), FewShape<ROWS>::kThreads}, static_cast<size_t>(ROWS) * a.pitch * sizeof(float), stream, a);
    return last_error();
}
template <int ROWS, bool WORDS>
bns_status few_head_of(const HeadProblem& p, HeadFew a, char* ws, bool backward, cudaStream_t stream) {
    a.status = reinterpret_cast<unsigned*>(ws);
    if (ROWS > kFewRowsBackward || !backward) {
        a.partial = reinterpret_cast<float2*>(ws + p.off_partial);
        a.target_logit = reinterpret_cast<float*>(ws + p.off_logit);
        return few_logits<ROWS, WORDS, false>(a, stream);
    }
    if constexpr (ROWS <= kFewRowsBackward) {
        a.G = reinterpret_cast<float*>(ws + p.off_G);
        a.sums = reinterpret_cast<float*>(ws + p.off_sums);
        a.chunks = p.few_chunks;
        a.per = p.few_per;
        a.groups = p.few_groups;
        const bns_status st = few_logits<ROWS, WORDS, true>(a, stream);
        if (st != BNS_OK) return st;
        launch(BNS_KERNEL_HEAD_PRODUCT, head_few_products_kernel<ROWS, WORDS>,
               Shape{static_cast<unsigned>(p.few_chunks * p.few_groups), static_cast<unsigned>(p.few_threads)}, 0, stream, a);
        const int64_t elements = static_cast<int64_t>(p.T) * p.D;
        launch(BNS_KERNEL_HEAD_VECTOR, head_few_join_kernel, Shape{static_cast<unsigned>(divide_up<int64_t>(elements, 32)), 256}, 0, stream, a);
    }
    return last_error();
}
template <bool WORDS>
bns_status few_head_in(const HeadProblem& p, const HeadFew& a, char* ws, bool backward, cudaStream_t stream) {
    switch (p.few) {
        case 1: return few_head_of<1, WORDS>(p, a, ws, backward, stream);
        case 2: return few_head_of<2, WORDS>(p, a, ws, backward, stream);
        case 4: return few_head_of<4, WORDS>(p, a, ws, backward, stream);
        case 8: return few_head_of<8, WORDS>(p, a, ws, backward, stream);
        case 16: return few_head_of<16, WORDS>(p, a, ws, backward, stream);
        default: return few_head_of<32, WORDS>(p, a, ws, backward, stream);
    }
}
bns_status few_head(const HeadProblem& p, const bns_head* sh, HeadFew a, char* ws, bool backward, cudaStream_t stream) {
    a.x_stride = sh->x_stride;
    a.w_stride = sh->w_stride;
    a.target64 = sh->target_is_int64;
    a.T = p.T;
    a.V = p.V;
    a.D = p.D;
    a.pitch = few_pitch(p.D, p.few_words);
    return p.few_words ? few_head_in<true>(p, a, ws, backward, stream) : few_head_in<false>(p, a, ws, backward, stream);
}

// ------------------------------------------------------------------------------------ distillation
bns_status check_distillation(const bns_distillation* sh) {
    if (!sh) return BNS_ERR_NULL;
    if (sh->rows < 0 || sh->vocabulary <= 0 || sh->vocabulary > 1 << 30 || sh->entries < 1 || sh->entries > kDistillMaxEntries ||
        sh->stride < sh->vocabulary || !(sh->temperature >= 1e-38f) || sh->temperature > 1e30f)    // log2(e) / temperature is finite
        return BNS_ERR_SHAPE;
    if (!known(sh->dtype) || !known(sh->teacher_dtype)) return BNS_ERR_DTYPE;
    return BNS_OK;
}

template <typename WHAT>
bns_status distill(const bns_distillation* sh, Distill a, cudaStream_t stream) {
    const size_t eb = elem_bytes(sh->dtype);
    if (!aligned(a.z, eb) || !aligned(a.dz, eb) || !aligned(a.teacher, elem_bytes(sh->teacher_dtype)) ||
        !aligned(a.index, sh->index_is_int64 ? 8 : 4) || !aligned(a.loss, 4) || !aligned(a.lse, 4) || !aligned(a.dloss, 4) ||
        !aligned(a.lse_in, 4))
        return BNS_ERR_ALIGN;
    a.z_stride = sh->stride;
    a.rows = sh->rows;
    a.V = sh->vocabulary;
    a.K = sh->entries;
    a.index64 = sh->index_is_int64;
    a.teacher_bf16 = sh->teacher_dtype == BNS_BF16;
    a.tau = sh->temperature;
    a.c = static_cast<float>(1.4426950408889634 / static_cast<double>(sh->temperature));
    constexpr bool backward = __is_same(WHAT, DistillBackward);
    const int vectors = std::max(1, a.V / (16 / static_cast<int>(eb)));
    const int64_t rows = sh->rows;
    // short rows take small blocks (8192 x 1000 bf16: 38 us against 100)
    const bool small = vectors <= kDistillSmall * 8 && a.K <= kDistillSmall * kDistillOwn && rows > 2 * sm_count();
    // A row that is read twice should still be in L2 the second time: long ones go over two blocks, so that half as many
    // are in flight.  Per 4096 rows with one block / two: bf16 50257 (98 KB) 179 / 248 us, 100277 (196 KB) 328 / 370, 112000
    // (219 KB) 376 / 385, 128256 (250 KB) 451 / 422, 200064 733 / 673; fp32 50257 (196 KB) 316 / 354, 65536
    // (256 KB) 458 / 401.
    const size_t row_bytes = static_cast<size_t>(a.V) * eb;
    a.parts = __is_same(WHAT, DistillStep) && row_bytes > (size_t{224} << 10) ? 2 : 1;
    // few rows are spread over the SMs
    while (a.parts < kDistillParts && rows * (a.parts + 1) <= 2 * sm_count() && vectors > a.parts * kDistillThreads) ++a.parts;
    a.per = divide_up(vectors, a.parts);
    if (rows * a.parts >= int64_t{1} << 31) return BNS_ERR_SHAPE;
    const unsigned parts = static_cast<unsigned>(a.parts), grid = static_cast<unsigned>(rows) * parts, cluster = backward ? 1 : parts;
    BNS_LM_BY_TYPE(sh->dtype, {
        if (small)
            launch(BNS_KERNEL_DISTILL, distill_kernel<T, WHAT, kDistillSmall>, Shape{grid, kDistillSmall, cluster}, 0, stream, a);
        else
            launch(BNS_KERNEL_DISTILL, distill_kernel<T, WHAT, kDistillThreads>, Shape{grid, kDistillThreads, cluster}, 0, stream, a);
    });
    return last_error();
}

}  // namespace

namespace bns {

int g_head_piece = 0;

bns_status lm_wait_timeouts(uint32_t* count, cudaStream_t stream) {
    if (cudaMemcpyFromSymbolAsync(count, g_lm_timeouts, sizeof(uint32_t), 0, cudaMemcpyDeviceToHost, stream) != cudaSuccess)
        return BNS_ERR_CUDA;
    return cudaStreamSynchronize(stream) == cudaSuccess ? BNS_OK : BNS_ERR_CUDA;
}

}  // namespace bns

extern "C" {

bns_status bns_rms_norm_forward(const bns_rows* shape, const void* x, int64_t x_stride, const void* residual,
                                int64_t residual_stride, const float* weight, float eps, void* y, void* h, float* rstd,
                                void* cuda_stream) {
    const bns_status st = check_rows(shape);
    if (st != BNS_OK) return st;
    return rms_forward<RmsNone>(shape, x, x_stride, residual, residual_stride, weight, eps, y, nullptr, h, rstd, cuda_stream);
}

bns_status bns_rms_norm_forward_quantized(const bns_rows* shape, const void* x, int64_t x_stride, const void* residual,
                                          int64_t residual_stride, const float* weight, float eps, int group, void* q,
                                          float* scales, void* h, float* rstd, void* cuda_stream) {
    const bns_status st = check_rows(shape);
    if (st != BNS_OK) return st;
    if (group != 0 && group != kRmsGroup) return BNS_ERR_RULE;
    if (group == 0)
        return rms_forward<RmsRowScale>(shape, x, x_stride, residual, residual_stride, weight, eps, q, scales, h, rstd, cuda_stream);
    return rms_forward<RmsGroupScale>(shape, x, x_stride, residual, residual_stride, weight, eps, q, scales, h, rstd, cuda_stream);
}

size_t bns_rms_norm_workspace_bytes(const bns_rows* shape) {
    if (check_rows(shape) != BNS_OK) return 0;
    return kHeaderBytes + align_up(static_cast<size_t>(rms_backward_blocks(shape->rows)) * shape->columns * sizeof(float));
}

bns_status bns_rms_norm_backward(const bns_rows* shape, const void* dy, int64_t dy_stride, const void* h, int64_t h_stride,
                                 const float* weight, const float* rstd, const void* dh, int64_t dh_stride, void* dx,
                                 float* dweight, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    const bns_status st = check_rows(shape);
    if (st != BNS_OK) return st;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (!dweight) return BNS_ERR_NULL;
    if (shape->rows == 0)
        return cudaMemsetAsync(dweight, 0, sizeof(float) * shape->columns, stream) == cudaSuccess ? BNS_OK : BNS_ERR_CUDA;
    if (!dy || !h || !weight || !rstd || !dx) return BNS_ERR_NULL;
    if (dy_stride < shape->columns || h_stride < shape->columns || (dh && dh_stride < shape->columns)) return BNS_ERR_SHAPE;
    const size_t eb = elem_bytes(shape->dtype);
    if (!aligned(dy, eb) || !aligned(h, eb) || !aligned(dh, eb) || !aligned(dx, eb) || !aligned(weight, 4) ||
        !aligned(rstd, 4) || !aligned(dweight, 4))
        return BNS_ERR_ALIGN;
    if (!workspace_fits(workspace, workspace_bytes, bns_rms_norm_workspace_bytes(shape))) return BNS_ERR_WORKSPACE;
    VectorRule rule(shape->columns, static_cast<int>(eb));
    rule.tensor(dy, dy_stride);
    rule.tensor(h, h_stride);
    rule.tensor(dh, dh_stride);
    rule.tensor(dx, shape->columns);
    if (!aligned(weight, 16) && rule.kind == VectorRule::kAligned) rule.kind = VectorRule::kPhase;
    const RmsPlan pl = plan_rms(shape->rows, shape->columns, shape->dtype, rule.kind, true);
    float* partial = reinterpret_cast<float*>(static_cast<char*>(workspace) + kHeaderBytes);
    const RmsBackward a{dy, h, dh, weight, rstd, dx, partial, shape->rows, dy_stride, h_stride, dh_stride, shape->columns,
                        1.f / static_cast<float>(shape->columns)};
    const Shape grid{pl.grid, pl.threads};
    BNS_LM_BY_TYPE_V(shape->dtype, pl.V, (rms_backward<T, V>(pl, grid, a, stream)));
    launch(BNS_KERNEL_RMS_BACKWARD, rms_dweight_kernel, Shape{static_cast<unsigned>(divide_up(shape->columns, 32)), 1024}, 0, stream,
           partial, static_cast<int>(pl.grid), shape->columns, dweight);
    return last_error();
}

size_t bns_linear_cross_entropy_workspace_bytes(const bns_head* shape, int backward) {
    if (check_head(shape) != BNS_OK) return 0;
    return plan_head(shape, backward != 0).total;
}

bns_status bns_linear_cross_entropy_forward(const bns_head* shape, const void* x, const void* w, const void* target, float* loss,
                                            float* lse, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    bns_status st = check_head(shape);
    if (st != BNS_OK) return st;
    if (!w) return BNS_ERR_NULL;
    if (shape->rows > 0 && (!x || !target || !loss || !lse)) return BNS_ERR_NULL;
    if (!aligned(x, 16) || !aligned(w, 16) || !aligned(target, shape->target_is_int64 ? 8 : 4) || !aligned(loss, 4) ||
        !aligned(lse, 4))
        return BNS_ERR_ALIGN;
    const HeadProblem p = plan_head(shape, false);
    if (!workspace_fits(workspace, workspace_bytes, p.total)) return BNS_ERR_WORKSPACE;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    char* ws = static_cast<char*>(workspace);
    if (p.T == 0) return cudaMemsetAsync(ws, 0, sizeof(uint32_t), stream) == cudaSuccess ? BNS_OK : BNS_ERR_CUDA;
    if (p.few) {
        HeadFew a{};
        a.x = static_cast<const float*>(x);
        a.w = static_cast<const float*>(w);
        a.target = target;
        st = few_head(p, shape, a, ws, false, stream);
        if (st != BNS_OK) return st;
        launch(BNS_KERNEL_HEAD_VECTOR, head_join_kernel, Shape{1, 1024}, 0, stream, reinterpret_cast<const float2*>(ws + p.off_partial),
               sm_count(), p.T, reinterpret_cast<const float*>(ws + p.off_logit), target, shape->target_is_int64, p.V, loss, lse,
               reinterpret_cast<unsigned*>(ws));
        return last_error();
    }
    Operand xs, rows;
    st = rows_of_x(p, shape, x, ws, stream, xs);
    if (st != BNS_OK) return st;
    HeadScalars* scalars = reinterpret_cast<HeadScalars*>(ws + p.off_scalars);
    float2* partial = reinterpret_cast<float2*>(ws + p.off_partial);
    int tiles = 0;
    for (int first = 0; first < p.V; first += p.piece) {
        const int count = std::min(p.piece, p.V - first);
        st = rows_of_w(p, shape, w, first, count, ws, stream, rows);
        if (st != BNS_OK) return st;
        HeadGemm g{};
        g.M = p.T;
        g.N = count;
        g.splits = 1;
        g.target = target;
        g.target64 = shape->target_is_int64;
        g.first = first;
        g.V = p.V;
        g.partial = partial + static_cast<size_t>(tiles) * p.T;
        g.target_logit = reinterpret_cast<float*>(ws + p.off_logit);
        g.status = first == 0 ? reinterpret_cast<unsigned*>(ws) : nullptr;
        g.a_scale = &scalars->x_scale;
        g.b_scale = &scalars->w_scale;
        BNS_LM_BY_TYPE(p.dtype, (st = head_gemm<kHeadLse, true, true, T>(BNS_KERNEL_HEAD_LOGITS, xs, rows, Operand{}, g, p.D, stream)));
        if (st != BNS_OK) return st;
        tiles += 2 * divide_up(count, head_columns(p.T, p.V));
    }
    launch(BNS_KERNEL_HEAD_VECTOR, head_join_kernel, Shape{static_cast<unsigned>(divide_up(p.T, 32)), 1024}, 0, stream, partial, tiles, p.T,
           reinterpret_cast<const float*>(ws + p.off_logit), target, shape->target_is_int64, p.V, loss, lse,
           reinterpret_cast<unsigned*>(ws));
    return last_error();
}

bns_status bns_linear_cross_entropy_backward(const bns_head* shape, const void* x, const void* w, const void* target,
                                             const float* lse, const float* dloss, void* dx, void* dw, void* workspace,
                                             size_t workspace_bytes, void* cuda_stream) {
    bns_status st = check_head(shape);
    if (st != BNS_OK) return st;
    if (!w || !dw) return BNS_ERR_NULL;
    if (shape->rows > 0 && (!x || !target || !lse || !dloss || !dx)) return BNS_ERR_NULL;
    if (!aligned(x, 16) || !aligned(w, 16) || !aligned(dx, 16) || !aligned(dw, 16) ||
        !aligned(target, shape->target_is_int64 ? 8 : 4) || !aligned(lse, 4) || !aligned(dloss, 4))
        return BNS_ERR_ALIGN;
    const HeadProblem p = plan_head(shape, true);
    if (!workspace_fits(workspace, workspace_bytes, p.total)) return BNS_ERR_WORKSPACE;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    char* ws = static_cast<char*>(workspace);
    const size_t eb = elem_bytes(p.dtype);
    if (p.T == 0)
        return cudaMemsetAsync(ws, 0, sizeof(uint32_t), stream) == cudaSuccess &&
                       cudaMemsetAsync(dw, 0, eb * p.V * p.D, stream) == cudaSuccess
                   ? BNS_OK
                   : BNS_ERR_CUDA;
    if (p.few) {
        HeadFew a{};
        a.x = static_cast<const float*>(x);
        a.w = static_cast<const float*>(w);
        a.target = target;
        a.lse = lse;
        a.dloss = dloss;
        a.dx = static_cast<float*>(dx);
        a.dw = static_cast<float*>(dw);
        return few_head(p, shape, a, ws, true, stream);
    }
    Operand xs, rows;
    st = rows_of_x(p, shape, x, ws, stream, xs);
    if (st != BNS_OK) return st;
    HeadScalars* scalars = reinterpret_cast<HeadScalars*>(ws + p.off_scalars);
    float* unit = &scalars->unit;
    // few rows: each warp finds the unit itself, under the first tile's copies; a launch costs some 3 us
    const bool find_unit = p.T <= 1024;
    if (!find_unit)
        launch(BNS_KERNEL_HEAD_VECTOR, head_unit_kernel, Shape{1, 1024}, 0, stream, target, shape->target_is_int64, dloss, p.T, p.V, unit,
               reinterpret_cast<unsigned*>(ws));
    float* sums = p.splits > 1 || p.pieces > 1 ? reinterpret_cast<float*>(ws + p.off_sums) : nullptr;
    for (int first = 0; first < p.V; first += p.piece) {
        const int count = std::min(p.piece, p.V - first);
        st = rows_of_w(p, shape, w, first, count, ws, stream, rows);
        if (st != BNS_OK) return st;
        HeadGemm g{};
        g.M = p.T;
        g.N = count;
        g.splits = 1;
        g.target = target;
        g.target64 = shape->target_is_int64;
        g.first = first;
        g.V = p.V;
        g.lse = lse;
        g.dloss = dloss;
        g.unit = unit;
        g.find_unit = find_unit;
        g.status = reinterpret_cast<unsigned*>(ws);
        g.a_scale = &scalars->x_scale;
        g.b_scale = &scalars->w_scale;
        const Operand G{ws + p.off_G, static_cast<int64_t>(p.terms) * kHeadN, p.T, kHeadN, p.terms, kHeadN, divide_up(count, kHeadN)};
        BNS_LM_BY_TYPE(p.dtype, (st = head_gemm<kHeadGrad, true, true, T>(BNS_KERNEL_HEAD_GRADIENT, xs, rows, G, g, p.D, stream)));
        if (st != BNS_OK) return st;
        HeadGemm o{};
        o.M = p.T;
        o.N = p.D;
        o.splits = p.splits;
        o.unit = unit;
        o.b_scale = &scalars->w_scale;
        o.out = dx;
        o.out_stride = p.D;
        o.sums = sums;
        o.add = first > 0;
        o.last = p.splits == 1 && first + count == p.V;
        BNS_LM_BY_TYPE(p.dtype, (st = head_gemm<kHeadOut, true, false, T>(BNS_KERNEL_HEAD_PRODUCT, G, rows, Operand{dx, p.D, p.T, p.D, 1, 0}, o, count, stream)));
        if (st != BNS_OK) return st;
        HeadGemm q{};
        q.M = count;
        q.N = p.D;
        q.splits = 1;
        q.unit = unit;
        if (p.splits > 1 && first + count == p.V) {
            q.join_sums = sums;
            q.join_out = dx;
            q.join_parts = p.splits;
            q.join_total = static_cast<int64_t>(p.T) * p.D;
        }
        q.b_scale = &scalars->x_scale;
        q.out = static_cast<char*>(dw) + static_cast<size_t>(first) * p.D * eb;
        q.out_stride = p.D;
        BNS_LM_BY_TYPE(p.dtype, (st = head_gemm<kHeadOut, false, false, T>(BNS_KERNEL_HEAD_PRODUCT, G, xs, Operand{q.out, p.D, count, p.D, 1, 0}, q, p.T, stream)));
        if (st != BNS_OK) return st;
    }
    return last_error();
}

bns_status bns_topk_distillation_forward(const bns_distillation* shape, const void* logits, const void* teacher, const void* index,
                                         float* loss, float* lse, void* cuda_stream) {
    const bns_status st = check_distillation(shape);
    if (st != BNS_OK) return st;
    if (shape->rows == 0) return BNS_OK;
    if (!logits || !teacher || !index || !loss || !lse) return BNS_ERR_NULL;
    Distill a{};
    a.z = logits;
    a.teacher = teacher;
    a.index = index;
    a.loss = loss;
    a.lse = lse;
    return distill<DistillForward>(shape, a, static_cast<cudaStream_t>(cuda_stream));
}

bns_status bns_topk_distillation_backward(const bns_distillation* shape, const void* logits, const void* teacher, const void* index,
                                          const float* lse, const float* dloss, void* dlogits, int64_t dlogits_stride,
                                          void* cuda_stream) {
    const bns_status st = check_distillation(shape);
    if (st != BNS_OK) return st;
    if (shape->rows == 0) return BNS_OK;
    if (!logits || !teacher || !index || !lse || !dloss || !dlogits) return BNS_ERR_NULL;
    if (dlogits_stride < shape->vocabulary) return BNS_ERR_SHAPE;
    Distill a{};
    a.z = logits;
    a.teacher = teacher;
    a.index = index;
    a.lse_in = lse;
    a.dloss = dloss;
    a.dz = dlogits;
    a.dz_stride = dlogits_stride;
    return distill<DistillBackward>(shape, a, static_cast<cudaStream_t>(cuda_stream));
}

bns_status bns_topk_distillation_step(const bns_distillation* shape, const void* logits, const void* teacher, const void* index,
                                      const float* dloss, float* loss, void* dlogits, int64_t dlogits_stride,
                                      void* cuda_stream) {
    const bns_status st = check_distillation(shape);
    if (st != BNS_OK) return st;
    if (shape->rows == 0) return BNS_OK;
    if (!logits || !teacher || !index || !dloss || !loss || !dlogits) return BNS_ERR_NULL;
    if (dlogits_stride < shape->vocabulary) return BNS_ERR_SHAPE;
    Distill a{};
    a.z = logits;
    a.teacher = teacher;
    a.index = index;
    a.dloss = dloss;
    a.loss = loss;
    a.dz = dlogits;
    a.dz_stride = dlogits_stride;
    return distill<DistillStep>(shape, a, static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
