// Host side of more language-model operators declared in include/bns.h: log probabilities of given tokens, norm + rotation
// of heads, norm over many gradients and clipping.  Checks, plans and launches; nothing here allocates device memory or
// synchronises the host.
#include <algorithm>

#include "bns_clip_kernels.cuh"
#include "bns_lm_host.h"
#include "bns_logp_kernels.cuh"
#include "bns_rotary_kernels.cuh"

namespace {

using namespace bns;

// ------------------------------------------------------------------------------------ token log probabilities
bns_status check_log_probs(const bns_token_log_probs* sh) {
    if (!sh) return BNS_ERR_NULL;
    if (sh->rows < 0 || sh->vocabulary <= 0 || sh->vocabulary > 1 << 30 || sh->entries < 0 || sh->entries > kLogpMaxTop ||
        sh->entries > sh->vocabulary || sh->stride < sh->vocabulary || !(sh->temperature >= 0.999e-6f) || sh->temperature > 1.001e6f)
        return BNS_ERR_SHAPE;
    if (!known(sh->dtype)) return BNS_ERR_DTYPE;
    return BNS_OK;
}

LogProbs log_probs_of(const bns_token_log_probs* sh, const void* logits, const void* token) {
    LogProbs a{};
    a.z = logits;
    a.token = token;
    a.z_stride = sh->stride;
    a.rows = sh->rows;
    a.V = sh->vocabulary;
    a.K = sh->entries;
    a.token64 = sh->token_is_int64;
    a.tau = sh->temperature;
    a.c = static_cast<float>(1.4426950408889634 / static_cast<double>(sh->temperature));
    return a;
}

template <typename T, int THREADS>
void logp_forward(const LogProbs& a, Shape shape, cudaStream_t stream) {
    if (a.K)
        launch(BNS_KERNEL_LOGP, logp_forward_kernel<T, true, THREADS>, shape, sizeof(TopShared<THREADS>), stream, a);
    else
        launch(BNS_KERNEL_LOGP, logp_forward_kernel<T, false, THREADS>, shape, 0, stream, a);
}

// ------------------------------------------------------------------------------------ heads' norm + rotation
bns_status check_head_norm(const bns_head_norm* sh) {
    if (!sh) return BNS_ERR_NULL;
    if (sh->batch < 0 || sh->length < 0 || static_cast<int64_t>(sh->batch) * sh->length > 0x7fffffff || sh->q_heads < 1 ||
        sh->q_heads > 32767 || sh->k_heads < 0 || sh->k_heads > 32767 || sh->head_dim < 2 || sh->head_dim > 1024 || sh->rotary < 2 ||
        sh->rotary > sh->head_dim || sh->rotary % 2 || sh->positions < 1 || !(sh->eps > 0.f))
        return BNS_ERR_SHAPE;
    for (int i = 0; i < 3; ++i)
        if (sh->q_strides[i] < 0 || (sh->k_heads && sh->k_strides[i] < 0)) return BNS_ERR_SHAPE;
    if (!known(sh->dtype)) return BNS_ERR_DTYPE;
    return BNS_OK;
}

struct HeadPlan {
    int V;           // elements of a vector
    int lanes;       // that share a head
    bool wide;       // more vectors than two for each of 32 lanes
    int words;       // angles (1) and weights (2) may be loaded in 16-byte words
};

// Whether all of the heads may be moved in vectors of V elements.
bool in_vectors(const bns_head_norm* sh, const int64_t* strides, int heads, const void* x, const void* dy, const void* y, int V) {
    const size_t bytes = static_cast<size_t>(V) * elem_bytes(sh->dtype);
    return aligned(x, bytes) && aligned(dy, bytes) && aligned(y, bytes) && (sh->batch == 1 || strides[0] % V == 0) &&
           (sh->length == 1 || strides[1] % V == 0) && (heads == 1 || strides[2] % V == 0);
}

HeadPlan plan_heads(const bns_head_norm* sh, const HeadNorm& a) {
    HeadPlan pl{};
    pl.V = 16 / elem_bytes(sh->dtype);
    while (pl.V > 1 && (sh->rotary / 2 % pl.V || (sh->head_dim - sh->rotary) % pl.V ||
                        !in_vectors(sh, sh->q_strides, sh->q_heads, a.q.x, a.q.dy, a.q.y, pl.V) ||
                        (sh->k_heads && !in_vectors(sh, sh->k_strides, sh->k_heads, a.k.x, a.k.dy, a.k.y, pl.V))))
        pl.V /= 2;
    auto share = [&] {
        const int units = sh->rotary / 2 / pl.V + divide_up(sh->head_dim - sh->rotary, 2 * pl.V);
        pl.lanes = 1;
        while (pl.lanes < 32 && pl.lanes < units) pl.lanes *= 2;
        pl.wide = units > 32;
    };
    share();
    // A warp with little to do at a position waits for angles and weights: half as large vectors make these half as many for a lane.  With more heads
    // than a few rounds of a warp, queries' and keys' together, or for the gradient more than one round of the smaller vectors each, that only holds
    // while there is no more than two 16-byte vectors for each thread that the SMs hold.  16384 positions (65536 in parentheses), bf16, vectors of
    // 16 / 8 bytes, forward: 4 + 1 heads of 64 20.0 / 16.1 us (76 / 61), 16 + 4 of 64 24.5 / 22.9 (96 / 92), 8 + 8 of 64 21.6 / 20.6 (85 / 80), 4 + 1 of 128 22.2 / 18.6
    // (84 / 72), but 32 + 32 of 32 28.3 / 30.3 (112 / 119) and 16 + 16 of 64 28.9 / 30.9 (115 / 123); 1024 positions of the last two 4.7 / 3.9 and 4.8 / 3.9.
    // Gradient: 4 + 1 of 64 24.8 / 19.9 (84 / 70), 8 + 8 of 32 25.1 / 19.3 (85 / 71), but 8 + 8 of 64 26.8 / 28.7 (92 / 105) and 16 + 16 of 32 26.6 / 27.6
    // (90 / 101); 1024 positions of the last two 7.0 / 5.9 and 7.5 / 6.1.
    const int slots = 32 / pl.lanes, rounds = divide_up(sh->q_heads, slots), all_rounds = rounds + divide_up(sh->k_heads, slots);
    const bool spare = a.tokens * (sh->q_heads + sh->k_heads) * sh->head_dim <= int64_t{sm_count()} * 2048 * 16;
    const bool one_each = 2 * std::max(sh->q_heads, sh->k_heads) <= slots;
    if (pl.V == 8 && (a.q.dy ? rounds == 1 && pl.lanes <= 4 && (one_each || spare) : rounds * pl.lanes <= 8 && (all_rounds <= 3 || spare))) {
        pl.V = 4;
        share();
    }
    pl.words = (aligned(a.cos, 16) && aligned(a.sin, 16) && sh->rotary / 2 % 4 == 0 ? 1 : 0) |
               (aligned(a.q.weight, 16) && aligned(a.k.weight, 16) ? 2 : 0);
    return pl;
}

HeadNorm problem_of(const bns_head_norm* sh, const float* cos, const float* sin, const void* position) {
    HeadNorm a{};
    a.cos = cos;
    a.sin = sin;
    a.position = position;
    a.tokens = static_cast<int64_t>(sh->batch) * sh->length;
    a.length = sh->length;
    a.D = sh->head_dim;
    a.R = sh->rotary;
    a.positions = sh->positions;
    a.position64 = sh->position_is_int64;
    a.interleaved = sh->interleaved;
    a.eps = sh->eps;
    a.inv_D = 1.f / static_cast<float>(sh->head_dim);
    // one batch, or batches that follow one another at the positions' stride, need no division
    const auto follows = [&](const int64_t* s) { return s[0] == s[1] * sh->length; };
    a.batched = sh->batch > 1 && !(follows(sh->q_strides) && (sh->k_heads == 0 || follows(sh->k_strides)));
    auto rows = [&](HeadRows& r, const int64_t* strides, int heads) {
        r.batch_stride = strides[0];
        r.position_stride = strides[1];
        r.head_stride = strides[2];
        r.heads = heads;
    };
    rows(a.q, sh->q_strides, sh->q_heads);
    rows(a.k, sh->k_strides, sh->k_heads);
    return a;
}

// Blocks of the gradient kernel at the most, each of which leaves a row of sums: what fits the SMs, or one for each chunk of heads.
constexpr int kHeadBlocks = 4;
constexpr double kHeadPosition = 1.5;    // (none / 1 / 2 / 5: 16384 positions of 16 + 4 heads of 80 bf16 62 / 50 / 50 / 52 us)
int head_norm_blocks(const bns_head_norm* sh) { return sh->q_heads + sh->k_heads + sm_count() * kHeadBlocks; }

// Rounds over the heads that a warp makes at one position, and the chunks that this makes, as even as they come out.
void share_heads(HeadRows& r, int slots, int most) {
    const int all = divide_up(r.heads, slots);
    r.chunks = divide_up(all, most);
    r.rounds = r.chunks ? divide_up(all, r.chunks) : 1;
}

// Forward: many rounds amortise the angles and weights that a warp fetches first (8192 positions of 32 + 8 heads of 128 bf16, up
// to 4 / 8 / 16 rounds: 35 / 31 / 31 us); few spread a small batch over the SMs (512 positions, aiming at 24 / 32 / 48 warps
// an SM: 4.2 / 3.9 / 5.2 us).
constexpr int kHeadWarps = 32, kHeadRounds = 16;
void plan_forward(HeadNorm& a, int slots) {
    const int64_t all = a.tokens * (divide_up(a.q.heads, slots) + divide_up(a.k.heads, slots));
    const int most = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(divide_up<int64_t>(all, kHeadWarps * sm_count()), kHeadRounds)));
    share_heads(a.q, slots, most);
    share_heads(a.k, slots, most);
}

// Gradient: blocks stay, and each chunk has some of them, in proportion to the time of a position: its rounds and what else a
// position takes, some kHeadPosition rounds.  The number of rounds is the one with which the last warp is done first.
void plan_backward(HeadNorm& a, int slots) {
    const int64_t tokens = divide_up<int64_t>(a.tokens, kRotaryWarps);
    HeadNorm best = a;
    double least = 1e300;
    for (int most = kHeadRounds; most >= 1; --most) {
        share_heads(a.q, slots, most);
        share_heads(a.k, slots, most);
        const double all = a.q.chunks * (a.q.rounds + kHeadPosition) + a.k.chunks * (a.k.rounds + kHeadPosition);
        double cost = 0;
        for (HeadRows* r : {&a.q, &a.k}) {
            if (!r->chunks) continue;
            r->blocks = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(tokens, static_cast<int64_t>(sm_count() * kHeadBlocks * (r->rounds + kHeadPosition) / all))));
            cost = std::max(cost, static_cast<double>(divide_up<int64_t>(tokens, r->blocks)) * (r->rounds + kHeadPosition));
        }
        if (cost < least) {
            least = cost;
            best = a;
        }
    }
    a = best;
}

// Blocks of a gradient launch that leave sums of the queries' and of the keys' weight.
struct HeadBlocks {
    int q, k;
};

template <typename T, int V, bool BACKWARD, bool INTERLEAVED>
HeadBlocks head_norm_of_vectors(HeadNorm a, const HeadPlan& pl, cudaStream_t stream) {
    // rounds in flight: two, but one where the gradient's registers hold no more (one / two: bf16 58 / 60 us, fp32 93 / 89)
    constexpr int kWide = 1024 / (64 * V), kDepth = BACKWARD && V == 8 ? 1 : 2;
    const int slots = 32 / pl.lanes;
    Shape shape{0, kRotaryWarps * 32};
    if (BACKWARD) {
        plan_backward(a, slots);
        shape.grid = static_cast<unsigned>(a.q.chunks * a.q.blocks + a.k.chunks * a.k.blocks);
    } else {
        plan_forward(a, slots);
        shape.grid = static_cast<unsigned>(divide_up<int64_t>(a.tokens, kRotaryWarps));
        shape.grid_y = static_cast<unsigned>(a.q.chunks + a.k.chunks);
    }
    if constexpr (BACKWARD) {
        const size_t smem = static_cast<size_t>(kRotaryWarps) * a.D * sizeof(float);
        if (pl.wide)
            launch(BNS_KERNEL_HEAD_NORM, head_norm_backward_kernel<T, V, kWide, 1, INTERLEAVED>, shape, smem, stream, a, pl.lanes, pl.words);
        else
            launch(BNS_KERNEL_HEAD_NORM, head_norm_backward_kernel<T, V, 1, kDepth, INTERLEAVED>, shape, smem, stream, a, pl.lanes, pl.words);
    } else {
        if (pl.wide)
            launch(BNS_KERNEL_HEAD_NORM, head_norm_forward_kernel<T, V, kWide, 1, INTERLEAVED>, shape, 0, stream, a, pl.lanes, pl.words);
        else
            launch(BNS_KERNEL_HEAD_NORM, head_norm_forward_kernel<T, V, 1, kDepth, INTERLEAVED>, shape, 0, stream, a, pl.lanes, pl.words);
    }
    return HeadBlocks{a.q.chunks * a.q.blocks, a.k.chunks * a.k.blocks};
}

template <typename T, int V, bool BACKWARD>
HeadBlocks head_norm_of(const HeadNorm& a, const HeadPlan& pl, cudaStream_t stream) {
    // a vector of one element holds a pair either way
    if constexpr (V > 1) {
        if (!a.interleaved) return head_norm_of_vectors<T, V, BACKWARD, false>(a, pl, stream);
    }
    return head_norm_of_vectors<T, V, BACKWARD, true>(a, pl, stream);
}

template <bool BACKWARD>
HeadBlocks head_norm(const HeadNorm& a, const HeadPlan& pl, int dtype, cudaStream_t stream) {
    if (dtype == BNS_F32) {
        if (pl.V == 4) return head_norm_of<F32, 4, BACKWARD>(a, pl, stream);
        if (pl.V == 2) return head_norm_of<F32, 2, BACKWARD>(a, pl, stream);
        return head_norm_of<F32, 1, BACKWARD>(a, pl, stream);
    }
    if (pl.V == 8) return head_norm_of<BF16, 8, BACKWARD>(a, pl, stream);
    if (pl.V == 4) return head_norm_of<BF16, 4, BACKWARD>(a, pl, stream);
    if (pl.V == 2) return head_norm_of<BF16, 2, BACKWARD>(a, pl, stream);
    return head_norm_of<BF16, 1, BACKWARD>(a, pl, stream);
}

// ------------------------------------------------------------------------------------ gradients
// Tensors that a launch takes: the kernels' arguments hold 32,764 bytes.  Few take a small list (the arguments of a launch are
// copied).
constexpr int kClipFew = 64, kClipMost = 1000;

int clip_blocks() { return sm_count() * kClipBlocks; }

bns_status check_gradients(const bns_gradients* list, bool out) {
    if (!list) return BNS_ERR_NULL;
    if (list->count < 0) return BNS_ERR_SHAPE;
    if (list->count && (!list->data || !list->elements || !list->dtype || (out && !list->out))) return BNS_ERR_NULL;
    for (int i = 0; i < list->count; ++i) {
        if (list->elements[i] < 0 || list->elements[i] > int64_t{1} << 40) return BNS_ERR_SHAPE;
        if (!known(list->dtype[i])) return BNS_ERR_DTYPE;
        if (list->elements[i] == 0) continue;
        if (!list->data[i] || (out && !list->out[i])) return BNS_ERR_NULL;
        const size_t eb = elem_bytes(list->dtype[i]);
        if (!aligned(list->data[i], eb) || (out && !aligned(list->out[i], eb))) return BNS_ERR_ALIGN;
    }
    return BNS_OK;
}

int clip_launches(const bns_gradients* list) { return std::max(1, divide_up(list->count, kClipMost)); }

// Tensors [begin, ...) with elements, as many as the list holds; returns where the next list begins.
template <int N>
int fill_list(const bns_gradients* list, int begin, bool out, ClipList<N>& to) {
    to.count = 0;
    to.in_place = 1;
    int64_t places = 0;
    int i = begin;
    for (; i < list->count && to.count < N; ++i) {
        if (list->elements[i] == 0) continue;
        const size_t eb = elem_bytes(list->dtype[i]);
        const int64_t n = list->elements[i];
        const int64_t head = std::min<int64_t>(n, static_cast<int64_t>((16 - reinterpret_cast<uintptr_t>(list->data[i]) % 16) % 16 / eb));
        const int k = to.count++;
        to.first[k] = places;
        to.in[k] = list->data[i];
        to.out[k] = out ? list->out[i] : nullptr;
        to.in_place &= to.out[k] == to.in[k];
        to.elements[k] = 2 * n + (list->dtype[i] == BNS_BF16);
        places += 1 + (n - head) / static_cast<int64_t>(16 / eb);
    }
    to.first[to.count] = places;
    return i;
}

// Places of a chunk: up to `most`, and such that what the SMs hold of blocks takes the line in whole rounds.
template <int N>
void share_out(ClipList<N>& list, int64_t most) {
    const int64_t each = divide_up<int64_t>(list.first[list.count], clip_blocks()), rounds = std::max<int64_t>(1, divide_up(each, most));
    list.chunk = static_cast<int>(std::max<int64_t>(1, divide_up(divide_up(each, rounds), int64_t{kClipThreads}))) * kClipThreads;
}
constexpr int64_t kSquaresChunk = 8192, kScaleChunk = 4096;    // 128 KB (3.7 GB: 534 us; shares in one piece 578) and 64 KB (6.5 TB/s; 128 KB 6.3)

struct ClipWork {
    double *total, *partial;
    float max_norm;
    float* norm;
    bool out;
};

template <int N>
void clip_lists(const bns_gradients* list, const ClipWork& w, cudaStream_t stream) {
    ClipList<N> here;
    int last = 0, count = 0;
    // forwards over the lists for the squares; an empty one has a sum of 0
    for (int begin = 0; begin < list->count || begin == 0;) {
        last = begin;
        begin = std::max(1, fill_list(list, begin, w.out, here));
        share_out(here, kSquaresChunk);
        const int grid = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(clip_blocks(), chunks_of(here))));
        launch(BNS_KERNEL_CLIP, clip_squares_kernel<N>, Shape{static_cast<unsigned>(grid), kClipThreads}, 0, stream, here, w.partial + count);
        count += grid;
    }
    const double* partial = w.partial;
    auto total = [&] { launch(BNS_KERNEL_CLIP, clip_norm_kernel, Shape{1, kClipThreads}, 0, stream, partial, count, w.total, w.norm); };
    if (!w.out) {
        total();
        return;
    }
    // Many blocks to scale: the sums are added up once, by a launch of its own.  3.7 GB in place and
    // below the limit: 597 us, with every block adding up and looking for its tensor 698.
    const bool many = list->count > kClipMost || divide_up<int64_t>(here.first[here.count], kScaleChunk) > 8 * clip_blocks();
    if (many) {
        total();
        partial = w.total;
        count = 1;
    }
    // the last list first, which is already at hand: its tensors may still be in L2
    auto scale = [&](float* norm) {
        share_out(here, kScaleChunk);
        launch(BNS_KERNEL_CLIP, clip_scale_kernel<N>, Shape{static_cast<unsigned>(std::max<int64_t>(1, chunks_of(here))), kClipThreads}, 0, stream,
               here, partial, count, w.max_norm, norm);
    };
    scale(w.norm);
    for (int begin = 0; begin < last;) {
        begin = fill_list(list, begin, true, here);
        scale(nullptr);
    }
}

bns_status clip(const bns_gradients* list, ClipWork w, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (!w.norm) return BNS_ERR_NULL;
    if (!aligned(w.norm, 4)) return BNS_ERR_ALIGN;
    if (!workspace_fits(workspace, workspace_bytes, bns_gradient_norm_workspace_bytes(list))) return BNS_ERR_WORKSPACE;
    w.total = static_cast<double*>(workspace);
    w.partial = reinterpret_cast<double*>(static_cast<char*>(workspace) + kHeaderBytes);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (list->count <= kClipFew)
        clip_lists<kClipFew>(list, w, stream);
    else
        clip_lists<kClipMost>(list, w, stream);
    return last_error();
}

}  // namespace

extern "C" {

bns_status bns_token_log_probs_forward(const bns_token_log_probs* shape, const void* logits, const void* token, float* logprob,
                                       float* entropy, float* lse, float* top_logprob, int32_t* top_index, void* cuda_stream) {
    const bns_status st = check_log_probs(shape);
    if (st != BNS_OK) return st;
    if (shape->rows == 0) return BNS_OK;
    if (!logits || !token || !logprob || !lse || (shape->entries && (!top_logprob || !top_index))) return BNS_ERR_NULL;
    const int eb = elem_bytes(shape->dtype);
    if (!aligned(logits, eb) || !aligned(token, shape->token_is_int64 ? 8 : 4) || !aligned(logprob, 4) || !aligned(entropy, 4) ||
        !aligned(lse, 4) || !aligned(top_logprob, 4) || !aligned(top_index, 4))
        return BNS_ERR_ALIGN;
    LogProbs a = log_probs_of(shape, logits, token);
    a.logp = logprob;
    a.entropy = entropy;
    a.lse = lse;
    a.top = top_logprob;
    a.index = top_index;
    const int vectors = std::max(1, a.V / (16 / eb));
    const int64_t rows = a.rows, sms = sm_count();
    // Threads of a block, with 1024 an SM.  Small blocks let more rows' ends lie under other rows' streams: bf16, 20
    // alternatives, 128 / 256 / 512 threads: 4096 x 32768 67 / 75 / 106 us, 2047 x 50257 53 / 57 / 72, 1024 x 131072 65 / 59 / 65;
    // without alternatives 2047 x 50257 39 / 40 / 47.  More than 32 alternatives want more threads' maxima: 2047 x 50257
    // with 64 72 / 68 / 82, unless a row has no more than some vectors for each thread (8192 x 4096 82 / 101).
    // Two to three long rows an SM are an uneven number of blocks of 256 threads, and large blocks have them done sooner.  256 / 512 threads, 370 rows, bf16
    // without alternatives: 20011 7.1 / 6.9, 32768 8.4 / 7.9, 50257 12.0 / 10.5, 131072 27.4 / 21.9, 262144 52 / 42; with 20: 40000 14.6 / 15.8, 50257
    // 16.9 / 17.1, 65536 18.7 / 18.1, 131072 33.3 / 29.1, 262144 59 / 52 (444 rows, three an SM: 131072 24.1 / 24.2 and 32.6 / 31.6).  fp32 gains where the
    // rows lie in L2: without alternatives 20000 7.1 / 7.6, 32768 9.4 / 8.9, 50001 14.1 / 12.8, 65536 17.6 / 15.7, but 80000 22.7 / 25.4; with 20
    // 32768 14.3 / 15.3, 50001 20.2 / 20.5, 65536 24.2 / 23.8, 131072 42 / 46.
    const bool uneven = rows > 2 * sms && rows < 3 * sms;
    const bool large = uneven && a.V >= (a.K ? 65536 : 32768) && (eb == 2 || rows * a.V * eb <= 96 << 20);
    const int threads = (vectors <= 1024 && rows > 2 * sms) || (vectors <= 8192 && rows > 8 * sms && a.K <= 32) ? kLogpSmall
                        : large                                                                                ? kLogpLarge
                                                                                                                : kLogpThreads;
    // Few rows are spread over the SMs, less thinly with alternatives, whose lists are joined (64 x 50257 fp32, 20: 8.7 us over
    // four blocks, 12.3 over eight; 16 x 32768 bf16 6.6 with eight vectors a thread, 8.3 with two).
    const int blocks = a.K ? 2 : 4, vectors_each = a.K ? 8 : 2;
    a.parts = 1;
    while (a.parts < kLogpParts && rows * (a.parts + 1) <= blocks * sms && vectors > a.parts * threads * vectors_each) ++a.parts;
    a.per = divide_up(vectors, a.parts);
    if (rows * a.parts >= int64_t{1} << 31) return BNS_ERR_SHAPE;
    const unsigned parts = static_cast<unsigned>(a.parts), grid = static_cast<unsigned>(rows) * parts;
    const Shape launch_shape{grid, static_cast<unsigned>(threads), parts};
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    BNS_LM_BY_TYPE(shape->dtype, {
        if (threads == kLogpSmall)
            (logp_forward<T, kLogpSmall>(a, launch_shape, stream));
        else if (threads == kLogpLarge)
            (logp_forward<T, kLogpLarge>(a, launch_shape, stream));
        else
            (logp_forward<T, kLogpThreads>(a, launch_shape, stream));
    });
    return last_error();
}

bns_status bns_token_log_probs_backward(const bns_token_log_probs* shape, const void* logits, const void* token, const float* lse,
                                        const float* entropy, const float* dlogprob, const float* dentropy, void* dlogits,
                                        int64_t dlogits_stride, void* cuda_stream) {
    const bns_status st = check_log_probs(shape);
    if (st != BNS_OK) return st;
    if (shape->rows == 0) return BNS_OK;
    if (!logits || !token || !lse || !dlogprob || !dlogits || (dentropy && !entropy)) return BNS_ERR_NULL;
    if (dlogits_stride < shape->vocabulary) return BNS_ERR_SHAPE;
    const int eb = elem_bytes(shape->dtype);
    if (!aligned(logits, eb) || !aligned(dlogits, eb) || !aligned(token, shape->token_is_int64 ? 8 : 4) || !aligned(lse, 4) ||
        !aligned(entropy, 4) || !aligned(dlogprob, 4) || !aligned(dentropy, 4))
        return BNS_ERR_ALIGN;
    LogProbs a = log_probs_of(shape, logits, token);
    a.lse_in = lse;
    a.entropy_in = entropy;
    a.dlogp = dlogprob;
    a.dentropy = dentropy;
    a.dz = dlogits;
    a.dz_stride = dlogits_stride;
    const int vectors = std::max(1, a.V / (16 / eb));
    const bool small = vectors <= kLogpSmall * kLogpDepth;
    const int threads = small ? kLogpSmall : kLogpThreads;
    a.parts = std::max(1, vectors / (2 * threads * kLogpDepth));
    while (a.rows * (a.parts + 1) <= 2 * sm_count() && vectors > a.parts * threads) ++a.parts;
    a.per = divide_up(vectors, a.parts);
    if (a.rows * a.parts >= int64_t{1} << 31) return BNS_ERR_SHAPE;
    a.walkers = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(a.parts, sm_count() * (1024 / threads) / a.rows)));
    a.walk = divide_up(vectors, a.walkers);
    const unsigned grid = static_cast<unsigned>(a.rows * a.parts);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    BNS_LM_BY_TYPE(shape->dtype, {
        if (small)
            launch(BNS_KERNEL_LOGP, logp_backward_kernel<T, kLogpSmall>, Shape{grid, kLogpSmall}, 0, stream, a);
        else
            launch(BNS_KERNEL_LOGP, logp_backward_kernel<T, kLogpThreads>, Shape{grid, kLogpThreads}, 0, stream, a);
    });
    return last_error();
}

bns_status bns_head_norm_rotary_forward(const bns_head_norm* shape, const void* q, const void* k, const float* q_weight,
                                        const float* k_weight, const float* cos, const float* sin, const void* position,
                                        void* q_out, void* k_out, void* cuda_stream) {
    const bns_status st = check_head_norm(shape);
    if (st != BNS_OK) return st;
    if (shape->batch == 0 || shape->length == 0) return BNS_OK;
    const bool keys = shape->k_heads > 0;
    if (!q || !q_weight || !cos || !sin || !position || !q_out || (keys && (!k || !k_weight || !k_out))) return BNS_ERR_NULL;
    const size_t eb = elem_bytes(shape->dtype);
    if (!aligned(q, eb) || !aligned(q_out, eb) || !aligned(q_weight, 4) || !aligned(cos, 4) || !aligned(sin, 4) ||
        !aligned(position, shape->position_is_int64 ? 8 : 4) || (keys && (!aligned(k, eb) || !aligned(k_out, eb) || !aligned(k_weight, 4))))
        return BNS_ERR_ALIGN;
    HeadNorm a = problem_of(shape, cos, sin, position);
    a.q.x = q;
    a.q.weight = q_weight;
    a.q.y = q_out;
    a.k.x = keys ? k : nullptr;
    a.k.weight = keys ? k_weight : nullptr;
    a.k.y = keys ? k_out : nullptr;
    head_norm<false>(a, plan_heads(shape, a), shape->dtype, static_cast<cudaStream_t>(cuda_stream));
    return last_error();
}

size_t bns_head_norm_rotary_workspace_bytes(const bns_head_norm* shape) {
    if (check_head_norm(shape) != BNS_OK) return 0;
    return kHeaderBytes + align_up(static_cast<size_t>(head_norm_blocks(shape)) * shape->head_dim * sizeof(float));
}

bns_status bns_head_norm_rotary_backward(const bns_head_norm* shape, const void* dq_out, const void* dk_out, const void* q,
                                         const void* k, const float* q_weight, const float* k_weight, const float* cos,
                                         const float* sin, const void* position, void* dq, void* dk, float* dq_weight,
                                         float* dk_weight, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    const bns_status st = check_head_norm(shape);
    if (st != BNS_OK) return st;
    const bool keys = shape->k_heads > 0;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (!dq_weight || (keys && !dk_weight)) return BNS_ERR_NULL;
    if (!aligned(dq_weight, 4) || !aligned(dk_weight, 4)) return BNS_ERR_ALIGN;
    auto clear = [&](float* weight) { return cudaMemsetAsync(weight, 0, sizeof(float) * shape->head_dim, stream) == cudaSuccess; };
    if (shape->batch == 0 || shape->length == 0) return clear(dq_weight) && (!dk_weight || clear(dk_weight)) ? BNS_OK : BNS_ERR_CUDA;
    if (!dq_out || !q || !q_weight || !cos || !sin || !position || !dq || (keys && (!dk_out || !k || !k_weight || !dk))) return BNS_ERR_NULL;
    const size_t eb = elem_bytes(shape->dtype);
    if (!aligned(dq_out, eb) || !aligned(q, eb) || !aligned(dq, eb) || !aligned(q_weight, 4) || !aligned(cos, 4) || !aligned(sin, 4) ||
        !aligned(position, shape->position_is_int64 ? 8 : 4) ||
        (keys && (!aligned(dk_out, eb) || !aligned(k, eb) || !aligned(dk, eb) || !aligned(k_weight, 4))))
        return BNS_ERR_ALIGN;
    if (!workspace_fits(workspace, workspace_bytes, bns_head_norm_rotary_workspace_bytes(shape))) return BNS_ERR_WORKSPACE;
    if (!keys && dk_weight && !clear(dk_weight)) return BNS_ERR_CUDA;
    HeadNorm a = problem_of(shape, cos, sin, position);
    a.q.x = q;
    a.q.dy = dq_out;
    a.q.weight = q_weight;
    a.q.y = dq;
    a.k.x = keys ? k : nullptr;
    a.k.dy = keys ? dk_out : nullptr;
    a.k.weight = keys ? k_weight : nullptr;
    a.k.y = keys ? dk : nullptr;
    a.partial = reinterpret_cast<float*>(static_cast<char*>(workspace) + kHeaderBytes);
    const HeadBlocks blocks = head_norm<true>(a, plan_heads(shape, a), shape->dtype, stream);
    launch(BNS_KERNEL_HEAD_NORM, head_weight_kernel, Shape{static_cast<unsigned>(divide_up(shape->head_dim, 32)), 1024, 1, keys ? 2u : 1u}, 0,
           stream, static_cast<const float*>(a.partial), blocks.q, blocks.k, shape->head_dim, dq_weight, dk_weight);
    return last_error();
}

size_t bns_gradient_norm_workspace_bytes(const bns_gradients* list) {
    if (check_gradients(list, false) != BNS_OK) return 0;
    return kHeaderBytes + align_up(static_cast<size_t>(clip_launches(list)) * clip_blocks() * sizeof(double));
}

bns_status bns_gradient_norm(const bns_gradients* list, float* norm, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    const bns_status st = check_gradients(list, false);
    if (st != BNS_OK) return st;
    return clip(list, ClipWork{nullptr, nullptr, 0.f, norm, false}, workspace, workspace_bytes, cuda_stream);
}

bns_status bns_clip_gradients(const bns_gradients* list, float max_norm, float* norm, void* workspace, size_t workspace_bytes,
                              void* cuda_stream) {
    const bns_status st = check_gradients(list, true);
    if (st != BNS_OK) return st;
    if (!(max_norm >= 0.f)) return BNS_ERR_SHAPE;
    return clip(list, ClipWork{nullptr, nullptr, max_norm, norm, true}, workspace, workspace_bytes, cuda_stream);
}

}  // extern "C"
