// What the host sides of the language-model operators share: sizes, alignment, launches, how rows may be moved.
#pragma once

#include "bns_elements.cuh"
#include "bns_host.h"

namespace bns {

constexpr size_t kAlign = 256;
constexpr size_t kHeaderBytes = 256;   // the status word

inline size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }
template <typename N>
N divide_up(N a, N b) {
    return (a + b - 1) / b;
}
inline int elem_bytes(int dtype) { return dtype == BNS_F32 ? 4 : 2; }
inline bool known(int dtype) { return dtype == BNS_F32 || dtype == BNS_BF16; }
inline bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
inline bool workspace_fits(const void* ws, size_t bytes, size_t need) { return ws && aligned(ws, kAlign) && bytes >= need; }

struct Shape {
    unsigned grid, threads, cluster = 1, grid_y = 1;
};

template <typename... KArgs, typename... Args>
void launch(int kind, void (*kernel)(KArgs...), Shape shape, size_t smem, cudaStream_t s, Args&&... args) {
    LaunchScope scope(kind, s);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(shape.grid, shape.grid_y);
    cfg.blockDim = dim3(shape.threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (g_pdl) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (shape.cluster > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = shape.cluster;
        attr[n].val.clusterDim.y = 1;
        attr[n++].val.clusterDim.z = 1;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    note_launch(cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...));
}

// How the rows of several tensors may be moved: in 16-byte vectors from the first column on, in such vectors from a column
// that depends on the row's phase (the same for all tensors in every row), or element by element.
struct VectorRule {
    enum Kind { kAligned, kPhase, kElements } kind = kAligned;
    VectorRule(int columns, int ebytes) : V(16 / ebytes), D(columns), eb(ebytes) {
        if (columns % V) kind = kPhase;
    }
    void tensor(const void* p, int64_t stride) { add(p, stride, eb); }
    void bytes(const void* p) { add(p, D, 1); }    // the dense 8-bit output: V elements are V bytes

private:
    int V, D, eb;
    bool first = true;
    uint64_t phase = 0, step = 0;
    void add(const void* p, int64_t stride, int size) {
        if (!p || kind == kElements) return;
        const uint64_t here = reinterpret_cast<uintptr_t>(p) / size % V, next = static_cast<uint64_t>(stride) % V;
        if (first) {
            phase = here;
            step = next;
            first = false;
        }
        if (here != phase || next != step)
            kind = kElements;
        else if (here || next)
            kind = kPhase;
    }
};

#define BNS_LM_BY_TYPE(dtype, CALL) \
    do {                            \
        if ((dtype) == BNS_F32) {   \
            using T = F32;          \
            CALL;                   \
        } else {                    \
            using T = BF16;         \
            CALL;                   \
        }                           \
    } while (0)

}  // namespace bns
