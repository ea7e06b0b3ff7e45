// What the host sides of the library share: launch counting and timing, launch errors, device queries.
// Defined in bns_api.cu.
#pragma once

#include <cuda_runtime.h>

#include "bns.h"

namespace bns {

constexpr int kMaxDevices = 64;

// Streaming multiprocessors of the current device.
int sm_count();

// Counts a launch and, with profiling on, brackets it with events.
struct LaunchScope {
    cudaStream_t stream;
    int kind;
    bool timed = false;
    cudaEvent_t start = nullptr, stop = nullptr;
    LaunchScope(int kind_, cudaStream_t s);
    ~LaunchScope();
    LaunchScope(const LaunchScope&) = delete;
    LaunchScope& operator=(const LaunchScope&) = delete;
};

// Records a launch's return code for this host thread; last_error() hands the verdict out and clears it.
void note_launch(cudaError_t err);
bns_status last_error();

// Ask for programmatic dependent launch (blocks may be scheduled while the previous kernel drains).
extern bool g_pdl;

// Most columns of the vocabulary that the head's gradient holds at a time; 0 = as many as its memory aim allows.
extern int g_head_piece;

// Adds the bounded waits that ran out in the language-model kernels on the current device (synchronises the stream).
bns_status lm_wait_timeouts(uint32_t* count, cudaStream_t stream);

}  // namespace bns
