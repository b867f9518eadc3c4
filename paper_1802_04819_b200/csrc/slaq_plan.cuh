// Host code of the plans over many tensors.
#pragma once

#include <algorithm>
#include <cstdint>
#include <utility>
#include <vector>

#include "slaq_internal.cuh"

namespace slaq {
namespace {

constexpr int64_t kMostElements = (int64_t)1 << 38;   // of a plan: its blocks are counted in 31 bits

size_t up(size_t n) { return (n + 255) & ~size_t(255); }
size_t size_of(int type) { return type == SLAQ_F32 ? 4 : 2; }

// Whether a call of the runtime did what it should.  An error that it left behind would be taken for that of a later call.
bool done(cudaError_t e) {
    if (e != cudaSuccess) (void)cudaGetLastError();
    return e == cudaSuccess;
}
// A stream that is captured, or cannot be asked: to wait for it would end the capture with an error.
bool captured(cudaStream_t st) {
    cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
    return !done(cudaStreamIsCapturing(st, &status)) || status != cudaStreamCaptureStatusNone;
}
template <class... Params, class... Args>
bool launch(void (*kernel)(Params...), int blocks, int threads, cudaStream_t st, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.stream = st;
    return done(cudaLaunchKernelEx(&cfg, kernel, args...));
}

// an interval of memory that meets one of `sorted`, which do not meet one another
bool meets(const std::vector<std::pair<uintptr_t, uintptr_t>>& sorted, uintptr_t lo, uintptr_t hi) {
    auto it = std::upper_bound(sorted.begin(), sorted.end(), std::make_pair(lo, UINTPTR_MAX));
    if (it != sorted.end() && it->first < hi) return true;
    return it != sorted.begin() && std::prev(it)->second > lo;
}

}  // namespace
}  // namespace slaq
