// A CUDA runtime without a GPU for the trainers' host code: device memory is host memory, kernels do nothing, and what a test asks to
// fail fails and leaves its error behind, as the runtime does.
#include <cuda_runtime_api.h>

#include <cstdint>
#include <cstdlib>
#include <cstring>
#include <map>

struct slaq_handle;

extern "C" {
int fake_launches = 0, fake_copies = 0;
int fake_capturing = 0;
int fake_capture_query_fails = 0;          // cudaStreamIsCapturing fails that often
int fake_copies_fail = 0;                  // cudaMemcpyAsync
int fake_launches_fail = 0;
const void* fake_last_kernel = nullptr;
size_t fake_last_bytes = 0;                // dynamic shared memory of the last launch

static cudaError_t last = cudaSuccess;
static std::map<const void*, int> limits;  // of dynamic shared memory, per kernel
static cudaError_t is(cudaError_t e) { return e == cudaSuccess ? e : last = e; }

int fake_limit(const void* kernel) { return limits.count(kernel) ? limits[kernel] : 48 * 1024; }
int slaq_append_losses_device(slaq_handle*, int32_t, const int32_t*, const double*, const double*, const int32_t*) { return 0; }

void** __cudaRegisterFatBinary(void*) { static void* h; return &h; }
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
void __cudaRegisterFunction(void**, const char*, char*, const char*, int, uint3*, uint3*, dim3*, dim3*, int*) {}
unsigned __cudaPushCallConfiguration(dim3, dim3, size_t, cudaStream_t) { return 0; }
cudaError_t __cudaPopCallConfiguration(dim3* g, dim3* b, size_t* s, void* st) {
    *g = *b = dim3(1), *s = 0, *(void**)st = nullptr;
    return cudaSuccess;
}
static cudaError_t launch(const void* kernel, size_t bytes) {
    if (fake_launches_fail > 0) return --fake_launches_fail, is(cudaErrorLaunchOutOfResources);
    if ((int)bytes > fake_limit(kernel)) return is(cudaErrorInvalidValue);
    ++fake_launches, fake_last_kernel = kernel, fake_last_bytes = bytes;
    return cudaSuccess;
}
cudaError_t cudaLaunchKernel(const void* kernel, dim3, dim3, void**, size_t bytes, cudaStream_t) { return launch(kernel, bytes); }
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void* kernel, void**) { return launch(kernel, c->dynamicSmemBytes); }
cudaError_t cudaFuncSetAttribute(const void* kernel, cudaFuncAttribute, int value) { limits[kernel] = value; return cudaSuccess; }
cudaError_t cudaOccupancyMaxActiveBlocksPerMultiprocessorWithFlags(int* n, const void*, int, size_t, unsigned) { *n = 4; return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int* v, cudaDeviceAttr, int) { *v = 148; return cudaSuccess; }
cudaError_t cudaGetDevice(int* d) { *d = 0; return cudaSuccess; }
cudaError_t cudaGetLastError() { const cudaError_t e = last; last = cudaSuccess; return e; }
cudaError_t cudaMalloc(void** p, size_t n) { *p = std::aligned_alloc(256, (n + 255) / 256 * 256); return *p ? cudaSuccess : is(cudaErrorMemoryAllocation); }
cudaError_t cudaFree(void* p) { std::free(p); return cudaSuccess; }
cudaError_t cudaMemcpyAsync(void* d, const void* s, size_t n, cudaMemcpyKind, cudaStream_t) {
    if (fake_copies_fail > 0) return --fake_copies_fail, is(cudaErrorStreamCaptureUnsupported);
    std::memcpy(d, s, n);
    ++fake_copies;
    return cudaSuccess;
}
cudaError_t cudaMemcpy2DAsync(void*, size_t, const void*, size_t, size_t, size_t, cudaMemcpyKind, cudaStream_t) {
    if (fake_copies_fail > 0) return --fake_copies_fail, is(cudaErrorStreamCaptureUnsupported);
    return cudaSuccess;
}
cudaError_t cudaMemsetAsync(void* d, int v, size_t n, cudaStream_t) { std::memset(d, v, n); return cudaSuccess; }
cudaError_t cudaStreamIsCapturing(cudaStream_t, cudaStreamCaptureStatus* s) {
    *s = fake_capturing ? cudaStreamCaptureStatusActive : cudaStreamCaptureStatusNone;
    if (fake_capture_query_fails > 0) return --fake_capture_query_fails, is(cudaErrorStreamCaptureImplicit);
    return cudaSuccess;
}
cudaError_t cudaStreamSynchronize(cudaStream_t) { return cudaSuccess; }
}
