// Mean losses of jobs over the rows that are theirs, as the scheduler's histories take them.
//
// Job j owns rows offsets[j] .. offsets[j+1).  A row counts with its weight (1 without weights), and not at all if its target is
// negative or its weight 0:  loss_j = -sum w_r logprob_r / sum w_r, in 64 bits: the scheduler works on differences of losses
// that a converged job reports at 1e-4 of their size and less.
#include "slaq_internal.cuh"

namespace slaq {
namespace {

constexpr int kThreads = 256;

__device__ double block_sum(double v, double* shared) {
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0;
    for (int w = 0; w < kThreads / 32; ++w) v += shared[w];
    return v;
}

__device__ __forceinline__ float weight_of(const int64_t* targets, const float* weights, int64_t r) {
    return targets && targets[r] < 0 ? 0.0f : weights ? weights[r] : 1.0f;
}

// The rows of job j; offsets that leave the array or run backwards give `bad`, and no row.
struct Rows {
    int64_t lo, hi;
    bool bad;
};
__device__ Rows rows_of(const int64_t* offsets, int64_t rows, int j) {
    const int64_t lo = offsets[j], hi = offsets[j + 1];
    if (lo < 0 || hi < lo || hi > rows) return {0, 0, true};
    return {lo, hi, false};
}

__global__ void __launch_bounds__(kThreads)
    row_grad_kernel(const int64_t* offsets, int64_t rows, const int64_t* targets, const float* weights, float* out) {
    __shared__ double shared[kThreads / 32];
    const auto [lo, hi, bad] = rows_of(offsets, rows, blockIdx.x);
    double w = 0.0;
    for (int64_t r = lo + threadIdx.x; r < hi; r += kThreads) w += weight_of(targets, weights, r);
    w = block_sum(w, shared);
    for (int64_t r = lo + threadIdx.x; r < hi; r += kThreads) {
        const float mine = weight_of(targets, weights, r);
        out[r] = mine == 0.0f ? 0.0f : (float)(-mine / w);
    }
}

__global__ void __launch_bounds__(kThreads)
    job_losses_kernel(const int64_t* offsets, int64_t rows, const int64_t* targets, const float* logprob, const float* weights, double* out) {
    __shared__ double shared[kThreads / 32];
    const auto [lo, hi, bad] = rows_of(offsets, rows, blockIdx.x);
    double w = 0.0, s = 0.0;
    for (int64_t r = lo + threadIdx.x; r < hi; r += kThreads) {
        const float mine = weight_of(targets, weights, r);
        if (mine != 0.0f) {
            w += mine;
            s += (double)mine * logprob[r];
        }
    }
    w = block_sum(w, shared);
    s = block_sum(s, shared);
    if (threadIdx.x == 0) out[blockIdx.x] = -s / w;   // NaN for a job without a row that counts
}

int done() { return cudaGetLastError() == cudaSuccess ? SLAQ_OK : SLAQ_E_CUDA; }

}  // namespace
}  // namespace slaq

extern "C" int slaq_job_row_grad(int32_t n_jobs, const int64_t* d_offsets, int64_t rows, const int64_t* d_targets, const float* d_weights,
                                 float* d_out_row_grad, void* cuda_stream) {
    using namespace slaq;
    if (n_jobs < 0 || rows < 0 || (n_jobs && (!d_offsets || !d_out_row_grad))) return SLAQ_E_ARG;
    if (n_jobs == 0) return SLAQ_OK;
    row_grad_kernel<<<n_jobs, kThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(d_offsets, rows, d_targets, d_weights, d_out_row_grad);
    return done();
}

extern "C" int slaq_job_losses(int32_t n_jobs, const int64_t* d_offsets, int64_t rows, const int64_t* d_targets, const float* d_logprob,
                               const float* d_weights, double* d_out_losses, void* cuda_stream) {
    using namespace slaq;
    if (n_jobs < 0 || rows < 0 || (n_jobs && (!d_offsets || !d_logprob || !d_out_losses))) return SLAQ_E_ARG;
    if (n_jobs == 0) return SLAQ_OK;
    job_losses_kernel<<<n_jobs, kThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(d_offsets, rows, d_targets, d_logprob, d_weights, d_out_losses);
    return done();
}

extern "C" int slaq_append_token_losses(slaq_t* h, int32_t n, const int32_t* d_job_ids, const int64_t* d_offsets, int64_t rows,
                                        const int64_t* d_targets, const float* d_logprob, const float* d_weights,
                                        const double* d_iter_times, const int32_t* d_cores_used, double* d_out_losses) {
    using namespace slaq;
    // the append's own checks come first, so that a refused call has launched nothing
    if (!h) return SLAQ_E_ARG;
    if (n > 0 && n <= h->max_jobs && d_job_ids && d_out_losses && !(d_cores_used && !d_iter_times)) {
        int device = -1;
        if (cudaGetDevice(&device) == cudaSuccess && device == h->device)
            if (const int rc = slaq_job_losses(n, d_offsets, rows, d_targets, d_logprob, d_weights, d_out_losses, h->stream)) {
                h->err = rc == SLAQ_E_ARG ? "offsets or logprob is null, or negative rows" : "job losses: a CUDA call failed";
                return rc;
            }
    }
    return slaq_append_losses_device(h, n, d_job_ids, d_out_losses, d_iter_times, d_cores_used);
}
