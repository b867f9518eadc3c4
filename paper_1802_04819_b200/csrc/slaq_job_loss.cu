// Mean losses of jobs over the rows that are theirs, as the scheduler's histories take them.
//
// Job j owns rows offsets[j] .. offsets[j+1).  A row counts with its weight (1 without weights), and not at all if its target is
// negative or its weight 0:  loss_j = -sum w_r logprob_r / sum w_r, in 64 bits: the scheduler works on differences of losses
// that a converged job reports at 1e-4 of their size and less.
//
// 12 to 20 bytes are read per row and little else happens, so what counts is that the threads have rows and that many are on their way.
// A warp, a block or a cluster of eight blocks works on a job, by the mean number of the jobs' rows: what is known without
// reading the offsets.  A job far longer than the others is then one block's, on one SM: 2,000 jobs of 10 rows and one of 2 M take 1.5 ms,
// 5,000 of 20 and one of 1 M 0.2 ms.  Every sum is taken in an order that the sizes alone decide.
#include <cooperative_groups.h>

#include <algorithm>

#include "slaq_internal.cuh"

namespace cg = cooperative_groups;

namespace slaq {
namespace {

constexpr int kCluster = 8;

struct JobArgs {
    int32_t n_jobs;
    const int64_t* offsets;
    int64_t rows;
    const int64_t* targets;
    const float *logprob, *weights;
    float* row_grad;
    double* losses;
};

struct Two {
    double w, s;
};

// The sums of a job's T threads, or of its cluster's blocks of T threads, in each of them.
template <int T, bool kClustered>
__device__ Two team_sum(Two v, Two* shared, Two* from_blocks) {
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        v.w += __shfl_xor_sync(~0u, v.w, o);
        v.s += __shfl_xor_sync(~0u, v.s, o);
    }
    if constexpr (T == 32) return v;
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
    __syncthreads();
    v = {0.0, 0.0};
    for (int w = 0; w < T / 32; ++w) v.w += shared[w].w, v.s += shared[w].s;
    if constexpr (kClustered) {
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();                                     // every block has begun
        if (threadIdx.x < kCluster) cluster.map_shared_rank(from_blocks, threadIdx.x)[cluster.block_rank()] = v;
        cluster.sync();
        v = {0.0, 0.0};
        for (int b = 0; b < kCluster; ++b) v.w += from_blocks[b].w, v.s += from_blocks[b].s;
    }
    return v;
}

// Eight rows of a thread, kStep apart, all loaded before the first is used: each(r, w, lp) with their weights (0 behind the end)
// and, if kLosses, their log probabilities.
constexpr int kBatch = 8;
template <bool kWhole, class T>
__device__ __forceinline__ void load_batch(T (&x)[kBatch], const T* from, int64_t r, int64_t end, int step) {
#pragma unroll
    for (int k = 0; k < kBatch; ++k) x[k] = kWhole || r + k * step < end ? __ldg(from + r + k * step) : T(0);
}
template <bool kWhole, bool kLosses, int kStep, class Each>
__device__ __forceinline__ void batch(const JobArgs& a, int64_t r, int64_t end, Each&& each) {
    long long t[kBatch] = {};
    float w[kBatch], lp[kBatch];
    if (a.targets) load_batch<kWhole>(t, reinterpret_cast<const long long*>(a.targets), r, end, kStep);
    if (kLosses) load_batch<kWhole>(lp, a.logprob, r, end, kStep);
    if (a.weights) {
        load_batch<kWhole>(w, a.weights, r, end, kStep);
    } else {
#pragma unroll
        for (int k = 0; k < kBatch; ++k) w[k] = kWhole || r + k * kStep < end ? 1.0f : 0.0f;
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
        if (t[k] < 0) w[k] = 0.0f;
    each(r, w, lp);
}
template <bool kLosses, int kStep, class Each>
__device__ __forceinline__ void for_rows(const JobArgs& a, int64_t first, int64_t end, Each&& each) {
    int64_t r = first;
    for (; r + (kBatch - 1) * kStep < end; r += kStep * kBatch) batch<true, kLosses, kStep>(a, r, end, each);
    if (r + kStep < end) {
        batch<false, kLosses, kStep>(a, r, end, each);
    } else if (r < end) {   // one row: most of what the threads of a short job have
        float w[kBatch] = {a.weights ? __ldg(a.weights + r) : 1.0f}, lp[kBatch] = {kLosses ? __ldg(a.logprob + r) : 0.0f};
        if (a.targets && __ldg(a.targets + r) < 0) w[0] = 0.0f;
        each(r, w, lp);
    }
}

// The rows of job j; offsets that leave the array or run backwards give none: the job's loss is then NaN, and its rows are not touched.
struct Rows {
    int64_t lo, hi;
};
__device__ __forceinline__ Rows rows_of(const JobArgs& a, int64_t j) {
    const int64_t lo = a.offsets[j], hi = a.offsets[j + 1];
    return lo < 0 || hi < lo || hi > a.rows ? Rows{0, 0} : Rows{lo, hi};
}

// Job j by T threads (numbered `tid`), or by the blocks of a cluster.
template <int T, bool kClustered, bool kLosses>
__device__ __forceinline__ void work_on(const JobArgs& a, int64_t j, Rows rows, int tid, int rank, Two* shared, Two* from_blocks) {
    constexpr int kStep = T * (kClustered ? kCluster : 1);
    const int64_t first = rows.lo + (int64_t)rank * T + tid;
    Two sum = {0.0, 0.0};
    for_rows<kLosses, kStep>(a, first, rows.hi, [&](int64_t, const float (&w)[kBatch], const float (&lp)[kBatch]) {
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            sum.w += w[k];
            if (kLosses) sum.s += w[k] != 0.0f ? (double)w[k] * lp[k] : 0.0;      // what does not count may be infinite or NaN
        }
    });
    sum = team_sum<T, kClustered>(sum, shared, from_blocks);
    if (kLosses) {
        if (tid == 0 && rank == 0) a.losses[j] = -sum.s / sum.w;   // NaN for a job without a row that counts
        return;
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");   // for zero_kernel, if it runs
    const double by = -1.0 / sum.w;
    for_rows<false, kStep>(a, first, rows.hi, [&](int64_t r, const float (&w)[kBatch], const float (&)[kBatch]) {
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
            if (r + k * kStep < rows.hi) a.row_grad[r + k * kStep] = w[k] != 0.0f ? (float)(w[k] * by) : 0.0f;
    });
}

// Zeros in the rows that no job counts.  A block knows the offsets of its own jobs; that the rows before the first and behind the last
// are nobody's follows only if none falls, and then every block has to look at all of them.  Where one does fall or leaves the array,
// each row is held against every job.
__device__ void zero_rest(const JobArgs& a) {
    bool bad = false;
    for (int64_t j = threadIdx.x; j < a.n_jobs; j += blockDim.x) bad |= a.offsets[j] < 0 || a.offsets[j + 1] < a.offsets[j] || a.offsets[j + 1] > a.rows;
    const int64_t n = (int64_t)gridDim.x * blockDim.x, at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (!__syncthreads_or(bad)) {
        for (int64_t r = at; r < a.offsets[0]; r += n) a.row_grad[r] = 0.0f;
        for (int64_t r = a.offsets[a.n_jobs] + at; r < a.rows; r += n) a.row_grad[r] = 0.0f;
        return;
    }
    for (int64_t r = at; r < a.rows; r += n) {
        bool counted = false;
        for (int64_t j = 0; j < a.n_jobs; ++j) {
            const Rows rows = rows_of(a, j);
            counted |= rows.lo <= r && r < rows.hi;
        }
        if (!counted) a.row_grad[r] = 0.0f;
    }
}
// .. and where there are too many jobs for that, zeros in all rows, before the kernel that writes the factors: it begins while these are
// written, and waits for them before its first factor.
__global__ void __launch_bounds__(512) zero_kernel(float* to, int64_t n) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int64_t step = (int64_t)gridDim.x * blockDim.x, at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    const int64_t head = min(n, (int64_t)((16 - ((uintptr_t)to & 15)) & 15) / 4), vectors = (n - head) / 4, tail = head + 4 * vectors;
    for (int64_t i = at; i < vectors; i += step) reinterpret_cast<float4*>(to + head)[i] = float4{0.0f, 0.0f, 0.0f, 0.0f};
    if (at < head) to[at] = 0.0f;
    if (at < n - tail) to[tail + at] = 0.0f;
}

// A block, or a cluster of blocks, for each job.
template <int T, bool kClustered, bool kLosses, bool kZeroRest>
__global__ void __launch_bounds__(T) jobs_kernel(JobArgs a) {
    __shared__ Two shared[T / 32], from_blocks[kCluster];
    if (kZeroRest) zero_rest(a);
    const int64_t j = kClustered ? blockIdx.x / kCluster : blockIdx.x;
    work_on<T, kClustered, kLosses>(a, j, rows_of(a, j), threadIdx.x, kClustered ? (int)cg::this_cluster().block_rank() : 0, shared, from_blocks);
}

// Short jobs: a warp for each; what is long among them is then done by all warps of its block.
constexpr int kShort = 2048, kBlockJobs = 16;
template <bool kLosses, bool kZeroRest>
__global__ void __launch_bounds__(32 * kBlockJobs) short_jobs_kernel(JobArgs a) {
    __shared__ Two shared[kBlockJobs];
    if (kZeroRest) zero_rest(a);
    const int64_t first = (int64_t)blockIdx.x * kBlockJobs, mine = first + (threadIdx.x >> 5);
    bool is_long = false;
    if (mine < a.n_jobs) {
        const Rows rows = rows_of(a, mine);
        is_long = rows.hi - rows.lo > kShort;
        if (!is_long) work_on<32, false, kLosses>(a, mine, rows, threadIdx.x & 31, 0, nullptr, nullptr);
    }
    if (!__syncthreads_or(is_long)) return;
    for (int64_t j = first; j < min(first + kBlockJobs, (int64_t)a.n_jobs); ++j) {
        const Rows rows = rows_of(a, j);
        if (rows.hi - rows.lo <= kShort) continue;
        work_on<32 * kBlockJobs, false, kLosses>(a, j, rows, threadIdx.x, 0, shared, nullptr);
        __syncthreads();
    }
}

// By the mean length.  Jobs of equal length (row factors, us; losses alike), a warp or 128 threads:
//       256 rows: 500 jobs 2.9 and 2.9, 2,000 3.0 and 5.4;   512: 500 jobs 3.8 and 2.8, 8,000 8.2 and 16.3;   1,024: 500 jobs 5.3 and 2.8, 2,000 5.5 and 5.0
// but 4,000 jobs of 1 to 2,000 rows, 490 on average, 25.3 and 22.6 us with both calls: a block of warps ends with its longest job.
// 128 or 512 threads:
//     2,048 rows: 160 jobs 3.1 and 4.1, 2,000 7.3 and 17.6;   4,096: 160 jobs 4.3 and 3.5, 2,000 14.7 and 18.5
// 512 threads, which take 0.23 us for 1,000 rows, or a cluster of eight blocks, of which 14 are 5 us and each further one 0.2 us, whatever they do:
//     16,384 rows: 4 jobs 5.2 and 6.2, 148 5.6 and 38;   32,768: 4 jobs 9.4 and 6.5, 16 9.4 and 9.6;   65,536: 32 jobs 16.6 and 10.5, 64 16.7 and 18.6;
//     262,144: 48 jobs 165 and 43
constexpr int64_t kWarpRows = 256, kSmallBlockRows = 2048, kClusterRows = 32768, kClusterRowsPerJob = 2048;

// Every block looks at all offsets while that is this many loads in all; zeros in a kernel of their own are another launch.  A fresh result, us on
// the device and in a call from Python, with all offsets looked at and with the other kernel:
//     700 jobs of 500 rows 4.5 / 6.8 and 3.9 / 9.0;   1,500 of 500 7.9 / 10.2 and 5.8 / 8.9;   2,000 of 200, 16 of them in a block, 5.5 / 6.9 and 4.0 / 9.0;
//     6,000 of 200 9.0 / 10.3 and 6.4 / 8.9;   4,000 of 500 23.6 / 24.6 and 10.1 / 12.3 (without any zeros 9.6 / 12.3)
constexpr int64_t kOffsetsLookedAt = (int64_t)1 << 19;
constexpr int64_t kFewRows = (int64_t)1 << 26;   // each of which may have to be held against all of these jobs

template <bool kLosses, bool kZeroRest>
int launch_jobs(const JobArgs& a, cudaStream_t st, bool behind_zeros) {
    const int64_t mean = a.rows / a.n_jobs;
    cudaLaunchConfig_t cfg = {};
    cfg.stream = st;
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[behind_zeros].id = cudaLaunchAttributeClusterDimension;
    attr[behind_zeros].val.clusterDim.x = kCluster;
    attr[behind_zeros].val.clusterDim.y = attr[behind_zeros].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = behind_zeros;
    cudaError_t e;
    if (mean <= kWarpRows) {
        cfg.gridDim = dim3((unsigned)((a.n_jobs + kBlockJobs - 1) / kBlockJobs));
        cfg.blockDim = dim3(32 * kBlockJobs);
        e = cudaLaunchKernelEx(&cfg, short_jobs_kernel<kLosses, kZeroRest>, a);
    } else if (mean <= kSmallBlockRows) {
        cfg.gridDim = dim3((unsigned)a.n_jobs);
        cfg.blockDim = dim3(128);
        e = cudaLaunchKernelEx(&cfg, jobs_kernel<128, false, kLosses, kZeroRest>, a);
    } else if (mean < kClusterRows || mean < kClusterRowsPerJob * a.n_jobs) {
        cfg.gridDim = dim3((unsigned)a.n_jobs);
        cfg.blockDim = dim3(512);
        e = cudaLaunchKernelEx(&cfg, jobs_kernel<512, false, kLosses, kZeroRest>, a);
    } else {
        cfg.gridDim = dim3((unsigned)a.n_jobs * kCluster);
        cfg.blockDim = dim3(1024);
        ++cfg.numAttrs;
        e = cudaLaunchKernelEx(&cfg, jobs_kernel<1024, true, kLosses, kZeroRest>, a);
    }
    if (e != cudaSuccess) (void)cudaGetLastError();
    return e == cudaSuccess ? SLAQ_OK : SLAQ_E_CUDA;
}

}  // namespace
}  // namespace slaq

extern "C" int slaq_job_row_grad(int32_t n_jobs, const int64_t* d_offsets, int64_t rows, const int64_t* d_targets, const float* d_weights,
                                 float* d_out_row_grad, int32_t zero_rest, void* cuda_stream) {
    using namespace slaq;
    if (n_jobs < 0 || rows < 0 || (n_jobs && (!d_offsets || (rows && !d_out_row_grad)))) return SLAQ_E_ARG;
    if (!aligned(d_offsets, d_targets, d_weights, d_out_row_grad)) return SLAQ_E_ARG;
    if (n_jobs == 0 || rows == 0) return n_jobs == 0 && rows && zero_rest ? SLAQ_E_ARG : SLAQ_OK;
    JobArgs a = {n_jobs, d_offsets, rows, d_targets, nullptr, d_weights, d_out_row_grad, nullptr};
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (!zero_rest) return launch_jobs<false, false>(a, st, false);
    const int64_t blocks = rows / n_jobs <= kWarpRows ? (n_jobs + kBlockJobs - 1) / kBlockJobs : n_jobs;
    if (blocks * n_jobs <= kOffsetsLookedAt && rows <= kFewRows) return launch_jobs<false, true>(a, st, false);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)std::min<int64_t>((rows + 4 * 512 - 1) / (4 * 512), 4 * 148));
    cfg.blockDim = dim3(512);
    cfg.stream = st;
    if (cudaLaunchKernelEx(&cfg, zero_kernel, d_out_row_grad, rows) != cudaSuccess) {
        (void)cudaGetLastError();
        return SLAQ_E_CUDA;
    }
    return launch_jobs<false, false>(a, st, true);
}

extern "C" int slaq_job_losses(int32_t n_jobs, const int64_t* d_offsets, int64_t rows, const int64_t* d_targets, const float* d_logprob,
                               const float* d_weights, double* d_out_losses, void* cuda_stream) {
    using namespace slaq;
    if (n_jobs < 0 || rows < 0 || (n_jobs && (!d_offsets || (rows && !d_logprob) || !d_out_losses))) return SLAQ_E_ARG;
    if (!aligned(d_offsets, d_targets, d_logprob, d_weights, d_out_losses)) return SLAQ_E_ARG;
    if (n_jobs == 0) return SLAQ_OK;
    JobArgs a = {n_jobs, d_offsets, rows, d_targets, d_logprob, d_weights, nullptr, d_out_losses};
    return launch_jobs<true, false>(a, static_cast<cudaStream_t>(cuda_stream), false);
}

extern "C" int slaq_append_token_losses(slaq_t* h, int32_t n, const int32_t* d_job_ids, const int64_t* d_offsets, int64_t rows,
                                        const int64_t* d_targets, const float* d_logprob, const float* d_weights,
                                        const double* d_iter_times, const int32_t* d_cores_used, double* d_out_losses) {
    using namespace slaq;
    // the append's own checks come first, so that a refused call has launched nothing
    if (!h) return SLAQ_E_ARG;
    if (!aligned(d_job_ids, d_offsets, d_targets, d_logprob, d_weights, d_iter_times, d_cores_used, d_out_losses)) {
        h->err = "an address that its elements' size does not divide";
        return SLAQ_E_ARG;
    }
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
