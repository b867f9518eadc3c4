// Log probabilities of given tokens with the entropy and the top alternatives of their rows, and their gradient.
//
// A row x[0..V) of logits, scale c, token t.  With m = max x, d_i = c (x_i - m), S = sum exp d_i:
//     log probability  d_t - ln S          entropy  ln S - (sum exp(d_i) d_i) / S
// Both terms of the entropy are non-negative, so nothing cancels.  What a later gradient needs of the row is kept as (m, S)
// and not as m c + ln S: a sum near 20 would carry 1e-6 of rounding into every probability.
#include "slaq_internal.cuh"
#include "slaq_rows.cuh"

namespace slaq {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxVocab = 1 << 22;
constexpr int kMaxTop = 32;

struct RowArgs {
    const void* logits;
    int64_t rows, stride;
    int32_t vocab, top;
    const int64_t* targets;
    float scale;
    float *logprob, *entropy, *norm;
    int32_t* top_ids;
    float* top_logprobs;
    const float *g_logprob, *g_entropy, *in_norm, *in_entropy;
    void* grad;
    int64_t grad_stride;
};

template <class T, class Op>
__device__ T block_reduce(T v, T* shared, Op op) {
    for (int o = 16; o; o >>= 1) v = op(v, __shfl_xor_sync(~0u, v, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
    __syncthreads();
    v = shared[0];
    for (int w = 1; w < kThreads / 32; ++w) v = op(v, shared[w]);
    return v;
}

struct RowStats {
    float m, s, log_s, entropy;
};

template <class E>
__device__ RowStats row_stats(const E* x, int V, float scale, float* shared) {
    auto plus = [](float a, float b) { return a + b; };
    float m = -CUDART_INF_F;
    for (int i = threadIdx.x; i < V; i += kThreads) m = max_nan(m, as_float(x[i]));
    m = block_reduce(m, shared, [](float a, float b) { return max_nan(a, b); });
    if (m != m || m == CUDART_INF_F) return {CUDART_NAN_F, CUDART_NAN_F, CUDART_NAN_F, CUDART_NAN_F};
    if (m == -CUDART_INF_F) return {m, 0.0f, -CUDART_INF_F, 0.0f};
    const float c = scale * kLog2E;
    float s = 0.0f, u = 0.0f;
    for (int i = threadIdx.x; i < V; i += kThreads) {
        const float t = fmaxf((as_float(x[i]) - m) * c, -200.0f);
        const float e = exp2_fast(t);
        s += e;
        u = fmaf(e, t, u);
    }
    s = block_reduce(s, shared, plus);
    u = block_reduce(u, shared, plus);
    return {m, s, logf(s), logf(s) - u / s * 0.6931471805599453f};
}

// the log probability of token t: NaN if there is no such token, -inf where the row or the token is masked
template <class E>
__device__ float given(const E* x, int V, int64_t t, const RowStats& r, float scale) {
    if (t >= V) return CUDART_NAN_F;
    if (r.m == -CUDART_INF_F) return r.m;
    return (as_float(x[t]) - r.m) * scale - r.log_s;
}

template <class E>
__global__ void __launch_bounds__(kThreads) logprobs_kernel(RowArgs a) {
    __shared__ float shared[kThreads / 32];
    __shared__ unsigned long long best[kThreads / 32];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const E* const x = static_cast<const E*>(a.logits) + row * a.stride;
        const int64_t t = a.targets ? a.targets[row] : 0;
        if (t < 0) {   // nobody asked for this row
            if (threadIdx.x == 0) {
                if (a.logprob) a.logprob[row] = 0.0f;
                if (a.entropy) a.entropy[row] = 0.0f;
                if (a.norm) a.norm[2 * row] = a.norm[2 * row + 1] = 0.0f;
            }
            for (int k = threadIdx.x; k < a.top; k += kThreads) {
                a.top_ids[row * a.top + k] = -1;
                a.top_logprobs[row * a.top + k] = -CUDART_INF_F;
            }
            continue;
        }
        const RowStats r = row_stats(x, a.vocab, a.scale, shared);
        if (threadIdx.x == 0) {
            if (a.logprob) a.logprob[row] = given(x, a.vocab, t, r, a.scale);
            if (a.entropy) a.entropy[row] = r.entropy;
            if (a.norm) a.norm[2 * row] = r.m, a.norm[2 * row + 1] = r.s;
        }
        unsigned long long last = ~0ull;
        for (int k = 0; k < a.top; ++k) {
            unsigned long long mine = 0;
            for (int i = threadIdx.x; i < a.vocab; i += kThreads) {
                const unsigned long long key = key_of(as_float(x[i]), i);
                if (key < last && key > mine) mine = key;
            }
            last = block_reduce(mine, best, [](unsigned long long p, unsigned long long q) { return p > q ? p : q; });
            if (threadIdx.x == 0) {
                a.top_ids[row * a.top + k] = last ? (int)position_of(last) : -1;
                a.top_logprobs[row * a.top + k] =
                    last ? r.m == -CUDART_INF_F ? r.m : (as_float(x[position_of(last)]) - r.m) * a.scale - r.log_s : -CUDART_INF_F;
            }
            if (!last) last = 1;   // the row has no more: every later key is below
        }
    }
}

// dx_i = c [ g (1[i = t] - p_i) - h p_i (ln p_i + H) ]
template <class E>
__device__ void write_gradient(const RowArgs& a, int64_t row, int64_t t, float m, float s, float log_s, float entropy, float g, float h) {
    const E* const x = static_cast<const E*>(a.logits) + row * a.stride;
    E* const out = static_cast<E*>(a.grad) + row * a.grad_stride;
    const float c = a.scale * kLog2E, per = 1.0f / s;
    const bool zero = t < 0 || m == -CUDART_INF_F, none = t >= a.vocab;
    for (int i = threadIdx.x; i < a.vocab; i += kThreads) {
        float y = 0.0f;
        if (none) {
            y = CUDART_NAN_F;
        } else if (!zero) {
            const float d = as_float(x[i]) - m, p = exp2_fast(d * c) * per;
            y = g * ((i == t ? 1.0f : 0.0f) - p);
            if (p > 0.0f && h != 0.0f) y -= h * p * (d * a.scale - log_s + entropy);
            y *= a.scale;
        }
        out[i] = from_float<E>(y);
    }
}

template <class E>
__global__ void __launch_bounds__(kThreads) grad_kernel(RowArgs a) {
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float s = a.in_norm[2 * row + 1];
        write_gradient<E>(a, row, a.targets[row], a.in_norm[2 * row], s, logf(s), a.in_entropy ? a.in_entropy[row] : 0.0f, a.g_logprob[row],
                          a.g_entropy ? a.g_entropy[row] : 0.0f);
    }
}

template <class E>
__global__ void __launch_bounds__(kThreads) loss_kernel(RowArgs a) {
    __shared__ float shared[kThreads / 32];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const E* const x = static_cast<const E*>(a.logits) + row * a.stride;
        const int64_t t = a.targets[row];
        RowStats r = {0.0f, 1.0f, 0.0f, 0.0f};
        if (t >= 0) r = row_stats(x, a.vocab, a.scale, shared);
        if (threadIdx.x == 0 && a.logprob) a.logprob[row] = t < 0 ? 0.0f : given(x, a.vocab, t, r, a.scale);
        __syncthreads();   // the gradient may take the logits' place
        write_gradient<E>(a, row, t, r.m, r.s, r.log_s, 0.0f, a.g_logprob[row], 0.0f);
    }
}

bool type_ok(int type) { return type == SLAQ_F32 || type == SLAQ_BF16 || type == SLAQ_F16; }
int64_t size_of(int type) { return type == SLAQ_F32 ? 4 : 2; }

// The gradient may lie in the logits' place, row for row, or apart from them; rows of both may alternate in one buffer.
bool overlap(const RowArgs& a, int64_t es) {
    const char *x = static_cast<const char*>(a.logits), *y = static_cast<const char*>(a.grad);
    const int64_t width = a.vocab * es;
    const char *x_end = x + (a.rows - 1) * a.stride * es + width, *y_end = y + (a.rows - 1) * a.grad_stride * es + width;
    if (x_end <= y || y_end <= x) return false;
    if (a.stride != a.grad_stride) return true;
    if (x == y) return false;
    const int64_t pitch = a.stride * es, apart = ((y - x) % pitch + pitch) % pitch;
    return apart < width || pitch - apart < width;
}

int check_rows(const RowArgs& a, int type) {
    if (!type_ok(type) || a.rows < 0 || a.vocab < 1 || !(a.scale > 0.0f) || a.scale > 3.0e38f) return SLAQ_E_ARG;
    if (a.vocab > kMaxVocab || a.rows > 0x7FFFFFFF) return SLAQ_E_RANGE;
    if (a.rows && (!a.logits || (a.rows > 1 && a.stride < 0))) return SLAQ_E_ARG;
    if (reinterpret_cast<uintptr_t>(a.logits) % size_of(type)) return SLAQ_E_ARG;
    return SLAQ_OK;
}
int check_gradient(const RowArgs& a, int type) {
    if (a.rows && (!a.targets || !a.grad || !a.g_logprob || (a.rows > 1 && a.grad_stride < a.vocab))) return SLAQ_E_ARG;
    if (reinterpret_cast<uintptr_t>(a.grad) % size_of(type)) return SLAQ_E_ARG;
    return a.rows && overlap(a, size_of(type)) ? SLAQ_E_ARG : SLAQ_OK;
}

int done() { return cudaGetLastError() == cudaSuccess ? SLAQ_OK : SLAQ_E_CUDA; }

template <class F>
int by_type(int type, F&& f) {
    if (type == SLAQ_F32) f(0.0f);
    else if (type == SLAQ_BF16) f(__nv_bfloat16());
    else f(__half());
    return done();
}

}  // namespace
}  // namespace slaq

extern "C" int slaq_token_logprobs(const void* d_logits, int type, int64_t rows, int32_t vocab, int64_t row_stride, const int64_t* d_targets,
                                   float scale, float* d_out_logprob, float* d_out_entropy, float* d_out_norm, int32_t top,
                                   int32_t* d_out_top_ids, float* d_out_top_logprobs, void* cuda_stream) {
    using namespace slaq;
    RowArgs a = {};
    a.logits = d_logits, a.rows = rows, a.vocab = vocab, a.stride = row_stride, a.targets = d_targets, a.scale = scale;
    a.logprob = d_out_logprob, a.entropy = d_out_entropy, a.norm = d_out_norm;
    a.top = top, a.top_ids = d_out_top_ids, a.top_logprobs = d_out_top_logprobs;
    if (const int rc = check_rows(a, type)) return rc;
    if (top < 0 || (top > 0 && rows && (!d_out_top_ids || !d_out_top_logprobs)) || (d_out_logprob && !d_targets && rows)) return SLAQ_E_ARG;
    if (top > kMaxTop) return SLAQ_E_RANGE;
    if (rows == 0) return SLAQ_OK;
    return by_type(type, [&](auto e) {
        logprobs_kernel<decltype(e)><<<(unsigned)rows, kThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(a);
    });
}

extern "C" int slaq_token_logprobs_grad(const void* d_logits, int type, int64_t rows, int32_t vocab, int64_t row_stride,
                                        const int64_t* d_targets, float scale, const float* d_norm, const float* d_entropy,
                                        const float* d_grad_logprob, const float* d_grad_entropy, void* d_out_grad, int64_t grad_stride,
                                        void* cuda_stream) {
    using namespace slaq;
    RowArgs a = {};
    a.logits = d_logits, a.rows = rows, a.vocab = vocab, a.stride = row_stride, a.targets = d_targets, a.scale = scale;
    a.in_norm = d_norm, a.in_entropy = d_entropy, a.g_logprob = d_grad_logprob, a.g_entropy = d_grad_entropy;
    a.grad = d_out_grad, a.grad_stride = grad_stride;
    if (const int rc = check_rows(a, type)) return rc;
    if (rows && (!d_norm || (d_grad_entropy && !d_entropy))) return SLAQ_E_ARG;
    if (const int rc = check_gradient(a, type)) return rc;
    if (rows == 0) return SLAQ_OK;
    return by_type(type, [&](auto e) {
        grad_kernel<decltype(e)><<<(unsigned)rows, kThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(a);
    });
}

extern "C" int slaq_token_loss(const void* d_logits, int type, int64_t rows, int32_t vocab, int64_t row_stride, const int64_t* d_targets,
                               float scale, const float* d_row_grad, float* d_out_logprob, void* d_out_grad, int64_t grad_stride,
                               void* cuda_stream) {
    using namespace slaq;
    RowArgs a = {};
    a.logits = d_logits, a.rows = rows, a.vocab = vocab, a.stride = row_stride, a.targets = d_targets, a.scale = scale;
    a.g_logprob = d_row_grad, a.logprob = d_out_logprob, a.grad = d_out_grad, a.grad_stride = grad_stride;
    if (const int rc = check_rows(a, type)) return rc;
    if (const int rc = check_gradient(a, type)) return rc;
    if (rows == 0) return SLAQ_OK;
    return by_type(type, [&](auto e) {
        loss_kernel<decltype(e)><<<(unsigned)rows, kThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(a);
    });
}
