// One AdamW step over the tensors of many jobs.
//
// Per element, in 32 bits and every operation rounded on its own:
//     g = grad grad_scale;   m = b1 m + (1-b1) g;   v = b2 v + (1-b2) g g;   r = sqrt v
//     p = p (1 - lr decay) - lr / (1 - b1^t) * m / (r / sqrt(1 - b2^t) + eps)
// States in 8 bits: 256 elements of a tensor share a scale; m is e4m3 times max|m|/448 and r (not v, whose range is twice as
// wide in octaves) e4m3 times max r/448.  The step itself works on the unrounded m and r of this step; the rounding, to
// nearest, is what the next step finds: at most 2^-4 of a value, 2^-10 of the block's scale where e4m3 is subnormal.  A
// second moment that is not zero never becomes zero: its element would then be divided by eps alone.
#include <cuda_fp8.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <utility>
#include <vector>

#include "slaq_internal.cuh"
#include "slaq_rows.cuh"

namespace slaq {
namespace {

constexpr int kBlock = 256;          // elements that share a scale, and what a warp works on at a time: 8 a lane
constexpr int kItemBlocks = 4;       // blocks of a work item
constexpr int kThreads = 256;
constexpr float kE4m3Max = 448.0f;
constexpr float kTiny = 7.888609052210118e-31f;   // 2^-100: a block with nothing above it is kept as zeros

struct TensorRef {
    void* param;
    float* master;
    void* avg;
    void* sq;
    float* avg_scale;
    float* sq_scale;
    int64_t n;
    int32_t group, pad;
};

// What a step needs of a group, ready for its next step: the block that finishes a step last moves it on.
struct Group {
    double lr, beta1, beta2;
    int64_t step;                    // steps taken
    float b1, a1, b2, a2, correct, eps, keep, size, grad_scale;
    int32_t pad;
};
static_assert(sizeof(Group) == 72, "read as whole words");

__host__ __device__ inline void for_next_step(Group& g) {
    const double t = (double)(g.step + 1);
    g.correct = (float)(1.0 / sqrt(1.0 - pow(g.beta2, t)));
    g.size = (float)(g.lr / (1.0 - pow(g.beta1, t)));
}

struct Item {
    int32_t tensor, block;           // blocks [block, block + kItemBlocks) of the tensor, as far as it goes
};

struct StepArgs {
    const TensorRef* tensors;
    const void* const* grads;
    const Item* items;
    int64_t n_items;
    Group* groups;
    int32_t n_groups;
    const int32_t* active;
    unsigned int* ticket;
};

template <class E>
__device__ __forceinline__ void load8(const E* from, int64_t i, int64_t n, bool wide, float (&x)[8]) {
    if (wide && i + 8 <= n) {
        alignas(16) E e[8];
#pragma unroll
        for (int k = 0; k < (int)sizeof(e) / 16; ++k) reinterpret_cast<uint4*>(e)[k] = reinterpret_cast<const uint4*>(from + i)[k];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = as_float(e[k]);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = i + k < n ? as_float(from[i + k]) : 0.0f;
    }
}
template <class E>
__device__ __forceinline__ void store8(E* to, int64_t i, int64_t n, bool wide, const float (&x)[8]) {
    if (wide && i + 8 <= n) {
        alignas(16) E e[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) e[k] = from_float<E>(x[k]);
#pragma unroll
        for (int k = 0; k < (int)sizeof(e) / 16; ++k) reinterpret_cast<uint4*>(to + i)[k] = reinterpret_cast<const uint4*>(e)[k];
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (i + k < n) to[i + k] = from_float<E>(x[k]);
    }
}

__device__ __forceinline__ float from_e4m3(uint8_t b) {
    return __half2float(__half(__nv_cvt_fp8_to_halfraw(b, __NV_E4M3)));
}
__device__ __forceinline__ void load8_codes(const uint8_t* from, int64_t i, int64_t n, bool wide, float scale, float (&x)[8]) {
    alignas(8) uint8_t b[8];
    if (wide && i + 8 <= n) {
        *reinterpret_cast<uint2*>(b) = *reinterpret_cast<const uint2*>(from + i);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) b[k] = i + k < n ? from[i + k] : 0;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = __fmul_rn(from_e4m3(b[k]), scale);
}
// The largest finite |x| of the warp, its scale out, and the codes.  What is not finite stays so in its own element (NaN).
template <bool kPositive>
__device__ __forceinline__ void store8_codes(uint8_t* to, int64_t i, int64_t n, bool wide, float* scale, int lane, const float (&x)[8]) {
    float most = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (i + k < n && fabsf(x[k]) < CUDART_INF_F) most = fmaxf(most, fabsf(x[k]));
    most = __uint_as_float(__reduce_max_sync(~0u, __float_as_uint(most)));
    const bool kept = most >= kTiny;
    const float inverse = kept ? __fdiv_rn(kE4m3Max, most) : 0.0f;
    if (lane == 0) *scale = kept ? __fdiv_rn(most, kE4m3Max) : 0.0f;
    alignas(8) uint8_t b[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        float y = __fmul_rn(x[k], inverse);
        if (kPositive && kept && x[k] > 0.0f) y = fmaxf(y, 0.001953125f);   // 2^-9, the smallest e4m3
        b[k] = fabsf(x[k]) < CUDART_INF_F ? __nv_cvt_float_to_fp8(y, __NV_SATFINITE, __NV_E4M3) : 0x7F;
    }
    if (wide && i + 8 <= n) {
        *reinterpret_cast<uint2*>(to + i) = *reinterpret_cast<const uint2*>(b);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (i + k < n) to[i + k] = b[k];
    }
}

template <class P, class G, bool kMaster, bool kEight>
__global__ void __launch_bounds__(kThreads) step_kernel(StepArgs a) {
    const int lane = threadIdx.x & 31;
    const int64_t warps = (int64_t)gridDim.x * (kThreads / 32);
    for (int64_t it = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); it < a.n_items; it += warps) {
        const Item item = a.items[it];
        const TensorRef t = a.tensors[item.tensor];
        if (a.active && a.active[t.group] <= 0) continue;
        const Group& c = a.groups[t.group];
        const float b1 = c.b1, a1 = c.a1, b2 = c.b2, a2 = c.a2, correct = c.correct, eps = c.eps, keep = c.keep, size = c.size, gs = c.grad_scale;
        const G* const grad = static_cast<const G*>(a.grads[item.tensor]);
        uintptr_t low = (uintptr_t)t.param | (uintptr_t)grad | (uintptr_t)t.master;
        if (!kEight) low |= (uintptr_t)t.avg | (uintptr_t)t.sq;
        const bool wide = (low & 15) == 0 && (!kEight || (((uintptr_t)t.avg | (uintptr_t)t.sq) & 7) == 0);
        for (int k = 0; k < kItemBlocks; ++k) {
            const int64_t block = item.block + k, i = block * kBlock + lane * 8;
            if (block * kBlock >= t.n) break;
            float p[8], g[8], m[8], v[8];
            load8(grad, i, t.n, wide, g);
            if (kMaster) load8(t.master, i, t.n, wide, p);
            else load8(static_cast<const P*>(t.param), i, t.n, wide, p);
            if (kEight) {
                load8_codes(static_cast<const uint8_t*>(t.avg), i, t.n, wide, t.avg_scale[block], m);
                load8_codes(static_cast<const uint8_t*>(t.sq), i, t.n, wide, t.sq_scale[block], v);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = __fmul_rn(v[j], v[j]);
            } else {
                load8(static_cast<const float*>(t.avg), i, t.n, wide, m);
                load8(static_cast<const float*>(t.sq), i, t.n, wide, v);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float x = __fmul_rn(g[j], gs);
                m[j] = __fadd_rn(__fmul_rn(b1, m[j]), __fmul_rn(a1, x));
                v[j] = __fadd_rn(__fmul_rn(b2, v[j]), __fmul_rn(a2, __fmul_rn(x, x)));
                const float r = __fsqrt_rn(v[j]);
                const float by = __fadd_rn(__fmul_rn(r, correct), eps);
                p[j] = __fsub_rn(__fmul_rn(p[j], keep), __fmul_rn(size, __fdiv_rn(m[j], by)));
                if (kEight) v[j] = r;
            }
            if (kMaster) store8(t.master, i, t.n, wide, p);
            store8(static_cast<P*>(t.param), i, t.n, wide, p);
            if (kEight) {
                store8_codes<false>(static_cast<uint8_t*>(t.avg), i, t.n, wide, t.avg_scale + block, lane, m);
                store8_codes<true>(static_cast<uint8_t*>(t.sq), i, t.n, wide, t.sq_scale + block, lane, v);
            } else {
                store8(static_cast<float*>(t.avg), i, t.n, wide, m);
                store8(static_cast<float*>(t.sq), i, t.n, wide, v);
            }
        }
    }
    // the last block moves the groups on to their next step
    __shared__ unsigned int arrived;
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        arrived = atomicAdd(a.ticket, 1u);
    }
    __syncthreads();
    if (arrived != gridDim.x - 1) return;
    for (int k = threadIdx.x; k < a.n_groups; k += kThreads)
        if (!a.active || a.active[k] > 0) {
            Group g = a.groups[k];
            ++g.step;
            for_next_step(g);
            a.groups[k].step = g.step;
            a.groups[k].correct = g.correct;
            a.groups[k].size = g.size;
        }
    if (threadIdx.x == 0) *a.ticket = 0;
}

__global__ void set_group_kernel(Group* groups, int32_t k, Group g, bool keep_step) {
    if (keep_step) g.step = groups[k].step;
    for_next_step(g);
    groups[k] = g;
}

__global__ void fill_items_kernel(const int32_t* first_item, int32_t n_tensors, Item* items) {
    const int t = blockIdx.x;
    for (int i = first_item[t] + threadIdx.x; i < first_item[t + 1]; i += blockDim.x) items[i] = {t, (i - first_item[t]) * kItemBlocks};
}

using StepFn = void (*)(StepArgs);
template <class P, class G>
StepFn pick(bool master, bool eight) {
    if (master) return eight ? step_kernel<P, G, true, true> : step_kernel<P, G, true, false>;
    return eight ? step_kernel<P, G, false, true> : step_kernel<P, G, false, false>;
}

size_t up(size_t n) { return (n + 255) & ~size_t(255); }

}  // namespace
}  // namespace slaq

struct slaq_adamw_handle {
    int device = 0;
    int32_t n_tensors = 0, n_groups = 0;
    int64_t n_items = 0;
    bool owns_ws = false;
    void* ws = nullptr;
    slaq::TensorRef* tensors = nullptr;
    void** grads = nullptr;
    int32_t* first_item = nullptr;
    slaq::Item* items = nullptr;
    slaq::Group* groups = nullptr;
    unsigned int* ticket = nullptr;
    slaq::StepFn step = nullptr;
    int blocks = 0;
    size_t grad_size = 0;                                        // bytes of a gradient's element
    std::vector<int64_t> numel;
    std::vector<std::pair<uintptr_t, uintptr_t>> written;        // sorted: what a step writes
    const char* err = "";
};

namespace slaq {
namespace {

int fail(slaq_adamw_handle* h, int code, const char* what) {
    h->err = what;
    return code;
}
bool on_device(const slaq_adamw_handle* h) {
    int d = -1;
    return cudaGetDevice(&d) == cudaSuccess && d == h->device;
}
bool group_ok(const slaq_adamw_group& g) {
    auto in = [](double x, double lo, double hi) { return x >= lo && x < hi; };
    return in(g.lr, 0.0, 1e30) && in(g.beta1, 0.0, 1.0) && in(g.beta2, 0.0, 1.0) && in(g.eps, 0.0, 1e30) && in(g.weight_decay, 0.0, 1e30) &&
           std::isfinite(g.grad_scale);
}
Group device_group(const slaq_adamw_group& g) {
    Group d = {};
    d.lr = g.lr, d.beta1 = g.beta1, d.beta2 = g.beta2, d.step = g.step;
    d.b1 = (float)g.beta1, d.a1 = (float)(1.0 - g.beta1), d.b2 = (float)g.beta2, d.a2 = (float)(1.0 - g.beta2);
    d.eps = (float)g.eps, d.keep = (float)(1.0 - g.lr * g.weight_decay), d.grad_scale = (float)g.grad_scale;
    for_next_step(d);
    return d;
}
size_t size_of(int type) { return type == SLAQ_F32 ? 4 : 2; }
int64_t items_of(int64_t n) { return (n + kBlock * kItemBlocks - 1) / (kBlock * kItemBlocks); }

// bytes of the plan's device memory, and with `h` where its parts lie
size_t layout(slaq_adamw_handle* h, char* base, int32_t n_tensors, int64_t n_items, int32_t n_groups) {
    size_t at = 0;
    auto part = [&](auto*& p, size_t bytes) {
        if (h) p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(base + at);
        at += up(bytes);
    };
    slaq_adamw_handle none;
    slaq_adamw_handle& o = h ? *h : none;
    part(o.tensors, sizeof(TensorRef) * (size_t)n_tensors);
    part(o.grads, sizeof(void*) * (size_t)n_tensors);
    part(o.first_item, sizeof(int32_t) * ((size_t)n_tensors + 1));
    part(o.items, sizeof(Item) * (size_t)n_items);
    part(o.groups, sizeof(Group) * (size_t)n_groups);
    part(o.ticket, sizeof(unsigned int));
    return at;
}

// an interval of memory that meets one of `sorted`, which do not meet one another
bool meets(const std::vector<std::pair<uintptr_t, uintptr_t>>& sorted, uintptr_t lo, uintptr_t hi) {
    auto it = std::upper_bound(sorted.begin(), sorted.end(), std::make_pair(lo, UINTPTR_MAX));
    if (it != sorted.end() && it->first < hi) return true;
    return it != sorted.begin() && std::prev(it)->second > lo;
}

int check_grads(slaq_adamw_handle* h, const void* const* grads) {
    for (int32_t t = 0; t < h->n_tensors; ++t) {
        if (!h->numel[t]) continue;
        const uintptr_t lo = (uintptr_t)grads[t];
        if (!lo || lo % h->grad_size) return fail(h, SLAQ_E_ARG, "a gradient is null or not aligned to its type");
        if (meets(h->written, lo, lo + h->grad_size * (size_t)h->numel[t])) return fail(h, SLAQ_E_ARG, "a gradient overlaps what the step writes");
    }
    return SLAQ_OK;
}

int create(slaq_adamw_handle* h, void* dev_ws, size_t bytes, int32_t n_tensors, const slaq_adamw_tensor* tensors, int32_t n_groups,
           const slaq_adamw_group* groups, int param_type, int grad_type, int state_bits, cudaStream_t st) {
    const bool eight = state_bits == 8;
    bool masters = false;
    std::vector<TensorRef> refs((size_t)n_tensors);
    std::vector<int32_t> first((size_t)n_tensors + 1, 0);
    std::vector<const void*> grads((size_t)n_tensors);
    h->numel.resize((size_t)n_tensors);
    int64_t items = 0;
    for (int32_t t = 0; t < n_tensors; ++t) {
        const slaq_adamw_tensor& x = tensors[t];
        if (x.n < 0 || x.group < 0 || x.group >= n_groups) return SLAQ_E_ARG;
        refs[t] = {x.param, x.master, x.exp_avg, x.exp_avg_sq, x.exp_avg_scale, x.exp_avg_sq_scale, x.n, x.group, 0};
        grads[t] = x.grad;
        h->numel[t] = x.n;
        first[t] = (int32_t)items;
        if (x.n >> 40) return SLAQ_E_RANGE;
        items += items_of(x.n);
        if (items > 0x7FFFFFFF / kItemBlocks) return SLAQ_E_RANGE;   // block indices are 32 bits wide
        if (!x.n) continue;
        if (!x.param || !x.exp_avg || !x.exp_avg_sq || (eight && (!x.exp_avg_scale || !x.exp_avg_sq_scale))) return SLAQ_E_ARG;
        masters |= x.master != nullptr;
        auto writes = [&](const void* p, size_t size, int64_t n) {
            if (!p) return true;
            h->written.emplace_back((uintptr_t)p, (uintptr_t)p + size * (size_t)n);
            return (uintptr_t)p % size == 0;
        };
        const int64_t blocks = (x.n + kBlock - 1) / kBlock;
        bool ok = writes(x.param, size_of(param_type), x.n) && writes(x.master, 4, x.n) && writes(x.exp_avg, eight ? 1 : 4, x.n) &&
                  writes(x.exp_avg_sq, eight ? 1 : 4, x.n);
        if (eight) ok = ok && writes(x.exp_avg_scale, 4, blocks) && writes(x.exp_avg_sq_scale, 4, blocks);
        if (!ok) return SLAQ_E_ARG;
    }
    first[n_tensors] = (int32_t)items;
    for (int32_t t = 0; t < n_tensors; ++t)
        if (masters && tensors[t].n && !tensors[t].master) return SLAQ_E_ARG;   // all tensors of a plan have a master copy, or none has
    std::sort(h->written.begin(), h->written.end());
    for (size_t k = 1; k < h->written.size(); ++k)
        if (h->written[k].first < h->written[k - 1].second) return SLAQ_E_ARG;   // a tensor listed twice, or overlapping ones
    h->n_tensors = n_tensors;
    h->n_groups = n_groups;
    h->n_items = items;
    h->grad_size = size_of(grad_type);
    if (const int rc = check_grads(h, grads.data())) return rc;
    if (param_type == SLAQ_F32) h->step = pick<float, float>(masters, eight);
    else if (param_type == SLAQ_BF16) h->step = grad_type == SLAQ_F32 ? pick<__nv_bfloat16, float>(masters, eight) : pick<__nv_bfloat16, __nv_bfloat16>(masters, eight);
    else h->step = grad_type == SLAQ_F32 ? pick<__half, float>(masters, eight) : pick<__half, __half>(masters, eight);
    if (cudaGetDevice(&h->device) != cudaSuccess) return SLAQ_E_CUDA;
    const size_t need = layout(nullptr, nullptr, n_tensors, items, n_groups);
    if (dev_ws) {
        if (((uintptr_t)dev_ws & 255) || bytes < need) return SLAQ_E_NOMEM;
        h->ws = dev_ws;
    } else {
        if (cudaMalloc(&h->ws, need) != cudaSuccess) {
            (void)cudaGetLastError();
            return SLAQ_E_NOMEM;
        }
        h->owns_ws = true;
    }
    layout(h, static_cast<char*>(h->ws), n_tensors, items, n_groups);
    std::vector<Group> gs((size_t)n_groups);
    for (int32_t k = 0; k < n_groups; ++k) gs[k] = device_group(groups[k]);
    auto to_device = [&](void* to, const void* from, size_t n) { return n == 0 || cudaMemcpyAsync(to, from, n, cudaMemcpyHostToDevice, st) == cudaSuccess; };
    int sm = 0, per_sm = 0;
    if (!to_device(h->tensors, refs.data(), sizeof(TensorRef) * refs.size()) || !to_device(h->grads, grads.data(), sizeof(void*) * grads.size()) ||
        !to_device(h->first_item, first.data(), sizeof(int32_t) * first.size()) || !to_device(h->groups, gs.data(), sizeof(Group) * gs.size()) ||
        cudaMemsetAsync(h->ticket, 0, sizeof(unsigned int), st) != cudaSuccess ||
        cudaDeviceGetAttribute(&sm, cudaDevAttrMultiProcessorCount, h->device) != cudaSuccess ||
        cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, h->step, kThreads, 0) != cudaSuccess)
        return SLAQ_E_CUDA;
    if (n_tensors) fill_items_kernel<<<n_tensors, 128, 0, st>>>(h->first_item, n_tensors, h->items);
    if (cudaGetLastError() != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess) return SLAQ_E_CUDA;   // the lists above end here
    const int64_t wanted = (items + kThreads / 32 - 1) / (kThreads / 32);
    h->blocks = (int)std::max<int64_t>(1, std::min<int64_t>(wanted, (int64_t)sm * std::max(per_sm, 1)));
    return SLAQ_OK;
}

}  // namespace
}  // namespace slaq

extern "C" {

size_t slaq_adamw_workspace_bytes(int32_t n_tensors, const int64_t* numels, int32_t n_groups) {
    if (n_tensors < 0 || n_groups < 1 || (n_tensors && !numels)) return 0;
    int64_t items = 0;
    for (int32_t t = 0; t < n_tensors; ++t) {
        if (numels[t] < 0 || numels[t] >> 40) return 0;
        items += slaq::items_of(numels[t]);
    }
    return slaq::layout(nullptr, nullptr, n_tensors, items, n_groups);
}

int slaq_adamw_create(void* dev_ws, size_t bytes, int32_t n_tensors, const slaq_adamw_tensor* tensors, int32_t n_groups,
                      const slaq_adamw_group* groups, int param_type, int grad_type, int state_bits, void* cuda_stream, slaq_adamw_t** out) {
    if (!out) return SLAQ_E_ARG;
    *out = nullptr;
    auto type_ok = [](int t) { return t == SLAQ_F32 || t == SLAQ_BF16 || t == SLAQ_F16; };
    if (n_tensors < 0 || n_groups < 1 || (n_tensors && !tensors) || !groups || !type_ok(param_type) || !type_ok(grad_type) ||
        (grad_type != SLAQ_F32 && grad_type != param_type) || (state_bits != 8 && state_bits != 32))
        return SLAQ_E_ARG;
    for (int32_t k = 0; k < n_groups; ++k)
        if (!slaq::group_ok(groups[k]) || groups[k].step < 0) return SLAQ_E_ARG;
    slaq_adamw_handle* h = new (std::nothrow) slaq_adamw_handle();
    if (!h) return SLAQ_E_NOMEM;
    int rc;
    try {
        rc = slaq::create(h, dev_ws, bytes, n_tensors, tensors, n_groups, groups, param_type, grad_type, state_bits, static_cast<cudaStream_t>(cuda_stream));
    } catch (const std::bad_alloc&) {
        rc = SLAQ_E_NOMEM;
    }
    if (rc < 0) {
        slaq_adamw_destroy(h);
        return rc;
    }
    *out = h;
    return SLAQ_OK;
}

int slaq_adamw_destroy(slaq_adamw_t* h) {
    if (!h) return SLAQ_OK;
    if (h->owns_ws && h->ws) cudaFree(h->ws);   // waits for the steps that still read it
    delete h;
    return SLAQ_OK;
}

const char* slaq_adamw_last_error(const slaq_adamw_t* h) { return h ? h->err : "null handle"; }

int slaq_adamw_step(slaq_adamw_t* h, const int32_t* d_active, void* cuda_stream) {
    if (!h) return SLAQ_E_ARG;
    if (!slaq::on_device(h)) return slaq::fail(h, SLAQ_E_ARG, "the plan's device is not the current one");
    slaq::StepArgs a = {h->tensors, h->grads, h->items, h->n_items, h->groups, h->n_groups, d_active, h->ticket};
    h->step<<<h->blocks, slaq::kThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(a);
    return cudaGetLastError() == cudaSuccess ? SLAQ_OK : slaq::fail(h, SLAQ_E_CUDA, "the step could not be launched");
}

int slaq_adamw_set_group(slaq_adamw_t* h, int32_t group, const slaq_adamw_group* g, void* cuda_stream) {
    if (!h) return SLAQ_E_ARG;
    if (!slaq::on_device(h)) return slaq::fail(h, SLAQ_E_ARG, "the plan's device is not the current one");
    if (!g || !slaq::group_ok(*g)) return slaq::fail(h, SLAQ_E_ARG, "a group's values are out of range");
    if (group < 0 || group >= h->n_groups) return slaq::fail(h, SLAQ_E_RANGE, "no such group");
    slaq_adamw_group v = *g;
    const bool keep = v.step < 0;
    if (keep) v.step = 0;
    slaq::set_group_kernel<<<1, 1, 0, static_cast<cudaStream_t>(cuda_stream)>>>(h->groups, group, slaq::device_group(v), keep);
    return cudaGetLastError() == cudaSuccess ? SLAQ_OK : slaq::fail(h, SLAQ_E_CUDA, "the group could not be set");
}

int slaq_adamw_set_grads(slaq_adamw_t* h, const void* const* grads, void* cuda_stream) {
    if (!h) return SLAQ_E_ARG;
    if (!slaq::on_device(h)) return slaq::fail(h, SLAQ_E_ARG, "the plan's device is not the current one");
    if (h->n_tensors == 0) return SLAQ_OK;
    if (!grads) return slaq::fail(h, SLAQ_E_ARG, "grads is null");
    if (const int rc = slaq::check_grads(h, grads)) return rc;
    cudaStreamCaptureStatus capturing = cudaStreamCaptureStatusNone;
    if (cudaStreamIsCapturing(static_cast<cudaStream_t>(cuda_stream), &capturing) != cudaSuccess || capturing != cudaStreamCaptureStatusNone)
        return slaq::fail(h, SLAQ_E_ARG, "gradients are not changed while the stream is captured");
    if (cudaMemcpyAsync(h->grads, grads, sizeof(void*) * (size_t)h->n_tensors, cudaMemcpyHostToDevice, static_cast<cudaStream_t>(cuda_stream)) != cudaSuccess)
        return slaq::fail(h, SLAQ_E_CUDA, "copy of the gradients' addresses");
    return SLAQ_OK;
}

int slaq_adamw_get_steps(slaq_adamw_t* h, int64_t* out_steps, void* cuda_stream) {
    if (!h) return SLAQ_E_ARG;
    if (!slaq::on_device(h)) return slaq::fail(h, SLAQ_E_ARG, "the plan's device is not the current one");
    if (!out_steps) return slaq::fail(h, SLAQ_E_ARG, "out_steps is null");
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (cudaMemcpy2DAsync(out_steps, sizeof(int64_t), &h->groups->step, sizeof(slaq::Group), sizeof(int64_t), (size_t)h->n_groups,
                          cudaMemcpyDeviceToHost, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess)
        return slaq::fail(h, SLAQ_E_CUDA, "copy of the steps");
    return SLAQ_OK;
}

}  // extern "C"
