// One AdamW step over the tensors of many jobs.
//
// Per element, in 32 bits:
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
constexpr int kThreads = 128;
constexpr bool kAhead = true;
constexpr int64_t kMostElements = (int64_t)1 << 38;   // of a plan: its blocks are counted in 31 bits
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
    int32_t group, first;            // the number of its first block among all tensors' blocks
};

// What a step needs of a group, ready for its next step: the block that finishes a step last moves it on.
struct Group {
    double lr, beta1, beta2, power1, power2;   // power: beta to the number of the next step
    int64_t step;                    // steps taken
    float b1, a1, b2, a2, correct, eps, keep, size, grad_scale;
    int32_t pad;
};

__host__ __device__ inline void corrections(Group& g) {
    g.correct = (float)(1.0 / sqrt(1.0 - g.power2));
    g.size = (float)(g.lr / (1.0 - g.power1));
}
__host__ __device__ inline void set_step(Group& g, int64_t step) {
    g.step = step;
    g.power1 = pow(g.beta1, (double)(step + 1));
    g.power2 = pow(g.beta2, (double)(step + 1));
    corrections(g);
}
// One product a step: a million steps put 1e-10 of their relative error into a power, which is 0 long before that.
__device__ inline void advance(Group& g) {
    ++g.step;
    g.power1 *= g.beta1;
    g.power2 *= g.beta2;
    corrections(g);
}

struct StepArgs {
    const TensorRef* tensors;
    const void* const* grads;
    const int32_t* tensor_of;        // per block
    int32_t n_blocks, n_groups;
    Group* groups;
    const int32_t* active;
    unsigned int* ticket;
};

// 8 elements as they lie in memory.
template <class E>
struct Raw {
    uint4 w[sizeof(E) / 2];
    __device__ __forceinline__ void load(const E* from) {
#pragma unroll
        for (int k = 0; k < (int)sizeof(E) / 2; ++k) w[k] = reinterpret_cast<const uint4*>(from)[k];
    }
    __device__ __forceinline__ void store(E* to) const {
#pragma unroll
        for (int k = 0; k < (int)sizeof(E) / 2; ++k) reinterpret_cast<uint4*>(to)[k] = w[k];
    }
    __device__ __forceinline__ void unpack(float (&x)[8]) const {
#pragma unroll
        for (int k = 0; k < 8; k += 2) {
            Vector<E> v;
            v.w = w[k * sizeof(E) / 16];
            split(v.at(k % Vector<E>::N / 2), x[k], x[k + 1]);
        }
    }
    __device__ __forceinline__ void pack(const float (&x)[8]) {
#pragma unroll
        for (int k = 0; k < 8; k += 2) {
            Vector<E> v;
            v.w = w[k * sizeof(E) / 16];
            v.put(k % Vector<E>::N / 2, pair_of(x[k], x[k + 1]));
            w[k * sizeof(E) / 16] = v.w;
        }
    }
};
// The elements i .. i + 8 of n; `whole`: all of them are there, and the address is a multiple of 16 bytes.
template <class E>
__device__ __forceinline__ void load8(const E* from, int64_t i, int64_t n, bool whole, float (&x)[8]) {
    if (whole) {
        Raw<E> r;
        r.load(from + i);
        r.unpack(x);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = i + k < n ? as_float(from[i + k]) : 0.0f;
    }
}
template <class E>
__device__ __forceinline__ void store8(E* to, int64_t i, int64_t n, bool whole, const float (&x)[8]) {
    if (whole) {
        Raw<E> r = {};
        r.pack(x);
        r.store(to + i);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (i + k < n) to[i + k] = from_float<E>(x[k]);
    }
}

// 8 codes and their scale
__device__ __forceinline__ void unpack_codes(uint2 b, float scale, float (&x)[8]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t w = k < 2 ? b.x : b.y;
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(k & 1 ? w >> 16 : w), __NV_E4M3);
        const float2 f = __half22float2(__half2(h));
        x[2 * k] = f.x * scale;
        x[2 * k + 1] = f.y * scale;
    }
}
__device__ __forceinline__ void load8_codes(const uint8_t* from, int64_t i, int64_t n, float scale, float (&x)[8]) {
    uint32_t b[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (i + k < n) b[k / 4] |= (uint32_t)from[i + k] << (k % 4 * 8);
    unpack_codes(make_uint2(b[0], b[1]), scale, x);
}
__device__ __forceinline__ float max_size(float a, float b) {   // max of |a| and |b|, sign aside; NaN as soon as one is
    float y;
    asm("max.NaN.xorsign.abs.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
// The codes of the warp's 256 values and their scale, largest / 448.  What is not finite stays so in its own element (NaN).
template <bool kPositive>
__device__ __forceinline__ uint2 to_codes(float* scale, int lane, const float (&x)[8]) {
    float most = x[0];
#pragma unroll
    for (int k = 1; k < 8; ++k) most = kPositive ? max_nan(most, x[k]) : max_size(most, x[k]);
    most = __uint_as_float(__reduce_max_sync(~0u, __float_as_uint(fabsf(most))));   // a NaN's bits stand above all
    const bool finite = most < CUDART_INF_F;
    if (!finite) {
        most = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (fabsf(x[k]) < CUDART_INF_F) most = fmaxf(most, fabsf(x[k]));
        most = __uint_as_float(__reduce_max_sync(~0u, __float_as_uint(most)));
    }
    const bool kept = most >= kTiny;
    const float inverse = kept ? __fdiv_rn(kE4m3Max, most) : 0.0f;
    if (lane == 0) *scale = kept ? __fdiv_rn(most, kE4m3Max) : 0.0f;
    float y[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) y[k] = x[k] * inverse;
    if (kPositive && kept) {
        constexpr float kLeast = 0.001953125f;   // 2^-9, the smallest code
        float least = y[0];
#pragma unroll
        for (int k = 1; k < 8; ++k) least = fminf(least, y[k]);
        if (least < kLeast)
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (x[k] > 0.0f) y[k] = fmaxf(y[k], kLeast);
    }
    uint32_t b[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        uint16_t two;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(two) : "f"(y[2 * k + 1]), "f"(y[2 * k]));
        b[k] = two;
        if (!finite) {
            if (!(fabsf(x[2 * k]) < CUDART_INF_F)) b[k] = (b[k] & 0xFF00u) | 0x7F;
            if (!(fabsf(x[2 * k + 1]) < CUDART_INF_F)) b[k] = (b[k] & 0xFFu) | 0x7F00;
        }
    }
    return make_uint2(__byte_perm(b[0], b[1], 0x5410), __byte_perm(b[2], b[3], 0x5410));
}
__device__ __forceinline__ void store8_codes(uint8_t* to, int64_t i, int64_t n, bool whole, uint2 b) {
    if (whole) {
        *reinterpret_cast<uint2*>(to + i) = b;
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (i + k < n) to[i + k] = (uint8_t)((k < 4 ? b.x : b.y) >> (k % 4 * 8));
    }
}

// sqrt and 1/x to 1 ulp or two, denormal arguments of the root included
__device__ __forceinline__ float root(float x) {
    float y;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float reciprocal(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// What a step needs of a group.
struct Numbers {
    float b1, a1, b2, a2, correct, eps, keep, size, grad_scale;
};
// 8 elements' step: new weights, first moments, and second moments (their roots, if kRoot)
template <bool kRoot>
__device__ __forceinline__ void step8(const Numbers& c, float (&p)[8], const float (&g)[8], float (&m)[8], float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float x = g[j] * c.grad_scale;
        m[j] = fmaf(c.b1, m[j], c.a1 * x);
        v[j] = fmaf(c.b2, v[j], c.a2 * (x * x));
        const float r = root(v[j]);
        p[j] = fmaf(-c.size, m[j] * reciprocal(fmaf(r, c.correct, c.eps)), p[j] * c.keep);
        if (kRoot) v[j] = r;
    }
}

template <bool kEight>
struct RawState : Raw<float> {
    __device__ __forceinline__ void load(const void* from, const float*, int64_t, int64_t i) { Raw<float>::load(static_cast<const float*>(from) + i); }
};
template <>
struct RawState<true> {
    uint2 w;
    float scale;
    __device__ __forceinline__ void load(const void* from, const float* scales, int64_t block, int64_t i) {
        w = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(from) + i);
        scale = scales[block];
    }
    __device__ __forceinline__ void unpack(float (&x)[8]) const { unpack_codes(w, scale, x); }
};

// Warp w of W takes blocks w, w + W, .. of all tensors' blocks in a row: the GPU's warps pass through a tensor side by side, which
// DRAM likes best (with a run of blocks for each warp it gave a sixth less), and what a tensor's blocks have in common is fetched
// again only when the tensor changes.
template <class P, class G, bool kMaster, bool kEight>
__global__ void __launch_bounds__(kThreads) step_kernel(StepArgs a) {
    using W = std::conditional_t<kMaster, float, P>;      // what the step works on
    const int lane = threadIdx.x & 31;
    const int warps = gridDim.x * (kThreads / 32);
    int at = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    auto tensor_of = [&](int b) { return (unsigned)b < (unsigned)a.n_blocks ? a.tensor_of[b] : -1; };   // n_blocks + 2 warps < 2^32
    int current = -1, tensor = tensor_of(at), next = tensor_of(at + warps);
    TensorRef t = {};
    const G* grad = nullptr;
    W* weights = nullptr;
    Numbers c = {};
    bool on = false, wide = false, fetched = false;
    Raw<G> rg;
    Raw<W> rw;
    RawState<kEight> ra, rs;
    float p[8], g[8], m[8], v[8];
    for (; tensor >= 0; at += warps) {
        const int after = tensor_of(at + 2 * warps);
        if (tensor != current) {
            current = tensor;
            t = a.tensors[tensor];
            on = !a.active || a.active[t.group] > 0;
            grad = static_cast<const G*>(a.grads[tensor]);
            weights = kMaster ? reinterpret_cast<W*>(t.master) : static_cast<W*>(t.param);
            const Group& group = a.groups[t.group];
            c = {group.b1, group.a1, group.b2, group.a2, group.correct, group.eps, group.keep, group.size, group.grad_scale};
            uintptr_t low = (uintptr_t)t.param | (uintptr_t)grad | (uintptr_t)weights;
            if (!kEight) low |= (uintptr_t)t.avg | (uintptr_t)t.sq;
            wide = (low & 15) == 0 && (!kEight || (((uintptr_t)t.avg | (uintptr_t)t.sq) & 7) == 0);
        }
        const bool more = next == current;
        tensor = next;
        next = after;
        if (!on) continue;
        const int64_t block = at - t.first, i = block * kBlock + lane * 8;
        const bool full = wide && (block + 1) * kBlock <= t.n;
        if (full) {
            auto load = [&](int64_t b) {
                const int64_t i = b * kBlock + lane * 8;
                rg.load(grad + i);
                rw.load(weights + i);
                ra.load(t.avg, t.avg_scale, b, i);
                rs.load(t.sq, t.sq_scale, b, i);
            };
            if (!fetched) load(block);
            rg.unpack(g);
            rw.unpack(p);
            ra.unpack(m);
            rs.unpack(v);
            fetched = kAhead && more && (block + warps + 1) * kBlock <= t.n;
            if (fetched) load(block + warps);             // on its way while this one is computed
            if (kEight)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] *= v[j];
        } else {                                          // a tensor's last block, or tensors that are not aligned
            const bool whole = wide && i + 8 <= t.n;
            load8(grad, i, t.n, whole, g);
            load8(weights, i, t.n, whole, p);
            if (kEight) {
                load8_codes(static_cast<const uint8_t*>(t.avg), i, t.n, t.avg_scale[block], m);
                load8_codes(static_cast<const uint8_t*>(t.sq), i, t.n, t.sq_scale[block], v);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] *= v[j];
            } else {
                load8(static_cast<const float*>(t.avg), i, t.n, whole, m);
                load8(static_cast<const float*>(t.sq), i, t.n, whole, v);
            }
        }
        const bool whole = full || (wide && i + 8 <= t.n);
        step8<kEight>(c, p, g, m, v);
        if (kMaster) store8(t.master, i, t.n, whole, p);
        store8(static_cast<P*>(t.param), i, t.n, whole, p);
        if (kEight) {
            store8_codes(static_cast<uint8_t*>(t.avg), i, t.n, whole, to_codes<false>(t.avg_scale + block, lane, m));
            store8_codes(static_cast<uint8_t*>(t.sq), i, t.n, whole, to_codes<true>(t.sq_scale + block, lane, v));
        } else {
            store8(static_cast<float*>(t.avg), i, t.n, whole, m);
            store8(static_cast<float*>(t.sq), i, t.n, whole, v);
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
            advance(g);
            a.groups[k] = g;
        }
    if (threadIdx.x == 0) *a.ticket = 0;
}

__global__ void set_group_kernel(Group* groups, int32_t k, Group g, bool keep_step) {
    if (keep_step) set_step(g, groups[k].step);
    groups[k] = g;
}

__global__ void fill_blocks_kernel(const TensorRef* tensors, int32_t* tensor_of) {
    const TensorRef t = tensors[blockIdx.x];
    const int n = (int)((t.n + kBlock - 1) / kBlock);
    for (int i = threadIdx.x; i < n; i += blockDim.x) tensor_of[t.first + i] = blockIdx.x;
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
    int32_t n_blocks = 0;
    bool owns_ws = false;
    void* ws = nullptr;
    slaq::TensorRef* tensors = nullptr;
    void** grads = nullptr;
    int32_t* tensor_of = nullptr;
    slaq::Group* groups = nullptr;
    unsigned int* ticket = nullptr;
    slaq::StepFn step = nullptr;
    int grid = 0;
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
    d.lr = g.lr, d.beta1 = g.beta1, d.beta2 = g.beta2;
    d.b1 = (float)g.beta1, d.a1 = (float)(1.0 - g.beta1), d.b2 = (float)g.beta2, d.a2 = (float)(1.0 - g.beta2);
    d.eps = (float)g.eps, d.keep = (float)(1.0 - g.lr * g.weight_decay), d.grad_scale = (float)g.grad_scale;
    set_step(d, g.step);
    return d;
}
size_t size_of(int type) { return type == SLAQ_F32 ? 4 : 2; }
int64_t blocks_of(int64_t n) { return (n + kBlock - 1) / kBlock; }
// bytes of the plan's device memory, and with `h` where its parts lie
size_t layout(slaq_adamw_handle* h, char* base, int32_t n_tensors, int64_t n_blocks, int32_t n_groups) {
    size_t at = 0;
    auto part = [&](auto*& p, size_t bytes) {
        if (h) p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(base + at);
        at += up(bytes);
    };
    slaq_adamw_handle none;
    slaq_adamw_handle& o = h ? *h : none;
    part(o.tensors, sizeof(TensorRef) * (size_t)n_tensors);
    part(o.grads, sizeof(void*) * (size_t)n_tensors);
    part(o.tensor_of, sizeof(int32_t) * (size_t)n_blocks);
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
    std::vector<const void*> grads((size_t)n_tensors);
    h->numel.resize((size_t)n_tensors);
    int64_t blocks = 0;
    for (int32_t t = 0; t < n_tensors; ++t) {
        const slaq_adamw_tensor& x = tensors[t];
        if (x.n < 0 || x.group < 0 || x.group >= n_groups) return SLAQ_E_ARG;
        if (x.n > kMostElements) return SLAQ_E_RANGE;
        refs[t] = {x.param, x.master, x.exp_avg, x.exp_avg_sq, x.exp_avg_scale, x.exp_avg_sq_scale, x.n, x.group, (int32_t)blocks};
        grads[t] = x.grad;
        h->numel[t] = x.n;
        blocks += blocks_of(x.n);
        if (blocks > kMostElements / kBlock) return SLAQ_E_RANGE;
        if (!x.n) continue;
        if (!x.param || !x.exp_avg || !x.exp_avg_sq || (eight && (!x.exp_avg_scale || !x.exp_avg_sq_scale))) return SLAQ_E_ARG;
        masters |= x.master != nullptr;
        auto writes = [&](const void* p, size_t size, int64_t n) {
            if (!p) return true;
            h->written.emplace_back((uintptr_t)p, (uintptr_t)p + size * (size_t)n);
            return (uintptr_t)p % size == 0;
        };
        const int64_t scales = blocks_of(x.n);
        bool ok = writes(x.param, size_of(param_type), x.n) && writes(x.master, 4, x.n) && writes(x.exp_avg, eight ? 1 : 4, x.n) &&
                  writes(x.exp_avg_sq, eight ? 1 : 4, x.n);
        if (eight) ok = ok && writes(x.exp_avg_scale, 4, scales) && writes(x.exp_avg_sq_scale, 4, scales);
        if (!ok) return SLAQ_E_ARG;
    }
    for (int32_t t = 0; t < n_tensors; ++t)
        if (masters && tensors[t].n && !tensors[t].master) return SLAQ_E_ARG;   // all tensors of a plan have a master copy, or none has
    std::sort(h->written.begin(), h->written.end());
    for (size_t k = 1; k < h->written.size(); ++k)
        if (h->written[k].first < h->written[k - 1].second) return SLAQ_E_ARG;   // a tensor listed twice, or overlapping ones
    h->n_tensors = n_tensors;
    h->n_groups = n_groups;
    h->n_blocks = (int32_t)blocks;
    h->grad_size = size_of(grad_type);
    if (const int rc = check_grads(h, grads.data())) return rc;
    if (param_type == SLAQ_F32) h->step = pick<float, float>(masters, eight);
    else if (param_type == SLAQ_BF16) h->step = grad_type == SLAQ_F32 ? pick<__nv_bfloat16, float>(masters, eight) : pick<__nv_bfloat16, __nv_bfloat16>(masters, eight);
    else h->step = grad_type == SLAQ_F32 ? pick<__half, float>(masters, eight) : pick<__half, __half>(masters, eight);
    if (cudaGetDevice(&h->device) != cudaSuccess) return SLAQ_E_CUDA;
    const size_t need = layout(nullptr, nullptr, n_tensors, blocks, n_groups);
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
    layout(h, static_cast<char*>(h->ws), n_tensors, blocks, n_groups);
    std::vector<Group> gs((size_t)n_groups);
    for (int32_t k = 0; k < n_groups; ++k) gs[k] = device_group(groups[k]);
    auto to_device = [&](void* to, const void* from, size_t n) { return n == 0 || cudaMemcpyAsync(to, from, n, cudaMemcpyHostToDevice, st) == cudaSuccess; };
    int sm = 0, per_sm = 0;
    if (!to_device(h->tensors, refs.data(), sizeof(TensorRef) * refs.size()) || !to_device(h->grads, grads.data(), sizeof(void*) * grads.size()) ||
        !to_device(h->groups, gs.data(), sizeof(Group) * gs.size()) ||
        cudaMemsetAsync(h->ticket, 0, sizeof(unsigned int), st) != cudaSuccess ||
        cudaDeviceGetAttribute(&sm, cudaDevAttrMultiProcessorCount, h->device) != cudaSuccess ||
        cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, h->step, kThreads, 0) != cudaSuccess)
        return SLAQ_E_CUDA;
    if (n_tensors) fill_blocks_kernel<<<n_tensors, 256, 0, st>>>(h->tensors, h->tensor_of);
    if (cudaGetLastError() != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess) return SLAQ_E_CUDA;   // the lists above end here
    const int64_t wanted = (blocks + kThreads / 32 - 1) / (kThreads / 32);
    h->grid = (int)std::max<int64_t>(1, std::min<int64_t>(wanted, (int64_t)sm * std::max(per_sm, 1)));
    return SLAQ_OK;
}

}  // namespace
}  // namespace slaq

extern "C" {

size_t slaq_adamw_workspace_bytes(int32_t n_tensors, const int64_t* numels, int32_t n_groups) {
    if (n_tensors < 0 || n_groups < 1 || (n_tensors && !numels)) return 0;
    int64_t blocks = 0;
    for (int32_t t = 0; t < n_tensors; ++t) {
        if (numels[t] < 0 || numels[t] > slaq::kMostElements) return 0;
        blocks += slaq::blocks_of(numels[t]);
    }
    return blocks > slaq::kMostElements / slaq::kBlock ? 0 : slaq::layout(nullptr, nullptr, n_tensors, blocks, n_groups);
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
    slaq::StepArgs a = {h->tensors, h->grads, h->tensor_of, h->n_blocks, h->n_groups, h->groups, d_active, h->ticket};
    h->step<<<h->grid, slaq::kThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(a);
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
