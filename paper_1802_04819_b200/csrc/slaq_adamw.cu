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
    int32_t group, first;            // the number of its first unit among all tensors' units
};

// A group's numbers for its next step; the block that finishes a step last moves them on.
struct Group {
    double power1, power2;           // beta to the number of the next step
    double beta1, beta2;
    int64_t step;                    // steps taken
    float b1, a1, b2, a2, eps, keep, lr, grad_scale;
};

__host__ __device__ inline void set_step(Group& g, int64_t step) {
    g.step = step;
    g.power1 = pow(g.beta1, (double)(step + 1));
    g.power2 = pow(g.beta2, (double)(step + 1));
}
// One product a step: a million steps put 1e-10 of their relative error into a power, which is 0 long before that.
__device__ inline void advance(Group& g) {
    ++g.step;
    g.power1 *= g.beta1;
    g.power2 *= g.beta2;
}

struct StepArgs {
    const TensorRef* tensors;
    const void* const* grads;
    const int32_t* tensor_of;        // per unit
    int32_t n_units, n_groups, unit; // blocks of a unit, a power of two
    Group* groups;
    const int32_t* active;
    unsigned int* ticket;
};

// Eight elements of a lane, two by two: the arithmetic is on pairs, which take one instruction together.
struct Eight {
    Pair at[4];
    __device__ __forceinline__ void get(int k, float& a, float& b) const { split(at[k], a, b); }
    __device__ __forceinline__ void set(int k, float a, float b) { at[k] = pair_of(a, b); }
};
// .. as they lie in memory
template <class E>
struct Raw {
    uint4 w[sizeof(E) / 2];
    __device__ __forceinline__ void load(const void* from) {
#pragma unroll
        for (int k = 0; k < (int)sizeof(E) / 2; ++k) w[k] = static_cast<const uint4*>(from)[k];
    }
    __device__ __forceinline__ void store(void* to) const {
#pragma unroll
        for (int k = 0; k < (int)sizeof(E) / 2; ++k) static_cast<uint4*>(to)[k] = w[k];
    }
    __device__ __forceinline__ Eight unpack() const {
        Eight x;
#pragma unroll
        for (int k = 0; k < 4; ++k) x.at[k] = Vector<E>{w[2 * k * sizeof(E) / 16]}.at(2 * k % Vector<E>::N / 2);
        return x;
    }
    __device__ __forceinline__ void pack(const Eight& x) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            Vector<E> v{w[2 * k * sizeof(E) / 16]};
            v.put(2 * k % Vector<E>::N / 2, x.at[k]);
            w[2 * k * sizeof(E) / 16] = v.w;
        }
    }
};
template <class E>
__device__ __forceinline__ void store_whole8(E* to, const Eight& x) {
    Raw<E> r = {};
    r.pack(x);
    r.store(to);
}
// .. element by element, as many as `n` of them there are
template <class E>
__device__ __forceinline__ Eight load_some(const E* from, int64_t n) {
    Eight x;
#pragma unroll
    for (int k = 0; k < 8; k += 2) x.set(k / 2, k < n ? as_float(from[k]) : 0.0f, k + 1 < n ? as_float(from[k + 1]) : 0.0f);
    return x;
}
template <class E>
__device__ __forceinline__ void store_some(E* to, int64_t n, const Eight& x) {
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
        float a, b;
        x.get(k / 2, a, b);
        if (k < n) to[k] = from_float<E>(a);
        if (k + 1 < n) to[k + 1] = from_float<E>(b);
    }
}

// 8 codes
__device__ __forceinline__ Eight unpack_codes(uint2 b) {
    Eight x;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t w = k < 2 ? b.x : b.y;
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(k & 1 ? w >> 16 : w), __NV_E4M3);
        const float2 f = __half22float2(__half2(h));
        x.set(k, f.x, f.y);
    }
    return x;
}
__device__ __forceinline__ uint2 load_some_codes(const uint8_t* from, int64_t n) {
    uint32_t b[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < n) b[k / 4] |= (uint32_t)from[k] << (k % 4 * 8);
    return make_uint2(b[0], b[1]);
}
__device__ __forceinline__ void store_some_codes(uint8_t* to, int64_t n, uint2 b) {
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < n) to[k] = (uint8_t)((k < 4 ? b.x : b.y) >> (k % 4 * 8));
}

__device__ __forceinline__ float max_size(float a, float b) {   // max of |a| and |b|, sign aside; NaN as soon as one is
    float y;
    asm("max.NaN.xorsign.abs.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
// The largest |x| of the warp, as bits: a NaN stands above all.
template <bool kPositive>
__device__ __forceinline__ float largest(const Eight& x) {
    float a, b;
    x.get(0, a, b);
    float most = kPositive ? max_nan(a, b) : max_size(a, b);
#pragma unroll
    for (int k = 1; k < 4; ++k) {
        x.get(k, a, b);
        most = kPositive ? max_nan(most, max_nan(a, b)) : max_size(most, max_size(a, b));
    }
    return __uint_as_float(__reduce_max_sync(~0u, __float_as_uint(fabsf(most))));
}
__device__ __forceinline__ float largest_finite(const Eight& x) {
    float most = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float a, b;
        x.get(k, a, b);
        if (fabsf(a) < CUDART_INF_F) most = fmaxf(most, fabsf(a));
        if (fabsf(b) < CUDART_INF_F) most = fmaxf(most, fabsf(b));
    }
    return __uint_as_float(__reduce_max_sync(~0u, __float_as_uint(most)));
}
template <bool kPositive>
__device__ __forceinline__ uint2 codes_of(const Eight& x, float inverse, bool finite) {
    Eight y;
#pragma unroll
    for (int k = 0; k < 4; ++k) y.at[k] = x.at[k] * pair_of(inverse, inverse);
    if (kPositive) {
        constexpr float kLeast = 0.001953125f;   // 2^-9, the smallest code
        float least = kLeast;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float a, b;
            y.get(k, a, b);
            least = fminf(least, fminf(a, b));
        }
        if (least < kLeast && inverse > 0.0f)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float a, b, p, q;
                x.get(k, a, b);
                y.get(k, p, q);
                y.set(k, a > 0.0f ? fmaxf(p, kLeast) : p, b > 0.0f ? fmaxf(q, kLeast) : q);
            }
    }
    uint32_t b[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float p, q;
        y.get(k, p, q);
        uint16_t two;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(two) : "f"(q), "f"(p));
        b[k] = two;
        if (!finite) {
            x.get(k, p, q);
            if (!(fabsf(p) < CUDART_INF_F)) b[k] = (b[k] & 0xFF00u) | 0x7F;
            if (!(fabsf(q) < CUDART_INF_F)) b[k] = (b[k] & 0xFFu) | 0x7F00;
        }
    }
    return make_uint2(__byte_perm(b[0], b[1], 0x5410), __byte_perm(b[2], b[3], 0x5410));
}
// Both states of the warp's 256 elements as codes, and their scales, largest x (1 / 448); a value becomes a code by (1 / largest) x 448.
// What is not finite stays so in its own element (NaN).
struct Codes {
    uint2 m, r;
    float m_scale, r_scale;
};
__device__ __forceinline__ Codes encode(const Eight& m, const Eight& r, int lane) {
    float most_m = largest<false>(m), most_r = largest<true>(r);
    const bool finite = most_m < CUDART_INF_F && most_r < CUDART_INF_F;
    if (!finite) most_m = largest_finite(m), most_r = largest_finite(r);
    // even lanes invert for m, odd ones for r; nothing is kept of what is too small
    const float most = lane & 1 ? most_r : most_m;
    const float inverse = most >= kTiny ? __frcp_rn(most) * kE4m3Max : 0.0f;
    constexpr float kPer = 1.0f / kE4m3Max;
    return {codes_of<false>(m, __shfl_sync(~0u, inverse, 0), finite), codes_of<true>(r, __shfl_sync(~0u, inverse, 1), finite),
            most_m >= kTiny ? most_m * kPer : 0.0f, most_r >= kTiny ? most_r * kPer : 0.0f};
}

// sqrt and 1/x to 1 ulp or two, denormal arguments of the root included.  A weight's step is then off by a few ulp of
// the step, which is far smaller than the weight: against 64 bits new weights are as exact as with correctly rounded operations (3.6e-8 and
// 4.2e-8 of their size).  With 32-bit states a root to the nearest takes 917 us where this one takes 886 (209 M bf16 weights with masters; without masters 772
// and 674), a division instead of the product with 1/x 1,043 (808).  With 8-bit states the division takes 720 us instead of 601.
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

// a + b of products that keep their own rounding: mul.rn.f32x2 and add.rn.f32x2 are merged, add.rn.f32 is not.
__device__ __forceinline__ Pair sum_of_products(Pair a, Pair b) {
    float p, q, r, t;
    split(a, p, q);
    split(b, r, t);
    return pair_of(__fadd_rn(p, r), __fadd_rn(q, t));
}

// What a step needs of a group.  1 - beta^t is a difference of 64-bit numbers (1e-3 at the first step for beta2 = 0.999), rounded to 32
// before the root and the division: up to 1.5 ulp of a step in all.  Both in 64 bits cost a step over 320 small tensors, in which every warp has
// one tensor, 9.5 us instead of 8.5, and 10 where the step's last block does it for the next.
struct Numbers {
    float b1, a1, b2, a2, correct, eps, keep, size, grad_scale;
};
__device__ __forceinline__ Numbers numbers_of(const Group& g) {
    return {g.b1, g.a1, g.b2, g.a2, __frsqrt_rn((float)(1.0 - g.power2)), g.eps, g.keep, __fdiv_rn(g.lr, (float)(1.0 - g.power1)), g.grad_scale};
}
// The step of 8 elements: new weights, first moments, and second moments.  With kCodes the states come as codes, whose units
// are m_scale and r_scale, and the roots of the second moments are returned.
//
// With codes, m, v and the root are rounded after every operation: a code is a decision, and the formula's own, taken operation by
// operation, is what a checkpoint or another implementation can be held to.  With fused products and a root good to 1 ulp, 51 of 16 M
// codes of m, 6 of v and the last bit of every fourth scale differed after two steps, and one code of v is 6 % of a weight's next step.
// It costs 8 %.
template <bool kCodes>
__device__ __forceinline__ void step8(const Numbers& c, float m_scale, float r_scale, Eight& p, const Eight& g, Eight& m, Eight& v) {
    auto two = [](float x) { return pair_of(x, x); };
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const Pair x = g.at[k] * two(c.grad_scale);
        if (kCodes) {
            const Pair old = v.at[k] * two(r_scale);
            m.at[k] = sum_of_products(two(c.b1) * (m.at[k] * two(m_scale)), two(c.a1) * x);
            v.at[k] = sum_of_products(two(c.b2) * (old * old), two(c.a2) * (x * x));
        } else {
            m.at[k] = fma2(two(c.b1), m.at[k], two(c.a1) * x);
            v.at[k] = fma2(two(c.a2) * x, x, two(c.b2) * v.at[k]);
        }
        float a, b;
        v.get(k, a, b);
        const Pair r = kCodes ? pair_of(__fsqrt_rn(a), __fsqrt_rn(b)) : pair_of(root(a), root(b));
        split(fma2(r, two(c.correct), two(c.eps)), a, b);
        p.at[k] = fma2(two(-c.size), m.at[k] * pair_of(reciprocal(a), reciprocal(b)), p.at[k] * two(c.keep));
        if (kCodes) v.at[k] = r;
    }
}

// The block that finishes a step last moves the groups on.
__device__ __forceinline__ void finish_step(const StepArgs& a) {
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
            advance(a.groups[k]);
        }
    if (threadIdx.x == 0) *a.ticket = 0;
}

template <bool kEight>
struct RawState : Raw<float> {
    __device__ __forceinline__ void load(const char* from, int block) { Raw<float>::load(from + (int64_t)block * (kBlock * 4)); }
};
template <>
struct RawState<true> {
    uint2 w;
    __device__ __forceinline__ void load(const char* from, int block) { w = *reinterpret_cast<const uint2*>(from + (int64_t)block * kBlock); }
};

// Warp w of W takes units w, w + W, .. of all tensors' units in a row, so that the GPU's warps pass through a tensor side by side, and
// what a tensor's blocks have in common is fetched again only when the tensor changes.  A lane's share of the next block, 48 to 128
// bytes, is asked for a block ahead, into registers.
//
// DRAM decides.  In 32 bits a unit is a block: with runs of four or eight blocks for each warp the step took a sixth longer (209 M
// bf16 weights with masters: 1040 us instead of 885, 6.60 TB/s).  And the next block is asked for behind this one's stores: asked
// for before them, while the block is computed, its loads come between the stores of other warps (967 us).  In 8 bits,
// where there is more to compute for a byte, it is the other way round (304 M fp32 weights: 783 us; behind the stores 875; 803 with the root to the nearest).
// Four thread blocks of four warps an SM are as many as the registers allow; more warps, with spills, were slower.
template <class P, class G, bool kMaster, bool kEight>
__global__ void __launch_bounds__(kThreads) step_kernel(StepArgs a) {
    using W = std::conditional_t<kMaster, float, P>;      // what the step works on
    constexpr int kState = kEight ? 1 : 4;
    const int lane = threadIdx.x & 31, unit = kEight ? a.unit : 1;
    const int warps = gridDim.x * (kThreads / 32);
    int at = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    auto tensor_of = [&](int u) { return (unsigned)u < (unsigned)a.n_units ? a.tensor_of[u] : -1; };   // n_units + 2 warps < 2^31
    int current = -1, tensor = tensor_of(at), next = tensor_of(at + warps);
    // of the current tensor; the addresses are those of the lane's 8 elements of block 0
    int first = 0, whole_blocks = 0, all_blocks = 0;
    int64_t n = 0;
    char *param = nullptr, *master = nullptr, *avg = nullptr, *sq = nullptr;
    const char* grad = nullptr;
    float *avg_scale = nullptr, *sq_scale = nullptr;
    Numbers c = {};
    bool on = false, fetched = false, have_scales = false;
    float scale_m = 0.0f, scale_r = 0.0f;                 // lane j: of the unit's j-th block
    Raw<G> rg;
    Raw<W> rw;
    RawState<kEight> ra, rs;
    auto load = [&](int b) {
        rg.load(grad + (int64_t)b * (kBlock * (int)sizeof(G)));
        rw.load((kMaster ? master : param) + (int64_t)b * (kBlock * (int)sizeof(W)));
        ra.load(avg, b);
        rs.load(sq, b);
    };
    for (; tensor >= 0; at += warps) {
        const int after = tensor_of(at + 2 * warps);
        if (tensor != current) {
            current = tensor;
            const TensorRef t = a.tensors[tensor];
            on = !a.active || a.active[t.group] > 0;
            first = t.first;
            n = t.n;
            const char* const g = static_cast<const char*>(a.grads[tensor]);
            uintptr_t low = (uintptr_t)t.param | (uintptr_t)g | (uintptr_t)t.master;
            if (!kEight) low |= (uintptr_t)t.avg | (uintptr_t)t.sq;
            const bool wide = (low & 15) == 0 && (!kEight || (((uintptr_t)t.avg | (uintptr_t)t.sq) & 7) == 0);
            whole_blocks = wide ? (int)(n / kBlock) : 0;
            all_blocks = (int)((n + kBlock - 1) / kBlock);
            grad = g + lane * 8 * sizeof(G);
            param = static_cast<char*>(t.param) + lane * 8 * sizeof(P);
            master = reinterpret_cast<char*>(t.master) + lane * 8 * 4;
            avg = static_cast<char*>(t.avg) + lane * 8 * kState;
            sq = static_cast<char*>(t.sq) + lane * 8 * kState;
            avg_scale = t.avg_scale + lane;
            sq_scale = t.sq_scale + lane;
            c = numbers_of(a.groups[t.group]);
        }
        const bool more = next == current;
        tensor = next;
        next = after;
        if (!on) continue;
        const int begin = (at - first) * unit, end = min(begin + unit, all_blocks), following = begin + warps * unit;
        float old_m = scale_m, old_r = scale_r, new_m = 0.0f, new_r = 0.0f;
        if constexpr (kEight) {
            if (!have_scales && begin + lane < end) old_m = avg_scale[begin], old_r = sq_scale[begin];
            have_scales = more;
            if (more && lane < unit && following + lane < all_blocks) scale_m = avg_scale[following], scale_r = sq_scale[following];
        }
        for (int block = begin; block < end; ++block) {
            P* const to = reinterpret_cast<P*>(param + (int64_t)block * (kBlock * (int)sizeof(P)));
            float* const to_master = reinterpret_cast<float*>(master + (int64_t)block * (kBlock * 4));
            char* const to_avg = avg + (int64_t)block * (kBlock * kState);
            char* const to_sq = sq + (int64_t)block * (kBlock * kState);
            Eight p, g, m, v;
            float by_m = 1.0f, by_r = 1.0f;
            if constexpr (kEight) by_m = __shfl_sync(~0u, old_m, block - begin), by_r = __shfl_sync(~0u, old_r, block - begin);
            auto from_codes = [&](uint2 codes_m, uint2 codes_r) { m = unpack_codes(codes_m), v = unpack_codes(codes_r); };
            Codes codes = {};
            if (block < whole_blocks) {
                if (!fetched) load(block);
                g = rg.unpack();
                p = rw.unpack();
                if constexpr (kEight) {
                    from_codes(ra.w, rs.w);
                } else {
                    m = ra.unpack();
                    v = rs.unpack();
                }
                const int ahead = block + 1 < end ? block + 1 : more ? following : whole_blocks;
                fetched = ahead < whole_blocks;
                if (kEight && fetched) load(ahead);
                step8<kEight>(c, by_m, by_r, p, g, m, v);
                if (kMaster) store_whole8(to_master, p);
                store_whole8(to, p);
                if constexpr (kEight) {
                    codes = encode(m, v, lane);
                    *reinterpret_cast<uint2*>(to_avg) = codes.m;
                    *reinterpret_cast<uint2*>(to_sq) = codes.r;
                } else {
                    store_whole8(reinterpret_cast<float*>(to_avg), m);
                    store_whole8(reinterpret_cast<float*>(to_sq), v);
                    if (fetched) load(ahead);
                }
            } else {                                      // a tensor's last block, or tensors that are not aligned
                const int64_t left = n - ((int64_t)block * kBlock + lane * 8);
                g = load_some(reinterpret_cast<const G*>(grad + (int64_t)block * (kBlock * (int)sizeof(G))), left);
                p = kMaster ? load_some(to_master, left) : load_some(to, left);
                if constexpr (kEight) {
                    from_codes(load_some_codes(reinterpret_cast<const uint8_t*>(to_avg), left), load_some_codes(reinterpret_cast<const uint8_t*>(to_sq), left));
                } else {
                    m = load_some(reinterpret_cast<const float*>(to_avg), left);
                    v = load_some(reinterpret_cast<const float*>(to_sq), left);
                }
                step8<kEight>(c, by_m, by_r, p, g, m, v);
                if (kMaster) store_some(to_master, left, p);
                store_some(to, left, p);
                if constexpr (kEight) {
                    codes = encode(m, v, lane);
                    store_some_codes(reinterpret_cast<uint8_t*>(to_avg), left, codes.m);
                    store_some_codes(reinterpret_cast<uint8_t*>(to_sq), left, codes.r);
                } else {
                    store_some(reinterpret_cast<float*>(to_avg), left, m);
                    store_some(reinterpret_cast<float*>(to_sq), left, v);
                }
            }
            if (kEight && lane == block - begin) new_m = codes.m_scale, new_r = codes.r_scale;
        }
        if (kEight && begin + lane < end) avg_scale[begin] = new_m, sq_scale[begin] = new_r;
    }
    finish_step(a);
}

template <int kBytes>
__device__ __forceinline__ void copy(void* to, const char* from) {
    const uint32_t at = (uint32_t)__cvta_generic_to_shared(to);
    if constexpr (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(at), "l"(from), "n"(kBytes) : "memory");
}
// Blocks of a tensor on their way to a warp, each lane having its own 8 elements: the next three, in shared memory.  A lane waits
// for its own copies only.
template <class W, class G>
struct Ahead {
    static constexpr int kDepth = 3, kSlots = kDepth + 1;     // the slot of the block before is free: its values have been used
    struct Slot {
        uint4 g[sizeof(G) / 2][32], w[sizeof(W) / 2][32];
        uint2 m[32], r[32];
    };
    struct Shared {
        Slot slot[kSlots];
    };
    Shared* const shared;
    const int lane;
    __device__ __forceinline__ Ahead(Shared* s) : shared(s), lane(threadIdx.x & 31) {}
    __device__ __forceinline__ void fetch(int n, bool there, const char* grad, const char* weights, const char* avg, const char* sq, int block) {
        if (there) {
            Slot& s = shared->slot[n % kSlots];
#pragma unroll
            for (int k = 0; k < (int)sizeof(G) / 2; ++k) copy<16>(&s.g[k][lane], grad + (int64_t)block * (kBlock * (int)sizeof(G)) + 16 * k);
#pragma unroll
            for (int k = 0; k < (int)sizeof(W) / 2; ++k) copy<16>(&s.w[k][lane], weights + (int64_t)block * (kBlock * (int)sizeof(W)) + 16 * k);
            copy<8>(&s.m[lane], avg + (int64_t)block * kBlock);
            copy<8>(&s.r[lane], sq + (int64_t)block * kBlock);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    // with the block's codes as they are: their scales are not in these numbers
    __device__ __forceinline__ void take(int n, Eight& grad, Eight& weights, Eight& avg, Eight& root) const {
        asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory");
        const Slot& s = shared->slot[n % kSlots];
        Raw<G> rg;
        Raw<W> rw;
#pragma unroll
        for (int k = 0; k < (int)sizeof(G) / 2; ++k) rg.w[k] = s.g[k][lane];
#pragma unroll
        for (int k = 0; k < (int)sizeof(W) / 2; ++k) rw.w[k] = s.w[k][lane];
        grad = rg.unpack(), weights = rw.unpack(), avg = unpack_codes(s.m[lane]), root = unpack_codes(s.r[lane]);
    }
};

// The same with 8-bit states where weights and gradients are of 16 bits and there is no master copy: a block is then 48 bytes a lane, and one ahead leaves 25 KB
// on their way to an SM where 40 are wanted.  Three ahead, and 32 blocks in a row, whose scales fill a line of each state:
// 599 us for 304 M elements (5.1 TB/s); with fused products and a root good to 1 ulp 528, then against 604 with one ahead.  It has 28 % of the
// warps resident and uses 69 % of the issue slots, but more warps do not help: registers for six, seven or eight blocks on an SM instead of
// five (78, 72, 64 instead of 96): 641, 672 and 745 us; two blocks ahead 608.  With more bytes a block three ahead lose (fp32: 1110 us against 790).
template <class P>
__global__ void __launch_bounds__(kThreads) deep_step_kernel(StepArgs a) {
    using Blocks = Ahead<P, P>;
    __shared__ typename Blocks::Shared shared[kThreads / 32];
    const int lane = threadIdx.x & 31, unit = a.unit;
    const int warps = gridDim.x * (kThreads / 32);
    for (int at = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); at < a.n_units;) {   // n_units + warps < 2^31
        const int tensor = a.tensor_of[at];
        const TensorRef t = a.tensors[tensor];
        const char* grad = static_cast<const char*>(a.grads[tensor]);
        const int all = (int)((t.n + kBlock - 1) / kBlock), unit0 = at - t.first;
        at += (((all + unit - 1) / unit - unit0 + warps - 1) / warps) * warps;            // behind all of the warp's units in this tensor
        if (a.active && a.active[t.group] <= 0) continue;
        const uintptr_t low = (uintptr_t)t.param | (uintptr_t)grad;
        const bool wide = (low & 15) == 0 && (((uintptr_t)t.avg | (uintptr_t)t.sq) & 7) == 0;
        const int whole = wide ? (int)(t.n / kBlock) : 0;
        // the addresses of the lane's 8 elements of block 0
        grad += lane * 8 * sizeof(P);
        char* const param = static_cast<char*>(t.param) + lane * 8 * sizeof(P);
        char* const avg = static_cast<char*>(t.avg) + lane * 8;
        char* const sq = static_cast<char*>(t.sq) + lane * 8;
        const Numbers c = numbers_of(a.groups[t.group]);
        Blocks blocks(shared + (threadIdx.x >> 5));
        auto after = [&](int b) { return ((b + 1) & (unit - 1)) && b + 1 < all ? b + 1 : (b & -unit) + warps * unit; };
        int ahead = unit0 * unit;
        for (int k = 0; k < Blocks::kDepth; ++k, ahead = after(ahead)) blocks.fetch(k, ahead < whole, grad, param, avg, sq, ahead);
        float scale_m = 0.0f, scale_r = 0.0f, old_m = 0.0f, old_r = 0.0f, new_m = 0.0f, new_r = 0.0f;   // lane j: of the unit's j-th block
        if (lane < unit && unit0 * unit + lane < all) scale_m = t.avg_scale[unit0 * unit + lane], scale_r = t.sq_scale[unit0 * unit + lane];
        int n = 0;
        for (int block = unit0 * unit; block < all; block = after(block), ++n) {
            const int place = block & (unit - 1);
            if (place == 0) {
                old_m = scale_m, old_r = scale_r;
                const int following = block + warps * unit + lane;
                if (lane < unit && following < all) scale_m = t.avg_scale[following], scale_r = t.sq_scale[following];
            }
            P* const to = reinterpret_cast<P*>(param + (int64_t)block * (kBlock * (int)sizeof(P)));
            char* const to_avg = avg + (int64_t)block * kBlock;
            char* const to_sq = sq + (int64_t)block * kBlock;
            const int64_t left = t.n - ((int64_t)block * kBlock + lane * 8);
            const float by_m = __shfl_sync(~0u, old_m, place), by_r = __shfl_sync(~0u, old_r, place);
            Eight p, g, m, v;
            Codes codes = {};
            auto step = [&] {
                step8<true>(c, by_m, by_r, p, g, m, v);
                codes = encode(m, v, lane);
            };
            if (block < whole) {
                blocks.take(n, g, p, m, v);
                blocks.fetch(n + Blocks::kDepth, ahead < whole, grad, param, avg, sq, ahead);
                step();
                store_whole8(to, p);
                *reinterpret_cast<uint2*>(to_avg) = codes.m;
                *reinterpret_cast<uint2*>(to_sq) = codes.r;
            } else {                                      // a tensor's last block, or tensors that are not aligned: nothing is ahead
                g = load_some(reinterpret_cast<const P*>(grad + (int64_t)block * (kBlock * (int)sizeof(P))), left);
                p = load_some(to, left);
                m = unpack_codes(load_some_codes(reinterpret_cast<const uint8_t*>(to_avg), left));
                v = unpack_codes(load_some_codes(reinterpret_cast<const uint8_t*>(to_sq), left));
                step();
                store_some(to, left, p);
                store_some_codes(reinterpret_cast<uint8_t*>(to_avg), left, codes.m);
                store_some_codes(reinterpret_cast<uint8_t*>(to_sq), left, codes.r);
            }
            ahead = after(ahead);
            if (lane == place) new_m = codes.m_scale, new_r = codes.r_scale;
            if ((place == unit - 1 || block == all - 1) && lane <= place) t.avg_scale[block - place + lane] = new_m, t.sq_scale[block - place + lane] = new_r;
        }
        asm volatile("cp.async.wait_all;" ::: "memory");   // nothing of this tensor's is on its way to the slots any more
    }
    finish_step(a);
}

__global__ void set_group_kernel(Group* groups, int32_t k, Group g, bool keep_step) {
    if (keep_step) set_step(g, groups[k].step);
    groups[k] = g;
}

__global__ void fill_units_kernel(const TensorRef* tensors, int unit, int32_t* tensor_of) {
    const TensorRef t = tensors[blockIdx.x];
    const int64_t blocks = (t.n + kBlock - 1) / kBlock;
    const int n = (int)((blocks + unit - 1) / unit);
    for (int i = threadIdx.x; i < n; i += blockDim.x) tensor_of[t.first + i] = blockIdx.x;
}

using StepFn = void (*)(StepArgs);
template <class P, class G>
constexpr bool deep() { return sizeof(P) == 2 && sizeof(G) == 2; }
template <class P, class G>
StepFn pick(bool master, bool eight) {
    if (master) return eight ? step_kernel<P, G, true, true> : step_kernel<P, G, true, false>;
    if (!eight) return step_kernel<P, G, false, false>;
    if constexpr (deep<P, G>()) return deep_step_kernel<P>;
    else return step_kernel<P, G, false, true>;
}

size_t up(size_t n) { return (n + 255) & ~size_t(255); }

}  // namespace
}  // namespace slaq

struct slaq_adamw_handle {
    int device = 0;
    int32_t n_tensors = 0, n_groups = 0;
    int32_t n_units = 0, unit = 1;
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
bool on_device(const slaq_adamw_handle* h) {
    int d = -1;
    return done(cudaGetDevice(&d)) && d == h->device;
}
// What the step computes with is finite in 32 bits, so that elements that are 0 stay so: the factor of the gradients, the decay, and the
// learning rate over 1 - beta1^t, which is largest at the first step.  eps is 0 or a normal number: the step's reciprocal takes what lies
// between for 0, and 0 x infinity would be the step of an element whose gradient and states are 0, which is 0 / eps = 0.
bool group_ok(const slaq_adamw_group& g) {
    constexpr double kLeastEps = 1.1754943508222875e-38, kMost = 3.4e38;   // 2^-126; 32 bits end at 3.4028e38
    auto in = [](double x, double lo, double hi) { return x >= lo && x < hi; };
    return in(g.lr, 0.0, 1e30) && in(g.beta1, 0.0, 1.0) && in(g.beta2, 0.0, 1.0) && (g.eps == 0.0 || in(g.eps, kLeastEps, 1e30)) &&
           in(g.weight_decay, 0.0, 1e30) && std::fabs(g.grad_scale) < kMost && g.lr * g.weight_decay < kMost && g.lr / (1.0 - g.beta1) < kMost &&
           g.step <= (int64_t)1 << 53;
}
Group device_group(const slaq_adamw_group& g) {
    Group d = {};
    d.lr = (float)g.lr, d.beta1 = g.beta1, d.beta2 = g.beta2;
    d.b1 = (float)g.beta1, d.a1 = (float)(1.0 - g.beta1), d.b2 = (float)g.beta2, d.a2 = (float)(1.0 - g.beta2);
    d.eps = (float)g.eps, d.keep = (float)(1.0 - g.lr * g.weight_decay), d.grad_scale = (float)g.grad_scale;
    set_step(d, g.step);
    return d;
}
size_t size_of(int type) { return type == SLAQ_F32 ? 4 : 2; }
int64_t blocks_of(int64_t n) { return (n + kBlock - 1) / kBlock; }
// bytes of the plan's device memory, and with `h` where its parts lie
size_t layout(slaq_adamw_handle* h, char* base, int32_t n_tensors, int64_t n_units, int32_t n_groups) {
    size_t at = 0;
    auto part = [&](auto*& p, size_t bytes) {
        if (h) p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(base + at);
        at += up(bytes);
    };
    slaq_adamw_handle none;
    slaq_adamw_handle& o = h ? *h : none;
    part(o.tensors, sizeof(TensorRef) * (size_t)n_tensors);
    part(o.grads, sizeof(void*) * (size_t)n_tensors);
    part(o.tensor_of, sizeof(int32_t) * (size_t)n_units);
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
    int64_t blocks = 0, units = 0;
    for (int32_t t = 0; t < n_tensors; ++t)
        if (tensors[t].n > 0 && tensors[t].n <= kMostElements) blocks += blocks_of(tensors[t].n);
    if (blocks > kMostElements / kBlock) return SLAQ_E_RANGE;
    // With 8-bit states a warp works on 8 blocks in a row (32 in the deep kernel), so that it reads and writes their scales at
    // once: where warps of several SMs wrote to one line of scales, these waited for one another (304 M elements in units of one
    // block: 774 us).  As far as there is a unit for every warp.
    bool any_master = false;
    for (int32_t t = 0; t < n_tensors; ++t) any_master |= tensors[t].n > 0 && tensors[t].master;
    int unit = !eight ? 1 : param_type != SLAQ_F32 && grad_type != SLAQ_F32 && !any_master ? 32 : 8;
    while (unit > 1 && blocks < (int64_t)unit * 148 * 16) unit /= 2;
    while (unit > 8 && blocks < (int64_t)unit * 8 * n_tensors) unit /= 2;   // short tensors end inside a unit (3,000 of 80 blocks: 120 us with 8, 134 with 32)
    for (int32_t t = 0; t < n_tensors; ++t) {
        const slaq_adamw_tensor& x = tensors[t];
        if (x.n < 0 || x.group < 0 || x.group >= n_groups) return SLAQ_E_ARG;
        if (x.n > kMostElements) return SLAQ_E_RANGE;
        refs[t] = {x.param, x.master, x.exp_avg, x.exp_avg_sq, x.exp_avg_scale, x.exp_avg_sq_scale, x.n, x.group, (int32_t)units};
        grads[t] = x.grad;
        h->numel[t] = x.n;
        units += (blocks_of(x.n) + unit - 1) / unit;
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
    h->n_units = (int32_t)units;
    h->unit = unit;
    h->grad_size = size_of(grad_type);
    if (const int rc = check_grads(h, grads.data())) return rc;
    if (param_type == SLAQ_F32) h->step = pick<float, float>(masters, eight);
    else if (param_type == SLAQ_BF16) h->step = grad_type == SLAQ_F32 ? pick<__nv_bfloat16, float>(masters, eight) : pick<__nv_bfloat16, __nv_bfloat16>(masters, eight);
    else h->step = grad_type == SLAQ_F32 ? pick<__half, float>(masters, eight) : pick<__half, __half>(masters, eight);
    if (!done(cudaGetDevice(&h->device))) return SLAQ_E_CUDA;
    if (captured(st)) return SLAQ_E_ARG;
    const size_t need = layout(nullptr, nullptr, n_tensors, blocks, n_groups);   // as many units as blocks: the size does not depend on the states
    if (dev_ws) {
        if (((uintptr_t)dev_ws & 255) || bytes < need) return SLAQ_E_NOMEM;
        h->ws = dev_ws;
    } else {
        if (!done(cudaMalloc(&h->ws, need))) return SLAQ_E_NOMEM;
        h->owns_ws = true;
    }
    layout(h, static_cast<char*>(h->ws), n_tensors, blocks, n_groups);
    std::vector<Group> gs((size_t)n_groups);
    for (int32_t k = 0; k < n_groups; ++k) gs[k] = device_group(groups[k]);
    auto to_device = [&](void* to, const void* from, size_t n) { return n == 0 || done(cudaMemcpyAsync(to, from, n, cudaMemcpyHostToDevice, st)); };
    int sm = 0, per_sm = 0;
    if (!to_device(h->tensors, refs.data(), sizeof(TensorRef) * refs.size()) || !to_device(h->grads, grads.data(), sizeof(void*) * grads.size()) ||
        !to_device(h->groups, gs.data(), sizeof(Group) * gs.size()) ||
        !done(cudaMemsetAsync(h->ticket, 0, sizeof(unsigned int), st)) || !done(cudaDeviceGetAttribute(&sm, cudaDevAttrMultiProcessorCount, h->device)) ||
        !done(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, h->step, kThreads, 0)))
        return SLAQ_E_CUDA;
    if (n_tensors && !launch(fill_units_kernel, n_tensors, 256, st, h->tensors, h->unit, h->tensor_of)) return SLAQ_E_CUDA;
    if (!done(cudaStreamSynchronize(st))) return SLAQ_E_CUDA;   // the lists above end here
    const int64_t wanted = (units + kThreads / 32 - 1) / (kThreads / 32);
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
    if (h->owns_ws && h->ws) slaq::done(cudaFree(h->ws));   // waits for the steps that still read it
    delete h;
    return SLAQ_OK;
}

const char* slaq_adamw_last_error(const slaq_adamw_t* h) { return h ? h->err : "null handle"; }

int slaq_adamw_step(slaq_adamw_t* h, const int32_t* d_active, void* cuda_stream) {
    if (!h) return SLAQ_E_ARG;
    if (!slaq::on_device(h)) return slaq::fail(h, SLAQ_E_ARG, "the plan's device is not the current one");
    if (!slaq::aligned(d_active)) return slaq::fail(h, SLAQ_E_ARG, "the list of active groups is not aligned to its type");
    slaq::StepArgs a = {h->tensors, h->grads, h->tensor_of, h->n_units, h->n_groups, h->unit, h->groups, d_active, h->ticket};
    return slaq::launch(h->step, h->grid, slaq::kThreads, static_cast<cudaStream_t>(cuda_stream), a) ? SLAQ_OK : slaq::fail(h, SLAQ_E_CUDA, "the step could not be launched");
}

int slaq_adamw_set_group(slaq_adamw_t* h, int32_t group, const slaq_adamw_group* g, void* cuda_stream) {
    if (!h) return SLAQ_E_ARG;
    if (!slaq::on_device(h)) return slaq::fail(h, SLAQ_E_ARG, "the plan's device is not the current one");
    if (!g || !slaq::group_ok(*g)) return slaq::fail(h, SLAQ_E_ARG, "a group's values are out of range");
    if (group < 0 || group >= h->n_groups) return slaq::fail(h, SLAQ_E_RANGE, "no such group");
    slaq_adamw_group v = *g;
    const bool keep = v.step < 0;
    if (keep) v.step = 0;
    const bool ok = slaq::launch(slaq::set_group_kernel, 1, 1, static_cast<cudaStream_t>(cuda_stream), h->groups, group, slaq::device_group(v), keep);
    return ok ? SLAQ_OK : slaq::fail(h, SLAQ_E_CUDA, "the group could not be set");
}

int slaq_adamw_set_grads(slaq_adamw_t* h, const void* const* grads, void* cuda_stream) {
    if (!h) return SLAQ_E_ARG;
    if (!slaq::on_device(h)) return slaq::fail(h, SLAQ_E_ARG, "the plan's device is not the current one");
    if (h->n_tensors == 0) return SLAQ_OK;
    if (!grads) return slaq::fail(h, SLAQ_E_ARG, "grads is null");
    if (const int rc = slaq::check_grads(h, grads)) return rc;
    if (slaq::captured(static_cast<cudaStream_t>(cuda_stream)))
        return slaq::fail(h, SLAQ_E_ARG, "gradients are not changed while the stream is captured");
    if (!slaq::done(cudaMemcpyAsync(h->grads, grads, sizeof(void*) * (size_t)h->n_tensors, cudaMemcpyHostToDevice, static_cast<cudaStream_t>(cuda_stream))))
        return slaq::fail(h, SLAQ_E_CUDA, "copy of the gradients' addresses");
    return SLAQ_OK;
}

int slaq_adamw_get_steps(slaq_adamw_t* h, int64_t* out_steps, void* cuda_stream) {
    if (!h) return SLAQ_E_ARG;
    if (!slaq::on_device(h)) return slaq::fail(h, SLAQ_E_ARG, "the plan's device is not the current one");
    if (!out_steps) return slaq::fail(h, SLAQ_E_ARG, "out_steps is null");
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (slaq::captured(st)) return slaq::fail(h, SLAQ_E_ARG, "the stream is being captured");
    if (!slaq::done(cudaMemcpy2DAsync(out_steps, sizeof(int64_t), &h->groups->step, sizeof(slaq::Group), sizeof(int64_t), (size_t)h->n_groups,
                                      cudaMemcpyDeviceToHost, st)) || !slaq::done(cudaStreamSynchronize(st)))
        return slaq::fail(h, SLAQ_E_CUDA, "copy of the steps");
    return SLAQ_OK;
}

}  // extern "C"
