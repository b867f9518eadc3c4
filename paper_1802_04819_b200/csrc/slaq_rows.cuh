// Rows of logits: 16-byte vectors of their elements, softmax sums in one pass, the largest elements.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>
#include <stdint.h>

#include <type_traits>

namespace slaq {

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float as_float(__half x) { return __half2float(x); }
template <class E> __device__ __forceinline__ E from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }

constexpr float kLog2E = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kGone = -200.0f;   // 2^kGone is 0 in 32 bits, and 0 x kGone is 0 where 0 x -inf is not

// 2^x to 2 ulp, 0 from -126 down.  Of a difference (x - m) scale log2(e) whose constant is rounded once: log probabilities are then within
// 1.3e-7 of 64 bits, relatively, where elementary operations in 32 bits with expf come to 0.8e-7.  expf in its place would cost more than
// anything else here does: 8,192 x 65,536 bf16 264 us instead of 168, loss and gradient of 4,096 x 128,000 528 instead of 400, the gradient
// alone of 4,096 x 128,000 403 instead of 322.
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// max that is NaN as soon as one operand is
__device__ __forceinline__ float max_nan(float a, float b) {
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
__device__ __forceinline__ float warp_max_nan(float x) {
    float y;
    asm("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
    return y;
}

// Unsigned integers in the order of the values, -0 equal to +0, NaN above everything.  No value maps to 0 or to
// 0xFFFFFFFF, so that a key of value and position can be told from "nothing" and from "nothing taken yet".
__device__ __forceinline__ uint32_t order_of(float x) {
    if (x != x) return 0xFFFFFFFEu;
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b ^ (b >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t order) { return __uint_as_float(order >> 31 ? order ^ 0x80000000u : ~order); }
// .. and with the position: of equal values the one further to the left is the larger
__device__ __forceinline__ unsigned long long key_of(float x, uint32_t i) {
    return (unsigned long long)order_of(x) << 32 | (0xFFFFFFFFu - i);
}
__device__ __forceinline__ uint32_t position_of(unsigned long long key) { return 0xFFFFFFFFu - (uint32_t)key; }

// ---- two numbers at a time ----
struct Pair {
    unsigned long long v;
};
__device__ __forceinline__ Pair pair_of(float a, float b) {
    Pair p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p.v) : "f"(a), "f"(b));
    return p;
}
__device__ __forceinline__ void split(Pair p, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p.v)); }
__device__ __forceinline__ Pair operator+(Pair a, Pair b) {
    Pair p;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(p.v) : "l"(a.v), "l"(b.v));
    return p;
}
__device__ __forceinline__ Pair operator*(Pair a, Pair b) {
    Pair p;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(p.v) : "l"(a.v), "l"(b.v));
    return p;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    Pair p;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(p.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return p;
}

// ---- 16 bytes of a row ----
template <class E>
struct Vector {
    static constexpr int N = 16 / (int)sizeof(E);
    uint4 w;

    __device__ __forceinline__ uint32_t word(int i) const { return i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w; }
    // elements 2 i and 2 i + 1
    __device__ __forceinline__ Pair at(int i) const {
        if constexpr (sizeof(E) == 4) return pair_of(__uint_as_float(word(2 * i)), __uint_as_float(word(2 * i + 1)));
        const uint32_t b = word(i);
        if constexpr (std::is_same_v<E, __nv_bfloat16>) return pair_of(__uint_as_float(b << 16), __uint_as_float(b & 0xFFFF0000u));
        if constexpr (std::is_same_v<E, __half>) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&b));
            return pair_of(f.x, f.y);
        }
    }
    __device__ __forceinline__ float max() const {
        if constexpr (sizeof(E) == 4) {
            return max_nan(max_nan(__uint_as_float(w.x), __uint_as_float(w.y)), max_nan(__uint_as_float(w.z), __uint_as_float(w.w)));
        } else {
            uint32_t m;
            if constexpr (std::is_same_v<E, __nv_bfloat16>) {
                asm("{.reg .b32 a, b;\n max.NaN.bf16x2 a, %1, %2;\n max.NaN.bf16x2 b, %3, %4;\n max.NaN.bf16x2 %0, a, b;}"
                    : "=r"(m) : "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w));
                return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
            } else {
                asm("{.reg .b32 a, b;\n max.NaN.f16x2 a, %1, %2;\n max.NaN.f16x2 b, %3, %4;\n max.NaN.f16x2 %0, a, b;}"
                    : "=r"(m) : "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w));
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&m));
                return max_nan(f.x, f.y);
            }
        }
    }
    __device__ __forceinline__ void put(int i, Pair p) {
        float a, b;
        split(p, a, b);
        uint32_t* const to = reinterpret_cast<uint32_t*>(&w);
        if constexpr (sizeof(E) == 4) {
            to[2 * i] = __float_as_uint(a), to[2 * i + 1] = __float_as_uint(b);
        } else if constexpr (std::is_same_v<E, __nv_bfloat16>) {
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(to[i]) : "f"(b), "f"(a));
        } else {
            asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(to[i]) : "f"(b), "f"(a));
        }
    }
    __device__ __forceinline__ float one(int e) const { return as_float(reinterpret_cast<const E*>(&w)[e]); }
};

// Elements off .. off + N - 1 of the 2 N elements of two vectors
template <class E>
__device__ __forceinline__ Vector<E> joined(const Vector<E>& a, const Vector<E>& b, int off) {
    uint32_t w[8] = {a.w.x, a.w.y, a.w.z, a.w.w, b.w.x, b.w.y, b.w.z, b.w.w};
    const int bytes = off * (int)sizeof(E);
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = bytes & 8 ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = bytes & 4 ? w[i + 1] : w[i];
    if constexpr (sizeof(E) == 2)
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], bytes & 2 ? 16 : 0);
    return {{w[0], w[1], w[2], w[3]}};
}
// elements by which an address lies behind a multiple of 16 bytes
template <class E>
__device__ __forceinline__ int skip_of(const E* p) { return (int)(reinterpret_cast<uintptr_t>(p) & 15) / (int)sizeof(E); }

// The 16-byte vectors that a row of V elements touches: the row begins with element `skip` of vector 0.  The vectors that lie
// inside the row, [lo, hi), are read and written whole; the others, at most one at each end, element by element, with -inf in
// the places outside.
template <class E>
struct Row {
    static constexpr int N = Vector<E>::N;
    const E* x;
    int V, skip, vectors, lo, hi;
    __device__ __forceinline__ Row(const E* row, int n) : x(row), V(n), skip(skip_of(row)) {
        vectors = (skip + n + N - 1) / N;
        lo = skip || n < N ? 1 : 0;
        hi = (skip + n) % N ? vectors - 1 : vectors;
        if (hi < lo) hi = lo;                              // one vector in all, not whole
    }
    __device__ __forceinline__ bool head() const { return lo == 1; }
    __device__ __forceinline__ bool tail() const { return hi < vectors; }
    __device__ __forceinline__ int first(int v) const { return v * N - skip; }   // the element a vector begins with
    __device__ __forceinline__ bool whole(int v) const { return v >= lo && v < hi; }
    __device__ __forceinline__ Vector<E> partial(int v) const {
        Vector<E> r;
        E* const e = reinterpret_cast<E*>(&r.w);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int i = first(v) + k;
            e[k] = i >= 0 && i < V ? x[i] : from_float<E>(-CUDART_INF_F);
        }
        return r;
    }
    static __device__ __forceinline__ Vector<E> load_at(const void* p) {
        Vector<E> r;
        asm("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.w.x), "=r"(r.w.y), "=r"(r.w.z), "=r"(r.w.w) : "l"(p));
        return r;
    }
    __device__ __forceinline__ Vector<E> load(int v) const {
        if (whole(v)) return load_at(x + first(v));
        return v >= 0 && v < vectors ? partial(v) : nothing();
    }
    static __device__ __forceinline__ Vector<E> nothing() {
        const uint32_t b = sizeof(E) == 4 ? 0xFF800000u : std::is_same_v<E, __half> ? 0xFC00FC00u : 0xFF80FF80u;
        return {{b, b, b, b}};
    }
};

// ---- softmax sums ----
// Of elements x seen so far: m = max x, s = sum 2^t, u = sum 2^t t with t = (x - m) c.  While only masked elements were seen
// m is -inf and the sums are 0.  A new maximum rescales the sums, t being shifted by the difference.
struct Sums {
    float m, s, u;
};
__device__ __forceinline__ float base_of(float m) { return m == -CUDART_INF_F ? 0.0f : m; }
// the sums with respect to `base` instead of their own maximum
__device__ __forceinline__ void rebase(Sums& a, float base, float c) {
    const float by = fmaxf((a.m - base) * c, kGone), f = exp2_fast(by);
    a.u = fmaf(a.s, by, a.u) * f;
    a.s *= f;
}
__device__ __forceinline__ Sums merged(Sums a, Sums b, float c) {
    const float m = max_nan(a.m, b.m), base = base_of(m);
    rebase(a, base, c);
    rebase(b, base, c);
    return {m, a.s + b.s, a.u + b.u};
}
__device__ __forceinline__ Sums warp_merged(Sums a, float c) {
    const float m = warp_max_nan(a.m);
    rebase(a, base_of(m), c);
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        a.s += __shfl_xor_sync(~0u, a.s, o);
        a.u += __shfl_xor_sync(~0u, a.u, o);
    }
    a.m = m;
    return a;
}

// U vectors more, whose largest element is `most`; u only if kEntropy
template <bool kEntropy, int U, class E>
__device__ __forceinline__ void add_vectors(Sums& a, const Vector<E> (&x)[U], float most, float c) {
    const float m = max_nan(a.m, most), base = base_of(m);
    rebase(a, base, c);
    a.m = m;
    const Pair off = pair_of(-base, -base), by = pair_of(c, c);
    Pair s = pair_of(0.0f, 0.0f), u = s;
#pragma unroll
    for (int k = 0; k < U; ++k)
#pragma unroll
        for (int i = 0; i < Vector<E>::N / 2; ++i) {
            float p, q;
            Pair t = (x[k].at(i) + off) * by;
            split(t, p, q);
            if (kEntropy) {
                p = fmaxf(p, kGone), q = fmaxf(q, kGone);
                t = pair_of(p, q);
            }
            const Pair e = pair_of(exp2_fast(p), exp2_fast(q));
            s = s + e;
            if (kEntropy) u = fma2(e, t, u);
        }
    float p, q;
    split(s, p, q);
    a.s += p + q;
    if (kEntropy) {
        split(u, p, q);
        a.u += p + q;
    }
}

// ---- the largest keys of a warp: lane i holds the i-th largest, 0 where there is none ----
template <class K>
__device__ __forceinline__ K larger_if(bool want, K a, K b) { return (a > b) == want ? a : b; }
template <class K>
__device__ __forceinline__ K merge_sorted(K a, K b_reversed) {
    const int lane = threadIdx.x & 31;
    a = a > b_reversed ? a : b_reversed;
#pragma unroll
    for (int o = 16; o; o >>= 1) a = larger_if(!(lane & o), a, __shfl_xor_sync(~0u, a, o));
    return a;
}
template <class K>
__device__ __forceinline__ K sorted(K a) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int n = 2; n <= 32; n *= 2)
#pragma unroll
        for (int o = n / 2; o; o >>= 1) a = larger_if(!(lane & o) == !(lane & n), a, __shfl_xor_sync(~0u, a, o));
    return a;
}
template <class K>
__device__ __forceinline__ K with_more(K best, K unsorted) {
    return merge_sorted(best, __shfl_sync(~0u, sorted(unsorted), 31 - (threadIdx.x & 31)));
}

}  // namespace slaq
