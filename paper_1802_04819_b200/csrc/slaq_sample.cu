// Tokens drawn from rows of logits with given random numbers.
//
// A row x[0..V), temperature T, uniform u.  With m = max x: w_i = exp((x_i - m) / T).  The order of a row is that of falling x, equal ones by
// rising id.  Kept is a prefix of that order: of the first k (S_k their sum) the shortest whose sum reaches p S_k, as far as w_i >= q.  With C the
// sum over what is kept, the token is the first by id at which the running sum over the kept ones exceeds u C.
//
// The result is an integer, and in a large vocabulary the sums of 32-bit weights are off by more than many a token's weight.  So sums come with a
// bound of their error; where a decision lies within it, the row is summed up again in 64 bits.
#include <cooperative_groups.h>

#include "slaq_internal.cuh"
#include "slaq_rows.cuh"

namespace cg = cooperative_groups;

namespace slaq {
namespace {

constexpr int kMaxVocab = 1 << 22;
constexpr double kMostTemperature = 1.0000001e30, kLeastTemperature = 0.9999999e-30;   // 1e30 and 1e-30, rounded to 32 bits or not
constexpr int kUnroll = 4;         // vectors that a lane has in flight

struct SampleArgs {
    const void* logits;
    int64_t rows, stride;
    int32_t vocab;
    const float* uniform;
    const float* temperatures;     // per row, or one for all
    const int32_t* top_ks;
    const float* top_ps;
    const float* min_ps;
    double temperature, top_p, min_p;
    int32_t top_k;
    int64_t* token;
    float *logprob, *kept_logprob;
    int32_t* kept;
};

// A row's numbers.
struct Asked {
    float u;
    double T, p, q;
    int k;
    int kind;                      // 0: to be drawn; 1: nobody asked; 2: numbers out of range
};
template <bool kFilter>
__device__ __forceinline__ Asked asked_of(const SampleArgs& a, int64_t row) {
    Asked r;
    r.u = a.uniform[row];
    r.T = a.temperatures ? (double)a.temperatures[row] : a.temperature;
    r.k = !kFilter ? 0 : a.top_ks ? a.top_ks[row] : a.top_k;
    r.p = !kFilter ? 1.0 : a.top_ps ? (double)a.top_ps[row] : a.top_p;
    r.q = !kFilter ? 0.0 : a.min_ps ? (double)a.min_ps[row] : a.min_p;
    const bool ok = r.u < 1.0f && (r.T == 0.0 || (r.T >= kLeastTemperature && r.T <= kMostTemperature)) && r.p >= 0.0 && r.p <= 1.0 && r.q >= 0.0 && r.q <= 1.0;
    r.kind = r.u < 0.0f ? 1 : ok ? 0 : 2;
    return r;
}
__device__ __forceinline__ void write(const SampleArgs& a, int64_t row, int64_t token, float logprob, float kept_logprob, int kept) {
    a.token[row] = token;
    if (a.logprob) a.logprob[row] = logprob;
    if (a.kept_logprob) a.kept_logprob[row] = kept_logprob;
    if (a.kept) a.kept[row] = kept;
}
// What is no draw: nobody asked, a NaN or an infinity in the row or its numbers, nothing but masked tokens.
__device__ __forceinline__ void write_none(const SampleArgs& a, int64_t row, int kind, float m) {
    const float x = kind == 1 ? 0.0f : kind == 0 && m == -CUDART_INF_F ? m : CUDART_NAN_F;
    write(a, row, -1, x, x, 0);
}
__device__ __forceinline__ bool is_finite(float x) { return fabsf(x) < CUDART_INF_F; }

// Weights in 32 bits: 2^t, t = x c - M with c = log2(e) / T rounded to 32 bits, M a whole number above m c, so that sums with another M are brought to
// this one exactly.  A weight is off by the exponential's 2^-22 and by |t| ln 2 times 2^-24, t's rounding, and c's (what c's puts on all weights alike
// cancels).  Of the sum S of V weights the mean of |t| is at most log2(V / S): the entropy of the shares is at most that of equal ones.
// Five additions in 32 bits lead to what is added up in 64.
constexpr float kMostExponent = 4194304.0f;                    // 2^22: beyond, M is not above m c by a little
struct Scale {
    double exact;                  // c before it is rounded
    float c;
    __device__ __forceinline__ explicit Scale(double T) : exact(1.4426950408889634 / T), c((float)exact) {}
    // Not below -2^22: a row whose largest element lies there is not weighed in 32 bits, and in the others what does lie there (masked by a large finite
    // number) weighs nothing, where a base of its own, a rounded one, would give it any weight.
    __device__ __forceinline__ float base(float m) const { return m == -CUDART_INF_F ? 0.0f : fmaxf(ceilf(m * c) + 1.0f, -kMostExponent); }
    __device__ __forceinline__ float exponent(float x, float M) const { return fmaf(x, c, -M); }
    __device__ __forceinline__ float weight(float x, float M) const { return exp2_fast(exponent(x, M)); }
    __device__ __forceinline__ bool holds(float m) const { return fabsf(m * c) <= kMostExponent; }
    // log2 of the largest element's weight with base M
    __device__ __forceinline__ double of_largest(float m, float M) const { return (double)m * c - M; }
};
// Bounds of a sum's error: of its weights alike, and through their exponents.
struct Error {
    double alike, exponents;
    __device__ __forceinline__ Error(int V, double S, const Scale& c)
        : alike(5.0 * 5.97e-8 + 2.4e-7), exponents(0.6932 * (5.97e-8 + fabs(c.c / c.exact - 1.0)) * fmax(log2((double)V / S), 0.0)) {}
    __device__ __forceinline__ double both() const { return alike + exponents; }
    // .. of the difference between the sum up to a token and u times the sum, near 0: (1 - u) of the errors before it and u of those behind
    __device__ __forceinline__ double at(double u) const { return alike * 2.0 * u * (1.0 - u) + exponents * fmax(u, 1.0 - u) + 1e-15; }
};

// Weights in 64 bits, of the largest 1: exp((x - m) / T) as 2^t, t = (x - m) c = k / 16 + f: a table of 2^(j / 16) and the series of 2^f
// to its seventh term, |f ln 2| <= 0.0217 (the next is 4e-16).  What is less than 2^-1000 counts as 0.  exp() takes three times as long for a row: its
// branches leave one weight at a time in work.
//
// The series' terms stand in constant memory, where an instruction finds them; as literals each takes two instructions of its own at every use (56
// instructions a weight instead of 46).
constexpr int kSteps = 16;
constexpr double kLn2Wide = 0.6931471805599453;
__constant__ double kSeries[8] = {1.0, kLn2Wide, kLn2Wide* kLn2Wide / 2.0, kLn2Wide* kLn2Wide* kLn2Wide / 6.0, kLn2Wide* kLn2Wide* kLn2Wide* kLn2Wide / 24.0,
                                        kLn2Wide* kLn2Wide* kLn2Wide* kLn2Wide* kLn2Wide / 120.0,
                                        kLn2Wide* kLn2Wide* kLn2Wide* kLn2Wide* kLn2Wide* kLn2Wide / 720.0, 422212465065984.0};   // .. and 1.5 x 2^48
__device__ __forceinline__ float not_below(double x) {
    float y;
    asm("cvt.rp.f32.f64 %0, %1;" : "=f"(y) : "d"(x));
    return y;
}
__device__ __forceinline__ float not_above(double x) {
    float y;
    asm("cvt.rm.f32.f64 %0, %1;" : "=f"(y) : "d"(x));
    return y;
}
struct Exact {
    double c, m;
    float least;                   // 0 below.  Rounded up: no exponent is below -1000, whatever a step of 32-bit numbers beside m is worth, and -inf always is 0
    const double* table;
    __device__ __forceinline__ Exact(float m, const Scale& s, const double* t)
        : c(s.exact), m(m), least(not_below((double)m - 1000.0 / s.exact)), table(t) {}
    // 0 if it is not wanted
    __device__ __forceinline__ double weight(float x, bool wanted = true) const {
        // r = (x - m) c + 1.5 x 2^48, whose last place is a 16th
        const double d = (double)x - m, r = fma(d, c, kSeries[7]), f = fma(d, c, kSeries[7] - r);
        const int k = __double2loint(r);
        double p = kSeries[6];
        p = fma(p, f, kSeries[5]);
        p = fma(p, f, kSeries[4]);
        p = fma(p, f, kSeries[3]);
        p = fma(p, f, kSeries[2]);
        p = fma(p, f, kSeries[1]);
        p = fma(p, f, kSeries[0]) * table[k & (kSteps - 1)];
        const bool on = wanted && x >= least;
        return __hiloint2double(on ? __double2hiint(p) + ((k & -kSteps) << 16) : 0, on ? __double2loint(p) : 0);
    }
};
// p S, rounded: it is not merged with the difference that is taken from it, so that a share of equal weights that comes out whole is the same in every kernel
__device__ __forceinline__ double share_of(double p, double S) {
    double x;
    asm("mul.rn.f64 %0, %1, %2;" : "=d"(x) : "d"(p), "d"(S));
    return x;
}
// 2^d for a whole number d <= 0, exactly; 0 far below
__device__ __forceinline__ double power(float d) { return d > -1000.0f ? __hiloint2double((1023 + (int)d) << 20, 0) : 0.0; }

// Kept are the elements above `value`, and those equal to it up to id `last`; nothing that is masked.
struct Cut {
    float value;
    uint32_t last;
    __device__ __forceinline__ bool keeps(float x, int i) const { return x > value || (x == value && (uint32_t)i <= last && x > -CUDART_INF_F); }
};
__device__ __forceinline__ Cut unmasked() { return {-CUDART_INF_F, 0}; }
__device__ __forceinline__ Cut tighter(const Cut& a, const Cut& b) { return a.value > b.value || (a.value == b.value && a.last < b.last) ? a : b; }

template <class T>
__device__ __forceinline__ T warp_sum(T x) {
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(~0u, x, o);
    return x;
}
template <class T>
__device__ __forceinline__ T warp_before(T x) {      // with its own
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const T y = __shfl_up_sync(~0u, x, o);
        if (lane >= o) x += y;
    }
    return x;
}

// .. and, from that, without it: not by subtraction, which would lose what is small beside its own
template <class T>
__device__ __forceinline__ T without_own(T in) {
    const T y = __shfl_up_sync(~0u, in, 1);
    return (threadIdx.x & 31) ? y : T(0);
}

// ---- T threads that work on a row: a block, or the blocks of a cluster ----
__device__ __forceinline__ int thread_index() { return (int)threadIdx.x; }
__device__ __forceinline__ int warp_index() { return (int)threadIdx.x >> 5; }
constexpr int kMaxCluster = 8;     // of blocks of 512
// Elements that are listed and sorted at most, intervals of a row's values, and groups of elements whose largest one is kept
template <int T>
struct Sizes {
    static constexpr int kListed = T == 128 ? 1024 : 2048, kBins = T == 128 ? 512 : 2048, kGroups = 2048;
};
template <int T>
struct Shared {
    static constexpr int W = T / 32, kRuns = T == 512 ? W * kMaxCluster : W;
    float most[kRuns];             // per run of the row, in a cluster in its first block
    double sum[kRuns];
    double table[kSteps];
    double more[W];
    int count[W];
    float block_most[kMaxCluster];
    double block_sum[kMaxCluster];
    double before, after;
    int found, listed, lowest, highest, before_it;
    uint32_t key_low, key_high;
};
template <int T>
struct Lists {                     // of the kernel with filters
    using S = Sizes<T>;
    union {
        struct {
            uint32_t hist[S::kBins], parts[S::kBins];
        };
        double weight[S::kListed];
    };
    union {
        unsigned long long key[S::kListed];
        float group[S::kGroups];   // until the list is made
    };
    uint32_t id[S::kListed];
};

template <int T>
__device__ __forceinline__ double team_sum(double x, Shared<T>& sh) {
    x = warp_sum(x);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh.more[warp_index()] = x;
    __syncthreads();
    x = 0.0;
#pragma unroll
    for (int w = 0; w < T / 32; ++w) x += sh.more[w];
    return x;
}
template <int T>
__device__ __forceinline__ int team_sum(int x, Shared<T>& sh) {
    x = __reduce_add_sync(~0u, x);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh.count[warp_index()] = x;
    __syncthreads();
    x = 0;
#pragma unroll
    for (int w = 0; w < T / 32; ++w) x += sh.count[w];
    return x;
}
// what the threads before this one have
template <int T>
__device__ __forceinline__ double team_before(double x, Shared<T>& sh) {
    const double in = warp_before(x), out = without_own(in);
    __syncthreads();
    if ((threadIdx.x & 31) == 31) sh.more[warp_index()] = in;
    __syncthreads();
    double before = 0.0;
    for (int w = 0; w < warp_index(); ++w) before += sh.more[w];
    return before + out;
}
template <int T>
__device__ __forceinline__ int team_before(int x, Shared<T>& sh) {
    const int in = warp_before(x);
    __syncthreads();
    if ((threadIdx.x & 31) == 31) sh.count[warp_index()] = in;
    __syncthreads();
    int before = in - x;
    for (int w = 0; w < warp_index(); ++w) before += sh.count[w];
    return before;
}
// `place` set to `value` for all, with a barrier on both sides
template <int T, class V>
__device__ __forceinline__ void set_all(V& place, V value) {
    __syncthreads();
    if (thread_index() == 0) place = value;
    __syncthreads();
}
template <int T>
__device__ __forceinline__ void fill_table(Shared<T>& sh) {
    __syncthreads();
    if (thread_index() < kSteps) sh.table[thread_index()] = exp2(thread_index() / (double)kSteps);
    __syncthreads();
}

// ---- a row's vectors ----
template <class E>
using Batch = Vector<E>[kUnroll];
// f(batch, number of its first vector) for the vectors [begin, end), a warp's lanes side by side; what is not in the row is -inf.
template <class E, class F>
__device__ __forceinline__ void over_vectors(const Row<E>& x, int begin, int end, F&& f) {
    const int lane = threadIdx.x & 31;
    for (int v = begin; v < end; v += 32 * kUnroll) {
        Batch<E> in;
        if (v >= x.lo && v + 32 * kUnroll <= min(end, x.hi)) {
            const E* const from = x.x + x.first(v + lane);
#pragma unroll
            for (int k = 0; k < kUnroll; ++k) in[k] = Row<E>::load_at(from + k * 32 * Vector<E>::N);
        } else {
#pragma unroll
            for (int k = 0; k < kUnroll; ++k) in[k] = v + lane + k * 32 < end ? x.load(v + lane + k * 32) : Row<E>::nothing();
        }
        f(in, v + lane);
    }
}
// .. a vector at a time: f(vector, its number)
template <class E, class F>
__device__ __forceinline__ void over_single(const Row<E>& x, int begin, int end, F&& f) {
    over_vectors(x, begin, end, [&](const Batch<E>& in, int v) {
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) f(in[k], v + k * 32);
    });
}
// .. element by element, two at a time: f(element, id)
template <class E, class F>
__device__ __forceinline__ void over_elements(const Row<E>& x, int begin, int end, F&& f) {
    over_single(x, begin, end, [&](const Vector<E>& in, int v) {
#pragma unroll 1
        for (int i = 0; i < Vector<E>::N / 2; ++i) {
            float y, z;
            split(in.at(i), y, z);
            f(y, x.first(v) + 2 * i), f(z, x.first(v) + 2 * i + 1);
        }
    });
}
template <class E>
__device__ __forceinline__ float largest(const Batch<E>& in) {
    float most = in[0].max();
#pragma unroll
    for (int k = 1; k < kUnroll; ++k) most = max_nan(most, in[k].max());
    return most;
}
template <class E>
__device__ __forceinline__ Pair weights_of(const Vector<E>& in, Pair by, Pair off) {
    constexpr int P = Vector<E>::N / 2;
    Pair e[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        float a, b;
        split(fma2(in.at(i), by, off), a, b);
        e[i] = pair_of(exp2_fast(a), exp2_fast(b));
    }
    Pair sum = e[0] + e[1];
    if constexpr (P == 4) sum = sum + (e[2] + e[3]);
    return sum;
}
template <class E>
__device__ __forceinline__ float weights_of(const Batch<E>& in, const Scale& c, float M) {
    const Pair off = pair_of(-M, -M), by = pair_of(c.c, c.c);
    Pair sum[kUnroll];
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) sum[k] = weights_of(in[k], by, off);
    float a, b;
    split((sum[0] + sum[1]) + (sum[2] + sum[3]), a, b);
    return a + b;
}
template <class E>
__device__ __forceinline__ float weights_of_one(const Vector<E>& in, const Scale& c, float M) {
    float a, b;
    split(weights_of(in, pair_of(c.c, c.c), pair_of(-M, -M)), a, b);
    return a + b;
}
// .. with -inf in the place of what is not wanted
template <class E, class F>
__device__ __forceinline__ void mask(Batch<E>& in, const Row<E>& x, int v, F&& wanted) {
#pragma unroll
    for (int k = 0; k < kUnroll; ++k)
#pragma unroll
        for (int i = 0; i < Vector<E>::N / 2; ++i) {
            float a, b;
            split(in[k].at(i), a, b);
            const int id = x.first(v + k * 32) + 2 * i;
            in[k].put(i, pair_of(wanted(a, id) ? a : -CUDART_INF_F, wanted(b, id + 1) ? b : -CUDART_INF_F));
        }
}

// The vectors that a warp of `warps` takes: neighbours, so that the warps' sums are those of runs of ids.
struct Runs {
    int vectors, per;
    __device__ __forceinline__ Runs(int vectors, int warps) : vectors(vectors), per(((vectors + warps - 1) / warps + 31) / 32 * 32) {}
    __device__ __forceinline__ int begin(int w) const { return min(w * per, vectors); }
    __device__ __forceinline__ int end(int w) const { return min((w + 1) * per, vectors); }
};

// Sums of runs with base M, each in sh.sum; all of them together.  Every warp adds them in the same order.
template <int T>
__device__ __forceinline__ double sum_of_runs(const Shared<T>& sh, int runs) {
    double s = 0.0;
    for (int r = threadIdx.x & 31; r < runs; r += 32) s += sh.sum[r];
    return warp_sum(s);
}
struct Total {
    float m, M;
    double S;
};
// A warp's run: its largest element and the sum of its weights with that one's base.  each(largest of a lane's batch)
template <class E, class F>
__device__ __forceinline__ void sum_run(const Row<E>& x, int begin, int end, const Scale& c, float& most, double& sum, F&& each) {
    float m = -CUDART_INF_F, M = 0.0f;
    double s = 0.0;
    over_vectors(x, begin, end, [&](const Batch<E>& in, int) {
        const float l = largest(in);
        each(l);
        if (!(l <= m)) {
            const float higher = c.base(l);
            s = m == -CUDART_INF_F ? 0.0 : s * power(M - higher);
            m = max_nan(m, l);
            M = higher;
        }
        s += (double)weights_of(in, c, M);
    });
    most = warp_max_nan(m);
    sum = warp_sum(m == -CUDART_INF_F ? 0.0 : s * power(M - c.base(most)));
}
// What the warps left in sh.most and sh.sum, brought to one base.
template <int T>
__device__ __forceinline__ Total join_runs(Shared<T>& sh, int runs, const Scale& c) {
    float m = -CUDART_INF_F;
    for (int r = threadIdx.x & 31; r < runs; r += 32) m = max_nan(m, sh.most[r]);
    Total t = {warp_max_nan(m), 0.0f, 0.0};
    t.M = c.base(t.m);
    for (int r = thread_index(); r < runs; r += T) sh.sum[r] *= power((sh.most[r] == -CUDART_INF_F ? -CUDART_INF_F : c.base(sh.most[r])) - t.M);
    __syncthreads();
    t.S = sum_of_runs(sh, runs);
    return t;
}
// The sums of the runs over what is kept, in 32-bit weights with base M; how many are kept.
template <class E, int T>
__device__ __noinline__ double fast_sums(const Row<E> x, const Scale c, float M, const Cut cut, Shared<T>& sh, int& kept) {
    const Runs runs(x.vectors, T / 32);
    const int warp = warp_index();
    double s = 0.0;
    int n = 0;
    over_vectors(x, runs.begin(warp), runs.end(warp), [&](const Batch<E>& given, int v) {
        if (!(largest(given) >= cut.value)) return;
        Batch<E> in;
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) in[k] = given[k];
        mask(in, x, v, [&](float y, int i) {
            const bool keep = cut.keeps(y, i);
            n += keep;
            return keep;
        });
        s += (double)weights_of(in, c, M);
    });
    s = warp_sum(s);
    kept = team_sum<T>(n, sh);
    if ((threadIdx.x & 31) == 0) sh.sum[warp] = s;
    __syncthreads();
    return sum_of_runs(sh, T / 32);
}
// .. in 64-bit weights
template <class E, int T>
__device__ __forceinline__ double exact_sums(const Row<E>& x, const Exact& w, const Cut& cut, Shared<T>& sh, int& kept) {
    const Runs runs(x.vectors, T / 32);
    const int warp = warp_index();
    double s = 0.0;
    int n = 0;
    over_single(x, runs.begin(warp), runs.end(warp), [&](const Vector<E>& in, int v) {
#pragma unroll 2                       // four weights at a time
        for (int i = 0; i < Vector<E>::N / 2; ++i) {
            float y, z;
            split(in.at(i), y, z);
            const bool keep_y = cut.keeps(y, x.first(v) + 2 * i), keep_z = cut.keeps(z, x.first(v) + 2 * i + 1);
            s += w.weight(y, keep_y) + w.weight(z, keep_z);
            n += keep_y + keep_z;
        }
    });
    s = warp_sum(s);
    kept = team_sum<T>(n, sh);
    if ((threadIdx.x & 31) == 0) sh.sum[warp] = s;
    __syncthreads();
    return sum_of_runs(sh, T / 32);
}

// The first element at which the running sum exceeds `target`: the run by sh.sum, the thread's part of that run, the element.  sh.found is the
// element, or -1, and sh.before and sh.after are the sums on its two sides.  weight(element, id); of_vector(vector, its number)
template <class E, int T, class Weight, class Sum>
__device__ __forceinline__ void find(const Row<E>& x, const Runs& runs, int n_runs, double target, Shared<T>& sh, Weight&& weight, Sum&& of_vector) {
    const int lane = threadIdx.x & 31, tid = thread_index();
    // the last run before which the sum does not exceed it, among those that weigh
    double before = 0.0, from_run = 0.0;
    int run = 0;
    for (int r0 = 0; r0 < n_runs; r0 += 32) {
        const double s = r0 + lane < n_runs ? sh.sum[r0 + lane] : 0.0, in = warp_before(s), out = without_own(in);
        const unsigned int here = __ballot_sync(~0u, s > 0.0 && before + out <= target);
        if (here) {
            const int l = 31 - __clz(here);
            run = r0 + l;
            from_run = before + __shfl_sync(~0u, out, l);
        }
        before += __shfl_sync(~0u, in, 31);
    }
    const int begin = runs.begin(run), end = runs.end(run), per = (end - begin + T - 1) / T;
    const int mine = begin + tid * per, stop = min(mine + per, end);
    double s = 0.0;
#pragma unroll 4
    for (int v = mine; v < stop; ++v) s += of_vector(x.load(v), v);
    const double from = from_run + team_before<T>(s, sh);
    if (tid == 0) sh.found = -1, sh.lowest = -1;
    __syncthreads();
    if (s > 0.0 && from <= target) atomicMax(&sh.lowest, tid);
    __syncthreads();
    // that thread's elements, its warp's lanes side by side
    const int owner = sh.lowest;
    if (owner >= 0 && tid >> 5 == owner >> 5) {
        double sum = __shfl_sync(~0u, from, owner & 31);
        const int v0 = begin + owner * per, v1 = min(v0 + per, end);
        int last = -1;
        double last_before = 0.0, last_after = 0.0;
        for (int i0 = max(x.first(v0), 0); i0 < min(x.first(v1), x.V); i0 += 32) {
            const int i = i0 + lane;
            const bool in_row = i < min(x.first(v1), x.V);
            const double w = in_row ? weight(as_float(x.x[i]), i) : 0.0;
            const double in = warp_before(w), out = without_own(in);
            const unsigned int here = __ballot_sync(~0u, w > 0.0 && sum + out <= target);
            if (here) {
                const int l = 31 - __clz(here);
                last = i0 + l;
                last_before = sum + __shfl_sync(~0u, out, l), last_after = sum + __shfl_sync(~0u, in, l);
            }
            sum += __shfl_sync(~0u, in, 31);
        }
        if (lane == 0) sh.found = last, sh.before = last_before, sh.after = last_after;
    }
    __syncthreads();
}

// Drawn from what is kept in 64 bits, sh.sum and C being its sums.  log2_S: of the whole row's sum.
template <class E, int T>
__device__ __forceinline__ void draw_exactly(const SampleArgs& a, int64_t row, const Row<E>& x, const Scale& c, const Exact& w, float u, const Cut& cut, double log2_S, double C,
                                             int kept, Shared<T>& sh) {
    auto weight = [&](float y, int i) { return w.weight(y, cut.keeps(y, i)); };
    find<E, T>(x, Runs(x.vectors, T / 32), T / 32, u * C, sh, weight, [&](const Vector<E>& in, int v) {
        double s = 0.0;
#pragma unroll 1
        for (int i = 0; i < Vector<E>::N / 2; ++i) {
            float y, z;
            split(in.at(i), y, z);
            s += weight(y, x.first(v) + 2 * i) + weight(z, x.first(v) + 2 * i + 1);
        }
        return s;
    });
    if (thread_index() == 0) {
        const int token = sh.found;
        const double z = token < 0 ? 0.0 : ((double)as_float(x.x[token]) - w.m) * c.exact, log2_C = log2(C);
        write(a, row, token, (float)((z - (log2_S == log2_S ? log2_S : log2_C)) * 0.6931471805599453), (float)((z - log2_C) * 0.6931471805599453), kept);
    }
}
template <class E, int T>
__device__ __forceinline__ void write_greedy(const SampleArgs& a, int64_t row, const Row<E>& x, float m, Shared<T>& sh) {
    set_all<T>(sh.found, 0x7FFFFFFF);
    const Runs runs(x.vectors, T / 32);
    int first = 0x7FFFFFFF;
    over_vectors(x, runs.begin(warp_index()), runs.end(warp_index()), [&](const Batch<E>& in, int v) {
#pragma unroll
        for (int k = 0; k < kUnroll; ++k)
            if (in[k].max() == m)
#pragma unroll
                for (int e = 0; e < Vector<E>::N; ++e)
                    if (in[k].one(e) == m) first = min(first, x.first(v + k * 32) + e);
    });
    if (first != 0x7FFFFFFF) atomicMin(&sh.found, first);
    __syncthreads();
    if (thread_index() == 0) write(a, row, sh.found, 0.0f, 0.0f, 1);
}

// The block's row, and in a cluster the part of it that the block takes.
template <int T>
struct Place {
    int rank = 0, blocks = 1;
    int64_t row = blockIdx.x;
    __device__ __forceinline__ Place() {
        if constexpr (T == 512) {
            rank = (int)cg::this_cluster().block_rank(), blocks = (int)cg::this_cluster().num_blocks();
            row = blockIdx.x / blocks;
        }
    }
    __device__ __forceinline__ int run() const { return rank * (T / 32) + warp_index(); }
    __device__ __forceinline__ int runs() const { return blocks * (T / 32); }
    // a barrier of all that work on the row
    __device__ __forceinline__ void sync() const {
        if (T == 512 && blocks > 1) cg::this_cluster().sync();
        else __syncthreads();
    }
    template <class P>
    __device__ __forceinline__ P* of_block(P* p, int r) const {
        if constexpr (T == 512)
            if (blocks > 1) return cg::this_cluster().map_shared_rank(p, r);
        return p;
    }
};

// ---- the whole distribution ----
// One pass over the row at the copy's rate (4,096 x 128,000 bf16: 162 us, 99 %), a second look at the run, the part and the vector in which the token is
// (188), and, for one row in twenty-five where 32 bits do not decide, the row once more in 64 (269 in all): 46 instructions a token there,
// 14 of them in 64 bits, whose chain is what it waits for.  More registers, four or eight weights at a time, the rows left to a kernel of its own with
// larger blocks (417 us: too few of them to share out evenly) were no faster.
template <class E, int T>
__global__ void __launch_bounds__(T) draw_kernel(SampleArgs a) {
    __shared__ Shared<T> sh;
    const Place<T> at;
    const int64_t row = at.row;
    const Asked r = asked_of<false>(a, row);
    if (r.kind) {
        if (at.rank == 0 && thread_index() == 0) write_none(a, row, r.kind, 0.0f);
        return;
    }
    const Row<E> x(static_cast<const E*>(a.logits) + row * a.stride, a.vocab);
    const Scale c(r.T == 0.0 ? 1.0 : r.T);
    const Runs runs(x.vectors, at.runs());
    float most;
    double sum;
    sum_run(x, runs.begin(at.run()), runs.end(at.run()), c, most, sum, [](float) {});
    if (T == 512 && at.blocks > 1) at.sync();                  // every block has begun
    if ((threadIdx.x & 31) == 0) at.of_block(sh.most, 0)[at.run()] = most, at.of_block(sh.sum, 0)[at.run()] = sum;
    at.sync();
    if (at.rank) return;
    const Total t = join_runs(sh, at.runs(), c);
    if (!is_finite(t.m)) {
        if (thread_index() == 0) write_none(a, row, 0, t.m);
        return;
    }
    if (r.T == 0.0) {
        write_greedy<E, T>(a, row, x, t.m, sh);
        return;
    }
    if (c.holds(t.m)) {
        const double target = r.u * t.S, margin = Error(a.vocab, t.S, c).at(r.u) * t.S;
        find<E, T>(x, runs, at.runs(), target, sh, [&](float y, int) { return (double)c.weight(y, t.M); },
                   [&](const Vector<E>& in, int) { return (double)weights_of_one(in, c, t.M); });
        const int token = sh.found;
        if (token >= 0 && target - sh.before >= margin && sh.after - target >= margin) {
            if (thread_index() == 0) {
                const double log2_S = log2(t.S) - c.of_largest(t.m, t.M);
                const float logprob = (float)((((double)as_float(x.x[token]) - t.m) * c.exact - log2_S) * 0.6931471805599453);
                write(a, row, token, logprob, logprob, 0);
            }
            return;
        }
        __syncthreads();
    }
    fill_table(sh);
    const Exact w(t.m, c, sh.table);
    int everything;
    const double S = exact_sums<E, T>(x, w, unmasked(), sh, everything);
    draw_exactly<E, T>(a, row, x, c, w, r.u, unmasked(), CUDART_NAN, S, 0, sh);
}

// ---- what is kept ----

// The list by rank, which is how many other keys are above: ids and weights.  No two keys are equal.
template <int T>
__device__ __forceinline__ void rank_list(Lists<T>& lists, int n, const Exact& w) {
    for (int i = thread_index(); i < n; i += T) {
        const unsigned long long mine = lists.key[i];
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) rank += lists.key[j] > mine;
        lists.id[rank] = position_of(mine);
        lists.weight[rank] = w.weight(value_of((uint32_t)(mine >> 32)));
    }
    __syncthreads();
}
// Keys fall from key[0] to key[n - 1], n <= kListed.  Distances below 64 stay in a warp's registers, two keys a lane: 2,048 keys take 15 passes
// through shared memory and six of those instead of 66 (34,000 cycles).
template <int T>
__device__ __forceinline__ void sort_list(unsigned long long* key, int n) {
    const int lane = threadIdx.x & 31;
    int size = 64;
    while (size < n) size *= 2;
    for (int i = n + thread_index(); i < size; i += T) key[i] = 0;
    __syncthreads();
    for (int k = 64; k <= size; k *= 2) {
        for (int j = k / 2; j >= 64; j /= 2) {
            for (int i = thread_index(); i < size / 2; i += T) {
                const int p = 2 * i - (i & (j - 1)), q = p + j;
                const unsigned long long x = key[p], y = key[q];
                if ((x < y) == !(p & k)) key[p] = y, key[q] = x;
            }
            __syncthreads();
        }
        for (int part = warp_index(); part < size / 64; part += T / 32) {
            unsigned long long a = key[part * 64 + lane], b = key[part * 64 + 32 + lane];
            const bool falls = !(part * 64 & k);
            if (k == 64) {
                a = sorted(a);
                b = __shfl_sync(~0u, sorted(b), 31 - lane);
            }
            const unsigned long long x = larger_if(falls, a, b), y = larger_if(!falls, a, b);
            a = x, b = y;
#pragma unroll
            for (int j = 16; j; j /= 2) {
                const bool first = !(lane & j) == falls;
                a = larger_if(first, a, __shfl_xor_sync(~0u, a, j));
                b = larger_if(first, b, __shfl_xor_sync(~0u, b, j));
            }
            key[part * 64 + lane] = a, key[part * 64 + 32 + lane] = b;
        }
        __syncthreads();
    }
}

// Intervals of the exponents t <= 0 of weights 2^t, from 0 down, kBins in 64 octaves.  With an interval's count goes the sum of what its exponents are
// beyond its beginning, in 256ths of it.  The sum of its weights then lies between the count times the weight at the mean exponent and what the chord
// over the interval gives: 6e-5 more at 32 an octave.
template <int kBins>
struct Intervals {
    static constexpr int kPerOctave = kBins / 64, kParts = 256;
    // to the nearest 256th: falls with the exponent, -inf last
    static __device__ __forceinline__ int depth(float t) {
        const float d = fminf(t * -(float)(kPerOctave * kParts), kBins * kParts - 1.0f);
        return __float_as_int(d + 12582912.0f) - 0x4B400000;      // 1.5 x 2^23
    }
    struct Bounds {
        float least, most;
    };
    static __device__ __forceinline__ Bounds sum_of(int b, uint32_t count, uint32_t parts) {
        if (count == 0) return {0.0f, 0.0f};
        constexpr float per = 1.0f / kPerOctave;
        // the roundings to 256ths, of exponents of up to 64 in 32 bits, and of this and what adds up a thread's intervals
        constexpr float slack = 0.36f / (kParts * kPerOctave) + 1.8e-5f;
        const float n = (float)count, mean = __fdividef((float)parts, n) * (1.0f / kParts), first = exp2_fast(b * -per), next = exp2_fast((b + 1) * -per);
        // the last interval goes on to 0
        return {b == kBins - 1 ? 0.0f : n * exp2_fast((b + mean) * -per) * (1.0f - slack), n * (first + (next - first) * mean) * (1.0f + slack)};
    }
};

// Looks for the border of what is kept: the intervals, an interval or two, in which it lies; the elements of those, listed and sorted.  What is
// too many for that is halved at the middle of its values, as often as it takes; if all are equal, the border is a matter of their ids.
template <class E, int T>
struct Search {
    static constexpr int kBins = Sizes<T>::kBins, kListed = Sizes<T>::kListed;
    using In = Intervals<kBins>;
    const Row<E> x;
    const Scale c;
    const Exact w;
    const float m;
    Shared<T>& sh;
    Lists<T>& lists;
    const Runs runs;

    __device__ __forceinline__ Search(const Row<E>& x, const Scale& c, const Total& t, Shared<T>& sh, Lists<T>& lists)
        : x(x), c(c), w(t.m, c, sh.table), m(t.m), sh(sh), lists(lists), runs(x.vectors, T / 32) {}
    __device__ __forceinline__ int begin() const { return runs.begin(warp_index()); }
    __device__ __forceinline__ int end() const { return runs.end(warp_index()); }
    // Of the exponent below the largest element's, for which 32 bits do.
    __device__ __forceinline__ int depth(float y) const { return In::depth((y - m) * c.c); }
    __device__ __forceinline__ int bin(float y) const { return depth(y) / In::kParts; }

    // kAll: nothing but what is masked is left out
    template <bool kAll>
    static __device__ __forceinline__ bool keeps(const Cut& in, float y, int i) { return kAll ? y > -CUDART_INF_F : in.keeps(y, i); }
    template <bool kAll>
    __device__ __forceinline__ void count(const Cut& in, bool parts) {
        __syncthreads();
        for (int b = thread_index(); b < kBins; b += T) lists.hist[b] = lists.parts[b] = 0;
        __syncthreads();
        over_elements(x, begin(), end(), [&](float y, int i) {
            if (!keeps<kAll>(in, y, i)) return;
            const int d = depth(y);
            atomicAdd(&lists.hist[d / In::kParts], 1u);
            if (parts) atomicAdd(&lists.parts[d / In::kParts], (uint32_t)(d % In::kParts));
        });
        __syncthreads();
    }
    // The first interval up to which there are n elements (sh.highest), how many there are before it (sh.before_it) and in it (sh.listed);
    // without so many, the last one.
    __device__ __forceinline__ void reach(int n) {
        constexpr int per = kBins / T;
        const int b0 = thread_index() * per;
        int mine = 0;
        for (int b = b0; b < b0 + per; ++b) mine += lists.hist[b];
        int sum = team_before<T>(mine, sh);
        if (sum < n && (sum + mine >= n || thread_index() == T - 1)) {
            int b = b0;
            for (; b < b0 + per - 1 && sum + (int)lists.hist[b] < n; ++b) sum += lists.hist[b];
            sh.lowest = sh.highest = b, sh.before_it = sum, sh.listed = lists.hist[b];
        }
        __syncthreads();
    }
    // The intervals sh.lowest to sh.highest in which the running sum reaches B, which is known to `margin`; the elements before and in them.
    __device__ __forceinline__ void bracket(double B, double margin) {
        constexpr int per = kBins / T;
        const int b0 = thread_index() * per;
        auto sum_of = [&](int b) { return In::sum_of(b, lists.hist[b], lists.parts[b]); };
        float hi = 0.0f, lo = 0.0f;
        for (int b = b0; b < b0 + per; ++b) {
            const auto s = sum_of(b);
            hi += s.most, lo += s.least;
        }
        double sum_hi = team_before<T>((double)hi, sh), sum_lo = team_before<T>((double)lo, sh);
        if (thread_index() == 0) sh.lowest = sh.highest = kBins - 1;
        __syncthreads();
        if (sum_hi + hi >= B - margin || sum_lo + lo >= B + margin)
            for (int b = b0; b < b0 + per; ++b) {
                const auto s = sum_of(b);
                sum_hi += s.most, sum_lo += s.least;
                if (sum_hi >= B - margin) atomicMin(&sh.lowest, b);
                if (sum_lo >= B + margin) atomicMin(&sh.highest, b);
                if (sum_lo >= B + margin) break;
            }
        __syncthreads();
        int before = 0, inside = 0;
        const int first = min(sh.lowest, sh.highest), last = sh.highest;
        for (int b = b0; b < b0 + per; ++b) (b < first ? before : inside) += b <= last ? lists.hist[b] : 0;
        before = team_sum<T>(before, sh), inside = team_sum<T>(inside, sh);
        __syncthreads();
        if (thread_index() == 0) sh.lowest = first, sh.before_it = before, sh.listed = inside;
        __syncthreads();
    }

    __device__ __forceinline__ void append(float y, int i) {
        const int n = atomicAdd(&sh.listed, 1);
        if (n < kListed) lists.key[n] = key_of(y, i);
    }
    // .. those elements of vector v of which the bits are set
    __device__ __forceinline__ void append(const Vector<E>& in, int v, uint32_t which) {
        if (!which) return;
        int n = atomicAdd(&sh.listed, __popc(which));
#pragma unroll 1
        for (; which; which &= which - 1, ++n) {
            const int e = __ffs(which) - 1;
            float y, z;
            split(in.at(e / 2), y, z);
            if (n < kListed) lists.key[n] = key_of(e & 1 ? z : y, x.first(v) + e);
        }
    }
    // Everything down to interval `hi`, which is as much as a list holds.
    __device__ __forceinline__ void list(int hi) {
        set_all<T>(sh.listed, 0);
        over_single(x, begin(), end(), [&](const Vector<E>& in, int v) {
            if (bin(in.max()) > hi) return;
            uint32_t which = 0;
#pragma unroll
            for (int e = 0; e < Vector<E>::N; ++e) which |= (uint32_t)(in.one(e) > -CUDART_INF_F && bin(in.one(e)) <= hi) << e;
            append(in, v, which);
        });
        __syncthreads();
    }
    __device__ __forceinline__ float value(int i) const { return value_of((uint32_t)(lists.key[i] >> 32)); }
    __device__ __forceinline__ Cut cut_at(int i) const { return {value(i), position_of(lists.key[i])}; }
    // The first of n places at which above + the running sum of lists.weight reaches B, or exceeds it; the last if none does.  sh.before and
    // sh.after: the sums on its two sides.
    template <bool kExceeds>
    __device__ __forceinline__ int reach_in_list(int n, double above, double B) {
        const int per = (n + T - 1) / T, i0 = min(thread_index() * per, n), i1 = min(i0 + per, n);
        double mine = 0.0;
        for (int i = i0; i < i1; ++i) mine += lists.weight[i];
        const double from = above + team_before<T>(mine, sh);
        set_all<T>(sh.found, n - 1);
        double sum = from;
        for (int i = i0; i < i1; ++i) {
            sum += lists.weight[i];
            if (kExceeds ? sum > B : sum >= B) {
                atomicMin(&sh.found, i);
                break;
            }
        }
        __syncthreads();
        const int at = sh.found;
        if (at >= i0 && at < i1) {
            sum = from;
            for (int i = i0; i < at; ++i) sum += lists.weight[i];
            sh.before = sum, sh.after = sum + lists.weight[at];
        }
        __syncthreads();
        return at;
    }

    // The border in intervals sh.lowest to sh.highest: of the first k elements of `in`, or (k = 0) of those whose sum reaches p times that of `in`,
    // in 64-bit weights.  With k = 0, `of` is that sum, and C and `kept` are the sum and the number of what is kept, sh.sum the runs' sums of it, unless
    // C is NaN.
    template <bool kAll>
    __device__ __forceinline__ Cut border(const Cut& in, int k, double p, double& of, double& C, int& kept) {
        const int lo = sh.lowest, hi = sh.highest;
        int above = sh.before_it, n = sh.listed;
        __syncthreads();
        if (thread_index() == 0) sh.key_low = 0xFFFFFFFFu, sh.key_high = 0, sh.listed = 0;
        __syncthreads();
        const bool fits = n <= kListed;
        double S = 0.0, A = 0.0, B = 0.0;
        uint32_t low = 0xFFFFFFFFu, high = 0;
        C = CUDART_NAN;
        over_single(x, begin(), end(), [&](const Vector<E>& v, int at) {
            if (k && bin(v.max()) > hi) return;
#pragma unroll 2
            for (int q = 0; q < Vector<E>::N / 2; ++q) {
                float y, z;
                split(v.at(q), y, z);
                const int id = x.first(at) + 2 * q;
                const int b_y = keeps<kAll>(in, y, id) ? bin(y) : kBins, b_z = keeps<kAll>(in, z, id + 1) ? bin(z) : kBins;
                if (k == 0) {
                    const double one = w.weight(y, b_y < kBins), two = w.weight(z, b_z < kBins);
                    S += one + two;
                    A += (b_y < lo ? one : 0.0) + (b_z < lo ? two : 0.0);
                }
                auto take = [&](float value, int i, int b) {
                    if (b < lo || b > hi) return;
                    if (fits) append(value, i);
                    else low = min(low, order_of(value)), high = max(high, order_of(value));
                };
                take(y, id, b_y), take(z, id + 1, b_z);
            }
        });
        if (k == 0) {
            of = team_sum<T>(S, sh);
            B = share_of(p, of);
            A = warp_sum(A);
            if ((threadIdx.x & 31) == 0) sh.sum[warp_index()] = A;
            __syncthreads();
            A = sum_of_runs(sh, T / 32);
        }
        if (!fits) {
            atomicMin(&sh.key_low, low), atomicMax(&sh.key_high, high);
            __syncthreads();
            uint32_t bottom = sh.key_low, top = sh.key_high;
            while (n > kListed && bottom < top) {
                const uint32_t middle = bottom + (top - bottom) / 2;       // the upper half: above it
                double s = 0.0;
                int upper = 0;
                low = 0xFFFFFFFFu, high = 0;
                over_elements(x, begin(), end(), [&](float y, int i) {
                    const uint32_t o = order_of(y);
                    if (o < bottom || o > top || !keeps<kAll>(in, y, i)) return;
                    if (o > middle) {
                        ++upper;
                        low = min(low, o);
                        if (k == 0) s += w.weight(y);
                    } else {
                        high = max(high, o);
                    }
                });
                upper = team_sum<T>(upper, sh);
                s = team_sum<T>(s, sh);
                __syncthreads();
                if (thread_index() == 0) sh.key_low = 0xFFFFFFFFu, sh.key_high = 0;
                __syncthreads();
                atomicMin(&sh.key_low, low), atomicMax(&sh.key_high, high);
                __syncthreads();
                if (k ? above + upper >= k : A + s >= B) bottom = sh.key_low, n = upper;
                else top = sh.key_high, above += upper, n -= upper, A += s;
            }
            if (bottom == top) {
                // all equal: the border is the id of the last one that is kept
                const float v = value_of(top);
                const int wanted = k ? k - above : (int)fmin(fmax(ceil((B - A) / w.weight(v)), 1.0), (double)n);
                int mine = 0;
                over_elements(x, begin(), end(), [&](float y, int i) { mine += y == v && keeps<kAll>(in, y, i); });
                mine = __reduce_add_sync(~0u, mine);
                __syncthreads();
                if ((threadIdx.x & 31) == 0) sh.count[warp_index()] = mine;
                set_all<T>(sh.found, 0);
                int before = 0;
                for (int r = 0; r < warp_index(); ++r) before += sh.count[r];
                if (before < wanted && before + mine >= wanted)            // in this warp's run
                    for (int v0 = begin(); v0 < end() && before < wanted; v0 += 32) {
                        const int at = v0 + (threadIdx.x & 31);
                        const Vector<E> in_v = at < end() ? x.load(at) : Row<E>::nothing();
                        auto is = [&](int e) { return in_v.one(e) == v && keeps<kAll>(in, v, x.first(at) + e); };
                        int equal = 0;
#pragma unroll
                        for (int e = 0; e < Vector<E>::N; ++e) equal += is(e);
                        const int up_to = warp_before(equal);
                        int rank = before + up_to - equal;
                        if (rank < wanted && rank + equal >= wanted)
#pragma unroll
                            for (int e = 0; e < Vector<E>::N; ++e)
                                if (is(e) && ++rank == wanted) sh.found = x.first(at) + e;
                        before += __shfl_sync(~0u, up_to, 31);
                    }
                __syncthreads();
                return {v, (uint32_t)sh.found};
            }
            set_all<T>(sh.listed, 0);
            over_elements(x, begin(), end(), [&](float y, int i) {
                const uint32_t o = order_of(y);
                if (o >= bottom && o <= top && keeps<kAll>(in, y, i)) append(y, i);
            });
        }
        __syncthreads();
        n = min(sh.listed, kListed);
        sort_list<T>(lists.key, n);
        if (k) return cut_at(min(k - above, n) - 1);
        for (int i = thread_index(); i < n; i += T) lists.weight[i] = w.weight(value(i));
        __syncthreads();
        const int at = reach_in_list<false>(n, A, B);
        if (fits) {
            // those of the list that are kept, to their runs
            double s = 0.0;
            for (int i = threadIdx.x & 31; i <= at; i += 32)
                if (((int)position_of(lists.key[i]) + x.skip) / Vector<E>::N / runs.per == warp_index()) s += lists.weight[i];
            s = warp_sum(s);
            if ((threadIdx.x & 31) == 0) sh.sum[warp_index()] += s;
            __syncthreads();
            C = sum_of_runs(sh, T / 32);
            kept = above + at + 1;
        }
        return cut_at(at);
    }
};

// Where weights, as 64 bits hold them, reach min_p: m + T ln q, and near 1, where many logits have the weight 1, as far below as that rounding goes.  Nothing
// below the first reaches it, everything from the second on does.
__device__ __forceinline__ float below_min_p(const Asked& r, float m) { return fminf(not_above((double)m + r.T * (log(r.q) * 1.0000001 - 4e-15)), m); }
__device__ __forceinline__ float above_min_p(const Asked& r, float m) { return fminf(not_below((double)m + r.T * (log(r.q) * 0.9999999 + 4e-15)), m); }
// The lowest logit that reaches it: a few trials
__device__ __forceinline__ float least_of(const Exact& w, const Asked& r, float m) {
    uint32_t lo = order_of(below_min_p(r, m)), hi = order_of(above_min_p(r, m));
    while (lo < hi) {
        const uint32_t middle = lo + (hi - lo) / 2;
        if (w.weight(value_of(middle)) >= r.q) hi = middle;
        else lo = middle + 1;
    }
    return value_of(hi);
}

// Rows of which more is kept than a list holds.  `counted`: by_count's, or of everything, are the counts that the search has.
template <class E, int T>
__device__ __noinline__ void draw_from_many(const SampleArgs& a, int64_t row, const Row<E> x, const Scale c, const Asked r, const Total t, bool by_count, bool counted,
                                            Shared<T>& sh, Lists<T>& lists) {
    const bool by_sum = r.p < 1.0, by_size = r.q > 0.0;
    fill_table(sh);
    Search<E, T> search(x, c, t, sh, lists);
    const Exact& w = search.w;
    const bool holds = c.holds(t.m);
    const double one = c.of_largest(t.m, t.M), to_largest = exp2(-one);      // where they hold
    Cut cut = unmasked();
    double log2_S = holds ? log2(t.S) - one : CUDART_NAN, of, C = CUDART_NAN;
    int n = 0;
    if (!holds && (by_count || by_size)) log2_S = log2(exact_sums<E, T>(x, w, unmasked(), sh, n));
    if (by_count) {
        if (!counted) search.template count<true>(unmasked(), false);
        search.reach(r.k);
        cut = search.template border<true>(unmasked(), r.k, 0.0, of, C, n);
    }
    if (by_sum) {
        const Cut in = cut;
        double about = t.S, error = 1e-13;
        if (!holds) {
            about = exact_sums<E, T>(x, w, in, sh, n);
        } else {
            if (by_count) about = fast_sums<E, T>(x, c, t.M, in, sh, n);
            error = Error(a.vocab, about, c).both();
            about *= to_largest;
        }
        if (by_count) search.template count<false>(in, true);
        else if (!counted) search.template count<true>(in, true);
        search.bracket(r.p * about, 2.0 * error * about);
        cut = tighter(in, by_count ? search.template border<false>(in, 0, r.p, of, C, n) : search.template border<true>(in, 0, r.p, of, C, n));
        if (!by_count) log2_S = log2(of);
    }
    if (by_size) {
        const Cut least = {least_of(w, r, t.m), 0xFFFFFFFFu}, both = tighter(cut, least);
        if (both.value != cut.value || both.last != cut.last) C = CUDART_NAN;
        cut = both;
    }
    if (holds && C != C) {
        C = fast_sums<E, T>(x, c, t.M, cut, sh, n);
        const double target = r.u * C, margin = Error(a.vocab, C, c).at(r.u) * C;
        auto weight = [&](float y, int i) { return cut.keeps(y, i) ? c.weight(y, t.M) : 0.0f; };
        find<E, T>(x, search.runs, T / 32, target, sh, [&](float y, int i) { return (double)weight(y, i); }, [&](const Vector<E>& in, int v) {
            float sum[2] = {0.0f, 0.0f};
#pragma unroll
            for (int e = 0; e < Vector<E>::N; ++e) sum[e & 1] += weight(in.one(e), x.first(v) + e);
            return (double)(sum[0] + sum[1]);
        });
        const int token = sh.found;
        if (token >= 0 && target - sh.before >= margin && sh.after - target >= margin) {
            if (thread_index() == 0) {
                const double z = ((double)as_float(x.x[token]) - t.m) * c.exact, log2_C = log2(C) - one;
                write(a, row, token, (float)((z - log2_S) * 0.6931471805599453), (float)((z - log2_C) * 0.6931471805599453), n);
            }
            return;
        }
        __syncthreads();
        C = CUDART_NAN;
    }
    if (C != C) C = exact_sums<E, T>(x, w, cut, sh, n);
    draw_exactly<E, T>(a, row, x, c, w, r.u, cut, log2_S, C, n, sh);
}

// Draws from a list of n elements that holds all that may be kept.  Of a share top_p alone it may fall short (unless `all_sizes`: min_p
// keeps nothing below it): false then.
template <class E, int T>
__device__ __noinline__ bool draw_from_list(const SampleArgs& a, int64_t row, const Row<E> x, const Scale c, const Asked r, const Total t, int n, bool by_count, bool all_sizes,
                                            Shared<T>& sh, Lists<T>& lists) {
    constexpr int kListed = Sizes<T>::kListed, kRanked = 256;
    const bool by_sum = r.p < 1.0, by_size = r.q > 0.0;
    const int tid = thread_index();
    if (n == 0) return false;
    fill_table(sh);
    Search<E, T> search(x, c, t, sh, lists);
    const Exact& w = search.w;
    // by rank: ids and weights
    if (n <= kRanked) {
        rank_list<T>(lists, n, w);
    } else {
        sort_list<T>(lists.key, n);
        for (int i = tid; i < n; i += T) {
            lists.id[i] = position_of(lists.key[i]);
            lists.weight[i] = w.weight(search.value(i));
        }
        __syncthreads();
    }
    double S = t.S * exp2(-c.of_largest(t.m, t.M));                // in 64-bit weights, to the error of its 32-bit ones
    int L = by_count ? min(r.k, n) : n;
    if (by_sum) {
        double of = S;
        if (by_count) {
            double mine = 0.0;
            for (int i = tid; i < L; i += T) mine += lists.weight[i];
            of = team_sum<T>(mine, sh);
        }
        int last = search.template reach_in_list<false>(L, 0.0, r.p * of);
        if (!by_count) {
            const double margin = Error(a.vocab, t.S, c).both() * S;
            if (!all_sizes && sh.after < r.p * of - margin) return false;
            if (r.p * of - sh.before < margin || fabs(sh.after - r.p * of) < margin) {
                int everything;
                S = exact_sums<E, T>(x, w, unmasked(), sh, everything);
                last = search.template reach_in_list<false>(L, 0.0, r.p * S);
                if (!all_sizes && sh.after < r.p * S) return false;
            }
        }
        L = last + 1;
    }
    if (by_size) {
        set_all<T>(sh.found, L);
        for (int i = tid; i < L; i += T)
            if (lists.weight[i] < r.q) {
                atomicMin(&sh.found, i);
                break;
            }
        __syncthreads();
        L = max(sh.found, 1);
    }
    double mine = 0.0;
    for (int i = tid; i < L; i += T) mine += lists.weight[i];
    const double C = team_sum<T>(mine, sh), target = r.u * C;
    // by id: of the tokens before which the sum does not exceed the target the last
    set_all<T>(sh.found, -1);
    if (L <= kRanked) {
        for (int i = tid; i < L; i += T) {
            const uint32_t id = lists.id[i];
            double before = 0.0;
#pragma unroll 4
            for (int j = 0; j < L; ++j) before += lists.id[j] < id ? lists.weight[j] : 0.0;
            if (lists.weight[i] > 0.0 && before <= target) atomicMax(&sh.found, (int)id);
        }
    } else {
        for (int i = tid; i < L; i += T) lists.key[i] = (unsigned long long)(0xFFFFFFFFu - lists.id[i]) << 32 | (uint32_t)i;
        sort_list<T>(lists.key, L);
        double by_id[kListed / T];
#pragma unroll
        for (int j = 0; j < kListed / T; ++j) by_id[j] = j * T + tid < L ? lists.weight[(uint32_t)lists.key[j * T + tid]] : 0.0;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kListed / T; ++j)
            if (j * T + tid < L) lists.weight[j * T + tid] = by_id[j];
        __syncthreads();
        const int first = search.template reach_in_list<true>(L, 0.0, target);
        if (tid == 0) {
            int i = first;
            while (i > 0 && lists.weight[i] == 0.0) --i;
            sh.found = (int)(0xFFFFFFFFu - (uint32_t)(lists.key[i] >> 32));
        }
    }
    __syncthreads();
    if (tid == 0) {
        const int token = sh.found;
        const double z = ((double)as_float(x.x[token]) - w.m) * c.exact * 0.6931471805599453;
        write(a, row, token, (float)(z - log(S)), (float)(z - log(C)), L);
    }
    return true;
}

// A lane's elements come in groups, of each of which the largest is kept while the row is summed up.  The k-th largest of these is at most the k-th
// largest element; and where the largest of the groups from some value on weigh as much as top_p of the sum, so do the elements from there on.  What
// reaches such a bound is in the few groups whose largest does: those are read once more, and what reaches it is listed.  Where
// that fails, the row's elements are counted, and listed if the counts allow it.
//
// 4,096 x 128,000 bf16, top 50: 270 to 295 us by the rows' likely tokens, of a row's 68,000 cycles (four at a time on an SM) 40,000 go to reading it, 12,000 to the bound, 8,000 to the
// list, 8,000 to the draw: latencies of a few dozen barriers.  Rows that keep thousands take ten times that: counting 40,000 cycles a row, 64-bit sums 110,000.
template <class E, int T>
__global__ void __launch_bounds__(T, T == 512 ? 2 : T == 256 ? 4 : 6) filter_kernel(SampleArgs a) {
    using Size = Sizes<T>;
    constexpr int kListed = Size::kListed, kGroupBins = Size::kBins < 1024 ? Size::kBins : 1024, kBlocks = T == 512 ? kMaxCluster : 1;
    using In = Intervals<kGroupBins>;
    extern __shared__ uint4 dynamic[];
    struct Both {
        Shared<T> sh;
        Lists<T> lists;
    };
    Both& both = *reinterpret_cast<Both*>(dynamic);
    Shared<T>& sh = both.sh;
    Lists<T>& lists = both.lists;
    const int tid = thread_index(), lane = tid & 31;
    const Place<T> at;
    const int64_t row = at.row;
    const Asked r = asked_of<true>(a, row);
    if (r.kind) {
        if (at.rank == 0 && tid == 0) write_none(a, row, r.kind, 0.0f);
        return;
    }
    const Row<E> x(static_cast<const E*>(a.logits) + row * a.stride, a.vocab);
    const Scale c(r.T == 0.0 ? 1.0 : r.T);
    const bool by_sum = r.p < 1.0, by_size = r.q > 0.0;
    bool by_count = r.k > 0 && r.k < a.vocab;
    const Runs runs(x.vectors, at.runs());
    const int begin = runs.begin(at.run()), end = runs.end(at.run());
    // batches of a lane to a group, and groups of a lane
    const int batches = (runs.per + 32 * kUnroll - 1) / (32 * kUnroll), span = (batches * T + Size::kGroups - 1) / Size::kGroups, groups = (batches + span - 1) / span;
    float most;
    double sum;
    {
        int n = 0, g = 0;
        float group = -CUDART_INF_F;
        sum_run(x, begin, end, c, most, sum, [&](float l) {
            group = max_nan(group, l);
            if (++n < span) return;
            lists.group[g++ * T + tid] = group;
            group = -CUDART_INF_F;
            n = 0;
        });
        for (; g < groups; ++g) {
            lists.group[g * T + tid] = group;
            group = -CUDART_INF_F;
        }
    }
    for (int b = tid; b < kGroupBins; b += T) lists.hist[b] = lists.parts[b] = 0;
    if (tid == 0) sh.listed = 0;
    if (lane == 0) sh.more[warp_index()] = most;
    at.sync();                                                 // every block has begun
    if (lane == 0) at.of_block(sh.most, 0)[at.run()] = most, at.of_block(sh.sum, 0)[at.run()] = sum;
    float block_most = (float)sh.more[0];
#pragma unroll
    for (int w = 1; w < T / 32; ++w) block_most = max_nan(block_most, (float)sh.more[w]);
    // The block's groups in intervals of their exponents with its own base.  Bases are whole numbers, so another's intervals are these, shifted.
    const bool counting = r.T != 0.0 && (by_count || by_sum), here = is_finite(block_most) && c.holds(block_most);
    double block_sum = 0.0;
    if (counting) {
        const float M = c.base(block_most);
        block_sum = team_sum<T>(here && lane == 0 && most > -CUDART_INF_F ? sum * power(c.base(most) - M) : 0.0, sh);
        if (here)
            for (int g = 0; g < groups; ++g) {
                const int d = In::depth(c.exponent(lists.group[g * T + tid], M));
                atomicAdd(&lists.hist[d / In::kParts], 1u);
                if (!by_count) atomicAdd(&lists.parts[d / In::kParts], (uint32_t)(d % In::kParts));
            }
    }
    if (tid < at.blocks) at.of_block(sh.block_most, tid)[at.rank] = block_most, at.of_block(sh.block_sum, tid)[at.rank] = block_sum;
    at.sync();
    float m = sh.block_most[0];
    for (int b = 1; b < at.blocks; ++b) m = max_nan(m, sh.block_most[b]);
    const bool holds = is_finite(m) && c.holds(m);
    float bound = -CUDART_INF_F;
    if (counting && holds) {
        const float M = c.base(m);
        double S = 0.0;
        for (int b = 0; b < at.blocks; ++b)
            if (sh.block_most[b] > -CUDART_INF_F && c.holds(sh.block_most[b])) S += sh.block_sum[b] * power(c.base(sh.block_most[b]) - M);
        constexpr int per = kGroupBins / T;
        const double wanted = by_count ? (double)r.k : r.p * S * (1.0 + 1e-5);
        uint32_t count[per] = {}, parts[per] = {};
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
            if (b >= at.blocks) continue;
            const float down = sh.block_most[b] > -CUDART_INF_F && c.holds(sh.block_most[b]) ? M - c.base(sh.block_most[b]) : 64.0f;
            const int by = (int)fminf(down, 64.0f) * In::kPerOctave;
            const uint32_t *const hist = at.of_block(lists.hist, b), *const part = at.of_block(lists.parts, b);
#pragma unroll
            for (int q = 0; q < per; ++q) {
                const int from = tid * per + q - by;
                if (from < 0 || from >= kGroupBins - 1) continue;      // the last interval holds whatever is below
                count[q] += hist[from];
                if (!by_count) parts[q] += part[from];
            }
        }
        double part[per], mine = 0.0;
#pragma unroll
        for (int q = 0; q < per; ++q) {
            part[q] = by_count ? (double)count[q] : (double)In::sum_of(tid * per + q, count[q], parts[q]).least;
            mine += part[q];
        }
        double before = team_before<T>(mine, sh);
        set_all<T>(sh.lowest, kGroupBins - 1);
        if (before + mine >= wanted)
#pragma unroll
            for (int q = 0; q < per; ++q) {
                before += part[q];
                if (before >= wanted && before > 0.0) atomicMin(&sh.lowest, tid * per + q);   // one at least, if none is wanted
            }
        __syncthreads();
        // below every element of the interval
        const int b = sh.lowest;
        if (b < kGroupBins - 1) bound = fminf(__double2float_rd(((double)M - (b + 1.01) / In::kPerOctave) / c.c), m);
    }
    bool all_sizes = false;
    if (by_size && !(by_count && by_sum) && is_finite(m)) {
        const float q = below_min_p(r, m);
        if (q >= bound) bound = q, all_sizes = true;
    }
    const bool listing = r.T != 0.0 && holds && (bound > -CUDART_INF_F || a.vocab <= kListed);
    if (listing) {
        int* const listed = at.of_block(&sh.listed, 0);
        uint16_t* const hit = reinterpret_cast<uint16_t*>(lists.id);
        set_all<T>(sh.found, 0);
        for (int g = 0; g < groups; ++g) {
            const float l = lists.group[g * T + tid];
            if (!(l >= bound) || l == -CUDART_INF_F) continue;
            const int n = atomicAdd(&sh.found, 1);
            if (n < 2 * kListed) hit[n] = (uint16_t)(g * T + tid);
        }
        at.sync();                                             // the list takes the groups' place
        unsigned long long* const key = at.of_block(lists.key, 0);
        const int hits = sh.found, each = span * kUnroll;
        if (hits > kListed) {
            if (tid == 0) atomicAdd(listed, hits);             // there are no fewer elements than groups
        } else {
            for (int n = tid; n < hits * each; n += T) {
                const int h = hit[n / each], g = h / T, of = h % T, k = n % each;
                const int v = runs.begin(at.rank * (T / 32) + of / 32) + (g * each + k) * 32 + of % 32;
                if (v >= runs.end(at.rank * (T / 32) + of / 32)) continue;
                const Vector<E> in = x.load(v);
                if (!(in.max() >= bound)) continue;
                auto take = [&](float y, int id) {
                    if (!(y >= bound) || y == -CUDART_INF_F) return;
                    const int i = atomicAdd(listed, 1);
                    if (i < kListed) key[i] = key_of(y, id);
                };
#pragma unroll 1
                for (int i = 0; i < Vector<E>::N / 2; ++i) {
                    float y, z;
                    split(in.at(i), y, z);
                    take(y, x.first(v) + 2 * i), take(z, x.first(v) + 2 * i + 1);
                }
            }
        }
        at.sync();
    } else {
        at.sync();                                             // the blocks have read one another's counts
    }
    if (at.rank) return;
    const Total t = join_runs(sh, at.runs(), c);
    if (!is_finite(t.m)) {
        if (tid == 0) write_none(a, row, 0, t.m);
        return;
    }
    if (r.T == 0.0) {
        write_greedy<E, T>(a, row, x, t.m, sh);
        return;
    }
    int n = sh.listed;
    if (listing && n <= kListed && draw_from_list<E, T>(a, row, x, c, r, t, n, by_count, all_sizes, sh, lists)) return;
    bool counted = false;
    if (by_count || by_sum) {
        Search<E, T> search(x, c, t, sh, lists);
        search.template count<true>(unmasked(), by_sum);
        counted = true;
        if (by_count) {
            search.reach(r.k);
            by_count = sh.before_it + sh.listed >= r.k;        // otherwise fewer are not masked
        }
        if (holds && !by_count && by_sum) {
            const double S = t.S * exp2(-c.of_largest(t.m, t.M));
            search.bracket(r.p * S, 2.0 * Error(a.vocab, t.S, c).both() * S);
        }
        n = sh.before_it + sh.listed;
        if (holds && (by_count || by_sum) && n <= kListed) {
            const int hi = sh.highest;
            search.list(hi);
            if (draw_from_list<E, T>(a, row, x, c, r, t, n, by_count, false, sh, lists)) return;
            counted = false;
        }
        __syncthreads();
    }
    draw_from_many<E, T>(a, row, x, c, r, t, by_count, counted, sh, lists);
}

// ---- few tokens: L lanes have one each, and everything in 64 bits ----
template <class E, int L, bool kFilter>
__global__ void __launch_bounds__(256) narrow_kernel(SampleArgs a) {
    const int lane = threadIdx.x & 31, sub = lane % L;
    const int64_t row = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L;
    const bool real = row < a.rows;
    const Asked r = asked_of<kFilter>(a, real ? row : 0);
    const bool mine = real && sub < a.vocab && r.kind == 0;
    const float x = mine ? as_float(static_cast<const E*>(a.logits)[row * a.stride + sub]) : -CUDART_INF_F;
    float m = x;
#pragma unroll
    for (int o = L / 2; o; o >>= 1) m = max_nan(m, __shfl_xor_sync(~0u, m, o));
    const bool greedy = r.T == 0.0, ok = is_finite(m);
    const double z = ok && mine && x > -CUDART_INF_F ? ((double)x - (double)m) / (greedy ? 1.0 : r.T) : -CUDART_INF;
    double w = exp(z), S = w;
#pragma unroll
    for (int o = L / 2; o; o >>= 1) S += __shfl_xor_sync(~0u, S, o);
    bool keep = x > -CUDART_INF_F;
    // A warp has two rows, of which one may be greedy and the other not: all lanes take part in what lanes exchange.
    if (kFilter || __any_sync(~0u, greedy)) {
        // how many are before this one in the row's order, and their sum
        int rank = 0;
        double before = 0.0;
#pragma unroll
        for (int j = 0; j < L; ++j) {
            const float y = __shfl_sync(~0u, x, j, L);
            const double v = __shfl_sync(~0u, w, j, L);
            const bool earlier = y > x || (y == x && j < sub);
            rank += earlier;
            if (earlier) before += v;
        }
        if (kFilter) {
            const bool counts = keep && (r.k <= 0 || rank < r.k);
            double of = counts ? w : 0.0;
#pragma unroll
            for (int o = L / 2; o; o >>= 1) of += __shfl_xor_sync(~0u, of, o);
            keep = counts && (rank == 0 || ((r.p >= 1.0 || before < r.p * of) && w >= r.q));
        }
        if (greedy) keep = x > -CUDART_INF_F && rank == 0;
    }
    // the running sum by id; the last token before which it does not exceed the target
    double upto = keep ? w : 0.0;
#pragma unroll
    for (int o = 1; o < L; o <<= 1) {
        const double y = __shfl_up_sync(~0u, upto, o, L);
        if (sub >= o) upto += y;
    }
    const double C = __shfl_sync(~0u, upto, L - 1, L), previous = __shfl_up_sync(~0u, upto, 1, L), out = sub ? previous : 0.0;
    const unsigned int all = L == 32 ? ~0u : ((1u << (L & 31)) - 1) << (lane & ~(L - 1));
    const unsigned int here = __ballot_sync(~0u, keep && w > 0.0 && out <= r.u * C) & all;
    const unsigned int kept = __ballot_sync(~0u, keep) & all;
    if (!real) return;
    if (r.kind || !ok) {
        if (sub == 0) write_none(a, row, r.kind, m);
    } else if (here ? lane == 31 - __clz(here) : sub == 0) {
        if (greedy) write(a, row, sub, 0.0f, 0.0f, 1);
        else write(a, row, here ? sub : -1, (float)(z - log(S)), (float)(z - log(C)), __popc(kept));
    }
}

// ---- some tokens: a lane has N neighbouring ones, and everything in 64 bits ----
// The largest order o such that at(o), which falls, is `enough`.  The lowest `skip` bits of all orders are alike for each sign.
template <class F>
__device__ __forceinline__ uint32_t last_order(int skip, F&& enough) {
    uint32_t o = 0;
#pragma unroll 1
    for (int b = 31; b >= skip; --b)
        if (enough(o | 1u << b)) o |= 1u << b;
    return o;
}
template <class E, int N, bool kFilter>
__global__ void __launch_bounds__(128) middle_kernel(SampleArgs a) {
    __shared__ double table[kSteps];
    if (threadIdx.x < kSteps) table[threadIdx.x] = exp2(threadIdx.x / (double)kSteps);
    __syncthreads();
    const int lane = threadIdx.x & 31;
    const int64_t row = (int64_t)blockIdx.x * 4 + warp_index();
    if (row >= a.rows) return;
    const Asked r = asked_of<kFilter>(a, row);
    if (r.kind) {
        if (lane == 0) write_none(a, row, r.kind, 0.0f);
        return;
    }
    const E* const from = static_cast<const E*>(a.logits) + row * a.stride;
    float x[N], m = -CUDART_INF_F;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int i = lane * N + j;
        x[j] = i < a.vocab ? as_float(from[i]) : -CUDART_INF_F;
        m = max_nan(m, x[j]);
    }
    m = warp_max_nan(m);
    if (!is_finite(m)) {
        if (lane == 0) write_none(a, row, 0, m);
        return;
    }
    if (r.T == 0.0) {
        int first = 0x7FFFFFFF;
#pragma unroll
        for (int j = N - 1; j >= 0; --j)
            if (x[j] == m) first = lane * N + j;
        first = __reduce_min_sync(~0u, first);
        if (lane == 0) write(a, row, first, 0.0f, 0.0f, 1);
        return;
    }
    const Scale c(r.T);
    const Exact exact(m, c, table);
    double w[N], mine = 0.0;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        w[j] = exact.weight(x[j]);
        mine += w[j];
    }
    const double S = warp_sum(mine);
    double C = S;
    uint32_t in = 0;               // bit j: x[j] is kept
    int kept = 0;
    if (kFilter) {
        constexpr int kSkip = sizeof(E) == 4 ? 0 : std::is_same_v<E, __half> ? 13 : 16;
        uint32_t order[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            order[j] = x[j] > -CUDART_INF_F ? order_of(x[j]) : 0u;
            in |= (uint32_t)(x[j] > -CUDART_INF_F) << j;
        }
        // Only those above `o` stay, and of those equal to it the first `n` by id.
        auto keep = [&](uint32_t o, int n) {
            int equal = 0;
#pragma unroll
            for (int j = 0; j < N; ++j) equal += order[j] >> kSkip == o >> kSkip && (in >> j & 1);
            int rank = without_own(warp_before(equal));
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const bool same = order[j] >> kSkip == o >> kSkip && (in >> j & 1);
                if (order[j] >> kSkip < o >> kSkip || (same && rank >= n)) in &= ~(1u << j);
                rank += same;
            }
        };
        if (r.k > 0 && r.k < (int)__reduce_add_sync(~0u, __popc(in))) {
            auto at_least = [&](uint32_t o) {
                int n = 0;
#pragma unroll
                for (int j = 0; j < N; ++j) n += order[j] >= o;
                return (int)__reduce_add_sync(~0u, n);
            };
            const uint32_t o = last_order(kSkip, [&](uint32_t y) { return at_least(y) >= r.k; });
            keep(o, r.k - at_least(o + (1u << kSkip)));
        }
        if (r.p < 1.0) {
            auto sum_from = [&](uint32_t o) {
                double s = 0.0;
#pragma unroll
                for (int j = 0; j < N; ++j) s += order[j] >= o && (in >> j & 1) ? w[j] : 0.0;
                return warp_sum(s);
            };
            const double B = share_of(r.p, sum_from(0));
            // the row's largest, if none is wanted
            const uint32_t top = order_of(m) >> kSkip << kSkip;
            const uint32_t o = B > 0.0 ? last_order(kSkip, [&](uint32_t y) { return sum_from(y) >= B; }) : top;
            const uint32_t above = o + (1u << kSkip);
            const double A = sum_from(above), each = exact.weight(value_of(o | (o >> 31 ? 0u : (1u << kSkip) - 1)));
            keep(o, (int)fmin(fmax(ceil((B - A) / each), 1.0), 1e9));
        }
        if (r.q > 0.0)
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (w[j] < r.q) in &= ~(1u << j);
        mine = 0.0;
#pragma unroll
        for (int j = 0; j < N; ++j) mine += in >> j & 1 ? w[j] : 0.0;
        kept = __reduce_add_sync(~0u, __popc(in));
    } else {
        in = ~0u;
    }
    // by id: the last token that weighs before which the sum does not exceed the target
    const double upto = warp_before(mine), before = without_own(upto);
    if (kFilter) C = __shfl_sync(~0u, upto, 31);
    const double target = r.u * C;
    const unsigned int here = __ballot_sync(~0u, mine > 0.0 && before <= target);
    if (lane != 31 - __clz(here)) return;
    double sum = before;
    int token = 0;
    float at = m;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const double v = in >> j & 1 ? w[j] : 0.0;
        if (v > 0.0 && sum <= target) token = lane * N + j, at = x[j];
        sum += v;
    }
    const double z = ((double)at - (double)m) * c.exact * 0.6931471805599453;
    write(a, row, token, (float)(z - log(S)), (float)(z - log(C)), kept);
}

// ---- launches ----

template <class F>
int by_type(int type, F&& f) {
    cudaError_t e;
    if (type == SLAQ_F32) e = f(0.0f);
    else if (type == SLAQ_BF16) e = f(__nv_bfloat16());
    else e = f(__half());
    if (e != cudaSuccess) (void)cudaGetLastError();
    return e == cudaSuccess ? SLAQ_OK : SLAQ_E_CUDA;
}
constexpr size_t kMostShared = 100 * 1024;
template <class... Params, class... Args>
cudaError_t launch(void (*kernel)(Params...), int64_t blocks, int threads, size_t smem, int cluster, cudaStream_t st, Args... args) {
    if (smem > 40 * 1024) {   // what a kernel may use is state that all host threads share: never what this call needs, always the most
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostShared);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1] = {};
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}
constexpr int kSms = 148;

template <class E, int T>
cudaError_t launch_team(const SampleArgs& a, bool filter, int cluster, cudaStream_t st) {
    constexpr size_t smem = sizeof(Shared<T>) + sizeof(Lists<T>);
    static_assert(smem <= kMostShared);
    return filter ? launch(filter_kernel<E, T>, a.rows * cluster, T, smem, cluster, st, a) : launch(draw_kernel<E, T>, a.rows * cluster, T, 0, cluster, st, a);
}
template <class E, int N>
cudaError_t launch_middle(const SampleArgs& a, bool filter, cudaStream_t st) {
    return launch(filter ? middle_kernel<E, N, true> : middle_kernel<E, N, false>, (a.rows + 3) / 4, 128, 0, 1, st, a);
}
template <class E, bool kFilter>
cudaError_t launch_narrow(const SampleArgs& a, cudaStream_t st) {
    if (a.vocab <= 16) return launch(narrow_kernel<E, 16, kFilter>, (a.rows + 15) / 16, 256, 0, 1, st, a);
    return launch(narrow_kernel<E, 32, kFilter>, (a.rows + 7) / 8, 256, 0, 1, st, a);
}
// Up to 32 tokens have a lane each (200,000 x 10 fp32: 51 us, with a share 85; a block to a row 367 and 2,769), up to 1,024 a warp's registers (60,000 x 400
// bf16: 77 us, with a share 321; in blocks 129 and 1,893).  Beyond, with more rows than SMs, blocks of 256: four on an SM hide one another's
// ends.  512 x 65,536 bf16: top 40 28 us, the whole distribution 52; with 512 threads 41 and 42, with 128 30 and 94.  4,096 x 128,000: 270 and 269,
// with 512 threads 350 and 283, with 128 277 and 390.  Up to 2,048 vectors and for more than two rows an SM, blocks of 128, in which less waits for less: 20,000 x
// 5,000 bf16, whole, top 50 and a share of 0.9, 112, 355 and 1,018 us, with 256 threads 164, 538 and 1,118; 20,000 x 1,100 80, 343 and 695 (146, 526, 891).  At
// 6,000 x 16,000 71, 130 and 539 (75, 186, 525), but for flat rows, which keep most of their tokens, 73, 132 and 1,028 (77, 186, 722).  300 x 5,000: 16, 15 and 54
// (13, 17, 42).  With fewer rows a cluster shares one: 64 x 130,001 fp32 11 us, a block alone 15.
template <class E>
cudaError_t launch_sample(const SampleArgs& a, bool filter, cudaStream_t st) {
    if (a.vocab <= 32) return filter ? launch_narrow<E, true>(a, st) : launch_narrow<E, false>(a, st);
    if (a.vocab <= 64) return launch_middle<E, 2>(a, filter, st);
    if (a.vocab <= 128) return launch_middle<E, 4>(a, filter, st);
    if (a.vocab <= 256) return launch_middle<E, 8>(a, filter, st);
    if (a.vocab <= 512) return launch_middle<E, 16>(a, filter, st);
    if (a.vocab <= 1024) return launch_middle<E, 32>(a, filter, st);
    const int vectors = (a.vocab + 2 * (Vector<E>::N - 1)) / Vector<E>::N;
    if (vectors <= 2048 && a.rows > 2 * kSms) return launch_team<E, 128>(a, filter, 1, st);
    if (a.rows > kSms) return launch_team<E, 256>(a, filter, 1, st);
    int cluster = 1;
    while (cluster < kMaxCluster && a.rows * cluster * 2 <= kSms && vectors / (2 * cluster) >= 512) cluster *= 2;
    return launch_team<E, 512>(a, filter, cluster, st);
}

}  // namespace
}  // namespace slaq

extern "C" int slaq_sample_tokens(const void* d_logits, int type, int64_t rows, int32_t vocab, int64_t row_stride, const float* d_uniform,
                                  double temperature, const float* d_temperatures, int32_t top_k, const int32_t* d_top_ks, double top_p,
                                  const float* d_top_ps, double min_p, const float* d_min_ps, int64_t* d_out_token, float* d_out_logprob,
                                  float* d_out_kept_logprob, int32_t* d_out_kept, void* cuda_stream) {
    using namespace slaq;
    SampleArgs a = {d_logits, rows, row_stride, vocab, d_uniform, d_temperatures, d_top_ks, d_top_ps, d_min_ps, temperature, top_p, min_p, top_k,
                    d_out_token, d_out_logprob, d_out_kept_logprob, d_out_kept};
    if (type != SLAQ_F32 && type != SLAQ_BF16 && type != SLAQ_F16) return SLAQ_E_ARG;
    auto share = [](double x) { return x >= 0.0 && x <= 1.0; };
    if (rows < 0 || vocab < 1 || (!d_temperatures && temperature != 0.0 && !(temperature >= kLeastTemperature && temperature <= kMostTemperature)) ||
        (!d_top_ps && !share(top_p)) || (!d_min_ps && !share(min_p)))
        return SLAQ_E_ARG;
    if (vocab > kMaxVocab || rows > 0x7FFFFFFF) return SLAQ_E_RANGE;
    if (rows && (!d_logits || !d_uniform || !d_out_token || (rows > 1 && row_stride < 0))) return SLAQ_E_ARG;
    if (reinterpret_cast<uintptr_t>(d_logits) % (type == SLAQ_F32 ? 4 : 2) ||
        !aligned(d_uniform, d_temperatures, d_top_ks, d_top_ps, d_min_ps, d_out_token, d_out_logprob, d_out_kept_logprob, d_out_kept))
        return SLAQ_E_ARG;
    if (rows == 0) return SLAQ_OK;
    const bool filter = d_out_kept || d_top_ks || d_top_ps || d_min_ps || top_k > 0 || top_p < 1.0 || min_p > 0.0;
    return by_type(type, [&](auto e) { return launch_sample<decltype(e)>(a, filter, static_cast<cudaStream_t>(cuda_stream)); });
}
