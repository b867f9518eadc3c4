// Tokens drawn from rows of logits with given random numbers.
//
// A row x[0..V), temperature T, uniform u.  With m = max x: w_i = exp((x_i - m) / T).  The order of a row is that of falling x, equal ones by
// rising id.  Kept is a prefix of that order: of the first k (S_k their sum) the shortest whose sum reaches p S_k, as far as w_i >= q.  With C the
// sum over what is kept, the token is the first by id at which the running sum over the kept ones exceeds u C.
//
// The result is an integer, and in a large vocabulary the sums of 32-bit weights are off by more than many a token's weight.  So sums come with a
// bound of their error; where a decision lies within it, the row is summed up again in 64 bits.
#include "slaq_internal.cuh"
#include "slaq_rows.cuh"

namespace slaq {
namespace {

constexpr int kMaxVocab = 1 << 22;
constexpr float kMostTemperature = 1e30f, kLeastTemperature = 1e-30f;
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
    float temperature, top_p, min_p;
    int32_t top_k;
    int64_t* token;
    float *logprob, *kept_logprob;
    int32_t* kept;
};

// A row's numbers.
struct Asked {
    float u, T, p, q;
    int k;
    int kind;                      // 0: to be drawn; 1: nobody asked; 2: numbers out of range
};
template <bool kFilter>
__device__ __forceinline__ Asked asked_of(const SampleArgs& a, int64_t row) {
    Asked r;
    r.u = a.uniform[row];
    r.T = a.temperatures ? a.temperatures[row] : a.temperature;
    r.k = !kFilter ? 0 : a.top_ks ? a.top_ks[row] : a.top_k;
    r.p = !kFilter ? 1.0f : a.top_ps ? a.top_ps[row] : a.top_p;
    r.q = !kFilter ? 0.0f : a.min_ps ? a.min_ps[row] : a.min_p;
    const bool ok = r.u < 1.0f && (r.T == 0.0f || (r.T >= kLeastTemperature && r.T <= kMostTemperature)) && r.p >= 0.0f && r.p <= 1.0f && r.q >= 0.0f && r.q <= 1.0f;
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

// Weights in 32 bits: 2^(x c - M), M a whole number above m c, so that sums of other M are brought to this one exactly.  c comes in two
// parts, which leaves two roundings of the exponent t: an error of at most 2^-23 |t| ln 2 of a weight, beside the exponential's own 2^-22.
// Of the sum S of V weights 2^t the mean of |t| is at most log2(V / S) - the entropy of the shares is at most that of equal ones.  Beyond
// kMostExponent the parts of c are not enough.
constexpr float kMostExponent = 65536.0f;
struct Scale {
    float hi, lo;
    double c;                      // log2(e) / T
    __device__ __forceinline__ explicit Scale(float T) {
        c = 1.4426950408889634 / (double)T;
        hi = __double2float_rz(c);
        lo = fmaxf((float)(c - (double)hi), 1e-38f);        // above 0: a masked token is -inf, whichever way
    }
    __device__ __forceinline__ float base(float m) const { return m == -CUDART_INF_F ? 0.0f : ceilf(m * hi) + 1.0f; }
    __device__ __forceinline__ float exponent(float x, float M) const { return fmaf(x, lo, fmaf(x, hi, -M)); }
    __device__ __forceinline__ float weight(float x, float M) const { return exp2_fast(exponent(x, M)); }
    __device__ __forceinline__ bool holds(float m) const { return fabsf(m * hi) <= kMostExponent; }
    // of a sum of V weights, relative to it: 5 additions in 32 bits, the exponential, the exponents
    __device__ __forceinline__ double error(int V, double S) const { return 5.0 * 5.97e-8 + 2.4e-7 + 8.3e-8 * fmax(log2((double)V / S), 0.0); }
};
// .. and in 64 bits
struct Exact {
    double m, by;
    __device__ __forceinline__ Exact(float most, float T) : m(most), by(1.0 / (double)T) {}
    __device__ __forceinline__ double weight(float x) const { return exp(((double)x - m) * by); }
};
// 2^d for a whole number d <= 0, exactly; 0 far below
__device__ __forceinline__ double power(float d) { return d > -1000.0f ? __hiloint2double((1023 + (int)d) << 20, 0) : 0.0; }

// Kept are the elements above `value`, and those equal to it up to id `last`.
struct Cut {
    float value;
    uint32_t last;
    __device__ __forceinline__ bool keeps(float x, int i) const { return x > value || (x == value && (uint32_t)i <= last && x > -CUDART_INF_F); }
};

__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(~0u, x, o);
    return x;
}
template <class T>
__device__ __forceinline__ T warp_before(T x) {      // inclusive prefix
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const T y = __shfl_up_sync(~0u, x, o);
        if (lane >= o) x += y;
    }
    return x;
}

// f(vectors, number of the first) for the row's vectors [begin, end), a warp's lanes side by side; what is not in the row is -inf.
template <class E, class F>
__device__ __forceinline__ void over_vectors(const Row<E>& x, int begin, int end, F&& f) {
    const int lane = threadIdx.x & 31;
    for (int v = begin; v < end; v += 32 * kUnroll) {
        Vector<E> in[kUnroll];
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
// .. element by element: f(element, id)
template <class E, class F>
__device__ __forceinline__ void over_elements(const Row<E>& x, int begin, int end, F&& f) {
    over_vectors(x, begin, end, [&](const Vector<E>(&in)[kUnroll], int v) {
#pragma unroll
        for (int k = 0; k < kUnroll; ++k)
#pragma unroll
            for (int e = 0; e < Vector<E>::N; ++e) f(in[k].one(e), x.first(v + k * 32) + e);
    });
}

// The part of a row's vectors that a warp of T / 32 takes: neighbours, so that the warps' sums are those of runs of ids.
template <int T>
struct Runs {
    int per;
    __device__ __forceinline__ explicit Runs(int vectors) : per(((vectors + T / 32 - 1) / (T / 32) + 31) / 32 * 32) {}
    __device__ __forceinline__ int begin(int w) const { return w * per; }
    __device__ __forceinline__ int end(int w, int vectors) const { return min((w + 1) * per, vectors); }
};

constexpr int kBins = 4096;        // of a histogram
constexpr int kListed = 2048;      // elements that are sorted at most

template <int T>
struct Block {
    float most[T / 32];
    double sum[T / 32], more[T / 32];
    int count[T / 32];
    int found, listed, lowest, highest, before_it;
    double before, after;
    uint32_t key_low, key_high;
};
struct Lists {                     // of the kernel with filters, behind its Block
    union {
        uint32_t hist[kBins];
        double weight[kListed];
    };
    unsigned long long key[kListed];
};

template <int T>
__device__ __forceinline__ double block_sum(double x, Block<T>& sh) {
    x = warp_sum(x);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh.more[threadIdx.x >> 5] = x;
    __syncthreads();
    x = 0.0;
    for (int w = 0; w < T / 32; ++w) x += sh.more[w];
    return x;
}
// what the threads before this one have, and in `all` what all have
template <int T>
__device__ __forceinline__ double block_before(double x, Block<T>& sh, double& all) {
    const double in = warp_before(x);
    __syncthreads();
    if ((threadIdx.x & 31) == 31) sh.more[threadIdx.x >> 5] = in;
    __syncthreads();
    double before = 0.0;
    all = 0.0;
    for (int w = 0; w < T / 32; ++w) {
        if (w < (int)(threadIdx.x >> 5)) before += sh.more[w];
        all += sh.more[w];
    }
    return before + (in - x);
}
template <int T>
__device__ __forceinline__ int block_before(int x, Block<T>& sh) {
    const int in = warp_before(x);
    __syncthreads();
    if ((threadIdx.x & 31) == 31) sh.count[threadIdx.x >> 5] = in;
    __syncthreads();
    int before = in - x;
    for (int w = 0; w < (int)(threadIdx.x >> 5); ++w) before += sh.count[w];
    return before;
}
// sh.<place> set to `value` for all; a barrier on both sides
template <class S, class V>
__device__ __forceinline__ void set_all(S& place, V value) {
    __syncthreads();
    if (threadIdx.x == 0) place = value;
    __syncthreads();
}

// The row's largest element m, its base M, the sum S, and in sh.sum those of the warps' runs, all in 32-bit weights.
struct Total {
    float m, M;
    double S;
};
template <class E, int T>
__device__ __forceinline__ Total sums_of_row(const Row<E>& x, const Scale& c, Block<T>& sh) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Runs<T> runs(x.vectors);
    float m = -CUDART_INF_F, M = 0.0f;
    double s = 0.0;
    over_vectors(x, runs.begin(warp), runs.end(warp, x.vectors), [&](const Vector<E>(&in)[kUnroll], int) {
        float most = in[0].max();
#pragma unroll
        for (int k = 1; k < kUnroll; ++k) most = max_nan(most, in[k].max());
        if (!(most <= m)) {
            const float higher = c.base(most);
            s = m == -CUDART_INF_F ? 0.0 : s * power(M - higher);
            m = max_nan(m, most);
            M = higher;
        }
        const Pair off = pair_of(-M, -M), hi = pair_of(c.hi, c.hi), lo = pair_of(c.lo, c.lo);
        Pair sum[kUnroll];
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
            constexpr int P = Vector<E>::N / 2;
            Pair e[P];
#pragma unroll
            for (int i = 0; i < P; ++i) {
                float a, b;
                split(fma2(in[k].at(i), lo, fma2(in[k].at(i), hi, off)), a, b);
                e[i] = pair_of(exp2_fast(a), exp2_fast(b));
            }
            sum[k] = e[0] + e[1];
            if constexpr (P == 4) sum[k] = sum[k] + (e[2] + e[3]);
        }
        float a, b;
        split((sum[0] + sum[1]) + (sum[2] + sum[3]), a, b);
        s += (double)(a + b);
    });
    const float most = warp_max_nan(m);
    if (lane == 0) sh.most[warp] = most;
    __syncthreads();
    Total t = {sh.most[0], 0.0f, 0.0};
#pragma unroll
    for (int w = 1; w < T / 32; ++w) t.m = max_nan(t.m, sh.most[w]);
    t.M = c.base(t.m);
    s = warp_sum(m == -CUDART_INF_F ? 0.0 : s * power(M - t.M));
    if (lane == 0) sh.sum[warp] = s;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < T / 32; ++w) t.S += sh.sum[w];
    return t;
}
// .. in 64-bit weights, of what is kept; the number of those
template <class E, int T>
__device__ __noinline__ double exact_sums(const Row<E>& x, const Exact& w, const Cut& cut, Block<T>& sh, int& kept) {
    const int warp = threadIdx.x >> 5;
    const Runs<T> runs(x.vectors);
    double s = 0.0;
    int n = 0;
    over_elements(x, runs.begin(warp), runs.end(warp, x.vectors), [&](float y, int i) {
        if (cut.keeps(y, i)) {
            s += w.weight(y);
            ++n;
        }
    });
    s = warp_sum(s);
    n = __reduce_add_sync(~0u, n);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh.sum[warp] = s, sh.count[warp] = n;
    __syncthreads();
    s = 0.0;
    kept = 0;
    for (int k = 0; k < T / 32; ++k) s += sh.sum[k], kept += sh.count[k];
    return s;
}

// The first element at which the running sum exceeds `target`: the run by sh.sum, then the threads' parts of that run.  sh.found is the
// element, or -1, and sh.before and sh.after are the sums on its two sides.
template <class E, int T, class Weight>
__device__ __forceinline__ void find(const Row<E>& x, double target, Block<T>& sh, Weight&& weight) {
    const Runs<T> runs(x.vectors);
    int run = 0;
    double before = 0.0;
    for (; run < T / 32 - 1 && before + sh.sum[run] <= target; ++run) before += sh.sum[run];
    set_all(sh.found, -1);
    const int begin = runs.begin(run), end = runs.end(run, x.vectors), per = (end - begin + T - 1) / T;
    const int mine = begin + (int)threadIdx.x * per, stop = min(mine + per, end);
    double s = 0.0;
    int last = -1;
    auto walk = [&](auto&& f) {
        for (int v = mine; v < stop; ++v) {
            const Vector<E> in = x.load(v);
#pragma unroll
            for (int e = 0; e < Vector<E>::N; ++e) f(in.one(e), x.first(v) + e);
        }
    };
    walk([&](float y, int i) {
        const double w = weight(y, i);
        s += w;
        if (w > 0.0) last = i;
    });
    double all;
    const double from = before + block_before<T>(s, sh, all);
    if (from <= target && target < from + s) {
        double sum = from;
        int at = -1;
        walk([&](float y, int i) {
            const double w = weight(y, i);
            if (at < 0 || sum <= target) {               // the last of them, where roundings leave no other
                if (w > 0.0) at = i, sh.before = sum, sh.after = sum + w;
                sum += w;
            }
        });
        sh.found = at;
    }
    __syncthreads();
    if (sh.found < 0) {                                  // between two threads' sums, by rounding: the last that weighs
        __syncthreads();
        if (last >= 0 && from <= target) atomicMax(&sh.found, last);
        if (threadIdx.x == 0) sh.before = sh.after = target;
        __syncthreads();
    }
}

// Drawn from what is kept, the row's own order, in 64 bits.  S: the sum over the whole row.
struct Drawn {
    int token;
    double logprob, kept_logprob;
};
template <class E, int T>
__device__ __noinline__ Drawn draw_exactly(const Row<E>& x, float m, float Temp, float u, Cut cut, double S, Block<T>& sh, int& kept) {
    const Exact w(m, Temp);
    const double C = exact_sums<E, T>(x, w, cut, sh, kept);
    if (S <= 0.0) S = C;
    find<E, T>(x, u * C, sh, [&](float y, int i) { return cut.keeps(y, i) ? w.weight(y) : 0.0; });
    Drawn d = {sh.found, 0.0, 0.0};
    const double z = d.token < 0 ? 0.0 : ((double)as_float(x.x[d.token]) - w.m) * w.by;
    d.logprob = z - log(S), d.kept_logprob = z - log(C);
    return d;
}

template <class E, int T>
__device__ __forceinline__ void write_greedy(const SampleArgs& a, int64_t row, const Row<E>& x, float m, Block<T>& sh) {
    set_all(sh.found, 0x7FFFFFFF);
    const Runs<T> runs(x.vectors);
    const int warp = threadIdx.x >> 5;
    int first = 0x7FFFFFFF;
    over_vectors(x, runs.begin(warp), runs.end(warp, x.vectors), [&](const Vector<E>(&in)[kUnroll], int v) {
#pragma unroll
        for (int k = 0; k < kUnroll; ++k)
            if (in[k].max() == m)
#pragma unroll
                for (int e = 0; e < Vector<E>::N; ++e)
                    if (in[k].one(e) == m) first = min(first, x.first(v + k * 32) + e);
    });
    if (first != 0x7FFFFFFF) atomicMin(&sh.found, first);
    __syncthreads();
    if (threadIdx.x == 0) write(a, row, sh.found, 0.0f, 0.0f, 1);
}

// ---- the whole distribution ----
template <class E, int T>
__global__ void __launch_bounds__(T) draw_kernel(SampleArgs a) {
    __shared__ Block<T> sh;
    const int64_t row = blockIdx.x;
    const Asked r = asked_of<false>(a, row);
    if (r.kind) {
        if (threadIdx.x == 0) write_none(a, row, r.kind, 0.0f);
        return;
    }
    const Row<E> x(static_cast<const E*>(a.logits) + row * a.stride, a.vocab);
    const Scale c(r.T == 0.0f ? 1.0f : r.T);
    const Total t = sums_of_row<E, T>(x, c, sh);
    if (!is_finite(t.m)) {
        if (threadIdx.x == 0) write_none(a, row, 0, t.m);
        return;
    }
    if (r.T == 0.0f) {
        write_greedy<E, T>(a, row, x, t.m, sh);
        return;
    }
    if (c.holds(t.m)) {
        const double target = r.u * t.S, margin = c.error(a.vocab, t.S) * t.S;
        find<E, T>(x, target, sh, [&](float y, int) { return (double)c.weight(y, t.M); });
        const int token = sh.found;
        if (token >= 0 && target - sh.before >= margin && sh.after - target >= margin) {
            if (threadIdx.x == 0) {
                const float logprob = (float)(((double)as_float(x.x[token]) * c.c - t.M - log2(t.S)) * 0.6931471805599453);
                write(a, row, token, logprob, logprob, 0);
            }
            return;
        }
        __syncthreads();
    }
    int kept;
    const Drawn d = draw_exactly<E, T>(x, t.m, r.T, r.u, Cut{-CUDART_INF_F, 0}, 0.0, sh, kept);
    if (threadIdx.x == 0) write(a, row, d.token, (float)d.logprob, (float)d.logprob, 0);
}

// ---- what is kept ----

// Keys fall from list[0] to list[n - 1]; n <= kListed.
template <int T>
__device__ __forceinline__ void sort_list(unsigned long long* list, int n) {
    int size = 32;
    while (size < n) size *= 2;
    for (int i = n + threadIdx.x; i < size; i += T) list[i] = 0;
    for (int k = 2; k <= size; k *= 2)
        for (int j = k / 2; j; j /= 2) {
            __syncthreads();
            for (int i = threadIdx.x; i < size / 2; i += T) {
                const int p = 2 * i - (i & (j - 1)), q = p + j;
                const unsigned long long x = list[p], y = list[q];
                if ((x < y) == !(p & k)) list[p] = y, list[q] = x;
            }
        }
    __syncthreads();
}

// Looks for the border of what is kept.
//
// The row's elements are counted in intervals of 1/64 of an octave of their weight, from the largest down.  The counts bound the running sum
// over the order from both sides, within 1.1 % of what lies above or below; so the border lies in few intervals.  The elements that
// may be kept, or, where those are too many, the ones of the intervals in question, are listed and sorted.  What is still too many for
// that is halved at the middle of their values, as often as it takes; if all are equal, the border is a matter of their ids.
template <class E, int T>
struct Search {
    const Row<E>& x;
    const Scale& c;
    const Exact w;
    const float M;
    const bool holds;
    const double shift;            // log2 of the 64-bit weight of what weighs 1 with base M
    Block<T>& sh;
    Lists& lists;
    int begin, end;                // the warp's run

    __device__ __forceinline__ Search(const Row<E>& x, const Scale& c, float Temp, const Total& t, Block<T>& sh, Lists& lists)
        : x(x), c(c), w(t.m, Temp), M(t.M), holds(c.holds(t.m)), shift(holds ? t.M - (double)t.m * c.c : 0.0), sh(sh), lists(lists) {
        const Runs<T> runs(x.vectors);
        begin = runs.begin(threadIdx.x >> 5), end = runs.end(threadIdx.x >> 5, x.vectors);
    }
    // Falls with the value, masked ones last.
    __device__ __forceinline__ int bin(float y) const {
        const float t = holds ? c.exponent(y, M) : (float)(((double)y - w.m) * c.c);
        return (int)fminf(t * -64.0f, kBins - 1.0f);
    }
    // bounds of the weight in interval b, with base M; the exponents' roundings, 2^-17 at 64, and the exponential's included
    static __device__ __forceinline__ float most(int b) { return exp2_fast(b * -0.015625f) * 1.00004f; }
    static __device__ __forceinline__ float least(int b) { return b == kBins - 1 ? 0.0f : exp2_fast((b + 1) * -0.015625f) * 0.99996f; }

    __device__ __forceinline__ void count(const Cut& in) {
        __syncthreads();
        for (int b = threadIdx.x; b < kBins; b += T) lists.hist[b] = 0;
        __syncthreads();
        over_elements(x, begin, end, [&](float y, int i) {
            if (in.keeps(y, i)) atomicAdd(&lists.hist[bin(y)], 1u);
        });
        __syncthreads();
    }
    // The first interval up to which there are n elements (sh.highest), how many there are before it (sh.before_it) and in it (sh.listed);
    // without so many, the last one.
    __device__ __forceinline__ void reach(int n) {
        constexpr int per = kBins / T;
        const int b0 = threadIdx.x * per;
        int mine = 0;
        for (int b = b0; b < b0 + per; ++b) mine += lists.hist[b];
        int sum = block_before<T>(mine, sh);
        if (sum < n && (sum + mine >= n || threadIdx.x == T - 1)) {
            int b = b0;
            for (; b < b0 + per - 1 && sum + (int)lists.hist[b] < n; ++b) sum += lists.hist[b];
            sh.lowest = sh.highest = b, sh.before_it = sum, sh.listed = lists.hist[b];
        }
        __syncthreads();
    }
    // The intervals sh.lowest to sh.highest in which the running sum reaches B; the elements before and in them.  B and S, the sum of all, with
    // base M, S to `slack` of itself.
    __device__ __forceinline__ void bracket(double B, double S, double slack) {
        constexpr int per = kBins / T;
        const int b0 = threadIdx.x * per;
        double hi = 0.0, lo = 0.0, all_hi, all_lo;
        for (int b = b0; b < b0 + per; ++b) hi += (double)lists.hist[b] * most(b), lo += (double)lists.hist[b] * least(b);
        double sum_hi = block_before<T>(hi, sh, all_hi), sum_lo = block_before<T>(lo, sh, all_lo);
        if (threadIdx.x == 0) sh.lowest = sh.highest = kBins - 1;
        __syncthreads();
        const double least_B = B - S * slack, most_B = B + S * slack;
        for (int b = b0; b < b0 + per; ++b) {
            const double h = lists.hist[b];
            sum_hi += h * most(b), sum_lo += h * least(b);
            if (sum_hi >= least_B) atomicMin(&sh.lowest, b);
            if (fmax(sum_lo, S * (1.0 - slack) - fmax(all_hi - sum_hi, 0.0) * (1.0 + 1e-12) - all_hi * 1e-14) >= most_B) atomicMin(&sh.highest, b);
        }
        __syncthreads();
        int before = 0, inside = 0;
        const int first = min(sh.lowest, sh.highest), last = sh.highest;
        for (int b = b0; b < b0 + per; ++b) (b < first ? before : inside) += b <= last ? lists.hist[b] : 0;
        const double all_before = block_sum<T>((double)before, sh), all_inside = block_sum<T>((double)inside, sh);
        if (threadIdx.x == 0) sh.lowest = first, sh.before_it = (int)all_before, sh.listed = (int)all_inside;
        __syncthreads();
    }

    // f(element, id) for the elements of `in` from interval lo to hi
    template <class F>
    __device__ __forceinline__ void over_bins(const Cut& in, int lo, int hi, F&& f) {
        over_vectors(x, begin, end, [&](const Vector<E>(&v)[kUnroll], int at) {
#pragma unroll
            for (int k = 0; k < kUnroll; ++k) {
                if (bin(v[k].max()) > hi) continue;
#pragma unroll
                for (int e = 0; e < Vector<E>::N; ++e) {
                    const float y = v[k].one(e);
                    const int i = x.first(at + k * 32) + e, b = bin(y);
                    if (in.keeps(y, i) && b >= lo && b <= hi) f(y, i);
                }
            }
        });
    }
    __device__ __forceinline__ void append(float y, int i) {
        const int n = atomicAdd(&sh.listed, 1);
        if (n < kListed) lists.key[n] = key_of(y, i);
    }
    // .. listed and sorted: how many there are, at most kListed
    __device__ __forceinline__ int list(const Cut& in, int lo, int hi) {
        set_all(sh.listed, 0);
        over_bins(in, lo, hi, [&](float y, int i) { append(y, i); });
        __syncthreads();
        const int n = min(sh.listed, kListed);
        sort_list<T>(lists.key, n);
        return n;
    }
    __device__ __forceinline__ float value(int i) const { return value_of((uint32_t)(lists.key[i] >> 32)); }
    __device__ __forceinline__ Cut cut_at(int i) const { return {value(i), position_of(lists.key[i])}; }
    __device__ __forceinline__ void weigh(int n) {
        for (int i = threadIdx.x; i < n; i += T) lists.weight[i] = w.weight(value(i));
        __syncthreads();
    }
    // The first of n places at which above + the running sum of lists.weight reaches B, or exceeds it; the last if none does.  sh.before and
    // sh.after: the sums on its two sides.
    template <bool kExceeds>
    __device__ __forceinline__ int reach_in_list(int n, double above, double B) {
        const int per = (n + T - 1) / T, i0 = min((int)threadIdx.x * per, n), i1 = min(i0 + per, n);
        double mine = 0.0, all;
        for (int i = i0; i < i1; ++i) mine += lists.weight[i];
        const double from = above + block_before<T>(mine, sh, all);
        set_all(sh.found, n - 1);
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

    // The border in intervals sh.lowest to sh.highest: of the first k elements (k > 0), or of those whose sum reaches B in 64-bit weights.
    __device__ __noinline__ Cut border(const Cut& in, int k, double B) {
        const int lo = sh.lowest, hi = sh.highest;
        int above = sh.before_it, n = sh.listed;
        __syncthreads();
        // what lies above, and the range of what is in question
        double A = 0.0;
        if (k == 0) {
            if (lo > 0) over_bins(in, 0, lo - 1, [&](float y, int) { A += w.weight(y); });
            A = block_sum<T>(A, sh);
        }
        if (n > kListed) {
            if (threadIdx.x == 0) sh.key_low = 0xFFFFFFFFu, sh.key_high = 0;
            __syncthreads();
            uint32_t low = 0xFFFFFFFFu, high = 0;
            over_bins(in, lo, hi, [&](float y, int) { low = min(low, order_of(y)), high = max(high, order_of(y)); });
            atomicMin(&sh.key_low, low), atomicMax(&sh.key_high, high);
            __syncthreads();
            uint32_t bottom = sh.key_low, top = sh.key_high;
            while (n > kListed && bottom < top) {
                const uint32_t middle = bottom + (top - bottom) / 2;       // the upper half: above it
                double s = 0.0;
                int upper = 0;
                low = 0xFFFFFFFFu, high = 0;
                over_elements(x, begin, end, [&](float y, int i) {
                    const uint32_t o = order_of(y);
                    if (o < bottom || o > top || !in.keeps(y, i)) return;
                    if (o > middle) {
                        ++upper;
                        low = min(low, o);
                        if (k == 0) s += w.weight(y);
                    } else {
                        high = max(high, o);
                    }
                });
                const int uppers = (int)block_sum<T>((double)upper, sh);
                s = block_sum<T>(s, sh);
                if (threadIdx.x == 0) sh.key_low = 0xFFFFFFFFu, sh.key_high = 0;
                __syncthreads();
                atomicMin(&sh.key_low, low), atomicMax(&sh.key_high, high);
                __syncthreads();
                if (k ? above + uppers >= k : A + s >= B) bottom = sh.key_low, n = uppers;
                else top = sh.key_high, above += uppers, n -= uppers, A += s;
            }
            if (bottom == top) {
                // all equal: the border is the id of the last one that is kept
                const float v = value_of(top);
                const double each = w.weight(v);
                const int wanted = k ? k - above : (int)fmin(fmax(ceil((B - A) / each), 1.0), (double)n);
                int mine = 0;
                over_elements(x, begin, end, [&](float y, int i) { mine += y == v && in.keeps(y, i); });
                mine = __reduce_add_sync(~0u, mine);
                __syncthreads();
                if ((threadIdx.x & 31) == 0) sh.count[threadIdx.x >> 5] = mine;
                set_all(sh.found, 0);
                int before = 0;
                for (int r = 0; r < (int)(threadIdx.x >> 5); ++r) before += sh.count[r];
                if (before < wanted && before + mine >= wanted)            // in this warp's run
                    for (int v0 = begin; v0 < end && before < wanted; v0 += 32) {
                        const int at = v0 + (threadIdx.x & 31);
                        const Vector<E> in_v = at < end ? x.load(at) : Row<E>::nothing();
                        auto is = [&](int e) { return in_v.one(e) == v && in.keeps(v, x.first(at) + e); };
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
            set_all(sh.listed, 0);
            over_elements(x, begin, end, [&](float y, int i) {
                const uint32_t o = order_of(y);
                if (o >= bottom && o <= top && in.keeps(y, i)) append(y, i);
            });
            __syncthreads();
            n = min(sh.listed, kListed);
            sort_list<T>(lists.key, n);
        } else {
            n = list(in, lo, hi);
        }
        if (k) return cut_at(min(k - above, n) - 1);
        weigh(n);
        return cut_at(reach_in_list<false>(n, A, B));
    }
};

__device__ __forceinline__ Cut tighter(const Cut& a, const Cut& b) {
    return a.value > b.value || (a.value == b.value && a.last < b.last) ? a : b;
}

// ---- with filters ----
template <class E, int T>
__global__ void __launch_bounds__(T) filter_kernel(SampleArgs a) {
    __shared__ Block<T> sh;
    extern __shared__ uint4 dynamic[];
    Lists& lists = *reinterpret_cast<Lists*>(dynamic);
    const int64_t row = blockIdx.x;
    const Asked r = asked_of<true>(a, row);
    if (r.kind) {
        if (threadIdx.x == 0) write_none(a, row, r.kind, 0.0f);
        return;
    }
    const Row<E> x(static_cast<const E*>(a.logits) + row * a.stride, a.vocab);
    const Scale c(r.T == 0.0f ? 1.0f : r.T);
    const Total t = sums_of_row<E, T>(x, c, sh);
    if (!is_finite(t.m)) {
        if (threadIdx.x == 0) write_none(a, row, 0, t.m);
        return;
    }
    if (r.T == 0.0f) {
        write_greedy<E, T>(a, row, x, t.m, sh);
        return;
    }
    Search<E, T> search(x, c, r.T, t, sh, lists);
    const Exact& w = search.w;
    const Cut all = {-CUDART_INF_F, 0};
    const bool by_sum = r.p < 1.0f, by_size = r.q > 0.0f;
    bool by_count = r.k > 0 && r.k < a.vocab;
    // the sum over the whole row in 64-bit weights, to `slack` of itself
    double S = search.holds ? t.S * exp2(search.shift) : 0.0, slack = search.holds ? c.error(a.vocab, t.S) : 0.0;
    int everything;
    if (!search.holds) S = exact_sums<E, T>(x, w, all, sh, everything);
    int n = 0;                         // what is listed, if that is all that may be kept
    if (a.vocab <= kListed) {
        n = search.list(all, 0, kBins - 1);
    } else {
        search.count(all);
        int hi = -1;
        if (by_count) {
            search.reach(r.k);
            if (sh.before_it + sh.listed < r.k) by_count = false;         // fewer are not masked
            else hi = sh.highest;
        }
        if (!by_count) {
            if (by_sum) {
                search.bracket(r.p * S * exp2(-search.shift), S * exp2(-search.shift), slack + 1e-12);
                hi = sh.highest;
            }
            if (by_size) {
                const int b = search.bin(__double2float_rd((double)t.m + (double)r.T * log((double)r.q))) + 1;
                if (hi < 0 || b < hi) hi = min(b, kBins - 1);
            }
        }
        if (hi >= 0) {
            int mine = 0;
            for (int b = threadIdx.x; b <= hi; b += T) mine += lists.hist[b];
            const int up_to = (int)block_sum<T>((double)mine, sh);
            if (up_to <= kListed) n = search.list(all, 0, hi);
        }
    }
    if (n > 0) {
        // the list holds all that may be kept
        search.weigh(n);
        const int K = by_count ? min(r.k, n) : n;
        int L = K;
        if (by_sum) {
            double of = S;
            if (by_count || a.vocab <= kListed) {
                double mine = 0.0;
                for (int i = threadIdx.x; i < K; i += T) mine += lists.weight[i];
                of = block_sum<T>(mine, sh);
            }
            L = search.template reach_in_list<false>(K, 0.0, r.p * of) + 1;
            const double near = of * slack;
            if (!by_count && a.vocab > kListed && slack > 0.0 && (r.p * of - sh.before < near || sh.after - r.p * of < near)) {
                S = exact_sums<E, T>(x, w, all, sh, everything);
                slack = 0.0;
                L = search.template reach_in_list<false>(K, 0.0, r.p * S) + 1;
            }
        }
        if (by_size) {
            set_all(sh.found, L);
            for (int i = threadIdx.x; i < L; i += T)
                if (lists.weight[i] < r.q) {
                    atomicMin(&sh.found, i);
                    break;
                }
            __syncthreads();
            L = max(sh.found, 1);
        }
        double mine = 0.0;
        for (int i = threadIdx.x; i < L; i += T) mine += lists.weight[i];
        const double C = block_sum<T>(mine, sh);
        if (a.vocab <= kListed) {
            double rest = 0.0;
            for (int i = L + threadIdx.x; i < n; i += T) rest += lists.weight[i];
            S = C + block_sum<T>(rest, sh);
        }
        // by id: the weights go with them
        __syncthreads();
        for (int i = threadIdx.x; i < L; i += T) lists.key[i] = (unsigned long long)(0xFFFFFFFFu - position_of(lists.key[i])) << 32 | (uint32_t)i;
        sort_list<T>(lists.key, L);
        double by_id[kListed / T];
#pragma unroll
        for (int j = 0; j < kListed / T; ++j) by_id[j] = j * T + threadIdx.x < L ? lists.weight[(uint32_t)lists.key[j * T + threadIdx.x]] : 0.0;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kListed / T; ++j)
            if (j * T + threadIdx.x < L) lists.weight[j * T + threadIdx.x] = by_id[j];
        __syncthreads();
        int at = search.template reach_in_list<true>(L, 0.0, r.u * C);
        if (threadIdx.x == 0) {
            while (at > 0 && lists.weight[at] == 0.0) --at;
            const int token = (int)(0xFFFFFFFFu - (uint32_t)(lists.key[at] >> 32));
            const double z = ((double)as_float(x.x[token]) - w.m) * w.by;
            write(a, row, token, (float)(z - log(S)), (float)(z - log(C)), L);
        }
        return;
    }
    // too many for a list
    Cut cut = all;
    if (by_count) {
        search.reach(r.k);
        cut = search.border(all, r.k, 0.0);
    }
    if (by_sum) {
        int kept;
        const double of = exact_sums<E, T>(x, w, cut, sh, kept);
        if (!by_count) S = of;
        search.count(cut);
        const double unit = exp2(-search.shift);
        search.bracket(r.p * of * unit, of * unit, 1e-12);
        cut = tighter(cut, search.border(cut, 0, r.p * of));
    }
    if (by_size) {
        float f = __double2float_ru((double)t.m + (double)r.T * log((double)r.q));
        if (w.weight(f) < r.q) f = nextafterf(f, CUDART_INF_F);
        else if (w.weight(nextafterf(f, -CUDART_INF_F)) >= r.q) f = nextafterf(f, -CUDART_INF_F);
        cut = tighter(cut, Cut{fminf(f, t.m), 0xFFFFFFFFu});
    }
    int kept;
    const Drawn d = draw_exactly<E, T>(x, t.m, r.T, r.u, cut, S, sh, kept);
    if (threadIdx.x == 0) write(a, row, d.token, (float)d.logprob, (float)d.kept_logprob, kept);
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
template <class... Params, class... Args>
cudaError_t launch(void (*kernel)(Params...), int64_t blocks, int threads, size_t smem, cudaStream_t st, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}
static_assert(sizeof(Lists) + sizeof(Block<512>) <= 48 * 1024, "more shared memory than a kernel may use unasked");

template <class E>
cudaError_t launch_sample(const SampleArgs& a, bool filter, cudaStream_t st) {
    if (!filter) {
        if (a.vocab <= 4096) return launch(draw_kernel<E, 64>, a.rows, 64, 0, st, a);
        return launch(draw_kernel<E, 256>, a.rows, 256, 0, st, a);
    }
    if (a.vocab <= kListed) return launch(filter_kernel<E, 128>, a.rows, 128, sizeof(Lists), st, a);
    return launch(filter_kernel<E, 512>, a.rows, 512, sizeof(Lists), st, a);
}

}  // namespace
}  // namespace slaq

extern "C" int slaq_sample_tokens(const void* d_logits, int type, int64_t rows, int32_t vocab, int64_t row_stride, const float* d_uniform,
                                  float temperature, const float* d_temperatures, int32_t top_k, const int32_t* d_top_ks, float top_p,
                                  const float* d_top_ps, float min_p, const float* d_min_ps, int64_t* d_out_token, float* d_out_logprob,
                                  float* d_out_kept_logprob, int32_t* d_out_kept, void* cuda_stream) {
    using namespace slaq;
    SampleArgs a = {d_logits, rows, row_stride, vocab, d_uniform, d_temperatures, d_top_ks, d_top_ps, d_min_ps, temperature, top_p, min_p, top_k,
                    d_out_token, d_out_logprob, d_out_kept_logprob, d_out_kept};
    if (type != SLAQ_F32 && type != SLAQ_BF16 && type != SLAQ_F16) return SLAQ_E_ARG;
    auto share = [](float x) { return x >= 0.0f && x <= 1.0f; };
    if (rows < 0 || vocab < 1 || (!d_temperatures && temperature != 0.0f && !(temperature >= kLeastTemperature && temperature <= kMostTemperature)) ||
        (!d_top_ps && !share(top_p)) || (!d_min_ps && !share(min_p)))
        return SLAQ_E_ARG;
    if (vocab > kMaxVocab || rows > 0x7FFFFFFF) return SLAQ_E_RANGE;
    if (rows && (!d_logits || !d_uniform || !d_out_token || (rows > 1 && row_stride < 0))) return SLAQ_E_ARG;
    if (reinterpret_cast<uintptr_t>(d_logits) % (type == SLAQ_F32 ? 4 : 2) ||
        !aligned(d_uniform, d_temperatures, d_top_ks, d_top_ps, d_min_ps, d_out_token, d_out_logprob, d_out_kept_logprob, d_out_kept))
        return SLAQ_E_ARG;
    if (rows == 0) return SLAQ_OK;
    const bool filter = d_out_kept || d_top_ks || d_top_ps || d_min_ps || top_k > 0 || top_p < 1.0f || min_p > 0.0f;
    return by_type(type, [&](auto e) { return launch_sample<decltype(e)>(a, filter, static_cast<cudaStream_t>(cuda_stream)); });
}
