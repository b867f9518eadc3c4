// Log probabilities of given tokens with the entropy and the top alternatives of their rows, and their gradient.
//
// A row x[0..V) of logits, scale c, token t.  With m = max x, d_i = c (x_i - m), S = sum exp d_i:
//     log probability  d_t - ln S          entropy  ln S - (sum exp(d_i) d_i) / S
// Both terms of the entropy are non-negative, so nothing cancels.  What a later gradient needs of the row is kept as (m, S)
// and not as m c + ln S: a sum near 20 would carry 1e-6 of rounding into every probability.
#include <cooperative_groups.h>

#include "slaq_internal.cuh"
#include "slaq_rows.cuh"

namespace cg = cooperative_groups;

namespace slaq {
namespace {

constexpr int kMaxVocab = 1 << 22;
constexpr int kMaxTop = 32;
constexpr float kMostScale = 1e30f;   // beyond, a scale times log2 e would not be finite
constexpr int kMaxCluster = 8;
constexpr int kUnroll = 4;         // vectors that a thread has in flight

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
    int32_t slice;                 // vectors per block of a cluster
};

template <class E>
__device__ __forceinline__ const E* row_of(const RowArgs& a, int64_t row) { return static_cast<const E*>(a.logits) + row * a.stride; }

// A row's outputs from its sums.
struct RowStats {
    float m, s, log_s, entropy;
};
__device__ __forceinline__ RowStats stats_of(const Sums& a) {
    if (a.m != a.m || a.m == CUDART_INF_F) return {CUDART_NAN_F, CUDART_NAN_F, CUDART_NAN_F, CUDART_NAN_F};
    if (a.m == -CUDART_INF_F) return {a.m, 0.0f, -CUDART_INF_F, 0.0f};
    const float log_s = logf(a.s);
    return {a.m, a.s, log_s, log_s - a.u / a.s * kLn2};
}
// the log probability of an element x: -inf where the row or the element is masked
__device__ __forceinline__ float logprob_of(float x, const RowStats& r, float scale) {
    return r.m == -CUDART_INF_F ? r.m : (x - r.m) * scale - r.log_s;
}
__device__ __forceinline__ void write_stats(const RowArgs& a, int64_t row, int64_t t, float x_t, const RowStats& r) {
    if (a.logprob) a.logprob[row] = t >= a.vocab ? CUDART_NAN_F : logprob_of(x_t, r, a.scale);
    if (a.entropy) a.entropy[row] = r.entropy;
    if (a.norm) reinterpret_cast<float2*>(a.norm)[row] = make_float2(r.m, r.s);
}
__device__ __forceinline__ void write_top(const RowArgs& a, int64_t row, int k, unsigned long long key, const RowStats& r) {
    a.top_ids[row * a.top + k] = key ? (int)position_of(key) : -1;
    a.top_logprobs[row * a.top + k] = key ? logprob_of(value_of((uint32_t)(key >> 32)), r, a.scale) : -CUDART_INF_F;
}
// a row that nobody asked for
__device__ __forceinline__ void write_nothing(const RowArgs& a, int64_t row, int thread, int threads) {
    if (thread == 0) {
        if (a.logprob) a.logprob[row] = 0.0f;
        if (a.entropy) a.entropy[row] = 0.0f;
        if (a.norm) reinterpret_cast<float2*>(a.norm)[row] = make_float2(0.0f, 0.0f);
    }
    for (int k = thread; k < a.top; k += threads) {
        a.top_ids[row * a.top + k] = -1;
        a.top_logprobs[row * a.top + k] = -CUDART_INF_F;
    }
}

// ---- the gradient of a row ----
//
// dx_i = c [ g (1[i = t] - p_i) - h p_i (ln p_i + H) ] with p_i = 2^t_i / S, t_i in units of log 2:
//      = 2^t_i (A + B t_i) + 1[i = t] c g,     B = -h c ln 2 / S,   A = -(g + h (H - ln S)) c / S
struct Gradient {
    float base, c, A, B, at_target;
    int target;
    int kind;                      // 0: as above; 1: zeros (nobody asked, or nothing but masked tokens); 2: NaN (no such token)
};
__device__ __forceinline__ Gradient gradient_of(const RowArgs& a, int64_t t, float m, float s, float log_s, float entropy, float g, float h) {
    Gradient r;
    r.base = base_of(m);
    r.c = a.scale * kLog2E;
    r.target = (int)(t < a.vocab ? t : -1);
    const float per = a.scale / s;
    r.B = -h * per * kLn2;
    r.A = -(h == 0.0f ? g : fmaf(h, entropy - log_s, g)) * per;
    r.at_target = g * a.scale;
    r.kind = t >= a.vocab ? 2 : t < 0 || m == -CUDART_INF_F ? 1 : 0;
    return r;
}
template <bool kEntropy>
__device__ __forceinline__ float gradient_at(const Gradient& r, float x, int i) {
    if (r.kind) return r.kind == 1 ? 0.0f : CUDART_NAN_F;
    float t = (x - r.base) * r.c, y = r.A;
    if (kEntropy) {
        t = t < kGone ? kGone : t;    // not fmaxf: NaN stays
        y = fmaf(r.B, t, y);
    }
    y *= exp2_fast(t);
    return i == r.target ? y + r.at_target : y;
}
// .. of a vector in which the target is not
template <bool kEntropy, class E>
__device__ __forceinline__ Vector<E> gradient_at(const Gradient& r, const Vector<E>& x) {
    constexpr int N = Vector<E>::N;
    Vector<E> out;
    const Pair off = pair_of(-r.base, -r.base), by = pair_of(r.c, r.c), A = pair_of(r.A, r.A), B = pair_of(r.B, r.B);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        float p, q;
        Pair t = (x.at(i) + off) * by, y = A;
        split(t, p, q);
        if (kEntropy) {
            p = p < kGone ? kGone : p, q = q < kGone ? kGone : q;
            y = fma2(B, pair_of(p, q), A);
        }
        out.put(i, y * pair_of(exp2_fast(p), exp2_fast(q)));
    }
    return out;
}
template <class E>
__device__ __forceinline__ void store_whole(E* to, const Vector<E>& x) {
    asm volatile("st.global.v4.b32 [%0], {%1, %2, %3, %4};" ::"l"(to), "r"(x.w.x), "r"(x.w.y), "r"(x.w.z), "r"(x.w.w) : "memory");
}
// What a thread adds to the whole vectors that it has written: the row's vector number v, which is not whole ..
template <bool kEntropy, class E>
__device__ __forceinline__ void store_partial(E* row, const Row<E>& r, int v, const Vector<E>& x, const Gradient& y) {
#pragma unroll
    for (int k = 0; k < Vector<E>::N; ++k) {
        const int i = r.first(v) + k;
        if (i >= 0 && i < r.V) row[i] = from_float<E>(gradient_at<kEntropy>(y, x.one(k), i));
    }
}
// .. and zeros, or NaN, where the row has no gradient
template <class E>
__device__ __forceinline__ Vector<E> gradient_of_kind(const Gradient& r) {
    Vector<E> out;
    const Pair p = r.kind == 1 ? pair_of(0.0f, 0.0f) : pair_of(CUDART_NAN_F, CUDART_NAN_F);
#pragma unroll
    for (int i = 0; i < Vector<E>::N / 2; ++i) out.put(i, p);
    return out;
}
// .. and what L lanes write vector by vector: the target's own term comes afterwards, from the thread that wrote its vector
template <bool kEntropy, class E>
__device__ __forceinline__ void store_vector(const Row<E>& to, E* row, int v, const Vector<E>& in, const Gradient& y) {
    if (v >= to.vectors) return;
    const Vector<E> out = y.kind ? gradient_of_kind<E>(y) : gradient_at<kEntropy>(y, in);
    if (to.whole(v)) {
        store_whole(row + to.first(v), out);
    } else {
        const E* const e = reinterpret_cast<const E*>(&out.w);
#pragma unroll
        for (int k = 0; k < Vector<E>::N; ++k)
            if ((unsigned)(to.first(v) + k) < (unsigned)to.V) row[to.first(v) + k] = e[k];
    }
}
// Where the gradient's row `to` is not aligned as the logits' row `from` is, each of its vectors begins with element `off` of one of
// theirs and the rest of it is in the next: lane `sub` of L has vectors sub, sub + L, .. and gets what it lacks from its neighbour.
__device__ __forceinline__ uint4 shuffled(unsigned int group, uint4 x, int lane, int L) {
    return {__shfl_sync(group, x.x, lane, L), __shfl_sync(group, x.y, lane, L), __shfl_sync(group, x.z, lane, L), __shfl_sync(group, x.w, lane, L)};
}
// vectors w, w + L, .. are here, w + 1, w + 1 + L, .. come; of those, lane L - 1 has its last already
template <int L, class E>
__device__ __forceinline__ void join_next(Vector<E> (&in)[kUnroll], const Vector<E>& last, int off, int sub, unsigned int group) {
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
        const Vector<E> next = {shuffled(group, sub == 0 && k + 1 < kUnroll ? in[(k + 1) % kUnroll].w : in[k].w, sub + 1, L)};
        in[k] = joined(in[k], k + 1 == kUnroll && sub == L - 1 ? last : next, off);
    }
}
// .. and w - 1, w - 1 + L, .. come; of those, lane 0 has its first already
template <int L, class E>
__device__ __forceinline__ void join_previous(Vector<E> (&in)[kUnroll], const Vector<E>& first, int off, int sub, unsigned int group) {
#pragma unroll
    for (int k = kUnroll - 1; k >= 0; --k) {
        const Vector<E> previous = {shuffled(group, sub == L - 1 && k ? in[(k + kUnroll - 1) % kUnroll].w : in[k].w, sub + L - 1, L)};
        in[k] = joined(k == 0 && sub == 0 ? first : previous, in[k], off);
    }
}
template <class E>
__device__ __forceinline__ int off_of(const Row<E>& from, const Row<E>& to) { return (from.skip - to.skip + Row<E>::N) % Row<E>::N; }
// the lanes of the L that share a row
template <int L>
__device__ __forceinline__ unsigned int group_of_lane() {
    return L == 32 ? ~0u : ((1u << (L & 31)) - 1) << (threadIdx.x & 31 & ~(L - 1));
}
template <class E>
__device__ __forceinline__ bool aligned_alike(const E* a, const E* b) { return ((reinterpret_cast<uintptr_t>(a) ^ reinterpret_cast<uintptr_t>(b)) & 15) == 0; }

// ---- few elements a row: L lanes share one, N elements each, kept in registers ----
template <class E, int L, int N, bool kGrad>
__global__ void __launch_bounds__(256) narrow_kernel(RowArgs a) {
    const int sub = threadIdx.x % L;
    const int64_t row = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L;
    const bool real = row < a.rows;
    const int64_t t = !real ? -1 : a.targets ? a.targets[row] : 0;
    const E* const from = row_of<E>(a, real ? row : 0);
    const float c = a.scale * kLog2E;
    float x[N], m = -CUDART_INF_F;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int i = sub + k * L;
        x[k] = t >= 0 && i < a.vocab ? as_float(from[i]) : -CUDART_INF_F;
        m = max_nan(m, x[k]);
    }
    const float x_t = t >= 0 && t < a.vocab ? as_float(from[t]) : 0.0f;   // before a gradient takes its place
#pragma unroll
    for (int o = L / 2; o; o >>= 1) m = max_nan(m, __shfl_xor_sync(~0u, m, o));
    Sums all = {m, 0.0f, 0.0f};
    const float base = base_of(m);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const float d = fmaxf((x[k] - base) * c, kGone), e = exp2_fast(d);
        all.s += e;
        all.u = fmaf(e, d, all.u);
    }
#pragma unroll
    for (int o = L / 2; o; o >>= 1) {
        all.s += __shfl_xor_sync(~0u, all.s, o);
        all.u += __shfl_xor_sync(~0u, all.u, o);
    }
    const RowStats r = stats_of(all);
    if (real && sub == 0) {
        if (t < 0) write_nothing(a, row, 0, 1);
        else write_stats(a, row, t, x_t, r);
    }
    if (kGrad) {
        __syncwarp();                  // the row's logits have been read by all of its lanes
        if (!real) return;
        const Gradient y = gradient_of(a, t, r.m, r.s, r.log_s, 0.0f, a.g_logprob[row], 0.0f);
        E* const to = static_cast<E*>(a.grad) + row * a.grad_stride;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int i = sub + k * L;
            if (i < a.vocab) to[i] = from_float<E>(gradient_at<false>(y, x[k], i));
        }
        return;
    }
    unsigned long long last = ~0ull;
    for (int n = 0; n < a.top; ++n) {
        unsigned long long best = 0;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int i = sub + k * L;
            const unsigned long long key = i < a.vocab ? key_of(x[k], i) : 0;
            if (key < last && key > best) best = key;
        }
#pragma unroll
        for (int o = L / 2; o; o >>= 1) {
            const unsigned long long other = __shfl_xor_sync(~0u, best, o);
            best = other > best ? other : best;
        }
        if (real && t >= 0 && sub == 0) write_top(a, row, n, best, r);
        last = best ? best : 1;        // the row has no more: every later key is below
    }
}

// ---- the loss and gradient of a row that L lanes hold in registers: 4 vectors a lane ----
// 60,000 x 400 bf16 27 us, fp32 41 us (71 % of the copy bandwidth; 47 us with registers for 9 blocks instead of 12 on an SM); 100,000 x 171
// bf16 26 us: what is done once a row bounds it, and rows that begin at no vector.
template <class E, int L>
__global__ void __launch_bounds__(128, 12) warp_loss_kernel(RowArgs a) {
    const int sub = threadIdx.x % L;
    const int64_t row = (int64_t)blockIdx.x * (128 / L) + threadIdx.x / L;
    if (row >= a.rows) return;
    const unsigned int group = group_of_lane<L>();
    const int64_t t = a.targets[row];
    const Row<E> x(row_of<E>(a, row), a.vocab);
    const float c = a.scale * kLog2E;
    Vector<E> v[kUnroll];
    RowStats r = {0.0f, 1.0f, 0.0f, 0.0f};
    float given = 0.0f;
    if (t >= 0) {
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) v[k] = x.load(k * L + sub);
        given = t < a.vocab ? as_float(x.x[t]) : 0.0f;
        float most = -CUDART_INF_F;
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) most = max_nan(most, v[k].max());
        if (L == 32) most = warp_max_nan(most);
        else
#pragma unroll
            for (int o = L / 2; o; o >>= 1) most = max_nan(most, __shfl_xor_sync(group, most, o));
        Sums all = {-CUDART_INF_F, 0.0f, 0.0f};
        add_vectors<false>(all, v, most, c);      // one maximum for all lanes: nothing to rescale
#pragma unroll
        for (int o = L / 2; o; o >>= 1) all.s += __shfl_xor_sync(group, all.s, o);
        r = stats_of(all);
        if (sub == 0) write_stats(a, row, t, given, r);
    } else {
        write_nothing(a, row, sub, L);
    }
    const Gradient y = gradient_of(a, t, r.m, r.s, r.log_s, 0.0f, a.g_logprob[row], 0.0f);
    E* const out = static_cast<E*>(a.grad) + row * a.grad_stride;
    const Row<E> to(out, a.vocab);
    if (const int off = off_of(x, to); off && y.kind == 0) {      // no lane has a vector behind the row's last
        if (x.skip > to.skip) join_next<L>(v, Row<E>::nothing(), off, sub, group);
        else join_previous<L>(v, Row<E>::nothing(), off, sub, group);
    }
    const int at = y.target >= 0 && y.kind == 0 ? (y.target + to.skip) / Row<E>::N : -1;
    __syncwarp(group);             // the row's logits have been read by all lanes
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) store_vector<false>(to, out, k * L + sub, v[k], y);
    if (at >= 0 && at % L == sub) out[y.target] = from_float<E>(gradient_at<false>(y, given, y.target));
}

// ---- rows that a team of T threads, or a cluster of such blocks, sums up in one pass ----

constexpr int kListed = 256;       // elements that reach the bound, before a slower way is taken
template <int T>
struct SumsShared {
    Sums warp[T / 32], cluster[kMaxCluster];
};
template <int T>
struct TopShared {
    uint32_t bound[T / 32][32];
    int listed, threads;
    uint16_t thread[T];
    unsigned long long list[kListed], warp[T / 32][32], cluster[T > 32 ? kMaxCluster : 1][32];
};
struct NoTop {
    int listed, threads;
};

template <int T>
__device__ __forceinline__ void team_sync() {
    if constexpr (T == 32) __syncwarp();
    else __syncthreads();
}
template <int T>
__device__ __forceinline__ Sums team_merged(Sums mine, Sums* shared, float c) {
    mine = warp_merged(mine, c);
    if constexpr (T == 32) return mine;
    const int lane = threadIdx.x & 31;
    if (lane == 0) shared[threadIdx.x >> 5] = mine;
    __syncthreads();
    return warp_merged(lane < T / 32 ? shared[lane] : Sums{-CUDART_INF_F, 0.0f, 0.0f}, c);
}
// The 32 largest keys of the team's warps, each warp's sorted, in its warp 0.
template <int T, class K>
__device__ __forceinline__ K team_top(K best, K (*shared)[32]) {
    const int lane = threadIdx.x & 31, warp = (threadIdx.x % T) >> 5;
#pragma unroll
    for (int half = T / 64; half; half >>= 1) {
        if (warp >= half && warp < 2 * half) shared[warp][lane] = best;
        __syncthreads();
        if (warp < half) best = merge_sorted(best, shared[warp + half][31 - lane]);
    }
    return best;
}

// The part of a row that a block of a cluster takes: its whole vectors [lo, lo + n), and the vectors at the ends.
template <class E>
struct Part {
    int lo, n;
    bool head, tail;
    __device__ __forceinline__ Part(const Row<E>& x, int rank, int blocks, int slice) {
        const int begin = rank * slice, end = min(begin + slice, x.vectors);
        lo = max(begin, x.lo);
        n = max(min(end, x.hi) - lo, 0);
        head = x.head() && rank == 0;
        tail = x.tail() && begin < x.vectors && end == x.vectors;
    }
};

// The sums of a thread's share of a part: every T-th of its whole vectors, which vector(i) gives, and `edge`.
template <bool kEntropy, int T, class E, class Get>
__device__ __forceinline__ Sums sums_of_part(const Part<E>& part, int tid, float c, const Vector<E>& edge, Get&& vector) {
    constexpr int U = kUnroll;
    Sums mine = {-CUDART_INF_F, 0.0f, 0.0f};
    int i = tid;
    const int ahead = 31 - (tid & 31);                 // a warp's lanes go the same way
    for (; i + ahead + (U - 1) * T < part.n; i += U * T) {
        Vector<E> in[U];
#pragma unroll
        for (int k = 0; k < U; ++k) in[k] = vector(i + k * T);
        float most = in[0].max();
#pragma unroll
        for (int k = 1; k < U; ++k) most = max_nan(most, in[k].max());
        add_vectors<kEntropy>(mine, in, most, c);
    }
    for (; i - (tid & 31) < part.n; i += U * T) {      // once, unless the last lanes have nothing where the first have all
        Vector<E> in[U];
#pragma unroll
        for (int k = 0; k < U; ++k) in[k] = i + k * T < part.n ? vector(i + k * T) : Row<E>::nothing();
        float most = in[0].max();
#pragma unroll
        for (int k = 1; k < U; ++k) most = max_nan(most, in[k].max());
        add_vectors<kEntropy>(mine, in, most, c);
    }
    if ((part.head && tid < 32) || (part.tail && tid >= T - 32)) {
        const Vector<E> in[1] = {edge};
        add_vectors<kEntropy>(mine, in, edge.max(), c);
    }
    return mine;
}
// The vector of the row that is not whole and belongs to this thread: -1 for none.
template <int T, class E>
__device__ __forceinline__ int edge_of(const Row<E>& x, const Part<E>& part, int tid) {
    return part.head && tid == 0 ? 0 : part.tail && tid == T - 1 ? x.vectors - 1 : -1;
}

template <class E, int T, bool kTop>
__global__ void __launch_bounds__(T < 128 ? 128 : T) stream_kernel(RowArgs a) {
    constexpr int kTeams = T < 128 ? 128 / T : 1;
    __shared__ SumsShared<T> sums_shared[kTeams];
    __shared__ std::conditional_t<kTop, TopShared<T>, NoTop> top_shared[kTeams];
    const int tid = threadIdx.x % T, team = threadIdx.x / T, lane = threadIdx.x & 31;
    auto& sh = sums_shared[team];
    auto& st = top_shared[team];
    int rank = 0, blocks = 1;
    int64_t row = (int64_t)blockIdx.x * kTeams + team;
    if constexpr (T > 32) {
        rank = (int)cg::this_cluster().block_rank(), blocks = (int)cg::this_cluster().num_blocks();
        row = blockIdx.x / blocks;
    }
    if (row >= a.rows) return;
    const int64_t t = a.targets ? a.targets[row] : 0;
    if (t < 0) {
        if (rank == 0) write_nothing(a, row, tid, T);
        return;
    }
    if (T > 32 && blocks > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // awaited before another block's memory is used
    if (kTop && tid == 0) st.listed = st.threads = 0;
    const Row<E> x(row_of<E>(a, row), a.vocab);
    const float x_t = rank == 0 && tid == 0 && a.logprob && t < a.vocab ? as_float(x.x[t]) : 0.0f;
    const float c = a.scale * kLog2E;
    const Part<E> part(x, rank, blocks, T > 32 ? a.slice : x.vectors);
    const char* const from = reinterpret_cast<const char*>(x.x + x.first(part.lo));
    const int edge = edge_of<T>(x, part, tid);
    const Vector<E> at_edge = edge >= 0 ? x.partial(edge) : Row<E>::nothing();
    auto vector = [&](int i) { return Row<E>::load_at(from + (int64_t)i * 16); };
    const Sums mine = sums_of_part<true, T>(part, tid, c, at_edge, vector);
    Sums all = team_merged<T>(mine, sh.warp, c);
    unsigned long long best = 0;
    if constexpr (kTop) {
        // Every thread's largest element is one of the row's: the top-th largest of these bounds the top-th largest element
        // from below.  Elements that reach the bound are in threads whose largest does: about `top` threads.  Those are read once
        // more; their elements from the bound on - a few more than wanted, unless many are equal - are listed and sorted.
        uint32_t order = sorted(order_of(mine.m));
        if constexpr (T > 32) {
            order = team_top<T>(order, st.bound);
            if (tid < 32) st.bound[0][lane] = order;
            __syncthreads();
            order = st.bound[0][a.top - 1];
        } else {
            order = __shfl_sync(~0u, order, a.top - 1);
            __syncwarp();
        }
        const float bound = value_of(order);              // NaN counts as above everything: "not below" is what is asked
        if (!(mine.m < bound)) st.thread[atomicAdd(&st.threads, 1)] = (uint16_t)tid;
        team_sync<T>();
        const int threads = st.threads;
        auto list = [&](float value, int i) {
            if (value < bound) return;
            const int at = atomicAdd(&st.listed, 1);
            if (at < kListed) st.list[at] = key_of(value, i);
        };
        constexpr int kAtOnce = 4;                        // a warp's threads whose vectors it has in flight
        for (int b = tid >> 5; b < threads; b += kAtOnce * (T / 32)) {
            int first[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) first[k] = b + k * (T / 32) < threads ? st.thread[b + k * (T / 32)] : part.n;
            for (int j = lane * T; j - lane * T < part.n; j += 32 * T) {
                Vector<E> q[kAtOnce];
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k) q[k] = first[k] + j < part.n ? vector(first[k] + j) : Row<E>::nothing();
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k)
                    if (first[k] + j < part.n && !(q[k].max() < bound)) {
                        const int n = x.first(part.lo + first[k] + j);
#pragma unroll
                        for (int e = 0; e < Vector<E>::N; ++e) list(q[k].one(e), n + e);
                    }
            }
        }
        if (edge >= 0)
            for (int i = max(x.first(edge), 0); i < min(x.first(edge + 1), x.V); ++i) list(as_float(x.x[i]), i);
        team_sync<T>();
        const int listed = st.listed;
        if (listed <= kListed) {
            if (tid < 32)
                for (int n = 0; n < listed; n += 32) best = with_more(best, n + lane < listed ? st.list[n + lane] : 0ull);
        } else {   // many are equal: every warp keeps the best it has seen, and takes only what is better
            auto take = [&](bool in, float value, int i) {
                const unsigned long long key = in ? key_of(value, i) : 0;
                const bool better = key > __shfl_sync(~0u, best, a.top - 1);
                if (__any_sync(~0u, better)) best = with_more(best, better ? key : 0ull);
            };
            for (int b = tid >> 5; b < threads; b += T / 32) {
                for (int j = (int)st.thread[b] + lane * T; j - lane * T < part.n; j += 32 * T) {
                    const Vector<E> q = j < part.n ? vector(j) : Row<E>::nothing();
#pragma unroll
                    for (int e = 0; e < Vector<E>::N; ++e) take(j < part.n, q.one(e), x.first(part.lo + j) + e);
                }
            }
            if ((part.head && tid < 32) || (part.tail && tid >= T - 32))
#pragma unroll
                for (int e = 0; e < Vector<E>::N; ++e) {
                    const int i = x.first(max(edge, 0)) + e;
                    take(edge >= 0 && i >= 0 && i < x.V, at_edge.one(e), i);
                }
            if constexpr (T > 32) best = team_top<T>(best, st.warp);
        }
    }
    if constexpr (T > 32) {
        if (blocks > 1) {
            cg::cluster_group cluster = cg::this_cluster();
            asm volatile("barrier.cluster.wait.aligned;" ::: "memory");    // every block has begun
            if (tid < 32 && rank) {
                if (lane == 0) cluster.map_shared_rank(&sh, 0)->cluster[rank] = all;
                if constexpr (kTop) cluster.map_shared_rank(&st, 0)->cluster[rank][lane] = best;
            }
            cluster.sync();
            if (rank) return;
            for (int b = 1; b < blocks; ++b) {
                all = merged(all, sh.cluster[b], c);
                if constexpr (kTop)
                    if (tid < 32) best = merge_sorted(best, st.cluster[b][31 - lane]);
            }
        }
        if (tid >= 32) return;
    }
    const RowStats r = stats_of(all);
    if (lane == 0) write_stats(a, row, t, x_t, r);
    if (kTop && lane < a.top) write_top(a, row, lane, best, r);
}

// The loss and its gradient of a long row.  The block's part of the row is copied to shared memory (by the thread that
// works on it: nothing to wait for but its own copies), summed up, and read again for the gradient when the cluster has
// agreed on m and S.  kResident false: it does not fit, and is read from global memory again.
template <class E, int T, bool kResident>
__global__ void __launch_bounds__(T) loss_kernel(RowArgs a) {
    constexpr int U = kUnroll, N = Vector<E>::N;
    __shared__ SumsShared<T> sh;
    extern __shared__ uint4 kept[];
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), blocks = (int)cluster.num_blocks(), tid = threadIdx.x;
    const int64_t row = blockIdx.x / blocks;
    const int64_t t = a.targets[row];
    const Row<E> x(row_of<E>(a, row), a.vocab);
    const Part<E> part(x, rank, blocks, a.slice);
    const char* const from = reinterpret_cast<const char*>(x.x + x.first(part.lo));
    const float c = a.scale * kLog2E;
    const int edge = edge_of<T>(x, part, tid);
    // the thread that writes the target's vector adds the target's own term
    const int at = t >= 0 && t < a.vocab ? ((int)t + x.skip) / N - part.lo : -1;
    const bool owner = at >= 0 && at < part.n && at % T == tid;
    Vector<E> at_edge = Row<E>::nothing();
    float x_t = 0.0f;
    Sums all = {0.0f, 1.0f, 0.0f};
    auto vector = [&](int i) {
        if (!kResident) return Row<E>::load_at(from + (int64_t)i * 16);
        Vector<E> v;
        v.w = kept[i];
        return v;
    };
    if (t >= 0) {
        if (blocks > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
        if (kResident) {
            const uint32_t to = (uint32_t)__cvta_generic_to_shared(kept);
#pragma unroll 4
            for (int i = tid; i < part.n; i += T)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + i * 16), "l"(from + (int64_t)i * 16) : "memory");
        }
        if (edge >= 0) at_edge = x.partial(edge);
        if ((owner || (rank == 0 && tid == 0)) && t < a.vocab) x_t = as_float(x.x[t]);
        if (kResident) asm volatile("cp.async.wait_all;" ::: "memory");
        all = team_merged<T>(sums_of_part<false, T>(part, tid, c, at_edge, vector), sh.warp, c);
        if (blocks > 1) {
            asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
            if (tid < blocks) cluster.map_shared_rank(&sh, tid)->cluster[rank] = all;
            cluster.sync();       // the logits have been read by everybody: the gradient may take their place
            all = sh.cluster[0];
            for (int b = 1; b < blocks; ++b) all = merged(all, sh.cluster[b], c);
        } else {
            __syncthreads();
        }
        if (rank == 0 && tid == 0) write_stats(a, row, t, x_t, stats_of(all));
    } else if (rank == 0 && tid == 0) {
        write_nothing(a, row, 0, 1);
    }
    const RowStats r = stats_of(all);
    const Gradient y = gradient_of(a, t, r.m, r.s, r.log_s, 0.0f, a.g_logprob[row], 0.0f);
    E* const to = static_cast<E*>(a.grad) + row * a.grad_stride;
    E* const out = to + x.first(part.lo);
    if (aligned_alike(to, x.x)) {
        int i = tid;
        if (y.kind) {
            const Vector<E> same = gradient_of_kind<E>(y);
            for (; i < part.n; i += T) store_whole(out + i * N, same);
        } else {
            for (; i + (U - 1) * T < part.n; i += U * T) {
                Vector<E> in[U];
#pragma unroll
                for (int k = 0; k < U; ++k) in[k] = vector(i + k * T);
#pragma unroll
                for (int k = 0; k < U; ++k) store_whole(out + (i + k * T) * N, gradient_at<false>(y, in[k]));
            }
            for (; i < part.n; i += T) store_whole(out + i * N, gradient_at<false>(y, vector(i)));
            if (owner) to[t] = from_float<E>(gradient_at<false>(y, x_t, (int)t));
        }
    } else if (part.n > 0) {
        // The rows of the gradient are aligned otherwise than the logits': each of its vectors comes from two of theirs, and at
        // the ends of the part up to N elements come one by one.
        const E* const elements = kResident ? reinterpret_cast<const E*>(kept) : reinterpret_cast<const E*>(from);
        const int first = x.first(part.lo), off = (x.skip - skip_of(to) + N) % N;
        auto one = [&](int i) { out[i] = from_float<E>(gradient_at<false>(y, as_float(elements[i]), first + i)); };
#pragma unroll 4
        for (int i = tid; i < part.n - 1; i += T)
            store_whole(out + i * N + off, y.kind ? gradient_of_kind<E>(y) : gradient_at<false>(y, joined(vector(i), vector(i + 1), off)));
        if (tid < N) one(tid < off ? tid : (part.n - 1) * N + tid);
        const int i_t = y.target >= 0 ? y.target - first : -1;
        if (i_t >= off && i_t < (part.n - 1) * N + off && (i_t - off) / N % T == tid) one(i_t);
    }
    if (edge >= 0) store_partial<false>(to, x, edge, at_edge, y);
}

// ---- the gradient alone, from the sums that the log probabilities left ----

__device__ __forceinline__ Gradient gradient_from_norm(const RowArgs& a, int64_t row) {
    const float2 n = reinterpret_cast<const float2*>(a.in_norm)[row];
    const float h = a.g_entropy ? a.g_entropy[row] : 0.0f;
    return gradient_of(a, a.targets[row], n.x, n.y, a.g_entropy ? logf(n.y) : 0.0f, a.g_entropy ? a.in_entropy[row] : 0.0f, a.g_logprob[row], h);
}

// L lanes take L kUnroll vectors of a row, as they lie in the gradient.  Nothing is shared and nothing waited for, so this runs at the
// copy's rate: 4,096 x 128,000 bf16 314 us (102 %), 2,048 x 50,001 with rows at every alignment 70 us (89 %), with the logits' rows
// aligned otherwise than the gradient's 73 us (element by element: 300).  Registers for five blocks on an SM: 334 us with those for four.
template <class E, bool kEntropy, int L>
__global__ void __launch_bounds__(256, 5) grad_kernel(RowArgs a, int segments) {
    const int sub = threadIdx.x % L;
    const int64_t item = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L, row = item / segments;
    if (row >= a.rows) return;
    const Row<E> from(row_of<E>(a, row), a.vocab);
    const int v = (int)(item - row * segments) * L * kUnroll + sub;
    E* const to = static_cast<E*>(a.grad) + row * a.grad_stride;
    const Row<E> x(to, a.vocab);
    Vector<E> in[kUnroll];
    const int off = off_of(from, x), w = from.skip < x.skip ? v - 1 : v;
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) in[k] = from.load(w + L * k);
    if (off) join_next<L>(in, sub == L - 1 ? from.load(w + L * (kUnroll - 1) + 1) : Row<E>::nothing(), off, sub, group_of_lane<L>());
    const Gradient y = gradient_from_norm(a, row);
    const int at = y.target >= 0 ? (y.target + x.skip) / Row<E>::N : -1;
    const bool owner = at >= v && (at - v) % L == 0 && at - v < L * kUnroll && y.kind == 0;
    const float x_t = owner ? as_float(from.x[y.target]) : 0.0f;
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) store_vector<kEntropy>(x, to, v + L * k, in[k], y);
    if (owner) to[y.target] = from_float<E>(gradient_at<kEntropy>(y, x_t, y.target));
}

// Few elements a row: L lanes share one, element by element.
template <class E, bool kEntropy, int L, int N>
__global__ void __launch_bounds__(256) narrow_grad_kernel(RowArgs a) {
    const int sub = threadIdx.x % L;
    const int64_t row = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L;
    if (row >= a.rows) return;
    const E* const from = row_of<E>(a, row);
    E* const to = static_cast<E*>(a.grad) + row * a.grad_stride;
    float x[N];
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = sub + k * L < a.vocab ? as_float(from[sub + k * L]) : 0.0f;
    const Gradient y = gradient_from_norm(a, row);
#pragma unroll
    for (int k = 0; k < N; ++k)
        if (sub + k * L < a.vocab) to[sub + k * L] = from_float<E>(gradient_at<kEntropy>(y, x[k], sub + k * L));
}

// ---- launches ----

bool type_ok(int type) { return type == SLAQ_F32 || type == SLAQ_BF16 || type == SLAQ_F16; }
int64_t size_of(int type) { return type == SLAQ_F32 ? 4 : 2; }

// The gradient may lie in the logits' place, row for row, or apart from them; rows of both may alternate in one buffer.
bool overlap(const RowArgs& a, int64_t es) {
    const char *x = static_cast<const char*>(a.logits), *y = static_cast<const char*>(a.grad);
    const int64_t width = a.vocab * es;
    const char *x_end = x + (a.rows - 1) * a.stride * es + width, *y_end = y + (a.rows - 1) * a.grad_stride * es + width;
    if (x_end <= y || y_end <= x) return false;
    if (a.rows > 1 && a.stride != a.grad_stride) return true;
    if (x == y) return false;
    if (a.rows == 1) return true;
    const int64_t pitch = a.stride * es, apart = ((y - x) % pitch + pitch) % pitch;
    return apart < width || pitch - apart < width;
}

int check_rows(const RowArgs& a, int type) {
    if (!type_ok(type) || a.rows < 0 || a.vocab < 1 || !(a.scale > 0.0f) || a.scale > kMostScale) return SLAQ_E_ARG;
    if (a.vocab > kMaxVocab || a.rows > 0x7FFFFFFF) return SLAQ_E_RANGE;
    if (a.rows && (!a.logits || (a.rows > 1 && a.stride < 0))) return SLAQ_E_ARG;
    if (reinterpret_cast<uintptr_t>(a.logits) % size_of(type)) return SLAQ_E_ARG;
    const bool ok = aligned(a.targets, a.logprob, a.entropy, a.top_ids, a.top_logprobs, a.g_logprob, a.g_entropy, a.in_entropy) &&
                    aligned(reinterpret_cast<const float2*>(a.norm), reinterpret_cast<const float2*>(a.in_norm));
    return ok ? SLAQ_OK : SLAQ_E_ARG;
}
int check_gradient(const RowArgs& a, int type) {
    if (a.rows && (!a.targets || !a.grad || !a.g_logprob || (a.rows > 1 && a.grad_stride < a.vocab))) return SLAQ_E_ARG;
    if (reinterpret_cast<uintptr_t>(a.grad) % size_of(type)) return SLAQ_E_ARG;
    return a.rows && overlap(a, size_of(type)) ? SLAQ_E_ARG : SLAQ_OK;
}

template <class F>
int by_type(int type, F&& f) {
    cudaError_t e;
    if (type == SLAQ_F32) e = f(0.0f);
    else if (type == SLAQ_BF16) e = f(__nv_bfloat16());
    else e = f(__half());
    if (e != cudaSuccess) (void)cudaGetLastError();
    return e == cudaSuccess ? SLAQ_OK : SLAQ_E_CUDA;
}

constexpr size_t kSliceBytes = 72 * 1024, kMostSlice = 200 * 1024;   // per block of the loss: three blocks on an SM, or one

template <class... Params, class... Args>
cudaError_t launch(void (*kernel)(Params...), int64_t blocks, int threads, size_t smem, int cluster, cudaStream_t st, Args... args) {
    if (smem > 40 * 1024) {   // what a kernel may use is state that all host threads share: never what this call needs, always the most
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostSlice);
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

// Vectors a row may touch, whatever its alignment.
template <class E>
int most_vectors(int vocab) { return (vocab + 2 * (Vector<E>::N - 1)) / Vector<E>::N; }
// What every block of a cluster takes of them: whole groups of 32.
int slice_of(int vectors, int blocks) { return ((vectors + blocks - 1) / blocks + 31) / 32 * 32; }

// Rows of at most this many elements are shared by a few lanes, the next by a warp with all its vectors in registers.
constexpr int kNarrow = 64;
template <class E>
bool fits_a_warp(int vocab) { return most_vectors<E>(vocab) <= 32 * kUnroll; }

template <class E, bool kGrad>
cudaError_t launch_narrow(const RowArgs& a, cudaStream_t st) {
    if (a.vocab <= 16) return launch(narrow_kernel<E, 4, 4, kGrad>, (a.rows + 63) / 64, 256, 0, 1, st, a);
    return launch(narrow_kernel<E, 16, 4, kGrad>, (a.rows + 15) / 16, 256, 0, 1, st, a);
}

template <class E, int T>
cudaError_t launch_stream(RowArgs a, int cluster, cudaStream_t st) {
    a.slice = slice_of(most_vectors<E>(a.vocab), cluster);
    const int64_t blocks = T == 32 ? (a.rows + 3) / 4 : a.rows * cluster;
    return launch(a.top ? stream_kernel<E, T, true> : stream_kernel<E, T, false>, blocks, T < 128 ? 128 : T, 0, cluster, st, a);
}

// A warp to a row while there are rows for all warps and a row is not too long for one (2,400 x 5,000 with 5 alternatives: 14.3 us, a
// block of 128 threads 18.5; 30,000 x 3,000: 39 and 68; but 2,000 x 16,000: 20.5 and 17.3).  With few rows a cluster shares one, as many
// blocks as make two on every SM (64 x 130,001 fp32: 11.0 us; four on every SM 12.1).  More threads where a block has the SM for
// itself (there 512 threads 12.0 us, 128 threads 17); with many rows several small blocks hide one another's ends better than
// large ones, up to a length: 8,192 x 32,768 bf16 98 us with 128 threads, 105 with 256; 8,192 x 65,536, which may touch 8,193 vectors and gets
// 256, 168 and 174 in a burst, 187 and 195 under load (512 threads: 242); 600 x 65,536 22.6 and 20.5; 2,048 x 65,536 fp32 90 and 84.
template <class E>
cudaError_t launch_logprobs(const RowArgs& a, cudaStream_t st) {
    if (a.vocab <= kNarrow) return launch_narrow<E, false>(a, st);
    const int vectors = most_vectors<E>(a.vocab);
    if (vectors <= 32 * kUnroll || (a.rows >= 16 * kSms && vectors <= 2048)) return launch_stream<E, 32>(a, 1, st);
    int cluster = 1;
    while (cluster < kMaxCluster && a.rows * cluster * 2 <= 2 * kSms && vectors / (2 * cluster) >= 256) cluster *= 2;
    const int each = vectors / cluster;
    const bool many = a.rows * cluster > 2 * kSms;
    if (each <= (many ? 8192 : 1024)) return launch_stream<E, 128>(a, cluster, st);
    if (each <= 4096 || many) return launch_stream<E, 256>(a, cluster, st);
    return launch_stream<E, 512>(a, cluster, st);
}

// A block's part of a row stays in shared memory; three blocks of 72 KB on an SM work in turn on loading, summing up and storing.
// 4,096 x 128,000 bf16 in clusters of four: 403 us, 79 % of the copy bandwidth (a step read twice from memory: 495 us; parts of 32 KB in
// clusters of eight 445; blocks of 512 threads 507).  What bounds it is the special function unit, two exponentials an element keep
// it busy 63 % of the time, and the turns: a block waits for its cluster once a row.  Exponentials by a polynomial in a quarter
// or half of the places were worth 2 % and nothing: 393 and 408 us.
template <class E>
cudaError_t launch_loss(RowArgs a, cudaStream_t st) {
    if (a.vocab <= kNarrow) return launch_narrow<E, true>(a, st);
    const int vectors = most_vectors<E>(a.vocab);
    // as few lanes as hold the row (100,000 x 171 bf16: 8 lanes 26 us, 32 lanes 82; 60,000 x 400: 16 lanes 27 us, 32 lanes 39)
    if (vectors <= 8 * kUnroll) return launch(warp_loss_kernel<E, 8>, (a.rows + 15) / 16, 128, 0, 1, st, a);
    if (vectors <= 16 * kUnroll) return launch(warp_loss_kernel<E, 16>, (a.rows + 7) / 8, 128, 0, 1, st, a);
    if (fits_a_warp<E>(a.vocab)) return launch(warp_loss_kernel<E, 32>, (a.rows + 3) / 4, 128, 0, 1, st, a);
    int cluster = 1;
    while (cluster < kMaxCluster && ((a.rows * cluster * 2 <= 2 * kSms && vectors / (2 * cluster) >= 256) || (size_t)slice_of(vectors, cluster) * 16 > kSliceBytes))
        cluster *= 2;
    a.slice = slice_of(vectors, cluster);
    const size_t bytes = (size_t)a.slice * 16;
    if (bytes > kMostSlice) return launch(loss_kernel<E, 512, false>, a.rows * cluster, 512, 0, cluster, st, a);
    if (a.slice <= 1536)   // 20,000 x 5,000 bf16: 88 us, with 256 threads 125; 8,000 x 16,000: 91 and 92
        return launch(loss_kernel<E, 128, true>, a.rows * cluster, 128, bytes, cluster, st, a);
    return launch(loss_kernel<E, 256, true>, a.rows * cluster, 256, bytes, cluster, st, a);
}

template <class E, bool kEntropy>
cudaError_t launch_grad(const RowArgs& a, cudaStream_t st) {
    auto blocks = [&](int64_t per) { return (a.rows + per - 1) / per; };
    if (a.vocab <= 16) return launch(narrow_grad_kernel<E, kEntropy, 4, 4>, blocks(256 / 4), 256, 0, 1, st, a);
    if (a.vocab <= kNarrow) return launch(narrow_grad_kernel<E, kEntropy, 16, 4>, blocks(256 / 16), 256, 0, 1, st, a);
    const int vectors = most_vectors<E>(a.vocab);
    if (vectors <= 8 * kUnroll) return launch(grad_kernel<E, kEntropy, 8>, blocks(256 / 8), 256, 0, 1, st, a, 1);
    if (vectors <= 16 * kUnroll) return launch(grad_kernel<E, kEntropy, 16>, blocks(256 / 16), 256, 0, 1, st, a, 1);
    const int segments = (vectors + 32 * kUnroll - 1) / (32 * kUnroll);
    const int64_t n = (a.rows * segments + 7) / 8;
    return n > 0x7FFFFFFF ? cudaErrorInvalidValue : launch(grad_kernel<E, kEntropy, 32>, n, 256, 0, 1, st, a, segments);
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
    return by_type(type, [&](auto e) { return launch_logprobs<decltype(e)>(a, static_cast<cudaStream_t>(cuda_stream)); });
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
        return d_grad_entropy ? launch_grad<decltype(e), true>(a, static_cast<cudaStream_t>(cuda_stream))
                              : launch_grad<decltype(e), false>(a, static_cast<cudaStream_t>(cuda_stream));
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
    return by_type(type, [&](auto e) { return launch_loss<decltype(e)>(a, static_cast<cudaStream_t>(cuda_stream)); });
}
