// The norms of groups of gradients over many tensors, and the gradients times the factors that clipping gives them.
//
//     norm_g = |scale| sqrt(sum x^2) over the group's tensors,     factor_g = min(1, most_g / norm_g)
//
// Squares are summed up in 32 bits as far as a lane has them in registers (at most 8 additions one after the other and the join of
// eight sums, 11 roundings, so 2^-20 of the sum at the very most and 2^-24 in the mean), and in 64 bits from there on, always in the same order.
// A product is rounded to 32 bits and then, for 16-bit types, to those: half a step and 2^-24.  Where 32
// bits do not hold the squares, gradients below 2^-50 or above 2^63, a lane takes them in 64.
#include <cmath>
#include <new>

#include "slaq_plan.cuh"
#include "slaq_rows.cuh"

namespace slaq {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kDeep = 8;                 // vectors that a lane has in flight
constexpr int kBatch = 32 * kDeep;       // vectors that a warp takes at a time
constexpr float kLeastSum = 7.888609052210118e-31f;   // 2^-100: what is lost of smaller squares is at most 2^-30 of it

struct GradRef {
    const void* grad;
    void* out;
    int64_t n;
    int32_t group, first, type, reserved;   // first: the number of its first unit among all units
};
// A group's units are neighbours, and so are the places in which the warps leave their sums.
struct GroupRef {
    int32_t first, units, place, places;
};

struct NormArgs {
    const GradRef* tensors;
    const GroupRef* groups;
    const int32_t* tensor_of;           // per unit
    double* sums;                       // per place
    int32_t n_units, n_groups, team, join_here;
    const int32_t* active;
    const float* mosts;
    double scale, most;
    float *norm, *factor;
    unsigned int* ticket;
};
struct ApplyArgs {
    const GradRef* tensors;
    const int32_t* tensor_of;
    int32_t n_units;
    const int32_t* active;
    const float* factor;
};

// A unit of a tensor is kBatch of its whole vectors.  The elements before and behind all of them belong to the first and the last unit.  A
// tensor's units are counted from its elements, whatever its alignment: the last may have no whole vector.
template <class E>
struct Part {
    static constexpr int N = Vector<E>::N;
    const E* x;
    int64_t before, vectors, at;        // elements before vector 0; the unit's first vector
    int head, tail;
    __device__ __forceinline__ Part(const GradRef& t, int k) : x(static_cast<const E*>(t.grad)) {
        before = min((int64_t)((N - skip_of(x)) % N), t.n);
        vectors = (t.n - before) / N;
        at = (int64_t)k * kBatch;
        head = k == 0 ? (int)before : 0;
        tail = (at + kBatch) * N >= t.n ? (int)(t.n - before - vectors * N) : 0;   // the tensor's last unit
    }
    __device__ __forceinline__ int64_t element(int64_t vector) const { return before + vector * N; }
    __device__ __forceinline__ bool whole() const { return at + kBatch <= vectors; }
    // those in no whole vector: at most 2 N - 2, a lane each
    __device__ __forceinline__ bool has_loose(int lane) const { return lane < head + tail; }
    __device__ __forceinline__ int64_t loose(int lane) const { return lane < head ? lane : element(vectors) + lane - head; }
};

// The sum of squares of a lane's vectors, `n` of them 32 vectors apart, in 64 bits.  Out of line: kept out of the registers of what runs.
template <class E>
__device__ __noinline__ double wide_squares(const E* from, int n) {
    double sum = 0.0;
#pragma unroll 1
    for (int k = 0; k < n; ++k)
#pragma unroll 1
        for (int i = 0; i < Vector<E>::N; ++i) {
            const double a = (double)as_float(from[k * 32 * Vector<E>::N + i]);
            sum = fma(a, a, sum);
        }
    return sum;
}
template <class E>
__device__ __forceinline__ double unit_squares(const GradRef& t, int k, int lane) {
    constexpr int N = Vector<E>::N, P = N / 2;
    const Part<E> u(t, k);
    const int64_t v = u.at + lane;
    const E* const from = u.x + u.element(v);
    Vector<E> in[kDeep];
    if (u.whole()) {
#pragma unroll
        for (int j = 0; j < kDeep; ++j) in[j] = Row<E>::load_at(from + j * 32 * N);
    } else {
#pragma unroll
        for (int j = 0; j < kDeep; ++j) in[j] = v + j * 32 < u.vectors ? Row<E>::load_at(from + j * 32 * N) : Vector<E>{{0, 0, 0, 0}};
    }
    const double loose = u.has_loose(lane) ? (double)as_float(u.x[u.loose(lane)]) : 0.0;
    Pair s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = pair_of(0.0f, 0.0f);
    uint32_t any = 0;
#pragma unroll
    for (int j = 0; j < kDeep; ++j) {
        any |= (in[j].w.x | in[j].w.y) | (in[j].w.z | in[j].w.w);
#pragma unroll
        for (int i = 0; i < P; ++i) s[(j * P + i) % 4] = fma2(in[j].at(i), in[j].at(i), s[(j * P + i) % 4]);
    }
    float a, b;
    split((s[0] + s[1]) + (s[2] + s[3]), a, b);
    a += b;
    double sum = (double)a;
    if (!(a >= kLeastSum && a < CUDART_INF_F) && (any & (sizeof(E) == 4 ? 0x7FFFFFFFu : 0x7FFF7FFFu)))
        sum = wide_squares(from, (int)min((u.vectors - v + 31) / 32, (int64_t)kDeep));
    return fma(loose, loose, sum);
}
template <class F>
__device__ __forceinline__ auto by_device_type(int type, F&& f) {
    if (type == SLAQ_F32) return f(0.0f);
    if (type == SLAQ_BF16) return f(__nv_bfloat16());
    return f(__half());
}
__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(~0u, x, o);
    return x;
}

__device__ __forceinline__ void write_norm(const NormArgs& a, int g, double sum) {
    const double norm = sqrt(sum) * a.scale, most = a.mosts ? (double)a.mosts[g] : a.most;
    a.norm[g] = (float)norm;
    if (a.factor) a.factor[g] = !(norm < CUDART_INF) || !(most >= 0.0) ? CUDART_NAN_F : norm > most ? (float)(most / norm) : 1.0f;
}

// 209 M bf16 in 300 tensors: 63 us (6.6 TB/s, 101 % of a copy); with the rare sum in 64 bits inline, which took the vectors out of registers, 115.  320
// small tensors of 160 jobs: 5.7 us, of which the launch is 2 and the join 1.5; with a warp a group in the join 23.  The threads of a group in the join go by the
// groups' mean, so one large group among many small ones is joined by one thread: 209 M elements beside 700 groups of 1,000 228 us.
//
// Warp w of W takes units w, w + W, ..  What says where a unit lies is asked for a unit ahead: with a tensor's units spread over all warps, most
// units of a warp are in another tensor than the one before.
template <class F>
__device__ __forceinline__ void for_units(const GradRef* tensors, const int32_t* tensor_of, int n_units, F&& f) {
    const int warps = gridDim.x * kWarps;
    int u = blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (u >= n_units) return;
    auto tensor_at = [&](int k) { return k < n_units ? tensor_of[k] : -1; };   // n_units + 2 warps < 2^31
    int next = tensor_at(u + warps);
    GradRef t = tensors[tensor_of[u]];
    for (; u < n_units; u += warps) {
        const GradRef ahead = next >= 0 ? tensors[next] : t;
        next = tensor_at(u + 2 * warps);
        f(u, t);
        t = ahead;
    }
}

// The warps' sums of the groups `first`, `first` + `step`, .., a team of threads a group.  All of the block's threads go round together.
__device__ __forceinline__ void join(const NormArgs& a, int first, int step, double* shared) {
    const int lane = threadIdx.x & 31, team = a.team, me = threadIdx.x & (team - 1);
    for (int k0 = first; k0 < a.n_groups; k0 += step) {
        const int k = k0 + (int)threadIdx.x / team;
        const bool here = k < a.n_groups && (!a.active || a.active[k] > 0);
        const GroupRef g = here ? a.groups[k] : GroupRef{0, 0, 0, 0};
        double s = 0.0;
        for (int i = me; i < g.places; i += 8 * team) {
            double x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = i + j * team < g.places ? __ldcg(a.sums + g.place + i + j * team) : 0.0;
#pragma unroll
            for (int j = 0; j < 8; ++j) s += x[j];
        }
        for (int o = min(team, 32) / 2; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
        if (team == kThreads) {
            if (lane == 0) shared[threadIdx.x >> 5] = s;
            __syncthreads();
            s = 0.0;
            for (int w = 0; w < kWarps; ++w) s += shared[w];
            __syncthreads();
        }
        if (me == 0 && k < a.n_groups) {
            if (here) {
                write_norm(a, k, s);
            } else {
                a.norm[k] = 0.0f;
                if (a.factor) a.factor[k] = 1.0f;
            }
        }
    }
}

// A warp leaves one sum for each group of which it had units.  The block that ends last joins them, unless there are so many groups that a launch
// of its own does it sooner.
__global__ void __launch_bounds__(kThreads) norm_kernel(NormArgs a) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, mine = blockIdx.x * kWarps + warp;
    int group = -1, last = 0;
    bool on = false;
    double sum = 0.0;
    auto leave = [&] {
        const double s = warp_sum(sum);
        const GroupRef g = a.groups[group];
        if (lane == 0) a.sums[g.place + (g.units > g.places ? mine : last - g.first)] = s;
    };
    for_units(a.tensors, a.tensor_of, a.n_units, [&](int u, const GradRef& t) {
        if (t.group != group) {
            if (on) leave();
            sum = 0.0;
            group = t.group;
            on = !a.active || a.active[group] > 0;
        }
        if (!on) return;
        last = u;
        sum += by_device_type(t.type, [&](auto e) { return unit_squares<decltype(e)>(t, u - t.first, lane); });
    });
    if (on) leave();
    if (!a.join_here) return;

    __shared__ unsigned int arrived;
    __shared__ double shared[kWarps];
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        arrived = atomicAdd(a.ticket, 1u);
        __threadfence();
    }
    __syncthreads();
    if (arrived != gridDim.x - 1) return;
    join(a, 0, kThreads / a.team, shared);
    if (threadIdx.x == 0) *a.ticket = 0;
}
__global__ void __launch_bounds__(kThreads) join_kernel(NormArgs a) {
    __shared__ double shared[kWarps];
    const int each = kThreads / a.team;
    join(a, blockIdx.x * each, gridDim.x * each, shared);
}

// 209 M bf16 into other tensors: 139 us, 92 % of a copy; into tensors that lie otherwise in 16 bytes, element by element, 527.
template <class E>
__device__ __forceinline__ void apply_unit(const GradRef& t, int k, int lane, float factor) {
    constexpr int N = Vector<E>::N;
    const Part<E> u(t, k);
    E* const y = static_cast<E*>(t.out);
    const Pair by = pair_of(factor, factor);
    auto product = [&](Vector<E> x) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) x.put(i, x.at(i) * by);
        return x.w;
    };
    const int64_t v = u.at + lane;
    const E* const from = u.x + u.element(v);
    if (skip_of(u.x) == skip_of(y)) {
        uint4* const to = reinterpret_cast<uint4*>(y + u.element(v));
        Vector<E> in[kDeep];
        if (u.whole()) {
#pragma unroll
            for (int j = 0; j < kDeep; ++j) in[j] = Row<E>::load_at(from + j * 32 * N);
#pragma unroll
            for (int j = 0; j < kDeep; ++j) to[j * 32] = product(in[j]);
        } else {
            for (int j = 0; j < kDeep; ++j)
                if (v + j * 32 < u.vectors) to[j * 32] = product(Row<E>::load_at(from + j * 32 * N));
        }
    } else {
        const int64_t end = u.element(min(u.at + kBatch, u.vectors));
        for (int64_t i = u.element(u.at) + lane; i < end; i += 32) y[i] = from_float<E>(as_float(u.x[i]) * factor);
    }
    if (u.has_loose(lane)) y[u.loose(lane)] = from_float<E>(as_float(u.x[u.loose(lane)]) * factor);
}

__global__ void __launch_bounds__(kThreads) apply_kernel(ApplyArgs a) {
    const int lane = threadIdx.x & 31;
    for_units(a.tensors, a.tensor_of, a.n_units, [&](int u, const GradRef& t) {
        const float factor = a.factor[t.group];
        if ((a.active && a.active[t.group] <= 0) || factor != factor || (factor == 1.0f && t.out == t.grad)) return;
        by_device_type(t.type, [&](auto e) {
            apply_unit<decltype(e)>(t, u - t.first, lane, factor);
            return 0;
        });
    });
}

__host__ __device__ inline int64_t units_of(int64_t n, int type) {
    const int64_t per = kBatch * (type == SLAQ_F32 ? 4 : 8);
    return (n + per - 1) / per;
}
__global__ void fill_grad_units_kernel(const GradRef* tensors, int32_t* tensor_of) {
    const GradRef t = tensors[blockIdx.x];
    const int n = (int)units_of(t.n, t.type);
    for (int i = threadIdx.x; i < n; i += blockDim.x) tensor_of[t.first + i] = blockIdx.x;
}

}  // namespace
}  // namespace slaq

struct slaq_grad_norms_handle {
    int device = 0;
    int32_t n_tensors = 0, n_groups = 0, n_units = 0, team = 0;
    bool owns_ws = false;
    void* ws = nullptr;
    slaq::GradRef* tensors = nullptr;
    slaq::GroupRef* groups = nullptr;
    int32_t* tensor_of = nullptr;
    double* sums = nullptr;
    unsigned int* ticket = nullptr;
    int norm_grid = 0, apply_grid = 0;
    std::vector<slaq::GradRef> refs;
    std::vector<char> in_place;
    const char* err = "";
};

namespace slaq {
namespace {

int fail(slaq_grad_norms_handle* h, int code, const char* what) {
    h->err = what;
    return code;
}
constexpr int kMostRounds = 3;           // of the joining block
bool on_device(const slaq_grad_norms_handle* h) {
    int d = -1;
    return done(cudaGetDevice(&d)) && d == h->device;
}
size_t layout(slaq_grad_norms_handle* h, char* base, int32_t n_tensors, int64_t n_units, int32_t n_groups) {
    size_t at = 0;
    auto part = [&](auto*& p, size_t bytes) {
        if (h) p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(base + at);
        at += up(bytes);
    };
    slaq_grad_norms_handle none;
    slaq_grad_norms_handle& o = h ? *h : none;
    part(o.tensors, sizeof(GradRef) * (size_t)n_tensors);
    part(o.groups, sizeof(GroupRef) * (size_t)n_groups);
    part(o.tensor_of, sizeof(int32_t) * (size_t)n_units);
    part(o.sums, sizeof(double) * (size_t)n_units);
    part(o.ticket, sizeof(unsigned int));
    return at;
}
// as many units as there are with the smallest vectors: the size does not depend on the types
int64_t most_units(int32_t n_tensors, const int64_t* numels) {
    int64_t n = 0;
    for (int32_t t = 0; t < n_tensors; ++t) n += units_of(numels[t], SLAQ_F32);
    return n;
}
// Units, and the steps of blocks and warps beyond them and beyond the groups, are counted in 31 bits.
constexpr int32_t kMost = 1 << 30;       // tensors, or groups
bool sizes_ok(int32_t n_tensors, const int64_t* numels, int32_t n_groups) {
    if (n_tensors > kMost || n_groups > kMost) return false;
    int64_t n = 0;
    for (int32_t t = 0; t < n_tensors; ++t) {
        if (numels[t] < 0 || numels[t] > kMostElements) return false;
        n += numels[t];
        if (n > kMostElements) return false;
    }
    return true;
}

// Addresses, alignments, and what is written: no two tensors' elements, and no gradient's that are not written in place.
int check(const std::vector<GradRef>& refs, const char** what) {
    std::vector<std::pair<uintptr_t, uintptr_t>> written;
    for (const GradRef& t : refs) {
        if (!t.n) continue;
        const uintptr_t size = size_of(t.type), g = (uintptr_t)t.grad, o = (uintptr_t)t.out;
        *what = "a gradient, or what it is written to, is null or not aligned to its type";
        if (!g || !o || g % size || o % size) return SLAQ_E_ARG;
        written.emplace_back(o, o + size * (uintptr_t)t.n);
    }
    *what = "tensors that overlap";
    std::sort(written.begin(), written.end());
    for (size_t k = 1; k < written.size(); ++k)
        if (written[k].first < written[k - 1].second) return SLAQ_E_ARG;
    for (const GradRef& t : refs)
        if (t.n && t.out != t.grad && meets(written, (uintptr_t)t.grad, (uintptr_t)t.grad + size_of(t.type) * (uintptr_t)t.n)) return SLAQ_E_ARG;
    return SLAQ_OK;
}

int create(slaq_grad_norms_handle* h, void* dev_ws, size_t bytes, int32_t n_tensors, const slaq_grad_tensor* tensors, int32_t n_groups, cudaStream_t st) {
    std::vector<int64_t> numels((size_t)n_tensors);
    for (int32_t t = 0; t < n_tensors; ++t) {
        const slaq_grad_tensor& x = tensors[t];
        if (x.n < 0 || x.group < 0 || x.group >= n_groups || (x.type != SLAQ_F32 && x.type != SLAQ_BF16 && x.type != SLAQ_F16)) return SLAQ_E_ARG;
        numels[t] = x.n;
    }
    if (!sizes_ok(n_tensors, numels.data(), n_groups)) return SLAQ_E_RANGE;
    h->n_tensors = n_tensors, h->n_groups = n_groups;
    h->refs.resize((size_t)n_tensors);
    h->in_place.resize((size_t)n_tensors);
    // units are numbered group by group
    std::vector<int64_t> first((size_t)n_groups + 1);
    for (int32_t t = 0; t < n_tensors; ++t) first[(size_t)tensors[t].group + 1] += units_of(tensors[t].n, tensors[t].type);
    for (int32_t k = 0; k < n_groups; ++k) first[(size_t)k + 1] += first[k];
    const int64_t n_units = first[n_groups];
    for (int32_t t = 0; t < n_tensors; ++t) {
        const slaq_grad_tensor& x = tensors[t];
        h->in_place[t] = !x.out;
        h->refs[t] = {x.grad, x.out ? x.out : const_cast<void*>(x.grad), x.n, x.group, 0, x.type, 0};
    }
    if (const int rc = check(h->refs, &h->err)) return rc;
    int sm = 0, per_norm = 0, per_apply = 0;
    if (!done(cudaGetDevice(&h->device)) || !done(cudaDeviceGetAttribute(&sm, cudaDevAttrMultiProcessorCount, h->device)) ||
        !done(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_norm, norm_kernel, kThreads, 0)) ||
        !done(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_apply, apply_kernel, kThreads, 0)))
        return SLAQ_E_CUDA;
    if (captured(st)) return SLAQ_E_ARG;
    h->n_units = (int32_t)n_units;
    auto grid = [&](int per) { return (int)std::max<int64_t>(1, std::min<int64_t>((n_units + kWarps - 1) / kWarps, (int64_t)sm * std::max(per, 1))); };
    h->norm_grid = grid(per_norm), h->apply_grid = grid(per_apply);
    const int64_t warps = (int64_t)h->norm_grid * kWarps;
    std::vector<GroupRef> groups((size_t)n_groups);
    int64_t place = 0;
    for (int32_t k = 0; k < n_groups; ++k) {
        const int64_t units = first[(size_t)k + 1] - first[k], places = std::min(units, warps);
        groups[k] = {(int32_t)first[k], (int32_t)units, (int32_t)place, (int32_t)places};
        place += places;
    }
    // A thread has eight sums in flight.
    h->team = place > (int64_t)n_groups * 256 ? kThreads : place > (int64_t)n_groups * 8 ? 32 : 1;
    for (int32_t t = 0; t < n_tensors; ++t) {
        h->refs[t].first = (int32_t)first[tensors[t].group];
        first[tensors[t].group] += units_of(tensors[t].n, tensors[t].type);
    }
    const int64_t most = most_units(n_tensors, numels.data());
    const size_t need = layout(nullptr, nullptr, n_tensors, most, n_groups);
    if (dev_ws) {
        if (((uintptr_t)dev_ws & 255) || bytes < need) return SLAQ_E_NOMEM;
        h->ws = dev_ws;
    } else {
        if (!done(cudaMalloc(&h->ws, need))) return SLAQ_E_NOMEM;
        h->owns_ws = true;
    }
    layout(h, static_cast<char*>(h->ws), n_tensors, most, n_groups);
    auto to_device = [&](void* to, const void* from, size_t n) { return n == 0 || done(cudaMemcpyAsync(to, from, n, cudaMemcpyHostToDevice, st)); };
    if (!to_device(h->tensors, h->refs.data(), sizeof(GradRef) * h->refs.size()) || !to_device(h->groups, groups.data(), sizeof(GroupRef) * groups.size()) ||
        !done(cudaMemsetAsync(h->ticket, 0, sizeof(unsigned int), st)))
        return SLAQ_E_CUDA;
    if (n_tensors && !launch(fill_grad_units_kernel, n_tensors, 256, st, h->tensors, h->tensor_of)) return SLAQ_E_CUDA;
    return done(cudaStreamSynchronize(st)) ? SLAQ_OK : SLAQ_E_CUDA;   // the lists above end here
}

}  // namespace
}  // namespace slaq

extern "C" {

size_t slaq_grad_norms_workspace_bytes(int32_t n_tensors, const int64_t* numels, int32_t n_groups) {
    if (n_tensors < 0 || n_groups < 1 || (n_tensors && !numels) || !slaq::sizes_ok(n_tensors, numels, n_groups)) return 0;
    return slaq::layout(nullptr, nullptr, n_tensors, slaq::most_units(n_tensors, numels), n_groups);
}

int slaq_grad_norms_create(void* dev_ws, size_t bytes, int32_t n_tensors, const slaq_grad_tensor* tensors, int32_t n_groups, void* cuda_stream,
                           slaq_grad_norms_t** out) {
    if (!out) return SLAQ_E_ARG;
    *out = nullptr;
    if (n_tensors < 0 || n_groups < 1 || (n_tensors && !tensors)) return SLAQ_E_ARG;
    slaq_grad_norms_handle* h = new (std::nothrow) slaq_grad_norms_handle();
    if (!h) return SLAQ_E_NOMEM;
    int rc;
    try {
        rc = slaq::create(h, dev_ws, bytes, n_tensors, tensors, n_groups, static_cast<cudaStream_t>(cuda_stream));
    } catch (const std::bad_alloc&) {
        rc = SLAQ_E_NOMEM;
    }
    if (rc < 0) {
        slaq_grad_norms_destroy(h);
        return rc;
    }
    *out = h;
    return SLAQ_OK;
}

int slaq_grad_norms_destroy(slaq_grad_norms_t* h) {
    if (!h) return SLAQ_OK;
    if (h->owns_ws && h->ws) slaq::done(cudaFree(h->ws));   // waits for the calls that still read it
    delete h;
    return SLAQ_OK;
}

const char* slaq_grad_norms_last_error(const slaq_grad_norms_t* h) { return h ? h->err : "null handle"; }

int slaq_grad_norms_measure(slaq_grad_norms_t* h, const int32_t* d_active, double scale, double max_norm, const float* d_max_norms, float* d_out_norm,
                            float* d_out_factor, void* cuda_stream) {
    if (!h) return SLAQ_E_ARG;
    if (!slaq::on_device(h)) return slaq::fail(h, SLAQ_E_ARG, "the plan's device is not the current one");
    if (!d_out_norm || !slaq::aligned(d_active) || !slaq::aligned(d_max_norms, d_out_norm, d_out_factor))
        return slaq::fail(h, SLAQ_E_ARG, "an address is null or not aligned to its type");
    if (!(std::fabs(scale) < 3.4e38) || !(max_norm >= 0.0)) return slaq::fail(h, SLAQ_E_ARG, "scale is not finite in 32 bits, or max_norm is negative or NaN");
    const int teams = slaq::kThreads / h->team, rounds = (h->n_groups + teams - 1) / teams;
    const bool join_here = rounds <= slaq::kMostRounds;
    slaq::NormArgs a = {h->tensors, h->groups, h->tensor_of, h->sums, h->n_units, h->n_groups, h->team, join_here, d_active, d_max_norms,
                        std::fabs(scale), max_norm, d_out_norm, d_out_factor, h->ticket};
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return slaq::launch(slaq::norm_kernel, h->norm_grid, slaq::kThreads, st, a) &&
                   (join_here || slaq::launch(slaq::join_kernel, std::min(rounds, 148 * 8), slaq::kThreads, st, a))
               ? SLAQ_OK : slaq::fail(h, SLAQ_E_CUDA, "the norms could not be launched");
}

int slaq_grad_norms_apply(slaq_grad_norms_t* h, const int32_t* d_active, const float* d_factor, void* cuda_stream) {
    if (!h) return SLAQ_E_ARG;
    if (!slaq::on_device(h)) return slaq::fail(h, SLAQ_E_ARG, "the plan's device is not the current one");
    if (!d_factor || !slaq::aligned(d_active) || !slaq::aligned(d_factor)) return slaq::fail(h, SLAQ_E_ARG, "an address is null or not aligned to its type");
    slaq::ApplyArgs a = {h->tensors, h->tensor_of, h->n_units, d_active, d_factor};
    return slaq::launch(slaq::apply_kernel, h->apply_grid, slaq::kThreads, static_cast<cudaStream_t>(cuda_stream), a)
               ? SLAQ_OK : slaq::fail(h, SLAQ_E_CUDA, "the factors could not be launched");
}

int slaq_grad_norms_set_grads(slaq_grad_norms_t* h, const void* const* grads, void* cuda_stream) {
    if (!h) return SLAQ_E_ARG;
    if (!slaq::on_device(h)) return slaq::fail(h, SLAQ_E_ARG, "the plan's device is not the current one");
    if (h->n_tensors == 0) return SLAQ_OK;
    if (!grads) return slaq::fail(h, SLAQ_E_ARG, "grads is null");
    try {
        std::vector<slaq::GradRef> refs = h->refs;
        for (int32_t t = 0; t < h->n_tensors; ++t) {
            refs[t].grad = grads[t];
            if (h->in_place[t]) refs[t].out = const_cast<void*>(grads[t]);
        }
        const char* what = "";
        if (const int rc = slaq::check(refs, &what)) return slaq::fail(h, rc, what);
        if (slaq::captured(static_cast<cudaStream_t>(cuda_stream)))
            return slaq::fail(h, SLAQ_E_ARG, "gradients are not changed while the stream is captured");
        if (!slaq::done(cudaMemcpyAsync(h->tensors, refs.data(), sizeof(slaq::GradRef) * refs.size(), cudaMemcpyHostToDevice, static_cast<cudaStream_t>(cuda_stream))))
            return slaq::fail(h, SLAQ_E_CUDA, "copy of the gradients' addresses");
        h->refs.swap(refs);
    } catch (const std::bad_alloc&) {
        return slaq::fail(h, SLAQ_E_NOMEM, "out of memory");
    }
    return SLAQ_OK;
}

}  // extern "C"
