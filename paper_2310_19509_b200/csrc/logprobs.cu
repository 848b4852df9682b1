// Log probabilities of given classes, entropy and the most probable classes of rows of logits.
//
//   lse = m + log s,  m = max x,  s = sum e^(x - m);   log p(c) = x_c - lse
//   entropy = -sum p log p = log s - u / s,  u = sum e^(x - m) (x - m)
//
// Bound: memory; the logits are read once.  Every thread keeps m, s and u of its own share and brings s and u down to a new
// maximum only when one comes (e^d, d = old - new: s' = e^d s, u' = e^d (u + d s)); shares are joined the same way.
//
// The k most probable classes come out of the same pass: the threads of a team are dealt to groups, and the k-th largest of
// the groups' maxima is a bound that at least k classes reach and few more.  Only threads whose own maximum reaches it go
// over their share again (k = 20 of 131072 classes: about 24 threads of 512, whose vectors all lanes of the team load
// together), and what they find is put in order by counting, value first, lower index first.  Rows in which too many classes
// reach the bound take their ties in the order of their indexes, or, when even the classes above it do not fit the list, one
// sweep a class.
//
// A row is worked on by a warp, by a CTA, or, when rows are fewer than SMs, by the CTAs of a cluster.
#include <algorithm>
#include <cmath>

#include "common.h"
#include "mxfp4.cuh"
#include "pipeline.cuh"

namespace sbnn {
namespace {

constexpr int kMaxTop = SBNN_LOGPROBS_MAX_TOP;
constexpr float kLog2E = 1.4426950408889634f;
constexpr float kFar = -1e30f;   // differences below it count as it: e^kFar = 0, and 0 * kFar is 0, which 0 * -inf is not

__device__ __forceinline__ float exp_of(float d) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d * kLog2E));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// Order of values: larger keys first.  -0 equals 0, NaN counts as -inf, 0 is below every value.
__device__ __forceinline__ uint32_t key_of(float v) {
    if (v != v) v = -INFINITY;
    const uint32_t b = __float_as_uint(v + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key); }
__device__ __forceinline__ unsigned long long entry_of(uint32_t key, int index) { return ((unsigned long long)key << 32) | (uint32_t)~index; }

struct Sums {
    float m, s, u;
};
__device__ __forceinline__ Sums join(const Sums& a, const Sums& b) {
    const float m = fmaxf(a.m, b.m);
    const float da = a.m == m ? 0.f : fmaxf(a.m - m, kFar), db = b.m == m ? 0.f : fmaxf(b.m - m, kFar);
    const float ea = exp_of(da), eb = exp_of(db);
    return {m, a.s * ea + b.s * eb, ea * (a.u + da * a.s) + eb * (b.u + db * b.s)};
}

// N values of a row, all at once: N / 2 packed pairs.
template <int N>
__device__ __forceinline__ void add_values(Sums& t, const float (&x)[N]) {
    float m = x[0];
#pragma unroll
    for (int i = 1; i < N; ++i) m = fmaxf(m, x[i]);
    if (m > t.m) {
        const float d = fmaxf(t.m - m, kFar), e = exp_of(d);
        t.u = e * (t.u + d * t.s);
        t.s *= e;
        t.m = m;
    }
    const float base = t.m == -INFINITY ? 0.f : t.m;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float d = max_nan(x[i] - base, kFar), e = exp_of(d);
        t.s += e;
        t.u = fmaf(e, d, t.u);
    }
}

struct Params {
    const void* x;
    const int32_t* targets;
    float *logprob, *entropy, *top_logprob;
    int32_t* top_index;
    int64_t ld;
    int rows, classes, ntargets, top, parts;
};

template <class T>
struct Vec {   // 16 bytes of a row
    static constexpr int N = 16 / (int)sizeof(T);
    alignas(16) T v[N];
};

// A row as 16-byte vectors on 16-byte boundaries; the first and the last may lie partly outside it.
template <class T>
struct Row {
    static constexpr int N = Vec<T>::N;
    const T* x;       // the row's first class
    int classes;
    int lead;         // places of vector 0 that are before the row
    int vectors;
    int full0, full1; // vectors [full0, full1) lie inside the row altogether
    __device__ Row(const T* row, int n) : x(row), classes(n) {
        lead = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
        vectors = (int)(((int64_t)lead + n + N - 1) / N);
        full0 = lead ? 1 : 0;
        full1 = (int)(((int64_t)lead + n) / N);
    }
    __device__ int index(int v, int j) const { return v * N - lead + j; }
    __device__ Vec<T> load_full(int v) const {
        Vec<T> r;
        *reinterpret_cast<uint4*>(r.v) = __ldg(reinterpret_cast<const uint4*>(x - lead) + v);
        return r;
    }
    // Values that are not of the row come as -inf; callers that look at single values ask inside() as well.
    __device__ Vec<T> load(int v) const {
        if (v >= full0 && v < full1) return load_full(v);
        Vec<T> r;
#pragma unroll
        for (int j = 0; j < N; ++j) r.v[j] = inside(v, j) ? __ldg(x + index(v, j)) : from_float<T>(-INFINITY);
        return r;
    }
    __device__ bool inside(int v, int j) const { return (uint32_t)index(v, j) < (uint32_t)classes; }
};

// Candidates and scratch of a team of NT threads.
template <int NT>
struct Team {
    static constexpr int WARPS = NT / 32;
    static constexpr int GROUPS = NT == 32 ? 32 : 64;
    static constexpr int CAP = NT == 512 ? 2048 : NT == 128 ? 1024 : 256;
    unsigned long long list[CAP], best[kMaxTop];
    Sums sums[WARPS], total;
    uint32_t keys[GROUPS];
    int flagged[NT];
    int scan[WARPS];
    int count, nflagged, ties;
    unsigned long long sweep[WARPS];
};
template <int NT>
__device__ __forceinline__ void team_sync() {
    if (NT == 32) __syncwarp();
    else __syncthreads();
}

// The `top` first of the vectors [v0, v1) of a row into t.best, in order; places that have no class get 0.
// mine: the key of the calling thread's largest value among vectors v0 + id, v0 + id + NT, ...; 0 without any.
template <class T, int NT>
__device__ void pick_top(Team<NT>& t, const Row<T>& row, int v0, int v1, int top, uint32_t mine) {
    constexpr int N = Vec<T>::N, GL = NT / Team<NT>::GROUPS;   // lanes of a group
    const int id = threadIdx.x % NT, lane = id & 31, warp = id >> 5;
    uint32_t g = mine;
#pragma unroll
    for (int o = 1; o < GL; o <<= 1) g = max(g, __shfl_xor_sync(~0u, g, o));
    if (id % GL == 0) t.keys[id / GL] = g;
    if (id == 0) t.count = t.nflagged = t.ties = 0;
    for (int i = id; i < top; i += NT) t.best[i] = 0;
    team_sync<NT>();
    // the top-th largest of the groups' maxima (their order among equal ones does not matter)
    uint32_t bound = 0;
#pragma unroll
    for (int h = 0; h < Team<NT>::GROUPS / 32; ++h) {
        const uint32_t k = t.keys[lane + 32 * h];
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < Team<NT>::GROUPS; ++j) rank += t.keys[j] > k || (t.keys[j] == k && j < lane + 32 * h);
        const uint32_t who = __ballot_sync(~0u, rank == top - 1);
        if (who) bound = __shfl_sync(~0u, k, __ffs(who) - 1);
    }
    if (mine >= bound && mine) t.flagged[atomicAdd(&t.nflagged, 1)] = id;
    team_sync<NT>();
    const int nflagged = t.nflagged, share = (v1 - v0 + NT - 1) / NT;
    for (int i = warp; i < nflagged; i += Team<NT>::WARPS) {
        const int first = v0 + t.flagged[i];
        for (int j = lane; j < share; j += 32) {
            const int v = first + j * NT;
            if (v >= v1) break;
            const Vec<T> q = row.load(v);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const uint32_t k = key_of(to_float(q.v[e]));
                if (k >= bound && row.inside(v, e)) {
                    if (k == bound) atomicAdd(&t.ties, 1);
                    const int at = atomicAdd(&t.count, 1);
                    if (at < Team<NT>::CAP) t.list[at] = entry_of(k, row.index(v, e));
                }
            }
        }
    }
    team_sync<NT>();
    int n = t.count;
    const int ties = t.ties;
    if (n > Team<NT>::CAP && n - ties <= Team<NT>::CAP - kMaxTop) {
        // those above the bound, and of those on it as many as are wanted, lowest indexes first
        team_sync<NT>();
        if (id == 0) t.count = 0;
        team_sync<NT>();
        for (int i = warp; i < nflagged; i += Team<NT>::WARPS) {
            const int first = v0 + t.flagged[i];
            for (int j = lane; j < share; j += 32) {
                const int v = first + j * NT;
                if (v >= v1) break;
                const Vec<T> q = row.load(v);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const uint32_t k = key_of(to_float(q.v[e]));
                    if (k > bound && row.inside(v, e)) t.list[atomicAdd(&t.count, 1)] = entry_of(k, row.index(v, e));
                }
            }
        }
        team_sync<NT>();
        const int above = t.count;
        int have = above;
        for (int c = v0; c < v1 && have < top; c += NT) {
            const int v = c + id;
            uint32_t on = 0;   // one bit a value
            if (v < v1) {
                const Vec<T> q = row.load(v);
#pragma unroll
                for (int e = 0; e < N; ++e) on |= (uint32_t)(key_of(to_float(q.v[e])) == bound && row.inside(v, e)) << e;
            }
            const int own = __popc(on);
            int before = own;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int w = __shfl_up_sync(~0u, before, o);
                if (lane >= o) before += w;
            }
            if (lane == 31) t.scan[warp] = before;
            team_sync<NT>();
            int all = 0;
            before -= own;
            for (int w = 0; w < Team<NT>::WARPS; ++w) {
                if (w < warp) before += t.scan[w];
                all += t.scan[w];
            }
            for (uint32_t b = on; b && have + before < top; b &= b - 1, ++before) t.list[have + before] = entry_of(bound, row.index(v, __ffs(b) - 1));
            have += all;
            team_sync<NT>();
        }
        n = min(have, max(top, above));
    } else if (n > Team<NT>::CAP) {
        unsigned long long last = ~0ull;
        for (int i = 0; i < top; ++i) {
            unsigned long long best = 0;
            for (int v = v0 + id; v < v1; v += NT) {
                const Vec<T> q = row.load(v);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const unsigned long long c = entry_of(key_of(to_float(q.v[e])), row.index(v, e));
                    if (row.inside(v, e) && c < last && c > best) best = c;
                }
            }
#pragma unroll
            for (int o = 16; o; o >>= 1) best = max(best, __shfl_xor_sync(~0u, best, o));
            if (lane == 0) t.sweep[warp] = best;
            team_sync<NT>();
            for (int w = 0; w < Team<NT>::WARPS; ++w) best = max(best, t.sweep[w]);
            if (id == 0) t.best[i] = best;
            last = best;
            team_sync<NT>();
        }
        return;
    }
    for (int i = id; i < n; i += NT) {
        const unsigned long long c = t.list[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += t.list[j] > c;
        if (rank < top) t.best[rank] = c;
    }
    team_sync<NT>();
}

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
template <class V>
__device__ __forceinline__ V load_remote(const V* p, int rank) {
    static_assert(sizeof(V) == 4 || sizeof(V) == 8, "one word");
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    V r;
    if (sizeof(V) == 4) {
        uint32_t w;
        asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(w) : "r"(a) : "memory");
        *reinterpret_cast<uint32_t*>(&r) = w;
    } else {
        unsigned long long w;
        asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(w) : "r"(a) : "memory");
        *reinterpret_cast<unsigned long long*>(&r) = w;
    }
    return r;
}

// NT = 32: eight rows a CTA, a warp each; else a row, or with parts > 1 one of the parts of a row that a cluster shares.
template <class T, int NT>
__global__ void __launch_bounds__(NT == 32 ? 256 : NT)
logprobs_kernel(const Params p) {
    constexpr int TEAMS = NT == 32 ? 8 : 1, N = Vec<T>::N, U = 4;
    __shared__ Team<NT> teams[TEAMS];
    grid_dependency_wait();
    grid_dependency_release();
    Team<NT>& t = teams[threadIdx.x / NT];
    const int id = threadIdx.x % NT, lane = id & 31, warp = id >> 5;
    const int64_t r = NT == 32 ? (int64_t)blockIdx.x * TEAMS + threadIdx.x / NT : blockIdx.x / p.parts;
    const int part = NT == 32 ? 0 : blockIdx.x % p.parts;
    if (r >= p.rows) return;   // whole warps, and never part of a cluster
    const Row<T> row(static_cast<const T*>(p.x) + r * p.ld, p.classes);
    const int v0 = (int)((int64_t)row.vectors * part / p.parts), v1 = (int)((int64_t)row.vectors * (part + 1) / p.parts);

    Sums a = {-INFINITY, 0.f, 0.f};
    auto one = [&](const Vec<T>& q) {
        float f[N];
#pragma unroll
        for (int j = 0; j < N; ++j) f[j] = to_float(q.v[j]);
        add_values(a, f);
    };
    int v = v0 + id;
    if (v < v1) one(row.load(v));
    v += NT;
    const int end = min(v1, row.full1);
    for (; v + (U - 1) * NT < end; v += U * NT) {
        Vec<T> q[U];
#pragma unroll
        for (int i = 0; i < U; ++i) q[i] = row.load_full(v + i * NT);
        float f[U * N];
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) f[i * N + j] = to_float(q[i].v[j]);
        add_values(a, f);
    }
    for (; v < v1; v += NT) one(row.load(v));

    if (p.top) pick_top<T, NT>(t, row, v0, v1, p.top, v0 + id < v1 ? key_of(a.m) : 0u);

#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const Sums b = {__shfl_xor_sync(~0u, a.m, o), __shfl_xor_sync(~0u, a.s, o), __shfl_xor_sync(~0u, a.u, o)};
        a = lane & o ? join(b, a) : join(a, b);   // the same order in both lanes
    }
    if (NT > 32) {
        if (lane == 0) t.sums[warp] = a;
        __syncthreads();
        a = t.sums[0];
        for (int w = 1; w < Team<NT>::WARPS; ++w) a = join(a, t.sums[w]);
    }
    if (NT > 32 && p.parts > 1) {
        if (id == 0) t.total = a;
        cluster_sync();
        if (part == 0) {
            for (int c = 1; c < p.parts; ++c) {
                const Sums b = {load_remote(&t.total.m, c), load_remote(&t.total.s, c), load_remote(&t.total.u, c)};
                a = join(a, b);
            }
            if (p.top) {
                const int n = p.parts * p.top;
                for (int i = id; i < n; i += NT) t.list[i] = i < p.top ? t.best[i] : load_remote(&t.best[i % p.top], i / p.top);
                __syncthreads();
                for (int i = id; i < n; i += NT) {
                    const unsigned long long c = t.list[i];
                    int rank = 0;
                    for (int j = 0; j < n; ++j) rank += t.list[j] > c;
                    if (rank < p.top && c) t.best[rank] = c;
                }
                __syncthreads();
            }
        }
        cluster_sync();
        if (part) return;
    }
    const float log_s = logf(a.s);
    if (id == 0 && p.entropy) p.entropy[r] = log_s - a.u / a.s;
    for (int i = id; i < p.ntargets; i += NT) {
        const int32_t c = p.targets[r * p.ntargets + i];
        float f = 0.f;
        if (c >= p.classes) f = NAN;
        else if (c >= 0) f = (to_float(row.x[c]) - a.m) - log_s;
        p.logprob[r * p.ntargets + i] = f;
    }
    for (int i = id; i < p.top; i += NT) {
        const unsigned long long c = t.best[i];
        p.top_index[r * p.top + i] = (int32_t)~(uint32_t)c;
        p.top_logprob[r * p.top + i] = (value_of((uint32_t)(c >> 32)) - a.m) - log_s;
    }
}

template <class T>
sbnn_status launch_as(const Params& given, cudaStream_t st) {
    Params p = given;
    const int64_t bytes = (int64_t)p.classes * sizeof(T);
    const int sms = device_sms();
    p.parts = 1;
    ChainedLaunchScope chained;
    if (bytes <= 4096 && p.rows >= 8 * sms) {
        SBNN_CUDA_TRY(launch_kernel(logprobs_kernel<T, 32>, dim3((unsigned)((p.rows + 7ll) / 8)), dim3(256), 0, st, p));
        return SBNN_OK;
    }
    if (bytes <= 16384) {
        SBNN_CUDA_TRY(launch_kernel(logprobs_kernel<T, 128>, dim3((unsigned)p.rows), dim3(128), 0, st, p));
        return SBNN_OK;
    }
    while (p.parts < 8 && (int64_t)p.rows * p.parts * 2 <= 2 * sms && bytes / (p.parts * 2) >= 8192) p.parts *= 2;
    if ((int64_t)p.rows * p.parts > 0x7fffffff) return fail(SBNN_ERR_SHAPE, "too many rows");
    SBNN_CUDA_TRY(launch_kernel_cluster(logprobs_kernel<T, 512>, dim3((unsigned)(p.rows * p.parts)), dim3(512), 0, st, (unsigned)p.parts, p));
    return SBNN_OK;
}

}  // namespace
}  // namespace sbnn

using namespace sbnn;

extern "C" sbnn_status sbnn_logprobs(const void* logits_dev, int type, int64_t ld, int rows, int classes, const int32_t* targets_dev, int ntargets,
                                     float* logprob_dev, float* entropy_dev, int top, int32_t* top_index_dev, float* top_logprob_dev,
                                     void* cuda_stream) {
    clear_error();
    if (!logits_dev) return fail(SBNN_ERR_NULL, "logits_dev must not be NULL");
    if (rows < 0 || classes <= 0 || ntargets < 0) return fail(SBNN_ERR_SHAPE, "bad shape rows=%d classes=%d ntargets=%d", rows, classes, ntargets);
    if (type != SBNN_F32 && type != SBNN_F16 && type != SBNN_BF16) return fail(SBNN_ERR_UNSUPPORTED, "logits_dev: unknown element type %d", type);
    if (classes > 1 << 30) return fail(SBNN_ERR_UNSUPPORTED, "%d classes: 2^30 at most", classes);
    if (ld < classes) return fail(SBNN_ERR_SHAPE, "rows of %d classes do not fit a stride of %lld", classes, (long long)ld);
    if (top < 0 || top > kMaxTop || top > classes)
        return fail(SBNN_ERR_SHAPE, "top=%d: 0 to %d, and not more than the %d classes", top, kMaxTop, classes);
    if (ntargets && (!targets_dev || !logprob_dev)) return fail(SBNN_ERR_NULL, "targets_dev and logprob_dev must not be NULL");
    if (top && (!top_index_dev || !top_logprob_dev)) return fail(SBNN_ERR_NULL, "top_index_dev and top_logprob_dev must not be NULL");
    if (!aligned16(logits_dev) || !aligned16(targets_dev) || !aligned16(logprob_dev) || !aligned16(entropy_dev) || !aligned16(top_index_dev) ||
        !aligned16(top_logprob_dev))
        return fail(SBNN_ERR_ALIGN, "device pointers must be 16-byte aligned");
    if (rows == 0) return SBNN_OK;
    const sbnn_status r = check_device();
    if (r != SBNN_OK) return r;
    Params p = {};
    p.x = logits_dev, p.targets = targets_dev, p.logprob = logprob_dev, p.entropy = entropy_dev;
    p.top_index = top_index_dev, p.top_logprob = top_logprob_dev;
    p.ld = ld, p.rows = rows, p.classes = classes, p.ntargets = ntargets, p.top = top;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    switch (type) {
        case SBNN_F32: return launch_as<float>(p, st);
        case SBNN_F16: return launch_as<__half>(p, st);
        default: return launch_as<__nv_bfloat16>(p, st);
    }
}
