// Log probabilities of given classes, entropy and the most probable classes of rows of logits.
//
//   lse = m + log s,  m = max x,  s = sum e^(x - m);   log p(c) = x_c - lse
//   entropy = -sum p log p = log s - u / s,  u = sum e^(x - m) (x - m)
//
// Bound: memory; the logits are read once.  Every thread keeps m, s and u of its own share; where that fits its registers
// (RES) it is held there and m is known before the first exponential, else s and u are brought down whenever a larger m comes
// (e^d, d = old - new: s' = e^d s, u' = e^d (u + d s)).  Shares are joined the same way.  Exponentials, sums and products are
// packed in pairs: 5.5 instructions a bf16 logit instead of 8.5.
//
// The k most probable classes come out of the same pass: the threads of a team are dealt to groups, and the k-th largest of
// the groups' maxima is a bound that at least k classes reach and few more.  Only threads whose own maximum reaches it look
// at their share again (k = 20 of 131072 classes: about 24 of 256), and what they find is put in order by counting, value
// first, lower index first.  Rows in which too many classes reach the bound take their ties in the order of their indexes,
// or, when even the classes above it do not fit the list, one sweep a class.
//
// A row is worked on by a warp (many short rows), by a CTA, or, when rows are few, by the CTAs of a cluster.
#include <algorithm>
#include <cmath>

#include "common.h"
#include "mxfp4.cuh"
#include "pipeline.cuh"

namespace sbnn {
namespace {

constexpr int kMaxTop = SBNN_LOGPROBS_MAX_TOP;
constexpr int kHeld = 8;        // 16-byte vectors of a row that a thread holds (RES)
constexpr float kLog2E = 1.4426950408889634f;
constexpr float kFar = -1e30f;   // differences below it count as it: e^kFar = 0, and 0 * kFar is 0, which 0 * -inf is not

__device__ __forceinline__ float exp2_of(float t) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));
    return r;
}
__device__ __forceinline__ float exp_of(float d) { return exp2_of(d * kLog2E); }
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
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
// The same sums over a larger maximum.
__device__ __forceinline__ Sums lower(const Sums& a, float m) {
    if (a.m == m) return a;
    const float d = fmaxf(a.m - m, kFar), e = exp_of(d);
    return {m, a.s * e, e * (a.u + d * a.s)};
}
__device__ __forceinline__ Sums join(const Sums& a, const Sums& b) {
    const float m = fmaxf(a.m, b.m);
    const Sums x = lower(a, m), y = lower(b, m);
    return {m, x.s + y.s, x.u + y.u};
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
    __device__ __forceinline__ void fill(float f) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = from_float<T>(f);
    }
};
// The largest of a vector (a NaN only if there is nothing else).
__device__ __forceinline__ float largest(const Vec<float>& q) { return fmaxf(fmaxf(q.v[0], q.v[1]), fmaxf(q.v[2], q.v[3])); }
__device__ __forceinline__ float largest(const Vec<__half>& q) {
    const __half2* w = reinterpret_cast<const __half2*>(q.v);
    const __half2 m = __hmax2(__hmax2(w[0], w[1]), __hmax2(w[2], w[3]));
    return fmaxf(__low2float(m), __high2float(m));
}
__device__ __forceinline__ float largest(const Vec<__nv_bfloat16>& q) {
    const __nv_bfloat162* w = reinterpret_cast<const __nv_bfloat162*>(q.v);
    const __nv_bfloat162 m = __hmax2(__hmax2(w[0], w[1]), __hmax2(w[2], w[3]));
    return fmaxf(__low2float(m), __high2float(m));
}

// Sums over a base that stays, in pairs.
struct Pairs {
    f32x2 s, u;
    __device__ Pairs() : s(0), u(0) {}
    template <class T>
    __device__ __forceinline__ void add(const Vec<T>& q, f32x2 minus_base) {
#pragma unroll
        for (int j = 0; j < Vec<T>::N; j += 2) {
            float d0, d1, t0, t1;
            unpack2(add2(pack2(to_float(q.v[j]), to_float(q.v[j + 1])), minus_base), d0, d1);
            const f32x2 d = pack2(max_nan(d0, kFar), max_nan(d1, kFar));
            unpack2(mul2(d, dup2(kLog2E)), t0, t1);
            const f32x2 e = pack2(exp2_of(t0), exp2_of(t1));
            s = add2(s, e);
            fma2(u, e, d);
        }
    }
    __device__ __forceinline__ void lower_by(float d) {   // to a base larger by -d
        const float e = exp_of(d);
        fma2(u, dup2(d), s);
        u = mul2(u, dup2(e));
        s = mul2(s, dup2(e));
    }
    __device__ __forceinline__ Sums over(float m) const {
        float a, b, c, d;
        unpack2(s, a, b);
        unpack2(u, c, d);
        return {m, a + b, c + d};
    }
};
__device__ __forceinline__ f32x2 minus_base(float m) { return dup2(m == -INFINITY ? 0.f : -m); }

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
    static constexpr int CAP = NT == 32 ? 256 : 2048;
    alignas(16) unsigned long long list[CAP];   // two at a time
    unsigned long long best[kMaxTop];
    Sums sums[WARPS], total;
    alignas(16) uint32_t keys[GROUPS];   // read four at a time
    uint32_t bound;
    int scan[WARPS];
    int count;
    unsigned long long sweep[WARPS];
};
template <int NT>
__device__ __forceinline__ void team_sync() {
    if (NT == 32) __syncwarp();
    else __syncthreads();
}

// Whole warp: the top-th largest of the groups' maxima, the smallest of those that fewer than `top` exceed.
template <int NT>
__device__ __forceinline__ uint32_t bound_of(const Team<NT>& t, int top) {
    constexpr int H = Team<NT>::GROUPS / 32;
    uint32_t k[H], bound = ~0u;
    int rank[H];
#pragma unroll
    for (int h = 0; h < H; ++h) k[h] = t.keys[(threadIdx.x & 31) + 32 * h], rank[h] = 0;
#pragma unroll
    for (int j = 0; j < Team<NT>::GROUPS; j += 4) {
        const uint4 o = *reinterpret_cast<const uint4*>(t.keys + j);
#pragma unroll
        for (int h = 0; h < H; ++h) rank[h] += (o.x > k[h]) + (o.y > k[h]) + (o.z > k[h]) + (o.w > k[h]);
    }
#pragma unroll
    for (int h = 0; h < H; ++h)
        if (rank[h] < top) bound = min(bound, k[h]);
    return __reduce_min_sync(~0u, bound);
}
// The classes of a vector that reach the bound, into the list as far as it goes.
template <class T, int NT>
__device__ __forceinline__ void take(Team<NT>& t, const Row<T>& row, const Vec<T>& q, int v, float bound) {
    uint32_t hits = 0;
#pragma unroll
    for (int e = 0; e < Vec<T>::N; ++e) hits |= (uint32_t)(to_float(q.v[e]) >= bound || bound == -INFINITY) << e;   // NaN counts as -inf
    if (!hits) return;
    if (v < row.full0 || v >= row.full1)
#pragma unroll
        for (int e = 0; e < Vec<T>::N; ++e)
            if (!row.inside(v, e)) hits &= ~(1u << e);
    int at = atomicAdd(&t.count, __popc(hits));
#pragma unroll
    for (int e = 0; e < Vec<T>::N; ++e)
        if (hits >> e & 1) {
            if (at < Team<NT>::CAP) t.list[at] = entry_of(key_of(to_float(q.v[e])), row.index(v, e));
            ++at;
        }
}

// More classes reach the bound than the list holds: the first `top` of the vectors [v0, v1) of a row, without order, into t.list;
// returns how many there are (at least `top` of those that exist, `done`: t.best is complete already).
template <class T, int NT>
__device__ __noinline__ int take_many(Team<NT>& t, const Row<T> row, int v0, int v1, int top, uint32_t bound, bool* done) {
    constexpr int N = Vec<T>::N;
    const int id = threadIdx.x % NT, lane = id & 31, warp = id >> 5;
    *done = false;
    team_sync<NT>();
    if (id == 0) t.count = 0;
    team_sync<NT>();
    int own_above = 0;
    for (int v = v0 + id; v < v1; v += NT) {
        const Vec<T> q = row.load(v);
#pragma unroll
        for (int e = 0; e < N; ++e) own_above += key_of(to_float(q.v[e])) > bound && row.inside(v, e);
    }
    if (own_above) atomicAdd(&t.count, own_above);
    team_sync<NT>();
    const int above = t.count;
    if (above <= Team<NT>::CAP - kMaxTop) {
        // those above the bound, and of those on it as many as are wanted, lowest indexes first
        team_sync<NT>();
        if (id == 0) t.count = 0;
        team_sync<NT>();
        for (int v = v0 + id; v < v1; v += NT) {
            const Vec<T> q = row.load(v);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const uint32_t k = key_of(to_float(q.v[e]));
                if (k > bound && row.inside(v, e)) t.list[atomicAdd(&t.count, 1)] = entry_of(k, row.index(v, e));
            }
        }
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
        team_sync<NT>();
        return min(have, max(top, above));
    }
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
    *done = true;
    return 0;
}

// W threads of a team, numbered by `id`: the `top` largest of n entries (n at most CAP) in order into t.best; places without an entry get 0.
template <int NT, int W>
__device__ __forceinline__ void order(Team<NT>& t, int n, int top, int id) {
    const int whole = (n + 7) & ~7;
    for (int i = id; i < top; i += W) t.best[i] = 0;
    if (id < whole - n) t.list[n + id] = 0;
    if (W == 32) __syncwarp();
    else __syncthreads();
    for (int i = id; i < n; i += W) {
        const unsigned long long c = t.list[i];
        int rank = 0;
        for (int j = 0; j < whole; j += 8) {
            ulonglong2 o[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) o[q] = *reinterpret_cast<const ulonglong2*>(t.list + j + 2 * q);
#pragma unroll
            for (int q = 0; q < 4; ++q) rank += (o[q].x > c) + (o[q].y > c);
        }
        if (rank < top && c) t.best[rank] = c;
    }
    if (W == 32) __syncwarp();
    else __syncthreads();
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
template <class T, int NT, bool RES>
__global__ void __launch_bounds__(256, 4)
logprobs_kernel(const Params p) {
    constexpr int TEAMS = NT == 32 ? 8 : 1, WARPS = Team<NT>::WARPS, GL = NT / Team<NT>::GROUPS, U = 4;
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
    const int mine0 = v0 + id;

    // the thread's share
    Vec<T> held[RES ? kHeld : 1];
    Sums a = {-INFINITY, 0.f, 0.f};
    Pairs sums;
    if (RES) {
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const int v = mine0 + i * NT;
            if (v < v1 && v >= row.full0 && v < row.full1) held[i] = row.load_full(v);
            else held[i].fill(-INFINITY);
        }
        // the first and the last vector of the row may be partly outside it
        for (int e = 0; e < 2; ++e) {
            const int v = e ? row.vectors - 1 : 0;
            if ((e ? row.full1 != row.vectors : row.full0) && v >= v0 && v < v1 && (v - v0) % NT == id) {
                const Vec<T> q = row.load(v);
#pragma unroll
                for (int i = 0; i < kHeld; ++i)
                    if (mine0 + i * NT == v) held[i] = q;
            }
        }
#pragma unroll
        for (int i = 0; i < kHeld; ++i) a.m = fmaxf(a.m, largest(held[i]));
        const f32x2 base = minus_base(a.m);
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            if (mine0 + i * NT < v1) sums.add(held[i], base);
    } else {
        auto raise = [&](float m) {
            if (m > a.m) {
                sums.lower_by(fmaxf(a.m - m, kFar));
                a.m = m;
            }
        };
        auto one = [&](int v) {
            const Vec<T> q = row.load(v);
            raise(largest(q));
            sums.add(q, minus_base(a.m));
        };
        int v = mine0;
        if (v < v1) one(v);
        v += NT;
        const int end = min(v1, row.full1);
        // U vectors are on their way while the U before them are added up
        if (v + (U - 1) * NT < end) {
            Vec<T> q[U];
#pragma unroll
            for (int i = 0; i < U; ++i) q[i] = row.load_full(v + i * NT);
            v += U * NT;
#pragma unroll 1
            for (;;) {
                const bool more = v + (U - 1) * NT < end;
                Vec<T> next[U];
                if (more)
#pragma unroll
                    for (int i = 0; i < U; ++i) next[i] = row.load_full(v + i * NT);
                float m = largest(q[0]);
#pragma unroll
                for (int i = 1; i < U; ++i) m = fmaxf(m, largest(q[i]));
                raise(m);
                const f32x2 base = minus_base(a.m);
#pragma unroll
                for (int i = 0; i < U; ++i) sums.add(q[i], base);
                if (!more) break;
#pragma unroll
                for (int i = 0; i < U; ++i) q[i] = next[i];
                v += U * NT;
            }
        }
        for (; v < v1; v += NT) one(v);
    }
    a = sums.over(a.m);

    // the groups' maxima; from them the row's, to which everybody brings down its sums, and the bound
    const uint32_t mine = mine0 < v1 ? key_of(a.m) : 0u;
    uint32_t g = mine;
#pragma unroll
    for (int o = 1; o < GL; o <<= 1) g = max(g, __shfl_xor_sync(~0u, g, o));
    if (id % GL == 0) t.keys[id / GL] = g;
    if (id == 0) t.count = 0;
    team_sync<NT>();
    uint32_t most = t.keys[lane];
    if (NT > 32) most = max(most, t.keys[lane + 32]);
    most = __reduce_max_sync(~0u, most);
    a = lower(a, value_of(most));
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        a.s += __shfl_xor_sync(~0u, a.s, o);
        a.u += __shfl_xor_sync(~0u, a.u, o);
    }
    if (NT > 32) {
        if (lane == 0) t.sums[warp] = a;
        if (p.top > 1 && warp == WARPS - 1) {
            const uint32_t b = bound_of<NT>(t, p.top);
            if (lane == 0) t.bound = b;
        }
        __syncthreads();
    }
    if (p.top) {
        const uint32_t bound = p.top == 1 ? most : NT == 32 ? bound_of<NT>(t, p.top) : t.bound;
        // The lanes of a warp read the shares of those among them that reach the bound again, from the L1 or the L2: of four at
        // a time where a share is no more than kHeld vectors.
        constexpr int L = RES ? kHeld : 32;   // lanes that look at a share
        const float least = bound ? value_of(bound) : -INFINITY;
        const int share = (v1 - v0 + NT - 1) / NT;
        for (uint32_t who = __ballot_sync(~0u, mine >= bound && mine); who;) {
            int from = -1;
#pragma unroll
            for (int q = 0; q < 32 / L; ++q) {
                if (lane / L == q && who) from = __ffs(who) - 1;
                who &= who - 1;
            }
            const int first = __shfl_sync(~0u, mine0, from & 31);
            if (from >= 0)
                for (int j = lane % L, v = first + j * NT; j < share && v < v1; j += L, v += L * NT) take<T, NT>(t, row, row.load(v), v, least);
        }
        team_sync<NT>();
        int n = t.count;
        bool done = false;
        if (n > Team<NT>::CAP) n = take_many<T, NT>(t, row, v0, v1, p.top, bound, &done);
        if (warp == 0 && !done) order<NT, 32>(t, n, p.top, lane);
    }
    if (NT > 32) {
        // the rest is the first warp's, of the first part
        if (warp == 0) {
            a = lane < WARPS ? t.sums[lane] : Sums{a.m, 0.f, 0.f};
#pragma unroll
            for (int o = WARPS / 2; o; o >>= 1) {
                a.s += __shfl_xor_sync(~0u, a.s, o);
                a.u += __shfl_xor_sync(~0u, a.u, o);
            }
            a.s = __shfl_sync(~0u, a.s, 0), a.u = __shfl_sync(~0u, a.u, 0);
        }
        if (p.parts > 1) {
            if (id == 0) t.total = a;
            cluster_sync();
            if (part == 0 && warp == 0) {
                for (int c = 1; c < p.parts; ++c) {
                    const Sums b = {load_remote(&t.total.m, c), load_remote(&t.total.s, c), load_remote(&t.total.u, c)};
                    a = join(a, b);
                }
            }
            if (part == 0 && p.top) {
                const int n = p.parts * p.top;   // at most NT
                if (id < n) t.list[id] = load_remote(&t.best[id % p.top], id / p.top);
                __syncthreads();
                order<NT, NT>(t, n, p.top, id);
            }
            cluster_sync();
        }
        if (part || warp) return;
    }
    const float log_s = logf(a.s);
    if (lane == 0 && p.entropy) p.entropy[r] = log_s - a.u / a.s;
    for (int i = lane; i < p.ntargets; i += 32) {
        const int32_t c = p.targets[r * p.ntargets + i];
        float f = 0.f;
        if (c >= p.classes) f = NAN;
        else if (c >= 0) f = (to_float(row.x[c]) - a.m) - log_s;
        p.logprob[r * p.ntargets + i] = f;
    }
    for (int i = lane; i < p.top; i += 32) {
        const unsigned long long c = t.best[i];
        p.top_index[r * p.top + i] = (int32_t)~(uint32_t)c;
        p.top_logprob[r * p.top + i] = (value_of((uint32_t)(c >> 32)) - a.m) - log_s;
    }
}

template <class T>
sbnn_status launch_as(const Params& given, cudaStream_t st) {
    Params p = given;
    // vectors of a row at most: one more where rows start anywhere
    const bool whole = p.ld % Vec<T>::N == 0;
    const int64_t vectors = ((int64_t)p.classes + (whole ? 1 : 2) * (Vec<T>::N - 1)) / Vec<T>::N;
    const int sms = device_sms();
    p.parts = 1;
    ChainedLaunchScope chained;
    if (vectors <= 32 * kHeld && p.rows >= 8 * sms) {
        SBNN_CUDA_TRY(launch_kernel(logprobs_kernel<T, 32, true>, dim3((unsigned)((p.rows + 7ll) / 8)), dim3(256), 0, st, p));
        return SBNN_OK;
    }
    while (p.parts < 8 && (int64_t)p.rows * p.parts * 2 <= 2 * sms && vectors / (p.parts * 2) >= 256) p.parts *= 2;
    if ((int64_t)p.rows * p.parts > 0x7fffffff) return fail(SBNN_ERR_SHAPE, "too many rows");
    // a part has at most one vector more than its share
    auto* const kernel = (vectors + p.parts - 1) / p.parts <= 256 * kHeld ? logprobs_kernel<T, 256, true> : logprobs_kernel<T, 256, false>;
    SBNN_CUDA_TRY(launch_kernel_cluster(kernel, dim3((unsigned)(p.rows * p.parts)), dim3(256), 0, st, (unsigned)p.parts, p));
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
