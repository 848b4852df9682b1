// Log probabilities of given classes, entropy and the most probable classes of rows of logits.
//
//   t = (x - m) log2 e,  m = max x,  s = sum 2^t,  u = sum 2^t t;   log p(c) = (t_c - log2 s) ln 2
//   entropy = -sum p log p = (log2 s - u / s) ln 2
//
// Bound: memory; the logits are read once.  Every thread keeps m, s and u of its own share; where that fits its registers
// (RES) it is held there and m is known before the first exponential, else s and u are brought down whenever a larger m comes
// (2^d, d the old one's t: s' = 2^d s, u' = 2^d (u + d s)).  Shares are joined the same way.  Exponentials, sums and products are
// packed in pairs.
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

#include "cluster.cuh"
#include "common.h"
#include "mxfp4.cuh"
#include "pipeline.cuh"

namespace sbnn {
namespace {

constexpr int kMaxTop = SBNN_LOGPROBS_MAX_TOP;
constexpr int kHeld = 8;        // 16-byte vectors of a row that a thread holds (RES)
constexpr float kLog2E = 1.4426950408889634f;
constexpr float kFar = -1e30f;   // a t below it counts as it: 2^kFar = 0, and 0 * kFar is 0, which 0 * -inf is not

__device__ __forceinline__ float exp2_of(float t) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));
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

// s and u of a share, relative to its largest logit m: of t = (x - m) log2(e), s = sum 2^t, u = sum 2^t t.  The scaled base m log2(e)
// is rounded once, b, and t = x log2(e) - b in one step: what that rounding moves it moves in every term and in the answers' own t alike.
// Beyond kHuge, where that rounding is no small number any more, t is (x - m) log2(e).
struct Sums {
    float m, s, u;
};
constexpr float kHuge = 1e6f;
__device__ __forceinline__ bool small(float m) { return fabsf(m) <= kHuge; }
// The logarithm of a probability from the sums of a row.
__device__ __forceinline__ float log_of(float x, float m, float log2_s) {
    constexpr float kLn2 = 0.6931471805599453f;
    return small(m) && fabsf(x) <= 1e37f ? (fmaf(x, kLog2E, -__fmul_rn(m, kLog2E)) - log2_s) * kLn2 : (x - m) - log2_s * kLn2;
}
__device__ __forceinline__ float shift(float from, float to) {   // t of the old base over the new one
    if (from == to) return 0.f;
    const float old = __fmul_rn(from, kLog2E);
    const float d = small(to) ? (small(from) ? __fsub_rn(old, __fmul_rn(to, kLog2E)) : fmaf(from, kLog2E, -__fmul_rn(to, kLog2E)))
                              : (small(from) ? fmaf(-to, kLog2E, old) : (from - to) * kLog2E);
    return fmaxf(d, kFar);
}
// The same sums over a larger maximum.
__device__ __forceinline__ Sums lower(const Sums& a, float m) {
    if (a.m == m) return a;
    const float d = shift(a.m, m), e = exp2_of(d);
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

// Logits of at most kLeast may be taken for it where the largest is above kFast: their exponentials are 0 all the same, and t stays finite.
template <class T>
struct Least;
template <>
struct Least<float> {
    static constexpr float kLeast = -1e38f, kFast = -kHuge;
    static __device__ __forceinline__ void clamp(Vec<float>& q) {
#pragma unroll
        for (int j = 0; j < 4; ++j) q.v[j] = max_nan(q.v[j], kLeast);
    }
};
template <>
struct Least<__half> {
    static constexpr float kLeast = -65504.f, kFast = -60000.f;
    static __device__ __forceinline__ void clamp(Vec<__half>& q) {
        __half2* w = reinterpret_cast<__half2*>(q.v);
        const __half2 least = __float2half2_rn(kLeast);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = __hmax2_nan(w[j], least);
    }
};
template <>
struct Least<__nv_bfloat16> {
    static constexpr float kLeast = -1e38f, kFast = -kHuge;
    static __device__ __forceinline__ void clamp(Vec<__nv_bfloat16>& q) {
        __nv_bfloat162* w = reinterpret_cast<__nv_bfloat162*>(q.v);
        const __nv_bfloat162 least = __float2bfloat162_rn(kLeast);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = __hmax2_nan(w[j], least);
    }
};

// Element e of a vector.
template <class T>
__device__ __forceinline__ float element(const Vec<T>& q, int e) {
    const uint4 w = *reinterpret_cast<const uint4*>(q.v);
    const int i = sizeof(T) == 4 ? e : e >> 1;
    const uint32_t x = i & 2 ? (i & 1 ? w.w : w.z) : (i & 1 ? w.y : w.x);
    if (sizeof(T) == 4) return __uint_as_float(x);
    const unsigned short h = (unsigned short)(e & 1 ? x >> 16 : x);
    T v;
    *reinterpret_cast<unsigned short*>(&v) = h;
    return to_float(v);
}
// A thread's sums, in pairs.
struct Pairs {
    float m;
    float2 s, u;
    __device__ Pairs() : m(-INFINITY), s(make_float2(0.f, 0.f)), u(make_float2(0.f, 0.f)) {}
    __device__ __forceinline__ void term(float2 t) {
        const float2 e = make_float2(exp2_of(t.x), exp2_of(t.y));
        s = __fadd2_rn(s, e);
        u = __ffma2_rn(e, t, u);
    }
    // The base for these, whose largest is returned, and what they add.
    template <class T, int V>
    __device__ __forceinline__ float raise(const Vec<T> (&q)[V]) {
        float most = largest(q[0]);
#pragma unroll
        for (int i = 1; i < V; ++i) most = fmaxf(most, largest(q[i]));
        if (most > m) {
            const float d = shift(m, most), e = exp2_of(d);
            u = __fmul2_rn(__ffma2_rn(make_float2(d, d), s, u), make_float2(e, e));
            s = __fmul2_rn(s, make_float2(e, e));
            m = most;
        }
        return most;
    }
    // What the first `there` of them add.
    template <class T, int V>
    __device__ __forceinline__ void terms(Vec<T> (&q)[V], int there) {
        if (m > Least<T>::kFast && m <= kHuge) {
            const float b = -__fmul_rn(m, kLog2E);
            const float2 scale = make_float2(kLog2E, kLog2E), base = make_float2(b, b);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (i >= there) break;
                Least<T>::clamp(q[i]);
#pragma unroll
                for (int j = 0; j < Vec<T>::N; j += 2) {
                    term(__ffma2_rn(make_float2(to_float(q[i].v[j]), to_float(q[i].v[j + 1])), scale, base));
                }
            }
        } else {   // rare, and little code: see take()
            const bool huge = !small(m);
            const float from = huge && m > -INFINITY ? m : 0.f, base = huge ? 0.f : -__fmul_rn(m, kLog2E);
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll 1
                for (int j = 0; i < there && j < Vec<T>::N; j += 2)
                    term(make_float2(max_nan(fmaf(element(q[i], j) - from, kLog2E, base), kFar), max_nan(fmaf(element(q[i], j + 1) - from, kLog2E, base), kFar)));
        }
    }
    template <class T, int V>
    __device__ __forceinline__ void add(Vec<T> (&q)[V]) {
        raise(q);
        terms(q, V);
    }
    template <class T>
    __device__ __forceinline__ void add(Vec<T> q) {
        Vec<T> one[1] = {q};
        add(one);
    }
    __device__ __forceinline__ Sums all() const {
        return {m, s.x + s.y, u.x + u.y};
    }
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
    static constexpr int CAP = NT == 32 ? 256 : 768;   // candidates; behind them, in the first part's memory, the answers of a row's parts
    alignas(16) unsigned long long list[NT == 32 ? CAP : CAP + 8 * kMaxTop];   // two at a time
    unsigned long long best[kMaxTop];
    Sums sums[WARPS];
    Sums part_sums[NT == 32 ? 1 : 8];
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
// Whole warp: the same of all the keys that its lanes have (0: none), the largest number that at least `top` reach, or one below it
// that no more reach; 0 where fewer exist.
template <int V>
__device__ __forceinline__ uint32_t bound_of_all(const uint32_t (&keys)[V], int top) {
    uint32_t bound = 0;
#pragma unroll 1
    for (uint32_t bit = 0x80000000u; bit; bit >>= 1) {
        int reach = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) reach += keys[i] >= (bound | bit);
        reach = __reduce_add_sync(~0u, reach);
        if (reach >= top) bound |= bit;
        if (reach == top) break;
    }
    return bound;
}
// The classes of a vector that reach the bound, into the list as far as it goes.  (Little code, called from one place of a kernel: a row's
// end runs it once a warp, and what is not in the instruction cache then is waited for.  Unrolled over the elements and at
// several places it made the 20 most probable classes of 2048 x 131072 cost 61 us.)
template <class T, int NT>
__device__ __forceinline__ void take(Team<NT>& t, const Row<T>& row, const Vec<T>& q, int v, float bound) {
    uint32_t hits = 0;
#pragma unroll
    for (int e = 0; e < Vec<T>::N; ++e) hits |= (uint32_t)(to_float(q.v[e]) >= bound) << e;
    if (bound == -INFINITY) hits = (1u << Vec<T>::N) - 1;   // NaN counts as -inf
#pragma unroll 1
    for (; hits; hits &= hits - 1) {
        const int e = __ffs(hits) - 1;
        if (!row.inside(v, e)) continue;
        const int at = atomicAdd(&t.count, 1);
        if (at < Team<NT>::CAP) t.list[at] = entry_of(key_of(element(q, e)), row.index(v, e));
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

// What is left of a row, or of the part [v0, v1) of it that a CTA has, when every thread has its sums `a` (has: of at least one vector):
// joins them, finds the most probable classes and, in the first part, writes the answers.  scan(reaches, least), called by whole warps,
// takes what is least or more out of the shares of the threads that reach the bound.
// tighter, of a warp: a better bound for many alternatives than that of its lanes' maxima, 0 without one.
template <class T, int NT, bool SHARED, class Scan>
__device__ __forceinline__ void finish(Team<NT>& t, const Params& p, const Row<T>& row, int64_t r, int part, int v0, int v1, bool has, Sums a,
                                       uint32_t tighter, Scan scan) {
    constexpr int WARPS = Team<NT>::WARPS, GL = NT / Team<NT>::GROUPS;
    const int id = threadIdx.x % NT, lane = id & 31, warp = id >> 5;
    // the groups' maxima; from them the row's, to which everybody brings down its sums, and the bound
    const uint32_t mine = has ? key_of(a.m) : 0u;
    uint32_t g = mine;
#pragma unroll
    for (int o = 1; o < GL; o <<= 1) g = max(g, __shfl_xor_sync(~0u, g, o));
    if (id % GL == 0) t.keys[id / GL] = g;
    if (id == 0) t.count = 0;
    team_sync<NT>();
    uint32_t most = t.keys[lane];
    if (NT > 32) most = max(most, t.keys[lane + 32]);
    most = __reduce_max_sync(~0u, most);
    a = lower(a, most ? value_of(most) : -INFINITY);
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
        const uint32_t bound = p.top == 1 ? most : NT > 32 ? t.bound : tighter ? tighter : bound_of<NT>(t, p.top);
        scan(mine >= bound && mine, bound ? value_of(bound) : -INFINITY);
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
        if (SHARED && p.parts > 1) {
            // the parts' answers go to the first part's memory; only that waits for the others, which end here
            cluster_wait();   // all CTAs of the cluster have begun
            if (warp == 0) {
                if (lane == 0) {
                    store_remote(remote_address(smem_u32(&t.part_sums[part].m), 0), __float_as_uint(a.m));
                    store_remote(remote_address(smem_u32(&t.part_sums[part].s), 0), __float_as_uint(a.s));
                    store_remote(remote_address(smem_u32(&t.part_sums[part].u), 0), __float_as_uint(a.u));
                }
                for (int i = lane; i < p.top; i += 32) store_remote(remote_address(smem_u32(&t.list[Team<NT>::CAP + part * p.top + i]), 0), t.best[i]);
            }
            cluster_arrive();
            if (part) return;
            cluster_wait();
            if (warp == 0) {
                a = t.part_sums[0];
                for (int c = 1; c < p.parts; ++c) a = join(a, t.part_sums[c]);
            }
            if (p.top) {
                const int n = p.parts * p.top;   // at most NT
                if (id < n) t.list[id] = t.list[Team<NT>::CAP + id];
                __syncthreads();
                order<NT, NT>(t, n, p.top, id);
            }
        }
        if (warp) return;
    }
    const float log2_s = log2f(a.s);
    if (lane == 0 && p.entropy) p.entropy[r] = (log2_s - a.u / a.s) * 0.6931471805599453f;
    for (int i = lane; i < p.ntargets; i += 32) {
        const int32_t c = p.targets[r * p.ntargets + i];
        float f = 0.f;
        if (c >= p.classes) f = NAN;
        else if (c >= 0) f = log_of(to_float(row.x[c]), a.m, log2_s);
        p.logprob[r * p.ntargets + i] = f;
    }
    for (int i = lane; i < p.top; i += 32) {
        const unsigned long long c = t.best[i];
        p.top_index[r * p.top + i] = (int32_t)~(uint32_t)c;
        p.top_logprob[r * p.top + i] = log_of(value_of((uint32_t)(c >> 32)), a.m, log2_s);
    }
}

// Rows that the threads of a team hold (kHeld vectors a thread at most).  NT = 32: eight rows a CTA, a warp each; else a row, or
// with parts > 1 one of the parts of a row that a cluster shares.
template <class T, int NT>
__global__ void __launch_bounds__(NT == 32 ? 256 : NT, NT == 512 ? 2 : NT == 128 ? 8 : 4)
logprobs_held_kernel(const Params p) {
    constexpr int TEAMS = NT == 32 ? 8 : 1;
    __shared__ Team<NT> teams[TEAMS];
    if (NT > 32 && p.parts > 1) cluster_arrive();   // see finish()
    grid_dependency_wait();
    grid_dependency_release();
    Team<NT>& t = teams[threadIdx.x / NT];
    const int id = threadIdx.x % NT;
    const int64_t r = NT == 32 ? (int64_t)blockIdx.x * TEAMS + threadIdx.x / NT : blockIdx.x / p.parts;
    const int part = NT == 32 ? 0 : blockIdx.x % p.parts;
    if (r >= p.rows) return;   // whole warps, and never part of a cluster
    const Row<T> row(static_cast<const T*>(p.x) + r * p.ld, p.classes);
    const int v0 = (int)((int64_t)row.vectors * part / p.parts), v1 = (int)((int64_t)row.vectors * (part + 1) / p.parts);
    const int mine0 = v0 + id;
    Vec<T> held[kHeld];
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
    // Nearly as many alternatives as lanes: the bound comes from the vectors' maxima, of which there are more (1731 x 422 bf16, top 32,
    // 45 us without and 15 with: the least of the lanes' maxima is reached by more classes than the list holds; 4 x 302, top 20, 5.6
    // and 6.8).
    uint32_t tighter = 0;
    if (NT == 32 && p.top > 24 && v1 > 32) {
        uint32_t keys[kHeld];
#pragma unroll
        for (int i = 0; i < kHeld; ++i) keys[i] = mine0 + i * NT < v1 ? key_of(largest(held[i])) : 0u;
        tighter = bound_of_all(keys, p.top);
    }
    Pairs sums;
    sums.raise(held);   // places without a vector are -inf
    sums.terms(held, mine0 < v1 ? (v1 - mine0 + NT - 1) / NT : 0);
    finish<T, NT, (NT > 32)>(t, p, row, r, part, v0, v1, mine0 < v1, sums.all(), tighter, [&](bool reaches, float least) {
        // eight lanes a share read it again, from the L1 or the L2
        for (uint32_t who = __ballot_sync(~0u, reaches); who;) {
            int from = -1;
#pragma unroll
            for (int q = 0; q < 32 / kHeld; ++q) {
                if ((threadIdx.x & 31) / kHeld == q && who) from = __ffs(who) - 1;
                who &= who - 1;
            }
            const int first = __shfl_sync(~0u, mine0, from & 31), v = first + (int)(threadIdx.x % kHeld) * NT;
            if (from >= 0 && v < v1) take<T, NT>(t, row, row.load(v), v, least);
        }
    });
}

// Longer rows, or parts of them.  Every thread has a ring of its own in shared memory, which asynchronous copies fill: kAhead vectors
// a group, two groups on their way while one is added up, 128 KB an SM (through registers it was half of that, and 2048 x 131072 bf16
// took 114 us; bulk copies into a ring of the whole CTA, with barriers, 114).  The largest of a group, or of several, is kept (rounded
// up to bf16), so that of the shares that reach the bound only the groups that do are read again.
constexpr int kAhead = 4, kBuckets = 16;
constexpr int kStreamSmem = 2 * kAhead * 256 * 16;

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
template <class T, bool SHARED>
__global__ void __launch_bounds__(256, 4)
logprobs_stream_kernel(const Params p) {
    constexpr int NT = 256, GROUP = kAhead * NT;
    __shared__ Team<NT> t;
    __shared__ __nv_bfloat16 tops[kBuckets][NT];
    extern __shared__ __align__(1024) uint4 ring[];   // [2][kAhead][NT]
    grid_dependency_wait();
    grid_dependency_release();
    const int id = threadIdx.x, lane = id & 31;
    const int parts = SHARED ? p.parts : 1;
    const int64_t r = blockIdx.x / parts;
    const int part = blockIdx.x % parts;
    const Row<T> row(static_cast<const T*>(p.x) + r * p.ld, p.classes);
    const int v0 = (int)((int64_t)row.vectors * part / parts), v1 = (int)((int64_t)row.vectors * (part + 1) / parts);
    const int mine0 = v0 + id, end = min(v1, row.full1);
    // A thread's first vector, which may be partly outside the row, then whole groups of vectors, then what is left.
    auto groups_of = [&](int first) { return max(0, (end - first - 1) / GROUP); };
    const int groups = groups_of(mine0);
    int wide = 0;   // 2^wide groups share a bucket; the last bucket is for the vectors that are in no group
    while ((groups_of(v0) >> wide) >= kBuckets - 1) ++wide;

    const uint4* const from = reinterpret_cast<const uint4*>(row.x - row.lead) + mine0 + NT;
    const uint32_t slots = smem_u32(ring + id);
    auto ask = [&](int g) {
        if (g < groups)
#pragma unroll
            for (int i = 0; i < kAhead; ++i) copy16(slots + (uint32_t)(((g & 1) * kAhead + i) * NT * 16), from + (int64_t)g * GROUP + i * NT);
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    ask(0);
    ask(1);
    Pairs sums;
    float others = -INFINITY, top = -INFINITY;
    auto alone = [&](int v) {
        const Vec<T> q = row.load(v);
        others = fmaxf(others, largest(q));
        sums.add(q);
    };
    if (mine0 < v1) alone(mine0);
#pragma unroll 1
    for (int g = 0; g < groups; ++g) {
        asm volatile("cp.async.wait_group 1;" ::: "memory");
        Vec<T> q[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) *reinterpret_cast<uint4*>(q[i].v) = ring[((g & 1) * kAhead + i) * NT + id];
        const float most = sums.raise(q);   // what was read from the ring is in registers now
        ask(g + 2);
        top = fmaxf(top, most);
        if (((g + 1) & ((1 << wide) - 1)) == 0 || g + 1 == groups) {
            tops[g >> wide][id] = __float2bfloat16_ru(top);
            top = -INFINITY;
        }
        sums.terms(q, kAhead);
    }
    for (int v = mine0 + NT + groups * GROUP; v < v1; v += NT) alone(v);
    tops[kBuckets - 1][id] = __float2bfloat16_ru(others);
    asm volatile("cp.async.wait_all;" ::: "memory");

    if (SHARED && p.parts > 1) cluster_arrive();   // see finish()
    finish<T, NT, SHARED>(t, p, row, r, part, v0, v1, mine0 < v1, sums.all(), 0u, [&](bool reaches, float least) {
        // share by share: a lane a bucket, then a lane a vector of those that reach it
        for (uint32_t who = __ballot_sync(~0u, reaches); who; who &= who - 1) {
            const int other = (id & ~31) + __ffs(who) - 1, first = v0 + other, n = groups_of(first);
            const bool hit = lane < kBuckets && (lane == kBuckets - 1 || (lane << wide) < n) && __bfloat162float(tops[lane % kBuckets][other]) >= least;
            for (uint32_t which = __ballot_sync(~0u, hit); which; which &= which - 1) {
                const int b = __ffs(which) - 1, tail = first + NT + n * GROUP;
                // the last bucket: the first vector and those behind the groups
                const int from = b == kBuckets - 1 ? tail - NT : first + NT + (b << wide) * GROUP;
                const int last = b == kBuckets - 1 ? v1 : first + NT + min(n, (b + 1) << wide) * GROUP;
#pragma unroll 1
                for (int i = lane; from + i * NT < last; i += 32) {
                    const int v = b == kBuckets - 1 && i == 0 ? first : from + i * NT;
                    take<T, NT>(t, row, row.load(v), v, least);
                }
            }
        }
    });
}

template <class T>
sbnn_status launch_as(const Params& given, cudaStream_t st) {
    Params p = given;
    // vectors of a row at most: one more where rows start anywhere
    const bool whole = p.ld % Vec<T>::N == 0 && aligned16(p.x);
    const int64_t vectors = ((int64_t)p.classes + (whole ? 1 : 2) * (Vec<T>::N - 1)) / Vec<T>::N;
    const int sms = device_sms();
    p.parts = 1;
    ChainedLaunchScope chained;
    // A warp a row: 64 x 1000 fp32 top 5 4.0 us (a CTA a row 4.3), 1000 x 1000 bf16 4.7 (10.2); but for many alternatives of few rows a CTA
    // has the tighter bound, as long as none of the groups that it takes has nothing: 64 x 1000 top 20 6.7 (4.7).
    if (vectors <= 32 * kHeld && (p.top <= 8 || p.rows > 2 * sms || vectors < 4 * p.top)) {
        SBNN_CUDA_TRY(launch_kernel(logprobs_held_kernel<T, 32>, dim3((unsigned)((p.rows + 7ll) / 8)), dim3(256), 0, st, p));
        return SBNN_OK;
    }
    // Few rows are shared by clusters: 100 x 262144 fp32 by 1, 2 and 4 CTAs 35, 28 and 28 us, 16 rows 28, 20 and 15, 300 x 100000 34, 43
    // and 52.
    while (p.parts < 8 && (int64_t)p.rows * p.parts * 2 <= 2 * sms && vectors / (p.parts * 2) >= 256) p.parts *= 2;
    if ((int64_t)p.rows * p.parts > 0x7fffffff) return fail(SBNN_ERR_SHAPE, "too many rows");
    const dim3 grid((unsigned)(p.rows * p.parts));
    const int64_t share = (vectors + p.parts - 1) / p.parts;
    // 512 threads hold a share where all run at once: 200 x 32000 bf16 7.6 us (streamed 10.9), 3166 x 20000 47 (38)
    // 128 threads a row where rows are more than the SMs hold of 256: 2169 x 1253 fp32, top 5, 10.1 us (17.6), 4000 x 3000 fp16 17.5 (32.3)
    if (share <= 128 * kHeld && p.rows > 2 * sms) {
        SBNN_CUDA_TRY(launch_kernel(logprobs_held_kernel<T, 128>, grid, dim3(128), 0, st, p));
    } else if (share <= 256 * kHeld) {
        SBNN_CUDA_TRY(launch_kernel_cluster(logprobs_held_kernel<T, 256>, grid, dim3(256), 0, st, (unsigned)p.parts, p));
    } else if (share <= 512 * kHeld && (int64_t)p.rows * p.parts <= 2 * sms) {
        SBNN_CUDA_TRY(launch_kernel_cluster(logprobs_held_kernel<T, 512>, grid, dim3(512), 0, st, (unsigned)p.parts, p));
    } else {
        auto* const kernel = p.parts > 1 ? logprobs_stream_kernel<T, true> : logprobs_stream_kernel<T, false>;
        const sbnn_status r = set_max_dyn_smem(reinterpret_cast<const void*>(kernel), kStreamSmem);
        if (r != SBNN_OK) return r;
        SBNN_CUDA_TRY(launch_kernel_cluster(kernel, grid, dim3(256), (size_t)kStreamSmem, st, (unsigned)p.parts, p));
    }
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
    if (reinterpret_cast<uintptr_t>(logits_dev) % (type == SBNN_F32 ? 4 : 2))
        return fail(SBNN_ERR_ALIGN, "logits_dev must lie on a multiple of its elements' size");
    if (!aligned16(targets_dev) || !aligned16(logprob_dev) || !aligned16(entropy_dev) || !aligned16(top_index_dev) ||
        !aligned16(top_logprob_dev))
        return fail(SBNN_ERR_ALIGN, "targets_dev and the outputs must be 16-byte aligned");
    if (rows == 0) return SBNN_OK;
    sbnn_status r = check_device();
    if (r != SBNN_OK) return r;
    if ((r = check_device_memory({logits_dev, targets_dev, logprob_dev, entropy_dev, top_index_dev, top_logprob_dev})) != SBNN_OK) return r;
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
