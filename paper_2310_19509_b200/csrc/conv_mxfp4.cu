// 1x1 convolution on microscaled 4-bit operands (layout: mxfp4.cuh), fp32 sums on the tensor cores.
//
//   y[m][o] = act( bias[o] + sum_b 2^(ex(m,b) + ew(o,b)) sum_{k in block b} cx(m,k) cw(o,k) )
//
// The tensor core multiplies e2m1 codes and applies the two scales of every 32 channels itself (kind::mxf4).  Weights are its
// A operand: a tile is 128 output channels (the lanes of tensor memory) x BN pixels (its columns), so
//   - the few pixels of a single token or a small batch are a narrow N (8 to 32) and the weights, which are what such a call
//     reads, pass through the wide operand once;
//   - a warp of the epilogue holds 32 consecutive channels of a pixel and stores them without a transposition.
// Both operands arrive by tiled copies (128-byte rows = 256 channels, 128-byte swizzle), scales by linear copies of their
// tiles and from shared into tensor memory by tcgen05.cp.  A pipeline stage keeps tensor-memory columns for its scales of its
// own, so that a copy into them never meets an MMA that still reads them.
// Calls of up to 32 pixels are rounded to 4 bits by the CTAs themselves (FUSED): one launch, and the rounding happens while
// the first weights are on their way.  Otherwise a launch ahead rounds them, and this one asks for its first weights meanwhile.
// Where tiles are fewer than SMs the channel steps of a tile are shared by the CTAs of a cluster, which add up their sums
// through each other's shared memory in the order of their ranks: results do not depend on timing.
//
// Bound: a single token by its weights and by how evenly its CTAs lie on the SMs (8192 -> 8192: 35.7 MB, 5.5 us at the copy rate, of
// 9.3; -> 32768, 143 MB, more than the L2 holds, 21.8 of 39.7: 128 or 256 equal CTAs fill 86 % of 148 SMs, and the DRAM was at 44 % of its
// peak at 71 MB; what is fixed is the 3.5 us that 0.5 MB take).  More pixels by what the L2 delivers, until the kernel of
// CTA pairs (conv_mxfp4_pair.cu) takes over.  Many pixels of few channels by the beginnings and ends of its tiles, which nothing
// overlaps (802816 pixels 32 -> 64 fp32 214 us of 47, the rounding ahead among them).
#include <cuda.h>

#include <algorithm>

#include "cluster.cuh"
#include "common.h"
#include "mxfp4.cuh"
#include "mxfp4_mma.cuh"
#include "pipeline.cuh"
#include "tcgen05.cuh"

namespace sbnn {

namespace {

constexpr int kThreads = 256;       // warp 0 copies, warp 1 issues MMAs, warps 4-7 drain; warps 2-7 round activations (FUSED)
constexpr int kABytes = 128 * 128;  // the weights of a step
constexpr int kMaxStages = 8;
constexpr int kFusedPixels = SBNN_MXFP4_DIRECT_ROWS;
constexpr int kMaxSmem = 227 * 1024, kHalfSmem = 113 * 1024;   // of one CTA, of two on an SM

struct Args {
    const uint8_t *w_scales, *x_scales;
    const float* bias;
    const void* x;          // FUSED: the activations as they are
    void* y;
    int64_t ldx, ldy;
    int x_type, y_type;
    int M, Cout, K;
    int bn;                 // pixels of a tile
    int ctiles;             // tiles of 128 output channels
    int steps, split;       // steps of a tile, CTAs that share them
    int stages;
    int relu;
    int early;              // the launch before this one in the stream rounds x and has seen the end of all before it
    int vec;                // FUSED: rows of x can be read 16 bytes at a time
    int* status;
};

struct Shared {
    uint64_t full[kMaxStages], empty[kMaxStages], done, ready;
    uint32_t tmem;
    int abort;
};

// Pixels of a tile that each CTA of a cluster finishes: a multiple of 4.
__host__ __device__ constexpr int exchange_width(int bn, int split) { return (bn + 4 * split - 1) / (4 * split) * 4; }

// What a launch needs of shared memory, by parts (all multiples of 1024 bytes except the last).
struct Layout {
    int a, b, sfa, sfb;     // a stage's operands; FUSED: b and sfb are those of one step and all steps of the CTA stay
    int stage;
    int exchange;           // what the CTAs of a cluster send each other
    int64_t resident, total;   // of any number of steps: past 32 bits from 2^20 on, long after no CTA has room for them
};
__host__ __device__ inline Layout layout_of(int bn, int stages, int steps, int split, bool fused) {
    const int own = (steps + split - 1) / split;
    Layout l;
    l.a = kABytes;
    l.b = bn * 128;
    l.sfa = 1024;
    l.sfb = 1024 * ((bn + 127) / 128);
    l.stage = l.a + l.sfa + (fused ? 0 : l.b + l.sfb);
    l.resident = fused ? (int64_t)own * (l.b + l.sfb) : 0;
    l.exchange = split > 1 ? split * exchange_width(bn, split) * 512 : 0;
    l.total = l.resident + stages * l.stage + l.exchange + 1024 + (int)sizeof(Shared);
    return l;
}
// Columns of tensor memory: sums, then the scales of the stages.
__host__ __device__ constexpr int sf_columns(int bn) { return 8 + 8 * ((bn + 127) / 128); }
__host__ __device__ inline uint32_t tmem_columns(int bn, int stages) {
    const int need = (bn + 31) / 32 * 32 + stages * sf_columns(bn);
    uint32_t c = 32;
    while ((int)c < need) c *= 2;
    return c;
}

__device__ __forceinline__ void umma_mxf4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
        : "memory");
}
// 512 bytes of scales into 4 columns, the same in each quarter of the lanes.
__device__ __forceinline__ void scales_to_tmem(uint32_t tmem, uint64_t d) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(d) : "memory");
}

// Polls without regard to the abort flag, a bounded number of times: what is in flight when a CTA gives up has to land first.
__device__ __forceinline__ void land(uint64_t* bar, uint32_t parity) {
    for (uint32_t i = 0; i < kWaitLimit && !mbar_try_wait(bar, parity); ++i) __nanosleep(64);
}

// ---- activations of a FUSED call: rounded by the CTA for the steps that it sums -------------------------
// A thread takes whole blocks, U of them at a time: 4 U loads are on their way before the first is used.  (Four lanes a block, 8
// channels each, read whole lines but need more rounds: 13 pixels 8192 -> 8192 14.4 us and one token 4096 -> 16384 10.6, like this
// 13.2 and 9.6.)
template <class T, bool VEC, int U>
__device__ __forceinline__ void round_blocks(const Args& a, uint8_t* b, uint8_t* sfb, int b_bytes, int sfb_bytes, int step0, int blocks, int i, int nt) {
    Eight<T> e[U][4];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int row = (i + u * nt) / blocks, blk = (i + u * nt) - row * blocks, k = (step0 * 8 + blk) * 32, n = a.K - k;
        const T* p = static_cast<const T*>(a.x) + row * a.ldx + k;
        if (VEC && n >= 32) {
#pragma unroll
            for (int q = 0; q < 4; ++q) load8(e[u][q], p + 8 * q);
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int j = 0; j < 8; ++j) e[u][q].v[j] = 8 * q + j < n ? __ldg(p + 8 * q + j) : from_float<T>(0.f);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int row = (i + u * nt) / blocks, blk = (i + u * nt) - row * blocks, s = blk >> 3, c = blk & 7;
        uint32_t m = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) m = max(m, largest_bits(e[u][q]));
        const uint32_t byte = mx_scale_byte(m);
        *reinterpret_cast<uint4*>(b + s * b_bytes + row * 128 + ((c ^ (row & 7)) << 4)) =
            make_uint4(encode8(e[u][0], byte), encode8(e[u][1], byte), encode8(e[u][2], byte), encode8(e[u][3], byte));
        sfb[s * sfb_bytes + (c >> 2) * 512 + row * 16 + (c & 3)] = (uint8_t)byte;   // row < 32
    }
}
template <class T, bool VEC>
__device__ __forceinline__ void round_pixels_as(const Args& a, uint8_t* b, uint8_t* sfb, int b_bytes, int sfb_bytes, int step0, int steps, int t, int nt) {
    const int blocks = steps * 8, total = a.M * blocks;
    int i = t;
    if (VEC && sizeof(T) == 2)
        for (; i + nt < total; i += 2 * nt) round_blocks<T, VEC, 2>(a, b, sfb, b_bytes, sfb_bytes, step0, blocks, i, nt);
#pragma unroll 1
    for (; i < total; i += nt) round_blocks<T, VEC, 1>(a, b, sfb, b_bytes, sfb_bytes, step0, blocks, i, nt);
}
template <class T>
__device__ __forceinline__ void round_pixels(const Args& a, uint8_t* b, uint8_t* sfb, int b_bytes, int sfb_bytes, int step0, int steps, int t, int nt) {
    if (a.vec) round_pixels_as<T, true>(a, b, sfb, b_bytes, sfb_bytes, step0, steps, t, nt);
    else round_pixels_as<T, false>(a, b, sfb, b_bytes, sfb_bytes, step0, steps, t, nt);
}

// ---- epilogue: one output channel a lane ---------------------------------------------------------------
template <class T>
struct Out {
    T* y;             // channel `o` of the tile's first pixel
    int64_t ldy;
    float bias;
    int relu, pixels; // pixels of the tile that there are
    bool mine;        // the lane's channel exists
    __device__ __forceinline__ void put(T* at, float sum) const {
        sum += bias;
        if (relu) sum = fmaxf(sum, 0.f);
        if (mine) *at = from_float<T>(sum);
    }
    template <int N>
    __device__ __forceinline__ void put(int c, const uint32_t (&v)[N]) const {
        T* at = y + c * ldy;
        if (c + N <= pixels) {
#pragma unroll
            for (int i = 0; i < N; ++i, at += ldy) put(at, __uint_as_float(v[i]));
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i, at += ldy)
                if (c + i < pixels) put(at, __uint_as_float(v[i]));
        }
    }
};
// Whole warp: columns [c0, c1) of its lanes, a multiple of 8.
template <class T>
__device__ __forceinline__ void drain(const Out<T>& out, uint32_t tmem, int c0, int c1) {
    int c = c0;
    for (; c + 32 <= c1; c += 32) {
        uint32_t v[32];
        __syncwarp();   // the stores of channels that there are not part the lanes
        tmem_ld(tmem + (uint32_t)c, v);
        tmem_ld_wait();
        out.put(c, v);
    }
    for (; c < c1; c += 8) {
        uint32_t v[8];
        __syncwarp();
        tmem_ld(tmem + (uint32_t)c, v);
        tmem_ld_wait();
        out.put(c, v);
    }
}

template <bool FUSED, class T>
__global__ void __launch_bounds__(kThreads, 2)
conv_mxfp4_kernel(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap xmap, const Args a) {
    extern __shared__ uint8_t raw[];
    uint8_t* const base = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    const Layout l = layout_of(a.bn, a.stages, a.steps, a.split, FUSED);
    uint8_t* const resident = base + a.stages * l.stage;
    uint8_t* const exchange = resident + l.resident;
    Shared& sh = *reinterpret_cast<Shared*>(exchange + l.exchange);
    // operands first, scales behind them: the operands of every stage start on 1024 bytes
    uint8_t* const scales = base + a.stages * (l.a + (FUSED ? 0 : l.b));
    const int op_stage = l.a + (FUSED ? 0 : l.b), sf_stage = l.sfa + (FUSED ? 0 : l.sfb);
    uint8_t* const resident_sf = resident + ((int)l.resident / (l.b + l.sfb)) * l.b;   // (what a launch has of it fits shared memory)

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int tile = blockIdx.x / a.split, rank = a.split > 1 ? (int)cluster_rank() : 0;
    const int ct = tile % a.ctiles, n0 = tile / a.ctiles * a.bn;
    const int step0 = (int)((int64_t)a.steps * rank / a.split), step1 = (int)((int64_t)a.steps * (rank + 1) / a.split), steps = step1 - step0;
    const int ktiles = mx_ktiles(a.K);
    const int first = n0 & 127, atoms = (first + a.bn + 127) >> 7;   // tiles of scales that the pixels of a tile lie in
    const int xtiles = (a.M + 127) >> 7;
    const uint32_t columns = tmem_columns(a.bn, a.stages), sf_cols = (uint32_t)sf_columns(a.bn);

    if (warp == 1) {
        tmem_alloc(&sh.tmem, columns);
    } else if (threadIdx.x == 0) {
        for (int i = 0; i < a.stages; ++i) {
            mbar_init(&sh.full[i], 1);
            mbar_init(&sh.empty[i], 1);
        }
        mbar_init(&sh.done, 1);
        mbar_init(&sh.ready, kThreads - 64);
        mbar_fence_init();
        sh.abort = 0;
        prefetch_map(&wmap);
        if (!FUSED) prefetch_map(&xmap);
    }
    __syncwarp();
    if (a.split > 1) cluster_arrive();   // waited for before the first store into another CTA's memory: all of the cluster have begun by then
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = sh.tmem;
    volatile int* const abort = &sh.abort;
    grid_dependency_release();   // every CTA has its tensor memory: what starts now waits for none of it
    if (warp || !a.early) grid_dependency_wait();

    if (warp == 0) {
        if (lane == 0) {
            int issued = 0, s = 0;
            uint32_t phase = 1;   // the first round finds every stage empty
            const int rows = FUSED ? 0 : min(atoms, xtiles - (n0 >> 7));
            const uint8_t* wsf = a.w_scales + ((int64_t)ct * ktiles + 2 * step0) * 512;
            const uint8_t* xsf = FUSED ? nullptr : a.x_scales + ((int64_t)(n0 >> 7) * ktiles + 2 * step0) * 512;
            // Weights do not depend on the launch that rounds the activations (early): those of the first round are on their way
            // while it still runs.
            const int ahead = a.early ? min(a.stages, steps) : 0;
            for (int i = 0; i < ahead; ++i) {
                const uint32_t sfbytes = 512u * (uint32_t)min(2, ktiles - 2 * (step0 + i));
                mbar_arrive_expect_tx(&sh.full[i], (uint32_t)op_stage + sfbytes * (uint32_t)(1 + rows));
                tensor_g2s_2d(base + i * op_stage, &wmap, (step0 + i) * 64, ct * 128, &sh.full[i]);
                bulk_g2s(scales + i * sf_stage, wsf + i * 1024, sfbytes, &sh.full[i]);
            }
            if (a.early) grid_dependency_wait();
            for (int ks = step0; ks < step1; ++ks, ++issued) {
                if (issued >= a.stages && !mbar_wait(&sh.empty[s], phase, abort, a.status, SBNN_ERR_TIMEOUT)) break;
                uint8_t* const op = base + s * op_stage;
                uint8_t* const sf = scales + s * sf_stage;
                const uint32_t sfbytes = 512u * (uint32_t)min(2, ktiles - 2 * ks);
                if (issued >= ahead) {
                    mbar_arrive_expect_tx(&sh.full[s], (uint32_t)op_stage + sfbytes * (uint32_t)(1 + rows));
                    tensor_g2s_2d(op, &wmap, ks * 64, ct * 128, &sh.full[s]);
                    bulk_g2s(sf, wsf, sfbytes, &sh.full[s]);
                }
                wsf += 1024;
                if (!FUSED) {
                    tensor_g2s_2d(op + l.a, &xmap, ks * 64, n0, &sh.full[s]);
                    for (int r = 0; r < rows; ++r) bulk_g2s(sf + l.sfa + r * 1024, xsf + (int64_t)r * ktiles * 512, sfbytes, &sh.full[s]);
                    xsf += 1024;
                }
                if (++s == a.stages) s = 0, phase ^= 1;
            }
            if (*abort)
                for (int i = max(0, issued - a.stages); i < issued; ++i) land(&sh.full[i % a.stages], (i / a.stages) & 1);
        }
    } else if (warp == 1) {
        bool ok = !FUSED || __all_sync(~0u, mbar_wait(&sh.ready, 0, abort, a.status, SBNN_ERR_TIMEOUT));
        const uint32_t tmem = __shfl_sync(~0u, sh.tmem, 0), tmem_sf = tmem + (uint32_t)((a.bn + 31) / 32 * 32);   // in uniform registers
        // Everything that the issuing lane needs is kept by addition: divisions and rebuilt descriptors of a step took longer
        // than its MMAs (one token, 8192 -> 16384: 25.1 us, like this 17.6).
        const uint64_t a0 = operand_desc(smem_u32(base)), b0 = operand_desc(FUSED ? smem_u32(resident) : smem_u32(base) + (uint32_t)l.a);
        const uint64_t sfa0 = scale_desc(smem_u32(scales)), sfb0 = scale_desc(FUSED ? smem_u32(resident_sf) : smem_u32(scales) + (uint32_t)l.sfa);
        const uint32_t idesc0 = mx_instr_desc(128, a.bn, 0), idesc1 = mx_instr_desc(128, a.bn, 1);
        int s = 0;
        uint32_t phase = 0;
        for (int i = 0; ok && i < steps; ++i) {
            if (!(ok = __all_sync(~0u, mbar_wait(&sh.full[s], phase, abort, a.status, SBNN_ERR_TIMEOUT)))) break;
            tc_fence_after_sync();
            const uint32_t tsfa = tmem_sf + (uint32_t)s * sf_cols, tsfb = tsfa + 8;
            const uint64_t ad = a0 + (uint32_t)(s * (op_stage >> 4)), bd = b0 + (uint32_t)(FUSED ? i * (l.b >> 4) : s * (op_stage >> 4));
            const uint64_t sa = sfa0 + (uint32_t)(s * (sf_stage >> 4)), sb = sfb0 + (uint32_t)(FUSED ? i * (l.sfb >> 4) : s * (sf_stage >> 4));
            const int n64 = min(4, (a.K - (step0 + i) * kStep + 63) >> 6);
            if (elect_one()) {
                const uint32_t tb0 = tsfb + (uint32_t)(first >> 5), tb1 = tb0 + 4u * (uint32_t)atoms;
                scales_to_tmem(tsfa, sa);
                for (int r = 0; r < atoms; ++r) scales_to_tmem(tsfb + 4 * r, sb + r * 64);
                if (n64 > 2) {
                    scales_to_tmem(tsfa + 4, sa + 32);
                    for (int r = 0; r < atoms; ++r) scales_to_tmem(tsfb + 4 * (atoms + r), sb + r * 64 + 32);
                }
                umma_mxf4(tmem, ad, bd, idesc0, tsfa, tb0, (uint32_t)i);
                if (n64 > 1) umma_mxf4(tmem, ad + 2, bd + 2, idesc1, tsfa, tb0, 1);
                if (n64 > 2) umma_mxf4(tmem, ad + 4, bd + 4, idesc0, tsfa + 4, tb1, 1);
                if (n64 > 3) umma_mxf4(tmem, ad + 6, bd + 6, idesc1, tsfa + 4, tb1, 1);
                umma_commit(&sh.empty[s]);
                if (i + 1 == steps) umma_commit(&sh.done);
            }
            __syncwarp();
            if (++s == a.stages) s = 0, phase ^= 1;
        }
        if (!ok) {   // the MMAs issued so far end before the tensor memory is given back
            if (elect_one()) umma_commit(&sh.done);
            __syncwarp();
            land(&sh.done, 0);
        }
    }
    if (FUSED && warp >= 2) {
        const int t = threadIdx.x - 64, nt = kThreads - 64;
        if (a.x_type == SBNN_F32) round_pixels<float>(a, resident, resident_sf, l.b, l.sfb, step0, steps, t, nt);
        else if (a.x_type == SBNN_F16) round_pixels<__half>(a, resident, resident_sf, l.b, l.sfb, step0, steps, t, nt);
        else round_pixels<__nv_bfloat16>(a, resident, resident_sf, l.b, l.sfb, step0, steps, t, nt);
        fence_async_smem();
        mbar_arrive(&sh.ready);
    }
    // All warps drain: two share a quarter of the lanes and halve the columns.
    __syncwarp();
    const bool ok = __all_sync(~0u, mbar_wait(&sh.done, 0, abort, a.status, SBNN_ERR_TIMEOUT));
    tc_fence_after_sync();
    const int row = (warp & 3) * 32 + lane, o = ct * 128 + row;
    const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const int middle = (a.bn / 8 + 1) / 2 * 8, c0 = warp < 4 ? 0 : middle, c1 = warp < 4 ? middle : a.bn;
    Out<T> out;
    out.mine = o < a.Cout;
    out.y = static_cast<T*>(a.y) + (int64_t)n0 * a.ldy + o;
    out.ldy = a.ldy;
    out.bias = a.bias && out.mine ? __ldg(a.bias + o) : 0.f;
    out.relu = a.relu;
    out.pixels = min(a.bn, a.M - n0);
    if (a.split == 1) {
        if (ok) drain(out, lanes, c0, c1);
    } else {
        // The CTAs send each other their sums, four pixels of a channel at a time; CTA r finishes pixels [r * width, (r + 1) * width).
        cluster_wait();
        const int width = exchange_width(a.bn, a.split);
        if (ok) {
            const uint32_t ex = smem_u32(exchange);
            int owner = c0 / width, first_of_owner = owner * width;
            for (int c = c0; c < c1; c += 8) {
                uint32_t v[8];
                __syncwarp();
                tmem_ld(lanes + (uint32_t)c, v);
                tmem_ld_wait();
#pragma unroll
                for (int h = 0; h < 8; h += 4) {
                    if (c + h >= first_of_owner + width) ++owner, first_of_owner += width;
                    const int slot = (rank * width + c + h - first_of_owner) / 4 * 128 + row;
                    if (c + h < out.pixels) store_remote(remote_address(ex + (uint32_t)slot * 16u, owner), v[h], v[h + 1], v[h + 2], v[h + 3]);
                }
            }
        }
        cluster_sync();
        if (ok) {
            const float4* const sent = reinterpret_cast<const float4*>(exchange);
            for (int c = warp < 4 ? 0 : 4; c < width && rank * width + c < out.pixels; c += 8) {
                float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
                for (int r = 0; r < a.split; ++r) {
                    const float4 g = sent[(r * width + c) / 4 * 128 + row];
                    f.x += g.x, f.y += g.y, f.z += g.z, f.w += g.w;
                }
                const uint32_t v[4] = {__float_as_uint(f.x), __float_as_uint(f.y), __float_as_uint(f.z), __float_as_uint(f.w)};
                out.put(rank * width + c, v);
            }
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    __syncwarp();
    if (warp == 1) tmem_dealloc(tmem, columns);
}

// ---- host ------------------------------------------------------------------------------------------
struct Plan {
    int bn, split, stages;
    bool fused, pair;
};
// Whether any number of CTAs up to 8 that share a tile's steps holds these few pixels of its steps beside two stages of weights.
bool can_round_inside(int64_t M, int K) {
    const int steps = (K + kStep - 1) / kStep;
    for (int split = 1; M <= kFusedPixels && split <= 8 && split <= steps; ++split)
        if (layout_of((int)(M + 7) / 8 * 8, 2, steps, split, true).total <= kMaxSmem) return true;
    return false;
}

// Microseconds that a launch of this kernel takes, and one of the kernel of CTA pairs, fitted to what they were measured at (their
// rounding apart): a CTA starts, fills its pipeline and drains in 2.4 + 0.024 BN, a step brings in 17 KB of weights and 136 bytes a
// pixel at 45 bytes a clock and SM, sharing a tile costs the exchange.  300 pixels 4096 -> 4096: tiles of 64 in two waves 18.0 (model
// 18.2), of pairs 10.4 (12.3); 588, 1024 -> 516 fp32: tiles of 64 shared by two 5.8 (5.6), pairs 8.5 (7.9); 2048, 256 -> 4096:
// tiles of 256 16.7 (18.4), pairs 11.3 (10.3); 8192, 8192 -> 8192: 327 (409: a step of wide tiles overlaps the next more than the model
// has it, where pairs are far ahead) and 192 (168).
double tile_us(int bn) { return 2.4 + 0.024 * bn; }
double step_us(int bn) { return 0.215 + 0.00168 * bn; }
double single_us(int64_t tiles, int steps, int bn, int split, int sms) {
    const int64_t waves = (tiles * split + sms - 1) / sms;
    return (double)waves * (tile_us(bn) + (double)((steps + split - 1) / split) * step_us(bn)) + (split > 1 ? 1.0 : 0.0);
}
double pair_us(int64_t M, int Cout, int steps, int y_bytes, int sms) {
    const int64_t tiles = ((M + 255) / 256) * (((int64_t)Cout + 255) / 256), waves = (tiles + sms / 2 - 1) / (sms / 2);
    const double sums = 0.36 * steps;   // 256 channels of a tile; its epilogue takes 3.4 (fp32 5.2), unless the sums of the next do
    return 6.5 + sums + (double)(waves - 1) * std::max(sums, y_bytes == 4 ? 5.2 : 3.4);
}

// The same for up to 32 pixels (one tile as wide as they are), where a step is bound by the chain of its copies and MMAs, 0.3 us, or
// 0.55 with two CTAs on an SM, and sharing a tile by the exchange; `pixels`: of those that the CTAs round themselves.  One token 8192 ->
// 8192 shared by 2 10.4, by 4 9.7; 4096 -> 4096 by 2, 4, 8 6.3, 5.5, 6.1; 1024 -> 1000 by 1, 2, 4 3.6, 4.2, 4.1.
double few_us(int64_t tiles, int steps, int split, int pixels, int sms) {
    const int own = (steps + split - 1) / split;
    const int64_t rounds = ((int64_t)pixels * own * 32 + 1535) / 1536;
    return 2.6 + (split > 1 ? 0.6 + 0.12 * split : 0.0) + own * (tiles * split > sms ? 0.55 : 0.3) * std::max(1.0, (double)(tiles * split) / (2 * sms)) +
           0.55 * (double)rounds;
}

// The width of a tile and the number of CTAs that share its steps, all resident at the same time, that take least by the model, or
// the kernel of pairs.
Plan plan_for(int64_t M, int Cout, int K, bool raw, int y_bytes, int sms) {
    const int ctiles = (Cout + 127) / 128, steps = (K + kStep - 1) / kStep;
    Plan p = {};
    double best = 1e30;
    if (M <= kFusedPixels) {
        // One plan for both entry points, as if the CTAs rounded the activations, so that their results are the same bits.  First
        // what is resident at once; else any cluster that holds its share of the activations; else none does: rounded ahead.
        p.bn = (int)(M + 7) / 8 * 8;
        for (int pass = 0; pass < 3 && best == 1e30; ++pass) {
            p.fused = raw && pass < 2;
            for (int split = 1; split <= 8 && split <= steps && (pass || split == 1 || ctiles * split <= 2 * sms); ++split) {
                const bool two = ctiles * split > sms && !pass;
                const auto stages_in = [&](bool fused) {
                    int n = 6;
                    while (n > 0 && layout_of(p.bn, n, steps, split, fused).total > (two ? kHalfSmem : kMaxSmem)) --n;
                    return n;
                };
                if (stages_in(pass < 2) < (two ? 3 : 2)) continue;
                const double us = few_us(ctiles, steps, split, (int)M, sms);
                if (us < best) best = us, p.split = split, p.stages = stages_in(p.fused);
            }
        }
        return p;
    }
    for (int bn = 64; bn <= 256; bn *= 2) {
        const int64_t tiles = ctiles * ((M + bn - 1) / bn);
        for (int split = 1; split <= 8 && split <= steps && (split == 1 || tiles * split <= sms); ++split) {
            int stages = bn <= 128 ? 6 : 4;
            while (stages > 1 && layout_of(bn, stages, steps, split, false).total > kMaxSmem) --stages;
            const double us = single_us(tiles, steps, bn, split, sms);
            if (stages >= 3 && us < best) best = us, p.bn = bn, p.split = split, p.stages = stages;
        }
    }
    p.pair = pair_us(M, Cout, steps, y_bytes, sms) < best;
    return p;
}
// The same for activations that the call has to round, and that it has room for in 4 bits or not.
Plan plan_rounding(int64_t M, int Cout, int K, bool room, int y_bytes, int sms) {
    const Plan p = plan_for(M, Cout, K, true, y_bytes, sms);
    // A CTA of a few pixels rounds all that it meets of them.  From three rounds of its threads on a launch ahead, which does it once, is
    // the quicker way, if there is room for its result: 16, 24 and 32 pixels 8192 -> 8192 12.7, 14.7 and 17.0 us, ahead 12.9, 13.1 and
    // 13.3; 32 pixels 4096 -> 4096 8.4 and 9.2.  The sums are the same.
    const int steps = (K + kStep - 1) / kStep;
    if (p.fused && room && M * ((steps + p.split - 1) / p.split) * 32 > 3 * 1536) return plan_for(M, Cout, K, false, y_bytes, sms);
    return p;
}

sbnn_status launch(const Args& given, const Plan& p, const uint8_t* w_codes, const uint8_t* x_codes, cudaStream_t st) {
    if (p.pair) {
        const MxProduct q = {w_codes, given.w_scales, x_codes, given.x_scales, given.bias, given.y, given.ldy, given.y_type, given.M, given.Cout, given.K,
                             given.relu, given.early};
        return conv_mxfp4_pair(q, st);
    }
    Args a = given;
    sbnn_status r = async_status_word(&a.status);
    if (r != SBNN_OK) return r;
    a.bn = p.bn;
    a.split = p.split;
    a.stages = p.stages;
    a.ctiles = (a.Cout + 127) / 128;
    a.steps = (a.K + kStep - 1) / kStep;
    const int64_t ctas = (int64_t)a.ctiles * (((int64_t)a.M + a.bn - 1) / a.bn) * a.split;
    if (ctas > 0x7fffffff) return fail(SBNN_ERR_SHAPE, "too many tiles");
    CUtensorMap wmap, xmap;
    const unsigned long long row_bytes = 16ull * mx_blocks(a.K), strides[1] = {row_bytes};
    const unsigned long long wdims[2] = {row_bytes / 2, (unsigned long long)a.Cout}, xdims[2] = {row_bytes / 2, (unsigned long long)a.M};
    const unsigned wbox[2] = {64, 128}, xbox[2] = {64, (unsigned)a.bn};
    if ((r = encode_tiled_map(&wmap, w_codes, 2, 2, wdims, strides, wbox, 128)) != SBNN_OK) return r;
    if (p.fused) xmap = wmap;
    else if ((r = encode_tiled_map(&xmap, x_codes, 2, 2, xdims, strides, xbox, 128)) != SBNN_OK) return r;
    auto* const kernel = a.y_type == SBNN_F32   ? (p.fused ? conv_mxfp4_kernel<true, float> : conv_mxfp4_kernel<false, float>)
                         : a.y_type == SBNN_F16 ? (p.fused ? conv_mxfp4_kernel<true, __half> : conv_mxfp4_kernel<false, __half>)
                                                : (p.fused ? conv_mxfp4_kernel<true, __nv_bfloat16> : conv_mxfp4_kernel<false, __nv_bfloat16>);
    if ((r = set_max_dyn_smem(reinterpret_cast<const void*>(kernel), kMaxSmem)) != SBNN_OK) return r;
    const size_t smem = (size_t)layout_of(a.bn, a.stages, a.steps, a.split, p.fused).total;
    ChainedLaunchScope chained;   // the set-up overlaps the end of the launch before
    SBNN_CUDA_TRY(launch_kernel_cluster(kernel, dim3((unsigned)ctas), dim3(kThreads), smem, st, (unsigned)a.split, wmap, xmap, a));
    return SBNN_OK;
}

int bytes_of(int type) { return type == SBNN_F32 ? 4 : 2; }

sbnn_status check_call(const uint8_t* w_codes, const uint8_t* w_scales, const float* bias, const void* y, int y_type, int64_t ldy, int M, int Cin,
                       int Cout, int flags) {
    if (M < 0 || Cin <= 0 || Cout <= 0) return fail(SBNN_ERR_SHAPE, "bad shape M=%d Cin=%d Cout=%d", M, Cin, Cout);
    if (M > 1 << 30 || Cin > 1 << 30 || Cout > 1 << 30) return fail(SBNN_ERR_UNSUPPORTED, "M=%d Cin=%d Cout=%d: 2^30 at most", M, Cin, Cout);
    if (y_type != SBNN_F32 && y_type != SBNN_F16 && y_type != SBNN_BF16) return fail(SBNN_ERR_UNSUPPORTED, "y_dev: unknown element type %d", y_type);
    if (ldy < Cout) return fail(SBNN_ERR_SHAPE, "y_dev: rows of %d elements do not fit a stride of %lld", Cout, (long long)ldy);
    if (flags & ~SBNN_RELU) return fail(SBNN_ERR_UNSUPPORTED, "unknown flag bits 0x%x", flags);
    if (!aligned16(w_codes) || !aligned16(w_scales) || !aligned16(bias) || !aligned16(y))
        return fail(SBNN_ERR_ALIGN, "device pointers must be 16-byte aligned");
    return SBNN_OK;
}

}  // namespace
}  // namespace sbnn

using namespace sbnn;

extern "C" sbnn_status sbnn_conv1x1_mxfp4_q(const uint8_t* w_codes_dev, const uint8_t* w_scales_dev, const float* bias_dev,
                                            const uint8_t* x_codes_dev, const uint8_t* x_scales_dev, void* y_dev, int y_type, int64_t ldy, int M,
                                            int Cin, int Cout, int flags, void* cuda_stream) {
    clear_error();
    if (!w_codes_dev || !w_scales_dev || !x_codes_dev || !x_scales_dev || !y_dev)
        return fail(SBNN_ERR_NULL, "weights, activations and y_dev must not be NULL");
    sbnn_status r = check_call(w_codes_dev, w_scales_dev, bias_dev, y_dev, y_type, ldy, M, Cin, Cout, flags);
    if (r != SBNN_OK) return r;
    if (!aligned16(x_codes_dev) || !aligned16(x_scales_dev)) return fail(SBNN_ERR_ALIGN, "device pointers must be 16-byte aligned");
    if (M == 0) return SBNN_OK;
    if ((r = check_device()) != SBNN_OK) return r;
    if ((r = check_device_memory({w_codes_dev, w_scales_dev, bias_dev, x_codes_dev, x_scales_dev, y_dev})) != SBNN_OK) return r;
    Args a = {};
    a.w_scales = w_scales_dev, a.x_scales = x_scales_dev, a.bias = bias_dev, a.y = y_dev, a.ldy = ldy, a.y_type = y_type;
    a.M = M, a.Cout = Cout, a.K = Cin, a.relu = flags & SBNN_RELU;
    return launch(a, plan_for(M, Cout, Cin, false, bytes_of(y_type), device_sms()), w_codes_dev, x_codes_dev, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" sbnn_status sbnn_conv1x1_mxfp4(const uint8_t* w_codes_dev, const uint8_t* w_scales_dev, const float* bias_dev, const void* x_dev,
                                          int x_type, int64_t ldx, void* y_dev, int y_type, int64_t ldy, int M, int Cin, int Cout, int flags,
                                          void* workspace_dev, int64_t workspace_bytes, void* cuda_stream) {
    clear_error();
    if (!w_codes_dev || !w_scales_dev || !x_dev || !y_dev) return fail(SBNN_ERR_NULL, "weights, x_dev and y_dev must not be NULL");
    sbnn_status r = check_call(w_codes_dev, w_scales_dev, bias_dev, y_dev, y_type, ldy, M, Cin, Cout, flags);
    if (r != SBNN_OK) return r;
    if (x_type != SBNN_F32 && x_type != SBNN_F16 && x_type != SBNN_BF16) return fail(SBNN_ERR_UNSUPPORTED, "x_dev: unknown element type %d", x_type);
    if (ldx < Cin) return fail(SBNN_ERR_SHAPE, "x_dev: rows of %d elements do not fit a stride of %lld", Cin, (long long)ldx);
    if (!aligned16(x_dev)) return fail(SBNN_ERR_ALIGN, "x_dev must be 16-byte aligned");
    const int64_t codes = (int64_t)M * 16 * mx_blocks(Cin), scales = ((int64_t)M + 127) / 128 * 512 * mx_ktiles(Cin);
    if (M > kFusedPixels) {
        if (!workspace_dev) return fail(SBNN_ERR_NULL, "more than %d pixels need a workspace", kFusedPixels);
        if (workspace_bytes < codes + scales)
            return fail(SBNN_ERR_SHAPE, "the workspace has %lld bytes, %lld are needed", (long long)workspace_bytes, (long long)(codes + scales));
        if (!aligned16(workspace_dev)) return fail(SBNN_ERR_ALIGN, "workspace_dev must be 16-byte aligned");
    }
    if (M == 0) return SBNN_OK;
    const bool room = workspace_dev && workspace_bytes >= codes + scales && aligned16(workspace_dev);
    if (!room && !can_round_inside(M, Cin))
        return fail(SBNN_ERR_NULL, "Cin=%d is too wide to be rounded without a workspace of %lld bytes", Cin, (long long)(codes + scales));
    if ((r = check_device()) != SBNN_OK) return r;
    if ((r = check_device_memory({w_codes_dev, w_scales_dev, bias_dev, x_dev, y_dev, workspace_dev})) != SBNN_OK) return r;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    Args a = {};
    a.w_scales = w_scales_dev, a.bias = bias_dev, a.y = y_dev, a.ldy = ldy, a.y_type = y_type;
    a.M = M, a.Cout = Cout, a.K = Cin, a.relu = flags & SBNN_RELU;
    const Plan p = plan_rounding(M, Cout, Cin, room, bytes_of(y_type), device_sms());
    if (p.fused) {
        a.x = x_dev, a.ldx = ldx, a.x_type = x_type;
        a.vec = ldx * bytes_of(x_type) % 16 == 0;
        return launch(a, p, w_codes_dev, nullptr, st);
    }
    uint8_t* const xc = static_cast<uint8_t*>(workspace_dev);
    a.x_scales = xc + codes;
    if ((r = mxfp4_quantize_launch(x_dev, x_type, ldx, xc, xc + codes, M, Cin, st)) != SBNN_OK) return r;
    a.early = 1;
    return launch(a, p, w_codes_dev, xc, st);
}

extern "C" sbnn_status sbnn_debug_plan_conv1x1_mxfp4(int M, int Cin, int Cout, int y_type, int activations, int sms, int* pair, int* pixels, int* split,
                                                     int* rounds, int64_t* shared_bytes) {
    clear_error();
    if (!pair || !pixels || !split || !rounds || !shared_bytes) return fail(SBNN_ERR_NULL, "the results must not be NULL");
    const sbnn_status r = check_call(nullptr, nullptr, nullptr, nullptr, y_type, Cout, M, Cin, Cout, 0);
    if (r != SBNN_OK) return r;
    if (M == 0 || sms < 2 || sms > 4096 || activations < 0 || activations > 2) return fail(SBNN_ERR_SHAPE, "bad call: M=%d sms=%d activations=%d", M, sms, activations);
    if (activations == 1 && !can_round_inside(M, Cin)) return fail(SBNN_ERR_NULL, "such a call needs a workspace");
    const Plan p = activations ? plan_rounding(M, Cout, Cin, activations == 2, bytes_of(y_type), sms) : plan_for(M, Cout, Cin, false, bytes_of(y_type), sms);
    *pair = p.pair;
    *pixels = p.pair ? 256 : p.bn;
    *split = p.pair ? 1 : p.split;
    *rounds = p.fused;
    *shared_bytes = p.pair ? 0 : layout_of(p.bn, p.stages, (Cin + kStep - 1) / kStep, p.split, p.fused).total;
    return SBNN_OK;
}
