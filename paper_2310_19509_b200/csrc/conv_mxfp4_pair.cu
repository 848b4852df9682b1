// 1x1 convolution on microscaled 4-bit operands for many pixels (see conv_mxfp4.cu for the operation and the small calls).
//
// Bound: with one CTA a tile, by what the L2 delivers: a 128 x 256 tile takes in 51 KB for 524 cycles of MMAs.  Here two CTAs
// of a cluster work on one 256 x 256 tile (cta_group::2): each holds half of either operand, 35 KB for the same cycles an SM, and
// the tensor cores of both read both halves.  Pixels are the A operand, so that a thread of the epilogue holds consecutive
// channels of a pixel: it packs them, stages them in shared memory and the copy engine writes whole 128-byte rows (a warp that
// stored 32 channels of a pixel at a time took 6 us for 128 x 256 sums).
//
// Tensor memory (512 columns): two sets of sums that overlap, [0, 256) and [136, 392), and scales of 5 stages, 24 columns each.
// The epilogue takes the overlapping half of a tile into registers first; the MMAs of the next tile start then.
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

constexpr int kThreads = 384;      // warp 0 copies, warp 1 of the first CTA issues MMAs, warps 4-7 and 8-11 drain
constexpr int kStages = 5;
constexpr int kOperand = 128 * 128;
constexpr int kStage = 2 * kOperand + 3 * 1024;   // both operands, scales of the CTA's pixels, scales of all channels of the tile
constexpr int kSecond = 136;       // first column of the second set of sums
constexpr int kScales = 392;       // first column of the scales
constexpr int kSlab = 128 * 128;   // staged output: 128 pixels x 128 bytes
constexpr int kGroup = 8;          // pixel tiles that share the channel tiles in the L2

struct PairShared {
    uint64_t full[kStages], empty[kStages], sums, freed;
    float bias[256];
    uint32_t tmem;
    int abort;
};
constexpr int kPairSmem = kStages * kStage + 2 * kSlab + (int)sizeof(PairShared) + 1024;
static_assert(kPairSmem <= 227 * 1024, "shared memory");
static_assert(kScales + 24 * kStages <= 512 && kSecond + 256 <= kScales, "tensor memory");

struct PairArgs {
    const float* bias;
    void* y;
    int64_t ldy;
    int M, Cout, K;
    int mtiles, ntiles;
    int relu, tiled_store;
    int early;              // the launch before this one in the stream rounds the pixels and has seen the end of all before it
    int* status;
};

// A copy whose bytes are counted by a barrier of either CTA of the pair (`bar`: its address in the cluster).
__device__ __forceinline__ void pair_g2s(void* dst, const void* map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void pair_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void pair_scales(uint32_t tmem, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
// One arrival at the barrier of this address in both CTAs once all MMAs issued so far are complete.
__device__ __forceinline__ void pair_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(smem_u32(bar)), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void pair_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Barriers that CTAs of the pair signal to each other are acquired at cluster scope.
__device__ __forceinline__ bool pair_wait(uint64_t* bar, uint32_t parity, volatile int* abort, int* status) {
    for (uint32_t i = 0; i < kWaitLimit; ++i) {
        uint32_t ok;
        asm volatile("{\n\t.reg .pred p;\n\t"
                     "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
                     "selp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
        if (ok) return true;
        if (i > 64) {
            if (*abort) return false;
            __nanosleep(64);
        }
    }
    *abort = 1;
    atomicCAS(status, 0, (int)SBNN_ERR_TIMEOUT);
    return false;
}
// The four warps of a group.  (Aligned instructions as well: see cluster.cuh.)
__device__ __forceinline__ void drain_sync(int group) {
    __syncwarp();
    asm volatile("bar.sync %0, 128;" ::"r"(1 + group) : "memory");
}
__device__ __forceinline__ bool drain_any(int group, bool v) {
    uint32_t r;
    __syncwarp();
    asm volatile("{\n\t.reg .pred p, q;\n\t"
                 "setp.ne.b32 p, %1, 0;\n\t"
                 "bar.red.or.pred q, %2, 128, p;\n\t"
                 "selp.u32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"((uint32_t)v), "r"(1 + group) : "memory");
    return r != 0;
}

// Tile number -> (pixel tile, channel tile): groups of pixel tiles pass over all channel tiles together.
__device__ __forceinline__ void tile_at(const PairArgs& a, int t, int& mt, int& nt) {
    const int group = t / (kGroup * a.ntiles), r = t - group * kGroup * a.ntiles, rows = min(kGroup, a.mtiles - group * kGroup);
    nt = r / rows;
    mt = group * kGroup + r - nt * rows;
}

template <class T>
__device__ __forceinline__ uint32_t pack_word(const float* f);
template <>
__device__ __forceinline__ uint32_t pack_word<float>(const float* f) { return __float_as_uint(f[0]); }
template <>
__device__ __forceinline__ uint32_t pack_word<__half>(const float* f) {
    const __half2 h = __floats2half2_rn(f[0], f[1]);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <>
__device__ __forceinline__ uint32_t pack_word<__nv_bfloat16>(const float* f) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(f[0], f[1]);
    return *reinterpret_cast<const uint32_t*>(&h);
}

template <class T>
__global__ void __launch_bounds__(kThreads, 1)
conv_mxfp4_pair_kernel(const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap xsmap,
                       const __grid_constant__ CUtensorMap wsmap, const __grid_constant__ CUtensorMap ymap, const PairArgs a) {
    extern __shared__ uint8_t raw[];
    uint8_t* const base = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    uint8_t* const slabs = base + 2 * kStages * kOperand;                // operands first, then the staged output, then scales
    uint8_t* const scales = slabs + 2 * kSlab;
    PairShared& sh = *reinterpret_cast<PairShared*>(scales + kStages * 3 * 1024);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)cluster_rank();
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1, tiles = a.mtiles * a.ntiles;
    const int steps = (a.K + kStep - 1) / kStep;

    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&sh.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&sh.full[i], 1);
            mbar_init(&sh.empty[i], 1);
        }
        mbar_init(&sh.sums, 1);
        mbar_init(&sh.freed, 16);
        mbar_fence_init();
        sh.abort = 0;
        prefetch_map(&xmap);
        prefetch_map(&wmap);
        prefetch_map(&xsmap);
        prefetch_map(&wsmap);
    }
    tc_fence_before_sync();
    __syncthreads();
    cluster_sync();   // both CTAs' barriers are set up
    tc_fence_after_sync();
    const uint32_t tmem = sh.tmem;
    volatile int* const abort = &sh.abort;
    grid_dependency_release();
    if (warp || !a.early) grid_dependency_wait();

    if (warp == 0) {
        if (lane == 0) {
            // Channels do not depend on the launch that rounds the pixels (early): those of the first stages are on their way while it
            // still runs.
            const int ahead = a.early ? min(kStages, steps) : 0;
            if (ahead) {
                int mt, nt;
                tile_at(a, pair, mt, nt);
                for (int i = 0; i < ahead; ++i) {
                    const uint32_t bar = remote_address(smem_u32(&sh.full[i]), 0);
                    if (rank == 0) mbar_arrive_expect_tx(&sh.full[i], 2 * kStage);
                    pair_g2s(base + i * 2 * kOperand + kOperand, &wmap, i * 64, nt * 256 + rank * 128, bar);
                    pair_g2s(scales + i * 3 * 1024 + 1024, &wsmap, i * 256, nt * 2, bar);
                }
                grid_dependency_wait();
            }
            int s = 0, used = 0;
            uint32_t phase = 1;
            bool ok = true;
            for (int t = pair; ok && t < tiles; t += pairs) {
                int mt, nt;
                tile_at(a, t, mt, nt);
                for (int i = 0; i < steps; ++i) {
                    if (used == kStages && !(ok = pair_wait(&sh.empty[s], phase, abort, a.status))) break;
                    if (used < kStages) ++used;
                    const uint32_t bar = remote_address(smem_u32(&sh.full[s]), 0);
                    uint8_t* const op = base + s * 2 * kOperand;
                    uint8_t* const sf = scales + s * 3 * 1024;
                    if (t != pair || i >= ahead) {
                        if (rank == 0) mbar_arrive_expect_tx(&sh.full[s], 2 * kStage);
                        pair_g2s(op + kOperand, &wmap, i * 64, nt * 256 + rank * 128, bar);
                        pair_g2s(sf + 1024, &wsmap, i * 256, nt * 2, bar);
                    }
                    pair_g2s(op, &xmap, i * 64, mt * 256 + rank * 128, bar);
                    pair_g2s(sf, &xsmap, i * 256, mt * 2 + rank, bar);
                    if (++s == kStages) s = 0, phase ^= 1;
                }
            }
            // what was issued before giving up lands before the memory is given back
            if (*abort)
                for (int i = 0; i < 1000; ++i) __nanosleep(1000);
        }
    } else if (warp == 1 && rank == 0) {
        const uint64_t a0 = operand_desc(smem_u32(base)), b0 = operand_desc(smem_u32(base + kOperand)), f0 = scale_desc(smem_u32(scales));
        const uint32_t idesc0 = mx_instr_desc(256, 256, 0), idesc1 = mx_instr_desc(256, 256, 1);
        const uint32_t tmem = __shfl_sync(~0u, sh.tmem, 0);   // in a uniform register
        int s = 0, done = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int t = pair; ok && t < tiles; t += pairs, ++done) {
            if (done && !(ok = __all_sync(~0u, pair_wait(&sh.freed, (done - 1) & 1, abort, a.status)))) break;
            tc_fence_after_sync();
            const uint32_t d = tmem + (done & 1 ? kSecond : 0);
            for (int i = 0; i < steps; ++i) {
                if (!(ok = __all_sync(~0u, pair_wait(&sh.full[s], phase, abort, a.status)))) break;
                tc_fence_after_sync();
                const uint32_t sfa = tmem + kScales + 24 * s, sfb = sfa + 8;
                const uint64_t ad = a0 + (uint32_t)(s * (2 * kOperand >> 4)), bd = b0 + (uint32_t)(s * (2 * kOperand >> 4)), fd = f0 + (uint32_t)(s * 192);
                const int n64 = min(4, (a.K - i * kStep + 63) >> 6);
                if (elect_one()) {
                    // scales in shared memory: pixels k-tile 0, 1; channels 0-127 k-tile 0, 1; channels 128-255 k-tile 0, 1
                    pair_scales(sfa, fd);
                    pair_scales(sfb, fd + 64);
                    pair_scales(sfb + 4, fd + 128);
                    if (n64 > 2) {
                        pair_scales(sfa + 4, fd + 32);
                        pair_scales(sfb + 8, fd + 96);
                        pair_scales(sfb + 12, fd + 160);
                    }
                    pair_mma(d, ad, bd, idesc0, sfa, sfb, (uint32_t)i);
                    if (n64 > 1) pair_mma(d, ad + 2, bd + 2, idesc1, sfa, sfb, 1);
                    if (n64 > 2) pair_mma(d, ad + 4, bd + 4, idesc0, sfa + 4, sfb + 8, 1);
                    if (n64 > 3) pair_mma(d, ad + 6, bd + 6, idesc1, sfa + 4, sfb + 8, 1);
                    pair_commit(&sh.empty[s]);
                    if (i + 1 == steps) pair_commit(&sh.sums);
                }
                __syncwarp();
                if (++s == kStages) s = 0, phase ^= 1;
            }
        }
        if (!ok) {
            if (elect_one()) pair_commit(&sh.sums);
            __syncwarp();
            for (int i = 0; i < 1000; ++i) __nanosleep(1000);
        }
    } else if (warp >= 4) {
        // Two groups of four warps: of the 128 columns of either half of a tile each takes 64, and has a slab of its own.
        constexpr int W = 128 / (int)sizeof(T);   // channels of a slab
        constexpr int E = 4 / (int)sizeof(T);     // channels of a 32-bit word
        const int group = (warp - 4) >> 2, thread = (threadIdx.x - 128) & 127, row = (warp & 3) * 32 + lane;
        const uint32_t freed = remote_address(smem_u32(&sh.freed), 0);
        uint8_t* const slab = slabs + group * kSlab;
        float* const bias = sh.bias + group * 128;   // of the group's channels: 64 of the first half of the tile, 64 of the second
        int done = 0;
        for (int t = pair; t < tiles; t += pairs, ++done) {
            int mt, nt;
            tile_at(a, t, mt, nt);
            const int m0 = mt * 256 + rank * 128, n0 = nt * 256 + group * 64;
            const int ob = n0 + (thread >> 6) * 128 + (thread & 63);
            bias[thread] = a.bias && ob < a.Cout ? __ldg(a.bias + ob) : 0.f;   // the group's last barrier was behind its last use
            if (drain_any(group, !pair_wait(&sh.sums, done & 1, abort, a.status))) break;
            tc_fence_after_sync();
            const uint32_t d = tmem + (done & 1 ? kSecond : 0) + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(group * 64);
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                const int half = (done & 1) ? h : 1 - h;   // the half that the next tile's sums overlap comes first
                uint32_t v[2][32];
                __syncwarp();   // the last stores part the lanes
                tmem_ld(d + (uint32_t)(half * 128), v[0]);
                tmem_ld(d + (uint32_t)(half * 128 + 32), v[1]);
                tmem_ld_wait();
                if (h == 0) {
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) pair_arrive(freed);
                }
#pragma unroll
                for (int c = 0; c < 64; c += W) {
                    const int o = n0 + half * 128 + c;
                    uint32_t w[32];
#pragma unroll
                    for (int j = 0; j < W; j += 4) {
                        const float4 b = *reinterpret_cast<const float4*>(bias + half * 64 + c + j);
                        float f[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            f[e] += __uint_as_float(v[(c + j + e) >> 5][(c + j + e) & 31]);
                            if (a.relu) f[e] = fmaxf(f[e], 0.f);
                        }
#pragma unroll
                        for (int e = 0; e < 4; e += E) w[(j + e) / E] = pack_word<T>(f + e);
                    }
                    if (thread == 0) bulk_wait_read_all();   // the store before this one has left the slab
                    drain_sync(group);
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        *reinterpret_cast<uint4*>(slab + row * 128 + ((q ^ (row & 7)) << 4)) = make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
                    if (a.tiled_store) {
                        fence_async_smem();
                        drain_sync(group);
                        if (thread == 0) {
                            if (o < a.Cout && m0 < a.M) tensor_s2g_2d(&ymap, o, m0, slab);
                            bulk_commit_group();
                        }
                    } else {
                        drain_sync(group);
                        // rows that the copy engine cannot address: a warp stores a row's channels, a lane every 32nd
                        T* const y = static_cast<T*>(a.y);
                        for (int r = warp & 3; r < 128 && m0 + r < a.M; r += 4)
#pragma unroll
                            for (int e = lane; e < W; e += 32)
                                if (o + e < a.Cout)
                                    y[(int64_t)(m0 + r) * a.ldy + o + e] =
                                        *reinterpret_cast<const T*>(slab + r * 128 + (((e * (int)sizeof(T) >> 4) ^ (r & 7)) << 4) + (e * (int)sizeof(T) & 15));
                    }
                }
            }
        }
        if (thread == 0) bulk_wait_all();
    }
    __syncwarp();
    tc_fence_before_sync();
    __syncthreads();
    cluster_sync();   // nothing of the pair's is in use any more
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

template <class T>
sbnn_status launch_as(const PairArgs& a, const CUtensorMap& xm, const CUtensorMap& wm, const CUtensorMap& xs, const CUtensorMap& ws,
                      const CUtensorMap& ym, cudaStream_t st) {
    const sbnn_status r = set_max_dyn_smem(reinterpret_cast<const void*>(&conv_mxfp4_pair_kernel<T>), kPairSmem);
    if (r != SBNN_OK) return r;
    const int64_t tiles = (int64_t)a.mtiles * a.ntiles;
    const int pairs = (int)std::min<int64_t>(tiles, device_sms() / 2);
    ChainedLaunchScope chained;
    SBNN_CUDA_TRY(launch_kernel_cluster(conv_mxfp4_pair_kernel<T>, dim3((unsigned)(2 * pairs)), dim3(kThreads), (size_t)kPairSmem, st, 2u, xm, wm, xs,
                                        ws, ym, a));
    return SBNN_OK;
}

}  // namespace

sbnn_status conv_mxfp4_pair(const MxProduct& p, cudaStream_t st) {
    PairArgs a = {};
    sbnn_status r = async_status_word(&a.status);
    if (r != SBNN_OK) return r;
    a.bias = p.bias, a.y = p.y, a.ldy = p.ldy, a.M = p.M, a.Cout = p.Cout, a.K = p.K, a.relu = p.relu, a.early = p.early;
    a.mtiles = (int)(((int64_t)p.M + 255) / 256), a.ntiles = (int)(((int64_t)p.Cout + 255) / 256);
    const int size = p.y_type == SBNN_F32 ? 4 : 2, ktiles = mx_ktiles(p.K);
    if ((int64_t)a.mtiles * a.ntiles > 0x3fffffff) return fail(SBNN_ERR_SHAPE, "too many tiles");
    a.tiled_store = p.ldy * size % 16 == 0 && (int64_t)p.Cout * size % 16 == 0;
    CUtensorMap xm, wm, xs, ws, ym;
    const unsigned long long row = 16ull * mx_blocks(p.K), srow = 512ull * ktiles, yrow = (unsigned long long)p.ldy * size;
    const unsigned long long xd[2] = {row / 2, (unsigned long long)p.M}, wd[2] = {row / 2, (unsigned long long)p.Cout};
    const unsigned long long xsd[2] = {srow / 4, (unsigned long long)(p.M + 127ll) / 128}, wsd[2] = {srow / 4, (unsigned long long)(p.Cout + 127ll) / 128};
    const unsigned long long yd[2] = {(unsigned long long)p.Cout, (unsigned long long)p.M};
    const unsigned box[2] = {64, 128}, xsbox[2] = {256, 1}, wsbox[2] = {256, 2}, ybox[2] = {128u / size, 128};
    if ((r = encode_tiled_map(&xm, p.x_codes, 2, 2, xd, &row, box, 128)) != SBNN_OK) return r;
    if ((r = encode_tiled_map(&wm, p.w_codes, 2, 2, wd, &row, box, 128)) != SBNN_OK) return r;
    if ((r = encode_tiled_map(&xs, p.x_scales, 4, 2, xsd, &srow, xsbox)) != SBNN_OK) return r;
    if ((r = encode_tiled_map(&ws, p.w_scales, 4, 2, wsd, &srow, wsbox)) != SBNN_OK) return r;
    if (!a.tiled_store) ym = xm;
    else if ((r = encode_tiled_map(&ym, p.y, size, 2, yd, &yrow, ybox, 128)) != SBNN_OK) return r;
    switch (p.y_type) {
        case SBNN_F32: return launch_as<float>(a, xm, wm, xs, ws, ym, st);
        case SBNN_F16: return launch_as<__half>(a, xm, wm, xs, ws, ym, st);
        default: return launch_as<__nv_bfloat16>(a, xm, wm, xs, ws, ym, st);
    }
}

}  // namespace sbnn
