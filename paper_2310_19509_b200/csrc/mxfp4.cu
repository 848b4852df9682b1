// Rounding to microscaled 4-bit floating point and back (layout and arithmetic: mxfp4.cuh).
//
// Bound: memory.  A bf16 element is two bytes to read and 17/32 of a byte to write, or the other way round: 16384 x 8192 take 57 and
// 54 us of 52 at the copy rate.
#include <algorithm>

#include "common.h"
#include "mxfp4.cuh"
#include "mxfp4_mma.cuh"
#include "pipeline.cuh"

namespace sbnn {
namespace {

// LPR lanes take a row, eight channels a lane: all 32 of a warp, or 16 or 8 where rows are no longer than 128 or 64 channels (60000 x 64 bf16
// to 4 bits 3.4 us, with 32 lanes 10).  A warp has four rows, whose loads are all on their way before the first is used, a CTA 32.
// (16 rows a warp, so that a CTA's scales are whole tiles: 16384 x 1024 bf16 14.8 us, like this 9.2; 16384 x 8192 fp32 89 and 87.)
// Rows that do not start on 16 bytes, or do not end with a whole vector, are read and written one element a lane and pass
// through shared memory (20000 x 1001 bf16 14.8 and 12.4 us there and back; through eight loads a lane 86 together).
constexpr int kThreads = 256, kRows = 4;

template <class T, bool VEC, int LPR>
__global__ void __launch_bounds__(kThreads)
quantize_kernel(const T* __restrict__ x, int64_t ldx, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales, int M, int K, int ktiles) {
    constexpr int ROWS = 8 * kRows, AT = 32 / LPR, BATCH = kRows / AT;   // AT: rows of a warp side by side
    __shared__ uint32_t tile[2][ROWS];   // [k-tile][row of the CTA]: four scale bytes each
    __shared__ Eight<T> turn[VEC ? 1 : kThreads];
    grid_dependency_wait();
    grid_dependency_release();   // behind the wait: what starts now knows all launches before this one to be done
    const int l = threadIdx.x % LPR, at = threadIdx.x % 32 / LPR, warp = threadIdx.x >> 5;
    const int wide = LPR == 32 ? (ktiles + 1) / 2 : 1, kt = blockIdx.x % wide * 2;
    const int64_t row0 = (int64_t)(blockIdx.x / wide) * ROWS;
    const int rows = (int)min((int64_t)ROWS, M - row0), k0 = kt * 128;
    const int64_t ldc = 16 * (int64_t)mx_blocks(K);
    const bool word = ((k0 + l * 8) & ~31) < K;   // the lane's word of codes exists
    // addresses by addition: built anew for each row they were a third of the instructions, and those are what bounds bf16
    const int r0 = warp * kRows + at;
    const T* p = x + (row0 + r0) * ldx + k0;
    Eight<T> e[BATCH];   // VEC: channels k0 + 8 l ..; else channel k0 + l + LPR j
#pragma unroll
    for (int i = 0; i < BATCH; ++i, p += AT * ldx) {
        const int r = r0 + i * AT;
        if (VEC) {
            if (r < rows && k0 + l * 8 < K) {
                load8(e[i], p + l * 8);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) e[i].v[j] = from_float<T>(0.f);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) e[i].v[j] = r < rows && k0 + l + LPR * j < K ? __ldg(p + l + LPR * j) : from_float<T>(0.f);
        }
    }
    uint8_t* to = codes + (row0 + r0) * ldc + (k0 >> 1) + l * 4;
#pragma unroll
    for (int i = 0; i < BATCH; ++i, to += AT * ldc) {
        const int r = r0 + i * AT;
        if (!VEC) {
            Eight<T>* const row = turn + (threadIdx.x - l);
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 8; ++j) row[0].v[l + LPR * j] = e[i].v[j];
            __syncwarp();
            e[i] = row[l];
        }
        uint32_t m = largest_bits(e[i]);
        m = max(m, __shfl_xor_sync(~0u, m, 1));
        m = max(m, __shfl_xor_sync(~0u, m, 2));
        const uint32_t byte = mx_scale_byte(m), c = encode8(e[i], byte);
        // one lane of each quad has a block's byte: four lanes' make a word.  Blocks behind the last channel are all zeros: byte 0.
        uint32_t w = byte << 8 * (l >> 2 & 3);
        w |= __shfl_xor_sync(~0u, w, 4);
        if (LPR > 8) w |= __shfl_xor_sync(~0u, w, 8);
        if (r < rows && word) *reinterpret_cast<uint32_t*>(to) = c;
        if ((l & 15) == 0) tile[l >> 4][r] = w;
    }
    // (stored by the warps as they have them, a word of two lanes a row: 16384 x 8192 bf16 74 us, like this 63)
    __syncthreads();
    const int h = threadIdx.x / ROWS, r = threadIdx.x % ROWS;
    if (threadIdx.x < (LPR == 32 ? 2 : 1) * ROWS && r < rows && kt + h < ktiles)
        *reinterpret_cast<uint32_t*>(scales + mx_scale_offset(row0 + r, 4 * (kt + h), ktiles)) = tile[h][r];
}

template <class T, bool VEC, int LPR>
__global__ void __launch_bounds__(kThreads)
dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, T* __restrict__ y, int64_t ldy, int M, int K, int ktiles) {
    constexpr int ROWS = 8 * kRows, AT = 32 / LPR, BATCH = kRows / AT;
    __shared__ Eight<T> turn[VEC ? 1 : kThreads];
    grid_dependency_wait();
    grid_dependency_release();
    const int l = threadIdx.x % LPR, at = threadIdx.x % 32 / LPR, warp = threadIdx.x >> 5;
    const int wide = LPR == 32 ? (ktiles + 1) / 2 : 1, kt = blockIdx.x % wide * 2;
    const int64_t row0 = (int64_t)(blockIdx.x / wide) * ROWS;
    const int rows = (int)min((int64_t)ROWS, M - row0), k0 = kt * 128;
    const int64_t ldc = 16 * (int64_t)mx_blocks(K);
    const bool word = ((k0 + l * 8) & ~31) < K;
    const int r0 = warp * kRows + at;
    const uint8_t* from = codes + (row0 + r0) * ldc + (k0 >> 1) + l * 4;
    const uint8_t* sf = scales + mx_scale_offset(row0 + r0, 4 * (kt + (l >> 4)), ktiles);   // the next row's is 16 bytes on: a CTA's rows share a tile
    uint32_t c[BATCH], s[BATCH];   // a word of codes, the scales of the four blocks that it is one of
#pragma unroll
    for (int i = 0; i < BATCH; ++i, from += AT * ldc) {
        c[i] = s[i] = 0;
        if (r0 + i * AT < rows && word) {
            c[i] = __ldg(reinterpret_cast<const uint32_t*>(from));
            s[i] = __ldg(reinterpret_cast<const uint32_t*>(sf + i * AT * 16));
        }
    }
    T* p = y + (row0 + r0) * ldy + k0;
#pragma unroll
    for (int i = 0; i < BATCH; ++i, p += AT * ldy) {
        const int r = r0 + i * AT;
        constexpr bool LINES = VEC && sizeof(T) == 4 && LPR == 32;
        float s0, s1;   // of the first and the last four of the lane's channels
        if (LINES) {
            // fp32: channels 4 l .. and 128 + 4 l .., so that both stores are whole lines (16384 x 8192: 99 us, 140 without)
            const uint32_t a = __shfl_sync(~0u, c[i], l >> 1), b = __shfl_sync(~0u, c[i], 16 + (l >> 1));
            const uint32_t sa = __shfl_sync(~0u, s[i], 0), sb = __shfl_sync(~0u, s[i], 16);
            c[i] = l & 1 ? (a >> 16) | (b & 0xFFFF0000u) : (a & 0xFFFFu) | (b << 16);
            s0 = mx_scale(sa >> 8 * (l >> 3) & 255u);
            s1 = mx_scale(sb >> 8 * (l >> 3) & 255u);
        } else {
            s0 = s1 = mx_scale(s[i] >> 8 * (l >> 2 & 3) & 255u);
        }
        __half2 h[4];
        mx_decode8(c[i], h);
        Eight<T> e;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 f = __half22float2(h[j]);
            put2(e, 2 * j, f.x * (j < 2 ? s0 : s1), f.y * (j < 2 ? s0 : s1));
        }
        if (LINES) {
            const float4* const f = reinterpret_cast<const float4*>(e.v);
            if (r < rows && k0 + 4 * l < K) *reinterpret_cast<float4*>(p + 4 * l) = f[0];
            if (r < rows && k0 + 128 + 4 * l < K) *reinterpret_cast<float4*>(p + 128 + 4 * l) = f[1];
        } else if (VEC) {
            if (r < rows && k0 + l * 8 < K) store8(e, p + l * 8);
        } else {
            Eight<T>* const row = turn + (threadIdx.x - l);
            __syncwarp();
            row[l] = e;
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (r < rows && k0 + l + LPR * j < K) p[l + LPR * j] = row[0].v[l + LPR * j];
        }
    }
}

// 16-byte accesses: every row starts on a 16-byte boundary, as the matrix does, and ends with a whole one.
bool whole_vectors(int64_t ld, int K, int elem_bytes) { return ld * elem_bytes % 16 == 0 && K % 8 == 0; }

sbnn_status check_matrix(const char* what, const void* p, int type, int64_t ld, int M, int K) {
    if (M < 0 || K <= 0) return fail(SBNN_ERR_SHAPE, "bad shape M=%d K=%d", M, K);
    if (K > 1 << 30) return fail(SBNN_ERR_UNSUPPORTED, "K=%d: 2^30 at most", K);
    if (type != SBNN_F32 && type != SBNN_F16 && type != SBNN_BF16) return fail(SBNN_ERR_UNSUPPORTED, "%s: unknown element type %d", what, type);
    if (ld < K) return fail(SBNN_ERR_SHAPE, "%s: rows of %d elements do not fit a stride of %lld", what, K, (long long)ld);
    if (!aligned16(p)) return fail(SBNN_ERR_ALIGN, "%s must be 16-byte aligned", what);
    return SBNN_OK;
}

// Lanes of a row, and the CTAs.
sbnn_status grid_of(int M, int K, int* lpr, unsigned* blocks) {
    *lpr = K > 128 ? 32 : K > 64 ? 16 : 8;
    const int64_t n = ((int64_t)M + 8 * kRows - 1) / (8 * kRows) * ((mx_ktiles(K) + 1) / 2);
    if (n > 0x7fffffff) return fail(SBNN_ERR_SHAPE, "tensor too large");
    *blocks = (unsigned)n;
    return SBNN_OK;
}

template <class T, bool VEC>
auto quantize_for(int lpr) { return lpr == 32 ? quantize_kernel<T, VEC, 32> : lpr == 16 ? quantize_kernel<T, VEC, 16> : quantize_kernel<T, VEC, 8>; }
template <class T, bool VEC>
auto dequantize_for(int lpr) { return lpr == 32 ? dequantize_kernel<T, VEC, 32> : lpr == 16 ? dequantize_kernel<T, VEC, 16> : dequantize_kernel<T, VEC, 8>; }

template <class T>
sbnn_status quantize_as(const void* x, int64_t ldx, uint8_t* codes, uint8_t* scales, int M, int K, cudaStream_t st) {
    int lpr;
    unsigned blocks;
    const sbnn_status r = grid_of(M, K, &lpr, &blocks);
    if (r != SBNN_OK) return r;
    auto* const kernel = whole_vectors(ldx, K, sizeof(T)) ? quantize_for<T, true>(lpr) : quantize_for<T, false>(lpr);
    ChainedLaunchScope chained;
    SBNN_CUDA_TRY(launch_kernel(kernel, dim3(blocks), dim3(kThreads), 0, st, static_cast<const T*>(x), ldx, codes, scales, M, K, mx_ktiles(K)));
    return SBNN_OK;
}
template <class T>
sbnn_status dequantize_as(const uint8_t* codes, const uint8_t* scales, void* y, int64_t ldy, int M, int K, cudaStream_t st) {
    int lpr;
    unsigned blocks;
    const sbnn_status r = grid_of(M, K, &lpr, &blocks);
    if (r != SBNN_OK) return r;
    auto* const kernel = whole_vectors(ldy, K, sizeof(T)) ? dequantize_for<T, true>(lpr) : dequantize_for<T, false>(lpr);
    ChainedLaunchScope chained;
    SBNN_CUDA_TRY(launch_kernel(kernel, dim3(blocks), dim3(kThreads), 0, st, codes, scales, static_cast<T*>(y), ldy, M, K, mx_ktiles(K)));
    return SBNN_OK;
}

}  // namespace

sbnn_status mxfp4_quantize_launch(const void* x, int x_type, int64_t ldx, uint8_t* codes, uint8_t* scales, int M, int K, cudaStream_t st) {
    switch (x_type) {
        case SBNN_F32: return quantize_as<float>(x, ldx, codes, scales, M, K, st);
        case SBNN_F16: return quantize_as<__half>(x, ldx, codes, scales, M, K, st);
        default: return quantize_as<__nv_bfloat16>(x, ldx, codes, scales, M, K, st);
    }
}

}  // namespace sbnn

using namespace sbnn;

extern "C" sbnn_status sbnn_mxfp4_bytes(int M, int K, int64_t* codes_bytes, int64_t* scales_bytes) {
    clear_error();
    if (!codes_bytes || !scales_bytes) return fail(SBNN_ERR_NULL, "codes_bytes and scales_bytes must not be NULL");
    if (M < 0 || K <= 0) return fail(SBNN_ERR_SHAPE, "bad shape M=%d K=%d", M, K);
    if (K > 1 << 30) return fail(SBNN_ERR_UNSUPPORTED, "K=%d: 2^30 at most", K);
    *codes_bytes = (int64_t)M * 16 * mx_blocks(K);
    *scales_bytes = (((int64_t)M + 127) / 128) * 512 * mx_ktiles(K);
    return SBNN_OK;
}

extern "C" sbnn_status sbnn_mxfp4_quantize(const void* x_dev, int x_type, int64_t ldx, uint8_t* codes_dev, uint8_t* scales_dev, int M, int K,
                                           void* cuda_stream) {
    clear_error();
    if (!x_dev || !codes_dev || !scales_dev) return fail(SBNN_ERR_NULL, "x_dev, codes_dev and scales_dev must not be NULL");
    sbnn_status r = check_matrix("x_dev", x_dev, x_type, ldx, M, K);
    if (r != SBNN_OK) return r;
    if (!aligned16(codes_dev) || !aligned16(scales_dev)) return fail(SBNN_ERR_ALIGN, "codes_dev and scales_dev must be 16-byte aligned");
    if (M == 0) return SBNN_OK;
    if ((r = check_device()) != SBNN_OK || (r = check_device_memory({x_dev, codes_dev, scales_dev})) != SBNN_OK) return r;
    return mxfp4_quantize_launch(x_dev, x_type, ldx, codes_dev, scales_dev, M, K, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" sbnn_status sbnn_mxfp4_dequantize(const uint8_t* codes_dev, const uint8_t* scales_dev, void* y_dev, int y_type, int64_t ldy, int M, int K,
                                             void* cuda_stream) {
    clear_error();
    if (!codes_dev || !scales_dev || !y_dev) return fail(SBNN_ERR_NULL, "codes_dev, scales_dev and y_dev must not be NULL");
    sbnn_status r = check_matrix("y_dev", y_dev, y_type, ldy, M, K);
    if (r != SBNN_OK) return r;
    if (!aligned16(codes_dev) || !aligned16(scales_dev)) return fail(SBNN_ERR_ALIGN, "codes_dev and scales_dev must be 16-byte aligned");
    if (M == 0) return SBNN_OK;
    if ((r = check_device()) != SBNN_OK || (r = check_device_memory({codes_dev, scales_dev, y_dev})) != SBNN_OK) return r;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    switch (y_type) {
        case SBNN_F32: return dequantize_as<float>(codes_dev, scales_dev, y_dev, ldy, M, K, st);
        case SBNN_F16: return dequantize_as<__half>(codes_dev, scales_dev, y_dev, ldy, M, K, st);
        default: return dequantize_as<__nv_bfloat16>(codes_dev, scales_dev, y_dev, ldy, M, K, st);
    }
}
