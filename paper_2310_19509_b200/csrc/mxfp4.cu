// Rounding to microscaled 4-bit floating point and back (layout and arithmetic: mxfp4.cuh).
//
// Bound: memory.  A bf16 element is two bytes to read and 17/32 of a byte to write, or the other way round; the arithmetic
// is about five instructions an element.
#include <algorithm>

#include "common.h"
#include "mxfp4.cuh"
#include "pipeline.cuh"

namespace sbnn {
namespace {

// A CTA takes 128 rows x 128 channels: 16 lanes a row, eight channels a lane, so that the CTA's scales are one whole tile of
// 512 bytes, gathered in shared memory and written in one piece.  The eight loads of a thread are independent and
// issued before the first is used.
constexpr int kRows = 128;

template <class T, bool VEC>
__global__ void __launch_bounds__(256)
quantize_kernel(const T* __restrict__ x, int64_t ldx, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales, int M, int K, int ktiles) {
    __shared__ uint32_t tile[kRows];   // [row % 32][row / 32]: four scale bytes each
    grid_dependency_wait();
    grid_dependency_release();   // behind the wait: what starts now knows all launches before this one to be done
    const int lane = threadIdx.x & 31, half = lane >> 4, part = lane & 15, warp = threadIdx.x >> 5;
    const int kt = blockIdx.x % ktiles;
    const int64_t row0 = (int64_t)(blockIdx.x / ktiles) * kRows;
    const int k = kt * 128 + part * 8;
    const int rows = (int)min((int64_t)kRows, M - row0), n = min(8, K - k);
    const int64_t ldc = 16 * (int64_t)mx_blocks(K);
    constexpr int IT = kRows / 16;
    Eight<T> e[IT];
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        const int r = i * 16 + warp * 2 + half;
        if (r < rows && n > 0) {
            load8<VEC>(e[i], x + (row0 + r) * ldx + k, n);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) e[i].v[j] = from_float<T>(0.f);
        }
    }
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        const int r = i * 16 + warp * 2 + half;
        uint32_t m = largest_bits(e[i]);
        m = max(m, __shfl_xor_sync(~0u, m, 1));
        m = max(m, __shfl_xor_sync(~0u, m, 2));
        uint32_t byte = mx_scale_byte(m);
        const uint32_t c = encode8(e[i], byte);
        if (r < rows && (k & ~31) < K) *reinterpret_cast<uint32_t*>(codes + (row0 + r) * ldc + (k >> 1)) = c;
        // the four scales of the row: one of each quad of lanes.  Blocks behind the last channel are all zeros: byte 0.
        byte <<= 8 * (part >> 2);
        byte |= __shfl_xor_sync(~0u, byte, 4);
        byte |= __shfl_xor_sync(~0u, byte, 8);
        if (part == 0) tile[(r & 31) * 4 + (r >> 5)] = byte;
    }
    __syncthreads();
    const int t = threadIdx.x;
    if (t < kRows && (t >> 2) + 32 * (t & 3) < rows)
        reinterpret_cast<uint32_t*>(scales + (row0 / kRows * ktiles + kt) * 512)[t] = tile[t];
}

// A lane takes the eight channels of one word of codes.
template <class T, bool VEC>
__global__ void __launch_bounds__(256)
dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, T* __restrict__ y, int64_t ldy, int M, int K, int ktiles) {
    grid_dependency_wait();
    grid_dependency_release();   // behind the wait: what starts now knows all launches before this one to be done
    const int lane = threadIdx.x & 31, half = lane >> 4, part = lane & 15, warp = threadIdx.x >> 5;
    const int kt = blockIdx.x % ktiles;
    const int64_t row0 = (int64_t)(blockIdx.x / ktiles) * kRows;
    const int k = kt * 128 + part * 8;
    const int rows = (int)min((int64_t)kRows, M - row0), n = min(8, K - k);
    if (n <= 0) return;
    const int64_t ldc = 16 * (int64_t)mx_blocks(K);
    const uint8_t* st = scales + (row0 / kRows * ktiles + kt) * 512;
    constexpr int IT = kRows / 16;
    uint32_t c[IT], byte[IT];
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        const int r = i * 16 + warp * 2 + half;
        c[i] = byte[i] = 0;
        if (r < rows) {
            c[i] = __ldg(reinterpret_cast<const uint32_t*>(codes + (row0 + r) * ldc + (k >> 1)));
            byte[i] = __ldg(st + (r & 31) * 16 + (r >> 5) * 4 + (part >> 2));
        }
    }
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        const int r = i * 16 + warp * 2 + half;
        const float s = mx_scale(byte[i]);
        __half2 h[4];
        mx_decode8(c[i], h);
        Eight<T> e;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 f = __half22float2(h[j]);
            e.v[2 * j] = from_float<T>(f.x * s);
            e.v[2 * j + 1] = from_float<T>(f.y * s);
        }
        if (r < rows) store8<VEC>(e, y + (row0 + r) * ldy + k, n);
    }
}

// 16-byte accesses: every row starts on a 16-byte boundary and ends with a whole one.
bool whole_vectors(const void* p, int64_t ld, int K, int elem_bytes) { return aligned16(p) && ld * elem_bytes % 16 == 0 && K % 8 == 0; }

sbnn_status check_matrix(const char* what, const void* p, int type, int64_t ld, int M, int K) {
    if (M < 0 || K <= 0) return fail(SBNN_ERR_SHAPE, "bad shape M=%d K=%d", M, K);
    if (type != SBNN_F32 && type != SBNN_F16 && type != SBNN_BF16) return fail(SBNN_ERR_UNSUPPORTED, "%s: unknown element type %d", what, type);
    if (ld < K) return fail(SBNN_ERR_SHAPE, "%s: rows of %d elements do not fit a stride of %lld", what, K, (long long)ld);
    if (!aligned16(p)) return fail(SBNN_ERR_ALIGN, "%s must be 16-byte aligned", what);
    return SBNN_OK;
}

sbnn_status grid_of(int M, int K, unsigned* blocks) {
    const int64_t n = (int64_t)((M + (int64_t)kRows - 1) / kRows) * mx_ktiles(K);
    if (n > 0x7fffffff) return fail(SBNN_ERR_SHAPE, "tensor too large");
    *blocks = (unsigned)n;
    return SBNN_OK;
}

template <class T>
sbnn_status quantize_as(const void* x, int64_t ldx, uint8_t* codes, uint8_t* scales, int M, int K, cudaStream_t st) {
    unsigned blocks;
    const sbnn_status r = grid_of(M, K, &blocks);
    if (r != SBNN_OK) return r;
    auto* const kernel = whole_vectors(x, ldx, K, sizeof(T)) ? quantize_kernel<T, true> : quantize_kernel<T, false>;
    ChainedLaunchScope chained;
    SBNN_CUDA_TRY(launch_kernel(kernel, dim3(blocks), dim3(256), 0, st, static_cast<const T*>(x), ldx, codes, scales, M, K, mx_ktiles(K)));
    return SBNN_OK;
}
template <class T>
sbnn_status dequantize_as(const uint8_t* codes, const uint8_t* scales, void* y, int64_t ldy, int M, int K, cudaStream_t st) {
    unsigned blocks;
    const sbnn_status r = grid_of(M, K, &blocks);
    if (r != SBNN_OK) return r;
    auto* const kernel = whole_vectors(y, ldy, K, sizeof(T)) ? dequantize_kernel<T, true> : dequantize_kernel<T, false>;
    ChainedLaunchScope chained;
    SBNN_CUDA_TRY(launch_kernel(kernel, dim3(blocks), dim3(256), 0, st, codes, scales, static_cast<T*>(y), ldy, M, K, mx_ktiles(K)));
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
    if ((r = check_device()) != SBNN_OK) return r;
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
    if ((r = check_device()) != SBNN_OK) return r;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    switch (y_type) {
        case SBNN_F32: return dequantize_as<float>(codes_dev, scales_dev, y_dev, ldy, M, K, st);
        case SBNN_F16: return dequantize_as<__half>(codes_dev, scales_dev, y_dev, ldy, M, K, st);
        default: return dequantize_as<__nv_bfloat16>(codes_dev, scales_dev, y_dev, ldy, M, K, st);
    }
}
