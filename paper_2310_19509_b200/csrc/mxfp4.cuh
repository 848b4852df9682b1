// Microscaled 4-bit floating point: element and scale arithmetic and the layout of a matrix in that form, shared by the
// kernels that write, read and multiply it.
//
// A block is 32 consecutive channels of a row.  Its scale is a power of two, 2^(byte - 127), two exponents below that of the
// block's largest magnitude, so the largest element lands in [4, 8) and is rounded to 4 or 6.  Elements are e2m1 (0, 0.5, 1, 1.5,
// 2, 3, 4, 6 and a sign).  A matrix [M][K]:
//   codes   [M][16 * ceil(K / 32)] bytes, the element of the lower index in the lower half of a byte
//   scales  tiles of 128 rows x 4 blocks, 512 bytes each, the tiles of the same rows next to each other; inside a tile the
//           order is row % 32, row / 32, block, which is the order that the tensor core's scale memory wants them in: a tile
//           is one linear copy into shared memory and one copy from there.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

namespace sbnn {

__host__ __device__ constexpr int mx_blocks(int k) { return (k + 31) / 32; }
__host__ __device__ constexpr int mx_ktiles(int k) { return (k + 127) / 128; }
// Offset of the scale of (row, block) in a matrix of `ktiles` tiles a row.
__host__ __device__ constexpr int64_t mx_scale_offset(int64_t row, int block, int ktiles) {
    return ((row >> 7) * ktiles + (block >> 2)) * 512 + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3);
}

// Scale byte of a block from the bits of its largest magnitude (as fp32, sign cleared): floor(log2) - 2, the smallest scale
// 2^-127; 255 (not a number) for a block with an infinity or a NaN.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t largest_bits) {
    const int e = (int)(largest_bits >> 23);
    return e == 255 ? 255u : (uint32_t)max(e - 2, 0);
}
// 2^(127 - byte): what a block's elements are multiplied by, exactly, before they are rounded to e2m1.  0 for byte 255: the
// codes of such a block are zeros (its scale makes them NaN).
__device__ __forceinline__ float mx_inverse_scale(uint32_t byte) { return byte == 255u ? 0.f : __uint_as_float((254u - byte) << 23); }
// 2^(byte - 127); 2^-127 is subnormal, 255 is NaN.
__device__ __forceinline__ float mx_scale(uint32_t byte) {
    return __uint_as_float(byte == 255u ? 0x7FC00000u : byte == 0u ? 0x00400000u : byte << 23);
}

// Eight values, already divided by the scale, as e2m1: rounded to nearest, ties to even, 6 above 6; v[0] in the lowest bits.
__device__ __forceinline__ uint32_t mx_encode8(const float (&v)[8]) {
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}
// The eight values that a word of codes stands for, without their scale, as four pairs of fp16.
__device__ __forceinline__ void mx_decode8(uint32_t codes, __half2 (&v)[4]) {
    uint32_t r[4];
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
        : "r"(codes));
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<__half2*>(&r[i]);
}

// ---- eight consecutive elements of a row, as they come from memory -------------------------------
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

template <class T>
struct Eight {
    alignas(16) T v[8];
};
// From and to 16-byte aligned memory.
template <class T>
__device__ __forceinline__ void load8(Eight<T>& e, const T* p) {
    const uint4* q = reinterpret_cast<const uint4*>(p);
    uint4* d = reinterpret_cast<uint4*>(e.v);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) * 8 / 16); ++i) d[i] = __ldg(q + i);
}
template <class T>
__device__ __forceinline__ void store8(const Eight<T>& e, T* p) {
    uint4* q = reinterpret_cast<uint4*>(p);
    const uint4* d = reinterpret_cast<const uint4*>(e.v);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) * 8 / 16); ++i) q[i] = d[i];
}
// Two values into places i and i + 1.
__device__ __forceinline__ void put2(Eight<float>& e, int i, float a, float b) { e.v[i] = a, e.v[i + 1] = b; }
__device__ __forceinline__ void put2(Eight<__half>& e, int i, float a, float b) { *reinterpret_cast<__half2*>(e.v + i) = __floats2half2_rn(a, b); }
__device__ __forceinline__ void put2(Eight<__nv_bfloat16>& e, int i, float a, float b) {
    *reinterpret_cast<__nv_bfloat162*>(e.v + i) = __floats2bfloat162_rn(a, b);
}
// Bits of the largest magnitude of the eight, as fp32.  Magnitudes are compared by their bits, which puts infinities and NaN
// on top.
template <class T>
__device__ __forceinline__ uint32_t largest_bits(const Eight<T>& e) {
    uint32_t m = 0;
    if (sizeof(T) == 4) {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(e.v);
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, w[i] & 0x7FFFFFFFu);
        return m;
    }
    const uint32_t* w = reinterpret_cast<const uint32_t*>(e.v);
#pragma unroll
    for (int i = 0; i < 4; ++i) m = __vmaxu2(m, w[i] & 0x7FFF7FFFu);
    const unsigned short top = (unsigned short)max(m & 0xFFFFu, m >> 16);
    T t;
    *reinterpret_cast<unsigned short*>(&t) = top;
    return __float_as_uint(to_float(t));
}
// The eight as e2m1 under the scale `byte`.
template <class T>
__device__ __forceinline__ uint32_t encode8(const Eight<T>& e, uint32_t byte) {
    const float inv = mx_inverse_scale(byte);
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = to_float(e.v[i]) * inv;
    const uint32_t codes = mx_encode8(f);
    return byte == 255u ? 0u : codes;
}

}  // namespace sbnn
