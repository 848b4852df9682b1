// What the two kernels that multiply microscaled 4-bit operands share: arguments, descriptors of block-scaled MMAs.
#pragma once

#include <stdint.h>

#include "pipeline.cuh"

namespace sbnn {

constexpr int kStep = 256;   // channels of a pipeline step: 128 bytes of codes a row

// Arguments of a product whose activations are rounded already.
struct MxProduct {
    const uint8_t *w_codes, *w_scales, *x_codes, *x_scales;
    const float* bias;
    void* y;
    int64_t ldy;
    int y_type, M, Cout, K, relu;
    int early;   // it follows the launch that rounds the activations, which has seen the end of all before it
};
// mxfp4.cu: rounds M rows of K elements (arguments checked by the callers).
sbnn_status mxfp4_quantize_launch(const void* x, int x_type, int64_t ldx, uint8_t* codes, uint8_t* scales, int M, int K, cudaStream_t st);
// conv_mxfp4_pair.cu: pairs of CTAs on 256 x 256 tiles.
sbnn_status conv_mxfp4_pair(const MxProduct& p, cudaStream_t st);

// Instruction descriptor: e2m1 x e2m1 -> fp32, both K-major, m x n, scales are powers of two (ue8m0), two a row and MMA;
// `half` says which two of the four bytes of a scale word.
__device__ __forceinline__ uint32_t mx_instr_desc(int m, int n, int half) {
    return ((uint32_t)(2 * half) << 4)         // B: scale factor id 0 or 2
           | (1u << 7) | (1u << 10)            // A and B: e2m1
           | ((uint32_t)(n >> 3) << 17) | (1u << 23) | ((uint32_t)(m >> 7) << 27)
           | ((uint32_t)(2 * half) << 29);     // A: scale factor id
}
// Descriptor of 512 bytes of scales in shared memory: 32 rows of 16 bytes, linear.
__device__ __forceinline__ uint64_t scale_desc(uint32_t smem) {
    uint64_t d = (uint64_t)((smem & 0x3FFFFu) >> 4);
    d |= (uint64_t)1 << 16;            // leading byte offset: not used, rows are 16 bytes
    d |= (uint64_t)(128 >> 4) << 32;   // groups of 8 rows are 128 bytes apart
    d |= (uint64_t)1 << 46;            // descriptor version; no swizzle
    return d;
}

}  // namespace sbnn
