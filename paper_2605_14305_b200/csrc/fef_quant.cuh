// The 4-bit output layer: its layout, and what its kernels share.
//
// A row of d weights is cut into groups of G = 32, 64 or 128; a weight is (q - z) * s with q in 0..15, one scale s
// (bfloat16) and one zero point z (0..15; 8 where the layer keeps none) per group.  q - z has five bits and s eight, so
// the product is exact in binary32.
//
// Layout (kBlock = 128 columns are a block; a row is padded to whole blocks):
//   packed [V][blocks * 64] bytes: of a block's sixteen 32-bit words, word 4 t + w holds the columns
//          32 w + 8 t .. 32 w + 8 t + 7, lowest nibble first.  16 consecutive bytes (one t) therefore hold eight
//          columns of every 32-column piece, which is what one lane of a matrix instruction's operand needs.
//   scale, zero [blocks][V rounded up to 32][128 / G]: what a block of consecutive rows needs lies together; the
//          entries behind d and V are zero.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "fef.h"
#include "fef_common.cuh"

namespace fef {
namespace quant {

constexpr int kBlock = 128;

struct Layer {
    const uint8_t* packed;
    const uint16_t* scale;
    const uint8_t* zero;  // or null
    int V, Vp, d, blocks, G;
};

struct ProductParams {
    Layer layer;
    const uint16_t* hidden;  // [rows][d]
    char* out;               // [rows][ldo]
    int64_t ldo;
    int rows;
    int32_t* status;         // or null; the kernel clears it
};

__device__ __forceinline__ float bf16_value(uint32_t h) { return __uint_as_float(h << 16); }

// The numbers q - z of the nibbles at bits 0..3 of a word's two halves (columns 0 and 4 of its eight; after shifts by 4, 8 and
// 12: 1 and 5, 2 and 6, 3 and 7), exact: 0x4300 | q is 128 + q in bfloat16, `centre` holds 128 + z twice.
__device__ __forceinline__ uint32_t centred_pair(uint32_t word, uint32_t centre) {
    uint32_t x, r;
    asm("lop3.b32 %0, %1, 0x000F000F, 0x43004300, 0xEA;" : "=r"(x) : "r"(word));  // (word & mask) | 128, 128
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(centre));
    return r;
}
__device__ __forceinline__ uint32_t centre_of(uint32_t z) { return 0x43004300u | z | z << 16; }

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// Logits from few hidden rows: false when this size is not for that kernel.
bool rows_kernel_takes(const ProductParams& P);
fef_status launch_rows_kernel(const ProductParams& P, fef_dtype dt, int dev, int sms, cudaStream_t stream);

// Logits from any number of rows.
size_t tiles_kernel_workspace(const ProductParams& P);
fef_status launch_tiles_kernel(const ProductParams& P, fef_dtype dt, void* workspace, int dev, int sms, cudaStream_t stream);

}  // namespace quant
}  // namespace fef
