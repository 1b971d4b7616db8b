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

// A nibble becomes a bfloat16 number by masking alone: the bit pattern v < 256 in the lower half of a bfloat16 (the mantissa
// and the lowest exponent bit) is the number v 2^-133, below and above the smallest normal number alike.  So the nibbles at
// bits 0..3 of each half of a word (columns 0 and 4 of its eight; after a shift by 8: 2 and 6) stand for q 2^-133, and those at
// bits 4..7 (1 and 5; 3 and 7) for 16 q 2^-133: two masks, one shift, two masks for eight weights.  The other operand is
// scaled by a power of two that keeps the products in binary32's normal range, a further 1/16 for the columns of the upper
// nibbles; all of this is exact, and the inverse is applied to the logits.
constexpr uint32_t kLowNibbles = 0x000F000Fu, kHighNibbles = 0x00F000F0u;
constexpr int kUsualShift = 100;

// The numbers q - z of such a pair (after shifts by 0, 4, 8, 12), exact: 0x4300 | q is 128 + q in bfloat16, `centre` holds 128 + z
// twice.  Three more instructions for four weights, and nothing left to correct.
__device__ __forceinline__ uint32_t centred_pair(uint32_t word, uint32_t centre) {
    uint32_t x, r;
    asm("lop3.b32 %0, %1, 0x000F000F, 0x43004300, 0xEA;" : "=r"(x) : "r"(word));  // (word & mask) | 128, 128
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(centre));
    return r;
}
__device__ __forceinline__ uint32_t centre_of(uint32_t z) { return 0x43004300u | z | z << 16; }

// The power of two a hidden row is scaled by, from the bfloat16 bits of its largest value: 2^100, or, for a row with values
// beyond 2^27 or with none above 2^-80, the one that brings its largest value near 2^126.  (An exponent of 255: the row holds
// NaN or an infinity, its logits are no numbers anyway.)
__device__ __forceinline__ int row_shift(uint32_t largest) {
    const int e = static_cast<int>(largest >> 7);   // biased
    return largest == 0u || (e >= 47 && e < 154) || e == 255 ? kUsualShift : 253 - e;
}
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }  // |e| < 127
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
