// The output layer in 4 bits: fef_lmhead_quantize, fef_lmhead_dequantize, and the entry point of
// fef_lmhead_logits_quantized (layout: fef_quant.cuh).
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "fef.h"
#include "fef_common.cuh"
#include "fef_device_math.cuh"
#include "fef_quant.cuh"

namespace fef {
namespace quant {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

// ------------------------------------------------------------------------------------------ quantize ----
struct QuantizeParams {
    const uint16_t* weight;  // [V][d]
    uint8_t* packed;
    uint16_t* scale;
    uint8_t* zero;  // or null
    int V, Vp, d, blocks, G;
    int32_t* status;
};

// One warp per block of one row: lane 8 w... holds the four columns 4 lane .. 4 lane + 3.
__global__ void __launch_bounds__(kThreads) quantize_kernel(const __grid_constant__ QuantizeParams P) {
    const int lane = threadIdx.x & 31;
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
    if (unit >= static_cast<int64_t>(P.Vp) * P.blocks) return;
    const int c = static_cast<int>(unit % P.blocks), v = static_cast<int>(unit / P.blocks);
    const int k = c * kBlock + lane * 4;
    float w[4] = {0.f, 0.f, 0.f, 0.f};
    const bool real = v < P.V && k < P.d;  // (d is a multiple of 32: a lane's four columns exist or do not)
    if (real) {
        const uint2 r = *reinterpret_cast<const uint2*>(P.weight + static_cast<int64_t>(v) * P.d + k);
        w[0] = __uint_as_float(r.x << 16);
        w[1] = __uint_as_float(r.x & 0xFFFF0000u);
        w[2] = __uint_as_float(r.y << 16);
        w[3] = __uint_as_float(r.y & 0xFFFF0000u);
    }
    float lo = fminf(fminf(w[0], w[1]), fminf(w[2], w[3])), hi = fmaxf(fmaxf(w[0], w[1]), fmaxf(w[2], w[3]));
    // (differences of infinities and NaN are NaN: bad stays 0 for numbers alone)
    float bad = (w[0] - w[0]) + (w[1] - w[1]) + (w[2] - w[2]) + (w[3] - w[3]);
    const int lanes = P.G / 4;
    for (int o = 1; o < lanes; o <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xFFFFFFFFu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xFFFFFFFFu, hi, o));
        bad += __shfl_xor_sync(0xFFFFFFFFu, bad, o);
    }
    lo = fminf(lo, 0.f);
    hi = fmaxf(hi, 0.f);
    const float range = P.zero ? __fdiv_rn(hi - lo, 15.f) : __fdiv_rn(fmaxf(hi, -lo), 7.f);
    uint16_t sbits = __bfloat16_as_ushort(__float2bfloat16_rn(range));
    if (!(range < INFINITY)) bad = range;
    if (bad != 0.f) sbits = 0x7FC0;  // the group's values are NaN
    const float s = bf16_value(sbits);
    float z = P.zero ? 0.f : 8.f;
    if (P.zero && s > 0.f) z = fminf(fmaxf(rintf(__fdiv_rn(-lo, s)), 0.f), 15.f);
    uint32_t nibbles = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float q = s > 0.f ? fminf(fmaxf(rintf(__fdiv_rn(w[j], s)) + z, 0.f), 15.f) : z;
        nibbles |= static_cast<uint32_t>(q) << (4 * j);
    }
    // columns 4 lane .. 4 lane + 3: piece w = lane / 8, t = (lane / 2) % 4, upper or lower half of the word
    if (v < P.V)
        *reinterpret_cast<uint16_t*>(P.packed + static_cast<int64_t>(v) * P.blocks * 64 + c * 64 + ((lane >> 1) & 3) * 16 +
                                     (lane >> 3) * 4 + (lane & 1) * 2) = static_cast<uint16_t>(nibbles);
    if (lane % lanes == 0) {
        const int64_t at = (static_cast<int64_t>(c) * P.Vp + v) * (kBlock / P.G) + lane / lanes;
        P.scale[at] = real ? sbits : uint16_t(0);
        if (P.zero) P.zero[at] = real ? static_cast<uint8_t>(z) : uint8_t(0);
        if (real && bad != 0.f) report(P.status, FEF_ERR_NONFINITE);
    }
}

// ---------------------------------------------------------------------------------------- dequantize ----
__global__ void __launch_bounds__(kThreads) dequantize_kernel(const __grid_constant__ Layer P, float* __restrict__ out) {
    const int lane = threadIdx.x & 31;
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
    if (unit >= static_cast<int64_t>(P.V) * P.blocks) return;
    const int c = static_cast<int>(unit % P.blocks), v = static_cast<int>(unit / P.blocks);
    const int k = c * kBlock + lane * 4;
    if (k >= P.d) return;
    const uint32_t nibbles = *reinterpret_cast<const uint16_t*>(P.packed + static_cast<int64_t>(v) * P.blocks * 64 + c * 64 +
                                                                ((lane >> 1) & 3) * 16 + (lane >> 3) * 4 + (lane & 1) * 2);
    const int64_t at = (static_cast<int64_t>(c) * P.Vp + v) * (kBlock / P.G) + lane * 4 / P.G;
    const float s = bf16_value(P.scale[at]);
    const int z = P.zero ? P.zero[at] : 8;
    float4 r;
    r.x = static_cast<float>(static_cast<int>(nibbles & 15u) - z) * s;
    r.y = static_cast<float>(static_cast<int>(nibbles >> 4 & 15u) - z) * s;
    r.z = static_cast<float>(static_cast<int>(nibbles >> 8 & 15u) - z) * s;
    r.w = static_cast<float>(static_cast<int>(nibbles >> 12) - z) * s;
    *reinterpret_cast<float4*>(out + static_cast<int64_t>(v) * P.d + k) = r;
}

// ---------------------------------------------------------------------------------------------- host ----
static bool layer_ok(int V, int d, int G) {
    return V >= 1 && V <= (1 << 28) && (G == 32 || G == 64 || G == 128) && d >= G && d <= (1 << 20) && d % G == 0;
}
static Layer make_layer(const void* packed, const void* scale, const void* zero, int V, int d, int G) {
    Layer W;
    W.packed = static_cast<const uint8_t*>(packed);
    W.scale = static_cast<const uint16_t*>(scale);
    W.zero = static_cast<const uint8_t*>(zero);
    W.V = V;
    W.Vp = (V + 31) / 32 * 32;
    W.d = d;
    W.blocks = (d + kBlock - 1) / kBlock;
    W.G = G;
    return W;
}
static bool aligned32(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 31) == 0; }
static bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
static int device_and_sms(int* dev) {
    static int sms[64];
    *dev = -1;
    if (cudaGetDevice(dev) != cudaSuccess || *dev < 0 || *dev >= 64) return 0;
    if (!sms[*dev] && cudaDeviceGetAttribute(&sms[*dev], cudaDevAttrMultiProcessorCount, *dev) != cudaSuccess) return 0;
    return sms[*dev];
}

}  // namespace quant
}  // namespace fef

extern "C" {

fef_status fef_lmhead_quantize(const void* weight, int V, int d, int group, void* packed, void* scale, void* zero,
                               int32_t* device_status, void* cuda_stream) {
    using namespace fef;
    using namespace fef::quant;
    if (!weight || !packed || !scale || !layer_ok(V, d, group)) return FEF_ERR_INVALID_ARG;
    if (!aligned16(weight) || !aligned32(packed) || !aligned16(scale) || !aligned16(zero)) return FEF_ERR_ALIGNMENT;
    int dev;
    const int sms = device_and_sms(&dev);
    if (sms < 1) return FEF_ERR_CUDA;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (device_status && cudaMemsetAsync(device_status, 0, sizeof(int32_t), stream) != cudaSuccess) return FEF_ERR_CUDA;
    QuantizeParams P;
    const Layer W = make_layer(packed, scale, zero, V, d, group);
    P.weight = static_cast<const uint16_t*>(weight);
    P.packed = static_cast<uint8_t*>(packed);
    P.scale = static_cast<uint16_t*>(scale);
    P.zero = static_cast<uint8_t*>(zero);
    P.V = V;
    P.Vp = W.Vp;
    P.d = d;
    P.blocks = W.blocks;
    P.G = group;
    P.status = device_status;
    const int64_t units = static_cast<int64_t>(W.Vp) * W.blocks;
    const int64_t grid = (units + kWarps - 1) / kWarps;
    if (grid > 0x7FFFFFFF) return FEF_ERR_INVALID_ARG;
    quantize_kernel<<<static_cast<unsigned>(grid), kThreads, 0, stream>>>(P);
    return cudaGetLastError() == cudaSuccess ? FEF_OK : FEF_ERR_CUDA;
}

fef_status fef_lmhead_dequantize(const void* packed, const void* scale, const void* zero, int V, int d, int group,
                                 float* values, void* cuda_stream) {
    using namespace fef;
    using namespace fef::quant;
    if (!packed || !scale || !values || !layer_ok(V, d, group)) return FEF_ERR_INVALID_ARG;
    if (!aligned32(packed) || !aligned16(scale) || !aligned16(zero) || !aligned16(values)) return FEF_ERR_ALIGNMENT;
    int dev;
    const int sms = device_and_sms(&dev);
    if (sms < 1) return FEF_ERR_CUDA;
    const Layer W = make_layer(packed, scale, zero, V, d, group);
    const int64_t grid = (static_cast<int64_t>(V) * W.blocks + kWarps - 1) / kWarps;
    if (grid > 0x7FFFFFFF) return FEF_ERR_INVALID_ARG;
    dequantize_kernel<<<static_cast<unsigned>(grid), kThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(W, values);
    return cudaGetLastError() == cudaSuccess ? FEF_OK : FEF_ERR_CUDA;
}

size_t fef_lmhead_logits_quantized_workspace_bytes(int rows, int V, int d, int group) {
    using namespace fef::quant;
    if (rows < 1 || rows > (1 << 24) || !layer_ok(V, d, group)) return 0;
    ProductParams P = {};
    P.layer = make_layer(nullptr, nullptr, nullptr, V, d, group);
    P.rows = rows;
    return rows_kernel_takes(P) ? 256 : tiles_kernel_workspace(P);
}

fef_status fef_lmhead_logits_quantized(const void* hidden, const void* packed, const void* scale, const void* zero, int rows,
                                       int V, int d, int group, void* logits, int64_t ldo, fef_dtype dt,
                                       void* workspace, size_t workspace_bytes, int32_t* device_status, void* cuda_stream) {
    using namespace fef;
    using namespace fef::quant;
    if (dt != FEF_F32 && dt != FEF_BF16) return FEF_ERR_DTYPE;
    if (!hidden || !packed || !scale || !logits || !layer_ok(V, d, group)) return FEF_ERR_INVALID_ARG;
    if (rows < 1 || rows > (1 << 24) || ldo < V) return FEF_ERR_INVALID_ARG;
    if (!aligned16(hidden) || !aligned32(packed) || !aligned16(scale) || !aligned16(zero) || !aligned16(logits) ||
        (ldo * (dt == FEF_F32 ? 4 : 2)) % 16)
        return FEF_ERR_ALIGNMENT;
    ProductParams P;
    P.layer = make_layer(packed, scale, zero, V, d, group);
    P.hidden = static_cast<const uint16_t*>(hidden);
    P.out = static_cast<char*>(logits);
    P.ldo = ldo;
    P.rows = rows;
    P.status = device_status;
    const bool few = rows_kernel_takes(P);
    if (!few && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < tiles_kernel_workspace(P)))
        return FEF_ERR_WORKSPACE;
    int dev;
    const int sms = device_and_sms(&dev);
    if (sms < 1) return FEF_ERR_CUDA;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (few) return launch_rows_kernel(P, dt, dev, sms, stream);
    return launch_tiles_kernel(P, dt, workspace, dev, sms, stream);
}

}  // extern "C"
