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
constexpr int kUnits = 4;

// ------------------------------------------------------------------------------------------ quantize ----
// unit / blocks, in 32 bits where they do.
__device__ __forceinline__ int64_t row_of_unit(int64_t unit, int blocks) {
    return unit >> 32 ? unit / blocks : static_cast<int64_t>(static_cast<uint32_t>(unit) / static_cast<uint32_t>(blocks));
}

struct QuantizeParams {
    const uint16_t* weight;  // [V][d]
    uint8_t* packed;
    uint16_t* scale;
    uint8_t* zero;  // or null
    int V, Vp, d, blocks, G;
    int32_t* status;
};

// Half a warp per block of one row, kUnits blocks in turn; a lane takes eight columns, one word of nibbles.  Bound by instruction issue
// (85 % of the issue slots used, 29 % of the memory's time: 40000 x 4096 in 151 us = 2.7 TB/s): the rounding of every weight and a
// division by the blocks per row for every block; with an IEEE division for every weight the whole took four times as long.
//
// rint(w / s) without a division: w and s are bfloat16 numbers, w / s is below 16, and so a quotient that is no tie lies at
// least 1/1020 from every tie: |w/s - (n + 1/2)| = |2 w - (2 n + 1) s| / (2 s), whose numerator, unless it is zero, is at least
// half a unit of s's last place when w >= s / 4, and s has 255 such units at most.  w * (1 / s) is off by less than 1e-5; rounded
// to multiples of 2^-11 it is an exact tie where w / s is one and else stays on its side, and is then rounded to even.
__device__ __forceinline__ int whole_quotient(float w, float inv) {
    constexpr float kGrid = 6144.f, kWhole = 12582912.f;   // 1.5 * 2^12 and 1.5 * 2^23: their last places are 2^-11 and 1
    return __float_as_int(fmaf(w, inv, kGrid) + (kWhole - kGrid)) - 0x4B400000;
}

template <int G, bool ZERO>
__device__ __forceinline__ void quantize_unit(const QuantizeParams& P, int64_t unit, int p, const uint4& raw) {
    const bool there = unit < static_cast<int64_t>(P.Vp) * P.blocks;
    const int64_t v = there ? row_of_unit(unit, P.blocks) : 0;
    const int c = there ? static_cast<int>(unit - v * P.blocks) : 0;
    const bool real = there && v < P.V && c * kBlock + p * 8 < P.d;  // (d is a multiple of 32: a lane's columns exist or do not)
    float w[8];
    unpack<FEF_BF16>(raw, w);
    // the largest magnitude, as bits (they order like the values; infinities and NaN are 0x7F80 and above)
    const uint32_t m2 = __vmaxu2(__vmaxu2(raw.x & 0x7FFF7FFFu, raw.y & 0x7FFF7FFFu), __vmaxu2(raw.z & 0x7FFF7FFFu, raw.w & 0x7FFF7FFFu));
    uint32_t most = max(m2 & 0xFFFFu, m2 >> 16);
    float lo = 0.f, hi = 0.f;
    if constexpr (ZERO) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            lo = fminf(lo, w[j]);
            hi = fmaxf(hi, w[j]);
        }
    }
    constexpr int kLanes = G / 8;
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1) {
        most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
        if constexpr (ZERO) {
            lo = fminf(lo, __shfl_xor_sync(0xFFFFFFFFu, lo, o));
            hi = fmaxf(hi, __shfl_xor_sync(0xFFFFFFFFu, hi, o));
        }
    }
    const float range = __fdiv_rn(ZERO ? hi - lo : bf16_value(most), ZERO ? 15.f : 7.f);
    const bool bad = most >= 0x7F80u || !(range < INFINITY);
    const uint16_t sbits = bad ? uint16_t(0x7FC0) : __bfloat16_as_ushort(__float2bfloat16_rn(range));  // (bad: the values are NaN)
    const float s = bf16_value(sbits);
    int z = ZERO ? 0 : 8;
    if (ZERO && s > 0.f) z = static_cast<int>(fminf(fmaxf(rintf(__fdiv_rn(-lo, s)), 0.f), 15.f));
    uint32_t nibbles = 0;
    if (s > 1e-30f) {   // (not NaN; 1 / s is an ordinary number)
        float inv;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            int q = whole_quotient(w[j], inv) + z;   // (without zero points |w / s| is below 7.04: nothing to clamp)
            if constexpr (ZERO) q = min(max(q, 0), 15);
            nibbles += static_cast<uint32_t>(q) << (4 * j);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float q = s > 0.f ? fminf(fmaxf(rintf(__fdiv_rn(w[j], s)) + static_cast<float>(z), 0.f), 15.f) : static_cast<float>(z);
            nibbles |= static_cast<uint32_t>(q) << (4 * j);
        }
    }
    // columns 32 (p / 4) + 8 (p % 4) ..: word 4 (p % 4) + p / 4 of the block
    if (there && v < P.V)
        *reinterpret_cast<uint32_t*>(P.packed + (v * P.blocks + c) * 64 + ((p & 3) * 4 + (p >> 2)) * 4) = nibbles;
    if (there && p % kLanes == 0) {
        const int64_t at = (static_cast<int64_t>(c) * P.Vp + v) * (kBlock / G) + p / kLanes;
        P.scale[at] = real ? sbits : uint16_t(0);
        if constexpr (ZERO) P.zero[at] = real ? static_cast<uint8_t>(z) : uint8_t(0);
        if (real && bad) report(P.status, FEF_ERR_NONFINITE);
    }
}

template <int G, bool ZERO>
__global__ void __launch_bounds__(kThreads) quantize_kernel(const __grid_constant__ QuantizeParams P) {
    const int lane = threadIdx.x & 31, p = lane & 15;   // piece of eight columns
    const int64_t unit0 = (static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5)) * (2 * kUnits) + (lane >> 4);
    uint4 raw[kUnits];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {   // (all loads first)
        const int64_t unit = unit0 + 2 * u;
        const int64_t v = row_of_unit(unit, P.blocks);
        const int k = static_cast<int>(unit - v * P.blocks) * kBlock + p * 8;
        raw[u] = v < P.V && k < P.d ? ld_global_nc_v4(P.weight + v * P.d + k) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) quantize_unit<G, ZERO>(P, unit0 + 2 * u, p, raw[u]);
}

// ---------------------------------------------------------------------------------------- dequantize ----
// The same lanes; bound by the bytes of the values written (40000 x 4096 in 136 us = 5.4 TB/s).
__global__ void __launch_bounds__(kThreads) dequantize_kernel(const __grid_constant__ Layer P, float* __restrict__ out) {
    const int lane = threadIdx.x & 31, p = lane & 15;
    const int64_t unit = (static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5)) * 2 + (lane >> 4);
    if (unit >= static_cast<int64_t>(P.V) * P.blocks) return;
    const int64_t v = row_of_unit(unit, P.blocks);
    const int c = static_cast<int>(unit - v * P.blocks), k = c * kBlock + p * 8;
    if (k >= P.d) return;
    const uint32_t q = __ldg(reinterpret_cast<const uint32_t*>(P.packed + unit * 64) + (p & 3) * 4 + (p >> 2));
    const int64_t at = (static_cast<int64_t>(c) * P.Vp + v) * (kBlock / P.G) + p * 8 / P.G;
    const float s = bf16_value(__ldg(P.scale + at));
    const int z = P.zero ? __ldg(P.zero + at) : 8;
    float y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = static_cast<float>(static_cast<int>(q >> (4 * j) & 15u) - z) * s;
    float* to = out + v * P.d + k;   // (a multiple of 32 bytes from the start)
    if (reinterpret_cast<uintptr_t>(to) & 31) {
        *reinterpret_cast<float4*>(to) = make_float4(y[0], y[1], y[2], y[3]);
        *reinterpret_cast<float4*>(to + 4) = make_float4(y[4], y[5], y[6], y[7]);
    } else {
        asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]),
                     "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7])
                     : "memory");
    }
}

template <int G>
static void launch_quantize(const QuantizeParams& P, unsigned grid, cudaStream_t stream) {
    if (P.zero)
        quantize_kernel<G, true><<<grid, kThreads, 0, stream>>>(P);
    else
        quantize_kernel<G, false><<<grid, kThreads, 0, stream>>>(P);
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
    const int64_t grid = (units + 2 * kUnits * kWarps - 1) / (2 * kUnits * kWarps);
    if (grid > 0x7FFFFFFF) return FEF_ERR_INVALID_ARG;
    switch (group) {
        case 32: launch_quantize<32>(P, static_cast<unsigned>(grid), stream); break;
        case 64: launch_quantize<64>(P, static_cast<unsigned>(grid), stream); break;
        default: launch_quantize<128>(P, static_cast<unsigned>(grid), stream);
    }
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
    const int64_t grid = (static_cast<int64_t>(V) * W.blocks + 2 * kWarps - 1) / (2 * kWarps);
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
