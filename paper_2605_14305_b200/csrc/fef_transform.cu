// fef_hidden_transform: hidden states through one layer of a prediction head, ahead of the output layer:
//   out[r, j] = act( sum_k hidden[r, k] weight[j, k] + bias[j] ) + residual[r, j],
// products of bfloat16 numbers summed in binary32, everything behind them in binary32, one rounding to the output's type.
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <math.h>
#include <stdint.h>

#include "fef.h"
#include "fef_common.cuh"
#include "fef_device_math.cuh"

namespace fef {
namespace head {

struct Params {
    const __nv_bfloat16* hidden;
    const __nv_bfloat16* weight;
    const __nv_bfloat16* bias;      // [n] or null
    const __nv_bfloat16* residual;  // or null
    void* out;
    int64_t ld_hidden, ld_residual, ldo;
    int rows, n, d;
    int32_t* status;
};

template <int ACT>
__device__ __forceinline__ float activate(float y) {
    if constexpr (ACT == FEF_ACT_RELU) return y <= 0.f ? 0.f : y;   // (NaN stays)
    if constexpr (ACT == FEF_ACT_SILU) return __fdividef(y, 1.f + ex2_approx(-1.4426950408889634f * y));
    if constexpr (ACT == FEF_ACT_GELU) return 0.5f * y * erfcf(-0.70710678118654752f * y);
    if constexpr (ACT == FEF_ACT_GELU_TANH) {
        // (1 + tanh z) / 2 = 1 / (1 + e^(-2 z)),  z = sqrt(2 / pi) (y + 0.044715 y^3)
        const float z2 = y * fmaf(0.044715f * y, y, 1.f) * (2.f * 0.79788456080286536f * 1.4426950408889634f);
        return y / (1.f + ex2_approx(-z2));
    }
    return y;
}

template <class T>
__device__ __forceinline__ void store(void* out, int64_t at, float y) {
    if constexpr (sizeof(T) == 4)
        static_cast<float*>(out)[at] = y;
    else
        static_cast<__nv_bfloat16*>(out)[at] = __float2bfloat16_rn(y);
}

constexpr int kTile = 64, kDeep = 32;

template <int ACT, class T>
__global__ void __launch_bounds__(256) transform_kernel(const __grid_constant__ Params P) {
    __shared__ float a[kDeep][kTile + 4], w[kDeep][kTile + 4];
    const int r0 = blockIdx.y * kTile, j0 = blockIdx.x * kTile;
    const int tr = threadIdx.x / 16, tj = threadIdx.x % 16;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < P.d; k0 += kDeep) {
        for (int e = threadIdx.x; e < kTile * kDeep; e += 256) {
            const int row = e / kDeep, k = e % kDeep;
            const bool in = k0 + k < P.d;
            a[k][row] = in && r0 + row < P.rows ? __bfloat162float(P.hidden[static_cast<int64_t>(r0 + row) * P.ld_hidden + k0 + k]) : 0.f;
            w[k][row] = in && j0 + row < P.n ? __bfloat162float(P.weight[static_cast<int64_t>(j0 + row) * P.d + k0 + k]) : 0.f;
        }
        __syncthreads();
        for (int k = 0; k < kDeep; ++k)
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int y = 0; y < 4; ++y) acc[x][y] = fmaf(a[k][tr * 4 + x], w[k][tj * 4 + y], acc[x][y]);
        __syncthreads();
    }
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const int r = r0 + tr * 4 + x, j = j0 + tj * 4 + y;
            if (r >= P.rows || j >= P.n) continue;
            float v = acc[x][y];
            if (P.bias) v += __bfloat162float(P.bias[j]);
            v = activate<ACT>(v);
            if (P.residual) v += __bfloat162float(P.residual[static_cast<int64_t>(r) * P.ld_residual + j]);
            store<T>(P.out, static_cast<int64_t>(r) * P.ldo + j, v);
        }
}

template <int ACT>
static void launch(const Params& P, fef_dtype dt, cudaStream_t stream) {
    const dim3 grid((P.n + kTile - 1) / kTile, (P.rows + kTile - 1) / kTile);
    if (dt == FEF_F32)
        transform_kernel<ACT, float><<<grid, 256, 0, stream>>>(P);
    else
        transform_kernel<ACT, __nv_bfloat16><<<grid, 256, 0, stream>>>(P);
}

}  // namespace head
}  // namespace fef

extern "C" fef_status fef_hidden_transform(const void* hidden, int64_t ld_hidden, const void* weight, const void* bias,
                                           const void* residual, int64_t ld_residual, int rows, int n, int d,
                                           fef_activation activation, void* out, int64_t ldo, fef_dtype dt,
                                           int32_t* device_status, void* cuda_stream) {
    using namespace fef::head;
    if (dt != FEF_F32 && dt != FEF_BF16) return FEF_ERR_DTYPE;
    if (!hidden || !weight || !out) return FEF_ERR_INVALID_ARG;
    if (rows < 1 || rows > FEF_MAX_TRANSFORM || n < 1 || n > FEF_MAX_TRANSFORM || d < 8 || d > FEF_MAX_TRANSFORM || d % 8)
        return FEF_ERR_INVALID_ARG;
    if (ld_hidden < d || ldo < n || (residual && ld_residual < n)) return FEF_ERR_INVALID_ARG;
    const int64_t most = 1ll << 40;   // (pitches in elements)
    if (ld_hidden > most || ldo > most || (residual && ld_residual > most)) return FEF_ERR_INVALID_ARG;
    if (activation < FEF_ACT_NONE || activation > FEF_ACT_GELU_TANH) return FEF_ERR_INVALID_ARG;
    const int esize = dt == FEF_F32 ? 4 : 2;
    if ((reinterpret_cast<uintptr_t>(hidden) & 15) || (reinterpret_cast<uintptr_t>(weight) & 15) || ld_hidden % 8 ||
        (reinterpret_cast<uintptr_t>(bias) & 1) || (reinterpret_cast<uintptr_t>(residual) & 1) ||
        (reinterpret_cast<uintptr_t>(out) & (esize - 1)) || (reinterpret_cast<uintptr_t>(device_status) & 3))
        return FEF_ERR_ALIGNMENT;
    // the output may be the residual itself, element for element, and overlaps nothing else
    struct Range {
        uintptr_t from, to;
        Range(const void* p, int64_t rows, int64_t pitch, int64_t cols, int64_t size)
            : from(reinterpret_cast<uintptr_t>(p)), to(from + static_cast<uintptr_t>(((rows - 1) * pitch + cols) * size)) {}
        bool meets(const Range& o) const { return from < o.to && o.from < to; }
    };
    const Range o(out, rows, ldo, n, esize);
    if (o.meets(Range(hidden, rows, ld_hidden, d, 2)) || o.meets(Range(weight, n, d, d, 2)) || (bias && o.meets(Range(bias, 1, n, n, 2))))
        return FEF_ERR_INVALID_ARG;
    if (residual && o.meets(Range(residual, rows, ld_residual, n, 2)) &&
        !(residual == out && dt == FEF_BF16 && (ld_residual == ldo || rows == 1)))
        return FEF_ERR_INVALID_ARG;
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return FEF_ERR_CUDA;

    Params P = {};
    P.hidden = static_cast<const __nv_bfloat16*>(hidden);
    P.weight = static_cast<const __nv_bfloat16*>(weight);
    P.bias = static_cast<const __nv_bfloat16*>(bias);
    P.residual = static_cast<const __nv_bfloat16*>(residual);
    P.out = out;
    P.ld_hidden = ld_hidden;
    P.ld_residual = ld_residual;
    P.ldo = ldo;
    P.rows = rows;
    P.n = n;
    P.d = d;
    P.status = device_status;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (device_status && cudaMemsetAsync(device_status, 0, sizeof(int32_t), stream) != cudaSuccess) return FEF_ERR_CUDA;
    switch (activation) {
        case FEF_ACT_NONE: launch<FEF_ACT_NONE>(P, dt, stream); break;
        case FEF_ACT_RELU: launch<FEF_ACT_RELU>(P, dt, stream); break;
        case FEF_ACT_SILU: launch<FEF_ACT_SILU>(P, dt, stream); break;
        case FEF_ACT_GELU: launch<FEF_ACT_GELU>(P, dt, stream); break;
        default: launch<FEF_ACT_GELU_TANH>(P, dt, stream); break;
    }
    return cudaGetLastError() == cudaSuccess ? FEF_OK : FEF_ERR_CUDA;
}
