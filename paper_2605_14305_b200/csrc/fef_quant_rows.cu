// fef_lmhead_logits_quantized for few hidden rows (up to 16): bound by the weight bytes.
//
// The weights are the left operand of m16n8k16 matrix instructions, 16 vocabulary rows at a time, the hidden rows the right
// one (8 or 16 columns).  A sum over k may be taken in any order as long as both operands agree on it, so a lane uses the
// columns as the packed layout hands them to it: 16 bytes of a row are the lane's share of a 128-column block, each of
// their four words two k-steps.  The products of a group are added up in binary32 by the matrix instructions, then
// scaled in binary32.
//
// One CTA per SM takes an even share of the vocabulary, in passes of up to 8 units of 32 rows.  A producer thread brings
// in two blocks (256 columns) of a pass's rows per stage by TMA, 128-byte-swizzled, with their scales and zero points; of the
// 16 consumer warps, warps i and i + 8 take unit i, one block of the stage each, and add their halves up at the end of
// the pass.  The hidden rows stay in shared memory, rearranged into operand order once.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "fef_device_math.cuh"
#include "fef_quant.cuh"
#include "fef_tensor_core.cuh"

namespace fef {
namespace quant {
namespace {

constexpr int kUnit = 32;                    // vocabulary rows of a warp: two 16-row operands
constexpr int kPassUnits = 8;
constexpr int kConsumers = 2 * kPassUnits;   // warps
constexpr int kThreads = (kConsumers + 1) * 32;
constexpr int kMaxStages = 6;
constexpr int kUnitBytes = kUnit * 128;      // one unit's rows, two blocks
constexpr size_t kSmemLimit = 232448;
constexpr unsigned long long kWaitNs = 1000000000ull;

struct Shared {
    uint64_t full[kMaxStages];
    uint64_t empty[kMaxStages];
    int abort_flag;
};

struct Plan {
    int units, pass_units, stages;
    uint32_t scale_bytes, zero_bytes;        // of one unit and block
    uint32_t scale_at, zero_at, stage_bytes; // offsets within a stage (scales of block 0, of block 1)
    uint32_t hidden_at, join_at, shared_at;
    size_t smem;
};

// Shared memory: stages (1024-byte aligned), hidden rows, the place where two warps join their sums, barriers.
Plan make_plan(const ProductParams& P, int sms) {
    Plan L = {};
    const Layer& W = P.layer;
    const int nt = P.rows > 8 ? 2 : 1;
    L.units = (W.V + kUnit - 1) / kUnit;
    const int grid = L.units < sms ? L.units : sms;
    const int share = (L.units + grid - 1) / grid;
    const int passes = (share + kPassUnits - 1) / kPassUnits;
    L.pass_units = (share + passes - 1) / passes;
    L.scale_bytes = kUnit * (kBlock / W.G) * 2;
    L.zero_bytes = W.zero ? kUnit * (kBlock / W.G) : 0;
    L.scale_at = L.pass_units * kUnitBytes;
    L.zero_at = L.scale_at + 2 * L.pass_units * L.scale_bytes;
    L.stage_bytes = (L.zero_at + 2 * L.pass_units * L.zero_bytes + 1023) / 1024 * 1024;
    const size_t hidden = static_cast<size_t>(W.blocks) * 2048 * nt;
    const size_t join = static_cast<size_t>(kPassUnits) * 8 * nt * 33 * 4;
    const size_t fixed = hidden + join + sizeof(Shared) + 1024;
    if (fixed + 2 * static_cast<size_t>(L.stage_bytes) > kSmemLimit) return L;  // stages stays 0: not for this kernel
    L.stages = static_cast<int>((kSmemLimit - fixed) / L.stage_bytes);
    if (L.stages > kMaxStages) L.stages = kMaxStages;
    L.hidden_at = L.stages * L.stage_bytes;
    L.join_at = L.hidden_at + static_cast<uint32_t>(hidden);
    L.shared_at = L.join_at + static_cast<uint32_t>(join);
    L.smem = L.shared_at + sizeof(Shared) + 1024;
    return L;
}

__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 lds_v4(uint32_t at) {
    uint4 r;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(at));
    return r;
}
// N scales (or zero points) of one row and block.
template <int N>
__device__ __forceinline__ void lds_u16s(uint32_t at, uint32_t (&v)[N]) {
    if constexpr (N == 1) {
        unsigned short x;
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(at));
        v[0] = x;
    } else {
        uint32_t w[N / 2];
        if constexpr (N == 2)
            asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(at));
        else
            asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at));
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = w[i / 2] >> (16 * (i & 1)) & 0xFFFFu;
    }
}
template <int N>
__device__ __forceinline__ void lds_u8s(uint32_t at, uint32_t (&v)[N]) {
    uint32_t w;
    if constexpr (N == 1)
        asm volatile("ld.shared.u8 %0, [%1];" : "=r"(w) : "r"(at));
    else if constexpr (N == 2)
        asm volatile("ld.shared.u16 %0, [%1];" : "=r"(w) : "r"(at));
    else
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w) : "r"(at));
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = w >> (8 * i) & 0xFFu;
}
// 1-D bulk copy global -> shared.
__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
                 "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}

template <int NT, int N, bool ZERO>   // 8 NT hidden rows, N groups per block
__global__ void __launch_bounds__(kThreads, 1)
product_rows_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ ProductParams P,
                    const __grid_constant__ Plan L, int out_bf16) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t base = smem_u32(smem);
    Shared& sh = *reinterpret_cast<Shared*>(smem + L.shared_at);
    volatile int* abort_flag = &sh.abort_flag;
    const Layer& W = P.layer;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < L.stages; ++s) {
            mbar_init(sh.full + s, 1);
            mbar_init(sh.empty + s, kConsumers);
        }
        sh.abort_flag = 0;
        mbar_fence_init();
        if (P.status && blockIdx.x == 0) *P.status = FEF_OK;
    }
    __syncthreads();

    const int unit_begin = static_cast<int>(static_cast<int64_t>(L.units) * blockIdx.x / gridDim.x);
    const int unit_end = static_cast<int>(static_cast<int64_t>(L.units) * (blockIdx.x + 1) / gridDim.x);
    const int steps = (W.blocks + 1) / 2;
    int issued = 0;

    if (warp == kConsumers) {
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int u0 = unit_begin; ok && u0 < unit_end; u0 += L.pass_units) {
                const int n = min(L.pass_units, unit_end - u0);
                for (int step = 0; step < steps; ++step) {
                    if (!mbar_wait_bounded(sh.empty + stage, phase ^ 1u, abort_flag, kWaitNs)) {
                        *abort_flag = 1;
                        report(P.status, FEF_ERR_TIMEOUT);
                        ok = false;
                        break;
                    }
                    const int blocks = min(2, W.blocks - 2 * step);
                    uint64_t* bar = sh.full + stage;
                    const uint32_t dst = base + stage * L.stage_bytes;
                    mbar_arrive_expect_tx(bar, n * (kUnitBytes + blocks * (L.scale_bytes + L.zero_bytes)));
                    for (int u = 0; u < n; ++u)
                        tma_load_2d(smem + stage * L.stage_bytes + u * kUnitBytes, &map, step * 128, (u0 + u) * kUnit, bar);
                    for (int h = 0; h < blocks; ++h) {
                        const int64_t at = (static_cast<int64_t>(2 * step + h) * W.Vp + static_cast<int64_t>(u0) * kUnit) * N;
                        bulk_copy(dst + L.scale_at + h * L.pass_units * L.scale_bytes, W.scale + at, n * L.scale_bytes, bar);
                        if constexpr (ZERO)
                            bulk_copy(dst + L.zero_at + h * L.pass_units * L.zero_bytes, W.zero + at, n * L.zero_bytes, bar);
                    }
                    ++issued;
                    if (++stage == L.stages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
            }
        }
    } else {
        // ---- hidden rows into operand order: 16 bytes per (block, word, row, t): columns 0 4, 1 5, 2 6, 3 7 of the eight
        const uint32_t hidden = base + L.hidden_at;
        for (int at = threadIdx.x; at < W.blocks * 128 * NT; at += kConsumers * 32) {
            const int t = at & 3, row = at / 4 % (8 * NT), cw = at / (32 * NT);
            const int k = (cw >> 2) * kBlock + (cw & 3) * 32 + t * 8;
            uint4 x = make_uint4(0u, 0u, 0u, 0u);
            if (row < P.rows && k < W.d) x = __ldg(reinterpret_cast<const uint4*>(P.hidden + static_cast<int64_t>(row) * W.d + k));
            uint4 y;
            y.x = __byte_perm(x.x, x.z, 0x5410);
            y.y = __byte_perm(x.x, x.z, 0x7632);
            y.z = __byte_perm(x.y, x.w, 0x5410);
            y.w = __byte_perm(x.y, x.w, 0x7632);
            *reinterpret_cast<uint4*>(smem + L.hidden_at + at * 16) = y;
        }
        asm volatile("bar.sync 1, %0;" ::"n"(kConsumers * 32) : "memory");

        const int half = warp >> 3, slot = warp & 7;
        const int g = lane >> 2, t = lane & 3;
        // Operand row g stands for vocabulary row g / 2 + 4 (g % 2) of its eight: a quarter-warp's two rows then lie in
        // different halves of the swizzled 128 bytes, and its 16-byte loads meet no bank twice.
        const int r = (g >> 1) + 4 * (g & 1);
        const uint32_t w_at = slot * kUnitBytes + r * 128 + (((half * 4 + t) ^ r) << 4);   // + 1024 per eight rows
        const uint32_t s_at = L.scale_at + half * L.pass_units * L.scale_bytes + (slot * kUnit + r) * N * 2;
        const uint32_t z_at = L.zero_at + half * L.pass_units * L.zero_bytes + (slot * kUnit + r) * N;
        float* join = reinterpret_cast<float*>(smem + L.join_at) + slot * 8 * NT * 33;
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        // (after a wait that ran out the passes go on without waits: the pairs' barriers stay matched)
        for (int u0 = unit_begin; u0 < unit_end; u0 += L.pass_units) {
            const bool mine = slot < min(L.pass_units, unit_end - u0);
            float acc[2][NT][4];
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[m][n][i] = 0.f;
            for (int step = 0; ok && step < steps; ++step) {
                if (!__all_sync(0xFFFFFFFFu, mbar_wait_bounded(sh.full + stage, phase, abort_flag, kWaitNs))) {
                    *abort_flag = 1;
                    if (lane == 0) report(P.status, FEF_ERR_TIMEOUT);
                    ok = false;
                    break;
                }
                const int block = 2 * step + half;
                if (mine && block < W.blocks) {
                    const uint32_t st = base + stage * L.stage_bytes;
                    uint4 q[4];        // operand rows g, g + 8 of both 16-row tiles
                    uint32_t s[4][N], z[4][N];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        q[i] = lds_v4(st + w_at + i * 1024);
                        lds_u16s<N>(st + s_at + i * 8 * N * 2, s[i]);
                        if constexpr (ZERO) lds_u8s<N>(st + z_at + i * 8 * N, z[i]);
                    }
                    const uint32_t h_at = hidden + block * (2048 * NT) + (g * 4 + t) * 16;
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        float part[2][NT][4];
                        uint32_t centre[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) centre[i] = ZERO ? centre_of(z[i][j]) : 0x43084308u;
#pragma unroll
                        for (int m = 0; m < 2; ++m)
#pragma unroll
                            for (int n = 0; n < NT; ++n)
#pragma unroll
                                for (int i = 0; i < 4; ++i) part[m][n][i] = 0.f;
#pragma unroll
                        for (int w = j * (4 / N); w < (j + 1) * (4 / N); ++w) {
                            uint4 h[NT];
#pragma unroll
                            for (int n = 0; n < NT; ++n) h[n] = lds_v4(h_at + w * (512 * NT) + n * 512);
#pragma unroll
                            for (int m = 0; m < 2; ++m) {
                                const uint4 &lo = q[2 * m], &hi = q[2 * m + 1];
                                const uint32_t a = w == 0 ? lo.x : w == 1 ? lo.y : w == 2 ? lo.z : lo.w;
                                const uint32_t b = w == 0 ? hi.x : w == 1 ? hi.y : w == 2 ? hi.z : hi.w;
                                const uint32_t ca = centre[2 * m], cb = centre[2 * m + 1];
                                const uint32_t a0 = nibble_pair(a, ca), b0 = nibble_pair(b, cb);
                                const uint32_t a1 = nibble_pair(a >> 4, ca), b1 = nibble_pair(b >> 4, cb);
                                const uint32_t a2 = nibble_pair(a >> 8, ca), b2 = nibble_pair(b >> 8, cb);
                                const uint32_t a3 = nibble_pair(a >> 12, ca), b3 = nibble_pair(b >> 12, cb);
#pragma unroll
                                for (int n = 0; n < NT; ++n) {
                                    mma_16816(part[m][n], a0, b0, a1, b1, h[n].x, h[n].y);
                                    mma_16816(part[m][n], a2, b2, a3, b3, h[n].z, h[n].w);
                                }
                            }
                        }
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            const float sa = bf16_value(s[2 * m][j]), sb = bf16_value(s[2 * m + 1][j]);
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                acc[m][n][0] = fmaf(part[m][n][0], sa, acc[m][n][0]);
                                acc[m][n][1] = fmaf(part[m][n][1], sa, acc[m][n][1]);
                                acc[m][n][2] = fmaf(part[m][n][2], sb, acc[m][n][2]);
                                acc[m][n][3] = fmaf(part[m][n][3], sb, acc[m][n][3]);
                            }
                        }
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(sh.empty + stage);
                if (++stage == L.stages) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
            // ---- the second block's warp hands its sums over; the first one's adds its own and stores them
            // (join[hidden row][vocabulary row of the unit], 33 words per row)
            if (half == 1) {
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            join[(n * 8 + 2 * t + (i & 1)) * 33 + m * 16 + (i >> 1) * 8 + r] = acc[m][n][i];
            }
            asm volatile("bar.sync %0, 64;" ::"r"(2 + slot) : "memory");
            if (half == 0) {
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float* at = join + (n * 8 + 2 * t + (i & 1)) * 33 + m * 16 + (i >> 1) * 8 + r;
                            *at += acc[m][n][i];
                        }
                __syncwarp();
                const int64_t v = static_cast<int64_t>(u0 + slot) * kUnit + lane;
                if (ok && mine && v < W.V) {
                    const int rows = min(8 * NT, P.rows);
                    for (int n = 0; n < rows; ++n) {
                        if (out_bf16)
                            reinterpret_cast<__nv_bfloat16*>(P.out)[n * P.ldo + v] = __float2bfloat16_rn(join[n * 33 + lane]);
                        else
                            reinterpret_cast<float*>(P.out)[n * P.ldo + v] = join[n * 33 + lane];
                    }
                }
            }
            asm volatile("bar.sync %0, 64;" ::"r"(2 + slot) : "memory");
        }
    }

    // copies still in flight after a wait that ran out get a bounded chance to land
    __syncthreads();
    if (*abort_flag && warp == kConsumers && lane == 0) {
        const int first = issued > L.stages ? issued - L.stages : 0;
        for (int k = first; k < issued; ++k) {
            volatile int never = 0;
            mbar_wait_bounded(sh.full + (k % L.stages), static_cast<uint32_t>((k / L.stages) & 1), &never, kWaitNs);
        }
    }
    __syncthreads();
}

bool g_attr[64][2][3][2];

template <int NT, int N, bool ZERO>
fef_status launch(const CUtensorMap& map, const ProductParams& P, const Plan& L, fef_dtype dt, int dev, int grid,
                  cudaStream_t stream) {
    bool& done = g_attr[dev][NT - 1][N / 2][ZERO];
    if (!done) {
        if (cudaFuncSetAttribute(product_rows_kernel<NT, N, ZERO>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 static_cast<int>(kSmemLimit)) != cudaSuccess)
            return FEF_ERR_CUDA;
        done = true;
    }
    product_rows_kernel<NT, N, ZERO><<<grid, kThreads, L.smem, stream>>>(map, P, L, dt == FEF_BF16);
    return cudaGetLastError() == cudaSuccess ? FEF_OK : FEF_ERR_CUDA;
}

template <int NT, int N>
fef_status launch_z(const CUtensorMap& map, const ProductParams& P, const Plan& L, fef_dtype dt, int dev, int grid,
                    cudaStream_t stream) {
    return P.layer.zero ? launch<NT, N, true>(map, P, L, dt, dev, grid, stream)
                        : launch<NT, N, false>(map, P, L, dt, dev, grid, stream);
}

template <int NT>
fef_status launch_g(const CUtensorMap& map, const ProductParams& P, const Plan& L, fef_dtype dt, int dev, int grid,
                    cudaStream_t stream) {
    switch (P.layer.G) {
        case 32: return launch_z<NT, 4>(map, P, L, dt, dev, grid, stream);
        case 64: return launch_z<NT, 2>(map, P, L, dt, dev, grid, stream);
        default: return launch_z<NT, 1>(map, P, L, dt, dev, grid, stream);
    }
}

}  // namespace

bool rows_kernel_takes(const ProductParams& P, int sms) { return P.rows <= 16 && make_plan(P, sms).stages >= 2; }

fef_status launch_rows_kernel(const ProductParams& P, fef_dtype dt, int dev, int sms, cudaStream_t stream) {
    const Plan L = make_plan(P, sms);
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return FEF_ERR_CUDA;
    CUtensorMap map;
    const Layer& W = P.layer;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(W.blocks) * 64, static_cast<cuuint64_t>(W.V)};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(W.blocks) * 64};
    const cuuint32_t box[2] = {128, kUnit}, elem[2] = {1, 1};
    if (fn(&map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(W.packed), dims, strides, box, elem,
           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return FEF_ERR_CUDA;
    const int grid = L.units < sms ? L.units : sms;
    return P.rows > 8 ? launch_g<2>(map, P, L, dt, dev, grid, stream) : launch_g<1>(map, P, L, dt, dev, grid, stream);
}

}  // namespace quant
}  // namespace fef
