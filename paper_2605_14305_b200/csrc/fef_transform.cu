// fef_hidden_transform: hidden states through one layer of a prediction head, ahead of the output layer:
//   out[r, j] = act( sum_k hidden[r, k] weight[j, k] + bias[j] ) + residual[r, j],
// products of bfloat16 numbers summed in binary32, everything behind them in binary32, one rounding to the output's type.
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <cooperative_groups.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <type_traits>

#include "fef.h"
#include "fef_common.cuh"
#include "fef_device_math.cuh"
#include "fef_tensor_core.cuh"

namespace cg = cooperative_groups;

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
    int act;        // fef_activation
    int out_f32;    // the output is float32, not bfloat16
    int wide_out, wide_residual;   // eight neighbours lie on 16-byte boundaries in every row
    int row_tiles, tiles, blocks;   // tiles of rows, all tiles, 64-deep blocks
    int split, split_log2;          // CTAs (one cluster) that share a tile's depth
    int share_log2;                 // rows of a tile that one of them finishes
    unsigned long long wait_ns;
    int32_t* status;
#ifdef FEF_TEST_HOOKS
    int withhold;   // CTA 0 never delivers its stage of this number (-1: none)
#endif
};

template <int ACT>
__device__ __forceinline__ float activate(float y) {
    if constexpr (ACT == FEF_ACT_RELU) return y <= 0.f ? 0.f : y;   // (NaN stays)
    if constexpr (ACT == FEF_ACT_SILU) return __fdividef(y, 1.f + ex2_approx(-1.4426950408889634f * y));
    if constexpr (ACT == FEF_ACT_GELU) {
        // Phi from Abramowitz and Stegun 7.1.26: erfc x = (a1 t + .. + a5 t^5) e^(-x^2), t = 1 / (1 + p x), within 1.5e-7 for x >= 0
        const float x = 0.70710678118654752f * fabsf(y);
        const float t = __fdividef(1.f, fmaf(0.3275911f, x, 1.f));
        const float poly = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
        const float tail = 0.5f * poly * ex2_approx(-1.4426950408889634f * x * x);
        return y * (y > 0.f ? 1.f - tail : tail);
    }
    if constexpr (ACT == FEF_ACT_GELU_TANH) {
        // (1 + tanh z) / 2 = 1 / (1 + e^(-2 z)),  z = sqrt(2 / pi) (y + 0.044715 y^3)
        const float z2 = y * fmaf(0.044715f * y, y, 1.f) * (2.f * 0.79788456080286536f * 1.4426950408889634f);
        return __fdividef(y, 1.f + ex2_approx(-z2));
    }
    return y;
}

// ---- kernels ----
// transform_kernel: a CTA takes 128 columns of the output (rows of the weight: the left operand, M = 128) by BN rows (hidden
// states: the right operand, N = BN), so that few hidden rows cost few columns of tensor memory and no padding of the weight
// stream.  Warp 0 brings 64-deep blocks of both operands through a ring by TMA (one thread), warp 1 issues the MMAs (one thread),
// warps 2-9 are the epilogue.  Accumulators are double-buffered.  With fewer tiles than SMs the CTAs of a thread-block cluster
// share a tile's depth: each finishes a share of the rows, whose sums the others write into its shared memory (writes there do not
// wait for an answer, reads would).
//
// transform_pair_kernel: two CTAs (a cluster) take 256 columns by 256 rows with tcgen05.mma.cta_group::2: each brings its own 128
// columns' weights and half of the hidden rows, which both tensor cores read.  Per SM a block is 32 KiB instead of the 48 KiB of
// a 128 x 256 tile of its own, whose copies and operand reads together are more than shared memory's 128 bytes a clock.
//
// Few rows are bound by the weights' stream and by starting and joining (1 row x 4096 x 4096: 7.8 us on the device for 5.2 us of bytes;
// 64 rows 9.3), many by the tensor cores (2048 x 4096 x 4096 with silu, bias and residual 52.5 us, 1.31 PFLOP/s; the bare product by the
// installed library 44.5).
constexpr int kBM = 128, kBK = 64;
constexpr int kWBytes = kBM * kBK * 2;
constexpr int kEpilogueWarps = 8;
constexpr int kThreads = 64 + 32 * kEpilogueWarps;
constexpr int kMaxSplit = 8;
constexpr int kChunk = 16;       // columns of tensor memory (rows of the output) that an epilogue warp takes at a time
constexpr int kTurnPitch = 36;   // (rows of 16 bytes that start in different banks)
constexpr unsigned long long kWaitNs = 1000000000ull;

template <int BN>
struct Shape {
    static constexpr int kHBytes = BN * kBK * 2;
    static constexpr int kStageBytes = kWBytes + kHBytes;
    static constexpr int kStages = BN == 256 ? 4 : BN == 128 ? 4 : BN == 64 ? 6 : 8;
    static constexpr int kTmemCols = 2 * BN;
    static constexpr size_t kRing = static_cast<size_t>(kStages) * kStageBytes;
    // Where the cluster's CTAs put what they add up to the rows that this one finishes: BN / split rows of 128 sums from each.  With 256
    // rows there is no room beside the ring, and a barrier more frees the ring for it.
    static constexpr size_t kSums = static_cast<size_t>(BN) * kBM * 4;
    static constexpr bool kSumsInRing = BN == 256;
    static constexpr size_t kBuffers = kRing + (kSumsInRing ? 0 : kSums);
    static_assert(!kSumsInRing || kRing >= kSums, "a tile's sums fit into the ring");
};
// binary32 accumulator, bfloat16 operands, both K-major
__device__ constexpr uint32_t instruction(int m, int n) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(m >> 4) << 24);
}

template <int STAGES>
struct Shared {
    uint64_t full[STAGES];
    uint64_t empty[STAGES];
    uint64_t tmem_full[2];
    uint64_t tmem_empty[2];
    uint64_t drained;
    uint32_t tmem_base;
    int abort_flag;
    alignas(16) float turn[kEpilogueWarps][kChunk * kTurnPitch];   // where a warp turns 16 x 32 sums round
};
template <int STAGES>
constexpr size_t smem_bytes(size_t ring) {
    return ring + sizeof(Shared<STAGES>) + 1024;
}

__device__ __forceinline__ void tmem_load16(uint32_t addr, float (&v)[16]) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}

__device__ __forceinline__ void tmem_store16(uint32_t addr, const float (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
        :: "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])), "r"(__float_as_uint(v[3])),
           "r"(__float_as_uint(v[4])), "r"(__float_as_uint(v[5])), "r"(__float_as_uint(v[6])), "r"(__float_as_uint(v[7])),
           "r"(__float_as_uint(v[8])), "r"(__float_as_uint(v[9])), "r"(__float_as_uint(v[10])), "r"(__float_as_uint(v[11])),
           "r"(__float_as_uint(v[12])), "r"(__float_as_uint(v[13])), "r"(__float_as_uint(v[14])), "r"(__float_as_uint(v[15])),
           "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_wait_stores() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// A whole warp's wait.  The producer and the MMA issuer run as whole warps, with one elected lane for the copies and MMAs
// themselves: descriptors, addresses and flags then are warp-uniform values.  With one lane in a branch of its own a block cost each of
// the two over 600 clocks, more than the MMAs of a 128 x 256 x 64 block.
__device__ __forceinline__ bool all_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag, unsigned long long limit_ns) {
    return __all_sync(0xFFFFFFFFu, mbar_wait_bounded(bar, parity, abort_flag, limit_ns));
}

// An epilogue warp's wait for a tile: one lane polls, and not all the time.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag, unsigned long long limit_ns) {
    int ok = 0;
    if ((threadIdx.x & 31) == 0) {
        for (int spin = 0; spin < 64 && !ok; ++spin) {
            ok = mbar_try_wait(bar, parity);
            if (!ok) __nanosleep(64);
        }
        if (!ok) ok = mbar_wait_bounded(bar, parity, abort_flag, limit_ns);
    }
    return __shfl_sync(0xFFFFFFFFu, ok, 0) != 0;
}

// f with the activation as a constant.
template <class F>
__device__ __forceinline__ void with_activation(int act, F f) {
    switch (act) {
        case FEF_ACT_RELU: f(std::integral_constant<int, FEF_ACT_RELU>()); break;
        case FEF_ACT_SILU: f(std::integral_constant<int, FEF_ACT_SILU>()); break;
        case FEF_ACT_GELU: f(std::integral_constant<int, FEF_ACT_GELU>()); break;
        case FEF_ACT_GELU_TANH: f(std::integral_constant<int, FEF_ACT_GELU_TANH>()); break;
        default: f(std::integral_constant<int, FEF_ACT_NONE>()); break;
    }
}

// Eight neighbours of one row of the output, columns j .. j + 7, as the eight bfloat16 numbers of a 16-byte vector.
__device__ __forceinline__ uint4 load_eight(const __nv_bfloat16* p, int j, int n, bool whole) {
    if (whole) return *reinterpret_cast<const uint4*>(p + j);
    uint32_t w[4];
    const unsigned short* h = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t a = j + 2 * i < n ? h[j + 2 * i] : 0u, b = j + 2 * i + 1 < n ? h[j + 2 * i + 1] : 0u;
        w[i] = a | b << 16;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// What a lane keeps for its eight columns.
struct Columns {
    int j;
    bool in, whole_out, whole_residual;
    uint4 bias;
    __device__ __forceinline__ void set(const Params& P, int first) {
        j = first;
        in = j < P.n;
        whole_out = P.wide_out && j + 8 <= P.n;
        whole_residual = P.wide_residual && j + 8 <= P.n;
        bias = P.bias ? load_eight(P.bias, j, P.n, false) : make_uint4(0u, 0u, 0u, 0u);
    }
    __device__ __forceinline__ uint4 residual(const Params& P, int64_t row) const {
        if (!P.residual || !in || row >= P.rows) return make_uint4(0u, 0u, 0u, 0u);
        return load_eight(P.residual + row * P.ld_residual, j, P.n, whole_residual);
    }
    template <int ACT>
    __device__ __forceinline__ void finish(const Params& P, const float (&sum)[8], const uint4& residual, int64_t row) const {
        if (!in || row >= P.rows) return;
        float b[8], r[8], y[8];
        unpack<FEF_BF16>(bias, b);
        unpack<FEF_BF16>(residual, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = activate<ACT>(sum[i] + b[i]) + r[i];
        if (P.out_f32) {
            float* out = static_cast<float*>(P.out) + row * P.ldo + j;
            if (whole_out) {
                *reinterpret_cast<float4*>(out) = make_float4(y[0], y[1], y[2], y[3]);
                *reinterpret_cast<float4*>(out + 4) = make_float4(y[4], y[5], y[6], y[7]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (j + i < P.n) out[i] = y[i];
            }
        } else {
            __nv_bfloat16* out = static_cast<__nv_bfloat16*>(P.out) + row * P.ldo + j;
            if (whole_out) {
                uint4 w;
                __nv_bfloat162 h[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(y[2 * i], y[2 * i + 1]);
                memcpy(&w, h, 16);
                *reinterpret_cast<uint4*>(out) = w;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (j + i < P.n) out[i] = __float2bfloat16_rn(y[i]);
            }
        }
    }
};

// The epilogue of one tile by one warp: its 32 columns of the output, every second chunk of 16 rows.  A lane reads sums as one column
// of 16 rows and finishes eight columns of every eighth row; residuals are fetched three chunks ahead, the first before the wait.
struct Residuals {
    uint4 ahead[3][2];
    __device__ __forceinline__ void fetch(const Params& P, const Columns& col, int r0, uint4 (&to)[2]) const {
        const int row = r0 + ((threadIdx.x & 31) >> 2);
        to[0] = col.residual(P, row);
        to[1] = col.residual(P, row + 8);
    }
    __device__ __forceinline__ void first(const Params& P, const Columns& col, int r0) {
#pragma unroll
        for (int q = 0; q < 3; ++q) fetch(P, col, r0 + q * 2 * kChunk, ahead[q]);
    }
};
// Sums of many products: the tensor cores truncate whenever they add to an accumulator, 2^-24 of it each time and always the same
// way (measured against 64 bits, products of random signs: 1.3 10^-7 of the result after 128 products, 10^-6 after 1024).  Where the
// output is binary32, an accumulator therefore takes 512 products at most; an epilogue warp adds up such parts in registers, rounding
// to nearest, and puts their sum where the last part was, to be finished like any other.  (A bfloat16 output is rounded to 2^-9 of
// itself: nothing to gain.)  Tiles of 256 rows would need more registers than there are; 2048 x 4096 x 4096 with a binary32
// output takes 83 us with pairs of 128 rows, 53 us with a bfloat16 output and pairs of 256.
constexpr int kLongBlocks = 8;
template <int BN>
struct Parts {
    static constexpr int kChunks = BN >= 2 * kChunk ? BN / (2 * kChunk) : 1;   // of a warp
    float v[kChunks][kChunk];
    // adds a part to the sums; the first one starts them, the last one takes them
    template <bool FIRST, bool LAST>
    __device__ __forceinline__ void add(uint32_t tmem, int half) {
#pragma unroll
        for (int q = 0; q < kChunks; ++q) {
            const int c = half * kChunk + q * 2 * kChunk;
            if (c >= BN) continue;
            float x[kChunk];
            tmem_load16(tmem + static_cast<uint32_t>(c), x);
#pragma unroll
            for (int i = 0; i < kChunk; ++i) {
                if (!FIRST) x[i] += v[q][i];
                if (!LAST) v[q][i] = x[i];
            }
            if (LAST) tmem_store16(tmem + static_cast<uint32_t>(c), x);
        }
    }
    __device__ __forceinline__ void take(int part, int parts, uint32_t tmem, int half) {
        if (part + 1 < parts) {
            if (part == 0) add<true, false>(tmem, half);
            else add<false, false>(tmem, half);
        } else if (part > 0) {
            add<false, true>(tmem, half);
            tmem_wait_stores();
        }
    }
};

template <int BN>
__device__ __forceinline__ void finish_tile(const Params& P, uint32_t tmem, const Columns& col, Residuals& res, int r0, int half,
                                            float* turn) {
    const int lane = threadIdx.x & 31;
#pragma unroll 1
    for (int c = half * kChunk; c < BN; c += 2 * kChunk) {
        if (r0 + c >= P.rows) break;   // (uniform over the warp)
        float v[kChunk];
        tmem_load16(tmem + static_cast<uint32_t>(c), v);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kChunk; ++i) turn[i * kTurnPitch + lane] = v[i];
        const uint4 now[2] = {res.ahead[0][0], res.ahead[0][1]};
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            res.ahead[q][0] = res.ahead[q + 1][0];
            res.ahead[q][1] = res.ahead[q + 1][1];
        }
        if (c + 6 * kChunk < BN) res.fetch(P, col, r0 + c + 6 * kChunk, res.ahead[2]);
        __syncwarp();
        with_activation(P.act, [&](auto act) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int in_chunk = 8 * k + (lane >> 2);
                const float4* from = reinterpret_cast<const float4*>(turn + in_chunk * kTurnPitch + (lane & 3) * 8);
                const float4 a = from[0], b = from[1];
                const float y[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
                col.finish<decltype(act)::value>(P, y, now[k], r0 + c + in_chunk);
            }
        });
    }
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory");
}

__device__ __forceinline__ void give_up(const Params& P, volatile int* abort_flag) {
    *abort_flag = 1;
    report(P.status, FEF_ERR_TIMEOUT);
}

template <int BN, bool SPLIT, bool LONG>
__global__ void __launch_bounds__(kThreads, 1)
transform_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_h,
                 const __grid_constant__ Params P) {
    using S = Shape<BN>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    Shared<S::kStages>& sh = *reinterpret_cast<Shared<S::kStages>*>(smem + S::kBuffers);
    volatile int* abort_flag = &sh.abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        prefetch_map(&map_w);
        prefetch_map(&map_h);
        for (int s = 0; s < S::kStages; ++s) {
            mbar_init(sh.full + s, 1);
            mbar_init(sh.empty + s, 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(sh.tmem_full + a, 1);
            mbar_init(sh.tmem_empty + a, kEpilogueWarps);
        }
        mbar_init(&sh.drained, 1);
        sh.abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == 1) tmem_alloc(&sh.tmem_base, S::kTmemCols);   // (one CTA per SM: the columns are always free)
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *reinterpret_cast<volatile uint32_t*>(&sh.tmem_base);

    cudaGridDependencySynchronize();
    // (cleared here and not by a launch of its own: the earliest report comes after a wait of a second)
    if (threadIdx.x == 0 && blockIdx.x == 0 && P.status) *P.status = FEF_OK;

    const int row_tiles = P.row_tiles, tiles = P.tiles;
    const int rank = SPLIT ? static_cast<int>(blockIdx.x) & (P.split - 1) : 0;   // (a power of two)
    const int first_tile = SPLIT ? static_cast<int>(blockIdx.x) >> P.split_log2 : static_cast<int>(blockIdx.x);
    const int stride = SPLIT ? tiles : static_cast<int>(gridDim.x);   // (SPLIT: one tile per cluster)
    const int kb_begin = SPLIT ? rank * P.blocks >> P.split_log2 : 0;
    const int kb_end = SPLIT ? (rank + 1) * P.blocks >> P.split_log2 : P.blocks;
    int issued = 0;   // stages put in flight (producer thread)
    const int parts_of_tile = LONG ? (kb_end - kb_begin + kLongBlocks - 1) / kLongBlocks : 1;
    int last_acc = 0;   // the accumulator that holds a tile's last part, then its sums (epilogue)

    if (warp == 0) {
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int tile = first_tile; ok && tile < tiles; tile += stride) {
            const int j0 = tile / row_tiles * kBM, r0 = tile % row_tiles * BN;
            for (int kb = kb_begin; kb < kb_end; ++kb) {
#ifdef FEF_TEST_HOOKS
                // Test build: nothing is copied from here on and nothing arrives, so the waits for it run out.
                if (blockIdx.x == 0 && P.withhold >= 0 && issued >= P.withhold) {
                    ok = false;
                    break;
                }
#endif
                if (!all_wait(sh.empty + stage, phase ^ 1u, abort_flag, P.wait_ns)) {
                    give_up(P, abort_flag);
                    ok = false;
                    break;
                }
                if (elect_one()) {
                    unsigned char* dst = smem + stage * S::kStageBytes;
                    mbar_arrive_expect_tx(sh.full + stage, S::kStageBytes);
                    tma_load_2d(dst, &map_w, kb * kBK, j0, sh.full + stage);
                    tma_load_2d(dst + kWBytes, &map_h, kb * kBK, r0, sh.full + stage);
                }
                __syncwarp();
                ++issued;
                if (++stage == S::kStages) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
        }
    } else if (warp == 1) {
        int stage = 0;
        uint32_t phase = 0;
        unsigned uses[2] = {0u, 0u}, count = 0;
        bool ok = true;
        const uint64_t desc = smem_desc_sw128(smem_u32(smem));
        for (int tile = first_tile; ok && tile < tiles; tile += stride)
            for (int part = 0; ok && part < parts_of_tile; ++part, ++count) {
                const int acc = count & 1;
                // the epilogue must have drained this accumulator (passes at once on its first use)
                if (!all_wait(sh.tmem_empty + acc, (uses[acc] & 1u) ^ 1u, abort_flag, P.wait_ns)) {
                    give_up(P, abort_flag);
                    ok = false;
                    break;
                }
                ++uses[acc];
                const uint32_t tmem_d = tmem_base + static_cast<uint32_t>(acc * BN);
                const int from = kb_begin + part * kLongBlocks, to = LONG ? min(from + kLongBlocks, kb_end) : kb_end;
                for (int kb = from; kb < to; ++kb) {
                    if (!all_wait(sh.full + stage, phase, abort_flag, P.wait_ns)) {
                        give_up(P, abort_flag);
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    if (elect_one()) {
                        const uint64_t desc_w = desc + static_cast<uint64_t>(stage * (S::kStageBytes >> 4));   // (16-byte units)
                        const uint64_t desc_h = desc_w + static_cast<uint64_t>(kWBytes >> 4);
#pragma unroll
                        for (int k = 0; k < kBK / 16; ++k)   // 32 bytes further along K inside the swizzle row
                            tc_mma(tmem_d, desc_w + static_cast<uint64_t>(2 * k), desc_h + static_cast<uint64_t>(2 * k),
                                   instruction(kBM, BN), (kb > from || k) ? 1u : 0u);
                        tc_commit(sh.empty + stage);   // arrives when these MMAs have read the stage
                        if (kb == to - 1) tc_commit(sh.tmem_full + acc);   // arrives when the accumulator is complete
                    }
                    __syncwarp();
                    if (++stage == S::kStages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
            }
        // everything issued has finished before the tensor memory goes back, after a wait that ran out too: this one does
        // not look at the abort flag
        if (elect_one()) tc_commit(&sh.drained);
        __syncwarp();
        volatile int never = 0;
        mbar_wait_bounded(&sh.drained, 0u, &never, kWaitNs);
    } else {
        const int quarter = warp & 3, half = (warp - 2) >> 2;   // the tensor-memory lanes this warp may read; its chunks
        const uint32_t lane_addr = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16);
        unsigned uses[2] = {0u, 0u}, count = 0;
        bool ok = true;
        for (int tile = first_tile; ok && tile < tiles; tile += stride) {
            const int r0 = tile % row_tiles * BN;
            Columns col;
            Residuals res;
            if constexpr (!SPLIT) {
                col.set(P, tile / row_tiles * kBM + quarter * 32 + (lane & 3) * 8);
                res.first(P, col, r0 + half * kChunk);
            }
            Parts<LONG ? BN : 16> parts;
            for (int part = 0; part < parts_of_tile; ++part, ++count) {
                const int acc = count & 1;
                if (!warp_wait(sh.tmem_full + acc, uses[acc] & 1u, abort_flag, P.wait_ns)) {
                    give_up(P, abort_flag);
                    ok = false;
                    break;
                }
                ++uses[acc];
                tc_fence_after();
                last_acc = acc;
                const uint32_t at = lane_addr + static_cast<uint32_t>(acc * BN);
                if constexpr (LONG) parts.take(part, parts_of_tile, at, half);
                if (part + 1 == parts_of_tile) {
                    if constexpr (SPLIT) break;   // (one tile: it is finished below, by the whole cluster)
                    finish_tile<BN>(P, at, col, res, r0, half, sh.turn[warp - 2]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(sh.tmem_empty + acc);   // the accumulator may be overwritten
            }
        }
    }

    // ---- teardown: copies still in flight after an abort get a bounded chance to land; then the tensor memory goes back
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (*abort_flag && threadIdx.x == 0) {
        const int first = issued > S::kStages ? issued - S::kStages : 0;
        for (int k = first; k < issued; ++k) {
            volatile int never = 0;
            mbar_wait_bounded(sh.full + (k % S::kStages), static_cast<uint32_t>((k / S::kStages) & 1), &never, kWaitNs);
        }
    }
    __syncthreads();
    if constexpr (SPLIT) {
        cg::cluster_group cluster = cg::this_cluster();
        unsigned char* sums = smem + (S::kSumsInRing ? 0 : S::kRing);
        const int r0 = first_tile % row_tiles * BN, rows = min(BN, P.rows - r0);
        const int share = BN >> P.split_log2;   // rows that a CTA finishes (of the tile's BN)
        // (every CTA's MMAs are complete and have read its ring, so it is free)
        if (S::kSumsInRing) cluster.sync();
        if (warp >= 2) {
            const int quarter = warp & 3, half = (warp - 2) >> 2;
            tc_fence_after();
#pragma unroll 1
            for (int c = half * kChunk; c < rows; c += 2 * kChunk) {
                float v[kChunk];
                tmem_load16(tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) + static_cast<uint32_t>(last_acc * BN + c), v);
#pragma unroll
                for (int i = 0; i < kChunk; ++i) {
                    const int owner = (c + i) >> P.share_log2;
                    float* to = cluster.map_shared_rank(reinterpret_cast<float*>(sums), owner);
                    to[(rank * share + ((c + i) & (share - 1))) * kBM + quarter * 32 + lane] = v[i];
                }
            }
            tc_fence_before();
        }
        Columns col;
        col.set(P, first_tile / row_tiles * kBM + (lane & 15) * 8);
        // this CTA's rows, two to a warp at a time, eight columns per lane
        constexpr int kStep = kThreads / 16;
        const int own = min(share, rows - rank * share), q0 = warp * 2 + (lane >> 4);
        uint4 add = q0 < own ? col.residual(P, r0 + rank * share + q0) : make_uint4(0u, 0u, 0u, 0u);
        cluster.sync();
        for (int q = q0; q < own; q += kStep) {
            float y[8] = {};
            for (int s = 0; s < P.split; ++s) {
                const float4* from = reinterpret_cast<const float4*>(sums) + (s * share + q) * (kBM / 4) + (lane & 15) * 2;
                const float4 a = from[0], b = from[1];
                const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] += x[i];
            }
            const int64_t row = r0 + rank * share + q;
            const uint4 next = q + kStep < own ? col.residual(P, row + kStep) : make_uint4(0u, 0u, 0u, 0u);
            with_activation(P.act, [&](auto act) { col.finish<decltype(act)::value>(P, y, add, row); });
            add = next;
        }
    }
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem_base, S::kTmemCols);
    }
}

// ------------------------------------------------------------------------ pairs ----
namespace pair {

template <int TN>   // rows of a pair's tile
struct Shape {
    static constexpr int kHBytes = TN / 2 * kBK * 2;
    static constexpr int kStageBytes = kWBytes + kHBytes;   // this CTA's 128 columns' weights and half of the pair's hidden rows
    static constexpr int kStages = TN == 256 ? 6 : TN == 128 ? 8 : 9;
    static constexpr size_t kRing = static_cast<size_t>(kStages) * kStageBytes;
};
constexpr int kTileN = 256;                // columns of a pair's tile

// The address that a barrier of this CTA has in the pair's first CTA.
__device__ __forceinline__ uint32_t in_first(const uint64_t* bar) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(smem_u32(bar)));
    return r;
}
__device__ __forceinline__ void load_2d(void* dst, const CUtensorMap* map, int c0, int c1, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];" ::"r"(
            smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void alloc(uint32_t* slot, uint32_t cols) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void dealloc(uint32_t base, uint32_t cols) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(cols) : "memory");
}
__device__ __forceinline__ void mma(uint32_t tmem_d, uint64_t desc_a, uint64_t desc_b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t"
        "}\n" ::"r"(tmem_d),
        "l"(desc_a), "l"(desc_b), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Arrives at both CTAs' barriers when everything issued so far has finished.
__device__ __forceinline__ void commit_both(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
                     smem_u32(bar)),
                 "h"(static_cast<uint16_t>(3))
                 : "memory");
}
__device__ __forceinline__ void arrive_in(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool try_wait_cluster(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return ok != 0;
}
// As mbar_wait_bounded, for arrivals from the other CTA.
__device__ __forceinline__ bool wait_cluster(uint64_t* bar, uint32_t parity, volatile int* abort_flag, unsigned long long limit_ns) {
    if (try_wait_cluster(bar, parity)) return true;
    const unsigned long long start = globaltimer_ns();
    for (int round = 0; round < kSpinRounds; ++round) {
        for (int spin = 0; spin < 64; ++spin)
            if (try_wait_cluster(bar, parity)) return true;
        if (*abort_flag) return false;
        if (globaltimer_ns() - start > limit_ns) return false;
    }
    return false;
}

template <int TN, bool LONG>
__global__ void __launch_bounds__(kThreads, 1)
transform_pair_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_h,
                      const __grid_constant__ Params P) {
    using S = Shape<TN>;
    constexpr int kStages = S::kStages, kStageBytes = S::kStageBytes, kTmemCols = 2 * TN;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    Shared<kStages>& sh = *reinterpret_cast<Shared<kStages>*>(smem + S::kRing);
    volatile int* abort_flag = &sh.abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = static_cast<int>(cluster.block_rank());

    if (threadIdx.x == 0) {
        prefetch_map(&map_w);
        prefetch_map(&map_h);
        for (int s = 0; s < kStages; ++s) {
            mbar_init(sh.full + s, 1);
            mbar_init(sh.empty + s, 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(sh.tmem_full + a, 1);
            mbar_init(sh.tmem_empty + a, 2 * kEpilogueWarps);
        }
        mbar_init(&sh.drained, 1);
        sh.abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == 1) alloc(&sh.tmem_base, kTmemCols);   // (one CTA per SM: the columns are always free)
    tc_fence_before();
    __syncthreads();
    cluster.sync();   // both CTAs' barriers stand before either is signalled from the other side
    tc_fence_after();
    const uint32_t tmem_base = *reinterpret_cast<volatile uint32_t*>(&sh.tmem_base);

    cudaGridDependencySynchronize();
    if (threadIdx.x == 0 && blockIdx.x == 0 && P.status) *P.status = FEF_OK;   // (as above)

    const int row_tiles = P.row_tiles, tiles = P.tiles, blocks = P.blocks;
    const int first_tile = static_cast<int>(blockIdx.x) / 2, stride = static_cast<int>(gridDim.x) / 2;
    const int parts_of_tile = LONG ? (blocks + kLongBlocks - 1) / kLongBlocks : 1;
    int issued = 0;

    if (warp == 0) {
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int tile = first_tile; ok && tile < tiles; tile += stride) {
            const int j0 = tile / row_tiles * kTileN + rank * 128, r0 = tile % row_tiles * TN + rank * (TN / 2);
            for (int kb = 0; kb < blocks; ++kb) {
#ifdef FEF_TEST_HOOKS
                if (blockIdx.x == 0 && P.withhold >= 0 && issued >= P.withhold) {
                    ok = false;
                    break;
                }
#endif
                if (!all_wait(sh.empty + stage, phase ^ 1u, abort_flag, P.wait_ns)) {
                    give_up(P, abort_flag);
                    ok = false;
                    break;
                }
                if (elect_one()) {
                    unsigned char* dst = smem + stage * kStageBytes;
                    // the first CTA's barrier counts both CTAs' bytes (its phase cannot end before its own thread's arrival)
                    if (rank == 0) mbar_arrive_expect_tx(sh.full + stage, 2 * kStageBytes);
                    const uint32_t bar = in_first(sh.full + stage);
                    load_2d(dst, &map_w, kb * kBK, j0, bar);
                    load_2d(dst + kWBytes, &map_h, kb * kBK, r0, bar);
                }
                __syncwarp();
                ++issued;
                if (++stage == kStages) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
        }
    } else if (warp == 1) {
        if (rank == 0) {
            int stage = 0;
            uint32_t phase = 0;
            unsigned uses[2] = {0u, 0u}, count = 0;
            bool ok = true;
            const uint64_t desc = smem_desc_sw128(smem_u32(smem));
            for (int tile = first_tile; ok && tile < tiles; tile += stride)
                for (int part = 0; ok && part < parts_of_tile; ++part, ++count) {
                    const int acc = count & 1;
                    if (!__all_sync(0xFFFFFFFFu, wait_cluster(sh.tmem_empty + acc, (uses[acc] & 1u) ^ 1u, abort_flag, P.wait_ns))) {
                        give_up(P, abort_flag);
                        ok = false;
                        break;
                    }
                    ++uses[acc];
                    const uint32_t tmem_d = tmem_base + static_cast<uint32_t>(acc * TN);
                    const int from = part * kLongBlocks, to = LONG ? min(from + kLongBlocks, blocks) : blocks;
                    for (int kb = from; kb < to; ++kb) {
                        if (!__all_sync(0xFFFFFFFFu, wait_cluster(sh.full + stage, phase, abort_flag, P.wait_ns))) {
                            give_up(P, abort_flag);
                            ok = false;
                            break;
                        }
                        tc_fence_after();
                        if (elect_one()) {
                            const uint64_t desc_w = desc + static_cast<uint64_t>(stage * (kStageBytes >> 4));
                            const uint64_t desc_h = desc_w + static_cast<uint64_t>(kWBytes >> 4);
#pragma unroll
                            for (int k = 0; k < kBK / 16; ++k)
                                mma(tmem_d, desc_w + static_cast<uint64_t>(2 * k), desc_h + static_cast<uint64_t>(2 * k),
                                    instruction(256, TN), (kb > from || k) ? 1u : 0u);
                            commit_both(sh.empty + stage);
                            if (kb == to - 1) commit_both(sh.tmem_full + acc);
                        }
                        __syncwarp();
                        if (++stage == kStages) {
                            stage = 0;
                            phase ^= 1u;
                        }
                    }
                }
            if (elect_one()) commit_both(&sh.drained);
            __syncwarp();
            volatile int never = 0;
            mbar_wait_bounded(&sh.drained, 0u, &never, kWaitNs);
        }
    } else {
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        const uint32_t lane_addr = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16);
        unsigned uses[2] = {0u, 0u}, count = 0;
        bool ok = true;
        for (int tile = first_tile; ok && tile < tiles; tile += stride) {
            const int r0 = tile % row_tiles * TN;
            Columns col;
            Residuals res;
            col.set(P, tile / row_tiles * kTileN + rank * 128 + quarter * 32 + (lane & 3) * 8);
            res.first(P, col, r0 + half * kChunk);
            Parts<LONG ? TN : 16> parts;
            for (int part = 0; part < parts_of_tile; ++part, ++count) {
                const int acc = count & 1;
                if (!warp_wait(sh.tmem_full + acc, uses[acc] & 1u, abort_flag, P.wait_ns)) {
                    give_up(P, abort_flag);
                    ok = false;
                    break;
                }
                ++uses[acc];
                tc_fence_after();
                const uint32_t at = lane_addr + static_cast<uint32_t>(acc * TN);
                if constexpr (LONG) parts.take(part, parts_of_tile, at, half);
                if (part + 1 == parts_of_tile) finish_tile<TN>(P, at, col, res, r0, half, sh.turn[warp - 2]);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) arrive_in(in_first(sh.tmem_empty + acc));
            }
        }
    }

    // ---- teardown, as above; the first CTA's barriers answer for both CTAs' copies, and neither leaves before the other is done
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (*abort_flag && rank == 0 && threadIdx.x == 0) {
        const int first = issued > kStages ? issued - kStages : 0;
        for (int k = first; k < issued; ++k) {
            volatile int never = 0;
            mbar_wait_bounded(sh.full + (k % kStages), static_cast<uint32_t>((k / kStages) & 1), &never, kWaitNs);
        }
    }
    __syncthreads();
    cluster.sync();
    if (warp == 1) {
        tc_fence_after();
        dealloc(tmem_base, kTmemCols);
    }
    cluster.sync();
}

}  // namespace pair

// ---- host ----
static cudaError_t allow_smem(const void* kernel, size_t smem, bool (&allowed)[64], int dev) {
    if (dev < 64 && allowed[dev]) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e == cudaSuccess && dev < 64) allowed[dev] = true;
    return e;
}
static cudaError_t launch_clusters(void (*kernel)(CUtensorMap, CUtensorMap, Params), const CUtensorMap& w, const CUtensorMap& h,
                                   const Params& P, int grid, int cluster, size_t smem, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(grid));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // barriers and tensor memory are set up while the
    attr[0].val.programmaticStreamSerializationAllowed = 1;            // kernel before this one drains
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(cluster);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, w, h, P);
}
// Boxes of 64 columns by w_box rows of the weight and h_box rows of the hidden states.
static bool maps(const Params& P, int w_box, int h_box, CUtensorMap* w, CUtensorMap* h) {
    return map_2d(w, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, P.weight, P.d, P.n, static_cast<uint64_t>(P.d) * 2, kBK, w_box,
                  CU_TENSOR_MAP_SWIZZLE_128B) &&
           map_2d(h, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, P.hidden, P.d, P.rows, static_cast<uint64_t>(P.ld_hidden) * 2, kBK, h_box,
                  CU_TENSOR_MAP_SWIZZLE_128B);
}

template <int BN, bool SPLIT, bool LONG>
static cudaError_t launch(const CUtensorMap& w, const CUtensorMap& h, const Params& P, int grid, int dev, cudaStream_t stream) {
    constexpr size_t smem = smem_bytes<Shape<BN>::kStages>(Shape<BN>::kBuffers);
    static bool allowed[64];   // large shared memory, per device
    const cudaError_t e = allow_smem(reinterpret_cast<const void*>(transform_kernel<BN, SPLIT, LONG>), smem, allowed, dev);
    if (e != cudaSuccess) return e;
    return launch_clusters(transform_kernel<BN, SPLIT, LONG>, w, h, P, grid, SPLIT ? P.split : 1, smem, stream);
}
static int log2_of(int power) {
    int r = 0;
    while ((1 << r) < power) ++r;
    return r;
}
template <int BN>
static cudaError_t run(Params& P, int split, bool in_parts, int sms, int dev, cudaStream_t stream) {
    CUtensorMap w, h;
    if (!maps(P, kBM, BN, &w, &h)) return cudaErrorUnknown;
    P.row_tiles = (P.rows + BN - 1) / BN;
    P.tiles = P.row_tiles * ((P.n + kBM - 1) / kBM);   // (2^26 at most)
    P.split = split;
    P.split_log2 = log2_of(split);
    P.share_log2 = log2_of(BN / split);
    const int grid = split > 1 ? P.tiles * split : P.tiles < sms ? P.tiles : sms;
    if constexpr (BN <= 128)   // (twice as many registers would not do for the parts of 256 rows)
        if (in_parts)
            return split > 1 ? launch<BN, true, true>(w, h, P, grid, dev, stream) : launch<BN, false, true>(w, h, P, grid, dev, stream);
    return split > 1 ? launch<BN, true, false>(w, h, P, grid, dev, stream) : launch<BN, false, false>(w, h, P, grid, dev, stream);
}
template <int TN, bool LONG>
static cudaError_t launch_pairs(const CUtensorMap& w, const CUtensorMap& h, const Params& P, int grid, int dev, cudaStream_t stream) {
    constexpr size_t smem = smem_bytes<pair::Shape<TN>::kStages>(pair::Shape<TN>::kRing);
    static bool allowed[64];
    const cudaError_t e = allow_smem(reinterpret_cast<const void*>(pair::transform_pair_kernel<TN, LONG>), smem, allowed, dev);
    if (e != cudaSuccess) return e;
    return launch_clusters(pair::transform_pair_kernel<TN, LONG>, w, h, P, grid, 2, smem, stream);
}
template <int TN>
static cudaError_t run_pairs(Params& P, bool in_parts, int sms, int dev, cudaStream_t stream) {
    CUtensorMap w, h;
    if (!maps(P, 128, TN / 2, &w, &h)) return cudaErrorUnknown;
    P.row_tiles = (P.rows + TN - 1) / TN;
    P.tiles = P.row_tiles * ((P.n + pair::kTileN - 1) / pair::kTileN);
    const int grid = 2 * (P.tiles < sms / 2 ? P.tiles : sms / 2);
    if constexpr (TN <= 128)   // (as above)
        if (in_parts) return launch_pairs<TN, true>(w, h, P, grid, dev, stream);
    return launch_pairs<TN, false>(w, h, P, grid, dev, stream);
}

// Which tiles, and how many CTAs to a tile.  Every choice is right for every call; what each takes was measured over 23 sizes (1 to
// 2048 rows, 256 to 8192 columns, 512 to 8192 deep), in microseconds and within a tenth or two:
//   a 64-deep block   0.22 + 0.00065 BN (a CTA of its own)   0.175 + 0.0006 TN (a pair)
//   the last epilogue   0.4 + 0.01 BN       setup   3.5, a pair's 4.7
//   handing the sums of a shared tile over   0.3 + 0.029 BN, with two CTAs 0.7 of that
// e.g. 64 rows x 3584 x 3584: BN = 64 and four CTAs 9.0 (predicted 9.3), one CTA 18.4 (18.8); 512 x 4096 x 4096: pairs of 128 rows
// 21.4 (22.4), BN = 128 25.1 (24.6); 1024 x 1024 x 1024: BN = 64 8.7 (8.7), pairs of 256 rows 15.1 (11.7).
struct Choice {
    int tile, split;
    bool pair, in_parts;   // in_parts: sums of more than 512 products for a binary32 output (tiles of up to 128 rows only)
};
static Choice choose(int rows, int n, int d, bool out_f32, int sms) {
    const int64_t columns = (n + kBM - 1) / kBM, pair_columns = (n + 255) / 256;
    const int blocks = (d + kBK - 1) / kBK;
    Choice best = {128, 1, false, false};
    double least = 1e300;
    auto offer = [&](int tile, int split, bool pair, double us) {
        const bool in_parts = out_f32 && (blocks + split - 1) / split > kLongBlocks;
        if (us < least && !(in_parts && tile > 128)) {
            least = us;
            best = {tile, split, pair, in_parts};
        }
    };
    for (int bn = 16; bn <= 256; bn *= 2) {
        if (bn >= 32 && bn >= 2 * rows) break;   // (the tile before holds all rows)
        const int64_t tiles = columns * ((rows + bn - 1) / bn);
        const double block = 0.22 + 0.00065 * bn;
        offer(bn, 1, false, 3.5 + 0.4 + 0.01 * bn + static_cast<double>((tiles + sms - 1) / sms) * blocks * block);
        // a cluster's CTAs run at the same time, each on an SM of its own; clusters of eight do not fill all of a GPU's
        for (int split = 2; split <= kMaxSplit && split * 2 <= blocks && tiles * split <= (split == 8 ? sms * 3 / 4 : sms); split *= 2)
            offer(bn, split, false, 3.5 + (blocks + split - 1) / split * block + (0.3 + 0.029 * bn) * (split == 2 ? 0.7 : 1.0));
    }
    for (int tn = 64; tn <= 256; tn *= 2) {
        const int64_t tiles = pair_columns * ((rows + tn - 1) / tn), pairs = sms / 2;
        if (pairs)
            offer(tn, 1, true, 4.7 + 0.4 + 0.01 * tn + static_cast<double>((tiles + pairs - 1) / pairs) * blocks * (0.175 + 0.0006 * tn));
    }
    return best;
}

}  // namespace head
}  // namespace fef

#ifdef FEF_TEST_HOOKS
// Test builds only: CTA 0 of the next call withholds its stages from this number on, and waits give up after `limit_ns`.
static int g_test_withhold = -1;
static unsigned long long g_test_wait_ns = 0;
extern "C" void fef_test_withhold_transform_once(int stage, unsigned long long limit_ns) {
    g_test_withhold = stage;
    g_test_wait_ns = limit_ns;
}
#endif

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
    const int64_t most = 1ll << 38;   // (pitches in elements)
    if (ld_hidden > most || ldo > most || (residual && ld_residual > most)) return FEF_ERR_INVALID_ARG;
    if (activation < FEF_ACT_NONE || activation > FEF_ACT_GELU_TANH) return FEF_ERR_INVALID_ARG;
    const int esize = dt == FEF_F32 ? 4 : 2;
    if ((reinterpret_cast<uintptr_t>(hidden) & 15) || (reinterpret_cast<uintptr_t>(weight) & 15) || ld_hidden % 8 ||
        (reinterpret_cast<uintptr_t>(bias) & 1) || (reinterpret_cast<uintptr_t>(residual) & 1) ||
        (reinterpret_cast<uintptr_t>(out) & (esize - 1)) || (reinterpret_cast<uintptr_t>(device_status) & 3))
        return FEF_ERR_ALIGNMENT;
    // the output may be the residual itself, element for element, and overlaps nothing else
    struct Range {
        uintptr_t from, to, pitch, width;
        Range(const void* p, int64_t rows, int64_t ld, int64_t cols, int64_t size)
            : from(reinterpret_cast<uintptr_t>(p)), to(from + static_cast<uintptr_t>(((rows - 1) * ld + cols) * size)),
              pitch(static_cast<uintptr_t>(ld * size)), width(static_cast<uintptr_t>(cols * size)) {}
        bool meets(const Range& o) const {
            if (from >= o.to || o.from >= to) return false;
            if (pitch != o.pitch) return true;
            // different columns of one buffer: o's rows start `off` bytes behind this one's, and end before the next
            const uintptr_t off = (o.from >= from ? o.from - from : pitch - (from - o.from) % pitch) % pitch;
            return off < width || off + o.width > pitch;
        }
    };
    const Range o(out, rows, ldo, n, esize);
    if (o.meets(Range(hidden, rows, ld_hidden, d, 2)) || o.meets(Range(weight, n, d, d, 2)) || (bias && o.meets(Range(bias, 1, n, n, 2))))
        return FEF_ERR_INVALID_ARG;
    if (residual && o.meets(Range(residual, rows, ld_residual, n, 2)) &&
        !(residual == out && dt == FEF_BF16 && (ld_residual == ldo || rows == 1)))
        return FEF_ERR_INVALID_ARG;
    int dev = -1, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1)
        return FEF_ERR_CUDA;

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
    P.act = activation;
    P.out_f32 = dt == FEF_F32;
    P.blocks = (d + kBK - 1) / kBK;
    P.wide_out = !(reinterpret_cast<uintptr_t>(out) & 15) && ldo * esize % 16 == 0;
    P.wide_residual = !(reinterpret_cast<uintptr_t>(residual) & 15) && ld_residual % 8 == 0;
    P.wait_ns = kWaitNs;
    P.status = device_status;
#ifdef FEF_TEST_HOOKS
    P.withhold = g_test_withhold;
    if (g_test_withhold >= 0) P.wait_ns = g_test_wait_ns;   // one call only
    g_test_withhold = -1;
#endif
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const Choice c = choose(rows, n, d, dt == FEF_F32, sms);
    cudaError_t e;
    if (c.pair)
        e = c.tile == 64    ? run_pairs<64>(P, c.in_parts, sms, dev, stream)
            : c.tile == 128 ? run_pairs<128>(P, c.in_parts, sms, dev, stream)
                            : run_pairs<256>(P, c.in_parts, sms, dev, stream);
    else
        e = c.tile == 16    ? run<16>(P, c.split, c.in_parts, sms, dev, stream)
            : c.tile == 32  ? run<32>(P, c.split, c.in_parts, sms, dev, stream)
            : c.tile == 64  ? run<64>(P, c.split, c.in_parts, sms, dev, stream)
            : c.tile == 128 ? run<128>(P, c.split, c.in_parts, sms, dev, stream)
                            : run<256>(P, c.split, c.in_parts, sms, dev, stream);
    return e == cudaSuccess ? FEF_OK : FEF_ERR_CUDA;
}
