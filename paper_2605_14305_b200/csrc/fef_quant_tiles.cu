// fef_lmhead_logits_quantized for any number of hidden rows: the fifth-generation tensor cores (tcgen05.mma), accumulators in
// tensor memory.
//
// prepare_kernel brings the hidden rows into the operand's form once (workspace): scaled by a power of two, the eight columns
// of every packed word in the order 0 4, 1 5, 2 6, 3 7 in which masking delivers them (fef_quant.cuh), with the sums of every
// group.  product_tiles_kernel then takes tiles of 128 vocabulary rows x NT hidden rows, one CTA per SM:
//   warps 8..15   weights: packed nibbles from global memory (kAhead blocks in flight per warp) to bfloat16 numbers in the
//                 128-byte-swizzled layout in shared memory;
//   warp 16       one thread brings the hidden rows of the same 128 columns in by TMA;
//   warp 17       one thread issues the MMAs (128 x NT x 16), a fresh accumulator for every group of a row's weights;
//   warps 0..7    take each group's accumulator out of tensor memory, subtract z times the group's sum, scale it and add it
//                 to the logits in registers: the vocabulary rows are the lanes, so a group's scale is one number per thread.
// The weights are the left operand for that reason.  Every wait is bounded.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "fef_device_math.cuh"
#include "fef_quant.cuh"
#include "fef_tensor_core.cuh"

namespace fef {
namespace quant {
namespace {

constexpr int kTileV = 128;                   // vocabulary rows of a tile
constexpr int kStages = 3;
constexpr int kAccumulators = 4;
constexpr int kABytes = kTileV * kBlock * 2;  // 32 KiB: two halves of 64 columns
constexpr int kAhead = 4;
constexpr int kEpilogueWarps = 8, kWeightWarps = 8;
constexpr int kThreads = (kEpilogueWarps + kWeightWarps + 2) * 32;
constexpr unsigned long long kWaitNs = 1000000000ull;

struct TileParams {
    ProductParams P;
    int tiles, row_blocks, items, padded;   // padded: hidden rows rounded up to whole tiles
    const float* sums;                      // [blocks * 128 / G][padded]
    const int* shifts;                      // [padded]
    int out_bf16;
};

struct Shared {
    uint64_t full[kStages];
    uint64_t empty[kStages];
    uint64_t acc_full[kAccumulators];
    uint64_t acc_empty[kAccumulators];
    uint64_t drained;
    uint32_t tmem_base;
    int abort_flag;
};

// ------------------------------------------------------------------------------------- hidden rows ----
struct PrepareParams {
    const uint16_t* hidden;   // [rows][d]
    uint16_t* operand;        // [padded][blocks * 128]
    float* sums;
    int* shifts;
    int rows, padded, d, blocks, words;   // words: 32-column pieces per group
    int32_t* status;
};
constexpr int kPrepareThreads = 256;

__global__ void __launch_bounds__(kPrepareThreads) prepare_kernel(const __grid_constant__ PrepareParams P) {
    __shared__ uint32_t s_top;
    cudaTriggerProgrammaticLaunchCompletion();   // (the tiles' kernel may begin to fetch weights; it waits for the rest)
    const int row = blockIdx.x, tid = threadIdx.x;
    if (P.status && row == 0 && tid == 0) *P.status = FEF_OK;
    if (tid == 0) s_top = 0u;
    __syncthreads();
    const uint16_t* src = P.hidden + static_cast<int64_t>(row) * P.d;
    const int pieces = P.blocks * 16;   // of eight columns; d is a multiple of 32
    auto load = [&](int p) {
        return row < P.rows && p * 8 < P.d ? __ldg(reinterpret_cast<const uint4*>(src) + p) : make_uint4(0u, 0u, 0u, 0u);
    };
    uint32_t top = 0u;
    for (int p = tid; p < pieces; p += kPrepareThreads) {
        const uint4 x = load(p);
        const uint32_t m = __vmaxu2(__vmaxu2(x.x & 0x7FFF7FFFu, x.y & 0x7FFF7FFFu), __vmaxu2(x.z & 0x7FFF7FFFu, x.w & 0x7FFF7FFFu));
        top = max(top, max(m & 0xFFFFu, m >> 16));
    }
    if (top != 0u) atomicMax(&s_top, top);
    __syncthreads();
    const int shift = row_shift(s_top);
    const float f0 = exp2_int(shift / 2), f1 = exp2_int(shift - shift / 2);
    if (tid == 0) P.shifts[row] = shift;
    for (int p = tid; p < pieces; p += kPrepareThreads) {   // (pieces is a multiple of 16: a group's lanes come together)
        const uint4 x = load(p);
        float v[8], total = 0.f;
        unpack<FEF_BF16>(x, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = v[j] * f0 * f1;
            total += v[j] * exp2_int(-67) * exp2_int(-66);
        }
        reinterpret_cast<uint4*>(P.operand + static_cast<int64_t>(row) * P.blocks * kBlock)[p] =
            make_uint4(bf16_pair(v[0], v[4]), bf16_pair(v[1] * 0.0625f, v[5] * 0.0625f), bf16_pair(v[2], v[6]),
                       bf16_pair(v[3] * 0.0625f, v[7] * 0.0625f));
        const unsigned lanes = __activemask();
        for (int o = 1; o < P.words * 4; o <<= 1) total += __shfl_xor_sync(lanes, total, o);
        if (p % (P.words * 4) == 0) P.sums[static_cast<int64_t>(p / (P.words * 4)) * P.padded + row] = total;
    }
}

// ------------------------------------------------------------------------------------------- tiles ----
// 16 consecutive columns of this thread's accumulator row; the caller waits for them.
__device__ __forceinline__ void tmem_load16(uint32_t addr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_wait_load() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
    return static_cast<uint64_t>(__float_as_uint(hi)) << 32 | __float_as_uint(lo);
}
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}

template <int NT, int N>   // hidden rows of a tile, groups per block
__global__ void __launch_bounds__(kThreads, 1)
product_tiles_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ TileParams T) {
    constexpr int kBBytes = NT * kBlock * 2, kStageBytes = kABytes + kBBytes;
    constexpr int kTmemCols = NT * kAccumulators;
    constexpr uint32_t kInstr = (1u << 4) | (1u << 7) | (1u << 10) | ((NT >> 3) << 17) | ((kTileV >> 4) << 24);
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    Shared& sh = *reinterpret_cast<Shared*>(smem + kStages * kStageBytes);
    volatile int* abort_flag = &sh.abort_flag;
    const ProductParams& P = T.P;
    const Layer& W = P.layer;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(sh.full + s, 1 + kWeightWarps);
            mbar_init(sh.empty + s, 1);
        }
        for (int a = 0; a < kAccumulators; ++a) {
            mbar_init(sh.acc_full + a, 1);
            mbar_init(sh.acc_empty + a, kEpilogueWarps);
        }
        mbar_init(&sh.drained, 1);
        sh.abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == 0) tmem_alloc(&sh.tmem_base, kTmemCols);  // (one CTA per SM: the columns are always free)
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *reinterpret_cast<volatile uint32_t*>(&sh.tmem_base);
    int issued = 0;
    auto gave_up = [&]() {
        *abort_flag = 1;
        if (lane == 0) report(P.status, FEF_ERR_TIMEOUT);
    };

    if (warp == kEpilogueWarps + kWeightWarps) {
        // ------------------------------------------------------------ hidden rows, one thread
        if (lane == 0) {
            cudaGridDependencySynchronize();
            int stage = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int item = blockIdx.x; ok && item < T.items; item += gridDim.x) {
                const int row0 = item % T.row_blocks * NT;
                for (int c = 0; c < W.blocks; ++c) {
                    if (!mbar_wait_bounded(sh.empty + stage, phase ^ 1u, abort_flag, kWaitNs)) {
                        gave_up();
                        ok = false;
                        break;
                    }
                    unsigned char* dst = smem + stage * kStageBytes + kABytes;
                    mbar_arrive_expect_tx(sh.full + stage, kBBytes);
                    tma_load_2d(dst, &map, c * kBlock, row0, sh.full + stage);
                    tma_load_2d(dst + kBBytes / 2, &map, c * kBlock + 64, row0, sh.full + stage);
                    ++issued;
                    if (++stage == kStages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
            }
        }
    } else if (warp == kEpilogueWarps + kWeightWarps + 1) {
        // -------------------------------------------------------------------------- MMAs, one thread
        if (lane == 0) {
            int stage = 0, acc = 0;
            uint32_t phase = 0, acc_phase = 0;
            bool ok = true;
            for (int item = blockIdx.x; ok && item < T.items; item += gridDim.x)
                for (int c = 0; ok && c < W.blocks; ++c) {
                    if (!mbar_wait_bounded(sh.full + stage, phase, abort_flag, kWaitNs)) {
                        gave_up();
                        ok = false;
                        break;
                    }
                    const uint32_t a_at = smem_u32(smem + stage * kStageBytes), b_at = a_at + kABytes;
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        if (!mbar_wait_bounded(sh.acc_empty + acc, acc_phase ^ 1u, abort_flag, kWaitNs)) {
                            gave_up();
                            ok = false;
                            break;
                        }
                        tc_fence_after();
#pragma unroll
                        for (int k = 0; k < 8 / N; ++k) {
                            const int step = j * (8 / N) + k, half = step / 4, inside = step % 4;
                            tc_mma(tmem_base + acc * NT,
                                   smem_desc_sw128(a_at + half * (kABytes / 2)) + static_cast<uint64_t>(2 * inside),
                                   smem_desc_sw128(b_at + half * (kBBytes / 2)) + static_cast<uint64_t>(2 * inside), kInstr,
                                   k != 0 ? 1u : 0u);
                        }
                        tc_commit(sh.acc_full + acc);
                        if (++acc == kAccumulators) {
                            acc = 0;
                            acc_phase ^= 1u;
                        }
                    }
                    if (ok) tc_commit(sh.empty + stage);   // arrives when these MMAs have read the stage
                    if (++stage == kStages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
            // everything issued has finished before the tensor memory goes back
            tc_commit(&sh.drained);
            mbar_wait_bounded(&sh.drained, 0u, abort_flag, kWaitNs);
        }
    } else if (warp >= kEpilogueWarps) {
        // ------------------------------------------------------------------------------------ weights
        // Warp w takes rows 16 w .. 16 w + 15 of the tile.  A lane's 16 bytes (one t) of a row are four chunks of eight columns of
        // the operand; rows r and r + 4 side by side in a quarter-warp lie in different halves of the swizzled 128 bytes.
        const int w = warp - kEpilogueWarps, g = lane >> 2, t = lane & 3;
        const int r = (g >> 1) + 4 * (g & 1);
        const int64_t pitch = static_cast<int64_t>(W.blocks) * 64;
        const int mine = blockIdx.x < T.items ? (T.items - 1 - blockIdx.x) / gridDim.x + 1 : 0;   // items of this CTA
        const int64_t count = static_cast<int64_t>(mine) * W.blocks;
        int64_t fetch_at = 0;
        int fetch_item = blockIdx.x, fetch_block = 0;
        const uint8_t* from[2];
        auto seek = [&]() {   // (rows behind V are read as the last one; their logits are not stored)
            const int64_t v = static_cast<int64_t>(fetch_item / T.row_blocks) * kTileV + w * 16 + r;
#pragma unroll
            for (int i = 0; i < 2; ++i) from[i] = W.packed + min(v + 8 * i, static_cast<int64_t>(W.V - 1)) * pitch + t * 16;
        };
        uint4 ahead[kAhead][2];
        auto fetch = [&](uint4 (&q)[2]) {   // past the end the last block is fetched again: no branch around the loads
#pragma unroll
            for (int i = 0; i < 2; ++i) q[i] = ld_global_nc_v4(from[i] + fetch_block * 64);
            const int more = fetch_at + 1 < count ? 1 : 0;
            fetch_at += more;
            fetch_block += more;
            if (fetch_block == W.blocks) {
                fetch_block = 0;
                fetch_item += gridDim.x;
                seek();
            }
        };
        if (count > 0) {
            seek();
#pragma unroll
            for (int i = 0; i < kAhead; ++i) fetch(ahead[i]);
            int stage = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int64_t at = 0; ok && at < count; at += kAhead) {
#pragma unroll
                for (int n = 0; n < kAhead; ++n) {
                    if (!ok || at + n >= count) break;
                    if (!__all_sync(0xFFFFFFFFu, mbar_wait_bounded(sh.empty + stage, phase ^ 1u, abort_flag, kWaitNs))) {
                        gave_up();
                        ok = false;
                        break;
                    }
                    unsigned char* dst = smem + stage * kStageBytes + (w * 16 + r) * 128;
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint4& q = ahead[n][i];
                            const uint32_t x = j == 0 ? q.x : j == 1 ? q.y : j == 2 ? q.z : q.w;
                            // chunk 4 j + t of the block's sixteen: half j / 2, column 4 (j % 2) + t of its eight
                            *reinterpret_cast<uint4*>(dst + (j / 2) * (kABytes / 2) + i * 1024 + (((j & 1) * 4 + t) ^ r) * 16) =
                                make_uint4(x & kLowNibbles, x & kHighNibbles, x >> 8 & kLowNibbles, x >> 8 & kHighNibbles);
                        }
                    fetch(ahead[n]);
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(sh.full + stage);
                    if (++stage == kStages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
            }
        }
    } else {
        // ----------------------------------------------------------------------------------- epilogue
        cudaGridDependencySynchronize();
        constexpr int kCols = NT / 2;                 // hidden rows of this warp
        const int quarter = warp & 3, col0 = (warp >> 2) * kCols;
        const uint32_t tmem = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) + col0;
        int acc = 0;
        uint32_t acc_phase = 0;
        bool ok = true;
        for (int item = blockIdx.x; ok && item < T.items; item += gridDim.x) {
            const int row0 = item % T.row_blocks * NT + col0;
            const int64_t v = static_cast<int64_t>(item / T.row_blocks) * kTileV + quarter * 32 + lane;
            const int64_t vs = min(v, static_cast<int64_t>(W.Vp - 1));
            uint64_t total[kCols / 2];
#pragma unroll
            for (int i = 0; i < kCols / 2; ++i) total[i] = 0ull;
            for (int c = 0; ok && c < W.blocks; ++c) {
#pragma unroll 1
                for (int j = 0; j < N; ++j) {
                    const int64_t at = (static_cast<int64_t>(c) * W.Vp + vs) * N + j;
                    const float s = bf16_value(__ldg(W.scale + at));
                    const float z = W.zero ? static_cast<float>(__ldg(W.zero + at)) : 8.f;
                    const uint64_t s2 = pair(s, s), z2 = pair(-z, -z);
                    const ulonglong2* x = reinterpret_cast<const ulonglong2*>(T.sums + static_cast<int64_t>(c * N + j) * T.padded + row0);
                    if (!__all_sync(0xFFFFFFFFu, mbar_wait_bounded(sh.acc_full + acc, acc_phase, abort_flag, kWaitNs))) {
                        gave_up();
                        ok = false;
                        break;
                    }
                    tc_fence_after();
#pragma unroll
                    for (int h = 0; h < kCols / 16; ++h) {
                        uint32_t d[16];
                        tmem_load16(tmem + acc * NT + h * 16, d);
                        ulonglong2 xs[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) xs[i] = x[h * 4 + i];
                        tmem_wait_load();
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const uint64_t sum = static_cast<uint64_t>(d[2 * i + 1]) << 32 | d[2 * i];
                            total[h * 8 + i] = fma_pair(fma_pair(z2, i & 1 ? xs[i / 2].y : xs[i / 2].x, sum), s2, total[h * 8 + i]);
                        }
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(sh.acc_empty + acc);
                    if (++acc == kAccumulators) {
                        acc = 0;
                        acc_phase ^= 1u;
                    }
                }
            }
            if (ok && v < W.V) {
#pragma unroll
                for (int i = 0; i < kCols; ++i) {
                    const int row = row0 + i;
                    if (row < P.rows) {
                        const int back = 133 - T.shifts[row];
                        const float y = __uint_as_float(static_cast<uint32_t>(i & 1 ? total[i / 2] >> 32 : total[i / 2])) *
                                        exp2_int(back / 2) * exp2_int(back - back / 2);
                        if (T.out_bf16)
                            reinterpret_cast<__nv_bfloat16*>(P.out)[row * P.ldo + v] = __float2bfloat16_rn(y);
                        else
                            reinterpret_cast<float*>(P.out)[row * P.ldo + v] = y;
                    }
                }
            }
        }
    }

    // ---- teardown: copies still in flight after a wait that ran out get a bounded chance to land; then the tensor memory
    //      goes back
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (*abort_flag && warp == kEpilogueWarps + kWeightWarps && lane == 0) {
        const int first = issued > kStages ? issued - kStages : 0;
        for (int k = first; k < issued; ++k) {
            volatile int never = 0;
            mbar_wait_bounded(sh.full + (k % kStages), static_cast<uint32_t>((k / kStages) & 1), &never, kWaitNs);
        }
    }
    __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        tmem_dealloc(tmem_base, kTmemCols);
    }
}

int tile_rows(int rows) { return rows <= 32 ? 32 : rows <= 64 ? 64 : 128; }
int64_t padded_rows(int rows) {
    const int nt = tile_rows(rows);
    return (static_cast<int64_t>(rows) + nt - 1) / nt * nt;
}
size_t round256(size_t n) { return (n + 255) / 256 * 256; }

struct Workspace {
    size_t operand, sums, shifts, total;
};
Workspace workspace_layout(const ProductParams& P) {
    Workspace L;
    const size_t rows = static_cast<size_t>(padded_rows(P.rows)), blocks = P.layer.blocks;
    L.operand = 0;
    L.sums = round256(rows * blocks * kBlock * 2);
    L.shifts = L.sums + round256(rows * blocks * (kBlock / P.layer.G) * 4);
    L.total = L.shifts + round256(rows * 4);
    return L;
}

bool g_attr[64][3][3];

template <int NT, int N>
fef_status launch(const CUtensorMap& map, const TileParams& T, int dev, int grid, cudaStream_t stream) {
    constexpr size_t smem = static_cast<size_t>(kStages) * (kABytes + NT * kBlock * 2) + sizeof(Shared) + 1024;
    bool& done = g_attr[dev][NT == 32 ? 0 : NT / 64][N / 2];
    if (!done) {
        if (cudaFuncSetAttribute(product_tiles_kernel<NT, N>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 static_cast<int>(smem)) != cudaSuccess)
            return FEF_ERR_CUDA;
        done = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, product_tiles_kernel<NT, N>, map, T) == cudaSuccess ? FEF_OK : FEF_ERR_CUDA;
}

template <int NT>
fef_status launch_g(const CUtensorMap& map, const TileParams& T, int dev, int grid, cudaStream_t stream) {
    switch (T.P.layer.G) {
        case 32: return launch<NT, 4>(map, T, dev, grid, stream);
        case 64: return launch<NT, 2>(map, T, dev, grid, stream);
        default: return launch<NT, 1>(map, T, dev, grid, stream);
    }
}

}  // namespace

size_t tiles_kernel_workspace(const ProductParams& P) { return workspace_layout(P).total; }

fef_status launch_tiles_kernel(const ProductParams& P, fef_dtype dt, void* workspace, int dev, int sms, cudaStream_t stream) {
    const Layer& W = P.layer;
    const Workspace L = workspace_layout(P);
    char* ws = static_cast<char*>(workspace);
    const int nt = tile_rows(P.rows);
    PrepareParams H;
    H.hidden = P.hidden;
    H.operand = reinterpret_cast<uint16_t*>(ws + L.operand);
    H.sums = reinterpret_cast<float*>(ws + L.sums);
    H.shifts = reinterpret_cast<int*>(ws + L.shifts);
    H.rows = P.rows;
    H.padded = static_cast<int>(padded_rows(P.rows));
    H.d = W.d;
    H.blocks = W.blocks;
    H.words = W.G / 32;
    H.status = P.status;
    TileParams T;
    T.P = P;
    T.tiles = (W.V + kTileV - 1) / kTileV;
    T.row_blocks = H.padded / nt;
    if (static_cast<int64_t>(T.tiles) * T.row_blocks > 0x7FFFFFFF) return FEF_ERR_INVALID_ARG;
    T.items = T.tiles * T.row_blocks;
    T.padded = H.padded;
    T.sums = H.sums;
    T.shifts = H.shifts;
    T.out_bf16 = dt == FEF_BF16;
    CUtensorMap map;
    const uint64_t cols = static_cast<uint64_t>(W.blocks) * kBlock;
    if (!map_2d(&map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, H.operand, cols, H.padded, cols * 2, 64, nt, CU_TENSOR_MAP_SWIZZLE_128B))
        return FEF_ERR_CUDA;
    prepare_kernel<<<H.padded, kPrepareThreads, 0, stream>>>(H);
    if (cudaGetLastError() != cudaSuccess) return FEF_ERR_CUDA;

    const int grid = T.items < sms ? T.items : sms;
    switch (nt) {
        case 32: return launch_g<32>(map, T, dev, grid, stream);
        case 64: return launch_g<64>(map, T, dev, grid, stream);
        default: return launch_g<128>(map, T, dev, grid, stream);
    }
}

}  // namespace quant
}  // namespace fef
