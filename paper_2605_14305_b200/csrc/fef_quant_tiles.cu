// fef_lmhead_logits_quantized for any number of hidden rows: the fifth-generation tensor cores (tcgen05.mma), accumulators in
// tensor memory.
//
// prepare_kernel brings the hidden rows into the operand's form once (workspace): the eight columns of every packed word in
// the order 0 4, 1 5, 2 6, 3 7 in which the nibbles come apart (fef_quant.cuh).  product_tiles_kernel then takes tiles of
// vocabulary rows x NT hidden rows, one CTA of 20 warps per SM: up to 64 hidden rows as two pipelines of 128 vocabulary rows that
// share the hidden rows and nothing else, beyond that as one pipeline with twice the warps.
//   8 warps  weights: packed nibbles from global memory (kAhead blocks in flight per warp) to the bfloat16 numbers q - z in tensor
//            memory, a vocabulary row per lane (through shared memory, writing and reading them took 512 of its cycles a block:
//            160 us at 64 rows x 126464 x 4096);
//   1 warp   brings the hidden rows of the same 128 columns in by TMA, and on a ring of their own the groups' scales (read from
//            global memory by the warps that need them, their latency set the pace);
//   1 warp a pipeline issues the MMAs (128 x NT x 16), a fresh accumulator for every group of a row's weights;
//   8 warps  take each group's accumulator out of tensor memory, scale it and add it to the logits in registers: the vocabulary
//            rows are the lanes, so a group's scale is one number per thread.  The weights are the left operand for that reason.
// A block's hand-overs from warp to warp and the instructions of the weights' and the epilogue's warps set the pace: hence few warps
// with much to do each, and waits that poll several barriers at once.  126464 x 4096 in groups of 128: 64 rows 119 us (102 when the
// logits stay in L2), 512 rows 700 us = 0.76 PFLOP/s.  A CTA takes whole tiles: 494 of 256 rows on 148 SMs are four rounds for
// 3.34, a sixth of the time at 64 rows.  Groups of 64 and 32 take 1.6 and 2.6 times as long (64 rows 164 and 270 us, 512 rows 980
// and 1700): the epilogue's waits, accumulators and arrivals are per group.  The epilogue has most to do, so the weights' warps
// subtract the zero points (taking them off the groups' sums took longer, and is inexact where a hidden value is large).
// Every wait is bounded.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stddef.h>

#include "fef_device_math.cuh"
#include "fef_quant.cuh"
#include "fef_tensor_core.cuh"

namespace fef {
namespace quant {
namespace {

constexpr int kPipeV = 128;                   // vocabulary rows of a pipeline
constexpr int kACols = kBlock / 2;            // 32-bit columns of a block of unpacked weights in tensor memory
constexpr int kMaxBStages = 6;                // ring of the hidden rows
constexpr int kSides = 4;                     // ring of the blocks' scales
constexpr int kRoleWarps = 4;                 // warps that share a pipeline's rows
constexpr int kThreads = (4 * kRoleWarps + 4) * 32;   // the last four warps: TMA, up to two issuers, idle
constexpr int kWeightWarp0 = 2 * kRoleWarps, kTmaWarp = 4 * kRoleWarps, kIssueWarp0 = kTmaWarp + 1;
constexpr int kLaunchRegs = 96;               // per thread
constexpr unsigned long long kWaitNs = 1000000000ull;

struct TileParams {
    ProductParams P;
    int tiles, row_blocks, items, padded;   // padded: hidden rows rounded up to whole tiles
    int out_bf16;
#ifdef FEF_TEST_HOOKS
    int withhold;   // CTA 0 never delivers its block of hidden rows of this number (-1: none)
#endif
};

// PIPES = 2: two pipelines, each with four warps for its weights and four for its epilogue.  PIPES = 1: one, whose weights two
// teams of four warps unpack block by block in turn, and whose hidden rows two teams of four take half each in the epilogue.
template <int NT, int PIPES>
struct Sizes {
    static constexpr int kTileV = PIPES * kPipeV, kTeams = 2 / PIPES, kCols = NT / kTeams;
    static_assert(kCols == 64, "");   // the registers' shares below are for 64 columns per thread of the epilogue
    static constexpr int kBBytes = NT * kBlock * 2, kBStages = NT == 128 ? 5 : 6;
    static_assert(kBStages <= kMaxBStages, "");
    // tensor memory of a pipeline: accumulators, then weights
    static constexpr int kAStages = PIPES == 2 ? 2 : 4;
    static constexpr int kPipeCols = 512 / PIPES, kAccumulators = 2;
    static_assert(kAccumulators * NT + kAStages * kACols <= kPipeCols, "");
    // Registers per thread that the three kinds of warpgroups keep of the launch's: the shares add up to its total exactly.
    // (Chosen so that nothing spills: with this much shared memory in use a spilled register comes back from L2.)
    static constexpr int kEpilogueRegs = 128, kWeightRegs = 80, kControlRegs = 64;
    static_assert(2 * kRoleWarps * (kEpilogueRegs + kWeightRegs) + 4 * kControlRegs == kThreads / 32 * kLaunchRegs, "");
    static constexpr int kAhead = 2;   // blocks of weights in flight per warp
};

struct Shared {
    uint64_t a_full[2][4];
    uint64_t a_empty[2][4];
    uint64_t acc_full[2][4];
    uint64_t acc_empty[2][4];
    uint64_t b_full[kMaxBStages];
    uint64_t b_empty[kMaxBStages];
    uint64_t side_full[kSides];
    uint64_t side_empty[kSides];
    uint64_t drained;
    uint32_t tmem_base;
    int abort_flag;
};

// ------------------------------------------------------------------------------------- hidden rows ----
struct PrepareParams {
    const uint16_t* hidden;   // [rows][d]
    uint16_t* operand;        // [padded][blocks * 128]
    int rows, d, blocks;
    int32_t* status;
};
constexpr int kPrepareThreads = 256;

__global__ void __launch_bounds__(kPrepareThreads) prepare_kernel(const __grid_constant__ PrepareParams P) {
    cudaTriggerProgrammaticLaunchCompletion();   // (the tiles' kernel may begin to fetch weights; it waits for the rest)
    const int row = blockIdx.x;
    if (P.status && row == 0 && threadIdx.x == 0) *P.status = FEF_OK;
    const uint4* src = reinterpret_cast<const uint4*>(P.hidden + static_cast<int64_t>(row) * P.d);
    uint4* to = reinterpret_cast<uint4*>(P.operand + static_cast<int64_t>(row) * P.blocks * kBlock);
    for (int p = threadIdx.x; p < P.blocks * 16; p += kPrepareThreads) {   // pieces of eight columns; d is a multiple of 32
        const uint4 x = row < P.rows && p * 8 < P.d ? __ldg(src + p) : make_uint4(0u, 0u, 0u, 0u);
        to[p] = make_uint4(__byte_perm(x.x, x.z, 0x5410), __byte_perm(x.x, x.z, 0x7632), __byte_perm(x.y, x.w, 0x5410),
                           __byte_perm(x.y, x.w, 0x7632));
    }
}

// ------------------------------------------------------------------------------------------- tiles ----
// A bounded wait that reads no clock as long as it is short (the hand-overs between warps set this kernel's pace).
__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    for (int poll = 0; poll < 32; ++poll)
        if (mbar_try_wait(bar, parity)) return true;
    return mbar_wait_bounded(bar, parity, abort_flag, kWaitNs);
}

// The warp's vote on what its lanes waited for.  A vote orders no memory accesses: the barrier behind it does, so that what one lane's
// wait has made visible to it (copies that landed, registers read out of tensor memory) is visible to all.
__device__ __forceinline__ bool all_waited(bool mine) {
    const bool all = __all_sync(0xFFFFFFFFu, mine);
    __syncwarp();
    return all;
}

// A warp waits for three barriers (given by their offset in Shared) at once, each polled by a lane of its own: one round trip.
__device__ __forceinline__ bool wait_for_all(Shared& sh, uint32_t o0, uint32_t p0, uint32_t o1, uint32_t p1, uint32_t o2, uint32_t p2) {
    const int lane = threadIdx.x & 31;
    const uint32_t offset = lane == 0 ? o0 : lane == 1 ? o1 : o2, parity = lane == 0 ? p0 : lane == 1 ? p1 : p2;
    uint64_t* bar = reinterpret_cast<uint64_t*>(reinterpret_cast<char*>(&sh) + offset);
    return all_waited(lane > 2 || wait_for(bar, parity, &sh.abort_flag));
}

// A place in a ring of S and the phase of its barriers.
template <int S>
struct Turn {
    int at = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void advance() {
        if (++at == S) {
            at = 0;
            phase ^= 1u;
        }
    }
};

// 16 consecutive columns of this thread's accumulator row; the caller waits for them.
__device__ __forceinline__ void tmem_load16(uint32_t addr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr));
}
// (the registers are tied to the wait, so that nothing that reads them moves before it)
__device__ __forceinline__ void tmem_wait_load(uint32_t (&r)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                   "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])::"memory");
}
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
    return static_cast<uint64_t>(__float_as_uint(hi)) << 32 | __float_as_uint(lo);
}
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}

// 1-D bulk copy global -> shared.
__device__ __forceinline__ void bulk_copy(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
                 "l"(src), "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}

// Of a block: the scales of all rows.
template <int N>
struct Side {
    uint16_t scale[2 * kPipeV * N];
};

// The lower word of smem_desc_sw128's descriptor (the upper one is the same for all), and the MMA that takes it and a left
// operand in tensor memory: D (+)= A * B^T.
__device__ __forceinline__ uint32_t desc_low(uint32_t smem_addr) { return (smem_addr >> 4 & 0x3FFFu) | 1u << 16; }
__device__ __forceinline__ void tc_mma_low(uint32_t tmem_d, uint32_t tmem_a, uint32_t b, uint32_t idesc, uint32_t accumulate) {
    constexpr uint32_t kHigh = 1024u >> 4 | 1u << 14 | 2u << 29;
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        ".reg .b64 db;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "mov.b64 db, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, {%6, %6, %6, %6}, p;\n\t"
        "}\n" ::"r"(tmem_d),
        "r"(tmem_a), "r"(b), "r"(idesc), "r"(accumulate), "r"(kHigh), "r"(0u)
        : "memory");
}
// 16 columns of this thread's row; the caller waits for the stores.
__device__ __forceinline__ void tmem_store16(uint32_t addr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(
            addr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// 32 bytes, 32-byte aligned.
__device__ __forceinline__ void load_sector(const void* p, uint32_t (&r)[8]) {
    asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "l"(p));
}

__device__ __forceinline__ void put_logit(float* at, float y) { *at = y; }
__device__ __forceinline__ void put_logit(__nv_bfloat16* at, float y) { *at = __float2bfloat16_rn(y); }

// One vocabulary row's logits of `kCols` hidden rows, the first `many` of which exist.
template <int kCols, typename Out>
__device__ __forceinline__ void store_column(Out* out, int64_t ldo, const uint64_t (&total)[kCols / 2], int many) {
#pragma unroll
    for (int i = 0; i < kCols; ++i) {
        if (i < many) put_logit(out, __uint_as_float(static_cast<uint32_t>(i & 1 ? total[i / 2] >> 32 : total[i / 2])));
        out += ldo;
    }
}

template <int NT, int PIPES, int N>   // hidden rows of a tile, pipelines, groups per block
__global__ void __launch_bounds__(kThreads, 1)
product_tiles_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ TileParams T) {
    using S = Sizes<NT, PIPES>;
    constexpr int kTileV = S::kTileV, kTeams = S::kTeams, kCols = S::kCols, kAStages = S::kAStages;
    constexpr int kAccumulators = S::kAccumulators, kAhead = S::kAhead;
    constexpr uint32_t kInstr = (1u << 4) | (1u << 7) | (1u << 10) | ((NT >> 3) << 17) | ((kPipeV >> 4) << 24);
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    Side<N>* side = reinterpret_cast<Side<N>*>(smem + S::kBStages * S::kBBytes);
    Shared& sh = *reinterpret_cast<Shared*>(side + kSides);
    volatile int* abort_flag = &sh.abort_flag;
    const ProductParams& P = T.P;
    const Layer& W = P.layer;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int p = 0; p < PIPES; ++p) {
            for (int s = 0; s < kAStages; ++s) {
                mbar_init(&sh.a_full[p][s], kRoleWarps);
                mbar_init(&sh.a_empty[p][s], 1);
            }
            for (int a = 0; a < kAccumulators; ++a) {
                mbar_init(&sh.acc_full[p][a], 1);
                mbar_init(&sh.acc_empty[p][a], kTeams * kRoleWarps);
            }
        }
        for (int s = 0; s < S::kBStages; ++s) {
            mbar_init(sh.b_full + s, 1);
            mbar_init(sh.b_empty + s, PIPES);
        }
        for (int q = 0; q < kSides; ++q) {
            mbar_init(sh.side_full + q, 1);
            mbar_init(sh.side_empty + q, 2 * kRoleWarps);
        }
        mbar_init(&sh.drained, PIPES);
        sh.abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == 0) tmem_alloc(&sh.tmem_base, 512);  // (one CTA per SM: the columns are always free)
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *reinterpret_cast<volatile uint32_t*>(&sh.tmem_base);
    int issued = 0, sides = 0;
    auto gave_up = [&]() {
        *abort_flag = 1;
        report(P.status, FEF_ERR_TIMEOUT);
    };
    const int items = blockIdx.x < T.items ? (T.items - 1 - blockIdx.x) / gridDim.x + 1 : 0;   // of this CTA
    const int count = items * W.blocks;

    if (warp >= kTmaWarp) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::kControlRegs));
    if (warp == kTmaWarp) {
        // ------------------------------------------------------------ hidden rows, one thread
        if (elect_one()) {
            cudaGridDependencySynchronize();
            Turn<S::kBStages> stage;
            Turn<kSides> slot;
            bool ok = true;
            for (int item = blockIdx.x; ok && item < T.items; item += gridDim.x) {
                const int row0 = item % T.row_blocks * NT;
                const int64_t v0 = static_cast<int64_t>(item / T.row_blocks) * kTileV;
                const uint32_t rows = static_cast<uint32_t>(min(static_cast<int64_t>(kTileV), W.Vp - v0));   // a multiple of 32
                for (int c = 0; c < W.blocks; ++c) {
#ifdef FEF_TEST_HOOKS
                    // Test build: nothing is copied from here on and nothing arrives, so the waits for it run out.
                    if (blockIdx.x == 0 && T.withhold >= 0 && issued >= T.withhold) {
                        ok = false;
                        break;
                    }
#endif
                    if (!wait_for(sh.b_empty + stage.at, stage.phase ^ 1u, abort_flag)) {
                        gave_up();
                        ok = false;
                        break;
                    }
                    unsigned char* dst = smem + stage.at * S::kBBytes;
                    mbar_arrive_expect_tx(sh.b_full + stage.at, S::kBBytes);
                    tma_load_2d(dst, &map, c * kBlock, row0, sh.b_full + stage.at);
                    tma_load_2d(dst + S::kBBytes / 2, &map, c * kBlock + 64, row0, sh.b_full + stage.at);
                    ++issued;
                    stage.advance();
                    if (!wait_for(sh.side_empty + slot.at, slot.phase ^ 1u, abort_flag)) {
                        gave_up();
                        ok = false;
                        break;
                    }
                    uint64_t* bar = sh.side_full + slot.at;
                    mbar_arrive_expect_tx(bar, rows * N * 2);
                    bulk_copy(side[slot.at].scale, W.scale + (static_cast<int64_t>(c) * W.Vp + v0) * N, rows * N * 2, bar);
                    ++sides;
                    slot.advance();
                }
            }
        }
    } else if (warp >= kIssueWarp0 + PIPES) {
        // (the control warpgroup's fourth warp)
    } else if (warp >= kIssueWarp0) {
        // -------------------------------------------------------------------------- MMAs
        // A whole warp runs the loop and the elected lane issues: in a branch of lane 0 alone, bringing the descriptors into
        // uniform registers took most of the time.
        const int pipe = warp - kIssueWarp0;
        const uint32_t b_base = desc_low(smem_u32(smem));
        const uint32_t tmem = tmem_base + pipe * S::kPipeCols;
        Turn<kAStages> a;
        Turn<S::kBStages> b;
        Turn<kAccumulators> acc;
        bool ok = true;
        for (int at = 0; ok && at < count; ++at) {
            const uint32_t a_at = tmem + kAccumulators * NT + a.at * kACols, b_at = b_base + b.at * (S::kBBytes / 16);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                if (!wait_for_all(sh, offsetof(Shared, a_full) + (pipe * 4 + a.at) * 8, a.phase, offsetof(Shared, b_full) + b.at * 8,
                                  b.phase, offsetof(Shared, acc_empty) + (pipe * 4 + acc.at) * 8, acc.phase ^ 1u)) {
                    gave_up();
                    ok = false;
                    break;
                }
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < 8 / N; ++k) {
                        const int step = j * (8 / N) + k, half = step / 4, inside = step % 4;
                        tc_mma_low(tmem + acc.at * NT, a_at + 8 * step,
                                   b_at + half * (S::kBBytes / 32) + 2 * inside, kInstr, k != 0 ? 1u : 0u);
                    }
                    tc_commit(&sh.acc_full[pipe][acc.at]);
                    if (j == N - 1) {   // (they arrive when these MMAs have read the stages)
                        tc_commit(&sh.a_empty[pipe][a.at]);
                        tc_commit(sh.b_empty + b.at);
                    }
                }
                __syncwarp();
                acc.advance();
            }
            a.advance();
            b.advance();
        }
        // everything issued has finished before the tensor memory goes back, after a wait that ran out too: this one does not
        // look at the abort flag (both issuers always commit, so it ends)
        if (elect_one()) tc_commit(&sh.drained);
        __syncwarp();
        volatile int never = 0;
        wait_for(&sh.drained, 0u, &never);
    } else if (warp >= kWeightWarp0) {
        // ------------------------------------------------------------------------------------ weights
        // A lane takes one row: the 64 bytes of a block are its word 4 t + w, of columns 32 w + 8 t .. + 7, for every t and w.
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::kWeightRegs));
        const int which = (warp - kWeightWarp0) / kRoleWarps, quarter = (warp - kWeightWarp0) % kRoleWarps;
        const int pipe = PIPES == 2 ? which : 0, team = PIPES == 2 ? 0 : which;
        const uint32_t tmem = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) + pipe * S::kPipeCols + kAccumulators * NT;
        const int blocks = (count - team + kTeams - 1) / kTeams;   // of this team
        int left = blocks, fetch_item = blockIdx.x, fetch_block = team;
        const uint8_t *fetch_w = nullptr, *fetch_z = nullptr;
        const bool zeros = W.zero != nullptr;
        auto seek = [&]() {   // (rows behind V are read as the last one; their logits are not stored)
            while (fetch_block >= W.blocks) {
                fetch_block -= W.blocks;
                fetch_item += gridDim.x;
            }
            const int64_t v = min(static_cast<int64_t>(fetch_item / T.row_blocks) * kTileV + pipe * kPipeV + quarter * 32 + lane,
                                  static_cast<int64_t>(W.V - 1));
            fetch_w = W.packed + v * (static_cast<int64_t>(W.blocks) * 64);
            fetch_z = W.zero + v * N;
        };
        struct Fetched {
            uint32_t q[2][8];   // words 4 t + w: t = 0, 1 and t = 2, 3
            uint32_t z;         // N zero points
        } ahead[kAhead];
        auto fetch = [&](Fetched& f) {   // past the end the last block is fetched again: no branch around the loads
#pragma unroll
            for (int i = 0; i < 2; ++i) load_sector(fetch_w + fetch_block * 64 + i * 32, f.q[i]);
            f.z = 0x08080808u;
            if (zeros) {
                const uint8_t* z = fetch_z + static_cast<int64_t>(fetch_block) * W.Vp * N;
                f.z = N == 1 ? __ldg(z) : N == 2 ? __ldg(reinterpret_cast<const uint16_t*>(z)) : __ldg(reinterpret_cast<const uint32_t*>(z));
            }
            const int more = left > 1 ? 1 : 0;
            left -= more;
            fetch_block += more * kTeams;
            if (fetch_block >= W.blocks) seek();
        };
        if (blocks > 0) {
            seek();
#pragma unroll
            for (int i = 0; i < kAhead; ++i) fetch(ahead[i]);
            Turn<kAStages> stage;
            stage.at = team;
            bool ok = true;
            // (after a wait that ran out the rest goes by without waits and arrivals)
            auto put = [&](const Fetched& f) {
                if (ok && !all_waited(lane > 0 || wait_for(&sh.a_empty[pipe][stage.at], stage.phase ^ 1u, abort_flag))) {
                    gave_up();
                    ok = false;
                }
                tc_fence_after();
#pragma unroll
                for (int w = 0; w < 4; ++w) {   // 32 columns of the operand
                    const uint32_t centre = centre_of(f.z >> (8 * (w * N / 4)) & 0xFFu);
                    uint32_t y[16];
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const uint32_t x = f.q[t >> 1][(t & 1) * 4 + w];
                        y[4 * t] = centred_pair(x, centre);
                        y[4 * t + 1] = centred_pair(x >> 4, centre);
                        y[4 * t + 2] = centred_pair(x >> 8, centre);
                        y[4 * t + 3] = centred_pair(x >> 12, centre);
                    }
                    tmem_store16(tmem + stage.at * kACols + w * 16, y);
                }
            };
            auto hand_over = [&]() {
                tmem_wait_store();
                tc_fence_before();
                __syncwarp();
                if (ok && lane == 0) mbar_arrive(&sh.a_full[pipe][stage.at]);
#pragma unroll
                for (int t = 0; t < kTeams; ++t) stage.advance();
            };
            int at = 0;
            for (; at + kAhead <= blocks; at += kAhead) {
#pragma unroll
                for (int n = 0; n < kAhead; ++n) {
                    put(ahead[n]);
                    fetch(ahead[n]);
                    hand_over();
                }
            }
#pragma unroll
            for (int n = 0; n < kAhead - 1; ++n)
                if (at + n < blocks) {
                    put(ahead[n]);
                    hand_over();
                }
        }
    } else {
        // ----------------------------------------------------------------------------------- epilogue
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::kEpilogueRegs));
        cudaGridDependencySynchronize();
        const int which = warp / kRoleWarps, quarter = warp % kRoleWarps;
        const int pipe = PIPES == 2 ? which : 0, col0 = PIPES == 2 ? 0 : which * kCols;
        const int row_in_tile = pipe * kPipeV + quarter * 32 + lane;
        const uint32_t tmem = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) + pipe * S::kPipeCols + col0;
        Turn<kAccumulators> acc;
        Turn<kSides> slot;
        bool ok = true;
        for (int item = blockIdx.x; ok && item < T.items; item += gridDim.x) {
            uint64_t total[kCols / 2];
#pragma unroll
            for (int i = 0; i < kCols / 2; ++i) total[i] = 0ull;
            for (int c = 0; ok && c < W.blocks; ++c) {
#pragma unroll 1
                for (int j = 0; j < N; ++j) {
                    const uint32_t full = offsetof(Shared, acc_full) + (pipe * 4 + acc.at) * 8;
                    if (!wait_for_all(sh, full, acc.phase, offsetof(Shared, side_full) + slot.at * 8, slot.phase, full, acc.phase)) {
                        gave_up();
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    // (the next part is under way while one is added up)
                    constexpr int kPart = 16, kParts = kCols / kPart;
                    uint32_t d[2][kPart];
                    tmem_load16(tmem + acc.at * NT, d[0]);
                    const float s = bf16_value(side[slot.at].scale[row_in_tile * N + j]);
                    const uint64_t s2 = pair(s, s);
#pragma unroll
                    for (int h = 0; h < kParts; ++h) {
                        uint32_t (&now)[kPart] = d[h & 1];
                        tmem_wait_load(now);
                        if (h + 1 < kParts) {
                            tmem_load16(tmem + acc.at * NT + (h + 1) * kPart, d[(h + 1) & 1]);
                        } else {   // all out: the accumulator may be written again
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(&sh.acc_empty[pipe][acc.at]);
                        }
#pragma unroll
                        for (int i = 0; i < kPart / 2; ++i) {
                            uint64_t& t = total[h * (kPart / 2) + i];
                            t = fma_pair(static_cast<uint64_t>(now[2 * i + 1]) << 32 | now[2 * i], s2, t);
                        }
                    }
                    // after the block's last group its scales too
                    __syncwarp();
                    if (lane == 1 && j == N - 1) mbar_arrive(sh.side_empty + slot.at);
                    acc.advance();
                }
                slot.advance();
            }
            const int row0 = item % T.row_blocks * NT + col0;
            const int64_t v = static_cast<int64_t>(item / T.row_blocks) * kTileV + row_in_tile;
            if (ok && v < W.V) {
                if (T.out_bf16)
                    store_column<kCols>(reinterpret_cast<__nv_bfloat16*>(P.out) + row0 * P.ldo + v, P.ldo, total, P.rows - row0);
                else
                    store_column<kCols>(reinterpret_cast<float*>(P.out) + row0 * P.ldo + v, P.ldo, total, P.rows - row0);
            }
        }
    }

    // ---- teardown: copies still in flight after a wait that ran out get a bounded chance to land; then the tensor memory
    //      goes back
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (*abort_flag && warp == kTmaWarp) {   // (the lanes that issued nothing have nothing to wait for)
        for (int k = issued > S::kBStages ? issued - S::kBStages : 0; k < issued; ++k) {
            volatile int never = 0;
            mbar_wait_bounded(sh.b_full + (k % S::kBStages), static_cast<uint32_t>((k / S::kBStages) & 1), &never, kWaitNs);
        }
        for (int k = sides > kSides ? sides - kSides : 0; k < sides; ++k) {
            volatile int never = 0;
            mbar_wait_bounded(sh.side_full + (k % kSides), static_cast<uint32_t>((k / kSides) & 1), &never, kWaitNs);
        }
    }
    __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        tmem_dealloc(tmem_base, 512);
    }
}

// Up to 64 rows two pipelines of 64, beyond them one of 128: with more rows the weights are unpacked half as often (126464 x 4096, 512
// rows: 650 against 705 us; 64 rows: 154 against 102).  Tiles of 32 rows take no less time than those of 64, which is the weights'.
int tile_rows(int rows) { return rows <= 64 ? 64 : 128; }
int64_t padded_rows(int rows) {
    const int nt = tile_rows(rows);
    return (static_cast<int64_t>(rows) + nt - 1) / nt * nt;
}
bool g_attr[64][2][3];
#ifdef FEF_TEST_HOOKS
int g_test_withhold = -1;
#endif

template <int NT, int PIPES, int N>
fef_status launch(const CUtensorMap& map, const TileParams& T, int dev, int grid, cudaStream_t stream) {
    constexpr size_t smem = Sizes<NT, PIPES>::kBStages * Sizes<NT, PIPES>::kBBytes + kSides * sizeof(Side<N>) + sizeof(Shared) + 1024;
    static_assert(smem <= 232448, "");
    bool& done = g_attr[dev][PIPES - 1][N / 2];
    if (!done) {
        // (a warpgroup that asks for more registers than the launch left waits for good: never launch with another number)
        cudaFuncAttributes attr;
        if (cudaFuncGetAttributes(&attr, product_tiles_kernel<NT, PIPES, N>) != cudaSuccess || (attr.numRegs + 7) / 8 * 8 != kLaunchRegs)
            return FEF_ERR_CUDA;
        if (cudaFuncSetAttribute(product_tiles_kernel<NT, PIPES, N>, cudaFuncAttributeMaxDynamicSharedMemorySize,
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
    return cudaLaunchKernelEx(&cfg, product_tiles_kernel<NT, PIPES, N>, map, T) == cudaSuccess ? FEF_OK : FEF_ERR_CUDA;
}

template <int NT, int PIPES>
fef_status launch_g(const CUtensorMap& map, const TileParams& T, int dev, int grid, cudaStream_t stream) {
    switch (T.P.layer.G) {
        case 32: return launch<NT, PIPES, 4>(map, T, dev, grid, stream);
        case 64: return launch<NT, PIPES, 2>(map, T, dev, grid, stream);
        default: return launch<NT, PIPES, 1>(map, T, dev, grid, stream);
    }
}

}  // namespace

size_t tiles_kernel_workspace(const ProductParams& P) {
    return (static_cast<size_t>(padded_rows(P.rows)) * P.layer.blocks * kBlock * 2 + 255) / 256 * 256;
}

fef_status launch_tiles_kernel(const ProductParams& P, fef_dtype dt, void* workspace, int dev, int sms, cudaStream_t stream) {
    const Layer& W = P.layer;
    const int nt = tile_rows(P.rows), tile_v = nt == 64 ? 2 * kPipeV : kPipeV;
    PrepareParams H;
    H.hidden = P.hidden;
    H.operand = static_cast<uint16_t*>(workspace);
    H.rows = P.rows;
    H.d = W.d;
    H.blocks = W.blocks;
    H.status = P.status;

    TileParams T;
    T.P = P;
    T.tiles = (W.V + tile_v - 1) / tile_v;
    T.padded = static_cast<int>(padded_rows(P.rows));
    T.row_blocks = T.padded / nt;
    if (static_cast<int64_t>(T.tiles) * T.row_blocks * W.blocks > 0x7FFFFFFF) return FEF_ERR_INVALID_ARG;   // (counted in 32 bits)
    T.items = T.tiles * T.row_blocks;
    T.out_bf16 = dt == FEF_BF16;
#ifdef FEF_TEST_HOOKS
    T.withhold = g_test_withhold;   // one call only
    g_test_withhold = -1;
#endif
    CUtensorMap map;
    const uint64_t cols = static_cast<uint64_t>(W.blocks) * kBlock;
    if (!map_2d(&map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, H.operand, cols, T.padded, cols * 2, 64, nt, CU_TENSOR_MAP_SWIZZLE_128B))
        return FEF_ERR_CUDA;
    prepare_kernel<<<T.padded, kPrepareThreads, 0, stream>>>(H);
    if (cudaGetLastError() != cudaSuccess) return FEF_ERR_CUDA;

    const int grid = T.items < sms ? T.items : sms;
    return nt == 64 ? launch_g<64, 2>(map, T, dev, grid, stream) : launch_g<128, 1>(map, T, dev, grid, stream);
}

}  // namespace quant
}  // namespace fef

#ifdef FEF_TEST_HOOKS
// Test builds only (never part of the shipped library): in the next product of more than 16 rows CTA 0 withholds the hidden rows of
// its block number `block`, so that the waits for them run out after their second.
extern "C" void fef_test_withhold_product_block_once(int block) { fef::quant::g_test_withhold = block; }
#endif
