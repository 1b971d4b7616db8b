// fef_lmhead_logits_quantized for few hidden rows (up to 16): bound by the weight bytes.
//
// The weights are the left operand of m16n8k16 matrix instructions, 16 vocabulary rows at a time, the hidden rows the right
// one (8 or 16 columns).  A sum over k may be taken in any order as long as both operands agree on it, so a lane uses the
// columns as the packed layout hands them to it: 16 bytes of a row are the lane's share of a 128-column block, each of
// their four words two k-steps.  In the same way operand row g of the i-th eight rows of a unit of 32 is vocabulary row
// 4 g + i: a lane's four scales lie together, and so do its four logits of a hidden row.
//
// Nibbles become the bfloat16 numbers (q - z) / 64 before they are multiplied, nine instructions for eight weights (low_pair below).
// Masking alone would be five, with the zero points taken off the group's sum, sum q x - z sum x; but then a large x loses the
// group's other products even where q = z, without a bound (logits off by 2e-3 at one channel of 1e5 in 4096).  The products of
// a group are added up in binary32 by the matrix instructions, then scaled in binary32; the 64 comes back with the logits.
//
// One CTA of 16 warps per SM takes an even share of the vocabulary in units of 32 rows; all blocks of its units in a row are
// cut into 16 equal runs, one per warp, so that all end together.  A unit that lies in more than one run is joined at the
// very end: the warps behind leave their sums in shared memory, the warp that holds its beginning adds them up, in order.
// Every warp loads its weights straight into registers,
// kAhead blocks ahead of the arithmetic: 126464 x 2048 bytes in this order and nothing else took 42 us (6.1 TB/s), as did TMA
// boxes through a shared-memory ring; with the arithmetic the ring took 75 us, its waits and hand-overs being most of the
// instructions.  The hidden rows stay in shared memory, rearranged into operand order once.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "fef_quant.cuh"

namespace fef {
namespace quant {
namespace {

constexpr int kUnit = 32;    // vocabulary rows of a warp: two 16-row operands
constexpr int kWarps = 16;
constexpr int kThreads = kWarps * 32;
constexpr size_t kSmemLimit = 232448;

struct Plan {
    int units;    // of the whole vocabulary
    size_t smem;  // hidden rows, one place per warp for the sums of a shared unit; 0: not for this kernel
};

Plan make_plan(const ProductParams& P) {
    Plan L = {};
    const int nt = P.rows > 8 ? 2 : 1;
    L.units = (P.layer.V + kUnit - 1) / kUnit;
    const size_t smem = static_cast<size_t>(P.layer.blocks) * 2048 * nt + kWarps * 1024 * nt;
    L.smem = smem <= kSmemLimit - 1024 ? smem : 0;
    return L;
}

__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The first product of a group: no earlier sum.
__device__ __forceinline__ void mma_16816_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                                uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// Two nibbles of a word, less their zero points: a nibble becomes a bfloat16 number by masking alone, since the bit pattern v < 256 in
// the lower half of a bfloat16 (the mantissa and the lowest exponent bit) is the number v 2^-133, below and above the smallest
// normal number alike.  Bits 0..3 of each half of a word (columns 0 and 4 of its eight; after a shift by 8: 2 and 6) stand for
// q 2^-133, bits 4..7 (1 and 5; 3 and 7) for 16 q 2^-133; one fused multiply-add takes either to (q - z) 2^-6, exactly.  The
// form with 128 + q (centred_pair) needs two more shifts, and the pipe of shifts and masks is the busiest: 54 against 51 us at 1 row x
// 126464 x 4096, 67 against 59 us at 8 rows x 152064 x 3584 in groups of 64 with zero points.
__device__ __forceinline__ uint32_t fma_bf16_pair(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
__device__ __forceinline__ uint32_t low_pair(uint32_t word, uint32_t centre) {
    return fma_bf16_pair(word & 0x000F000Fu, 0x7F007F00u, centre);   // 2^127
}
__device__ __forceinline__ uint32_t high_pair(uint32_t word, uint32_t centre) {
    return fma_bf16_pair(word & 0x00F000F0u, 0x7D007D00u, centre);   // 2^123
}
// -z / 64 twice, from byte `i` of a word of zero points.
__device__ __forceinline__ uint32_t centre_of_byte(uint32_t z, int i) {
    return fma_bf16_pair(__byte_perm(z, 0u, 0x4040u + 0x0101u * i), 0xFF00FF00u, 0u);   // -2^127
}
constexpr uint32_t kCentre8 = 0xBE00BE00u;   // -8 / 64

// What a warp needs of one block of its unit: operand rows 4 g + i, their scales and zero points.
template <int N, bool ZERO>
struct Fetched {
    uint4 q[4];
    uint32_t s[2 * N];          // 4 rows x N groups, two to a word
    uint32_t z[ZERO ? N : 1];   // ..., four to a word
    __device__ __forceinline__ uint32_t scale(int i, int j) const { return s[(i * N + j) / 2] >> (16 * ((i * N + j) & 1)) & 0xFFFFu; }
    __device__ __forceinline__ uint32_t centre(int i, int j) const {
        return ZERO ? centre_of_byte(z[(i * N + j) / 4], (i * N + j) & 3) : kCentre8;
    }
};

template <int NT, int N, bool ZERO>   // 8 NT hidden rows, N groups per block
__global__ void __launch_bounds__(kThreads, 1)
product_rows_kernel(const __grid_constant__ ProductParams P, const __grid_constant__ Plan L, int out_bf16) {
    extern __shared__ __align__(16) unsigned char smem[];
    constexpr int kAhead = NT == 1 ? 3 : 2;
    const Layer& W = P.layer;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, t = lane & 3;
    const int unit_begin = static_cast<int>(static_cast<int64_t>(L.units) * blockIdx.x / gridDim.x);
    const int unit_end = static_cast<int>(static_cast<int64_t>(L.units) * (blockIdx.x + 1) / gridDim.x);
    const int64_t total_blocks = static_cast<int64_t>(unit_end - unit_begin) * W.blocks;
    auto run_begin = [&](int w) { return static_cast<int>(total_blocks * w / kWarps); };
    const int begin = run_begin(warp), end = run_begin(warp + 1);
    const int64_t pitch = static_cast<int64_t>(W.blocks) * 64;

    // ---- the flat sequence of this warp's blocks, fetched ahead.  Past its end the last block is fetched again: with a branch
    //      around the loads, waiting for one block's waits for the blocks behind it too (52 against 45 us for the loads alone).
    int fetch_at = begin, fetch_unit = unit_begin + begin / W.blocks, fetch_block = begin % W.blocks;
    const uint8_t* fetch_w;
    uint32_t row_at[4];
    auto seek = [&]() {   // (rows behind V are read as the last one; their logits are not stored)
        const int64_t v = static_cast<int64_t>(fetch_unit) * kUnit + 4 * g;
        const int64_t v0 = min(v, static_cast<int64_t>(W.V - 1));
        fetch_w = W.packed + v0 * pitch + t * 16;
#pragma unroll
        for (int i = 0; i < 4; ++i) row_at[i] = static_cast<uint32_t>((min(v + i, static_cast<int64_t>(W.V - 1)) - v0) * pitch);
    };
    auto fetch = [&](Fetched<N, ZERO>& f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f.q[i] = ld_global_nc_v4(fetch_w + row_at[i] + fetch_block * 64);
        const int64_t at = (static_cast<int64_t>(fetch_block) * W.Vp + static_cast<int64_t>(fetch_unit) * kUnit + 4 * g) * N;
        if constexpr (N == 1) {
            const uint2 x = __ldg(reinterpret_cast<const uint2*>(W.scale + at));
            f.s[0] = x.x;
            f.s[1] = x.y;
        } else {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const uint4 x = __ldg(reinterpret_cast<const uint4*>(W.scale + at) + i);
                f.s[4 * i] = x.x;
                f.s[4 * i + 1] = x.y;
                f.s[4 * i + 2] = x.z;
                f.s[4 * i + 3] = x.w;
            }
        }
        if constexpr (ZERO) {
#pragma unroll
            for (int i = 0; i < N; ++i) f.z[i] = __ldg(reinterpret_cast<const uint32_t*>(W.zero + at) + i);
        }
        const int more = fetch_at + 1 < end ? 1 : 0;
        fetch_at += more;
        fetch_block += more;
        if (fetch_block == W.blocks) {
            fetch_block = 0;
            ++fetch_unit;
            seek();
        }
    };
    Fetched<N, ZERO> ahead[kAhead];
    seek();
#pragma unroll
    for (int i = 0; i < kAhead; ++i) fetch(ahead[i]);

    // ---- hidden rows into operand order: 16 bytes per (block, word, row, t), columns 0 4, 1 5, 2 6, 3 7 of the eight
    constexpr int kPieces = 32 * NT;   // 16-byte pieces per block and word
    const int pieces = W.blocks * 4 * kPieces;
    for (int at0 = threadIdx.x; at0 < pieces; at0 += 4 * kThreads) {
        uint4 x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {   // (four loads in flight)
            const int at = at0 + u * kThreads, cw = at / kPieces, k = (cw >> 2) * kBlock + (cw & 3) * 32 + (at & 3) * 8;
            const int row = at / 4 % (8 * NT);
            x[u] = make_uint4(0u, 0u, 0u, 0u);
            if (at < pieces && row < P.rows && k < W.d)
                x[u] = __ldg(reinterpret_cast<const uint4*>(P.hidden + static_cast<int64_t>(row) * W.d + k));
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (at0 + u * kThreads < pieces)
                *reinterpret_cast<uint4*>(smem + (at0 + u * kThreads) * 16) =
                    make_uint4(__byte_perm(x[u].x, x[u].z, 0x5410), __byte_perm(x[u].x, x[u].z, 0x7632),
                               __byte_perm(x[u].y, x[u].w, 0x5410), __byte_perm(x[u].y, x[u].w, 0x7632));
    }
    __syncthreads();

    // ---- the units
    float acc[2][NT][4];
    auto clear = [&]() {
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[m][n][i] = 0.f;
    };
    auto multiply = [&](const Fetched<N, ZERO>& f, int block) {
        const unsigned char* h_at = smem + block * (2048 * NT) + lane * 16;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            float sum[2][NT][4];
            uint32_t centre[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) centre[i] = f.centre(i, j);
#pragma unroll
            for (int w = j * (4 / N); w < (j + 1) * (4 / N); ++w) {
                uint4 h[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n) h[n] = *reinterpret_cast<const uint4*>(h_at + w * (512 * NT) + n * 512);
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    const uint4 &lo = f.q[2 * m], &hi = f.q[2 * m + 1];
                    const uint32_t a = w == 0 ? lo.x : w == 1 ? lo.y : w == 2 ? lo.z : lo.w;
                    const uint32_t b = w == 0 ? hi.x : w == 1 ? hi.y : w == 2 ? hi.z : hi.w;
                    const uint32_t ca = centre[2 * m], cb = centre[2 * m + 1];
                    const uint32_t a0 = low_pair(a, ca), b0 = low_pair(b, cb), a1 = high_pair(a, ca), b1 = high_pair(b, cb);
                    const uint32_t a2 = low_pair(a >> 8, ca), b2 = low_pair(b >> 8, cb);
                    const uint32_t a3 = high_pair(a >> 8, ca), b3 = high_pair(b >> 8, cb);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        if (w == j * (4 / N))
                            mma_16816_first(sum[m][n], a0, b0, a1, b1, h[n].x, h[n].y);
                        else
                            mma_16816(sum[m][n], a0, b0, a1, b1, h[n].x, h[n].y);
                        mma_16816(sum[m][n], a2, b2, a3, b3, h[n].z, h[n].w);
                    }
                }
            }
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const float sa = bf16_value(f.scale(2 * m, j)), sb = bf16_value(f.scale(2 * m + 1, j));
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    acc[m][n][0] = fmaf(sum[m][n][0], sa, acc[m][n][0]);
                    acc[m][n][1] = fmaf(sum[m][n][1], sa, acc[m][n][1]);
                    acc[m][n][2] = fmaf(sum[m][n][2], sb, acc[m][n][2]);
                    acc[m][n][3] = fmaf(sum[m][n][3], sb, acc[m][n][3]);
                }
            }
        }
    };
    // Lane (g, t) holds vocabulary rows 4 g .. 4 g + 3 of hidden rows 8 n + 2 t + c: acc[0][n][c], acc[0][n][2 + c],
    // acc[1][n][c], acc[1][n][2 + c].
    auto store = [&](int unit) {
        const int64_t v = static_cast<int64_t>(unit) * kUnit + 4 * g;
        const int many = static_cast<int>(min(max(W.V - v, static_cast<int64_t>(0)), static_cast<int64_t>(4)));
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int row = n * 8 + 2 * t + c;
                if (row >= P.rows) continue;
                const float y[4] = {acc[0][n][c] * 64.f, acc[0][n][2 + c] * 64.f, acc[1][n][c] * 64.f, acc[1][n][2 + c] * 64.f};
                const int64_t at = row * P.ldo + v;
                if (out_bf16) {
                    __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(P.out) + at;
                    if (many == 4)
                        *reinterpret_cast<uint2*>(o) = make_uint2(bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3]));
                    else
                        for (int i = 0; i < 4; ++i)
                            if (i < many) o[i] = __float2bfloat16_rn(y[i]);
                } else {
                    float* o = reinterpret_cast<float*>(P.out) + at;
                    if (many == 4)
                        *reinterpret_cast<float4*>(o) = make_float4(y[0], y[1], y[2], y[3]);
                    else
                        for (int i = 0; i < 4; ++i)
                            if (i < many) o[i] = y[i];
                }
            }
    };
    float4* places = reinterpret_cast<float4*>(smem + W.blocks * 2048 * NT);   // [warp][2 NT][lane]
    if (P.status && blockIdx.x == 0 && threadIdx.x == 0) *P.status = FEF_OK;
    clear();
    int at = begin, unit = unit_begin + begin / W.blocks, block = begin % W.blocks;
    bool whole = block == 0;   // the sums go back to the unit's first block
    auto next_block = [&]() {
        ++at;
        ++block;
        if (!whole && (block == W.blocks || at == end)) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    places[warp * (64 * NT) + (2 * n + c) * 32 + lane] =
                        make_float4(acc[0][n][c], acc[0][n][2 + c], acc[1][n][c], acc[1][n][2 + c]);
        } else if (block == W.blocks) {
            store(unit);
        }
        if (block == W.blocks) {
            clear();
            block = 0;
            whole = true;
            ++unit;
        }
    };
    while (at + kAhead <= end) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            multiply(ahead[i], block);
            fetch(ahead[i]);
            next_block();
        }
    }
#pragma unroll
    for (int i = 0; i < kAhead - 1; ++i)
        if (at < end) {
            multiply(ahead[i], block);
            next_block();
        }
    __syncthreads();
    if (begin < end && whole && block > 0) {   // the unit goes on in the runs behind
        int left = W.blocks - block;
        for (int w = warp + 1; left > 0; ++w) {
            const int run = run_begin(w + 1) - run_begin(w);
            if (run > 0) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const float4 x = places[w * (64 * NT) + (2 * n + c) * 32 + lane];
                        acc[0][n][c] += x.x;
                        acc[0][n][2 + c] += x.y;
                        acc[1][n][c] += x.z;
                        acc[1][n][2 + c] += x.w;
                    }
            }
            left -= run;
        }
        store(unit);
    }
}

bool g_attr[64][2][3][2];

template <int NT, int N, bool ZERO>
fef_status launch(const ProductParams& P, const Plan& L, fef_dtype dt, int dev, int grid, cudaStream_t stream) {
    bool& done = g_attr[dev][NT - 1][N / 2][ZERO];
    if (!done) {
        if (cudaFuncSetAttribute(product_rows_kernel<NT, N, ZERO>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 static_cast<int>(kSmemLimit - 1024)) != cudaSuccess)
            return FEF_ERR_CUDA;
        done = true;
    }
    product_rows_kernel<NT, N, ZERO><<<grid, kThreads, L.smem, stream>>>(P, L, dt == FEF_BF16);
    return cudaGetLastError() == cudaSuccess ? FEF_OK : FEF_ERR_CUDA;
}

template <int NT, int N>
fef_status launch_z(const ProductParams& P, const Plan& L, fef_dtype dt, int dev, int grid, cudaStream_t stream) {
    return P.layer.zero ? launch<NT, N, true>(P, L, dt, dev, grid, stream) : launch<NT, N, false>(P, L, dt, dev, grid, stream);
}

template <int NT>
fef_status launch_g(const ProductParams& P, const Plan& L, fef_dtype dt, int dev, int grid, cudaStream_t stream) {
    switch (P.layer.G) {
        case 32: return launch_z<NT, 4>(P, L, dt, dev, grid, stream);
        case 64: return launch_z<NT, 2>(P, L, dt, dev, grid, stream);
        default: return launch_z<NT, 1>(P, L, dt, dev, grid, stream);
    }
}

}  // namespace

bool rows_kernel_takes(const ProductParams& P) { return P.rows <= 16 && make_plan(P).smem > 0; }

fef_status launch_rows_kernel(const ProductParams& P, fef_dtype dt, int dev, int sms, cudaStream_t stream) {
    const Plan L = make_plan(P);
    const int grid = L.units < sms ? L.units : sms;
    return P.rows > 8 ? launch_g<2>(P, L, dt, dev, grid, stream) : launch_g<1>(P, L, dt, dev, grid, stream);
}

}  // namespace quant
}  // namespace fef
