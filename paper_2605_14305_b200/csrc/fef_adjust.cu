// fef_logits_adjust: penalties for repeated tokens, biases and grammar masks on the logits of speculative
// windows, with the normaliser of every adjusted row (the input of fef_spec_verify_with_norms).
//
// For window b, position i and vocabulary id x, in binary32:
//   h = occurrences of x in tokens[b, :] and among the window's drafts j < i,
//   a = the same without the first prompt_len[b] tokens,
//   y = l                                    if h = 0
//       l / rep (l > 0), l * rep (l <= 0)    if h > 0
//   y = y + (bias[x] - (freq * a + pres * [a > 0])),   y = -inf where the mask's bit is 0,
//   out = y rounded to the logits' type,     log2_norm = log2 sum_x 2^(out_x * log2(e) / T).
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "fef.h"
#include "fef_common.cuh"
#include "fef_device_math.cuh"

namespace fef {
namespace adj {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kIdsPerThread = 8;                       // one 16-byte vector of bfloat16, two of binary32
constexpr int kChunk = kThreads * kIdsPerThread;       // vocabulary ids per CTA
constexpr int kRowsInFlight = 4;                       // rows whose loads a thread has in flight together
constexpr uint32_t kInPrompt = 0x80000000u;            // history word: seen in the prompt; low bits count the answer

struct Params {
    const char* logits;
    char* out;
    int64_t ld_bytes;
    const int32_t* tokens;       // [B][L]
    const int32_t* prompt_len;   // [B] or null
    const int32_t* drafts;       // [B][K] or null
    const int32_t* row_len;      // [B] or null
    const float* penalties;      // [B][3] or null
    const float* bias;           // or null
    int64_t bias_stride;
    const uint32_t* allowed;     // or null
    int64_t allowed_stride_b, allowed_stride_k;
    int L, B, K, V, chunks, rows_per_cta;
    float c;                     // log2(e) / T
    double c_law, norm_scale;    // the law's scale in double precision, and what turns its normaliser into one for log2(e) / T
    float2* partials;            // [B * K][chunks]: (largest logit m, sum of 2^((l - m) c))
    double* log2_norm;           // [B * K]
};

__device__ __forceinline__ uint4 ld_stream_v4(const void* p) {
    // (not .nc: the output may be the input)
    uint4 r;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
                 : "l"(p)
                 : "memory");
    return r;
}

template <int DT>
struct Row8 {  // a thread's eight logits of one row, as stored
    uint4 v[DT == FEF_F32 ? 2 : 1];
};

template <int DT>
__device__ __forceinline__ void unpack8(const Row8<DT>& r, float (&l)[8]) {
    if constexpr (DT == FEF_F32) {
        unpack<FEF_F32>(r.v[0], *reinterpret_cast<float(*)[4]>(&l[0]));
        unpack<FEF_F32>(r.v[1], *reinterpret_cast<float(*)[4]>(&l[4]));
    } else {
        unpack<FEF_BF16>(r.v[0], l);
    }
}

// Two binary32 numbers as one operand.
__device__ __forceinline__ uint64_t two(float a, float b) { return static_cast<uint64_t>(__float_as_uint(b)) << 32 | __float_as_uint(a); }
__device__ __forceinline__ float first_of(uint64_t x) { return __uint_as_float(static_cast<uint32_t>(x)); }
__device__ __forceinline__ float second_of(uint64_t x) { return __uint_as_float(static_cast<uint32_t>(x >> 32)); }
__device__ __forceinline__ uint64_t add_two(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul_two(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// Largest of the warp's numbers (NaN does not count).
__device__ __forceinline__ float warp_max_f32(float x) {
    float r;
    asm("redux.sync.max.f32 %0, %1, 0xFFFFFFFF;" : "=f"(r) : "f"(x));
    return r;
}
// Bits 0..3 at the tops of four bytes, and bytes filled with the top bit of one of them (selectors 8 + byte).
__device__ __forceinline__ uint32_t byte_tops(uint32_t bits) { return (bits & 15u) * 0x10204080u; }
__device__ __forceinline__ uint32_t spread_tops(uint32_t tops, uint32_t selectors) {
    uint32_t r;
    asm("prmt.b32 %0, %1, 0, %2;" : "=r"(r) : "r"(tops), "r"(selectors));
    return r;
}
__device__ __forceinline__ uint32_t pick(uint32_t x, uint32_t otherwise, uint32_t mask) { return (x & mask) | (otherwise & ~mask); }

// Rounds to the stored type, -inf where the mask's bit is 0; l becomes the stored values.
template <int DT>
__device__ __forceinline__ Row8<DT> pack8(float (&l)[8], uint32_t allowed) {
    Row8<DT> r;
    uint32_t w[DT == FEF_F32 ? 8 : 4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t tops = byte_tops(allowed >> (4 * h));
        if constexpr (DT == FEF_F32) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                w[4 * h + j] = pick(__float_as_uint(l[4 * h + j]), 0xFF800000u, spread_tops(tops, 0x8888u + 0x1111u * j));
        } else {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const __nv_bfloat162 v = __floats2bfloat162_rn(l[4 * h + 2 * j], l[4 * h + 2 * j + 1]);
                w[2 * h + j] = pick(*reinterpret_cast<const uint32_t*>(&v), 0xFF80FF80u, spread_tops(tops, j == 0 ? 0x9988u : 0xBBAAu));
            }
        }
    }
    r.v[0] = make_uint4(w[0], w[1], w[2], w[3]);
    if constexpr (DT == FEF_F32) r.v[1] = make_uint4(w[4], w[5], w[6], w[7]);
    unpack8<DT>(r, l);
    return r;
}

// l / rep for l > 0, l * rep otherwise; `inv` = 1 / rep.  The quotient takes one step of Markstein's correction (an infinite one
// skips it).
__device__ __forceinline__ float repeat_penalty(float l, float rep, float inv) {
    const float q = l * inv, fixed = fmaf(fmaf(-q, rep, l), inv, q);
    return l > 0.f ? (q < INFINITY ? fixed : q) : l * rep;
}

// One CTA per 2048 ids of a window and a run of its positions; a thread keeps eight ids over all of them: their additive term and
// repetition flags in registers, their counts in shared memory, so that the text is counted once and a position's draft is added
// for the positions behind it without a barrier.  Four rows are in flight per thread.  The bound is memory (every logit read
// and written once) with instruction issue close behind: 64 windows x 32 x 126464 bfloat16 with every rule and the normalisers
// 215 to 225 us by GPU = 5.0 TB/s (0.78 of the copy rate), 16 x 32 x 152064 binary32 118 to 123 us = 5.2 TB/s.  More resident CTAs pay
// although a few registers spill (on one GPU, bfloat16: three 245, four 219, five 212 us; binary32: two 129, three 119, four 139).
template <int DT, bool NORM>
__global__ void __launch_bounds__(kThreads, DT == FEF_F32 ? 3 : 5) adjust_kernel(const __grid_constant__ Params P) {
    __shared__ uint32_t s_hist[kChunk];
    __shared__ int s_draft[FEF_MAX_K];
    __shared__ float2 s_part[NORM ? FEF_MAX_K : 1][kWarps];
    constexpr int E = Elem<DT>::kBytes;

    const int b = blockIdx.z, k0 = blockIdx.y * P.rows_per_cta;
    const int n = P.row_len ? min(max(__ldg(P.row_len + b), 0), P.K) : P.K;
    const int k1 = min(k0 + P.rows_per_cta, n);
    if (k0 >= k1) return;  // uniform over the CTA
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int chunk0 = blockIdx.x * kChunk, x0 = chunk0 + tid * kIdsPerThread;
    const int valid = min(max(P.V - x0, 0), kIdsPerThread);

    // ---- what stands in the text of this chunk's ids
    float rep = 1.f, freq = 0.f, pres = 0.f;
    const bool counting = P.penalties != nullptr, drafts = counting && P.drafts != nullptr;
    if (counting) {
        rep = __ldg(P.penalties + 3 * b);
        freq = __ldg(P.penalties + 3 * b + 1);
        pres = __ldg(P.penalties + 3 * b + 2);
        for (int j = tid; j < kChunk; j += kThreads) s_hist[j] = 0u;
        if (tid < P.K) s_draft[tid] = P.drafts && tid < k1 ? __ldg(P.drafts + static_cast<int64_t>(b) * P.K + tid) : -1;
        __syncthreads();
        const int prompt = P.prompt_len ? __ldg(P.prompt_len + b) : 0;
        const int32_t* text = P.tokens + static_cast<int64_t>(b) * P.L;
        const unsigned width = min(P.V - chunk0, kChunk);
        for (int t0 = tid; t0 < P.L; t0 += 4 * kThreads) {
            int id[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) id[u] = t0 + u * kThreads < P.L ? __ldg(text + t0 + u * kThreads) : -1;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const unsigned at = static_cast<unsigned>(id[u]) - chunk0;  // (a negative id ends far above `width`)
                if (at < width) {
                    if (t0 + u * kThreads < prompt)
                        atomicOr(s_hist + at, kInPrompt);
                    else
                        atomicAdd(s_hist + at, 1u);
                }
            }
        }
        if (tid < k0) {
            const unsigned at = static_cast<unsigned>(s_draft[tid]) - chunk0;
            if (at < width) atomicAdd(s_hist + at, 1u);
        }
        __syncthreads();
    }

    // ---- the additive term and the repetition flags of this thread's ids
    const float inv = 1.f / rep;
    uint64_t add[kIdsPerThread / 2];
    unsigned repeated = 0u;
    // (from here on a thread's eight counts are its own)
    auto term = [&](int j) {
        const float bias = P.bias && j < valid ? __ldg(P.bias + b * P.bias_stride + x0 + j) : 0.f;
        const uint32_t h = counting ? s_hist[tid * kIdsPerThread + j] : 0u, a = h & ~kInPrompt;
        if (h) repeated |= 1u << j;
        return a ? bias - fmaf(freq, static_cast<float>(a), pres) : bias;
    };
#pragma unroll
    for (int j = 0; j < kIdsPerThread; j += 2) {
        const float t = term(j);
        add[j / 2] = two(t, term(j + 1));
    }
    unsigned anywhere = rep != 1.f ? __reduce_or_sync(0xFFFFFFFFu, repeated) : 0u;   // ids that some lane has to penalise

    const int64_t row0 = static_cast<int64_t>(b) * P.K;
    const char* src = P.logits + row0 * P.ld_bytes + static_cast<int64_t>(x0) * E;
    char* dst = P.out + row0 * P.ld_bytes + static_cast<int64_t>(x0) * E;
    const unsigned char* bits = P.allowed
        ? reinterpret_cast<const unsigned char*>(P.allowed + b * P.allowed_stride_b) + (x0 >> 3) : nullptr;

    const unsigned exist = (1u << valid) - 1u;   // ids behind V: -inf, never stored
    const int64_t to_out = dst - src;            // (the same place of the output)
    const bool whole = __all_sync(0xFFFFFFFFu, valid == kIdsPerThread);
    const char* from = src + k0 * P.ld_bytes;
    if (bits) bits += k0 * P.allowed_stride_k * 4;

    // Up to four rows: all of them and all ids there (FULL), or any.
    auto batch = [&](auto full, int i0) {
        constexpr bool FULL = decltype(full)::value;
        Row8<DT> raw[kRowsInFlight];
        unsigned mask[kRowsInFlight];
#pragma unroll
        for (int r = 0; r < kRowsInFlight; ++r) {
            const char* p = from + r * P.ld_bytes;
            mask[r] = 0xFFu;
            if (FULL || (i0 + r < k1 && valid)) {
                if (FULL || valid == kIdsPerThread) {
                    raw[r].v[0] = ld_stream_v4(p);
                    if constexpr (DT == FEF_F32) raw[r].v[1] = ld_stream_v4(p + 16);
                } else {
                    float l[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        l[j] = 0.f;
                        if (j < valid) {
                            if constexpr (DT == FEF_F32)
                                l[j] = *reinterpret_cast<const volatile float*>(p + 4 * j);
                            else
                                l[j] = __uint_as_float(
                                    static_cast<uint32_t>(*reinterpret_cast<const volatile unsigned short*>(p + 2 * j)) << 16);
                        }
                    }
                    raw[r] = pack8<DT>(l, 0xFFu);
                }
                if (bits) mask[r] = __ldg(bits + r * P.allowed_stride_k * 4);
            }
        }
        float top[kRowsInFlight], sum[kRowsInFlight];
#pragma unroll
        for (int r = 0; r < kRowsInFlight; ++r) {
            top[r] = sum[r] = 0.f;
            if (FULL || i0 + r < k1) {   // (uniform over the CTA)
                float l[8];
                unpack8<DT>(raw[r], l);
                if (anywhere) {   // (uniform over the warp, and so is every test in it)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (anywhere >> j & 1u) {
                            const float y = repeat_penalty(l[j], rep, inv);
                            l[j] = repeated >> j & 1u ? y : l[j];
                        }
                }
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const uint64_t y = add_two(two(l[j], l[j + 1]), add[j / 2]);
                    l[j] = first_of(y);
                    l[j + 1] = second_of(y);
                }
                const Row8<DT> w = pack8<DT>(l, FULL ? mask[r] : mask[r] & exist);
                char* q = const_cast<char*>(from) + r * P.ld_bytes + to_out;
                if (FULL || valid == kIdsPerThread) {
                    *reinterpret_cast<uint4*>(q) = w.v[0];
                    if constexpr (DT == FEF_F32) *reinterpret_cast<uint4*>(q + 16) = w.v[1];
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (j < valid) {
                            if constexpr (DT == FEF_F32)
                                reinterpret_cast<float*>(q)[j] = l[j];
                            else
                                reinterpret_cast<unsigned short*>(q)[j] = static_cast<unsigned short>(__float_as_uint(l[j]) >> 16);
                        }
                }
                if constexpr (NORM) {
                    // Relative to the warp's largest logit, subtracted before the scaling: a row whose entries are all the
                    // type's lowest value then has a normaliser like any other.
                    const float m = warp_max_f32(fmaxf(fmaxf(fmaxf(l[0], l[1]), fmaxf(l[2], l[3])),
                                                       fmaxf(fmaxf(l[4], l[5]), fmaxf(l[6], l[7]))));
                    top[r] = m > -INFINITY ? m : 0.f;
                    const uint64_t down = two(-top[r], -top[r]), c2 = two(P.c, P.c);
                    float s[4];
#pragma unroll
                    for (int j = 0; j < 8; j += 2) {
                        const uint64_t e = mul_two(add_two(two(l[j], l[j + 1]), down), c2);
                        s[j / 2] = ex2_approx(first_of(e)) + ex2_approx(second_of(e));
                    }
                    sum[r] = (s[0] + s[1]) + (s[2] + s[3]);
                }
                // the draft of this position counts for the positions behind it
                if (drafts) {
                    const unsigned at = static_cast<unsigned>(s_draft[i0 + r]) - x0;
                    const bool mine = at < static_cast<unsigned>(valid);
                    if (__any_sync(0xFFFFFFFFu, mine)) {
                        if (mine) {
                            ++s_hist[tid * kIdsPerThread + at];
                            const float t = term(static_cast<int>(at));
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                if (at == static_cast<unsigned>(j))
                                    add[j / 2] = j & 1 ? two(first_of(add[j / 2]), t) : two(t, second_of(add[j / 2]));
                        }
                        anywhere = rep != 1.f ? __reduce_or_sync(0xFFFFFFFFu, repeated) : 0u;
                    }
                }
            }
        }
        if constexpr (NORM) {
            // four rows' sums over the warp with six shuffles: lanes 8 r .. 8 r + 7 end with row r's
            static_assert(kRowsInFlight == 4, "");
            const bool upper = lane & 16, odd = lane & 8;
            float a = upper ? sum[2] : sum[0], c = upper ? sum[3] : sum[1];
            a += __shfl_xor_sync(0xFFFFFFFFu, upper ? sum[0] : sum[2], 16);
            c += __shfl_xor_sync(0xFFFFFFFFu, upper ? sum[1] : sum[3], 16);
            float s = (odd ? c : a) + __shfl_xor_sync(0xFFFFFFFFu, odd ? a : c, 8);
            s += __shfl_xor_sync(0xFFFFFFFFu, s, 4);
            s += __shfl_xor_sync(0xFFFFFFFFu, s, 2);
            s += __shfl_xor_sync(0xFFFFFFFFu, s, 1);
            const int r = lane >> 3;
            const float t = upper ? (odd ? top[3] : top[2]) : (odd ? top[1] : top[0]);
            if ((lane & 7) == 0 && (FULL || i0 + r < k1)) s_part[i0 + r - k0][warp] = make_float2(t, s);
        }
        from += kRowsInFlight * P.ld_bytes;
        if (bits) bits += kRowsInFlight * P.allowed_stride_k * 4;
    };
    int i0 = k0;
    if (whole)
        for (; i0 + kRowsInFlight <= k1; i0 += kRowsInFlight) batch(std::true_type{}, i0);
    for (; i0 < k1; i0 += kRowsInFlight) batch(std::false_type{}, i0);
    if constexpr (NORM) {
        __syncthreads();
        // The warps' sums are added up in double precision, eight lanes per row: a term then carries three roundings of its
        // argument (two for bfloat16), two ex2 and nine roundings of sums, 1.9e-6 in all; added up in binary32 it would be 2.4e-6,
        // and the residual draw counts on 2e-6.
        const int parts = (k1 - k0) * kWarps;
        for (int at0 = warp * 32; at0 < parts; at0 += kThreads) {
            const int at = at0 + lane, i = at / kWarps;
            const float2 p = at < parts ? s_part[i][at % kWarps] : make_float2(0.f, 0.f);
            float m = p.y != 0.f ? p.x : -INFINITY;
#pragma unroll
            for (int o = 1; o < kWarps; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
            double s = p.y != 0.f ? static_cast<double>(p.y) * ex2_approx((p.x - m) * P.c) : 0.0;
#pragma unroll
            for (int o = 1; o < kWarps; o <<= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
            if (at < parts && at % kWarps == 0) P.partials[(row0 + k0 + i) * P.chunks + blockIdx.x] = make_float2(m, static_cast<float>(s));
        }
    }
}

// log2 of the row sums from the chunks' partial sums, in double precision: one warp per row.  A bfloat16 law is the one that the
// draws and the verification evaluate: with log2(e) / T rounded to binary32 (c), and its normaliser scaled as theirs are.
__global__ void __launch_bounds__(kThreads) adjust_norm_kernel(const __grid_constant__ Params P) {
    cudaGridDependencySynchronize();
    const int lane = threadIdx.x & 31;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
    if (row >= static_cast<int64_t>(P.B) * P.K) return;
    const int b = static_cast<int>(row / P.K), i = static_cast<int>(row - static_cast<int64_t>(b) * P.K);
    const int n = P.row_len ? min(max(__ldg(P.row_len + b), 0), P.K) : P.K;
    if (i >= n) {
        if (lane == 0) P.log2_norm[row] = 0.0;
        return;
    }
    double m = -INFINITY, s = 0.0;
    for (int c = lane; c < P.chunks; c += 32) {
        const float2 p = P.partials[row * P.chunks + c];
        if (p.y != 0.f) {  // (a NaN sum poisons the row)
            const double nm = fmax(m, static_cast<double>(p.x));
            s = (m > -INFINITY ? s * exp2((m - nm) * P.c_law) : 0.0) +
                static_cast<double>(p.y) * exp2((static_cast<double>(p.x) - nm) * P.c_law);
            m = nm;
        }
    }
    const double top = warp_max(m);
    const double sum = warp_sum(m > -INFINITY ? s * exp2((m - top) * P.c_law) : 0.0);
    if (lane == 0)
        P.log2_norm[row] = sum > 0.0 && sum < INFINITY ? (top * P.c_law + log2(sum)) * P.norm_scale : static_cast<double>(NAN);
}

static int chunks_of(int V) { return (V + kChunk - 1) / kChunk; }

static bool sizes_ok(int B, int K, int V) {
    return B >= 1 && B <= FEF_MAX_B && K >= 1 && K <= FEF_MAX_K && V >= 1 && V <= (1 << 28);
}

template <int DT>
static void launch(const Params& P, int splits, bool norm, cudaStream_t stream) {
    const dim3 grid(P.chunks, splits, P.B);
    if (norm)
        adjust_kernel<DT, true><<<grid, kThreads, 0, stream>>>(P);
    else
        adjust_kernel<DT, false><<<grid, kThreads, 0, stream>>>(P);
}

}  // namespace adj
}  // namespace fef

extern "C" {

size_t fef_logits_adjust_workspace_bytes(int B, int K, int V) {
    using namespace fef::adj;
    if (!sizes_ok(B, K, V)) return 0;
    return static_cast<size_t>(B) * K * chunks_of(V) * sizeof(float2);
}

fef_status fef_logits_adjust(const void* logits, void* out, int B, int K, int V, int64_t ld, fef_dtype dt,
                             const int32_t* tokens, int L, const int32_t* prompt_len, const int32_t* draft_tokens,
                             const int32_t* row_len, const float* penalties, const float* bias, int64_t bias_stride,
                             const uint32_t* allowed, int64_t allowed_stride_b, int64_t allowed_stride_k,
                             float temperature, double* log2_norm, void* workspace, size_t workspace_bytes,
                             void* cuda_stream) {
    using namespace fef;
    using namespace fef::adj;
    if (dt != FEF_F32 && dt != FEF_BF16) return FEF_ERR_DTYPE;
    if (!logits || !out || !sizes_ok(B, K, V) || ld < V) return FEF_ERR_INVALID_ARG;
    if (L < 0 || L > (1 << 24) || (L > 0 && !tokens)) return FEF_ERR_INVALID_ARG;
    if (!(temperature >= 0.0f) || isinf(temperature)) return FEF_ERR_INVALID_ARG;
    if (bias && bias_stride != 0 && bias_stride < V) return FEF_ERR_INVALID_ARG;
    const int64_t words = (static_cast<int64_t>(V) + 31) / 32;
    if (allowed && ((allowed_stride_b != 0 && allowed_stride_b < words) || (allowed_stride_k != 0 && allowed_stride_k < words)))
        return FEF_ERR_INVALID_ARG;
    const int esize = dt == FEF_F32 ? 4 : 2;
    if ((reinterpret_cast<uintptr_t>(logits) & 15) || (reinterpret_cast<uintptr_t>(out) & 15) || ((ld * esize) & 15))
        return FEF_ERR_ALIGNMENT;
    for (const void* p : {static_cast<const void*>(tokens), static_cast<const void*>(prompt_len),
                          static_cast<const void*>(draft_tokens), static_cast<const void*>(row_len),
                          static_cast<const void*>(penalties), static_cast<const void*>(bias),
                          static_cast<const void*>(allowed)})
        if (reinterpret_cast<uintptr_t>(p) & 3) return FEF_ERR_ALIGNMENT;
    if (reinterpret_cast<uintptr_t>(log2_norm) & 7) return FEF_ERR_ALIGNMENT;
    const uintptr_t bytes = static_cast<uintptr_t>(B) * K * ld * esize;
    const uintptr_t from = reinterpret_cast<uintptr_t>(logits), to = reinterpret_cast<uintptr_t>(out);
    if (from != to && from < to + bytes && to < from + bytes) return FEF_ERR_INVALID_ARG;  // in place, or apart
    if (log2_norm && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) ||
                      workspace_bytes < fef_logits_adjust_workspace_bytes(B, K, V)))
        return FEF_ERR_WORKSPACE;

    Params P = {};
    const double c = 1.4426950408889634074 / (temperature == 0.0f ? 1.0 : static_cast<double>(temperature));
    P.c = static_cast<float>(c);
    P.c_law = dt == FEF_F32 ? c : static_cast<double>(P.c);
    P.norm_scale = c / P.c_law;
    if (!(P.c > 0.f) || isinf(P.c)) return FEF_ERR_INVALID_ARG;

    int dev = -1, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1)
        return FEF_ERR_CUDA;

    P.logits = static_cast<const char*>(logits);
    P.out = static_cast<char*>(out);
    P.ld_bytes = ld * esize;
    P.tokens = tokens;
    P.prompt_len = prompt_len;
    P.drafts = draft_tokens;
    P.row_len = row_len;
    P.penalties = penalties;
    P.bias = bias;
    P.bias_stride = bias_stride;
    P.allowed = allowed;
    P.allowed_stride_b = allowed_stride_b;
    P.allowed_stride_k = allowed_stride_k;
    P.L = L;
    P.B = B;
    P.K = K;
    P.V = V;
    P.chunks = chunks_of(V);
    P.partials = static_cast<float2*>(workspace);
    P.log2_norm = log2_norm;
    // A window's positions are shared out over CTAs only as far as the SMs need them (eight CTAs each): every CTA reads the text.
    int64_t splits = (static_cast<int64_t>(sms) * 8 + static_cast<int64_t>(P.chunks) * B - 1) / (static_cast<int64_t>(P.chunks) * B);
    const int most = (K + kRowsInFlight - 1) / kRowsInFlight;
    if (splits > most) splits = most;
    P.rows_per_cta = ((K + static_cast<int>(splits) - 1) / static_cast<int>(splits) + kRowsInFlight - 1) / kRowsInFlight * kRowsInFlight;
    splits = (K + P.rows_per_cta - 1) / P.rows_per_cta;

    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (dt == FEF_F32)
        launch<FEF_F32>(P, static_cast<int>(splits), log2_norm != nullptr, stream);
    else
        launch<FEF_BF16>(P, static_cast<int>(splits), log2_norm != nullptr, stream);
    if (cudaGetLastError() != cudaSuccess) return FEF_ERR_CUDA;
    if (log2_norm) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(static_cast<unsigned>((static_cast<int64_t>(B) * K + kWarps - 1) / kWarps));
        cfg.blockDim = dim3(kThreads);
        cfg.stream = stream;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        if (cudaLaunchKernelEx(&cfg, adjust_norm_kernel, P) != cudaSuccess) return FEF_ERR_CUDA;
    }
    return FEF_OK;
}

}  // extern "C"
