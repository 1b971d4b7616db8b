// fef_law_truncate, fef_draft_sample_truncated: the laws softmax(l / T) of speculative windows cut to their top-k, top-p
// and min-p sets, and one token of each cut law, drawn with one given random number per position.
//
// Entries of a row stand in one order: larger logit first, lower id among equal ones, -inf not at all.  With M the row's
// largest logit and w_x = 2^((l_x - M) log2(e) / T):
//   n_k  the first min(top_k, entries);  n_p  the shortest prefix of those whose weight is at least top_p of theirs;
//   n_m  the entries with w_x >= min_p;   the law keeps the first n = min(n_k, n_p, n_m).
//   cut = (logit, id) of the n-th entry,  log2_norm = M log2(e) / T + log2(sum of the kept weights),
//   token = the lowest id x for which the kept weights of ids <= x sum to more than u * (sum of the kept weights).
//
// Which entry a border falls on is decided by sums that differ by one entry's weight, 10^-6 of the whole and less, so weights
// are evaluated in double precision and summed as 64-bit integers (w 2^F, F = 62 - log2 V rounded down): such sums are exact,
// whatever the order in which threads add them.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "fef.h"
#include "fef_common.cuh"
#include "fef_device_math.cuh"

namespace fef {
namespace trunc {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kBins = 2048;
constexpr int kBinsPerThread = kBins / kThreads;
constexpr uint32_t kStreamDraft = 2u;   // the draft draws' Philox stream

struct Params {
    const char* logits;
    int64_t ld_bytes;
    const int32_t* row_len;     // [B] or null
    const int32_t* top_k;       // [B] or null
    const float* top_p;         // [B] or null
    const float* min_p;         // [B] or null
    int B, K, V;
    int vec_elems;              // entries of a row in whole 16-byte vectors
    double T, c;                // temperature and log2(e) / T
    double one;                 // 2^F: the weight 1
    const float* uniforms;      // [B, K], or null: Philox
    uint64_t seed;
    uint32_t step;
    const uint32_t* round;      // device word added to step, or null
    int32_t* tokens;            // null: no draws
    float* conf;
    double* log2_norm;
    float* cut_logit;
    int32_t* cut_id;
    int32_t* kept;
    int32_t* status;
};

struct Shared {
    unsigned long long mass[kBins];
    unsigned count[kBins];
    unsigned long long warp_mass[kWarps];
    unsigned warp_count[kWarps];
    double red[kWarps];
    unsigned long long found, lo, hi, above_mass;
    unsigned above_count, in_bin;
    int bad;
};

// Monotone map of a binary32 number that is no NaN to 32 bits, and back.
__device__ __forceinline__ uint32_t order_of(float l) {
    const uint32_t u = __float_as_uint(l + 0.f);   // (-0 becomes +0: the two are equal)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
// An entry's place in the order: the larger, the earlier.
__device__ __forceinline__ unsigned long long place_of(float l, int x) {
    return static_cast<unsigned long long>(order_of(l)) << 32 | (0xFFFFFFFFu - static_cast<uint32_t>(x));
}

struct Row {
    const char* base;
    int V, vec_elems;
    float top;            // largest logit
    double c, one;
    __device__ __forceinline__ unsigned long long weight(float l) const {
        return __double2ull_rn(exp2((static_cast<double>(l) - static_cast<double>(top)) * c) * one);
    }
};

// f(logit, id) for every entry of the row but -inf.
template <int DT, class F>
__device__ __forceinline__ void for_each(const Row& r, F f) {
    constexpr int N = Elem<DT>::kPerVec;
    for (int v = threadIdx.x; v < r.vec_elems / N; v += kThreads) {
        const uint4 w = ld_global_nc_v4(r.base + static_cast<int64_t>(v) * 16);
        float l[N];
        unpack<DT>(w, l);
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (l[i] != -INFINITY) f(l[i], v * N + i);
    }
    for (int x = r.vec_elems + threadIdx.x; x < r.V; x += kThreads) {
        const float l = load_logit<DT>(r.base, x);
        if (l != -INFINITY) f(l, x);
    }
}

__device__ __forceinline__ unsigned long long warp_sum_u64(unsigned long long v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// Sum over the CTA, in every thread.
__device__ unsigned long long block_sum(unsigned long long v, Shared& sh) {
    v = warp_sum_u64(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh.warp_mass[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0;
    for (int w = 0; w < kWarps; ++w) v += sh.warp_mass[w];
    return v;
}

// The first place, from the largest down, at which `enough(count, mass)` of the entries down to it holds; the places are
// those that each(f) hands to f(place, weight), all in [lo, hi], and all distinct.  `enough` is monotone and true for all of
// them together (otherwise the last place with an entry is returned).  Every level cuts the range into 2048 bins and goes on
// with the one the border is in.
template <class Each, class Enough>
__device__ unsigned long long select(Each each, Enough enough, unsigned long long lo, unsigned long long hi, Shared& sh) {
    unsigned long long above_mass = 0;
    unsigned above_count = 0;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (;;) {
        const int bits = 64 - __clzll(static_cast<long long>(hi - lo) | 1ll);
        const int shift = bits > 11 ? bits - 11 : 0;
        __syncthreads();
        for (int b = threadIdx.x; b < kBins; b += kThreads) {
            sh.mass[b] = 0;
            sh.count[b] = 0;
        }
        if (threadIdx.x == 0) sh.in_bin = 0;
        __syncthreads();
        each([&](unsigned long long place, auto&& weight) {
            if (place >= lo && place <= hi) {
                const int b = kBins - 1 - static_cast<int>((place - lo) >> shift);   // bin 0 is the largest
                atomicAdd(&sh.count[b], 1u);
                atomicAdd(&sh.mass[b], weight());
            }
        });
        __syncthreads();
        unsigned n[kBinsPerThread], ns = 0;
        unsigned long long m[kBinsPerThread], ms = 0;
#pragma unroll
        for (int j = 0; j < kBinsPerThread; ++j) {
            n[j] = sh.count[threadIdx.x * kBinsPerThread + j];
            m[j] = sh.mass[threadIdx.x * kBinsPerThread + j];
            ns += n[j];
            ms += m[j];
        }
        unsigned pn = ns;   // inclusive prefix over the warp, then what the warps before hold
        unsigned long long pm = ms;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned on = __shfl_up_sync(0xFFFFFFFFu, pn, o);
            const unsigned long long om = __shfl_up_sync(0xFFFFFFFFu, pm, o);
            if (lane >= o) {
                pn += on;
                pm += om;
            }
        }
        if (lane == 31) {
            sh.warp_count[warp] = pn;
            sh.warp_mass[warp] = pm;
        }
        __syncthreads();
        pn += above_count - ns;
        pm += above_mass - ms;
        unsigned all = above_count;
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) {
                pn += sh.warp_count[w];
                pm += sh.warp_mass[w];
            }
            all += sh.warp_count[w];
        }
#pragma unroll
        for (int j = 0; j < kBinsPerThread; ++j) {
            if (n[j]) {
                const bool before = pn > 0 && enough(pn, pm);
                const bool last = pn + n[j] == all;
                if (!before && (last || enough(pn + n[j], pm + m[j]))) {   // one bin of all
                    sh.above_count = pn;
                    sh.above_mass = pm;
                    sh.in_bin = n[j];
                    const unsigned long long from = lo + (static_cast<unsigned long long>(kBins - 1 - (threadIdx.x * kBinsPerThread + j)) << shift);
                    sh.lo = from;
                    const unsigned long long to = from + ((1ull << shift) - 1);
                    sh.hi = to < hi ? to : hi;
                }
            }
            pn += n[j];
            pm += m[j];
        }
        __syncthreads();
        lo = sh.lo;
        hi = sh.hi;
        above_count = sh.above_count;
        above_mass = sh.above_mass;
        if (shift == 0) return lo;
        if (sh.in_bin <= 1) {   // (0: there was no entry at all)
            each([&](unsigned long long place, auto&&) {
                if (place >= lo && place <= hi) sh.found = place;
            });
            __syncthreads();
            return sh.found;
        }
    }
}

// One row by the whole CTA, every step a pass over the row.
template <int DT>
__device__ void row_by_passes(const Params& P, int64_t at, int b, int i, Shared& sh) {
    Row r;
    r.base = P.logits + at * P.ld_bytes;
    r.V = P.V;
    r.vec_elems = P.vec_elems;
    r.c = P.c;
    r.one = P.one;

    float top = -INFINITY;
    int bad = 0;
    for_each<DT>(r, [&](float l, int) {
        bad |= !(l < INFINITY);
        top = fmaxf(top, l);
    });
    const int k = P.top_k ? __ldg(P.top_k + b) : 0;
    const float p = P.top_p ? __ldg(P.top_p + b) : 1.f, m = P.min_p ? __ldg(P.min_p + b) : 0.f;
    double u = 0.0;
    if (P.tokens) {
        if (P.uniforms) {
            u = __ldg(P.uniforms + at);
        } else {
            const uint4 w = philox4x32_10(make_uint4(kStreamDraft << 30, static_cast<uint32_t>(b), static_cast<uint32_t>(i),
                                                     P.step + (P.round ? __ldg(P.round) : 0u)),
                                          make_uint2(static_cast<uint32_t>(P.seed), static_cast<uint32_t>(P.seed >> 32)));
            u = uniform_from_word(w.x);
        }
    }
    bad |= p != p || m != m || u != u;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    __syncthreads();
    if (threadIdx.x == 0) sh.bad = 0;
    if ((threadIdx.x & 31) == 0) sh.red[threadIdx.x >> 5] = top;
    __syncthreads();
    if (bad) sh.bad = 1;
    for (int w = 0; w < kWarps; ++w) top = fmaxf(top, static_cast<float>(sh.red[w]));
    __syncthreads();
    if (sh.bad || top == -INFINITY) {
        if (threadIdx.x == 0) {
            const float nan = __int_as_float(0x7FC00000);
            P.log2_norm[at] = nan;
            P.cut_logit[at] = nan;
            P.cut_id[at] = -1;
            if (P.kept) P.kept[at] = 0;
            if (P.tokens) P.tokens[at] = -1;
            if (P.conf) P.conf[at] = -1.f;
            report(P.status, FEF_ERR_NONFINITE);
        }
        return;
    }
    r.top = top;

    auto places = [&](auto f) {
        for_each<DT>(r, [&](float l, int x) { f(place_of(l, x), [&] { return r.weight(l); }); });
    };
    const unsigned long long first = place_of(-3.402823466e38f, 0x7FFFFFFF), last = place_of(top, 0);
    const bool k_on = k > 0 && k < P.V, p_on = p < 1.f, m_on = m > 0.f;
    unsigned long long cut = 0;   // the smallest place in the law; 0: all of them
    if (k_on) {
        const unsigned most = static_cast<unsigned>(k);
        cut = select(places, [=](unsigned n, unsigned long long) { return n >= most; }, first, last, sh);
    }
    if (p_on) {
        unsigned long long sum = 0;
        for_each<DT>(r, [&](float l, int x) { sum += place_of(l, x) >= cut ? r.weight(l) : 0ull; });
        const double target = static_cast<double>(p) * static_cast<double>(block_sum(sum, sh));
        const unsigned long long cut_p =
            select(places, [=](unsigned, unsigned long long s) { return static_cast<double>(s) >= target; }, first, last, sh);
        cut = max(cut, cut_p);
    }
    if (m_on) {   // w >= m where l - M >= T ln m
        const double least = P.T * log(fmin(static_cast<double>(m), 1.0));
        unsigned long long lowest = ~0ull;
        for_each<DT>(r, [&](float l, int x) {
            if (static_cast<double>(l) - static_cast<double>(top) >= least) lowest = min(lowest, place_of(l, x));
        });
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) lowest = min(lowest, __shfl_xor_sync(0xFFFFFFFFu, lowest, o));
        __syncthreads();
        if ((threadIdx.x & 31) == 0) sh.warp_mass[threadIdx.x >> 5] = lowest;
        __syncthreads();
        for (int w = 0; w < kWarps; ++w) lowest = min(lowest, sh.warp_mass[w]);
        cut = max(cut, lowest);
    }
    unsigned long long sum = 0;
    unsigned n = 0;
    for_each<DT>(r, [&](float l, int x) {
        if (place_of(l, x) >= cut) {
            sum += r.weight(l);
            ++n;
        }
    });
    const unsigned long long total = block_sum(sum, sh);
    const unsigned kept = static_cast<unsigned>(block_sum(n, sh));
    if (threadIdx.x == 0) {
        P.log2_norm[at] = static_cast<double>(top) * P.c + log2(static_cast<double>(total) / P.one);
        P.cut_logit[at] = cut ? logit_of(static_cast<uint32_t>(cut >> 32)) : -INFINITY;
        P.cut_id[at] = cut ? static_cast<int>(0xFFFFFFFFu - static_cast<uint32_t>(cut)) : -1;
        if (P.kept) P.kept[at] = static_cast<int>(kept);
    }
    if (!P.tokens) return;
    const double target = fmin(fmax(u, 0.0), 1.0 - 0x1p-24) * static_cast<double>(total);
    auto by_id = [&](auto f) {
        for_each<DT>(r, [&](float l, int x) {
            if (place_of(l, x) >= cut) f(0xFFFFFFFFull - static_cast<unsigned>(x), [&] { return r.weight(l); });
        });
    };
    const unsigned long long drawn =
        select(by_id, [=](unsigned, unsigned long long s) { return static_cast<double>(s) > target; },
               0xFFFFFFFFull - static_cast<unsigned>(P.V - 1), 0xFFFFFFFFull, sh);
    if (threadIdx.x == 0) {
        const int x = static_cast<int>(0xFFFFFFFFull - drawn);
        P.tokens[at] = x;
        if (P.conf)
            P.conf[at] = static_cast<float>(exp2((static_cast<double>(load_logit<DT>(r.base, x)) - static_cast<double>(top)) * P.c) *
                                            (P.one / static_cast<double>(total)));
    }
}

template <int DT>
__global__ void __launch_bounds__(kThreads) truncate_kernel(const __grid_constant__ Params P) {
    __shared__ Shared sh;
    const int64_t rows = static_cast<int64_t>(P.B) * P.K;
    for (int64_t at = blockIdx.x; at < rows; at += gridDim.x) {
        const int b = static_cast<int>(at / P.K), i = static_cast<int>(at - static_cast<int64_t>(b) * P.K);
        if (P.row_len && i >= __ldg(P.row_len + b)) {
            if (threadIdx.x == 0) {
                P.log2_norm[at] = 0.0;
                P.cut_logit[at] = 0.f;
                P.cut_id[at] = -1;
                if (P.kept) P.kept[at] = 0;
                if (P.tokens) P.tokens[at] = -1;
                if (P.conf) P.conf[at] = -1.f;
            }
            continue;
        }
        row_by_passes<DT>(P, at, b, i, sh);
        __syncthreads();
    }
}

static fef_status truncate(const void* logits, const int32_t* row_len, int B, int K, int V, int64_t ld, fef_dtype dt,
                           float temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                           const float* uniforms, uint64_t seed, uint32_t step, const uint32_t* device_round, int32_t* tokens,
                           float* conf, double* log2_norm, float* cut_logit, int32_t* cut_id, int32_t* kept,
                           int32_t* device_status, void* cuda_stream) {
    if (dt != FEF_F32 && dt != FEF_BF16) return FEF_ERR_DTYPE;
    if (!logits || !log2_norm || !cut_logit || !cut_id) return FEF_ERR_INVALID_ARG;
    if (B < 1 || B > FEF_MAX_B || K < 1 || K > FEF_MAX_K || V < 1 || V > FEF_MAX_TRUNCATE_V || ld < V) return FEF_ERR_INVALID_ARG;
    if (!(temperature > 0.0f) || isinf(temperature)) return FEF_ERR_INVALID_ARG;
    const double c = 1.4426950408889634074 / static_cast<double>(temperature);
    if (isinf(static_cast<float>(c))) return FEF_ERR_INVALID_ARG;
    const int esize = dt == FEF_F32 ? 4 : 2;
    if ((reinterpret_cast<uintptr_t>(logits) & 15) || ((ld * esize) & 15)) return FEF_ERR_ALIGNMENT;
    for (const void* q : {static_cast<const void*>(row_len), static_cast<const void*>(top_k), static_cast<const void*>(top_p),
                          static_cast<const void*>(min_p), static_cast<const void*>(uniforms),
                          static_cast<const void*>(device_round), static_cast<const void*>(tokens), static_cast<const void*>(conf),
                          static_cast<const void*>(cut_logit), static_cast<const void*>(cut_id), static_cast<const void*>(kept),
                          static_cast<const void*>(device_status)})
        if (reinterpret_cast<uintptr_t>(q) & 3) return FEF_ERR_ALIGNMENT;
    if (reinterpret_cast<uintptr_t>(log2_norm) & 7) return FEF_ERR_ALIGNMENT;
    int dev = -1, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1)
        return FEF_ERR_CUDA;

    Params P = {};
    P.logits = static_cast<const char*>(logits);
    P.ld_bytes = ld * esize;
    P.row_len = row_len;
    P.top_k = top_k;
    P.top_p = top_p;
    P.min_p = min_p;
    P.B = B;
    P.K = K;
    P.V = V;
    P.vec_elems = static_cast<int>(static_cast<int64_t>(V) * esize / 16 * 16 / esize);
    P.T = temperature;
    P.c = c;
    int bits = 0;   // the weights of V entries, each at most 2^F, sum to at most 2^62
    while ((1 << bits) < V) ++bits;
    P.one = static_cast<double>(1ull << (62 - bits));
    P.uniforms = uniforms;
    P.seed = seed;
    P.step = step;
    P.round = device_round;
    P.tokens = tokens;
    P.conf = conf;
    P.log2_norm = log2_norm;
    P.cut_logit = cut_logit;
    P.cut_id = cut_id;
    P.kept = kept;
    P.status = device_status;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (device_status && cudaMemsetAsync(device_status, 0, sizeof(int32_t), stream) != cudaSuccess) return FEF_ERR_CUDA;
    const int64_t rows = static_cast<int64_t>(B) * K, most = static_cast<int64_t>(sms) * 4;
    const unsigned grid = static_cast<unsigned>(rows < most ? rows : most);
    if (dt == FEF_F32)
        truncate_kernel<FEF_F32><<<grid, kThreads, 0, stream>>>(P);
    else
        truncate_kernel<FEF_BF16><<<grid, kThreads, 0, stream>>>(P);
    return cudaGetLastError() == cudaSuccess ? FEF_OK : FEF_ERR_CUDA;
}

}  // namespace trunc
}  // namespace fef

extern "C" {

fef_status fef_law_truncate(const void* logits, const int32_t* row_len, int B, int K, int V, int64_t ld, fef_dtype dt,
                            float temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                            double* log2_norm, float* cut_logit, int32_t* cut_id, int32_t* kept, int32_t* device_status,
                            void* cuda_stream) {
    return fef::trunc::truncate(logits, row_len, B, K, V, ld, dt, temperature, top_k, top_p, min_p, nullptr, 0, 0, nullptr,
                                nullptr, nullptr, log2_norm, cut_logit, cut_id, kept, device_status, cuda_stream);
}

fef_status fef_draft_sample_truncated(const void* draft_logits, const int32_t* row_len, int B, int K, int V, int64_t ld,
                                      fef_dtype dt, float temperature, const int32_t* top_k, const float* top_p,
                                      const float* min_p, const float* uniforms, uint64_t seed, uint32_t step,
                                      const uint32_t* device_round, int32_t* draft_tokens, float* conf, double* log2_norm,
                                      float* cut_logit, int32_t* cut_id, int32_t* kept, int32_t* device_status,
                                      void* cuda_stream) {
    if (!draft_tokens) return FEF_ERR_INVALID_ARG;
    return fef::trunc::truncate(draft_logits, row_len, B, K, V, ld, dt, temperature, top_k, top_p, min_p, uniforms, seed, step,
                                device_round, draft_tokens, conf, log2_norm, cut_logit, cut_id, kept, device_status, cuda_stream);
}

}  // extern "C"
