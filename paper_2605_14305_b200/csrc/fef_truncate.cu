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
// are evaluated in double precision and summed as 64-bit integers (w 2^F, F = 62 - ceil(log2 V)): such sums are exact,
// whatever the order in which threads add them.
//
// A CTA has one row; memory bounds it from below (a row once, 259 MB and 40 us for 32 windows x 32 x 126464 bfloat16).  Three ways, each
// handing on what it cannot decide:
//   row_by_candidates  where the border is among few entries, as top-k's, min-p's and a steep law's top-p's are: a sample of the row tells a
//                      floor safely below the border, one pass notes down what is above it and only sums the rest, and the border and
//                      the draw are found among what was noted down.  One read of the row; bound by that and by the instructions of
//                      looking at every entry (64 windows x 32 x 126464 bfloat16, top-k 50: 118 us, with draws 133; 4.4 and 3.9 TB/s)
//   row_by_values      where it is among many (a flat law's top-p): the row is counted by value, then read once more (from memory: four
//                      rows to an SM are a little more than L2 holds).  Bound by the shared-memory atomics of the counting and, with
//                      draws, the weights of all entries before the border (flat rows of that size, top-p 0.9: 286 us, with draws 392;
//                      16 windows x 32 x 152064 binary32 237 and 248)
//   row_by_passes      whatever is left, and rows that are errors: some ten passes, 0.5 ms a row
// Candidates against counting every row: top-k 50 118 against 244 us, of 16 windows x 32 x 152064 binary32 62 against 128; counting
// against passes: 165 against 3850 us at 32 windows of flat bfloat16 rows.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "fef.h"
#include "fef_common.cuh"
#include "fef_device_math.cuh"

namespace fef {
namespace trunc {

// With more candidates the row is counted by value instead (64 windows x 32 x 126464 bfloat16, top-p 0.9 with draws: 227 us; with 1500
// in its place 270, 3000 239; 1 window x 32, top-p 0.95: 50, 55, 55).
constexpr float kManyCandidates = 4000.f;
constexpr int kMaxChunks = 252;    // stretches of a row whose kept weight is summed up for the draw
constexpr int kValueBins = 3842;   // of one sign: 30 binades of 128 bfloat16 numbers, what is below, what is above
constexpr int kRowBins = 2 * kValueBins;
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
    double one;                 // 2^F, the weight 1,
    int ones;                   // and F
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

struct Border {                      // an entry with its weight, what stands before it, and the weight of all
    unsigned long long place, mass, above_mass, all_mass;
    unsigned above_count;
};
// For selections: so much of all weights (and of `rest`, which is not among them).
struct Share {
    double p, rest, target;
    __device__ __forceinline__ void begin(unsigned long long all_mass) { target = p * (static_cast<double>(all_mass) + rest); }
    __device__ __forceinline__ bool operator()(unsigned, unsigned long long mass) const { return static_cast<double>(mass) >= target; }
};
template <class Enough>
__device__ __forceinline__ auto tell_all(Enough& enough, unsigned long long all_mass, int) -> decltype(enough.begin(all_mass)) {
    enough.begin(all_mass);
}
template <class Enough>
__device__ __forceinline__ void tell_all(Enough&, unsigned long long, long) {}

extern __shared__ __align__(16) unsigned char trunc_smem[];   // (begins with the table of 2^(i / 256))

// Monotone map of a binary32 number that is no NaN to 32 bits, and back.
__device__ __forceinline__ uint32_t order_of(float l) {
    const uint32_t u = __float_as_uint(l + 0.f);   // (-0 becomes +0: the two are equal)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
// An entry's place in the order: the larger, the earlier.  (bfloat16: the lower half of a logit's order says nothing.)
constexpr int kIdBits = 20;
constexpr uint32_t kIdMask = (1u << kIdBits) - 1u;
static_assert(FEF_MAX_TRUNCATE_V <= 1 << kIdBits, "ids fit");
template <int DT>
__device__ __forceinline__ unsigned long long place_of_order(uint32_t k, uint32_t x) {
    return static_cast<unsigned long long>(DT == FEF_F32 ? k : k >> 16) << kIdBits | (kIdMask - x);
}
template <int DT>
__device__ __forceinline__ unsigned long long place_of(float l, int x) {
    return place_of_order<DT>(order_of(l), static_cast<uint32_t>(x));
}
template <int DT>
__device__ __forceinline__ float logit_at(unsigned long long place) {
    const uint32_t k = static_cast<uint32_t>(place >> kIdBits);
    return logit_of(DT == FEF_F32 ? k : k & 0x8000u ? k << 16 : k << 16 | 0xFFFFu);
}
__device__ __forceinline__ int id_at(unsigned long long place) { return static_cast<int>(kIdMask - (static_cast<uint32_t>(place) & kIdMask)); }
// Ids as places: the lowest comes first.
__device__ __forceinline__ unsigned long long place_of_id(int x) { return kIdMask - static_cast<unsigned>(x); }

struct Row {
    const char* base;
    int V, vec_elems;
    float top;            // largest logit
    double c, one;
    double c256;          // 256 c,
    float c256_f;         // in binary32
    int ones;             // F: the weight 1 is 2^F
    // 2^((l - top) c) in units of 2^-F, as the product of two numbers: with y its exponent, 2^y = 2^(k / 256) 2^(f / 256), k a whole
    // number next to 256 y (from binary32), the first factor from a table, the second as its Taylor series (|f| < 0.51: the next term
    // is 1.5 10^-13).  For y > -900.  It takes seven operations in double precision, an addition of the product included: these set the
    // pace where every entry's weight is needed.
    __device__ __forceinline__ void factors(float l, double& a, double& b) const {
        constexpr double kRound = 6755399441055744.0;   // 1.5 * 2^52: whole numbers stand in the low bits
        constexpr double g = 0.6931471805599453094 / 256.0;
        const int k = __float2int_rn((l - top) * c256_f);
        const double f = fma(static_cast<double>(l) - static_cast<double>(top), c256, kRound - __hiloint2double(0x43380000 - (k < 0), k));
        double t = fma(f, g * g * g / 6.0, g * g / 2.0);
        t = fma(f, t, g);
        a = fma(f, t, 1.0);
        const double power = reinterpret_cast<const double*>(trunc_smem)[k & 255];
        b = __hiloint2double(__double2hiint(power) + (((k >> 8) + ones) << 20), __double2loint(power));
    }
    // The same, rounded to a whole number; 2^-1 and less is 0.
    __device__ __forceinline__ unsigned long long weight(float l) const {
        double a, b;
        factors(l, a, b);
        return (l - top) * c256_f >= -256.f * 64.f ? __double2ull_rn(a * b) : 0ull;   // (64 powers of two below: nothing, by far)
    }
};

__device__ __forceinline__ unsigned long long warp_sum_u64(unsigned long long v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

template <int DT>
__device__ constexpr float lowest_logit() {
    return DT == FEF_F32 ? -3.402823466e38f : -3.38953139e38f;
}

// Bits of the halves of a packed pair that are at least `from` (both halves of from2), all or none set.
__device__ __forceinline__ uint32_t at_least(uint32_t w, uint32_t from2) {
    uint32_t r;
    asm("set.ge.u32.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(w), "r"(from2));
    return r;
}

__device__ __forceinline__ uint32_t equal_to(uint32_t w, uint32_t from2) {
    uint32_t r;
    asm("set.eq.u32.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(w), "r"(from2));
    return r;
}
__device__ __forceinline__ uint32_t max_nan_two(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
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
__device__ __forceinline__ uint64_t fma_two(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// Bins in the order of the entries ("ranks") and what stands in them.
template <int DT>
struct Bins {
    static constexpr float kAbove = 16.f, kScale = 96.f;   // binary32: powers of two above the sampled largest, bins per power
    float c, anchor;   // binary32: c and the sampled largest logit
    uint32_t low;      // bfloat16: the magnitude (as bits) that bin 0 of a sign ends below

    __device__ __forceinline__ int of(float l) const {   // (binary32)
        return static_cast<int>(min(__float2uint_rz(fmaf(anchor - l, c, kAbove) * kScale), static_cast<unsigned>(kRowBins - 1)));
    }
    // bfloat16: table index of a rank and back to its number
    __device__ static __forceinline__ int at(int rank) { return DT == FEF_F32 ? rank : rank < kValueBins ? kValueBins - 1 - rank : rank; }
    __device__ __forceinline__ float value(int rank) const {
        if constexpr (DT == FEF_F32) {
            return anchor - ((static_cast<float>(rank) + 0.5f) / kScale - kAbove) / c;
        } else {
            const int m = rank < kValueBins ? kValueBins - 1 - rank : rank - kValueBins;   // magnitude
            const uint32_t bits = m == 0 ? 0u : (low - 1u + static_cast<uint32_t>(m)) << 16;
            return __uint_as_float(rank < kValueBins ? bits : bits | 0x80000000u);
        }
    }
};

// What a position asks for.
struct Limits {
    int k;
    float p, m;
    double u;
    bool k_on, p_on, m_on, bad;
    // w >= m where l - M >= this
    __device__ __forceinline__ double least(const Params& P) const { return P.T * log(fmin(static_cast<double>(m), 1.0)); }
};

__device__ __forceinline__ Limits limits_of(const Params& P, int64_t at, int b, int i) {
    Limits r;
    r.k = P.top_k ? __ldg(P.top_k + b) : 0;
    r.p = P.top_p ? __ldg(P.top_p + b) : 1.f;
    r.m = P.min_p ? __ldg(P.min_p + b) : 0.f;
    r.u = 0.0;
    if (P.tokens) {
        if (P.uniforms) {
            r.u = __ldg(P.uniforms + at);
        } else {
            const uint4 w = philox4x32_10(make_uint4(kStreamDraft << 30, static_cast<uint32_t>(b), static_cast<uint32_t>(i),
                                                     P.step + (P.round ? __ldg(P.round) : 0u)),
                                          make_uint2(static_cast<uint32_t>(P.seed), static_cast<uint32_t>(P.seed >> 32)));
            r.u = uniform_from_word(w.x);
        }
    }
    r.k_on = r.k > 0 && r.k < P.V;
    r.p_on = r.p < 1.f;
    r.m_on = r.m > 0.f;
    r.bad = r.p != r.p || r.m != r.m || r.u != r.u;
    r.u = fmin(fmax(r.u, 0.0), 1.0 - 0x1p-24);
    return r;
}

// A position without a law: behind its window's end, or (error) one whose row or limits are no numbers.
__device__ __forceinline__ void write_none(const Params& P, int64_t at, bool error) {
    const float nan = __int_as_float(0x7FC00000);
    P.log2_norm[at] = error ? nan : 0.0;
    P.cut_logit[at] = error ? nan : 0.f;
    P.cut_id[at] = -1;
    if (P.kept) P.kept[at] = 0;
    if (P.tokens) P.tokens[at] = -1;
    if (P.conf) P.conf[at] = -1.f;
    if (error) report(P.status, FEF_ERR_NONFINITE);
}

// The law is known: its smallest place (0: nothing is cut), its weight and its entries.
template <int DT>
__device__ __forceinline__ void write_law(const Params& P, int64_t at, const Row& r, unsigned long long cut,
                                          unsigned long long total, unsigned kept) {
    P.log2_norm[at] = static_cast<double>(r.top) * P.c + log2(static_cast<double>(total) / P.one);
    P.cut_logit[at] = cut ? logit_at<DT>(cut) : -INFINITY;
    P.cut_id[at] = cut ? id_at(cut) : -1;
    if (P.kept) P.kept[at] = static_cast<int>(kept);
}

template <int DT>
__device__ __forceinline__ void write_token(const Params& P, int64_t at, const Row& r, unsigned long long total, int x) {
    P.tokens[at] = x;
    if (P.conf)
        P.conf[at] = static_cast<float>(exp2((static_cast<double>(load_logit<DT>(r.base, x)) - static_cast<double>(r.top)) * P.c) *
                                        (P.one / static_cast<double>(total)));
}

// One row by a CTA of kThreads threads.
template <int kThreads>
struct Rows {
    static constexpr int kWarps = kThreads / 32;
    static constexpr int kBins = kThreads > 512 ? kThreads : 512;   // of a selection
    static constexpr int kBinsLog2 = kThreads > 512 ? 10 : 9;
    static constexpr int kBinsPerThread = kBins / kThreads;
    static constexpr int kSampleBins = 1024;
    static constexpr int kSampleBinsPerThread = kSampleBins / kThreads;
    static constexpr int kSampleOctaveLog2 = 7;   // bins per octave of the distance below the sample's largest
    static constexpr int kSample = 16 * kThreads; // entries a row's sample holds
    static constexpr int kAll = 16 * kThreads;    // rows of so many entries are noted down whole
    static constexpr int kWarpList = kAll / kWarps + 32;   // candidates a warp can note down (its share of such a row, and of the row's end)
    static constexpr int kList = kWarps * kWarpList;
    static constexpr int kRowBinsPerThread = (kRowBins + kThreads - 1) / kThreads;
    // So few candidates are all compared with one another, kFewShare threads to each; the work grows with the square.
    static constexpr int kFew = kThreads / 2 < 256 ? kThreads / 2 : 256;
    static constexpr int kFewShare = kThreads / kFew;
    static_assert(kRowBins * 4 <= kList * 8, "the bins fit where the candidates are later");
    static_assert(kMaxChunks < kThreads, "a thread for each stretch");

    struct Shared {
        double table[256];               // 2^(i / 256)
        union {
            struct {                     // a selection
                unsigned long long mass[kBins];
                unsigned count[kBins];
            };
            unsigned sample[kSampleBins];
            struct {                         // few candidates
                ulonglong2 loose[kFew];      // place and weight, as they come; later by rank, with the id in the place's stead
                unsigned long long ranked[kFew], upto[kFew];   // by rank: place, weight of all down to it
            };
        };
        union {
            struct {
                uint32_t id[kList];      // candidates: warp w's at w * kWarpList
                uint32_t key[kList];     // their logits' order
            };
            unsigned bin[kRowBins];      // entries by value, until the candidates are noted down
        };
        unsigned listed[kWarps];
        unsigned long long chunk[kMaxChunks + 1];
        unsigned long long warp_mass[kWarps];
        unsigned warp_count[kWarps];
        float red_f[kWarps][2];
        double red[kWarps];
        unsigned long long few_place[32], few_weight[32];   // a bin with few entries
        unsigned few;
        unsigned long long lo, hi, above_mass;
        unsigned above_count, in_bin;
        Border border;
        float from;                      // candidates are the logits from here on
        int bad;
        int loc_rank;                    // a border among the bins: its bin, what stands before it
        unsigned loc_n;
        unsigned long long loc_m;
    };

    // f(logit, id) for every entry of the row but -inf.
    template <int DT, class F>
    static __device__ __forceinline__ void for_each(const Row& r, F f) {
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

    // Sum over the CTA, in every thread.
    static __device__ unsigned long long block_sum(unsigned long long v, Shared& sh) {
        v = warp_sum_u64(v);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) sh.warp_mass[threadIdx.x >> 5] = v;
        __syncthreads();
        v = 0;
        for (int w = 0; w < kWarps; ++w) v += sh.warp_mass[w];
        return v;
    }

    static __device__ unsigned long long block_min(unsigned long long v, Shared& sh) {
    #pragma unroll
        for (int o = 16; o > 0; o >>= 1) v = min(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
        __syncthreads();
        if ((threadIdx.x & 31) == 0) sh.warp_mass[threadIdx.x >> 5] = v;
        __syncthreads();
        for (int w = 0; w < kWarps; ++w) v = min(v, sh.warp_mass[w]);
        return v;
    }

    // The first place, from the largest down, at which `enough(count, mass)` of the entries down to it holds; the places are
    // those that each(f) hands to f(place, weight), all in [lo, hi], and all distinct.  `enough` is monotone; where it does not hold
    // for all of them together, the last place is returned.  Every level cuts the range into 512 bins and goes on with the one
    // the border is in; one with at most 32 entries is settled by a warp.
    // above_count, above_mass: what stands before all of them.  `enough` is told their weight first, if it asks for it.
    template <class Each, class Enough>
    static __device__ Border select(Each each, Enough enough, unsigned long long lo, unsigned long long hi, Shared& sh, unsigned above_count = 0,
                             unsigned long long above_mass = 0) {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        unsigned long long all_mass = 0;
        for (bool first = true;; first = false) {
            const int bits = 64 - __clzll(static_cast<long long>(hi - lo) | 1ll);
            const int shift = bits > kBinsLog2 ? bits - kBinsLog2 : 0;
            __syncthreads();
            for (int b = threadIdx.x; b < kBins; b += kThreads) {
                sh.mass[b] = 0;
                sh.count[b] = 0;
            }
            if (threadIdx.x == 0) sh.few = 0;
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
            unsigned long long here = 0;
    #pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const unsigned wn = sh.warp_count[w];
                const unsigned long long wm = sh.warp_mass[w];
                if (w < warp) {
                    pn += wn;
                    pm += wm;
                }
                all += wn;
                here += wm;
            }
            if (first) {
                all_mass = here;
                tell_all(enough, all_mass, 0);
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
                        const unsigned long long from =
                            lo + (static_cast<unsigned long long>(kBins - 1 - (threadIdx.x * kBinsPerThread + j)) << shift);
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
            if (sh.in_bin <= 32) {
                each([&](unsigned long long place, auto&& weight) {
                    if (place >= lo && place <= hi) {
                        const unsigned at = atomicAdd(&sh.few, 1u);
                        sh.few_place[at] = place;
                        sh.few_weight[at] = weight();
                    }
                });
                __syncthreads();
                if (warp == 0) {
                    const int have = static_cast<int>(sh.few);
                    const unsigned long long mine = lane < have ? sh.few_place[lane] : 0ull;
                    unsigned c = above_count;
                    unsigned long long s = above_mass;
                    for (int j = 0; j < have; ++j)
                        if (sh.few_place[j] > mine) {
                            ++c;
                            s += sh.few_weight[j];
                        }
                    const bool before = c > 0 && enough(c, s);
                    if (lane < have && !before && (c + 1 == above_count + have || enough(c + 1, s + sh.few_weight[lane]))) {
                        sh.border.place = mine;
                        sh.border.mass = sh.few_weight[lane];
                        sh.border.all_mass = all_mass;
                        sh.border.above_mass = s;
                        sh.border.above_count = c;
                    }
                }
                __syncthreads();
                return sh.border;
            }
        }
    }

    // ------------------------------------------------------------------ passes over the row ----
    // One row by the whole CTA, every step a pass over the row: right for every row, and slow.
    template <int DT>
    static __device__ void row_by_passes(const Params& P, int64_t at, const Limits& lim, Row& r, Shared& sh) {
        float top = -INFINITY;
        int bad = lim.bad;
        for_each<DT>(r, [&](float l, int) {
            bad |= !(l < INFINITY);
            top = fmaxf(top, l);
        });
    #pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        __syncthreads();
        if (threadIdx.x == 0) sh.bad = 0;
        if ((threadIdx.x & 31) == 0) sh.red_f[threadIdx.x >> 5][0] = top;
        __syncthreads();
        if (bad) sh.bad = 1;
        for (int w = 0; w < kWarps; ++w) top = fmaxf(top, sh.red_f[w][0]);
        __syncthreads();
        if (sh.bad || top == -INFINITY) {
            if (threadIdx.x == 0) write_none(P, at, true);
            return;
        }
        r.top = top;

        auto places = [&](auto f) {
            for_each<DT>(r, [&](float l, int x) { f(place_of<DT>(l, x), [&] { return r.weight(l); }); });
        };
        const unsigned long long first = place_of<DT>(lowest_logit<DT>(), P.V - 1), last = place_of<DT>(top, 0);
        unsigned long long cut = 0;   // the smallest place in the law; 0: all of them
        if (lim.k_on) {
            const unsigned most = static_cast<unsigned>(lim.k);
            cut = select(places, [=](unsigned n, unsigned long long) { return n >= most; }, first, last, sh).place;
        }
        if (lim.p_on) {
            unsigned long long sum = 0;
            for_each<DT>(r, [&](float l, int x) { sum += place_of<DT>(l, x) >= cut ? r.weight(l) : 0ull; });
            const double target = static_cast<double>(lim.p) * static_cast<double>(block_sum(sum, sh));
            cut = max(cut, select(places, [=](unsigned, unsigned long long s) { return static_cast<double>(s) >= target; }, first, last,
                                  sh).place);
        }
        if (lim.m_on) {
            const double least = lim.least(P);
            unsigned long long lowest = ~0ull;
            for_each<DT>(r, [&](float l, int x) {
                if (static_cast<double>(l) - static_cast<double>(top) >= least) lowest = min(lowest, place_of<DT>(l, x));
            });
            cut = max(cut, block_min(lowest, sh));
        }
        unsigned long long sum = 0;
        unsigned n = 0;
        for_each<DT>(r, [&](float l, int x) {
            if (place_of<DT>(l, x) >= cut) {
                sum += r.weight(l);
                ++n;
            }
        });
        const unsigned long long total = block_sum(sum, sh);
        const unsigned kept = static_cast<unsigned>(block_sum(n, sh));
        if (threadIdx.x == 0) write_law<DT>(P, at, r, cut, total, kept);
        if (!P.tokens) return;
        const double target = lim.u * static_cast<double>(total);
        auto by_id = [&](auto f) {
            for_each<DT>(r, [&](float l, int x) {
                if (place_of<DT>(l, x) >= cut) f(place_of_id(x), [&] { return r.weight(l); });
            });
        };
        const unsigned long long drawn = select(by_id, [=](unsigned, unsigned long long s) { return static_cast<double>(s) > target; },
                                                place_of_id(P.V - 1), place_of_id(0), sh).place;
        if (threadIdx.x == 0) write_token<DT>(P, at, r, total, id_at(drawn));
    }

    // ---------------------------------------------------------------------- candidates ----
    // One pass over the row.  A sample of it says from which logit on the entries are noted down ("candidates") so that the law's
    // border is among them; the rest is only summed, in binary32, where top_p needs the whole row's weight.  What the sample says is
    // a guess and is checked afterwards: the candidates are the row's first entries in any case, so a border among them is the
    // border, provided that their exact weight and the rest's, whatever its rounding, put it there.

    // From which logit on?  False: no rule, or more candidates than there is room for.
    template <int DT>
    static __device__ bool candidates_from(const Params& P, const Row& r, const Limits& lim, Shared& sh, float& ref_logit) {
        constexpr int N = Elem<DT>::kPerVec;
        constexpr int kPerWarp = kSample / (kWarps * 32 * N);   // vectors of a lane
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        constexpr float lowest = lowest_logit<DT>();
        ref_logit = 0.f;
        if (r.V <= kAll) {   // room for all
            if (threadIdx.x == 0) sh.from = lowest;
            return true;
        }
        if (!lim.k_on && !lim.p_on && !lim.m_on) return false;
        const int chunks = r.vec_elems / (32 * N);   // of 512 bytes; V > kAll = kSample: there are as many as the sample takes
        float x[kPerWarp * N], top = -INFINITY;
    #pragma unroll
        for (int j = 0; j < kPerWarp; ++j) {
            const int s = warp * kPerWarp + j;
            const int chunk = static_cast<int>((static_cast<int64_t>(2 * s + 1) * chunks) / (2 * kPerWarp * kWarps));
            unpack<DT>(ld_global_nc_v4(r.base + (static_cast<int64_t>(chunk) * 32 + lane) * 16), *reinterpret_cast<float(*)[N]>(x + j * N));
        }
    #pragma unroll
        for (int j = 0; j < kPerWarp * N; ++j) top = fmaxf(top, x[j]);
    #pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        if (lane == 0) sh.red_f[warp][0] = top;
        for (int b = threadIdx.x; b < kSampleBins; b += kThreads) sh.sample[b] = 0;
        if (threadIdx.x == 0) {
            sh.from = lowest;
            sh.few = 0;   // candidates in the sample
        }
        __syncthreads();
    #pragma unroll
        for (int w = 0; w < kWarps; ++w) top = fmaxf(top, sh.red_f[w][0]);
        __syncthreads();
        if (top == -INFINITY) return true;   // (nothing but masked entries seen: those that are left may be few)
        if (!(top < INFINITY)) return false;
        ref_logit = top;
        // distance below the largest sampled logit, in powers of two of the weight; 128 bins per octave of (distance + 1)
        const float c = static_cast<float>(P.c);
    #pragma unroll
        for (int j = 0; j < kPerWarp * N; ++j)
            if (x[j] > -INFINITY)
                atomicAdd(&sh.sample[min((__float_as_uint(fmaf(top - x[j], c, 1.f)) - 0x3F800000u) >> (23 - kSampleOctaveLog2), kSampleBins - 1u)], 1u);
        __syncthreads();
        auto edge = [](int b) { return __uint_as_float(0x3F800000u + (static_cast<unsigned>(b) << (23 - kSampleOctaveLog2))) - 1.f; };
        unsigned n[kSampleBinsPerThread], cn = 0;
        float w[kSampleBinsPerThread], cw = 0.f;
        const int b0 = threadIdx.x * kSampleBinsPerThread;
    #pragma unroll
        for (int j = 0; j < kSampleBinsPerThread; ++j) {
            n[j] = sh.sample[b0 + j];
            w[j] = static_cast<float>(n[j]) * ex2_approx(-0.5f * (edge(b0 + j) + edge(b0 + j + 1)));
            cn += n[j];
            cw += w[j];
        }
        unsigned pn = cn;
        float pw = cw;
    #pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned on = __shfl_up_sync(0xFFFFFFFFu, pn, o);
            const float ow = __shfl_up_sync(0xFFFFFFFFu, pw, o);
            if (lane >= o) {
                pn += on;
                pw += ow;
            }
        }
        if (lane == 31) {
            sh.warp_count[warp] = pn;
            sh.red_f[warp][1] = pw;
        }
        __syncthreads();
        pn -= cn;
        pw -= cw;
        float all = 0.f;
    #pragma unroll
        for (int v = 0; v < kWarps; ++v) {
            if (v < warp) {
                pn += sh.warp_count[v];
                pw += sh.red_f[v][1];
            }
            all += sh.red_f[v][1];
        }
        const float share = static_cast<float>(kSample) / static_cast<float>(r.V);
        int bin = -1;   // the candidates go down to this bin's end
        if (lim.k_on) {   // as many in the sample as the first k have there five standard deviations above the mean
            const float mean = static_cast<float>(lim.k) * share;
            const unsigned need = static_cast<unsigned>(mean + 5.f * sqrtf(mean) + 5.f);
            unsigned at = pn;
    #pragma unroll
            for (int j = 0; j < kSampleBinsPerThread; ++j) {
                if (at < need && at + n[j] >= need) bin = b0 + j;
                at += n[j];
            }
        } else if (lim.p_on) {
            // The row's weight, rather too low than too high: the sample's largest four count as themselves, the others for their share.
            float single = 0.f;
            unsigned at = pn;
    #pragma unroll
            for (int j = 0; j < kSampleBinsPerThread; ++j) {
                at += n[j];
                if (at <= 4) single += w[j];
            }
    #pragma unroll
            for (int o = 16; o > 0; o >>= 1) single += __shfl_xor_sync(0xFFFFFFFFu, single, o);
            if (lane == 0) sh.red_f[warp][0] = single;
            __syncthreads();
            single = 0.f;
    #pragma unroll
            for (int v = 0; v < kWarps; ++v) single += sh.red_f[v][0];
            const float whole = single + (all - single) / share;
            const float may_miss = (1.f - fmaxf(lim.p, 0.f)) * whole * share * 0.85f;   // what the sample may hold below the border
            float below = all - pw;
    #pragma unroll
            for (int j = 0; j < kSampleBinsPerThread; ++j) {
                const float next = below - w[j];
                if (n[j] && below > may_miss && next <= may_miss) bin = b0 + j;
                below = next;
            }
        }
        if (bin >= 0 && bin < kSampleBins - 1) {   // (one thread, give or take the sums' rounding)
            sh.from = top - edge(bin + 1) / c;
            unsigned at = pn;
    #pragma unroll
            for (int j = 0; j < kSampleBinsPerThread; ++j)
                if (b0 + j <= bin) at += n[j];
            sh.few = at;
        }
        __syncthreads();
        float from = fmaxf(sh.from, lowest);
        if (lim.m_on && !(lim.k_on && lim.p_on)) {   // (top_p of the first k needs all of them)
            from = fmaxf(from, __double2float_rd(fmax(static_cast<double>(top) + lim.least(P), static_cast<double>(lowest))));
            unsigned few = 0;
    #pragma unroll
            for (int j = 0; j < kPerWarp * N; ++j) few += x[j] >= from;
            few = __reduce_add_sync(0xFFFFFFFFu, few);
            if (lane == 0) sh.warp_count[warp] = few;
            __syncthreads();
            few = 0;
    #pragma unroll
            for (int v = 0; v < kWarps; ++v) few += sh.warp_count[v];
            if (threadIdx.x == 0) sh.few = few;
            __syncthreads();
        }
        const bool many = static_cast<float>(sh.few) > share * fminf(0.8f * kList, kManyCandidates);
        if (DT == FEF_BF16) {   // rounded down
            uint32_t bits = __float_as_uint(from);
            if (bits & 0x80000000u) bits += 0xFFFFu;
            from = fmaxf(__uint_as_float(bits & 0xFFFF0000u), lowest);
        }
        __syncthreads();
        if (threadIdx.x == 0) sh.from = from;
        return !many;
    }

    // The pass: ids of the entries from `from` on into the warps' lists, and with SUM the others' sum of 2^(l c - ref).
    // NaN anywhere makes the sum NaN (without SUM it is looked for).  Returns the thread's sum.
    // EQUAL: the entries equal to `from` only.
    template <int DT, bool SUM, bool EQUAL = false>
    static __device__ float note_candidates(const Row& r, float from, float c, float ref, Shared& sh) {
        constexpr int N = Elem<DT>::kPerVec;
        constexpr int kBatch = 4;
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        const unsigned before = (1u << lane) - 1u;
        uint32_t* list = sh.id + warp * kWarpList;
        unsigned listed = 0;
        uint64_t sum[2] = {0u, 0u};       // two binary32 sums each
        uint32_t seen[2] = {0u, 0u};      // (bfloat16) the largest so far, NaN where there was one
        bool nan = false;
        const uint32_t from2 = __float_as_uint(from) | __float_as_uint(from) >> 16;
        const uint64_t c2 = two(c, c), ref2 = two(-ref, -ref);
        const int chunks = r.vec_elems / (32 * N);
        constexpr uint32_t kMinusInf = DT == FEF_F32 ? 0xFF800000u : 0xFF80FF80u;

        auto note = [&](bool hit, int x) {
            const unsigned hits = __ballot_sync(0xFFFFFFFFu, hit);
            const unsigned at = listed + __popc(hits & before);
            if (hit && at < kWarpList) list[at] = static_cast<uint32_t>(x);
            listed += __popc(hits);
        };
        auto fetch = [&](int chunk, uint4 (&w)[kBatch]) {
    #pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                const int at = chunk + j * kWarps;
                w[j] = make_uint4(kMinusInf, kMinusInf, kMinusInf, kMinusInf);
                if (at < chunks) w[j] = ld_global_nc_v4(r.base + (static_cast<int64_t>(at) * 32 + lane) * 16);
            }
        };
        uint4 w[kBatch], next[kBatch];
        fetch(warp, w);
    #pragma unroll 1
        for (int chunk = warp; chunk < chunks; chunk += kBatch * kWarps) {
            fetch(chunk + kBatch * kWarps, next);
            uint32_t mask = 0;
    #pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                uint32_t v[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
                if constexpr (DT == FEF_BF16) {
    #pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const uint32_t hit = EQUAL ? equal_to(v[q], from2) : at_least(v[q], from2);
                        mask |= hit & (0x00010001u << (4 * j + q));
                        if constexpr (SUM) {
                            v[q] = (v[q] & ~hit) | (0xFF80FF80u & hit);
                            const uint64_t x = fma_two(static_cast<uint64_t>(v[q] & 0xFFFF0000u) << 32 | v[q] << 16, c2, ref2);
                            sum[q & 1] = add_two(sum[q & 1], two(ex2_approx(first_of(x)), ex2_approx(second_of(x))));
                        } else {
                            seen[q & 1] = max_nan_two(seen[q & 1], v[q]);
                        }
                    }
                } else {
    #pragma unroll
                    for (int q = 0; q < 4; q += 2) {
                        const float a = __uint_as_float(v[q]), b = __uint_as_float(v[q + 1]);
                        const bool hit_a = EQUAL ? a == from : a >= from, hit_b = EQUAL ? b == from : b >= from;
                        mask |= (hit_a ? 1u << (4 * j + q) : 0u) | (hit_b ? 2u << (4 * j + q) : 0u);
                        if constexpr (SUM) {
                            const uint64_t x = fma_two(two(hit_a ? -INFINITY : a, hit_b ? -INFINITY : b), c2, ref2);
                            sum[q >> 1] = add_two(sum[q >> 1], two(ex2_approx(first_of(x)), ex2_approx(second_of(x))));
                        } else {
                            nan |= a != a || b != b;
                        }
                    }
                }
            }
            while (__any_sync(0xFFFFFFFFu, mask != 0u)) {
                const int bit = __ffs(mask) - 1;
                int x;
                if constexpr (DT == FEF_BF16)   // bit 16 h + 4 j + q: half h of word q of vector j
                    x = ((chunk + ((bit >> 2) & 3) * kWarps) * 32 + lane) * N + (bit & 3) * 2 + (bit >> 4);
                else
                    x = ((chunk + (bit >> 2) * kWarps) * 32 + lane) * N + (bit & 3);
                note(mask != 0u, x);
                mask &= mask - 1u;
            }
    #pragma unroll
            for (int j = 0; j < kBatch; ++j) w[j] = next[j];
        }
        for (int x0 = chunks * 32 * N + warp * 32; x0 < r.V; x0 += kThreads) {   // what is behind the last whole chunk
            const int x = x0 + lane;
            const float a = x < r.V ? load_logit<DT>(r.base, x) : -INFINITY;
            const bool hit = EQUAL ? a == from : a >= from;
            note(hit, x);
            if constexpr (SUM)
                sum[0] = add_two(sum[0], two(ex2_approx(fmaf(hit ? -INFINITY : a, c, -ref)), 0.f));
            else
                nan |= a != a;
        }
        if (lane == 0) sh.listed[warp] = listed;
        if constexpr (SUM) return (first_of(sum[0]) + second_of(sum[0])) + (first_of(sum[1]) + second_of(sum[1]));
        if constexpr (DT == FEF_BF16) {
            const uint32_t all = max_nan_two(seen[0], seen[1]);
            nan |= (all & 0x7FFFu) > 0x7F80u || (all >> 16 & 0x7FFFu) > 0x7F80u;
        }
        return nan ? __int_as_float(0x7FC00000) : 0.f;
    }

    // Few candidates: each one's rank and the weight down to it, by comparing it with all; every rule then is a number of ranks.  False:
    // the rest's weight is too near to call, or the border is not among them (nothing has been written).
    template <int DT>
    static __device__ __forceinline__ bool row_of_few(const Params& P, int64_t at, const Limits& lim, const Row& r, Shared& sh, int n, float from,
                                                      double rest, double slack) {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        const int mine = threadIdx.x / kFewShare, part = threadIdx.x % kFewShare;
        const unsigned listed = sh.listed[warp];
        const unsigned before = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? sh.listed[lane] : 0u);
        for (unsigned j = lane; j < listed; j += 32) {
            const uint32_t key = sh.key[warp * kWarpList + j];
            sh.loose[before + j] = make_ulonglong2(place_of_order<DT>(key, sh.id[warp * kWarpList + j]), r.weight(logit_of(key)));
        }
        __syncthreads();
        // the sum of those that `precede` own, over all of the first `count`
        auto sum_over = [&](int count, unsigned long long own, unsigned& rank) {
            unsigned long long sum = 0;
            rank = 0;
            if (mine < count)
                for (int j = part; j < count; j += kFewShare) {
                    const ulonglong2 o = sh.loose[j];
                    if (o.x > own) {
                        ++rank;
                        sum += o.y;
                    }
                }
    #pragma unroll
            for (int o = 1; o < kFewShare; o <<= 1) {
                rank += __shfl_xor_sync(0xFFFFFFFFu, rank, o);
                sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
            }
            return sum;
        };
        ulonglong2 own = make_ulonglong2(0ull, 0ull);
        if (mine < n) own = sh.loose[mine];
        unsigned rank;
        const unsigned long long above = sum_over(n, own.x, rank);
        const bool writes = mine < n && part == 0;
        if (writes) {
            sh.ranked[rank] = own.x;
            sh.upto[rank] = above + own.y;
        }
        __syncthreads();
        if (writes) sh.loose[rank] = make_ulonglong2(own.x & kIdMask, own.y);
        const bool everything = from == lowest_logit<DT>();
        const int t = threadIdx.x;
        int kept = n + 1;   // entries down to the border (n + 1: not known)
        if (lim.k_on) {
            if (n < lim.k && !everything) {
                if (lim.p_on || !lim.m_on) return false;
            } else {
                kept = min(lim.k, n);
            }
        }
        if (lim.p_on) {
            const double p = lim.p, sum = static_cast<double>(sh.upto[(lim.k_on ? kept : n) - 1]);
            const double target = p * (sum + rest), least = p * (sum + rest * (1.0 - slack));
            if (sum < least) {   // beyond the candidates
                if (!lim.m_on) return false;
            } else {
                const int n_p = __syncthreads_count(t < n && !(static_cast<double>(sh.upto[t]) >= target)) + 1;
                if (n_p > n) return false;
                const double most_of_it = p * (sum + rest * (1.0 + slack) + slack * 0x1p-20 * P.one);
                if (rest > 0.0 && !(static_cast<double>(sh.upto[n_p - 1]) >= most_of_it && (n_p == 1 || static_cast<double>(sh.upto[n_p - 2]) < least)))
                    return false;
                kept = min(kept, n_p);
            }
        }
        if (lim.m_on) {
            const double least = lim.least(P);
            const int n_m = __syncthreads_count(
                t < n && static_cast<double>(logit_at<DT>(sh.ranked[t < n ? t : 0])) - static_cast<double>(r.top) >= least);
            // (as below: with entries beyond the candidates in the set it is no border)
            if (everything || static_cast<double>(from) - static_cast<double>(r.top) <= least) kept = min(kept, n_m);
        }
        if (kept > n && !everything) return false;
        const unsigned long long cut = kept > n ? 0ull : sh.ranked[kept - 1];
        kept = min(kept, n);
        const unsigned long long total = sh.upto[kept - 1];
        if (threadIdx.x == 0) write_law<DT>(P, at, r, cut, total, static_cast<unsigned>(kept));
        if (!P.tokens) return true;
        // The draw: the same by the ids.
        __syncthreads();
        const double target = lim.u * static_cast<double>(total);
        if (mine < kept) own = sh.loose[mine];
        const unsigned long long lower = sum_over(kept, own.x, rank);
        if (mine < kept && part == 0 && static_cast<double>(lower + own.y) > target && !(static_cast<double>(lower) > target))
            write_token<DT>(P, at, r, total, id_at(own.x));   // one thread
        return true;
    }

    // The thread's share of the weight of the entries below `from`.  (Four loads at a time, and no rounding to whole numbers before the
    // thread's sum: a call of 1 window x 32 with such a row: 62 us when the passes did this, 53 now.)
    template <int DT>
    static __device__ __noinline__ double sum_below(const Row r, float from) {
        constexpr int N = Elem<DT>::kPerVec;
        constexpr int kBatch = 4;
        const int vectors = r.vec_elems / N;
        const float weightless = r.top - 64.f / static_cast<float>(r.c);
        double sum = 0.0;
        auto add = [&](float l) {
            double a, b;
            r.factors(l, a, b);
            if (l < from && l >= weightless) sum = fma(a, b, sum);
        };
    #pragma unroll 1
        for (int v = threadIdx.x; v < vectors; v += kBatch * kThreads) {
            uint4 w[kBatch];
    #pragma unroll
            for (int j = 0; j < kBatch; ++j)
                if (v + j * kThreads < vectors) w[j] = ld_global_nc_v4(r.base + static_cast<int64_t>(v + j * kThreads) * 16);
    #pragma unroll
            for (int j = 0; j < kBatch; ++j)
                if (v + j * kThreads < vectors) {
                    float l[N];
                    unpack<DT>(w[j], l);
    #pragma unroll
                    for (int i = 0; i < N; ++i) add(l[i]);
                }
        }
        for (int x = r.vec_elems + threadIdx.x; x < r.V; x += kThreads) add(load_logit<DT>(r.base, x));
        return sum;
    }

    // False: the row needs the other path (nothing has been written).
    template <int DT>
    static __device__ bool row_by_candidates(const Params& P, int64_t at, const Limits& lim, Row& r, Shared& sh) {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        float ref_logit;
        if (!candidates_from<DT>(P, r, lim, sh, ref_logit)) return false;
        __syncthreads();
        const float from = sh.from, c = static_cast<float>(P.c), ref = ref_logit * c;
        const bool with_sum = lim.p_on && !lim.k_on;
        const float mine = with_sum ? note_candidates<DT, true>(r, from, c, ref, sh) : note_candidates<DT, false>(r, from, c, ref, sh);
        __syncwarp();
        const unsigned listed = sh.listed[warp];
        uint32_t* id = sh.id + warp * kWarpList;
        uint32_t* key = sh.key + warp * kWarpList;
        uint32_t top = 0;
        for (unsigned j = lane; j < min(listed, static_cast<unsigned>(kWarpList)); j += 32) {
            key[j] = order_of(load_logit<DT>(r.base, id[j]));
            top = max(top, key[j]);
        }
        top = __reduce_max_sync(0xFFFFFFFFu, top);
        const double part = warp_sum(static_cast<double>(mine));
        if (lane == 0) {
            sh.red[warp] = part;
            sh.warp_count[warp] = top;
        }
        __syncthreads();
        double rest = 0.0;
        unsigned all = 0, most = 0;
        for (int v = 0; v < kWarps; ++v) {
            rest += sh.red[v];
            top = max(top, sh.warp_count[v]);
            all += sh.listed[v];
            most = max(most, sh.listed[v]);
        }
        __syncthreads();
        if (!(rest < INFINITY) || most > kWarpList || all == 0) return false;
        r.top = logit_of(top);
        if (!(r.top < INFINITY)) return false;

        auto each = [&](auto f) {
            for (unsigned j = lane; j < listed; j += 32) {
                const uint32_t k = key[j];
                f(place_of_order<DT>(k, id[j]), [&] { return r.weight(logit_of(k)); });
            }
        };
        const unsigned long long first = place_of<DT>(from, P.V - 1), last = place_of<DT>(r.top, 0);
        const bool everything = from == lowest_logit<DT>();
        // in units of the weights; the terms' relative error: their argument (its rounding and c's, 2^-24 of at most 40; smaller
        // terms are below 2^-40), the exponential's 2^-22, and as many additions as a thread makes in a row
        rest = with_sum ? rest * exp2(static_cast<double>(ref) - static_cast<double>(r.top) * static_cast<double>(c)) * P.one : 0.0;
        double slack = 4.0e-6 + (static_cast<double>(r.V) / (4 * kThreads) + 32.0) * 0x1p-24;
        if (all <= kFew) {
            if (row_of_few<DT>(P, at, lim, r, sh, static_cast<int>(all), from, rest, slack)) return true;
            __syncthreads();
        }
        unsigned long long cut = 0, total = 0;   // the border, and
        unsigned kept = 0;                       // what stands down to it (0: not known yet)
        auto take = [&](const Border& b) {
            if (b.place >= cut) {
                cut = b.place;
                total = b.above_mass + b.mass;
                kept = b.above_count + 1u;
            }
        };
        if (lim.k_on) {
            if (all < static_cast<unsigned>(lim.k) && !everything) {
                if (lim.p_on || !lim.m_on) return false;
            } else {
                const unsigned n_k = static_cast<unsigned>(lim.k);
                take(select(each, [=](unsigned n, unsigned long long) { return n >= n_k; }, first, last, sh));
            }
        }
        if (lim.p_on && lim.k_on) {   // of what top_k leaves
            const double target = static_cast<double>(lim.p) * static_cast<double>(total);
            take(select(each, [=](unsigned, unsigned long long s) { return static_cast<double>(s) >= target; }, first, last, sh));
        } else if (lim.p_on) {
            const double p = lim.p;
            for (;;) {
                const Border b = select(each, Share{p, rest, 0.0}, first, last, sh);
                const double listed_sum = static_cast<double>(b.all_mass), target = p * (listed_sum + rest);
                const double least = p * (listed_sum + rest * (1.0 - slack)), most_of_it = p * (listed_sum + rest * (1.0 + slack) + slack * 0x1p-20 * P.one);
                if (listed_sum < least) {   // beyond the candidates
                    if (!lim.m_on) return false;
                    break;
                }
                const double with_it = static_cast<double>(b.above_mass + b.mass);
                const bool sure = with_it >= (rest > 0.0 ? most_of_it : target) && (b.above_count == 0 || static_cast<double>(b.above_mass) < least);
                if (sure || rest == 0.0 || slack == 0.0) {
                    if (!(with_it >= target)) return false;
                    take(b);
                    break;
                }
                // too near to call (one row in 300): the rest once more, in double precision
                rest = static_cast<double>(block_sum(__double2ull_rn(sum_below<DT>(r, from)), sh));
                slack = 0.0;
            }
        }
        if (lim.m_on) {
            const double least = lim.least(P);
            unsigned long long lowest = ~0ull;
            each([&](unsigned long long place, auto&&) {
                if (static_cast<double>(logit_at<DT>(place)) - static_cast<double>(r.top) >= least)
                    lowest = min(lowest, place);
            });
            lowest = block_min(lowest, sh);
            // (entries beyond the candidates may belong to the set too: then it is no border, and another rule's is above it)
            if ((everything || static_cast<double>(from) - static_cast<double>(r.top) <= least) && lowest > cut) {
                cut = lowest;
                kept = 0;
            }
        }
        if (!cut && !everything) return false;
        if (kept == 0) {
            unsigned long long sum = 0;
            unsigned n = 0;
            each([&](unsigned long long place, auto&& weight) {
                if (place >= cut) {
                    sum += weight();
                    ++n;
                }
            });
            total = block_sum(sum, sh);
            kept = static_cast<unsigned>(block_sum(n, sh));
        }
        if (threadIdx.x == 0) write_law<DT>(P, at, r, cut, total, kept);
        if (!P.tokens) return true;
        const double target = lim.u * static_cast<double>(total);
        auto by_id = [&](auto f) {
            each([&](unsigned long long place, auto&& weight) {
                if (place >= cut) f(place & kIdMask, weight);
            });
        };
        const unsigned long long drawn = select(by_id, [=](unsigned, unsigned long long s) { return static_cast<double>(s) > target; },
                                                place_of_id(P.V - 1), place_of_id(0), sh).place;
        if (threadIdx.x == 0) write_token<DT>(P, at, r, total, id_at(drawn));
        return true;
    }

    // --------------------------------------------------------------------- values counted ----
    // Where candidates are too many, or the sample misled: one pass counts the row's entries by value, which places the border; a second
    // pass notes down the few entries near it and sums the weights before it, stretch by stretch for the draw.
    //   bfloat16: a bin is one number (30 binades of either sign), so all sums over the row follow from the counts, exactly (but for
    //   numbers near zero, see there), and the second pass looks for the entries equal to the border's number.
    //   binary32: bins are 1/96 of a power of two of the weight wide, masses are estimates, and the border is looked for among the bins
    //   within the estimates' error of it; the second pass sums exactly, over the whole row where top_p needs that.
    // A row of either kind that its bins do not hold (values out of their range that matter, borders in a bin of leftovers, more equal
    // entries than there is room for) takes the passes above.

    // The first pass.  Returns the thread's largest logit (binary32), and sets bad where there is a NaN (or, bfloat16, anything a bin
    // of leftovers cannot tell from one).
    template <int DT>
    static __device__ __forceinline__ float count_values(const Row& r, const Bins<DT>& bins, Shared& sh, bool& bad) {
        constexpr int N = Elem<DT>::kPerVec;
        constexpr int kBatch = 4;
        const int vectors = r.vec_elems / N;
        float top = -INFINITY;
        uint32_t largest = 0;
        char* table = reinterpret_cast<char*>(sh.bin);
        const uint32_t low2 = (bins.low - 1u) * 0x10001u, high2 = (bins.low - 1u + kValueBins - 1) * 0x10001u;
        auto count_bf16 = [&](uint32_t w, bool second) {   // a pair, as two indexes of four bytes each
            const uint32_t a = w & 0x7FFF7FFFu;
            largest = __vmaxu2(largest, a);
            const uint32_t t = (__vminu2(__vmaxu2(a, low2), high2) - low2 + ((w >> 15) & 0x00010001u) * kValueBins) << 2;
            atomicAdd(reinterpret_cast<unsigned*>(table + (t & 0xFFFFu)), 1u);
            if (second) atomicAdd(reinterpret_cast<unsigned*>(table + (t >> 16)), 1u);
        };
        auto count_f32 = [&](float l) {
            asm("max.NaN.f32 %0, %1, %2;" : "=f"(top) : "f"(top), "f"(l));
            atomicAdd(&sh.bin[bins.of(l)], 1u);
        };
    #pragma unroll 1
        for (int v0 = threadIdx.x; v0 < vectors; v0 += kBatch * kThreads) {
            uint4 w[kBatch];
    #pragma unroll
            for (int j = 0; j < kBatch; ++j)
                if (v0 + j * kThreads < vectors) w[j] = ld_global_nc_v4(r.base + static_cast<int64_t>(v0 + j * kThreads) * 16);
    #pragma unroll
            for (int j = 0; j < kBatch; ++j)
                if (v0 + j * kThreads < vectors) {
                    const uint32_t v[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
    #pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        if constexpr (DT == FEF_BF16)
                            count_bf16(v[q], true);
                        else
                            count_f32(__uint_as_float(v[q]));
                    }
                }
        }
        for (int x = r.vec_elems + threadIdx.x; x < r.V; x += kThreads) {
            const float l = load_logit<DT>(r.base, x);
            if constexpr (DT == FEF_BF16)
                count_bf16(__float_as_uint(l) >> 16, false);
            else
                count_f32(l);
        }
        if constexpr (DT == FEF_BF16)
            bad |= (largest & 0xFFFFu) > 0x7F80u || (largest >> 16) > 0x7F80u;
        else
            bad |= !(top < INFINITY);
        return top;
    }

    // The second pass.  Entries from `weigh` on have their weights summed into sh.chunk, those of [near, before) go into the warps' lists
    // (their ids), and with REST the weights of [far, near) are summed up for the thread.  (Sums in double precision, in a fixed
    // order, and rounded to the weights' units stretch by stretch.)
    struct Limits4 {
        float weigh, before, near, far;
    };
    template <int DT, bool REST>
    static __device__ __forceinline__ double gather_near(const Row& r, int pieces_per_chunk, const Limits4& at, Shared& sh) {
        constexpr int N = Elem<DT>::kPerVec;
        constexpr int kBatch = 4;
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        const unsigned lower = (1u << lane) - 1u;
        const int pieces = r.vec_elems / (32 * N);
        const int chunks = (pieces + pieces_per_chunk - 1) / pieces_per_chunk;
        uint32_t* list = sh.id + warp * kWarpList;
        unsigned listed = 0;
        double rest = 0.0;
        auto note = [&](bool hit, int x) {
            const unsigned hits = __ballot_sync(0xFFFFFFFFu, hit);
            const unsigned at = listed + __popc(hits & lower);
            if (hit && at < kWarpList) list[at] = static_cast<uint32_t>(x);
            listed += __popc(hits);
        };
        // (chunk `chunks` is what is behind the last whole piece)
        for (int c = warp; c <= chunks; c += kWarps) {
            double sum = 0.0;
            if (c < chunks) {
                const int end = min((c + 1) * pieces_per_chunk, pieces);
    #pragma unroll 1
                for (int p = c * pieces_per_chunk; p < end; p += kBatch) {   // (pieces_per_chunk is a multiple of kBatch)
                    uint4 w[kBatch];
    #pragma unroll
                    for (int j = 0; j < kBatch; ++j)
                        if (p + j < end) w[j] = ld_global_nc_v4(r.base + (static_cast<int64_t>(p + j) * 32 + lane) * 16);
                    uint32_t mask = 0;
    #pragma unroll
                    for (int j = 0; j < kBatch; ++j)
                        if (p + j < end) {
                            float l[N];
                            unpack<DT>(w[j], l);
                            bool any = false;
    #pragma unroll
                            for (int i = 0; i < N; ++i) {
                                mask |= l[i] >= at.near && l[i] < at.before ? 1u << (j * N + i) : 0u;
                                any |= l[i] >= at.weigh;
                            }
                            if (REST || __any_sync(0xFFFFFFFFu, any)) {
    #pragma unroll
                                for (int i = 0; i < N; ++i) {
                                    double a, b;
                                    r.factors(l[i], a, b);
                                    if (l[i] >= at.weigh) sum = fma(a, b, sum);
                                    if (REST && l[i] >= at.far && l[i] < at.near) rest = fma(a, b, rest);
                                }
                            }
                        }
                    while (__any_sync(0xFFFFFFFFu, mask != 0u)) {
                        const int bit = max(__ffs(mask) - 1, 0);
                        note(mask != 0u, ((p + bit / N) * 32 + lane) * N + bit % N);
                        mask &= mask - 1u;
                    }
                }
            } else {
                for (int x0 = pieces * 32 * N; x0 < r.V; x0 += 32) {
                    const int x = x0 + lane;
                    const float l = x < r.V ? load_logit<DT>(r.base, x) : -INFINITY;
                    note(l >= at.near && l < at.before && x < r.V, x);
                    if (l >= at.weigh) sum += static_cast<double>(r.weight(l));
                    if (REST && l >= at.far && l < at.near) rest += static_cast<double>(r.weight(l));
                }
            }
            sum = warp_sum(sum);
            if (lane == 0) sh.chunk[c] = __double2ull_rn(sum);
        }
        if (lane == 0) sh.listed[warp] = listed;
        return rest;
    }

    // The same for bfloat16 where the border is a positive number: weights come from a table of all positive numbers from it on.  False:
    // there are more entries equal to the border than there is room for beside the table.
    static constexpr int kTies = 128;
    static_assert((kValueBins - 2) * 8 + kWarps * kTies * 4 <= kList * 8, "the table and the ties fit where the candidates are otherwise");
    static __device__ __forceinline__ bool gather_with_table(const Row& r, int pieces_per_chunk, float border, uint32_t low, Shared& sh) {
        constexpr int N = Elem<FEF_BF16>::kPerVec;
        constexpr int kBatch = 4;
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        const unsigned lower = (1u << lane) - 1u;
        unsigned long long* table = reinterpret_cast<unsigned long long*>(sh.id);
        uint32_t* list = reinterpret_cast<uint32_t*>(table + kValueBins - 2) + warp * kTies;
        const uint32_t at_border = __float_as_uint(border) >> 16, at_top = __float_as_uint(r.top) >> 16;
        for (uint32_t a = at_border + threadIdx.x; a <= at_top; a += kThreads) table[a - low] = r.weight(__uint_as_float(a << 16));
        __syncthreads();
        const uint32_t border2 = at_border * 0x10001u;
        const int pieces = r.vec_elems / (32 * N);
        const int chunks = (pieces + pieces_per_chunk - 1) / pieces_per_chunk;
        unsigned listed = 0;
        auto note = [&](bool hit, int x) {
            const unsigned hits = __ballot_sync(0xFFFFFFFFu, hit);
            const unsigned at = listed + __popc(hits & lower);
            if (hit && at < kTies) list[at] = static_cast<uint32_t>(x);
            listed += __popc(hits);
        };
        for (int c = warp; c <= chunks; c += kWarps) {   // (chunk `chunks` is what is behind the last whole piece)
            unsigned long long sum = 0;
            if (c < chunks) {
                const int end = min((c + 1) * pieces_per_chunk, pieces);
    #pragma unroll 1
                for (int p = c * pieces_per_chunk; p < end; p += kBatch) {
                    uint4 w[kBatch];
    #pragma unroll
                    for (int j = 0; j < kBatch; ++j) {
                        w[j] = make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u);
                        if (p + j < end) w[j] = ld_global_nc_v4(r.base + (static_cast<int64_t>(p + j) * 32 + lane) * 16);
                    }
                    uint32_t mask = 0;
    #pragma unroll
                    for (int j = 0; j < kBatch; ++j) {
                        const uint32_t v[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
    #pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const uint32_t a = v[q] & 0xFFFFu, b = v[q] >> 16;   // (a negative number is beyond the largest)
                            mask |= equal_to(v[q], border2) & (0x00010001u << (4 * j + q));
                            if (a - at_border - 1u < at_top - at_border) sum += table[a - low];
                            if (b - at_border - 1u < at_top - at_border) sum += table[b - low];
                        }
                    }
                    while (__any_sync(0xFFFFFFFFu, mask != 0u)) {
                        const int bit = max(__ffs(mask) - 1, 0);   // bit 16 h + 4 j + q: half h of word q of vector j
                        note(mask != 0u, ((p + (bit >> 2 & 3)) * 32 + lane) * N + (bit & 3) * 2 + (bit >> 4));
                        mask &= mask - 1u;
                    }
                }
            } else {
                for (int x0 = pieces * 32 * N; x0 < r.V; x0 += 32) {
                    const int x = x0 + lane;
                    const float l = x < r.V ? load_logit<FEF_BF16>(r.base, x) : -INFINITY;
                    note(l == border, x);
                    if (l > border) sum += r.weight(l);
                }
            }
            sum = warp_sum_u64(sum);
            if (lane == 0) sh.chunk[c] = sum;
        }
        const bool fits = listed <= kTies;
        if (__syncthreads_and(fits) == 0) return false;
        // the ties move to where the warps' lists are
        uint32_t mine[(kTies + 31) / 32];
    #pragma unroll
        for (int j = 0; j < (kTies + 31) / 32; ++j) mine[j] = j * 32 + lane < listed ? list[j * 32 + lane] : 0u;
        __syncthreads();
    #pragma unroll
        for (int j = 0; j < (kTies + 31) / 32; ++j)
            if (j * 32 + lane < listed) sh.id[warp * kWarpList + j * 32 + lane] = mine[j];
        if (lane == 0) sh.listed[warp] = listed;
        return true;
    }

    // False: the row needs the passes (nothing has been written).
    template <int DT>
    static __device__ bool row_by_values(const Params& P, int64_t at, const Limits& lim, Row& r, Shared& sh) {
        constexpr int N = Elem<DT>::kPerVec;
        constexpr int kPerThread = kRowBinsPerThread;
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        if (r.V <= kAll) return false;
        if (DT == FEF_F32 && lim.k_on && lim.p_on) return false;   // (two borders, one inside the other)
        const float c = static_cast<float>(P.c);

        // ---- where the bins lie, from a sample
        Bins<DT> bins;
        bins.c = c;
        {
            constexpr int kPerWarp = kSample / (kWarps * 32 * N);
            const int pieces = r.vec_elems / (32 * N);
            float x[kPerWarp * N], top = -INFINITY, size = 0.f;
    #pragma unroll
            for (int j = 0; j < kPerWarp; ++j) {
                const int s = warp * kPerWarp + j;
                const int piece = static_cast<int>((static_cast<int64_t>(2 * s + 1) * pieces) / (2 * kPerWarp * kWarps));
                unpack<DT>(ld_global_nc_v4(r.base + (static_cast<int64_t>(piece) * 32 + lane) * 16), *reinterpret_cast<float(*)[N]>(x + j * N));
            }
    #pragma unroll
            for (int j = 0; j < kPerWarp * N; ++j) top = fmaxf(top, x[j]);
    #pragma unroll
            for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
            __syncthreads();
            if (lane == 0) sh.red_f[warp][0] = top;
            __syncthreads();
            for (int w = 0; w < kWarps; ++w) top = fmaxf(top, sh.red_f[w][0]);
            if (!(top > -INFINITY && top < INFINITY)) return false;
            bins.anchor = top;
            bins.low = 0;
            if constexpr (DT == FEF_BF16) {
                // the binades of what may weigh anything (64 powers of two below the largest sampled weight end it), and one more; with
                // smaller logits about, the range reaches so far that what lies beyond it weighs nothing
                const float end = top - 64.f / c;
                int far = 0;
    #pragma unroll
                for (int j = 0; j < kPerWarp * N; ++j) {
                    if (x[j] >= end)
                        size = fmaxf(size, fabsf(x[j]));
                    else
                        far = 1;
                }
    #pragma unroll
                for (int o = 16; o > 0; o >>= 1) size = fmaxf(size, __shfl_xor_sync(0xFFFFFFFFu, size, o));
                far = __any_sync(0xFFFFFFFFu, far);
                __syncthreads();
                if (lane == 0) {
                    sh.red_f[warp][0] = size;
                    sh.red_f[warp][1] = far ? 1.f : 0.f;
                }
                __syncthreads();
                float any_far = 0.f;
                for (int w = 0; w < kWarps; ++w) {
                    size = fmaxf(size, sh.red_f[w][0]);
                    any_far = fmaxf(any_far, sh.red_f[w][1]);
                }
                if (any_far > 0.f) size = fmaxf(size, 64.f / c);
                // binades low .. low + 29, the last but one that of `size`
                const int exponent = static_cast<int>(__float_as_uint(size) >> 23) + 1;
                const int first = min(max(exponent - 29, 1), 254 - 29);
                bins.low = static_cast<uint32_t>(first) << 7;
            }
        }
        for (int b = threadIdx.x; b < kRowBins; b += kThreads) sh.bin[b] = 0;
        if (threadIdx.x == 0) sh.bad = 0;
        __syncthreads();

        // ---- first pass
        bool bad = false;
        float top = count_values<DT>(r, bins, sh, bad);
        if (bad) sh.bad = 1;
        __syncthreads();
        unsigned ns = 0;
        int first_used = kRowBins;   // the thread's first rank with an entry
        const int rank0 = threadIdx.x * kPerThread;
        for (int j = 0; j < kPerThread; ++j) {
            const int rank = rank0 + j;
            const unsigned n = rank < kRowBins ? sh.bin[Bins<DT>::at(rank)] : 0u;
            if (n && !ns) first_used = rank;
            ns += n;
        }
        // the largest logit
        if constexpr (DT == FEF_F32) {
    #pragma unroll
            for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
            if (lane == 0) sh.red_f[warp][0] = top;
        } else {
            const int first = __reduce_min_sync(0xFFFFFFFFu, first_used);
            if (lane == 0) sh.warp_count[warp] = static_cast<unsigned>(first);
        }
        __syncthreads();
        if constexpr (DT == FEF_F32) {
            for (int w = 0; w < kWarps; ++w) top = fmaxf(top, sh.red_f[w][0]);
        } else {
            unsigned first = kRowBins;
            for (int w = 0; w < kWarps; ++w) first = min(first, sh.warp_count[w]);
            top = bins.value(static_cast<int>(first));
        }
        // Leftovers.  Above the range: the passes.  Behind it: nothing that weighs anything, or the passes.
        const unsigned above_range = sh.bin[Bins<DT>::at(0)], behind = sh.bin[Bins<DT>::at(kRowBins - 1)];
        __syncthreads();
        if (sh.bad || above_range) return false;
        r.top = top;
        if (behind && r.weight(bins.value(kRowBins - 1))) return false;
        constexpr int kLowFirst = kValueBins - 1;   // (bfloat16) the ranks of what is too small to tell apart, counted as zeros
        if constexpr (DT == FEF_BF16) {
            // Numbers that are no zeros among them put the sums out by 2^-29 of the largest logit's exponent times their weight.  A few
            // hardly ever matter (one row in a thousand has one); where they might, by 2^-45 of the largest weight, it is the passes' turn.
            const unsigned low = sh.bin[Bins<DT>::at(kLowFirst)] + sh.bin[Bins<DT>::at(kLowFirst + 1)];
            const float smallest = __uint_as_float(bins.low << 16);
            if (low && static_cast<float>(low) * ex2_approx(-top * c) * smallest * c > 0x1p-45f) {
                bool other = false;
                for_each<DT>(r, [&](float l, int) { other |= l != 0.f && fabsf(l) < smallest; });
                if (__syncthreads_or(other)) return false;
            }
        }
        auto leftover = [&](int rank) { return rank == kRowBins - 1 || (DT == FEF_BF16 && (rank == kLowFirst || rank == kLowFirst + 1)); };

        // ---- counts and weights before each thread's bins (binary32: weights are estimates, of a bin's middle)
        auto count_at = [&](int rank) { return rank < kRowBins ? sh.bin[Bins<DT>::at(rank)] : 0u; };
        using Mass = typename std::conditional<DT == FEF_BF16, unsigned long long, double>::type;
        auto bits_of = [](Mass m) {
            if constexpr (DT == FEF_BF16) return m;
            else return static_cast<unsigned long long>(__double_as_longlong(m));
        };
        auto mass_of = [](unsigned long long b) {
            if constexpr (DT == FEF_BF16) return b;
            else return __longlong_as_double(static_cast<long long>(b));
        };
        auto weight_at = [&](int rank) -> Mass {
            if (rank >= kRowBins - 1) return 0;
            if constexpr (DT == FEF_BF16) return r.weight(bins.value(rank));
            else return static_cast<double>(ex2_approx(Bins<DT>::kAbove - (static_cast<float>(rank) + 0.5f) / Bins<DT>::kScale));
        };
        Mass ms = 0;
    #pragma unroll 4
        for (int j = 0; j < kPerThread; ++j) ms += weight_at(rank0 + j) * count_at(rank0 + j);
        unsigned pn = ns;
        Mass pm = ms;
    #pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned on = __shfl_up_sync(0xFFFFFFFFu, pn, o);
            const Mass om = __shfl_up_sync(0xFFFFFFFFu, pm, o);
            if (lane >= o) {
                pn += on;
                pm += om;
            }
        }
        if (lane == 31) {
            sh.warp_count[warp] = pn;
            sh.warp_mass[warp] = bits_of(pm);
        }
        __syncthreads();
        pn -= ns;
        pm -= ms;
        Mass mass = 0;
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) {
                pn += sh.warp_count[w];
                pm += mass_of(sh.warp_mass[w]);
            }
            mass += mass_of(sh.warp_mass[w]);
        }
        // The first bin, from the largest down, with which `enough` holds: sh.loc_rank, and what stands before it (false: there is none).
        // The thread it belongs to is found first, then a warp looks at that thread's bins.
        auto locate = [&](auto enough) {
            __syncthreads();
            if (threadIdx.x == 0) sh.loc_rank = -1;
            __syncthreads();
            if (ns && !(pn > 0 && enough(pn, pm)) && enough(pn + ns, pm + ms)) {
                sh.loc_rank = rank0;
                sh.loc_n = pn;
                sh.loc_m = bits_of(pm);
            }
            __syncthreads();
            if (sh.loc_rank < 0) return false;
            if (warp == 0) {
                static_assert(kPerThread <= 32, "a lane for each of a thread's bins");
                const int rank = sh.loc_rank + lane;
                const unsigned n = lane < kPerThread ? count_at(rank) : 0u;
                const Mass m = n ? weight_at(rank) * n : 0;
                unsigned un = n;
                Mass um = m;
    #pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const unsigned on = __shfl_up_sync(0xFFFFFFFFu, un, o);
                    const Mass om = __shfl_up_sync(0xFFFFFFFFu, um, o);
                    if (lane >= o) {
                        un += on;
                        um += om;
                    }
                }
                un += sh.loc_n;
                um += mass_of(sh.loc_m);
                const unsigned there = __ballot_sync(0xFFFFFFFFu, n && enough(un, um));
                if (lane == __ffs(there) - 1) {
                    sh.loc_rank = rank;
                    sh.loc_n = un - n;
                    sh.loc_m = bits_of(um - m);
                }
            }
            __syncthreads();
            return true;
        };
        const bool cut_on = lim.k_on || lim.p_on || lim.m_on;
        const double least = lim.m_on ? lim.least(P) : 0.0;

        // ---- the ranks the border is among
        int rank_a = kRowBins, rank_b = kRowBins;   // first and last
        unsigned before_n;                          // entries before them,
        unsigned long long before_m = 0;            // and (bfloat16) their weight
        unsigned want = 0xFFFFFFFFu;                // (bfloat16) entries in the law
        if (!cut_on) {
            before_n = static_cast<unsigned>(r.V) - behind;
            if (behind) {   // those of them that are not -inf belong to the law
                unsigned finite = 0;
                for_each<DT>(r, [&](float, int) { ++finite; });
                before_n = static_cast<unsigned>(block_sum(finite, sh));
            }
            if constexpr (DT == FEF_BF16) before_m = mass;
        } else if constexpr (DT == FEF_BF16) {
            // how many entries each rule keeps; the fewest are the law
            unsigned long long of_first = mass;   // weight of what top_k leaves
            if (lim.k_on) {
                want = static_cast<unsigned>(lim.k);
                if (!locate([=](unsigned n, unsigned long long) { return n >= want; })) return false;
                of_first = sh.loc_m + weight_at(sh.loc_rank) * (want - sh.loc_n);
            }
            if (lim.p_on) {
                const double target = static_cast<double>(lim.p) * static_cast<double>(of_first);
                if (!locate([=](unsigned, unsigned long long m) { return static_cast<double>(m) >= target; })) return false;
                // the fewest of the number's entries that reach it (one at least)
                const unsigned long long w = weight_at(sh.loc_rank), m = sh.loc_m;
                unsigned few = 1, many = count_at(sh.loc_rank);
                while (few < many) {
                    const unsigned mid = few + (many - few) / 2;
                    if (static_cast<double>(m + w * mid) >= target)
                        many = mid;
                    else
                        few = mid + 1;
                }
                want = min(want, sh.loc_n + few);
            }
            if (lim.m_on) {
                unsigned upto = 0, n = pn;   // entries down to the thread's last bin that belongs to the set
                for (int j = 0; j < kPerThread; ++j) {
                    const unsigned count = count_at(rank0 + j);
                    n += count;
                    if (count && static_cast<double>(bins.value(rank0 + j)) - static_cast<double>(top) >= least) upto = n;
                }
                want = min(want, 0xFFFFFFFFu - static_cast<unsigned>(block_min(0xFFFFFFFFu - upto, sh)));
            }
            if (want == 0 || !locate([=](unsigned n, unsigned long long) { return n >= want; })) return false;
            rank_a = rank_b = sh.loc_rank;
            before_n = sh.loc_n;
            before_m = sh.loc_m;
            if (leftover(rank_a)) return false;
        } else {
            // every rule gives a range of ranks; the border is not before the first range's first rank nor behind its last
            if (lim.k_on) {
                const unsigned k = static_cast<unsigned>(lim.k);
                if (!locate([=](unsigned n, double) { return n >= k; })) return false;
                rank_a = rank_b = sh.loc_rank;
            }
            if (lim.p_on) {
                // (a bin's weight is off by less than 0.4 % where it matters, on either side of the border)
                const double p = lim.p, whole = mass, error = 0.02 * fmax(p, 0.0) * (1.0 - fmax(p, 0.0)) * whole;
                if (!locate([=](unsigned, double m) { return m >= p * whole - error; })) return false;
                rank_a = min(rank_a, sh.loc_rank);
                if (!locate([=](unsigned, double m) { return m >= p * whole + error; })) return false;
                rank_b = min(rank_b, sh.loc_rank);
            }
            if (lim.m_on) {
                const int rank = bins.of(static_cast<float>(static_cast<double>(top) + least));
                rank_a = min(rank_a, rank - 1);
                rank_b = min(rank_b, rank + 1);
            }
            if (rank_a > rank_b || rank_b >= kRowBins - 1) return false;
            __syncthreads();
            if (rank0 <= rank_a && rank_a < rank0 + kPerThread) {
                unsigned count = pn;
                for (int j = 0; rank0 + j < rank_a; ++j) count += sh.bin[rank0 + j];
                sh.loc_n = count;
            }
            __syncthreads();
            before_n = sh.loc_n;
        }
        __syncthreads();   // (the bins make room for the candidates)

        // ---- second pass
        const int pieces = r.vec_elems / (32 * N);
        const int per_chunk = ((pieces + kMaxChunks - 1) / kMaxChunks + 3) / 4 * 4;
        const int chunks = (pieces + per_chunk - 1) / per_chunk;
        const float border = DT == FEF_BF16 && cut_on ? bins.value(rank_a) : -INFINITY;
        Limits4 where;
        if constexpr (DT == FEF_BF16) {
            const float weightless = top - 64.f / c;   // (so far below the largest logit nothing has a weight)
            where.before = cut_on ? nextafterf(border, INFINITY) : -INFINITY;
            where.near = cut_on ? border : -INFINITY;
            where.weigh = fmaxf(where.before, weightless);
            where.far = where.weigh;
        } else {
            // the lowest numbers of the ranks before rank_a, up to rank_b and before the last: found by halving, so that an entry is
            // placed by comparisons
            __syncthreads();
            if (threadIdx.x < 3) {
                const int rank = threadIdx.x == 0 ? min(rank_a - 1, kRowBins - 2) : threadIdx.x == 1 ? min(rank_b, kRowBins - 2) : kRowBins - 2;
                uint32_t in = order_of(top), out = order_of(lowest_logit<DT>()) - 1u;   // (the largest logit's rank is at most rank_b)
                if (bins.of(top) > rank) in += 1u;   // nothing is before the border
                while (in - out > 1u && in <= order_of(top)) {
                    const uint32_t mid = out + (in - out) / 2;
                    if (bins.of(logit_of(mid)) <= rank)
                        in = mid;
                    else
                        out = mid;
                }
                sh.red_f[threadIdx.x][0] = logit_of(in);
            }
            __syncthreads();
            where.before = where.weigh = sh.red_f[0][0];
            where.near = cut_on ? sh.red_f[1][0] : where.before;
            where.far = sh.red_f[2][0];
            __syncthreads();
        }
        const bool need_rest = DT == FEF_F32 && lim.p_on;
        bool by_chunks = P.tokens != nullptr;   // the draw goes by the stretches' sums, not by the candidates
        unsigned long long rest = 0;
        if constexpr (DT == FEF_BF16) {
            if (!cut_on) {
                if (P.tokens) gather_near<DT, false>(r, per_chunk, where, sh);
                else if (lane == 0) sh.listed[warp] = 0;
            } else {
                bool noted = false;
                if (P.tokens && want <= static_cast<unsigned>(kList) / 8 * 7) {   // a law of few entries: all of them are candidates
                    note_candidates<DT, false>(r, border, 0.f, 0.f, sh);
                    __syncthreads();
                    unsigned longest = 0;
                    for (int w = 0; w < kWarps; ++w) longest = max(longest, sh.listed[w]);
                    noted = longest <= kWarpList;   // (or they are too many in one warp's share)
                    __syncthreads();
                }
                if (noted) {
                    by_chunks = false;
                    before_n = 0;
                    before_m = 0;
                } else if (P.tokens) {
                    if (!(border > 0.f && gather_with_table(r, per_chunk, border, bins.low, sh))) {
                        __syncthreads();
                        gather_near<DT, false>(r, per_chunk, where, sh);
                    }
                } else {
                    note_candidates<DT, false, true>(r, border, 0.f, 0.f, sh);
                }
            }
        } else {
            double mine = 0.0;
            if (need_rest)
                mine = gather_near<DT, true>(r, per_chunk, where, sh);
            else
                gather_near<DT, false>(r, per_chunk, where, sh);
            mine = warp_sum(mine);
            if (lane == 0) sh.red[warp] = mine;
        }
        __syncthreads();
        if constexpr (DT == FEF_F32) {
            double all = 0.0;
            for (int w = 0; w < kWarps; ++w) all += sh.red[w];
            rest = __double2ull_rn(all);
            unsigned long long sum = 0;
            for (int i = threadIdx.x; i <= chunks; i += kThreads) sum += sh.chunk[i];
            before_m = block_sum(sum, sh);
        }
        const unsigned listed = sh.listed[warp];
        unsigned most = 0;
        for (int w = 0; w < kWarps; ++w) most = max(most, sh.listed[w]);
        if (most > kWarpList) return false;
        uint32_t* id = sh.id + warp * kWarpList;
        uint32_t* key = sh.key + warp * kWarpList;
        for (unsigned j = lane; j < listed; j += 32) key[j] = order_of(load_logit<DT>(r.base, id[j]));
        __syncwarp();
        auto each = [&](auto f) {
            for (unsigned j = lane; j < listed; j += 32) {
                const uint32_t k = key[j];
                f(place_of_order<DT>(k, id[j]), [&] { return r.weight(logit_of(k)); });
            }
        };

        // ---- the border
        unsigned long long first = ~0ull, last = 0, cut = 0;   // (where the candidates stand, so that the first level's bins divide them)
        if (cut_on) {
            each([&](unsigned long long place, auto&&) {
                first = min(first, place);
                last = max(last, place);
            });
            first = block_min(first, sh);
            last = ~block_min(~last, sh);
        }
        if constexpr (DT == FEF_BF16) {
            if (cut_on) cut = select(each, [=](unsigned n, unsigned long long) { return n >= want; }, first, last, sh, before_n, before_m).place;
        } else if (cut_on) {
            unsigned long long near_mine = 0;
            unsigned near_n = 0;
            each([&](unsigned long long, auto&& weight) {
                near_mine += weight();
                ++near_n;
            });
            const unsigned long long near = block_sum(near_mine, sh);
            near_n = static_cast<unsigned>(block_sum(near_n, sh));
            if (near_n == 0) return false;
            if (lim.k_on && before_n + near_n >= static_cast<unsigned>(lim.k)) {
                const unsigned k = static_cast<unsigned>(lim.k);
                if (before_n >= k) return false;
                cut = select(each, [=](unsigned n, unsigned long long) { return n >= k; }, first, last, sh, before_n, before_m).place;
            }
            if (lim.p_on) {
                const double target = static_cast<double>(lim.p) * static_cast<double>(before_m + near + rest);
                if (before_n && static_cast<double>(before_m) >= target) return false;
                if (static_cast<double>(before_m + near) >= target)
                    cut = max(cut, select(each, [=](unsigned, unsigned long long s) { return static_cast<double>(s) >= target; }, first, last, sh,
                                          before_n, before_m).place);
            }
            if (lim.m_on) {
                unsigned long long lowest = ~0ull;
                unsigned behind_it = 0;
                each([&](unsigned long long place, auto&&) {
                    if (static_cast<double>(logit_at<DT>(place)) - static_cast<double>(r.top) >= least)
                        lowest = min(lowest, place);
                    else
                        behind_it = 1;
                });
                lowest = block_min(lowest, sh);
                behind_it = static_cast<unsigned>(block_sum(behind_it, sh));
                if (lowest == ~0ull) return false;          // it lies before the candidates
                // the last candidate that belongs to the set is its last entry if a candidate that does not follows, or the candidates go
                // further down than the limit
                if (behind_it || rank_b >= bins.of(static_cast<float>(static_cast<double>(r.top) + least)) + 1) cut = max(cut, lowest);
            }
            if (!cut) return false;
        }
        unsigned long long sum = 0;
        unsigned kept = 0;
        const int entries_per_chunk = per_chunk * 32 * N;
        each([&](unsigned long long place, auto&& weight) {
            if (place >= cut) {
                const unsigned long long w = weight();
                sum += w;
                ++kept;
                const int x = id_at(place);
                if (by_chunks) atomicAdd(&sh.chunk[x < pieces * 32 * N ? x / entries_per_chunk : chunks], w);
            }
        });
        const unsigned long long total = before_m + block_sum(sum, sh);
        kept = before_n + static_cast<unsigned>(block_sum(kept, sh));
        if (threadIdx.x == 0) write_law<DT>(P, at, r, cut, total, kept);
        if (!P.tokens) return true;

        const double target = lim.u * static_cast<double>(total);
        if (!by_chunks) {
            auto by_id = [&](auto f) {
                each([&](unsigned long long place, auto&& weight) {
                    if (place >= cut) f(place & kIdMask, weight);
                });
            };
            const unsigned long long drawn = select(by_id, [=](unsigned, unsigned long long s) { return static_cast<double>(s) > target; },
                                                    place_of_id(P.V - 1), place_of_id(0), sh).place;
            if (threadIdx.x == 0) write_token<DT>(P, at, r, total, id_at(drawn));
            return true;
        }

        // ---- the draw: the stretch that the number falls into, then the entry
        if (threadIdx.x == 0) {
            sh.in_bin = 0;
            sh.above_mass = 0;
        }
        __syncthreads();
        {
            const unsigned long long m = static_cast<int>(threadIdx.x) <= chunks ? sh.chunk[threadIdx.x] : 0ull;
            unsigned long long upto = m;
    #pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const unsigned long long om = __shfl_up_sync(0xFFFFFFFFu, upto, o);
                if (lane >= o) upto += om;
            }
            if (lane == 31) sh.warp_mass[warp] = upto;
            __syncthreads();
            for (int w = 0; w < warp; ++w) upto += sh.warp_mass[w];
            if (m && static_cast<double>(upto) > target && !(static_cast<double>(upto - m) > target)) {   // one thread
                sh.in_bin = threadIdx.x;
                sh.above_mass = upto - m;
            }
        }
        __syncthreads();
        const int stretch = static_cast<int>(sh.in_bin);
        const unsigned long long before_it = sh.above_mass;
        const int x_begin = stretch * entries_per_chunk < pieces * 32 * N && stretch < chunks ? stretch * entries_per_chunk : pieces * 32 * N;
        const int x_end = stretch < chunks ? min(x_begin + entries_per_chunk, pieces * 32 * N) : r.V;
        auto by_id = [&](auto f) {
            for (int x = x_begin + threadIdx.x; x < x_end; x += kThreads) {
                const float l = load_logit<DT>(r.base, x);
                if (l != -INFINITY && place_of<DT>(l, x) >= cut) f(place_of_id(x), [&] { return r.weight(l); });
            }
        };
        const unsigned long long drawn = select(by_id, [=](unsigned, unsigned long long s) { return static_cast<double>(s) > target; },
                                                place_of_id(x_end - 1), place_of_id(x_begin), sh, 1u, before_it).place;
        if (threadIdx.x == 0) write_token<DT>(P, at, r, total, id_at(drawn));
        return true;
    }
};

template <int kThreads, int DT>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads) truncate_kernel(const __grid_constant__ Params P) {
    using R = Rows<kThreads>;
    typename R::Shared& sh = *reinterpret_cast<typename R::Shared*>(trunc_smem);
    const int64_t at = blockIdx.x;
    const int b = static_cast<int>(at / P.K), i = static_cast<int>(at - static_cast<int64_t>(b) * P.K);
    if (gridDim.x == 1 && P.status) {
        if (threadIdx.x == 0) *P.status = FEF_OK;
        __syncthreads();   // (an error is reported after it)
    }
    if (P.row_len && i >= __ldg(P.row_len + b)) {
        if (threadIdx.x == 0) write_none(P, at, false);
        return;
    }
    if (threadIdx.x < 256) sh.table[threadIdx.x] = exp2(static_cast<double>(threadIdx.x) / 256.0);
    const Limits lim = limits_of(P, at, b, i);
    Row r;
    r.base = P.logits + at * P.ld_bytes;
    r.V = P.V;
    r.vec_elems = P.vec_elems;
    r.c = P.c;
    r.one = P.one;
    r.ones = P.ones;
    r.c256 = 256.0 * P.c;
    r.c256_f = static_cast<float>(r.c256);
    __syncthreads();
    if (!lim.bad && (R::template row_by_candidates<DT>(P, at, lim, r, sh) || R::template row_by_values<DT>(P, at, lim, r, sh))) return;
    R::template row_by_passes<DT>(P, at, lim, r, sh);
}

template <int kThreads, int DT>
static cudaError_t launch(const Params& P, int dev, cudaStream_t stream) {
    constexpr int smem = sizeof(typename Rows<kThreads>::Shared);
    static bool allowed[64];   // large shared memory, per device
    if (dev >= 64 || !allowed[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(truncate_kernel<kThreads, DT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
        if (dev < 64) allowed[dev] = true;
    }
    truncate_kernel<kThreads, DT><<<static_cast<unsigned>(P.B * P.K), kThreads, smem, stream>>>(P);
    return cudaGetLastError();
}
// Few rows: more threads to each, as many as an SM holds when there is an SM for every row.  Many: four rows to an SM, so that one's
// selections hide behind the others' streams.  (Short rows have no work for more threads.)
template <int DT>
static cudaError_t launch(const Params& P, int dev, int sms, cudaStream_t stream) {
    const int64_t rows = static_cast<int64_t>(P.B) * P.K;
    if (rows <= sms && P.V > 8192) return launch<1024, DT>(P, dev, stream);
    if (rows <= 2 * sms && P.V > 4096) return launch<512, DT>(P, dev, stream);
    return launch<256, DT>(P, dev, stream);
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
    P.ones = 62 - bits;
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
    // (one row's CTA clears the status by itself: 2 us less; of several, one could do so after another's report)
    if (device_status && B * K > 1 && cudaMemsetAsync(device_status, 0, sizeof(int32_t), stream) != cudaSuccess) return FEF_ERR_CUDA;
    const cudaError_t e = dt == FEF_F32 ? launch<FEF_F32>(P, dev, sms, stream) : launch<FEF_BF16>(P, dev, sms, stream);
    return e == cudaSuccess ? FEF_OK : FEF_ERR_CUDA;
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
