// The next token from a row of logits and a given random number: temperature, top-k, top-p, min-p.
//
// The row's order is larger logit first, lower index among equals; weights w = 2^((l - l_max) log2(e) / temperature).  Every filter keeps a beginning of the
// order - k tokens; as many as reach p of those k tokens' sum; those of at least min_p times the largest weight - and the token drawn is the first whose running sum
// passes u times the sum of what is kept.  So all of it is the same question: where, in the order, does a running count or a running sum reach a target?
//
// Nothing is sorted.  A histogram over the logits in steps of 2^(1/32) of a weight, 4096 bins of counts or of sums in LDS, says in which bin that is; the
// bin's tokens - some hundred of them for a usual row - are collected, and each finds its own place among them.  A bin of more than kList is cut again by the
// bits of its logits, and equal logits by their index, until few are left.  Two or three passes over the row, the first from memory.
//
// The histogram is laid from the largest of the row's first logits, which is known before the others have arrived; only where a later one's weight is more than
// 2^64 times its own, or where the first are all masked and the others stand below zero, is it laid again.
//
// Sums are exact: a bin's tokens add 2^(their place in the bin), which is near 1, as whole multiples of 2^-44 with a relative error of 2^-43, and the bin's sum, or
// that of the first of its tokens, is scaled by 2^(-bin / 32) once, by a product of whole numbers that is cut off.  Whole numbers add up to the same
// whichever wavefront comes first, and a border between two tokens is where 64-bit arithmetic has it but for 2^-40 of the sum.  With weights in fp32 it would
// be up to 2^-24 off, which is another token once in some hundred thousand rows.
//
// Bound by one CU's instructions - the vector units are busy 63 % of a lone row's time - and by the way of a pass's first logits, not by memory: of a row's 26 us in an earlier
// build the pass that lays sums took 11, the sums over the bins 1, each pass that collects 4.  50304 logits in fp32: one row, top-p 24.8 us; 64 rows, top-k of 50, top-p and
// min-p 18.2 us, with fp16 logits 18.0; 512 rows of different settings 61 us, 1.7 TB/s.  A row's logits do not fit its registers, and a row on more than one CU would
// need a workspace of the caller's.
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include "sample_params.h"
#include "device_utils.h"

// A token's bin and its place in it are worked out in several places and have to be the same numbers in all of them: no product joins a sum but where
// fma() says so.
#pragma clang fp contract(off)

namespace cfpp {

typedef unsigned long long u64;

constexpr int kBins = 4096, kCut = 2048, kList = 512, kBinsToOctave = 32;     // kCut: bins of a bin's own histogram
// Bins above the reference; as many below it.  (512 of 2048: 0.4 us less, but where the histogram of one of 64 rows is laid again 59.3 us for 35.0.)
constexpr float kAbove = 2048.f;
// Rows up to which a row has a CU's 1024 threads; more, and two rows share it.  (No filter: one row 25.6 us, with 512 threads 29.9; 64 rows 27.7 and 33.4; 512 rows, each
// with 1024 threads, 65.7, with 512 51.3.)
constexpr int kSampleOneEach = 256;

// 2^(63 - k / 32), to the nearest
__constant__ const u64 kOctave[kBinsToOctave] = {
    0x8000000000000000ull, 0x7d41d96db915019dull, 0x7a92be8a92436616ull, 0x77f25ccdee6d7ae6ull, 0x75606373ee921c97ull, 0x72dc8373be41a454ull, 0x70666f76154a7089ull,
    0x6dfddbcbed791babull, 0x6ba27e656b4eb57aull, 0x69540ec8f895722dull, 0x6712460a8fc24072ull, 0x64dcdec3371793d1ull, 0x62b39508aa836d6full, 0x6096266533384a2bull,
    0x5e8451cfac061b5full, 0x5c7dd7a3b17dcf75ull, 0x5a827999fcef3242ull, 0x5891fac0e95612c8ull, 0x56ac1f752150a563ull, 0x54d0ad5a753e077cull, 0x52ff6b54d8a89c75ull,
    0x513821818624b40cull, 0x4f7a993048d088d7ull, 0x4dc69cdceaa72a9cull, 0x4c1bf828c6dc54b8ull, 0x4a7a77d47f7b84b1ull, 0x48e1e9b9d588e19bull, 0x47521cc5a2e6a9e0ull,
    0x45cae0f1f545eb73ull, 0x444c0740496d4294ull, 0x42d561b3e6243d8aull, 0x4166c34c5615d0ecull};

// larger logits have larger keys (no NaN)
__device__ __forceinline__ unsigned sample_key(float v)
{
    const unsigned b = __float_as_uint(v + 0.f);           // (both zeros are equal)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float sample_of_key(unsigned k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
// the order as one number, the first the smallest
__device__ __forceinline__ u64 sample_place(unsigned key, int i) { return (u64)~key << 32 | (unsigned)i; }
__device__ __forceinline__ float sample_of_place(u64 place) { return sample_of_key(~(unsigned)(place >> 32)); }

template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned dpp_add(unsigned v)
{
    return v + (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 dpp_add(u64 v)
{
    const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)v, CTRL, ROWS, 0xF, false);
    const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)(v >> 32), CTRL, ROWS, 0xF, false);
    return v + ((u64)hi << 32 | lo);
}
// the sum over this lane and those before it, of 16 and of 64 lanes
template <class V>
__device__ __forceinline__ V row_scan(V v)
{
    v = dpp_add<0x111, 0xF>(v);                            // from 1, 2, 4, 8 lanes before
    v = dpp_add<0x112, 0xF>(v);
    v = dpp_add<0x114, 0xF>(v);
    return dpp_add<0x118, 0xF>(v);
}
template <class V>
__device__ __forceinline__ V wave_scan(V v)
{
    v = row_scan(v);
    v = dpp_add<0x142, 0xA>(v);                            // the sum of the row before to rows 1 and 3, of the first half to the second
    return dpp_add<0x143, 0xC>(v);
}
__device__ __forceinline__ unsigned lane_value(unsigned v, int lane) { return (unsigned)__builtin_amdgcn_readlane((int)v, lane); }
// a value that all lanes have, in scalar registers
__device__ __forceinline__ unsigned uniform(unsigned v) { return (unsigned)__builtin_amdgcn_readfirstlane((int)v); }
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float uniform(float v) { return __uint_as_float(uniform(__float_as_uint(v))); }
__device__ __forceinline__ u64 uniform(u64 v) { return (u64)uniform((unsigned)(v >> 32)) << 32 | uniform((unsigned)v); }
__device__ __forceinline__ double uniform(double v) { return __longlong_as_double((long long)uniform((u64)__double_as_longlong(v))); }
__device__ __forceinline__ u64 lane_value(u64 v, int lane) { return (u64)lane_value((unsigned)(v >> 32), lane) << 32 | lane_value((unsigned)v, lane); }

template <int T>
struct SampleShared {
    static constexpr int kWaves = T / 64;
    u64 mass[kBins];                                       // sums of the bins, then those of all bins before
    unsigned count[kBins];
    u64 place[kList], weight[kList], ahead[kList];         // the list's tokens; their weights; the sum of those before, of the same bin
    unsigned rank[kList];
    u64 wave_mass[2][kWaves];
    unsigned wave_count[2][kWaves];
    float wave_max[2][kWaves];
    int n_list, bin, other;
    unsigned below, before_count, lo, hi, kept, first;
    u64 before_mass, value, found_place, sum_of_kept;
    u64 octave[kBinsToOctave];                             // kOctave
};

// Sums of a value over the workgroup: those of the threads before this one, and of all.  `turn` alternates, so that a second call need not wait for the first one's readers.
template <int T>
__device__ __forceinline__ void block_scan(SampleShared<T> &s, int turn, unsigned own_count, u64 own_mass, unsigned &count, u64 &mass, unsigned &all_count, u64 &all_mass)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned c = wave_scan(own_count);
    const u64 m = wave_scan(own_mass);
    if (lane == 63) { s.wave_count[turn][wave] = c; s.wave_mass[turn][wave] = m; }
    __syncthreads();
    const unsigned wc = row_scan(s.wave_count[turn][lane & (T / 64 - 1)]);
    const u64 wm = row_scan(s.wave_mass[turn][lane & (T / 64 - 1)]);
    all_count = lane_value(wc, T / 64 - 1);
    all_mass = lane_value(wm, T / 64 - 1);
    count = c - own_count + (wave ? lane_value(wc, wave - 1) : 0u);
    mass = m - own_mass + (wave ? lane_value(wm, wave - 1) : 0ull);
}
template <int T>
__device__ __forceinline__ float block_max(SampleShared<T> &s, int turn, float v)
{
    v = wave_max(v);
    if ((threadIdx.x & 63) == 0) s.wave_max[turn][threadIdx.x >> 6] = v;
    __syncthreads();
    return uniform(wave_max(s.wave_max[turn][threadIdx.x & (T / 64 - 1)]));
}
// a b + c, with c in registers that stay as they are (the compiler copies a constant for every sum that it may overwrite)
__device__ __forceinline__ double fma_keep(double a, double b, double c)
{
    double r;
    asm("v_fma_f64 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
__device__ __forceinline__ float max4(f32x4 v, float m) { return fmaxf(fmaxf(m, fmaxf(v[0], v[1])), fmaxf(v[2], v[3])); }

// A row's logits, four to a thread that follow one another; what lies behind the row as minus infinity, a NaN stays one.  FEW: of less than four
template <int T, bool F16, bool FEW>
struct SampleRow {
    static constexpr int kThreads = T, STEP = 4 * T;
    const void *at;
    int vocab;
    // (the last ones of the row in place of those behind it; rows may begin at any logit)
    __device__ __forceinline__ f32x4 raw(int i) const
    {
        typedef std::conditional_t<F16, _Float16, float> L;
        typedef L L4 __attribute__((ext_vector_type(4), aligned(sizeof(L))));
        if constexpr (FEW) {
            const CFPP_GLOBAL L *p = (const CFPP_GLOBAL L *)at;
            const float last = (float)p[vocab - 1];
            return f32x4{(float)p[0], (float)p[min(1, vocab - 1)], last, last};         // (the histogram's reference is one of the row's)
        } else {
            const L4 x = *(const CFPP_GLOBAL L4 *)((const CFPP_GLOBAL char *)at + (unsigned)min(i, vocab - 4) * (unsigned)sizeof(L));
            return f32x4{(float)x[0], (float)x[1], (float)x[2], (float)x[3]};
        }
    }
    // first(the first vector, which may hold logits twice or stand for ones behind the row), then f(four logits, index of the first) for all; all threads of the workgroup
    // together.  One vector is on its way while another is looked at: two or four of each are no faster (one row 25.6 and 25.7 us for 24.8, 64 rows with a top-k of 50 18.5 and
    // 18.4 for 17.8; 512 rows 51.3 and 58.2 for 53.0, with a top-k of 50 39.6 and 42.7 for 36.7)
    template <class First, class Fn>
    __device__ __forceinline__ void each(First first, Fn f) const
    {
        int own = 4 * (int)threadIdx.x;
        asm volatile("" : "+v"(own));                      // (so that no pass keeps its addresses in registers for the next one)
        f32x4 next = raw(own);
        first(next);
#pragma unroll 1
        for (int at = 0; at < vocab; at += STEP) {
            const int i = at + own;
            f32x4 v = next;
            next = raw(i + STEP);                          // (past the end: the last ones again)
            if (at + STEP > vocab) {                       // (uniform) the row's end: what was loaded is `off` logits too early
                const int off = FEW ? 0 : max(i - (vocab - 4), 0);
                const f32x4 y = v;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    float z = y[c];
#pragma unroll
                    for (int k = c + 1; k < 4; ++k) z = off == k - c ? y[k] : z;
                    v[c] = i + c < vocab ? z : -INFINITY;
                }
            }
            f(v, i);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    template <class Fn>
    __device__ __forceinline__ void each(Fn f) const
    {
        each([](auto &) {}, f);
    }
};

struct SampleHow {
    float tau, top_p, min_p, uniform;
    int top_k;
    __device__ __forceinline__ double slope() const { return 1.4426950408889634 * kBinsToOctave / (double)tau; }       // bins to a logit
};

// Whether only the tokens that equal the largest weigh anything: it is infinite, or one step of the largest number is more bins than there are
__device__ __forceinline__ bool sample_level(const SampleHow &how, float most) { return most == INFINITY || (double)fabsf(most) * how.slope() > 0x1p40; }

// Below this temperature, where a bin is less than 2^-100 of a logit, a row is taken kUnsteep times as large, logits and temperature: 32 bits do not reach the slope.
// Tokens that weigh anything are so close to a largest one so small that this is exact; others may become minus infinity.
constexpr float kSteep = 0x1p-95f, kUnsteep = 0x1p64f;

// The token of a row.  !KNOWN: `most`, the largest logit, is found here.  false: only the tokens that equal it weigh anything, or the row is a steep one; nothing
// is answered then.  KNOWN: the logits are fit_one() of the row's, and `most` is the largest of them.  s.mass and s.count are zero.
template <bool KNOWN, class Row, class Fit, class Answer>
__device__ __forceinline__ bool sample_row(SampleShared<Row::kThreads> &s, const Row &R, const SampleHow &how, Fit fit_one, float &most, Answer answer)
{
    constexpr int T = Row::kThreads, EACH = kBins / T, EACH_CUT = kCut / T;
    const int tid = threadIdx.x;
    // for fp32 at least so many bins that infinite differences stay infinite (the largest finite one is no thousandth of a bin then), at most so many, of a steep row,
    // that none becomes NaN
    const double bounded = uniform(fmin(fmax(how.slope(), 1e-42), 1e37)), slope = how.tau < INFINITY ? bounded : 0.0;     // (none: all logits weigh the same)
    // Differences of logits are halved: two finite logits may be further apart than the type reaches.  (What the smallest numbers lose is 2^-150 of the slope.)
    const float slope_of_half = uniform((float)(2.0 * bounded));
    float ref = 0.f, half_ref = 0.f;                       // its bin is kAbove
    double shift = 0.0;
    auto refer = [&](float to) {
        ref = to;
        half_ref = uniform(0.5f * ref);
        shift = uniform((double)ref * slope + ((double)kAbove - 0.5));
    };
    auto depth_of = [&](float v) { return fmaf(fmaf(v, -0.5f, half_ref), slope_of_half, kAbove); };            // (never rises with v; infinite for minus infinity)
    auto bin_of = [&](float v) { return (int)__builtin_amdgcn_fmed3f(depth_of(v), 0.f, kBins - 1.f); };          // (no NaN)
    auto in_bins = [](float depth) { return __float_as_uint(depth) < __float_as_uint((float)kBins); };            // (neither less than zero nor NaN)
    // 2^(-f / 32) in multiples of 2^-44, f the token's place in its bin from its middle: -1/2 to 1/2
    auto weight_in = [&](float v, int bin) {
        const double f = fma((double)v, -slope, shift) - (double)bin;
        double p = fma_keep(161364.9745385843, f, -29798760.585014474);        // (fitted to the least relative error, 2^-43.5)
        p = fma_keep(p, f, 4127059964.301119);
        p = fma_keep(p, f, -381061692379.1814);
        p = fma_keep(p, f, 17592186044416.0);
        return (u64)__double_as_longlong(p + 4503599627370496.0) - 0x4330000000000000ull;      // (2^52 more, and the last bits are the number)
    };
    int top_bin = 0;                                       // the largest logit's
    auto scaled = [&](int bin, u64 sum) {                  // sum 2^((top_bin - bin) / 32), cut off
        const int below = bin - top_bin;                   // (of a bin that has something, not less than zero)
        return __umul64hi(sum << 1, s.octave[below & (kBinsToOctave - 1)]) >> min((unsigned)below / kBinsToOctave, 63u);
    };
    // a token's weight over a sum (its own, not the difference of two sums that are cut off)
    auto part_of = [&](u64 place, u64 of) {
        const float v = sample_of_place(place);
        const int bin = bin_of(v), below = bin - top_bin;
        return (float)(ldexp((double)weight_in(v, bin) * (double)s.octave[below & (kBinsToOctave - 1)], -63 - below / kBinsToOctave) / (double)of);
    };
    auto fit = [&](f32x4 v) {
        if constexpr (KNOWN)
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] = fit_one(v[c]);
        return v;
    };
    // f of the tokens that pick() is true of; a vector of four without any costs nothing more
    auto some = [&](auto pick, auto f) {
        R.each([&](f32x4 x, int i) {
            const f32x4 v = fit(x);
            bool on[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) on[c] = pick(v[c]);
            if (!(on[0] || on[1] || on[2] || on[3])) return;
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (on[c] && v[c] > -INFINITY) f(v[c], i + c);  // (no NaN either)
        });
    };
    bool by_k = how.top_k > 0 && how.top_k < R.vocab;
    const bool by_p = how.top_p < 1.f, by_m = how.min_p > 0.f, small = R.vocab <= kList;
    int n_k = by_k ? how.top_k : R.vocab;                  // (at most so many: minus infinities are found later)
    u64 k_place = ~0ull;                                   // of the last token that top-k keeps

    // kStageAll: the few tokens that top-k leaves, and some more, are in the list: all filters there (64 rows of 50304, here / the other way: a k of 50 18.4 / 34.9 us, 320 32.0 / 35.4,
    // 400 35.0 / 35.3, 480 38.1 / 35.4).  Otherwise the places where top-k ends, where top-p or min-p does, whichever comes first, and of the draw, one after the other
    enum { kStageAll, kStageK, kStageCut, kStageDraw };
    const int behind_k = by_p || by_m ? kStageCut : kStageDraw;
    int stage = small || (by_k && n_k <= kList * 3 / 4) ? kStageAll : by_k ? kStageK : behind_k;
    enum { kNone, kCounts, kMasses, kBoth };
    int built = kNone;                                     // what the histogram holds: running numbers or sums of the bins before
    bool dirty = false, known = KNOWN, cut = false;        // the histogram is to be cleared; `most` is known; top-p or min-p has cut
    unsigned kept = 0, all_count = 0;
    u64 mass = 0, all_mass = 0;                            // mass: of what is kept; all_: of all bins
    const double least = uniform(by_m ? log2((double)fminf(how.min_p, 1.f)) : 0.0);     // of a kept token's logarithm, by min-p
    int turn = 0;
    auto clear = [&]() {
        __syncthreads();
        for (int b = tid; b < kBins; b += T) { s.count[b] = 0u; s.mass[b] = 0ull; }
        __syncthreads();
    };
    auto drawn = [&](u64 sum) {
        const double u = how.uniform;
        return min((u64)floor(fmin(u > 0.0 ? u : 0.0, 1.0) * (double)sum) + 1ull, sum);
    };
    auto level = [&](float v) { return ((double)v - (double)most) * slope * (1.0 / kBinsToOctave); };
    if constexpr (KNOWN) {
        refer(most);
        top_bin = uniform(bin_of(most));
    }
    for (;;) {
        const bool counts = stage <= kStageK;
        if ((counts ? built != kCounts && built != kBoth : built != kMasses) && !(small && known)) {
            // Where top-k ends among many the sums are laid along with the numbers, so that no second pass has to lay those of the tokens it keeps: all bins behind the one where it ends
            // have the same sum then, that of what is kept (a k of 600: 64 rows of 50304 41.8 -> 37.0 us, 512 rows 88.4 -> 76.5).
            const bool both = stage == kStageK;
            if (dirty) clear();
            dirty = true;
            float seen = -INFINITY;
            unsigned n = 0;                                // tokens
            const bool number = !by_k && stage == kStageDraw && !cut;
            // a pass that lays the histogram; the first one from the largest of the first logits on
            auto lay = [&](auto first) {
                R.each([&](auto &x) {
                    if constexpr (decltype(first)::value) {
                        const float m = block_max(s, 0, 4 * tid < R.vocab ? max4(x, -INFINITY) : -INFINITY);
                        refer(fabsf(m) < INFINITY ? m : 0.f);
                    }
                }, [&](f32x4 x, int i) {
                    f32x4 v = fit(x);
                    if constexpr (decltype(first)::value) seen = max4(v, seen);
                    if (small) return;                     // (uniform)
                    if (counts) {                          // (uniform)
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            if (v[c] > -INFINITY) atomicAdd(&s.count[bin_of(v[c])], 1u);
                        if (!both) return;
                    } else if (by_k) {                     // (uniform)
#pragma unroll
                        for (int c = 0; c < 4; ++c) v[c] = sample_place(sample_key(v[c]), i + c) > k_place ? -INFINITY : v[c];
                    }
                    if (number)                            // (uniform)
#pragma unroll
                        for (int c = 0; c < 4; ++c) n += v[c] > -INFINITY;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const float y = depth_of(v[c]);
                        const int b = (int)y;
                        const u64 w = weight_in(v[c], b);
                        if (in_bins(y)) atomicAdd(&s.mass[b], w);
                        if (c & 1) __builtin_amdgcn_sched_barrier(0);          // (four side by side take more registers than there are)
                    }
                });
            };
            if (!known) {
                lay(std::true_type{});
                most = block_max(s, 1, seen);
                known = true;
                if (most == -INFINITY) {
                    if (tid == 0) answer(-1, 0.f, 0);
                    return true;
                }
                if (how.tau < kSteep || sample_level(how, most)) return false;
                // (uniform) out of reach, or below the zero that stands in for first logits that are all masked: the histogram from the largest on
                if (depth_of(most) < 0.f || depth_of(most) > kAbove) {
                    refer(most);
                    if (!small) {
                        n = 0;
                        clear();
                        lay(std::false_type{});
                    }
                }
                top_bin = uniform(bin_of(most));
            } else {
                lay(std::false_type{});
            }
            __syncthreads();
            if (!small) {
                const bool masses = !counts || both;
                unsigned c[EACH], c0 = 0, c1;
                u64 m[EACH], m0 = 0, m1;
#pragma unroll
                for (int k = 0; k < EACH; ++k) {
                    const int b = EACH * tid + k;
                    c[k] = c0;
                    m[k] = m0;
                    if (counts) c0 += s.count[b];
                    if (!masses) continue;
                    if (const u64 in = s.mass[b]) m0 += scaled(b, in);         // (most of the bins have nothing)
                }
                block_scan(s, turn ^= 1, c0, m0, c1, m1, all_count, all_mass);
#pragma unroll
                for (int k = 0; k < EACH; ++k) {
                    if (counts) s.count[EACH * tid + k] = c1 + c[k];
                    if (masses) s.mass[EACH * tid + k] = m1 + m[k];
                }
                if (masses) all_mass = uniform(all_mass);
                if (masses && !cut) {
                    mass = all_mass;
                    kept = both ? min((unsigned)n_k, all_count) : (unsigned)n_k;
                    if (number) {
                        unsigned none;
                        u64 none_of, no_sum;
                        block_scan(s, turn ^= 1, n, 0ull, none, none_of, kept, no_sum);
                    }
                }
                __syncthreads();
                built = both ? kBoth : counts ? kCounts : kMasses;
                if (counts && all_count <= (unsigned)n_k) {                    // (uniform) top-k keeps all that there is
                    n_k = (int)all_count;
                    by_k = false;
                    if (all_count > (unsigned)kList) {
                        stage = behind_k;
                        if (both) built = kMasses;
                        continue;
                    }
                    stage = kStageAll;
                }
            }
        }
        // where the target is reached: the bin, and what stands before it
        u64 target = (u64)n_k;
        if (stage == kStageCut) target = by_p ? min(max((u64)ceil((double)how.top_p * (double)all_mass), 1ull), all_mass) : 1ull;
        if (stage == kStageDraw) target = drawn(mass);
        target = uniform(target);
        if (small) {
            if (tid == 0) s.bin = kBins;
        } else {
#pragma unroll
            for (int k = 0; k < EACH; ++k) {
                const int b = EACH * tid + k;
                const u64 from = counts ? s.count[b] : s.mass[b], to = counts ? (b + 1 < kBins ? s.count[b + 1] : all_count) : b + 1 < kBins ? min(s.mass[b + 1], all_mass) : all_mass;
                if (from < target && target <= to) {
                    s.bin = b; s.other = (int)min(to, (u64)kBins); s.before_count = (unsigned)from; s.before_mass = from;
                }
            }
        }
        if (tid == 0) { s.n_list = 0; s.lo = ~0u; s.hi = 0u; s.below = 0u; }
        if (tid < kList) { s.rank[tid] = 0u; s.ahead[tid] = 0ull; }
        __syncthreads();
        const int bin = uniform(s.bin);
        unsigned before_count = uniform(s.before_count);
        u64 before_in = 0;
        const u64 before_mass = uniform(s.before_mass);    // before_in: of the bin's own tokens, unscaled
        const bool all = stage == kStageAll;
        if (all && !small && s.other > kList) {            // (uniform) more tokens than the list has places for
            stage = kStageK;
            __syncthreads();
            continue;
        }
        bool by_list = true;                               // whether the cut is to be found in a list
        unsigned kept_m = ~0u;
        u64 mass_m = ~0ull;
        if (stage == kStageCut && by_m) {
            // min-p ends in one of the bins m_lo .. m_hi (fp32 and fp64 may put a logit on either side of a border).  Where top-p ends in a bin before them, min-p
            // keeps more; otherwise the tokens before and in them are numbered and added up.
            const double at = ((double)ref - (double)most) * slope + (double)kAbove - least * kBinsToOctave;
            const int m_lo = (int)fmin(fmax(at - 0.01, 0.0), (double)kBins), m_hi = (int)fmin(fmax(at + 0.01, 0.0), (double)kBins);
            by_list = by_p && bin <= m_hi;
            if (!by_p || bin >= m_lo) {                    // (uniform)
                // (behind the last bin nothing has a weight that counts, but it does as a token kept)
                const float from = m_lo < kBins ? (float)m_lo : (float)(at - 0.01), to = m_lo < kBins ? (float)(m_hi + 1) : (float)(at + 0.01);
                unsigned n = 0;
                u64 in[2] = {0, 0};
                some([&](float v) {
                    const float y = depth_of(v);
                    n += y < from;
                    return y >= from && y < to;
                }, [&](float v, int i) {
                    if ((by_k && sample_place(sample_key(v), i) > k_place) || !(level(v) >= least)) return;
                    const int b = (int)depth_of(v);
                    ++n;
                    if (b < kBins) in[b - m_lo] += weight_in(v, b);
                });
                unsigned none;
                u64 none_of;
                block_scan(s, turn ^= 1, n, in[0], none, none_of, kept_m, in[0]);
                block_scan(s, turn ^= 1, 0u, in[1], none, none_of, n, in[1]);
                kept_m = min(kept_m, (unsigned)n_k);       // (those before the bins are numbered wherever top-k ends)
                mass_m = m_lo < kBins ? s.mass[m_lo] : all_mass;
                if (m_lo < kBins && in[0]) mass_m = s.mass[m_lo] + scaled(m_lo, in[0]);
                if (m_hi < kBins && m_hi > m_lo && in[1]) mass_m = s.mass[m_hi] + scaled(m_hi, in[1]);
                mass_m = min(mass_m, all_mass);            // (what top-k keeps)
            }
        }
        if (by_list) {
            // what is looked at: the bin; keys k_lo .. k_hi of it; the indexes i_lo .. i_hi of the key k_lo
            int depth = 0, i_lo = 0, i_hi = 0;
            unsigned k_lo = 0, k_hi = 0;
            // (where numbers are asked for the first and last bins have all that lies outside of them)
            const float from = all || (counts && bin == 0) ? -INFINITY : (float)bin, to = counts && bin >= kBins - 1 ? NAN : (float)(bin + 1);
            // what is near lies between two logits, which two comparisons tell for nearly all others: the bounds are a hundredth of a bin further than fp32 puts anything
            auto logit_at = [&](double depth) { return uniform((float)((double)ref - (depth - (double)kAbove) / slope)); };
            const float v_lo = to == to ? logit_at((double)to + 0.01) : -INFINITY, v_hi = from > -INFINITY ? logit_at((double)from - 0.01) : INFINITY;
            auto near = [&](float v) { return v >= v_lo && v <= v_hi; };
            auto is_near = [&](float v) {
                const float y = depth_of(v);
                return y >= from && !(y >= to);
            };
            auto inside = [&](float v, int i) {
                if (!is_near(v)) return false;
                if (depth > 0) {
                    const unsigned key = sample_key(v);
                    if (key < k_lo || key > k_hi || (depth == 2 && (i < i_lo || i > i_hi))) return false;
                }
                return counts || !by_k || sample_place(sample_key(v), i) <= k_place;
            };
            for (int round = 0;; ++round) {
                auto collect = [&](float v, int i) {
                    if (!inside(v, i)) return;
                    const int at = atomicAdd(&s.n_list, 1);
                    if (at >= kList) return;
                    s.place[at] = sample_place(sample_key(v), i);
                };
                if (stage == kStageCut && round == 0) {    // (what stands before a token that is kept is kept)
                    unsigned below = 0;
                    some([&](float v) { below += v > v_hi; return near(v); }, [&](float v, int i) {
                        below += depth_of(v) < from;
                        collect(v, i);
                    });
                    below = wave_scan(below);
                    if ((tid & 63) == 63 && below) atomicAdd(&s.below, below);
                } else {
                    some(near, collect);
                }
                __syncthreads();
                if (stage == kStageCut && round == 0) before_count = uniform(s.below);
                if (s.n_list <= kList || round == 4) break;                    // (a cut by a logit's 32 bits takes three rounds at most, by the index one)
                // too many for the list: a histogram of what is inside
                if (depth == 0) {
                    some(near, [&](float v, int i) {
                        if (!inside(v, i)) return;
                        const unsigned key = sample_key(v);
                        atomicMin(&s.lo, key);
                        atomicMax(&s.hi, key);
                    });
                    __syncthreads();
                    k_lo = uniform(s.lo); k_hi = uniform(s.hi);
                    depth = 1;
                }
                if (depth == 1 && k_lo == k_hi) { depth = 2; i_lo = 0; i_hi = R.vocab - 1; }
                const unsigned span = depth == 1 ? k_hi - k_lo : (unsigned)(i_hi - i_lo);
                int shift_by = 0;
                while (span >> shift_by >= (unsigned)kCut) ++shift_by;
                clear();
                built = kNone;
                some(near, [&](float v, int i) {
                    if (!inside(v, i)) return;
                    const unsigned b = (depth == 1 ? k_hi - sample_key(v) : (unsigned)(i - i_lo)) >> shift_by;
                    atomicAdd(&s.count[b], 1u);
                    if (!counts) atomicAdd(&s.mass[b], weight_in(v, bin));
                });
                __syncthreads();
                unsigned c = 0, none;
                u64 m = 0, none_of;
#pragma unroll
                for (int k = 0; k < EACH_CUT; ++k) { c += s.count[EACH_CUT * tid + k]; m += s.mass[EACH_CUT * tid + k]; }
                block_scan(s, turn ^= 1, c, m, c, m, none, none_of);
                c += before_count;
                m += before_in;
#pragma unroll
                for (int k = 0; k < EACH_CUT; ++k) {
                    const unsigned cb = s.count[EACH_CUT * tid + k];
                    const u64 mb = s.mass[EACH_CUT * tid + k];
                    if (counts ? c < target && target <= c + cb : before_mass + scaled(bin, m) < target && target <= before_mass + scaled(bin, m + mb)) {
                        s.other = EACH_CUT * tid + k; s.before_count = c; s.value = m;
                    }
                    c += cb; m += mb;
                }
                if (tid == 0) s.n_list = 0;
                __syncthreads();
                before_count = uniform(s.before_count);
                before_in = uniform(s.value);
                const unsigned b = uniform((unsigned)s.other);
                if (depth == 1) {
                    k_hi -= b << shift_by;
                    k_lo = max(k_lo, k_hi - min(k_hi, (1u << shift_by) - 1u));
                } else {
                    i_lo += (int)(b << shift_by);
                    i_hi = min(i_hi, i_lo + (1 << shift_by) - 1);
                }
            }
            // every token counts those before it; where there are threads enough, several for a token
            const int n = uniform(min(s.n_list, kList));
            if (tid < n) {
                const float v = sample_of_place(s.place[tid]);
                const int b = bin_of(v);
                u64 w = weight_in(v, b);
                if (counts && !(depth_of(v) < (float)kBins)) w = 0ull;         // (the last bin has all that lies behind it)
                if (all) w = scaled(b, w);
                s.weight[tid] = w;
            }
            __syncthreads();
            int wide = 64;
            while (wide < n) wide <<= 1;                   // (a power of two up to kList, which divides the threads)
            const int mine = tid & (wide - 1), share = (n + T / wide - 1) / (T / wide), j0 = tid / wide * share, j1 = min(j0 + share, n);
            u64 place = ~0ull, w = 0ull;
            if (mine < n) {
                place = s.place[mine];
                w = s.weight[mine];
                unsigned rank = 0;
                u64 ahead = 0;
#pragma unroll 4
                for (int j = j0; j < j1; ++j) {
                    const bool before = s.place[j] < place;
                    rank += before;
                    ahead += before ? s.weight[j] : 0ull;
                }
                if (rank) {
                    atomicAdd(&s.rank[mine], rank);
                    atomicAdd(&s.ahead[mine], ahead);
                }
            }
            if (tid == 0) s.kept = 0u;
            __syncthreads();
            // one thread to a token from here on: its number in the order, and the sums up to it and with it
            const bool token = tid < n;
            unsigned rank = 0;
            u64 sum = 0, with = 0;
            if (token) {
                rank = before_count + s.rank[tid];
                sum = s.ahead[tid];
                with = sum + w;
                if (!all && !counts) {
                    sum = before_mass + scaled(bin, before_in + sum);
                    with = before_mass + scaled(bin, before_in + with);
                }
            }
            if (all) {
                n_k = min(n_k, n);                         // (tokens behind the first n_k are in the list too)
                rank = tid < n ? s.rank[tid] : 0u;
                if (token && rank == (unsigned)n_k - 1u) s.value = with;
                __syncthreads();
                u64 p_target = ~0ull;
                if (by_p) p_target = max((u64)ceil((double)how.top_p * (double)s.value), 1ull);
                const bool ok = token && rank < (unsigned)n_k && sum < p_target && (!by_m || level(sample_of_place(place)) >= least);
                const unsigned long long of_wave = __ballot(ok);
                if ((tid & 63) == 0 && of_wave) atomicAdd(&s.kept, (unsigned)__popcll(of_wave));
                __syncthreads();
                const unsigned n_kept = s.kept;            // (the first of the order)
                if (token && rank == n_kept - 1u) s.sum_of_kept = with;
                __syncthreads();
                const u64 in_all = s.sum_of_kept, at = drawn(in_all);
                if (ok && sum < at && at <= with) answer((int)(unsigned)place, part_of(place, in_all), (int)n_kept);
                return true;
            }
            if (token && (counts ? rank + 1u == target : sum < target && target <= with)) {
                if (built == kBoth) with = s.mass[bin] + scaled(bin, with);
                s.found_place = place; s.value = with; s.kept = rank + 1u;
            }
            __syncthreads();
        }
        if (stage == kStageK) {
            k_place = uniform(s.found_place);
            if (built == kBoth) {                          // (otherwise laid anew)
                mass = all_mass = uniform(s.value);
                kept = (unsigned)n_k;
                built = kMasses;
            }
            stage = behind_k;
        } else if (stage == kStageCut) {
            kept = kept_m;
            mass = mass_m;
            if (by_list) {
                kept = uniform(min(kept, s.kept));
                mass = uniform(min(mass, s.value));
            }
            cut = true;
            stage = kStageDraw;
        } else {
            if (tid == 0) answer((int)(unsigned)s.found_place, part_of(s.found_place, mass), (int)kept);
            return true;
        }
        __syncthreads();                                   // (what was found has been read)
    }
}

template <int T, bool F16, bool FEW>
__global__ void __launch_bounds__(T, 4) k_sample(SampleParams P)
{
    __shared__ SampleShared<T> s;
    const int tid = threadIdx.x, row = blockIdx.x;
    int at = row;
    if (P.pos) {                                           // (uniform)
        at = *P.pos;
        if (at < 0 || at >= P.max_seq) return;
    }
    const SampleRow<T, F16, FEW> R{static_cast<const char *>(P.logits) + (size_t)row * P.stride * (F16 ? 2 : 4), P.vocab};
    SampleHow how{P.temperature ? P.temperature[row] : 1.f, P.top_p ? P.top_p[row] : 1.f, P.min_p ? P.min_p[row] : 0.f, P.uniform[at], P.top_k ? P.top_k[row] : 0};
    int shown = -1;                                        // tokens that the filters keep, where that is known beforehand
    auto answer = [&](int token, float prob, int kept) {
        if (P.pos) {
            P.tokens[at + 1] = max(token, 0);
            *P.pos = at + 1;
            return;
        }
        P.tokens[row] = token;
        if (P.probs) P.probs[row] = prob;
        if (P.kept) P.kept[row] = shown >= 0 ? shown : kept;
    };
    for (int b = tid; b < kBins; b += T) { s.count[b] = 0u; s.mass[b] = 0ull; }
    if (tid < kBinsToOctave) s.octave[tid] = kOctave[tid];
    if (!(how.tau > 0.f) || how.top_k == 1 || how.top_p <= 0.f) {              // (uniform) the first of the order
        float most = -INFINITY;
        int first = 0x7fffffff;
        R.each([&](f32x4 v, int i) {
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (v[c] > most) { most = v[c]; first = i + c; }               // (a thread's indexes rise)
        });
        if (tid == 0) s.first = 0x7fffffffu;
        const float all = block_max(s, 0, most);
        if (most == all && first != 0x7fffffff) atomicMin(&s.first, (unsigned)first);
        __syncthreads();
        if (tid == 0) {
            if (s.first == 0x7fffffffu) answer(-1, 0.f, 0);
            else answer((int)s.first, 1.f, 1);
        }
        return;
    }
    float most = -INFINITY;
    if (sample_row<false>(s, R, how, [](float v) { return v; }, most, answer)) return;
    // Either the row is steep, or only the tokens that equal the largest weigh anything.  Where that is infinite the others are no part of the order; where the temperature is
    // so low they are, and are kept where nothing cuts them off.
    if (most < INFINITY && !(how.top_p < 1.f) && !(how.min_p > 0.f)) {         // (uniform)
        unsigned n = 0, none, valid;
        u64 none_of, no_sum;
        R.each([&](f32x4 v, int) {
#pragma unroll
            for (int c = 0; c < 4; ++c) n += v[c] > -INFINITY;
        });
        block_scan(s, 0, n, 0ull, none, none_of, valid, no_sum);
        shown = how.top_k > 0 ? min(how.top_k, (int)valid) : (int)valid;
    }
    __syncthreads();
    for (int b = tid; b < kBins; b += T) { s.count[b] = 0u; s.mass[b] = 0ull; }
    __syncthreads();
    const bool steep = !sample_level(how, most);
    const float top = most;
    how.tau = steep ? how.tau * kUnsteep : 1.f;
    most = steep ? most * kUnsteep : 0.f;
    sample_row<true>(s, R, how, [=](float v) { return steep ? v * kUnsteep : v == top ? 0.f : -INFINITY; }, most, answer);
}

template <int T, bool F16>
static void launch_of(const SampleParams &P, int n_rows, hipStream_t s)
{
    if (P.vocab < 4) hipLaunchKernelGGL((k_sample<T, F16, true>), dim3(n_rows), dim3(T), 0, s, P);
    else hipLaunchKernelGGL((k_sample<T, F16, false>), dim3(n_rows), dim3(T), 0, s, P);
}

hipError_t launch_sample(const SampleParams &P, int type, int n_rows, hipStream_t s)
{
    const bool many = n_rows > kSampleOneEach;
    if (type == kLogitsF16) many ? launch_of<512, true>(P, n_rows, s) : launch_of<1024, true>(P, n_rows, s);
    else many ? launch_of<512, false>(P, n_rows, s) : launch_of<1024, false>(P, n_rows, s);
    return hipGetLastError();
}

}  // namespace cfpp
