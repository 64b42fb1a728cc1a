// The next token from a row of logits and a given random number: temperature, top-k, top-p, min-p.
//
// The row's order is larger logit first, lower index among equals; weights w = 2^((l - l_max) log2(e) / temperature).  Every filter keeps a beginning of the
// order - k tokens; as many as reach p of those k tokens' sum; those of at least min_p times the largest weight - and the token drawn is the first whose running sum
// passes u times the sum of what is kept.  So all of it is the same question: where, in the order, does a running count or a running sum reach a target?
//
// Nothing is sorted.  A histogram over (l_max - l) in steps of 2^(1/64) of a weight, 4096 bins of counts and of sums in LDS, says in which bin that is; the bin's
// tokens - tens of them for a usual row - are collected, and each finds its own place among them.  A bin of more than kList is cut again by the bits of its
// logits, and equal logits by their index, until few are left.
//
// Weights are whole multiples of 2^-45 of the largest, from a value with 2^-40 of relative error: their sums are exact in 64-bit integers whatever
// the order, so that results do not depend on which of a workgroup's wavefronts comes first, and a border between two tokens is where 64-bit arithmetic
// has it.  With weights in fp32 it would be up to 2^-24 off, which is another token once in some hundred thousand rows.
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include "sample_params.h"
#include "device_utils.h"

// A token's weight is worked out in several places and has to be the same number in all of them: no product joins a sum but where fma() says so.
#pragma clang fp contract(off)

namespace cfpp {

typedef unsigned long long u64;

constexpr int kSampleThreads = 1024, kSampleWaves = kSampleThreads / 64;
constexpr int kBins = 4096, kBinsEach = kBins / kSampleThreads, kList = 256;
constexpr float kBinsToOctave = 64.f;

// 2^t for t <= 0 as a multiple of 2^-45; zero below 2^-46
__device__ __forceinline__ u64 sample_weight(double t)
{
    t = fmax(t, -100.0);
    const double n = rint(t), f = t - n;                   // f in [-1/2, 1/2]
    // the series of 2^f: ln(2)^k / k!, its next term is below 2^-41
    double p = 7.054911620801122e-09;
    p = fma(p, f, 1.0178086009239699e-07);
    p = fma(p, f, 1.321548679014431e-06);
    p = fma(p, f, 1.525273380405984e-05);
    p = fma(p, f, 1.5403530393381609e-04);
    p = fma(p, f, 1.3333558146428441e-03);
    p = fma(p, f, 9.618129107628477e-03);
    p = fma(p, f, 5.550410866482158e-02);
    p = fma(p, f, 2.402265069591007e-01);
    p = fma(p, f, 6.931471805599453e-01);
    p = fma(p, f, 1.0);
    // (2^52 more, and the last bits of the fraction are the whole number)
    return __double_as_longlong(ldexp(p, (int)n + 45) + 4503599627370496.0) - 0x4330000000000000ull;
}

// larger logits have larger keys (no NaN)
__device__ __forceinline__ unsigned sample_key(float v)
{
    const unsigned b = __float_as_uint(v == 0.f ? 0.f : v);                    // (both zeros are equal)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float sample_of_key(unsigned k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

template <class T>
__device__ __forceinline__ T wave_scan(T v)                // the sum over this lane and those before
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const T o = __shfl_up(v, m, 64);
        if (lane >= m) v += o;
    }
    return v;
}

// four logits that follow one another, NaN as minus infinity; what lies behind the row likewise
template <bool F16>
struct SampleRow {
    const void *at;
    int vocab;
    bool infinite;                     // the largest logit is: weights of one and of zero
    __device__ __forceinline__ float value(float v) const
    {
        if (infinite) return v == INFINITY ? 0.f : -INFINITY;
        return v == v ? v : -INFINITY;
    }
    __device__ __forceinline__ f32x4 raw(int i) const
    {
        f32x4 v = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        if constexpr (F16) {
            typedef _Float16 h4 __attribute__((ext_vector_type(4), aligned(2)));
            const _Float16 *p = static_cast<const _Float16 *>(at) + i;
            if (i + 4 <= vocab) {                          // (rows may begin at any logit)
                const h4 x = *(const CFPP_GLOBAL h4 *)p;
                v = f32x4{(float)x[0], (float)x[1], (float)x[2], (float)x[3]};
            } else {
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (i + c < vocab) v[c] = (float)p[c];
            }
        } else {
            typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
            const float *p = static_cast<const float *>(at) + i;
            if (i + 4 <= vocab) {
                v = *(const CFPP_GLOBAL f4 *)p;
            } else {
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (i + c < vocab) v[c] = p[c];
            }
        }
        return v;
    }
    // f(logit, index) for this thread's tokens that are not minus infinity
    template <class Fn>
    __device__ __forceinline__ void each(Fn f) const
    {
        f32x4 next = raw(4 * (int)threadIdx.x);
        for (int i = 4 * (int)threadIdx.x; i < vocab; i += 4 * kSampleThreads) {
            const f32x4 x = next;
            next = raw(i + 4 * kSampleThreads);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const float v = value(x[c]);
                if (v > -INFINITY) f(v, i + c);
            }
        }
    }
};

// where in the order a target is reached
struct SampleFound { unsigned key; int index, count; u64 mass, weight; };      // count, mass: of the order up to this token and with it

struct SampleShared {
    unsigned count[kBins];
    u64 mass[kBins];
    unsigned key[kList];
    int index[kList];
    u64 weight[kList];
    u64 wave_mass[kSampleWaves];
    unsigned wave_count[kSampleWaves];
    float wave_max[kSampleWaves];
    int n_list, bin, bin_n;
    unsigned before_count, lo, hi;
    u64 before_mass;
    SampleFound found;
};

template <bool F16>
__global__ void __launch_bounds__(kSampleThreads) k_sample(SampleParams P)
{
    __shared__ SampleShared s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row = blockIdx.x;
    const SampleRow<F16> all{static_cast<const char *>(P.logits) + (size_t)row * P.stride * (F16 ? 2 : 4), P.vocab, false};
    const float tau = P.temperature ? P.temperature[row] : 1.f, top_p = P.top_p ? P.top_p[row] : 1.f, min_p = P.min_p ? P.min_p[row] : 0.f;
    const int top_k = P.top_k ? P.top_k[row] : 0;
    auto answer = [&](int token, float prob, int kept) {
        P.tokens[row] = token;
        if (P.probs) P.probs[row] = prob;
        if (P.kept) P.kept[row] = kept;
    };
    // the largest logit, and how many there are
    float most = -INFINITY;
    int valid = 0;
    all.each([&](float v, int) { most = fmaxf(most, v); ++valid; });
    most = wave_max(most);
    valid = wave_scan(valid);
    if (lane == 63) { s.wave_max[wave] = most; s.wave_count[wave] = (unsigned)valid; }
    if (tid == 0) s.lo = 0x7fffffffu;
    __syncthreads();
    valid = 0;
#pragma unroll
    for (int w = 0; w < kSampleWaves; ++w) { most = fmaxf(most, s.wave_max[w]); valid += (int)s.wave_count[w]; }
    if (valid == 0) {                                      // (uniform, as the ways out below)
        if (tid == 0) answer(-1, 0.f, 0);
        return;
    }
    if (!(tau > 0.f) || top_k == 1 || top_p <= 0.f) {      // the first of the order
        all.each([&](float v, int i) { if (v == most) atomicMin(&s.lo, (unsigned)i); });
        __syncthreads();
        if (tid == 0) answer((int)s.lo, 1.f, 1);
        return;
    }
    SampleRow<F16> R = all;
    if (most == INFINITY) {
        R.infinite = true;
        most = 0.f;
        valid = 0;                                         // (counted again)
        R.each([&](float, int) { ++valid; });
        valid = wave_scan(valid);
        __syncthreads();                                   // (wave_count has been read)
        if (lane == 63) s.wave_count[wave] = (unsigned)valid;
        __syncthreads();
        valid = 0;
        for (int w = 0; w < kSampleWaves; ++w) valid += (int)s.wave_count[w];
    }
    const double octaves = 1.4426950408889634 / (double)tau, least = min_p > 0.f ? log2((double)fminf(min_p, 1.f)) : -INFINITY;
    const float to_bin = fminf(fmaxf((float)octaves * kBinsToOctave, 1e-30f), 1e30f);          // (so that no product is none)
    auto level = [&](float v) { return ((double)v - (double)most) * octaves; };
    auto bin_of = [&](float v) { return (int)fminf((most - v) * to_bin, kBins - 1.f); };       // (never rises with v)
    const bool by_k = top_k > 0 && top_k < valid, by_p = top_p < 1.f;
    // the last token that top-k keeps
    unsigned k_key = 0;
    int k_index = 0x7fffffff;
    auto in_k = [&](unsigned key, int i) { return key > k_key || (key == k_key && i <= k_index); };

    enum { kStageK, kStageP, kStageDraw };
    unsigned kept = 0;
    u64 mass = 0;                                          // of what is kept
    bool built = false, cut = false;                       // cut: top-p has
    unsigned my_count = 0;                                 // running sums of the bins before this thread's
    u64 my_mass = 0, all_k = 0;                            // all_k: the sum of what top-k keeps
    for (int stage = by_k ? kStageK : by_p ? kStageP : kStageDraw; stage <= kStageDraw; ++stage) {
        if (stage == kStageP && !by_p) continue;
        const bool counts = stage == kStageK;
        u64 target = (u64)top_k;
        if (!built) {
            // counts of all tokens, or counts and sums of those that top-k and min-p keep
            __syncthreads();
            for (int b = tid; b < kBins; b += kSampleThreads) { s.count[b] = 0u; s.mass[b] = 0ull; }
            __syncthreads();
            u64 total = 0;                                 // over what top-k keeps
            if (counts) {
                R.each([&](float v, int) { atomicAdd(&s.count[bin_of(v)], 1u); });
            } else {
                R.each([&](float v, int i) {
                    if (!in_k(sample_key(v), i)) return;
                    const double t = level(v);
                    const u64 w = sample_weight(t);
                    total += w;
                    if (t < least) return;
                    const int b = bin_of(v);
                    atomicAdd(&s.count[b], 1u);
                    atomicAdd(&s.mass[b], w);
                });
            }
            __syncthreads();
            my_count = 0; my_mass = 0;
            for (int b = kBinsEach * tid; b < kBinsEach * (tid + 1); ++b) { my_count += s.count[b]; my_mass += s.mass[b]; }
            const unsigned c = wave_scan(my_count);
            const u64 m = wave_scan(my_mass), t = wave_scan(total);
            if (lane == 63) { s.wave_count[wave] = c; s.wave_mass[wave] = m; }
            __syncthreads();
            my_count = c - my_count; my_mass = m - my_mass;
            unsigned n = 0;
            u64 sum = 0;
#pragma unroll 4
            for (int w = 0; w < kSampleWaves; ++w) {
                if (w == wave) { my_count += n; my_mass += sum; }
                n += s.wave_count[w]; sum += s.wave_mass[w];
            }
            if (!cut) { kept = n; mass = sum; }
            __syncthreads();
            if (lane == 63) s.wave_mass[wave] = t;
            __syncthreads();
            if (stage == kStageP) {
                all_k = 0;
#pragma unroll 4
                for (int w = 0; w < kSampleWaves; ++w) all_k += s.wave_mass[w];
            }
            built = true;
        }
        if (stage == kStageP) {
            target = (u64)ceil((double)top_p * (double)all_k);
            if (target > mass) continue;                   // min-p keeps less
            target = max(target, 1ull);
        }
        if (stage == kStageDraw) {
            const double u = P.uniform[row];
            const double at = floor(fmin(u > 0.0 ? u : 0.0, 1.0) * (double)mass);
            target = min((u64)at + 1ull, mass);
        }
        // the bin in which the target is reached
        {
            unsigned c = my_count;
            u64 m = my_mass;
            for (int b = kBinsEach * tid; b < kBinsEach * (tid + 1); ++b) {
                const unsigned cb = s.count[b];
                const u64 mb = s.mass[b];
                if (counts ? c < target && target <= c + cb : m < target && target <= m + mb) {
                    s.bin = b; s.bin_n = (int)cb; s.before_count = c; s.before_mass = m;
                }
                c += cb; m += mb;
            }
        }
        if (tid == 0) { s.n_list = 0; s.lo = ~0u; s.hi = 0u; }
        __syncthreads();
        int n = s.bin_n, bin = s.bin;
        unsigned before_count = s.before_count;
        u64 before_mass = s.before_mass;
        auto taken = [&](float v, int i) { return counts || (in_k(sample_key(v), i) && level(v) >= least); };
        // what is looked at: the bin; keys k_lo .. k_hi; the indexes i_lo .. i_hi of the key k_lo
        int depth = 0, i_lo = 0, i_hi = 0;
        unsigned k_lo = 0, k_hi = 0;
        auto inside = [&](float v, int i) {
            if (depth == 0) return bin_of(v) == bin && taken(v, i);
            const unsigned key = sample_key(v);
            return key >= k_lo && key <= k_hi && (depth == 1 || (i >= i_lo && i <= i_hi)) && bin_of(v) == bin && taken(v, i);
        };
        // (a cut by 32 bits of the logit takes three rounds at most, one by the index one)
        for (int round = 0; round < 4 && n > kList; ++round) {                 // (uniform)
            if (depth == 0) {
                R.each([&](float v, int i) {
                    if (!inside(v, i)) return;
                    const unsigned key = sample_key(v);
                    atomicMin(&s.lo, key);
                    atomicMax(&s.hi, key);
                });
                __syncthreads();
                k_lo = s.lo; k_hi = s.hi;
                depth = 1;
            }
            if (depth == 1 && k_lo == k_hi) { depth = 2; i_lo = 0; i_hi = P.vocab - 1; }
            const unsigned span = depth == 1 ? k_hi - k_lo : (unsigned)(i_hi - i_lo);
            int shift = 0;
            while (span >> shift >= (unsigned)kBins) ++shift;
            auto slice = [&](float v, int i) { return (depth == 1 ? k_hi - sample_key(v) : (unsigned)(i - i_lo)) >> shift; };
            __syncthreads();
            for (int b = tid; b < kBins; b += kSampleThreads) { s.count[b] = 0u; s.mass[b] = 0ull; }
            __syncthreads();
            R.each([&](float v, int i) {
                if (!inside(v, i)) return;
                const unsigned b = slice(v, i);
                atomicAdd(&s.count[b], 1u);
                if (!counts) atomicAdd(&s.mass[b], sample_weight(level(v)));
            });
            __syncthreads();
            unsigned c0 = 0;
            u64 m0 = 0;
            for (int b = kBinsEach * tid; b < kBinsEach * (tid + 1); ++b) { c0 += s.count[b]; m0 += s.mass[b]; }
            const unsigned c1 = wave_scan(c0);
            const u64 m1 = wave_scan(m0);
            if (lane == 63) { s.wave_count[wave] = c1; s.wave_mass[wave] = m1; }
            __syncthreads();
            unsigned c = before_count + c1 - c0;
            u64 m = before_mass + m1 - m0;
            for (int w = 0; w < wave; ++w) { c += s.wave_count[w]; m += s.wave_mass[w]; }
            for (int b = kBinsEach * tid; b < kBinsEach * (tid + 1); ++b) {
                const unsigned cb = s.count[b];
                const u64 mb = s.mass[b];
                if (counts ? c < target && target <= c + cb : m < target && target <= m + mb) {
                    s.bin = b; s.bin_n = (int)cb; s.before_count = c; s.before_mass = m;
                }
                c += cb; m += mb;
            }
            __syncthreads();
            n = s.bin_n;
            before_count = s.before_count; before_mass = s.before_mass;
            const unsigned b = (unsigned)s.bin;
            if (depth == 1) {
                k_hi -= b << shift;
                k_lo = max(k_lo, k_hi - min(k_hi, (1u << shift) - 1u));
            } else {
                i_lo += (int)(b << shift);
                i_hi = min(i_hi, i_lo + (1 << shift) - 1);
            }
            built = false;                                 // (the histogram is another one now)
            __syncthreads();
        }
        R.each([&](float v, int i) {
            if (!inside(v, i)) return;
            const int at = atomicAdd(&s.n_list, 1);
            if (at >= kList) return;                       // (n tokens)
            s.key[at] = sample_key(v);
            s.index[at] = i;
        });
        __syncthreads();
        n = min(n, kList);
        u64 w = 0;
        if (tid < n) {
            w = sample_weight(level(sample_of_key(s.key[tid])));
            s.weight[tid] = w;
        }
        __syncthreads();
        if (tid < n) {
            const unsigned key = s.key[tid];
            const int i = s.index[tid];
            unsigned c = before_count;
            u64 m = before_mass;
            for (int j = 0; j < n; ++j) {
                const bool ahead = s.key[j] > key || (s.key[j] == key && s.index[j] < i);
                c += ahead;
                m += ahead ? s.weight[j] : 0ull;
            }
            if (counts ? c + 1 == target : m < target && target <= m + w) s.found = SampleFound{key, i, (int)c + 1, m + w, w};
        }
        __syncthreads();
        const SampleFound f = s.found;
        if (stage == kStageK) {
            k_key = f.key; k_index = f.index;
            built = false;
        } else if (stage == kStageP) {
            kept = (unsigned)f.count; mass = f.mass;
            cut = true;
        } else if (tid == 0) {
            answer(f.index, (float)((double)f.weight / (double)mass), (int)kept);
        }
        __syncthreads();
    }
}

hipError_t launch_sample(const SampleParams &P, int type, int n_rows, hipStream_t s)
{
    if (type == kLogitsF16) hipLaunchKernelGGL(k_sample<true>, dim3(n_rows), dim3(kSampleThreads), 0, s, P);
    else hipLaunchKernelGGL(k_sample<false>, dim3(n_rows), dim3(kSampleThreads), 0, s, P);
    return hipGetLastError();
}

}  // namespace cfpp
