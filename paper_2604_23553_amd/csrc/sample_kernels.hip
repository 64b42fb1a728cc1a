// The next token from a row of logits and a given random number: temperature, top-k, top-p, min-p.
//
// The row's order is larger logit first, lower index among equals; weights w = 2^((l - l_max) log2(e) / temperature).  Every filter keeps a beginning of the
// order - k tokens; as many as reach p of those k tokens' sum; those of at least min_p times the largest weight - and the token drawn is the first whose running sum
// passes u times the sum of what is kept.  So all of it is the same question: where, in the order, does a running count or a running sum reach a target?
//
// Nothing is sorted.  A histogram over (l_max - l) in steps of 2^(1/32) of a weight, 2048 bins of counts and of sums in LDS, says in which bin that is; the bin's
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

constexpr int kBins = 2048, kList = 512;
// Rows up to which a row has a CU's 1024 threads; more, and two rows share it
constexpr int kSampleOneEach = 256;
constexpr float kBinsToOctave = 32.f, kWeightless = 47.f * kBinsToOctave;     // from there on weights are zero

// 2^t for t <= 0 as a multiple of 2^-45; zero from 2^-46 down, and for NaN
__device__ __forceinline__ u64 sample_weight(double t)
{
    t = fmax(t, -100.0);
    const double whole = t + 6755399441055744.0;           // (1.5 2^52 more: the last bits are the whole number, rounded)
    const double f = t - (whole - 6755399441055744.0);     // in [-1/2, 1/2]
    // 2^f = 1 + f q(f), q fitted to the least relative error, 2^-40.1
    double p = 1.317893346165606e-06;
    p = fma(p, f, 1.5309156203092946e-05);
    p = fma(p, f, 1.5403825462733238e-04);
    p = fma(p, f, 1.3333454860442664e-03);
    p = fma(p, f, 9.618128616123461e-03);
    p = fma(p, f, 5.550410935266362e-02);
    p = fma(p, f, 2.4022650698110598e-01);
    p = fma(p, f, 6.931471805482123e-01);
    p = fma(p, f, 1.0);
    // times 2^(45 + the whole number), by the exponent; 2^52 more, and the last bits are the weight
    const u64 scaled = (u64)__double_as_longlong(p) + ((u64)((unsigned)__double_as_longlong(whole) + 45u) << 52);
    return (u64)__double_as_longlong(__longlong_as_double((long long)scaled) + 4503599627370496.0) - 0x4330000000000000ull;
}

// larger logits have larger keys (no NaN)
__device__ __forceinline__ unsigned sample_key(float v)
{
    const unsigned b = __float_as_uint(v + 0.f);           // (both zeros are equal)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float sample_of_key(unsigned k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
// the order as one number, the first the smallest
__device__ __forceinline__ u64 sample_place(unsigned key, int i) { return (u64)~key << 32 | (unsigned)i; }

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
__device__ __forceinline__ u64 lane_value(u64 v, int lane) { return (u64)lane_value((unsigned)(v >> 32), lane) << 32 | lane_value((unsigned)v, lane); }

template <int T>
struct SampleShared {
    static constexpr int kWaves = T / 64;
    u64 mass[kBins];
    unsigned count[kBins];
    u64 place[kList], sorted[kList], weight[kList];        // tokens as they were collected; in order, and their weights
    u64 wave_mass[2][kWaves];
    unsigned wave_count[2][kWaves];
    float wave_max[kWaves];
    int n_list, bin;
    unsigned below, before_count, bin_n, lo, hi, kept, first;
    u64 before_mass, value, found_place, found_mass, found_weight;
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

// A row's logits, four to a thread that follow one another; NaN and what lies behind the row as minus infinity.  FEW: of less than four
template <int T, bool F16, bool FEW>
struct SampleRow {
    static constexpr int kThreads = T;
    const void *at;
    int vocab;
    // (the last ones of the row in place of those behind it; rows may begin at any logit)
    __device__ __forceinline__ f32x4 raw(int i) const
    {
        typedef std::conditional_t<F16, _Float16, float> L;
        typedef L L4 __attribute__((ext_vector_type(4), aligned(sizeof(L))));
        const CFPP_GLOBAL L *p = (const CFPP_GLOBAL L *)at;
        if constexpr (FEW) {
            return f32x4{(float)p[0], (float)p[min(1, vocab - 1)], (float)p[vocab - 1], 0.f};
        } else {
            const L4 x = *(const CFPP_GLOBAL L4 *)(p + min(i, vocab - 4));
            return f32x4{(float)x[0], (float)x[1], (float)x[2], (float)x[3]};
        }
    }
    // f(four logits, index of the first), all threads of the workgroup together; INFINITE: of a row whose largest logit is, 0 and minus infinity.  A NaN
    // stays one.
    template <bool INFINITE, class Fn>
    __device__ __forceinline__ void each(Fn f) const
    {
        constexpr int STEP = 4 * T, AT = FEW ? 1 : 4;             // four vectors are on their way while four others are looked at
        int own = 4 * (int)threadIdx.x;
        asm volatile("" : "+v"(own));                      // (so that no pass keeps its addresses in registers for the next one)
        f32x4 next[AT];
#pragma unroll
        for (int j = 0; j < AT; ++j) next[j] = raw(own + j * STEP);
#pragma unroll 1
        for (int base = 0; base < vocab; base += AT * STEP) {
            f32x4 x[AT];
#pragma unroll
            for (int j = 0; j < AT; ++j) x[j] = next[j];
#pragma unroll
            for (int j = 0; j < AT; ++j) next[j] = raw(own + base + (AT + j) * STEP);          // (past the end: the last ones again)
#pragma unroll
            for (int j = 0; j < AT; ++j) {
                const int at = base + j * STEP, i = at + own;
                if (at >= vocab) break;                    // (uniform)
                f32x4 v = x[j];
                if (at + STEP > vocab) {                   // (uniform) the row's end: what was loaded is `off` logits too early
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
                if constexpr (INFINITE)
#pragma unroll
                    for (int c = 0; c < 4; ++c) v[c] = v[c] == INFINITY ? 0.f : -INFINITY;
                f(v, i);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
};

struct SampleHow { float tau, top_p, min_p, uniform; int top_k; };

// The token of a row whose largest logit is `most`.  s.mass and s.count are zero.
template <bool INFINITE, class Row, class Answer>
__device__ __forceinline__ void sample_row(SampleShared<Row::kThreads> &s, const Row &R, const SampleHow &how, float most, Answer answer)
{
    constexpr int T = Row::kThreads, EACH = kBins / T;
    const int tid = threadIdx.x;
    const double octaves = 1.4426950408889634 / (double)how.tau;
    const double least = how.min_p > 0.f ? log2((double)fminf(how.min_p, 1.f)) : -1.7976931348623157e308;
    const float to_bin = fminf(fmaxf((float)octaves * kBinsToOctave, 1e-30f), 1e30f);          // (so that no product is none)
    auto level = [&](float v) { return ((double)v - (double)most) * octaves; };
    auto depth_of = [&](float v) { return (most - v) * to_bin; };              // (never rises with v)
    auto bin_of = [&](float v) { return (int)fminf(depth_of(v), kBins - 1.f); };
    // f of the tokens that pick() is true of; a vector of four without any costs nothing more
    auto each = [&](auto f) { R.template each<INFINITE>(f); };
    auto some = [&](auto pick, auto f) {
        R.template each<INFINITE>([&](f32x4 v, int i) {
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
    const bool by_p = how.top_p < 1.f, small = R.vocab <= kList;
    int n_k = by_k ? how.top_k : R.vocab;                  // (at most so many: minus infinities are found later)
    u64 k_place = ~0ull;                                   // of the last token that top-k keeps

    // kStageAll: the few tokens that top-k leaves, and some more, are in the list: all filters there.  Otherwise the places where top-k ends, where top-p does,
    // and of the draw, one after the other
    enum { kStageAll, kStageK, kStageP, kStageDraw };
    int stage = small || (by_k && n_k <= kList / 2) ? kStageAll : by_k ? kStageK : by_p ? kStageP : kStageDraw;
    enum { kNone, kCounts, kMasses };
    int built = kNone;                                     // what the histogram holds
    bool dirty = false, cut = false;                       // the histogram is to be cleared; top-p has cut
    unsigned kept = 0, my_count = 0;                       // my_: running sums of the bins before this thread's
    u64 mass = 0, my_mass = 0, all_k = 0;                  // mass: of what is kept; all_k: of what top-k keeps
    const bool by_m = how.min_p > 0.f;
    int turn = 0;
    auto clear = [&]() {
        __syncthreads();
        for (int b = tid; b < kBins; b += T) { s.count[b] = 0u; s.mass[b] = 0ull; }
        __syncthreads();
    };
    auto scan = [&](unsigned &all_count, u64 &all_mass) {
        __syncthreads();
        unsigned c = 0;
        u64 m = 0;
#pragma unroll
        for (int b = 0; b < EACH; ++b) { c += s.count[EACH * tid + b]; m += s.mass[EACH * tid + b]; }
        block_scan(s, turn ^= 1, c, m, my_count, my_mass, all_count, all_mass);
    };
    // the bin in which the running count or sum reaches the target
    auto find = [&](bool counts, u64 target, unsigned c, u64 m) {
#pragma unroll
        for (int b = 0; b < EACH; ++b) {
            const unsigned cb = s.count[EACH * tid + b];
            const u64 mb = s.mass[EACH * tid + b];
            if (counts ? c < target && target <= c + cb : m < target && target <= m + mb) {
                s.bin = EACH * tid + b; s.bin_n = cb; s.before_count = c; s.before_mass = m;
            }
            c += cb; m += mb;
        }
    };
    for (;;) {
        const bool counts = stage <= kStageK;
        if (built != (counts ? kCounts : kMasses) && !small) {
            if (dirty) clear();
            dirty = true;
            unsigned n;
            u64 sum, total = 0;
            if (counts) {
                each([&](f32x4 v, int) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (v[c] > -INFINITY) atomicAdd(&s.count[bin_of(v[c])], 1u);
                });
                scan(n, sum);
                built = kCounts;
                if (n <= (unsigned)n_k) {                  // (uniform) top-k keeps all that there is
                    n_k = (int)n;
                    by_k = false;
                    if (n > (unsigned)kList) { stage = by_p ? kStageP : kStageDraw; continue; }
                    stage = kStageAll;
                }
            } else {
                // what min-p keeps is a beginning of the order too: its number and sum, beside the histogram of all that top-k keeps
                const bool number = by_m || !(by_p || by_k);
                unsigned reaches = 0;
                each([&](f32x4 v, int i) {
                    if (by_k) {                            // (uniform)
#pragma unroll
                        for (int c = 0; c < 4; ++c) v[c] = sample_place(sample_key(v[c]), i + c) > k_place ? -INFINITY : v[c];
                    }
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const double t = level(v[c]);
                        const u64 w = sample_weight(t);
                        const float y = depth_of(v[c]);
                        if (y < kWeightless) atomicAdd(&s.mass[(int)y], w);
                        if (number) {                      // (uniform)
                            const bool on = t >= least;
                            reaches += on;
                            total += on ? w : 0ull;
                        }
                    }
                });
                scan(n, all_k);
                if (!cut) {
                    kept = (unsigned)n_k;
                    mass = all_k;
                    if (number) {
                        unsigned none;
                        u64 before;
                        block_scan(s, turn ^= 1, reaches, total, none, before, kept, sum);
                        if (by_m) mass = sum;
                    }
                }
                built = kMasses;
            }
        }
        u64 target = (u64)n_k;
        if (stage == kStageP) {
            target = (u64)ceil((double)how.top_p * (double)all_k);
            target = min(max(target, 1ull), all_k);
        }
        auto drawn = [&](u64 sum) {
            const double u = how.uniform;
            return min((u64)floor(fmin(u > 0.0 ? u : 0.0, 1.0) * (double)sum) + 1ull, sum);
        };
        if (stage == kStageDraw) target = drawn(mass);
        if (!small) find(counts, target, my_count, my_mass);
        else if (tid == 0) { s.bin = kBins; s.bin_n = 0u; s.before_count = 0u; s.before_mass = 0ull; }
        if (tid == 0) { s.n_list = 0; s.below = 0u; s.lo = ~0u; s.hi = 0u; }
        __syncthreads();
        const int bin = s.bin;
        unsigned before_count = s.before_count;
        u64 before_mass = s.before_mass;
        if (stage == kStageAll) {
            if (before_count + s.bin_n > (unsigned)kList) { stage = kStageK; __syncthreads(); continue; }      // (uniform)
            before_count = 0u;
        }
        const bool all = stage == kStageAll;
        auto taken = [&](float v, int i) { return counts || !by_k || sample_place(sample_key(v), i) <= k_place; };
        // what is looked at: the bin; keys k_lo .. k_hi of it; the indexes i_lo .. i_hi of the key k_lo
        int depth = 0, i_lo = 0, i_hi = 0;
        unsigned k_lo = 0, k_hi = 0;
        const float from = all ? -1.f : (float)bin, to = bin >= kBins - 1 ? NAN : (float)(bin + 1);              // (the last bin has all that is left)
        auto near = [&](float v) {
            const float y = depth_of(v);
            return y >= from && !(y >= to);
        };
        auto inside = [&](float v, int i) {
            if (depth > 0) {
                const unsigned key = sample_key(v);
                if (key < k_lo || key > k_hi || (depth == 2 && (i < i_lo || i > i_hi))) return false;
            }
            return all || taken(v, i);
        };
        for (int round = 0;; ++round) {
            auto collect = [&](float v, int i) {
                if (!inside(v, i)) return;
                const int at = atomicAdd(&s.n_list, 1);
                if (at < kList) s.place[at] = sample_place(sample_key(v), i);
            };
            if (stage == kStageP && round == 0) {          // (what stands before a token that is kept is kept)
                unsigned below = 0;
                some([&](float v) { below += depth_of(v) < from; return near(v); }, collect);
                below = wave_scan(below);
                if ((tid & 63) == 63 && below) atomicAdd(&s.below, below);
            } else {
                some(near, collect);
            }
            __syncthreads();
            if (stage == kStageP && round == 0) before_count = s.below;
            if (s.n_list <= kList || round == 4) break;    // (a cut by a logit's 32 bits takes three rounds at most, by the index one)
            // too many for the list: a histogram of what is inside
            if (depth == 0) {
                some(near, [&](float v, int i) {
                    if (!inside(v, i)) return;
                    const unsigned key = sample_key(v);
                    atomicMin(&s.lo, key);
                    atomicMax(&s.hi, key);
                });
                __syncthreads();
                k_lo = s.lo; k_hi = s.hi;
                depth = 1;
            }
            if (depth == 1 && k_lo == k_hi) { depth = 2; i_lo = 0; i_hi = R.vocab - 1; }
            const unsigned span = depth == 1 ? k_hi - k_lo : (unsigned)(i_hi - i_lo);
            int shift = 0;
            while (span >> shift >= (unsigned)kBins) ++shift;
            clear();
            built = kNone;
            some(near, [&](float v, int i) {
                if (!inside(v, i)) return;
                const unsigned b = (depth == 1 ? k_hi - sample_key(v) : (unsigned)(i - i_lo)) >> shift;
                atomicAdd(&s.count[b], 1u);
                if (!counts) atomicAdd(&s.mass[b], sample_weight(level(v)));
            });
            unsigned n;
            u64 sum;
            scan(n, sum);
            find(counts, target, before_count + my_count, before_mass + my_mass);
            if (tid == 0) s.n_list = 0;
            __syncthreads();
            before_count = s.before_count; before_mass = s.before_mass;
            const unsigned b = (unsigned)s.bin;
            if (depth == 1) {
                k_hi -= b << shift;
                k_lo = max(k_lo, k_hi - min(k_hi, (1u << shift) - 1u));
            } else {
                i_lo += (int)(b << shift);
                i_hi = min(i_hi, i_lo + (1 << shift) - 1);
            }
        }
        const int n = min(s.n_list, kList);
        // the list in order: every token counts those before it
        if (tid < n) {
            const u64 own = s.place[tid];
            int rank = 0;
#pragma unroll 2
            for (int j = 0; j < n; ++j) rank += s.place[j] < own;
            s.sorted[rank] = own;
            s.weight[rank] = sample_weight(level(sample_of_key(~(unsigned)(own >> 32))));
        }
        __syncthreads();
        const u64 place = tid < n ? s.sorted[tid] : ~0ull, w = tid < n ? s.weight[tid] : 0ull;
        unsigned none, none_of;
        u64 sum, list_mass;
        block_scan(s, turn ^= 1, 0u, w, none, sum, none_of, list_mass);
        sum += before_mass;                                // of the order before this thread's token
        if (all) {
            n_k = min(n_k, n);                             // (tokens behind the first n_k are in the list too)
            if (tid == n_k - 1) s.value = sum + w;
            if (tid == 0) s.kept = 0u;
            __syncthreads();
            u64 p_target = ~0ull;
            if (by_p) p_target = max((u64)ceil((double)how.top_p * (double)s.value), 1ull);
            const bool ok = tid < n_k && sum < p_target && level(sample_of_key(~(unsigned)(place >> 32))) >= least;
            const unsigned long long of_wave = __ballot(ok);
            if ((tid & 63) == 0 && of_wave) atomicAdd(&s.kept, (unsigned)__popcll(of_wave));
            __syncthreads();
            const int n_kept = (int)s.kept;                // (the first of the order)
            if (tid == n_kept - 1) s.found_mass = sum + w;
            __syncthreads();
            const u64 at = drawn(s.found_mass);
            if (sum < at && at <= sum + w && tid < n_kept) answer((int)(unsigned)place, (float)((double)w / (double)s.found_mass), n_kept);
            return;
        }
        if (tid < n && (counts ? before_count + tid + 1 == target : sum < target && target <= sum + w)) {
            s.found_place = place; s.found_mass = sum + w; s.found_weight = w; s.kept = before_count + tid + 1;
        }
        __syncthreads();
        if (stage == kStageK) {
            k_place = s.found_place;
            stage = by_p ? kStageP : kStageDraw;
        } else if (stage == kStageP) {
            kept = min(kept, s.kept);
            mass = min(mass, s.found_mass);
            cut = true;
            stage = kStageDraw;
        } else {
            if (tid == 0) answer((int)(unsigned)s.found_place, (float)((double)s.found_weight / (double)mass), (int)kept);
            return;
        }
    }
}

template <int T, bool F16, bool FEW>
__global__ void __launch_bounds__(T) k_sample(SampleParams P)
{
    __shared__ SampleShared<T> s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row = blockIdx.x;
    const SampleRow<T, F16, FEW> R{static_cast<const char *>(P.logits) + (size_t)row * P.stride * (F16 ? 2 : 4), P.vocab};
    const SampleHow how{P.temperature ? P.temperature[row] : 1.f, P.top_p ? P.top_p[row] : 1.f, P.min_p ? P.min_p[row] : 0.f, P.uniform[row], P.top_k ? P.top_k[row] : 0};
    auto answer = [&](int token, float prob, int kept) {
        P.tokens[row] = token;
        if (P.probs) P.probs[row] = prob;
        if (P.kept) P.kept[row] = kept;
    };
    for (int b = tid; b < kBins; b += T) { s.count[b] = 0u; s.mass[b] = 0ull; }
    if (tid == 0) s.first = 0x7fffffffu;
    float most = -INFINITY;
    R.template each<false>([&](f32x4 v, int) { most = fmaxf(fmaxf(most, fmaxf(v[0], v[1])), fmaxf(v[2], v[3])); });
    most = wave_max(most);
    if (lane == 0) s.wave_max[wave] = most;
    __syncthreads();
    most = wave_max(s.wave_max[lane & (T / 64 - 1)]);
    if (most == -INFINITY) {                               // (uniform, as the ways out below)
        if (tid == 0) answer(-1, 0.f, 0);
        return;
    }
    if (!(how.tau > 0.f) || how.top_k == 1 || how.top_p <= 0.f) {              // the first of the order
        R.template each<false>([&](f32x4 v, int i) {
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (v[c] == most) atomicMin(&s.first, (unsigned)(i + c));
        });
        __syncthreads();
        if (tid == 0) answer((int)s.first, 1.f, 1);
        return;
    }
    if (most == INFINITY) sample_row<true>(s, R, how, 0.f, answer);
    else sample_row<false>(s, R, how, most, answer);
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
