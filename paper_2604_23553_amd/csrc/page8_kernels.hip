// Rows of K and V into a cache of 8-bit codes and back out of it (tree_params.h has the pool's layout).
//
// A row x of d values of one head: a = max |x|, code = C x / a rounded to the nearest code, ties to even, and read back as fp16(code a / C); C = 127
// (int8) or 448 (e4m3).  a is one of the row's fp16 values, so it is kept without loss.  C x is exact in fp32, and the quotient's distance from
// the middle of two codes is none or more than 2^-21 of it, so one correctly rounded quotient gives the code that exact arithmetic gives.  A row with
// an infinite or NaN value has a = NaN and codes of zero: all of it is read back as NaN.
//
// V lies by dimension, 16 positions to 16 bytes, so what can be written at once are rows whose slots follow one another inside of a granule:
// a run.  A workgroup has the runs that begin in 16 rows of the call - up to 31 rows - for a few heads of K or of V; V's codes meet in LDS.  A single row to a
// run, as in a decode step, writes its V codes byte by byte.
//
// Bound by memory where there are many rows (append of 4096 rows of 32 heads of 128, 101 MB: 24.9 us, 4.0 TB/s; a large copy has 4.6), by launch and one way to memory and
// back where there are few (64 rows in pages of their own 5.0 us).
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include "tree_params.h"
#include "device_utils.h"
#include "half_split.h"

namespace cfpp {

typedef unsigned p8_u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned short p8_u16x8 __attribute__((ext_vector_type(8)));
typedef float p8_f32x2 __attribute__((ext_vector_type(2)));

constexpr int kP8Window = 16, kP8Most = 2 * kP8Window - 1;

// The runs of a window, as bits of rows window .. window + 31; every lane of the wavefront has the same
struct P8Runs {
    unsigned starts, row_bits;         // rows that begin a run; rows of these runs
    int first, n;                      // the set: rows first .. first + n - 1 of the window
    __device__ __forceinline__ bool of(const Page8Rows &P, int window)
    {
        const int lane = threadIdx.x & 63, i = lane & 31, row = window * kP8Window + i, limit = P.pg.n_pages * P.pg.page;
        const int slot = row < P.n_rows ? P.slots[row] : -1, before = row > 0 && row <= P.n_rows ? P.slots[row - 1] : -1;
        const bool valid = slot >= 0 && slot < limit, on = valid && before >= 0 && slot == before + 1 && (slot & 15) != 0;
        const unsigned goes_on = (unsigned)__ballot(on), any = (unsigned)__ballot(valid);
        starts = any & ~goes_on & ((1u << kP8Window) - 1u);
        if (!starts) return false;
        first = __builtin_ctz(starts);
        const unsigned stop = ~goes_on & ~((1u << kP8Window) - 1u);            // the first row behind the window that begins something else
        const int end = min(stop ? __builtin_ctz(stop) : 32, kP8Window + 15);
        n = end - first;
        row_bits = any & (end < 32 ? (1u << end) - 1u : ~0u) & ~((1u << first) - 1u);
        return true;
    }
    __device__ __forceinline__ unsigned single() const     // runs of one row
    {
        return starts & ~((row_bits & ~starts) >> 1);
    }
    __device__ __forceinline__ int length(int at) const    // of the run that begins with row `at` of the window
    {
        const unsigned rest = row_bits & ~starts, up = at < 31 ? rest >> (at + 1) : 0u;
        return 1 + __builtin_ctz(~up);
    }
};

__device__ __forceinline__ unsigned char *p8_granule_of(const Page8Rows &P, int slot, int head)
{
    const int page = slot / P.pg.page, at = slot - page * P.pg.page;
    return P.pool + (((size_t)page * P.pg.heads + head) * (P.pg.page >> 4) + (at >> 4)) * page8_granule(P.pg.d);
}

// the lanes that have a row of a head, 8 dimensions each: 8 or 16 (of which head_dim 80 uses ten)
template <int D> constexpr int p8_lanes() { return D == 64 ? 8 : 16; }
// heads of a workgroup: two dimensions of V to a thread, or as few as have 16 rows for 256 threads
template <int D> constexpr int p8_heads(bool few) { return few ? (D == 64 ? 2 : 1) : 512 / D; }

template <int LANES>
__device__ __forceinline__ unsigned p8_most(unsigned v)
{
    auto up = [](unsigned a, auto ctrl) { return max(a, (unsigned)__builtin_amdgcn_update_dpp(0, (int)a, decltype(ctrl)::value, 0xF, 0xF, true)); };
    v = up(v, std::integral_constant<int, kDppXor1>{});
    v = up(v, std::integral_constant<int, kDppXor2>{});
    v = up(v, std::integral_constant<int, kDppHalfMirror>{});
    if constexpr (LANES == 16) v = up(v, std::integral_constant<int, kDppMirror>{});
    return v;
}

// the correctly rounded quotient y / a; inv = 1 / a, rounded.  One register, so that it is rounded to fp32 before it is to fp16: rounded to fp16 at once
// (v_fma_mixlo) the last sum, which is off by 2^-48 of itself, would put ties on either side
__device__ __forceinline__ float p8_quotient(float y, float a, float inv)
{
    const float q = y * inv;
    return split_value(fmaf(fmaf(-q, a, y), inv, q));
}

template <int D, bool INT8, bool FEW>
__global__ void __launch_bounds__(256) k_page8_append(Page8Rows P)
{
    constexpr int LANES = p8_lanes<D>(), HEADS = p8_heads<D>(FEW), EACH = HEADS * kP8Window * LANES / 256, PIECES = D / 8, PITCH = HEADS * D;
    constexpr float C = INT8 ? 127.f : 448.f;
    __shared__ __align__(16) unsigned char codes[kP8Most][PITCH];
    __shared__ int slot_of[32];
    P8Runs runs;
    if (!runs.of(P, blockIdx.x)) return;                   // (uniform)
    const int tid = threadIdx.x, window = blockIdx.x * kP8Window, head0 = blockIdx.y * HEADS;
    const bool v_rows = blockIdx.z != 0;
    if (tid < 32) slot_of[tid] = (runs.row_bits >> tid) & 1 ? P.slots[window + tid] : -1;
    const unsigned single = runs.single();
    const __half *from = v_rows ? P.v : P.k;
    __syncthreads();
    for (int half = 0; half < runs.n; half += kP8Window) {
        u32x4 x[EACH];
        int slot[EACH];
#pragma unroll
        for (int u = 0; u < EACH; ++u) {                   // 16 rows of a head follow one another
            const int e = tid + 256 * u, piece = e % LANES, j = half + e / LANES % kP8Window, head = head0 + e / (LANES * kP8Window);
            slot[u] = j < runs.n && piece < PIECES && head < P.pg.heads ? slot_of[runs.first + j] : -1;
            x[u] = u32x4{0u, 0u, 0u, 0u};
            if (slot[u] >= 0)
                x[u] = __builtin_nontemporal_load(as_global(reinterpret_cast<const u32x4 *>(from + (size_t)(window + runs.first + j) * P.stride + (size_t)head * D + piece * 8)));
        }
#pragma unroll
        for (int u = 0; u < EACH; ++u) {
            const int e = tid + 256 * u, piece = e % LANES, j = half + e / LANES % kP8Window, hb = e / (LANES * kP8Window);
            // sizes as whole numbers: those of NaN are above infinity's, infinity's above all others'
            const p8_u16x8 bits = __builtin_bit_cast(p8_u16x8, x[u] & 0x7fff7fffu);
            unsigned most = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) most = max(most, (unsigned)bits[i]);
            most = p8_most<LANES>(most);
            const bool finite = most < 0x7c00u;
            const float a = __half2float(__ushort_as_half((unsigned short)most)), inv = finite && most ? 1.f / a : 0.f;
            unsigned out[2];
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                float q[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = unpack_h2(x[u][2 * w + (i >> 1)]);
                    q[i] = finite ? p8_quotient((i & 1 ? f.y : f.x) * C, a, inv) : 0.f;
                }
                if constexpr (INT8) {
                    unsigned b[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) b[i] = (unsigned)(int)rintf(q[i]) & 255u;
                    out[w] = b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24;
                } else {
                    out[w] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false), true);
                }
            }
            if (slot[u] < 0) continue;
            unsigned char *g = p8_granule_of(P, slot[u], head0 + hb);
            const int t = slot[u] & 15;
            if (v_rows) *reinterpret_cast<p8_u32x2 *>(&codes[j][hb * D + piece * 8]) = p8_u32x2{out[0], out[1]};
            else *as_global(reinterpret_cast<p8_u32x2 *>(g + (t >> 2) * 4 * D + (piece >> 1) * 64 + (t & 3) * 16 + (piece & 1) * 8)) = p8_u32x2{out[0], out[1]};
            if (piece == 0) *as_global(reinterpret_cast<unsigned short *>(g + 32 * D + (v_rows ? 32 : 0) + 2 * t)) = (unsigned short)(finite ? most : 0x7e00u);
        }
    }
    if (!v_rows) return;                                   // (uniform)
    __syncthreads();
    // single rows together, a byte of a dimension to a thread: a wavefront's are in eight lines
    if (single)
#pragma unroll 4
        for (int e = tid; e < runs.n * PITCH; e += 256) {
            const int j = e / PITCH, x = e - j * PITCH, hb = x / D, dim = x - hb * D;
            if (head0 + hb >= P.pg.heads || !((single >> (runs.first + j)) & 1)) continue;
            const int slot = slot_of[runs.first + j];
            *as_global(p8_granule_of(P, slot, head0 + hb) + 16 * D + dim * 16 + (slot & 15)) = codes[j][x];
        }
    for (unsigned left = runs.starts & ~single; left; left &= left - 1) {
        const int at = __builtin_ctz(left), len = runs.length(at), slot = slot_of[at], t0 = slot & 15;         // (uniform)
        for (int e = tid; e < PITCH; e += 256) {
            const int hb = e / D, dim = e - hb * D;
            if (head0 + hb >= P.pg.heads) break;
            unsigned char *to = p8_granule_of(P, slot, head0 + hb) + 16 * D + dim * 16;
            const unsigned char *c = &codes[at - runs.first][e];
            if (len == 16) {
                u32x4 w;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    w[k] = (unsigned)c[4 * k * PITCH] | (unsigned)c[(4 * k + 1) * PITCH] << 8 | (unsigned)c[(4 * k + 2) * PITCH] << 16 | (unsigned)c[(4 * k + 3) * PITCH] << 24;
                *as_global(reinterpret_cast<u32x4 *>(to)) = w;
            } else {
                for (int i = 0; i < len; ++i) *as_global(to + t0 + i) = c[i * PITCH];
            }
        }
    }
}

// fp16 of two codes, the low 16 bits of c, times their rows' largest values (the products have at most 18 significant bits)
template <bool INT8>
__device__ __forceinline__ unsigned p8_read(unsigned c, float a0, float a1)
{
    constexpr float C = INT8 ? 127.f : 448.f;
    float f[2];
    if constexpr (INT8) {
        f[0] = (float)(int)(signed char)(c & 255u);
        f[1] = (float)(int)(signed char)((c >> 8) & 255u);
    } else {
        const p8_f32x2 v = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false);
        f[0] = v[0];
        f[1] = v[1];
    }
    return (unsigned)__half_as_ushort(__float2half_rn(p8_quotient(f[0] * a0, C, 1.f / C))) |
           (unsigned)__half_as_ushort(__float2half_rn(p8_quotient(f[1] * a1, C, 1.f / C))) << 16;
}

// V: a thread has two dimensions of a head and all positions of a run, which it writes one after the other, 256 bytes of a row to a wavefront; nothing
// goes through LDS (16384 rows of 8 heads of 128, 101 MB: 27.7 us through it, 24.1 so, 4.2 TB/s; a large copy has 4.6).
template <int D, bool INT8, bool FEW>
__global__ void __launch_bounds__(256) k_page8_read(Page8Rows P)
{
    constexpr int LANES = p8_lanes<D>(), HEADS = p8_heads<D>(FEW), EACH = HEADS * kP8Window * LANES / 256, PIECES = D / 8;
    __shared__ int slot_of[32];
    P8Runs runs;
    if (!runs.of(P, blockIdx.x)) return;                   // (uniform)
    const int tid = threadIdx.x, window = blockIdx.x * kP8Window, head0 = blockIdx.y * HEADS;
    if (tid < 32) slot_of[tid] = (runs.row_bits >> tid) & 1 ? P.slots[window + tid] : -1;
    __syncthreads();
    if (blockIdx.z != 0) {
        const int hb = tid / (D / 2), dim = 2 * (tid - hb * (D / 2)), head = head0 + hb;
        if (hb >= HEADS || head >= P.pg.heads) return;
        for (unsigned left = runs.starts; left; left &= left - 1) {
            const int at = __builtin_ctz(left), len = runs.length(at), slot = slot_of[at], t0 = slot & 15;     // (uniform)
            const unsigned char *g = p8_granule_of(P, slot, head);
            const u32x4 x = *as_global(reinterpret_cast<const u32x4 *>(g + 16 * D + dim * 16)), y = *as_global(reinterpret_cast<const u32x4 *>(g + 16 * D + dim * 16 + 16));
            u32x4 most[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) most[u] = *as_global(reinterpret_cast<const u32x4 *>(g + 32 * D + 32 + 16 * u));
            __half *to = P.v + (size_t)(window + at) * P.stride + (size_t)head * D + dim;
#pragma unroll
            for (int t = 0; t < 16; ++t) {
                if (t < t0 || t >= t0 + len) continue;     // (uniform)
                const float2 a2 = unpack_h2(most[t >> 3][(t >> 1) & 3]);
                const float a = t & 1 ? a2.y : a2.x;
                const unsigned c = ((x[t >> 2] >> 8 * (t & 3)) & 255u) | ((y[t >> 2] >> 8 * (t & 3)) & 255u) << 8;
                *as_global(reinterpret_cast<unsigned *>(to + (size_t)(t - t0) * P.stride)) = p8_read<INT8>(c, a, a);
            }
        }
        return;
    }
    for (int half = 0; half < runs.n; half += kP8Window) {
        p8_u32x2 x[EACH];
        unsigned short most[EACH];
        int slot[EACH];
#pragma unroll
        for (int u = 0; u < EACH; ++u) {                   // 16 rows of a head follow one another
            const int e = tid + 256 * u, piece = e % LANES, j = half + e / LANES % kP8Window, head = head0 + e / (LANES * kP8Window);
            slot[u] = j < runs.n && piece < PIECES && head < P.pg.heads ? slot_of[runs.first + j] : -1;
            x[u] = p8_u32x2{0u, 0u};
            most[u] = 0;
            if (slot[u] < 0) continue;
            const unsigned char *g = p8_granule_of(P, slot[u], head);
            const int t = slot[u] & 15;
            x[u] = *as_global(reinterpret_cast<const p8_u32x2 *>(g + (t >> 2) * 4 * D + (piece >> 1) * 64 + (t & 3) * 16 + (piece & 1) * 8));
            most[u] = *as_global(reinterpret_cast<const unsigned short *>(g + 32 * D + 2 * t));
        }
#pragma unroll
        for (int u = 0; u < EACH; ++u) {
            if (slot[u] < 0) continue;
            const int e = tid + 256 * u, piece = e % LANES, j = half + e / LANES % kP8Window, head = head0 + e / (LANES * kP8Window);
            const float a = __half2float(__ushort_as_half(most[u]));
            u32x4 out;
#pragma unroll
            for (int w = 0; w < 4; ++w) out[w] = p8_read<INT8>((x[u][w >> 1] >> 16 * (w & 1)) & 0xffffu, a, a);
            *as_global(reinterpret_cast<u32x4 *>(P.k + (size_t)(window + runs.first + j) * P.stride + (size_t)head * D + piece * 8)) = out;
        }
    }
}

// Up to so many workgroups of many heads there are some of few: 64 rows of 32 heads of 80, each in a page of its own, are 48 of six heads or 256 of one.
// us a call in a graph, few / many, by the workgroups of many heads:
//     rows apart, 32 heads of 80     48     180    240    264    360    540            rows that follow one another     48     240    264    360    540    768
//     append                         4.4    7.1    8.5    8.9   10.5   17.4                                             4.2    5.3    5.6    6.2    7.7   10.9
//                                  / 11.0  12.9   13.4   13.6   15.2   16.3                                          / 10.2   10.4   10.5   11.0   11.5   14.4
//     read                          10.6   11.3   12.1   13.2   13.6   19.5                                             5.2    6.1    6.3    6.8    8.2    8.9
//                                  / 10.5  11.0   11.4   12.5   13.3   15.2                                           / 7.4    7.7    7.7    7.8    8.1    8.4
// An append turns at about 500 of them where rows lie apart, behind 1000 where they follow one another, a read of rows that follow at about 500; one of rows that lie apart never gains.
// 32 heads of 128 and 8 heads of 64 or of 128 do the same.  Of few always, an append of 4096 rows of 32 heads of 128 takes 32.4 us for 23.7, a read of 16384 rows of 8 heads 35.6
// for 24.1.
constexpr int kP8Few = 256;
template <int D, bool INT8, bool FEW>
static hipError_t launch_of(const Page8Rows &P, bool append, hipStream_t s)
{
    const dim3 grid((P.n_rows + kP8Window - 1) / kP8Window, (P.pg.heads + p8_heads<D>(FEW) - 1) / p8_heads<D>(FEW), 2);
    if (append) hipLaunchKernelGGL((k_page8_append<D, INT8, FEW>), grid, dim3(256), 0, s, P);
    else hipLaunchKernelGGL((k_page8_read<D, INT8, FEW>), grid, dim3(256), 0, s, P);
    return hipGetLastError();
}
template <int D>
static hipError_t launch_type(const Page8Rows &P, int type, bool append, hipStream_t s)
{
    const int most = p8_heads<D>(false);
    const bool few = (long long)((P.n_rows + kP8Window - 1) / kP8Window) * ((P.pg.heads + most - 1) / most) * 2 <= kP8Few;
    if (type == kPage8Int8) return few ? launch_of<D, true, true>(P, append, s) : launch_of<D, true, false>(P, append, s);
    return few ? launch_of<D, false, true>(P, append, s) : launch_of<D, false, false>(P, append, s);
}
static hipError_t launch(const Page8Rows &P, int type, bool append, hipStream_t s)
{
    switch (P.pg.d) {
    case 64: return launch_type<64>(P, type, append, s);
    case 80: return launch_type<80>(P, type, append, s);
    default: return launch_type<128>(P, type, append, s);
    }
}
hipError_t launch_page8_append(const Page8Rows &P, int type, hipStream_t s) { return launch(P, type, true, s); }
hipError_t launch_page8_read(const Page8Rows &P, int type, hipStream_t s) { return launch(P, type, false, s); }

}  // namespace cfpp
