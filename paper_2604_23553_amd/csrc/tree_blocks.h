// What the attentions over pages share (tree_attention.hip, page8_attention.hip): block-table lookups, masks, outputs, and the sums that the
// pieces of a tile leave for each other.
#pragma once
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include "tree_params.h"
#include "device_utils.h"
#include "half_split.h"
#include "prefill_device.h"

namespace cfpp {

typedef _Float16 ta_f16x8 __attribute__((ext_vector_type(8)));
typedef unsigned ta_u32x2 __attribute__((ext_vector_type(2)));

constexpr int kTaThreads = 256, kTaWaves = kTaThreads / 64, kTaRow = 32, kTaStep = kTaRow * kTaWaves;

// Up to so many query rows to a tile its last workgroup adds the pieces, above it a launch does, which has all CUs for the up to 128 rows of sums: 64 nodes
// behind 8000 49 / 38 us, 200 behind 300 25.3 / 16.5, 26 behind 500 14.2 / 13.1, 26 behind 4096 19.3 / 18.6.  With 16 rows the launch costs more: one token behind
// 4096 14.4 / 15.7.
constexpr int kTaLastJoins = 16;

constexpr float kTaLowest = -3.402823466e38f;

// A granule of 16 positions lies in one page.
struct TaPick { int page, in; };                           // table entry, granule inside of its page

struct TaPages {
    const int *table;
    int page16, n_pages, last;                             // last: the piece's last granule
    unsigned inv;
    size_t per_page, head;
    // Granules are looked up well ahead of their request, by scalar loads: a vector load's wait would wait for the rows that are on their way too.
    __device__ __forceinline__ TaPick pick(int granule) const
    {
        const int g = min(granule, last);
        // g / page16: inv is ceil(2^32 / page16), so the product is at most one too large
        int p = (int)__umulhi((unsigned)g, inv);
        if (page16 == 1) p = g;
        else if (p * page16 > g) --p;
        p = __builtin_amdgcn_readfirstlane(p);
        return TaPick{reinterpret_cast<const __attribute__((address_space(4))) int *>(reinterpret_cast<uintptr_t>(table))[p], g - p * page16};
    }
    // elements into the K or V half of the pool; an entry outside of it is read as the last page (largest() tells)
    __device__ __forceinline__ size_t place(const TaPick &k) const
    {
        return (size_t)min((unsigned)k.page, (unsigned)n_pages - 1u) * per_page + head + (size_t)k.in * 256;
    }
    // the largest of this lane's entries of the granules first .. last: n_pages or more where one lies outside the pool
    __device__ __forceinline__ unsigned largest(int first, int lane) const
    {
        unsigned most = 0;
        for (int p = first / page16 + lane; p <= last / page16; p += 64) most = max(most, (unsigned)table[p]);
        return most;
    }
};

// largest of the four lanes that share lane % 16
__device__ __forceinline__ float ta_max4(float v)
{
    auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
    p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
constexpr float kTaUp = 9.f, kTaSlack = 6.f;               // (together at most 2^15, of fp16's 2^16)

// 32 bits of "sees position t .. t + 31" of a node: cached positions, then its words; any t, its request's last position behind it or not
__device__ __forceinline__ unsigned ta_window(const unsigned *words, int n_words, int t, int len, int nodes)
{
    const int rel = t - len;                               // node number of the first bit
    if (rel <= -32) return ~0u;
    auto word = [&](int w) -> unsigned {
        if (w < 0) return ~0u;
        const int left = nodes - 32 * w;
        if (left <= 0) return 0u;
        return words[min(w, n_words - 1)] & (left < 32 ? (1u << left) - 1u : ~0u);
    };
    const int w = rel >> 5, sh = rel & 31;
    return __funnelshift_r(word(w), word(w + 1), sh);
}

// four dimensions of a query row's output; STACK: of a node among a stack's rows, as its output projection takes them, heads and remainders
template <int D, bool STACK>
__device__ __forceinline__ void ta_deliver(const TreeAttention &P, const TreeItem &it, int head, int qr, int dim, f32x4 s, float l)
{
    const int G = P.group, node = qr / G, qh = head * G + (qr - node * G);
    f32x4 v = s / l;
    if (l == 0.f) {                                        // every score was minus infinity, or nothing is seen
        const int words = tree_words(P.b.max_nodes);
        bool any = it.len > 0;
        for (int w = 0; w < words; ++w) {
            const int left = it.nodes - 32 * w;
            any = any || (left > 0 && (P.b.masks[(size_t)(it.first + node) * words + w] & (left < 32 ? (1u << left) - 1u : ~0u)));
        }
        const float z = any ? NAN : 0.f;
        v = f32x4{z, z, z, z};
    }
    if constexpr (STACK) {
        const int row = it.first + node, k = qh * D + dim, width = P.n_heads * D;
        __half *to = P.planes + (P.narrow ? ng_at(row, k, width, kNgSet) : pf_at(row, k, width));
        __align__(8) __half hi[4], lo[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) split_half(v[e], hi[e], lo[e]);
        *as_global(reinterpret_cast<ta_u32x2 *>(to)) = *reinterpret_cast<const ta_u32x2 *>(hi);
        *as_global(reinterpret_cast<ta_u32x2 *>(to + (P.narrow ? 8 * kNgSet : kPfLo))) = *reinterpret_cast<const ta_u32x2 *>(lo);
        return;
    }
    ta_u32x2 o;
    o.x = (unsigned)__half_as_ushort(__float2half_rn(v[0])) | (unsigned)__half_as_ushort(__float2half_rn(v[1])) << 16;
    o.y = (unsigned)__half_as_ushort(__float2half_rn(v[2])) | (unsigned)__half_as_ushort(__float2half_rn(v[3])) << 16;
    *as_global(reinterpret_cast<ta_u32x2 *>(P.out + (size_t)(it.first + node) * P.out_stride + (size_t)qh * D + dim)) = o;
}

// 16 bytes that another workgroup of the launch reads or has written, as xwg_store and xwg_load (device scope), at an offset of a buffer
__device__ __forceinline__ __amdgpu_buffer_rsrc_t ta_sums(char *p) { return __builtin_amdgcn_make_buffer_rsrc(p, 0, 0x7fffffff, 0x00020000); }
constexpr int kTaDevice = 16;                              // sc1
__device__ __forceinline__ f32x4 ta_load(__amdgpu_buffer_rsrc_t b, unsigned off) { return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(b, (int)off, 0, kTaDevice)); }
__device__ __forceinline__ void ta_store(__amdgpu_buffer_rsrc_t b, unsigned off, f32x4 v) { __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), b, (int)off, 0, kTaDevice); }

__device__ __forceinline__ void xwg_store2(float *p, float a, float b)                  // p 8-byte aligned
{
    const unsigned long long w = ((unsigned long long)__float_as_uint(b) << 32) | (unsigned long long)__float_as_uint(a);
    __hip_atomic_store(as_global(reinterpret_cast<unsigned long long *>(p)), w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Where a tile's pieces leave their sums: [piece][key head], each [row][D] and then (maximum, weight) of each row
template <int D>
struct TaSlot {
    __amdgpu_buffer_rsrc_t sums;
    float *p;
    unsigned at;                       // bytes
    int tile_rows;
    __device__ __forceinline__ TaSlot(const TreePlanLayout &L, char *plan, const TreeItem &it, int H, int head, int piece)
        : sums(ta_sums(plan + L.sums)), p(reinterpret_cast<float *>(plan + L.sums)),
          at((unsigned)(((size_t)max(it.slot + piece, 0) * H + head) * (L.tile_rows * (D + 2)) * 4)), tile_rows(L.tile_rows)
    {
    }
    __device__ __forceinline__ void put(int i, int dim, f32x4 s) const { ta_store(sums, at + (i * D + dim) * 4, s); }
    __device__ __forceinline__ void put_ml(int i, float m, float l) const { xwg_store2(p + at / 4 + tile_rows * D + 2 * i, m, l); }
};

// The tile's last workgroup adds the pieces in order.
template <int D, bool STACK>
__device__ __forceinline__ void ta_join(const TreeAttention &P, const TreePlanLayout &L, char *plan, const TreeItem &it, int H, int head, int rows, int *last_one)
{
    constexpr int D4 = D / 4;
    const int tid = threadIdx.x;
    unsigned *counter = reinterpret_cast<unsigned *>(plan + L.counters) + (size_t)it.slot * H + head;
    xwg_wait_stores();
    __syncthreads();
    if (tid == 0) *last_one = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (unsigned)it.pieces - 1;
    __syncthreads();
    if (!*last_one) return;
    const TaSlot<D> slot(L, plan, it, H, head, 0);
    const unsigned step = (unsigned)(H * L.tile_rows * (D + 2) * 4);       // from piece to piece
    for (int e = tid; e < rows * D4; e += kTaThreads) {
        const int i = e / D4, dim = 4 * (e - i * D4);
        const unsigned at = slot.at + (i * D + dim) * 4;
        const float *ml_at = slot.p + slot.at / 4 + L.tile_rows * D + 2 * i;
        float M = kTaLowest, l = 0.f;
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
        constexpr int AT = 12;                             // in flight together (past the last: the last again)
        for (int z = 0; z < it.pieces; z += AT) {
            float2 ml[AT];
            f32x4 a[AT];
#pragma unroll
            for (int u = 0; u < AT; ++u) {
                const int q = min(z + u, it.pieces - 1);
                ml[u] = xwg_load2(ml_at + (size_t)q * (step / 4));
                a[u] = ta_load(slot.sums, at + q * step);
            }
#pragma unroll
            for (int u = 0; u < AT; ++u) {
                if (z + u >= it.pieces) continue;          // (uniform)
                const float mn = fmaxf(M, ml[u].x), c0 = __builtin_amdgcn_exp2f(M - mn), c1 = __builtin_amdgcn_exp2f(ml[u].x - mn);
                l = l * c0 + ml[u].y * c1;
                s = s * c0 + a[u] * c1;
                M = mn;
            }
        }
        ta_deliver<D, STACK>(P, it, head, it.tile * L.tile_rows + i, dim, s, l);
    }
    if (tid == 0) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

}  // namespace cfpp
