// Attention over a cache in 8 bits: the nodes of a step's requests, usually one new token each, over their request's cached positions and
// what their masks show.  Batch, plan, masks and the sums that pieces leave are those of tree_attention.hip.
//
// A position's K and V rows of a head are codes times a scale: k = c a_K / C, v = c a_V / C, a the row's largest absolute value and C the largest
// code (127, 448).  With s_t = q . c_t (a_K / C) log2(e) / sqrt d the output is sum_t 2^(s_t) c_t (a_V / C) / sum_t 2^(s_t).  Codes are small
// numbers that fp16 holds exactly, so both products run on v_mfma_f32_16x16x32_f16 with the codes as they are, and the scales go to the scores
// and to the weights:
//   S = K Q^T      (16 positions x 16 query rows)
//   O^T += V^T P^T (16 dimensions x 16 query rows), P_t = 2^(s_t) a_V
// A wavefront has 64 positions at a time, one granule of 16 to each group of 16 lanes: tile T of S has positions 4 T .. 4 T + 3 of all four
// granules, so that after four tiles a lane holds the 16 positions of its own group's granule - the ones whose V codes, 16 bytes of its
// dimension, it loads.  P needs no exchange, V no transposition: the granule holds V by dimension and K in the tiles' order, and every load
// is a run of at least 256 bytes.  Nothing goes through LDS but the wavefronts' sums at the end.
//
// Bound by the way of the codes from memory once there are many (32 requests behind 3000 to 8191 of 32 heads of 128: 1.55 GB in 251 us, 6.2 TB/s of the 7.0
// that reads reach; 64 requests of up to 3000 positions and 8 heads of 128: 222 MB in 47.5, 4.7).  Where there are few it is bound by launch and first loads (one token
// behind 128 positions of 8 heads of 64, a piece to each head, 6.2 us) and by the pieces' way to each other through memory, which no split made shorter (behind 4096 of 32
// heads of 80, 16 pieces, 12.2; behind 131072 of two heads of 64 with 8 query heads each 16.9).  More pieces: 768 to 2048 workgroups 52 to 56 us for the 64 requests;
// workgroups of 8 wavefronts 54; a third workgroup to a CU needs 20 more registers than head_dim 128 leaves.
//
// More than 16 query rows to a request are taken 16 at a time, each time with the codes read again: simple, and right for a few drafted nodes, but from 33 rows on an fp16 pool is
// the faster one (64 requests of up to 3000 positions of hidden 2560, fp16 / int8: 9 nodes 163 / 107 us, 36 nodes 181 / 298; 8 requests of 32 nodes 92 / 88, of 64 113 / 159).
//
// What enters the second product is fp16, head cut off and exact remainder cut off, 2^-21 of it.  a_V may be anything from 2^-24 to 2^16, so the
// reference of the running maximum is that of s_t + e_t with a_V = f_t 2^(e_t): the largest *contribution* is near 2^9 whatever the scales are, and the weight
// itself, for the sum, is 2^(s_t + e_t) 2^(-e_t) in fp32.
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include "tree_blocks.h"

namespace cfpp {

typedef _Float16 p8_f16x2 __attribute__((ext_vector_type(2)));

constexpr int kP8Step = 64;                                // positions to a wavefront at a time

// four codes as fp16: exact
template <bool INT8>
__device__ __forceinline__ ta_u32x2 p8_values(unsigned x)
{
    ta_u32x2 r;
    if constexpr (INT8) {
        x ^= 0x80808080u;                                  // c + 128, then 0x6400 | (c + 128) is 1024 + 128 + c
        const p8_f16x2 off = {(_Float16)-1152.f, (_Float16)-1152.f};
        r[0] = __builtin_bit_cast(unsigned, __builtin_bit_cast(p8_f16x2, __builtin_amdgcn_perm(0x64646464u, x, 0x04010400u)) + off);
        r[1] = __builtin_bit_cast(unsigned, __builtin_bit_cast(p8_f16x2, __builtin_amdgcn_perm(0x64646464u, x, 0x04030402u)) + off);
    } else {
        r[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)x, 1.f, false));
        r[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)x, 1.f, true));
    }
    return r;
}
template <bool INT8>
__device__ __forceinline__ ta_f16x8 p8_values8(unsigned a, unsigned b)
{
    const ta_u32x2 x = p8_values<INT8>(a), y = p8_values<INT8>(b);
    return __builtin_bit_cast(ta_f16x8, u32x4{x[0], x[1], y[0], y[1]});
}

template <bool ONCE, class T>
__device__ __forceinline__ T p8_load(const unsigned char *p)
{
    if constexpr (ONCE) return __builtin_nontemporal_load(as_global(reinterpret_cast<const T *>(p)));
    else return *as_global(reinterpret_cast<const T *>(p));
}

// what a wavefront holds of 64 positions
template <int D, bool ONCE>
struct P8Row {
    static constexpr int KL = D / 64, NT = D / 16;
    static constexpr bool ODD = D % 64 != 0;               // 16 dimensions are left: 4 to each group of lanes
    u32x4 k[4][KL], v[NT], ka[2], va[2];
    unsigned kt[ODD ? 4 : 1];
    // gk, gv: this lane's granules
    __device__ __forceinline__ void keys(const unsigned char *gk, int lane)
    {
        const unsigned char *p = gk + (lane >> 4) * 64 + (lane & 3) * 16;
#pragma unroll
        for (int T = 0; T < 4; ++T) {
#pragma unroll
            for (int b = 0; b < KL; ++b) k[T][b] = p8_load<ONCE, u32x4>(p + T * 4 * D + b * 256);
            if constexpr (ODD) kt[T] = p8_load<ONCE, unsigned>(gk + T * 4 * D + KL * 256 + (lane & 3) * 16 + (lane >> 4) * 4);
        }
    }
    __device__ __forceinline__ void values(const unsigned char *gv, int lane)
    {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            ka[u] = p8_load<ONCE, u32x4>(gv + 32 * D + 16 * u);
            va[u] = p8_load<ONCE, u32x4>(gv + 32 * D + 32 + 16 * u);
        }
        const unsigned char *p = gv + 16 * D + (lane & 15) * 16;
#pragma unroll
        for (int t = 0; t < NT; ++t) v[t] = p8_load<ONCE, u32x4>(p + t * 256);
    }
};

// sum over the four lanes that share lane % 16
__device__ __forceinline__ float p8_sum4(float v)
{
    auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// The pieces of a tile of up to 16 query rows, added in order.  Up to kP8Join by the last workgroup that ends, more by the last ones of groups of about as many
// as there are groups, whose sums the last of these adds: 128 pieces one after the other would be eleven trips to memory of a single workgroup
// (one token of two heads of 64 behind 131072 positions 24.6 -> 16.6 us); 16 are one trip.
constexpr int kP8Join = 16;
template <int D>
__device__ __forceinline__ void p8_join(const TreeAttention &P, const TreePlanLayout &L, char *plan, const TreeItem &it, int H, int head, int rows, int *last_one)
{
    constexpr int D4 = D / 4, AT = 16, EACH = (16 * D4 + kTaThreads - 1) / kTaThreads;
    const int tid = threadIdx.x;
    const unsigned step = (unsigned)(H * L.tile_rows * (D + 2) * 4);       // from piece to piece
    unsigned *counters = reinterpret_cast<unsigned *>(plan + L.counters);
    auto last = [&](int number, int of) {                  // whether this workgroup is the last of so many; the counter is zero again then
        unsigned *c = counters + (size_t)number * H + head;
        xwg_wait_stores();
        __syncthreads();
        if (tid == 0) {
            const bool is = __hip_atomic_fetch_add(c, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (unsigned)of - 1;
            *last_one = is;
            if (is) __hip_atomic_store(c, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        return *last_one != 0;
    };
    // pieces first, first + apart, ..: `n` of them
    f32x4 sum[EACH];
    float m[EACH], l[EACH];
    auto add = [&](int first, int apart, int n) {
        const TaSlot<D> slot(L, plan, it, H, head, first);
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            const int e = tid + k * kTaThreads, i = min(e / D4, rows - 1), dim = 4 * (e - e / D4 * D4);
            const unsigned at = slot.at + (i * D + dim) * 4;
            const float *ml_at = slot.p + slot.at / 4 + L.tile_rows * D + 2 * i;
            m[k] = kTaLowest; l[k] = 0.f; sum[k] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (k > 0 && k * kTaThreads >= rows * D4) break;               // (uniform)
            for (int z = 0; z < n; z += AT) {
                float2 ml[AT];
                f32x4 a[AT];
#pragma unroll
                for (int u = 0; u < AT; ++u) {             // (past the last: the last again)
                    const int q = min(z + u, n - 1) * apart;
                    ml[u] = xwg_load2(ml_at + (size_t)q * (step / 4));
                    a[u] = ta_load(slot.sums, at + q * step);
                }
#pragma unroll
                for (int u = 0; u < AT; ++u) {
                    if (z + u >= n) continue;              // (uniform)
                    const float mn = fmaxf(m[k], ml[u].x), c0 = __builtin_amdgcn_exp2f(m[k] - mn), c1 = __builtin_amdgcn_exp2f(ml[u].x - mn);
                    l[k] = l[k] * c0 + ml[u].y * c1;
                    sum[k] = sum[k] * c0 + a[u] * c1;
                    m[k] = mn;
                }
            }
        }
    };
    int apart = 1, groups = it.pieces;
    if (it.pieces > kP8Join) {
        while (apart * apart < it.pieces) ++apart;
        groups = (it.pieces + apart - 1) / apart;
        const int g = it.piece / apart, first = g * apart, n = min(apart, it.pieces - first);
        if (!last(it.slot + first, n)) return;
        add(first, 1, n);
        __syncthreads();                                   // (the maxima have been read)
        const TaSlot<D> slot(L, plan, it, H, head, first);
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            const int e = tid + k * kTaThreads, i = e / D4, dim = 4 * (e - i * D4);
            if (i >= rows) continue;
            slot.put(i, dim, sum[k]);
            if (dim == 0) slot.put_ml(i, m[k], l[k]);
        }
    }
    // (the first group has the tile's own number, and its second piece's number is no group's)
    if (!last(it.pieces > kP8Join ? it.slot + 1 : it.slot, groups)) return;
    add(0, apart, groups);
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        const int e = tid + k * kTaThreads, i = e / D4, dim = 4 * (e - i * D4);
        if (i < rows) ta_deliver<D, false>(P, it, head, it.tile * L.tile_rows + i, dim, sum[k], l[k]);
    }
}

// ONCE: every row is read by one workgroup only
template <int D, bool INT8, bool ONCE>
__global__ void __launch_bounds__(kTaThreads, 2) k_page8_attention(TreeAttention P, TreePlanLayout L, const unsigned char *pool, char *plan, int subs)
{
    constexpr int NT = D / 16, KL = D / 64, W = kTaWaves, TR = 16, D4 = D / 4, GB = 32 * D + 64;
    constexpr bool ODD = D % 64 != 0;
    constexpr float C = INT8 ? 127.f : 448.f;
    __shared__ __align__(16) float sums[W * TR * (D + 2)];
    __shared__ unsigned smask[TR][kTreeMaxNodes / 32];
    __shared__ int last_one;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, kg = lane >> 4;
    const int H = P.pg.heads, unit = (int)blockIdx.x / subs, sub = (int)blockIdx.x - unit * subs, item = unit / H, head = unit - item * H;
    const TreePlanHead &plan_head = *reinterpret_cast<const TreePlanHead *>(plan);
    const TreeItem it = reinterpret_cast<const TreeItem *>(plan + L.items)[item];
    if (plan_head.key != L.key || item >= plan_head.items) return;             // (a plan that was made for other sizes, or never)
    const int n_rows = it.nodes * P.group, first = it.tile * L.tile_rows + 16 * sub, rows = min(TR, n_rows - first);
    if (rows <= 0) return;
    TaPages pages;
    pages.table = P.b.table + (size_t)it.request * P.b.stride;
    pages.page16 = P.pg.page >> 4; pages.n_pages = P.pg.n_pages; pages.last = (it.t1 - 1) >> 4; pages.inv = P.page16_inv;
    pages.per_page = (size_t)H * pages.page16;
    pages.head = (size_t)head * pages.page16;
    struct Four { const unsigned char *g[4]; bool bad[4]; };
    auto look = [&](int base) {                            // the granules of positions base .. base + 63
        Four f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const TaPick k = pages.pick((base >> 4) + i);
            f.bad[i] = (unsigned)k.page >= (unsigned)pages.n_pages;
            f.g[i] = pool + ((size_t)min((unsigned)k.page, (unsigned)pages.n_pages - 1u) * pages.per_page + pages.head + k.in) * GB;
        }
        return f;
    };
    auto mine = [](const auto (&x)[4], int i) { const auto a = i & 1 ? x[1] : x[0], b = i & 1 ? x[3] : x[2]; return i & 2 ? b : a; };

    P8Row<D, ONCE> r;
    int base = it.t0 + kP8Step * wave;
    Four f = look(base);
    bool bad = mine(f.bad, kg);
    r.keys(mine(f.g, col >> 2), lane);
    r.values(mine(f.g, kg), lane);
    f = look(base + kP8Step * W);
    const bool tail = it.t1 > it.len;
    const int words = tree_words(P.b.max_nodes);
    if (tail) {
        for (int e = tid; e < TR * words; e += kTaThreads) {
            const int i = e / words, node = min(first + i, n_rows - 1) / P.group;
            smask[i][e - i * words] = P.b.masks[(size_t)(it.first + node) * words + (e - i * words)];
        }
    }
    // Q^T of this lane's query row: dimensions 64 b + 16 kg + 8 h .. + 7
    ta_f16x8 q[KL][2];
    ta_f16x8 qt;
    {
        const int qr = min(first + col, n_rows - 1), node = qr / P.group;
        const __half *at = P.q + (size_t)(it.first + node) * P.q_stride + (size_t)(head * P.group + (qr - node * P.group)) * D;
#pragma unroll
        for (int b = 0; b < KL; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h) q[b][h] = __builtin_bit_cast(ta_f16x8, load16(at + 64 * b + 16 * kg + 8 * h));
        if constexpr (ODD) {
            const ta_u32x2 x = *as_global(reinterpret_cast<const ta_u32x2 *>(at + 64 * KL + 4 * kg));
            qt = __builtin_bit_cast(ta_f16x8, u32x4{x[0], x[1], 0u, 0u});
        }
    }
    if (tail) __syncthreads();                             // (uniform)
    const float scale = 1.44269504088896340736f / sqrtf((float)D) / C;
    f32x4 O[NT];
    float m_run = kTaLowest, l = 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t) O[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (; base < it.t1; base += kP8Step * W) {
        f32x4 S[4];
#pragma unroll
        for (int T = 0; T < 4; ++T) {
            S[T] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int b = 0; b < KL; ++b) {
                S[T] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p8_values8<INT8>(r.k[T][b][0], r.k[T][b][1]), q[b][0], S[T], 0, 0, 0);
                S[T] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p8_values8<INT8>(r.k[T][b][2], r.k[T][b][3]), q[b][1], S[T], 0, 0, 0);
            }
            // Four dimensions of a lane's eight.  Not the instruction of half the depth (v_mfma_f32_16x16x16_f16): the compiler lets a vector instruction overwrite the registers
            // of its third operand three or four places behind it, which is too soon while it still waits for that operand from an instruction of the other depth.  Two of the
            // four sums were wrong; with wait states ahead of it or behind it they were right.  In a chain of one instruction that distance is enough.
            if constexpr (ODD) {
                const ta_u32x2 x = p8_values<INT8>(r.kt[T]);
                S[T] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(ta_f16x8, u32x4{x[0], x[1], 0u, 0u}), qt, S[T], 0, 0, 0);
            }
        }
        const bool more = base + kP8Step * W < it.t1;      // (uniform)
        if (more) r.keys(mine(f.g, col >> 2), lane);
        // s + e: a block table's entry outside the pool makes every score that is seen no number
        const float ks = bad ? NAN : scale;
        const bool masked = base + kP8Step > min(it.len, it.t1);               // (uniform)
        unsigned seen = 0xffffu;                           // of this lane's row and granule
        if (masked) {
            const int t = base + 16 * kg, left = it.t1 - t;
            seen = tail ? ta_window(smask[col], words, t, it.len, it.nodes) : ~0u;
            seen &= left >= 16 ? 0xffffu : left <= 0 ? 0u : (1u << left) - 1u;
        }
        float u[16], most = -INFINITY;
        int e[16];
        float av[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const unsigned a = r.va[i >> 3][(i >> 1) & 3], b = r.ka[i >> 3][(i >> 1) & 3];
            const float2 ah = unpack_h2(a), bh = unpack_h2(b);
            av[i] = i & 1 ? ah.y : ah.x;
            // a_V's exponent: 2^-e a_V is from 1 to 2; a row of zeros has that of fp16's smallest number
            e[i] = max((int)(__float_as_uint(av[i]) >> 23) - 127, -24);
            u[i] = fmaf(S[i >> 2][i & 3], (i & 1 ? bh.y : bh.x) * ks, (float)e[i]);
            if (masked) u[i] = (seen >> i) & 1 ? u[i] : -INFINITY;
            most = fmaxf(most, u[i]);
        }
        if (__any(most > m_run + kTaSlack)) {
            const float mn = fmaxf(m_run, ta_max4(most)), corr = __builtin_amdgcn_exp2f(m_run - mn);
            m_run = mn;
            l *= corr;
#pragma unroll
            for (int t = 0; t < NT; ++t) O[t] *= corr;
        }
        const float up = kTaUp - m_run;
        float minus = -1.f;
        asm("" : "+v"(minus));
        u32x4 hi[2], lo[2];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float p[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int i = 2 * j + h;
                const float x = __builtin_amdgcn_exp2f(u[i] + up), back = __uint_as_float((unsigned)(127 - e[i]) << 23);      // 2^-e
                float w = x * back, y = av[i] * back * x;
                if (masked && !((seen >> i) & 1)) { w = 0.f; y = 0.f; }
                l += w;
                p[h] = split_value(y);
            }
            const auto a = __builtin_amdgcn_cvt_pkrtz(p[0], p[1]);
            const auto b = __builtin_amdgcn_cvt_pkrtz(fmaf((float)a[0], minus, p[0]), fmaf((float)a[1], minus, p[1]));
            hi[j >> 2][j & 3] = __builtin_bit_cast(unsigned, a);
            lo[j >> 2][j & 3] = __builtin_bit_cast(unsigned, b);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            // Bytes 0x7f and 0xff are none of e4m3's numbers and are never written; where nothing was, in positions that no row sees, behind the last or in a page that an
            // entry outside the pool is read as, they may lie, and a weight of zero times NaN is NaN for all rows.  One bit less and they are finite.
            if (!INT8 && masked)
#pragma unroll
                for (int w = 0; w < 4; ++w) r.v[t][w] &= ~((((r.v[t][w] & 0x7f7f7f7fu) + 0x01010101u) >> 7) & 0x01010101u);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const ta_f16x8 v = p8_values8<INT8>(r.v[t][2 * h], r.v[t][2 * h + 1]);
                O[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, __builtin_bit_cast(ta_f16x8, hi[h]), O[t], 0, 0, 0);
                O[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, __builtin_bit_cast(ta_f16x8, lo[h]), O[t], 0, 0, 0);
            }
        }
        if (more) {
            r.values(mine(f.g, kg), lane);
            bad = mine(f.bad, kg);
            f = look(base + 2 * kP8Step * W);
        }
    }
    l = p8_sum4(l);
    // the wavefronts' sums: [wave][row][D], maxima and weights [wave][row]
    float *wm = sums + W * TR * D, *wl = wm + W * TR;
    if (col < rows) {
        const int at = wave * TR + col;
#pragma unroll
        for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4 *>(sums + at * D + 16 * t + 4 * kg) = O[t] * (1.f / C);
        if (kg == 0) { wm[at] = m_run; wl[at] = l; }
    }
    __syncthreads();
    const TaSlot<D> slot(L, plan, it, H, head, it.piece);
    for (int x = tid; x < rows * D4; x += kTaThreads) {
        const int i = x / D4, dim = 4 * (x - i * D4);
        float M = wm[i], lt = 0.f;
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 1; v < W; ++v) M = fmaxf(M, wm[v * TR + i]);
#pragma unroll
        for (int v = 0; v < W; ++v) {
            const float ew = __builtin_amdgcn_exp2f(wm[v * TR + i] - M);
            lt += wl[v * TR + i] * ew;
            s += *reinterpret_cast<const f32x4 *>(sums + (v * TR + i) * D + dim) * ew;
        }
        if (it.pieces == 1) {
            ta_deliver<D, false>(P, it, head, first + i, dim, s, lt);
        } else {
            slot.put(16 * sub + i, dim, s);
            if (dim == 0) slot.put_ml(16 * sub + i, M, lt);
        }
    }
    if (it.pieces > 1 && L.tile_rows <= kTaLastJoins) p8_join<D>(P, L, plan, it, H, head, rows, &last_one);
}

template <int D, bool INT8>
static hipError_t launch_of(const TreeAttention &P, const TreePlanLayout &L, const unsigned char *pool, char *plan, hipStream_t s)
{
    const int subs = page8_subtiles(L);
    const dim3 grid((unsigned)L.work * P.pg.heads * subs);
    if (subs == 1) hipLaunchKernelGGL((k_page8_attention<D, INT8, true>), grid, dim3(kTaThreads), 0, s, P, L, pool, plan, subs);
    else hipLaunchKernelGGL((k_page8_attention<D, INT8, false>), grid, dim3(kTaThreads), 0, s, P, L, pool, plan, subs);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || L.tile_rows <= kTaLastJoins ? e : launch_tree_join(P, L, plan, s);
}

hipError_t launch_page8_attention(const TreeAttention &A, const unsigned char *pool, int type, char *plan, hipStream_t s)
{
    TreeAttention P = A;
    const TreePlanLayout L = tree_plan_layout(P.pg, P.n_heads, P.b.requests, P.b.max_rows, P.b.max_nodes, P.b.stride);
    const unsigned page16 = (unsigned)P.pg.page >> 4;
    P.page16_inv = (unsigned)(((1ull << 32) + page16 - 1) / page16);
    const bool i8 = type == kPage8Int8;
    switch (P.pg.d) {
    case 64: return i8 ? launch_of<64, true>(P, L, pool, plan, s) : launch_of<64, false>(P, L, pool, plan, s);
    case 80: return i8 ? launch_of<80, true>(P, L, pool, plan, s) : launch_of<80, false>(P, L, pool, plan, s);
    default: return i8 ? launch_of<128, true>(P, L, pool, plan, s) : launch_of<128, false>(P, L, pool, plan, s);
    }
}

}  // namespace cfpp
