// Attention of drafted trees over a paged cache, the ancestor masks it reads and its launch plan.
//
// A node's output is softmax(q K^T / sqrt d) V over its request's cached positions, which every node sees, and the nodes of its
// own mask.  The query rows of a request that share a key head - its nodes, times the query heads to a key head - are the columns of
// both products (v_mfma_f32_16x16x32_f16), so a K and V row is read once for up to 64 of them:
//   S = K Q^T      (16 positions x 16 query rows): a lane holds row lane % 16 and positions 4 (lane / 16) .. + 3
//   O^T += V^T P^T (16 dimensions x 16 query rows): a lane's 8 K values are the positions of its own scores in two tiles of 16, so
//                  that P needs no exchange.  V goes through LDS of the wavefront's own, transposed, two positions to a word.
// One pass over the positions with the running maximum and sum of the softmax; a workgroup has a piece of a request's positions for one
// key head, its four wavefronts every fourth row of 32 of them, each with sums of its own that are joined in LDS in order.  Requests of
// few rows are cut into pieces until the CUs are full (k_tree_plan); the last workgroup of a tile adds the pieces in order.
// Weights enter the matrix instruction as two fp16 values, head and remainder, 2^14 times their size: 2^-22 of each and 2^-38 of the largest, as near
// as the sums in 32 bits are.  Queries and keys are fp16 as they come.
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include "tree_params.h"
#include "device_utils.h"
#include "half_split.h"

namespace cfpp {

typedef _Float16 ta_f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 ta_f16x4 __attribute__((ext_vector_type(4)));

constexpr int kTaThreads = 256, kTaWaves = kTaThreads / 64, kTaRow = 32, kTaStep = kTaRow * kTaWaves;
constexpr int kTaStride = kTaRow + 4;                      // halves between V's dimensions in LDS
constexpr int kTaWgs = 512;                                // workgroups that the pieces aim at
constexpr float kTaLowest = -3.402823466e38f;

// ---- the plan --------------------------------------------------------------------------------------
TreePlanLayout tree_plan_layout(const PageDims &pg, int n_heads, int requests, int max_rows, int max_nodes, int stride)
{
    TreePlanLayout L;
    const long long group = n_heads / pg.heads;
    L.tile_rows = tree_tile_rows((int)(group * max_nodes));
    const long long each = (group * max_nodes + L.tile_rows - 1) / L.tile_rows * requests, all = group * max_rows / L.tile_rows + requests;
    L.tiles = (int)(each < all ? each : all);
    L.want = (kTaWgs + pg.heads - 1) / pg.heads;
    L.work = L.want + L.tiles;                             // (pieces of a tile: its share of `want`, rounded up)
    size_t o = align_up(sizeof(TreePlanHead), 256);
    L.items = o; o = align_up(o + (size_t)L.work * sizeof(TreeItem), 256);
    L.counters = o; o = align_up(o + (size_t)L.tiles * pg.heads * 4, 256);
    // tiles of more than one piece have less than twice `want` of them in all
    L.sums = o; o = align_up(o + (size_t)2 * L.want * pg.heads * L.tile_rows * (pg.d + 2) * 4, 256);
    L.total = o;
    // what the plan depends on, as one number
    unsigned k = 0x7ee5u;
    for (int v : {pg.heads, pg.d, pg.page, pg.n_pages, n_heads, requests, max_rows, max_nodes, stride}) k = (k ^ (unsigned)v) * 0x9e3779b1u;
    L.key = (int)(k | 1u);
    return L;
}

// Rows of a request that take part: all or none
__device__ __forceinline__ int tree_rows(const PageDims &pg, const TreeBatch &b, int r, int &first)
{
    first = b.row_start[r];
    const int n = b.row_start[r + 1] - first, len = b.lens[r];
    if (n <= 0 || n > b.max_nodes || first < 0 || first + n > b.max_rows || len < 0 || (long long)len + n > (long long)b.stride * pg.page) return 0;
    return b.slots && b.slots[first] < 0 ? 0 : n;
}

// A request's masks by pointer doubling: after round k a node's words hold its 2^k nearest ancestors and itself, and the node that stands
// 2^k above it is known.  One workgroup has a request, one thread a node.
__device__ __forceinline__ void tree_masks(const PageDims &pg, const TreeBatch &b, int r)
{
    constexpr int W = kTreeMaxNodes / 32;
    __shared__ unsigned m[kTreeMaxNodes][W + 1];
    __shared__ int up[kTreeMaxNodes];
    const int i = threadIdx.x, words = tree_words(b.max_nodes);
    int first;
    const int n = tree_rows(pg, b, r, first);
    unsigned own[W];
#pragma unroll
    for (int w = 0; w < W; ++w) own[w] = i >> 5 == w ? 1u << (i & 31) : 0u;
    int at = i < n ? b.parents[first + i] : -1;
    if (at >= i) at = -1;
    for (int k = 1; k < n; k <<= 1) {                      // (uniform)
#pragma unroll
        for (int w = 0; w < W; ++w) m[i][w] = own[w];
        up[i] = at;
        __syncthreads();
        if (at >= 0) {
#pragma unroll
            for (int w = 0; w < W; ++w) own[w] |= m[at][w];
            at = up[at];
        }
        __syncthreads();
    }
    if (i >= n) return;
    int depth = -1;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        depth += __popc(own[w]);
        if (w < words) b.masks[(size_t)(first + i) * words + w] = own[w];
    }
    b.positions[first + i] = b.lens[r] + depth;
}

// The work list, by one workgroup: with tiles_r tiles of query rows, a request's positions are cut into pieces of C, a multiple of what the wavefronts take
// at a time, so that all pieces come to `want` and one more for each tile at most.
__device__ __forceinline__ void tree_work(const PageDims &pg, const TreeBatch &b, int group, const TreePlanLayout &L, char *plan)
{
    __shared__ int items[kTreeMaxRequests], multi[kTreeMaxRequests], tiles[kTreeMaxRequests];     // running sums
    __shared__ int wave_part[3][kTaWaves];
    __shared__ long long wave_total[kTaWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, R = b.requests, each = (R + kTaThreads - 1) / kTaThreads;
    const int lo = min(tid * each, R), hi = min(lo + each, R);
    int first;
    long long total = 0;
    for (int r = lo; r < hi; ++r) {
        const int n = tree_rows(pg, b, r, first), t = (n * group + L.tile_rows - 1) / L.tile_rows;
        tiles[r] = t;
        items[r] = n > 0 ? b.lens[r] + n : 0;              // (positions, for the moment)
        total += (long long)t * items[r];
    }
    for (int m = 1; m < 64; m <<= 1) total += __shfl_xor(total, m, 64);
    if (lane == 0) wave_total[wave] = total;
    __syncthreads();
    total = 0;
    for (int w = 0; w < kTaWaves; ++w) total += wave_total[w];
    const long long least = (total + L.want - 1) / L.want, C = (least + kTaStep - 1) / kTaStep * kTaStep;
    // (C is at least kTaStep wherever there is a position)
    int sum[3] = {0, 0, 0};
    for (int r = lo; r < hi; ++r) {
        const int t = tiles[r], pieces = t > 0 ? (int)((items[r] + C - 1) / C) : 0;
        sum[0] += t * pieces;
        sum[1] += pieces > 1 ? t * pieces : 0;
        sum[2] += t;
        items[r] = sum[0]; multi[r] = sum[1]; tiles[r] = sum[2];
    }
    int before[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        int s = sum[k];
        for (int m = 1; m < 64; m <<= 1) {
            const int o = __shfl_up(s, m, 64);
            if (lane >= m) s += o;
        }
        if (lane == 63) wave_part[k][wave] = s;
        before[k] = s - sum[k];
    }
    __syncthreads();
    for (int k = 0; k < 3; ++k)
        for (int w = 0; w < wave; ++w) before[k] += wave_part[k][w];
    for (int r = lo; r < hi; ++r) { items[r] += before[0]; multi[r] += before[1]; tiles[r] += before[2]; }
    __syncthreads();
    const int n_items = R > 0 ? items[R - 1] : 0;
    if (tid == 0) {
        reinterpret_cast<TreePlanHead *>(plan)->items = n_items;
        reinterpret_cast<TreePlanHead *>(plan)->key = L.key;
    }
    TreeItem *list = reinterpret_cast<TreeItem *>(plan + L.items);
    for (int i = tid; i < n_items; i += kTaThreads) {
        int a = 0, z = R - 1;                              // the first request whose sum is above i
        while (a < z) {
            const int mid = (a + z) >> 1;
            if (items[mid] > i) z = mid;
            else a = mid + 1;
        }
        const int r = a, t0 = r > 0 ? tiles[r - 1] : 0, n_tiles = tiles[r] - t0, at = i - (r > 0 ? items[r - 1] : 0);
        TreeItem it;
        it.request = r;
        it.nodes = tree_rows(pg, b, r, it.first);
        it.len = b.lens[r];
        it.pieces = (items[r] - (r > 0 ? items[r - 1] : 0)) / n_tiles;
        it.piece = at / n_tiles;                           // (the tiles of a piece follow one another: they read the same rows)
        it.tile = at - it.piece * n_tiles;
        it.slot = it.pieces > 1 ? (r > 0 ? multi[r - 1] : 0) + it.tile * it.pieces : -1;
        it.t0 = (int)(it.piece * C);
        it.t1 = (int)min((long long)it.len + it.nodes, (it.piece + 1) * C);
        it.counter = t0 + it.tile;
        it.pad = 0;
        list[i] = it;
    }
    unsigned *counters = reinterpret_cast<unsigned *>(plan + L.counters);
    for (int i = tid; i < L.tiles * pg.heads; i += kTaThreads) counters[i] = 0u;
}

__global__ void __launch_bounds__(kTaThreads) k_tree_plan(PageDims pg, TreeBatch b, int group, TreePlanLayout L, char *plan)
{
    static_assert(kTaThreads == kTreeMaxNodes, "a thread for each node");
    if (blockIdx.x == 0) tree_work(pg, b, group, L, plan);
    else tree_masks(pg, b, (int)blockIdx.x - 1);
}

hipError_t launch_tree_plan(const PageDims &pg, const TreeBatch &b, int n_heads, char *plan, hipStream_t s)
{
    const TreePlanLayout L = tree_plan_layout(pg, n_heads, b.requests, b.max_rows, b.max_nodes, b.stride);
    hipLaunchKernelGGL(k_tree_plan, dim3(b.requests + 1), dim3(kTaThreads), 0, s, pg, b, n_heads / pg.heads, L, plan);
    return hipGetLastError();
}

// ---- the attention -----------------------------------------------------------------------------------
// A granule of 16 positions lies in one page.
struct TaPlace { size_t at; bool good; };                  // elements into the K or V half of the pool

struct TaPages {
    const int *table;
    int page16, n_pages, last;                             // last: the piece's last granule
    unsigned inv;
    size_t per_page, head;
    __device__ __forceinline__ TaPlace place(int granule) const
    {
        const int g = min(granule, last);
        // g / page16: inv is ceil(2^32 / page16), so the product is at most one too large
        int p = (int)__umulhi((unsigned)g, inv);
        if (page16 == 1) p = g;
        else if (p * page16 > g) --p;
        const int page = __builtin_amdgcn_readfirstlane(table[p]);
        TaPlace w;
        w.good = (unsigned)page < (unsigned)n_pages;
        w.at = (size_t)(w.good ? page : 0) * per_page + head + (size_t)(g - p * page16) * 256;
        return w;
    }
};

// what a wavefront holds of a row of 32 positions
template <int D>
struct TaRow {
    static constexpr int KS = (D + 31) / 32, UN = (D / 8 * (kTaRow / 2) + 63) / 64;
    u32x4 k[2][KS], v[UN][2];
    bool good[2];
    __device__ __forceinline__ void request(const __half *K, const __half *V, const TaPages &pages, unsigned slab, int row, int lane)
    {
        const int n = lane & 15, kg = lane >> 4;
        TaPlace w[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            w[t] = pages.place(2 * row + t);
            good[t] = w[t].good;
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int s = 0; s < KS; ++s) k[t][s] = load16_stream(K + w[t].at + (unsigned)min(2 * s + (kg >> 1), D / 16 - 1) * slab + n * 16u + (kg & 1) * 8u);
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            const int e = min(lane + 64 * u, D / 8 * (kTaRow / 2) - 1), pc = e / (kTaRow / 2), tp = e % (kTaRow / 2);
            const __half *from = V + (tp >= 8 ? w[1].at : w[0].at) + (unsigned)(pc >> 1) * slab + (unsigned)(2 * (tp & 7)) * 16u + (pc & 1) * 8u;
#pragma unroll
            for (int i = 0; i < 2; ++i) v[u][i] = load16_stream(from + 16 * i);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    // V, transposed, to LDS: [dimension][kTaStride]; positions from `end` on as zeros
    __device__ __forceinline__ void store(__half *vt, int row, int end, int lane) const
    {
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            const int e = lane + 64 * u, pc = e / (kTaRow / 2), tp = e % (kTaRow / 2), t = row * kTaRow + 2 * tp;
            if (D / 8 * (kTaRow / 2) % 64 != 0 && e >= D / 8 * (kTaRow / 2)) break;
            const bool ok = tp >= 8 ? good[1] : good[0];
            const u32x4 a = ok && t < end ? v[u][0] : u32x4{0u, 0u, 0u, 0u}, b = ok && t + 1 < end ? v[u][1] : u32x4{0u, 0u, 0u, 0u};
            unsigned *to = reinterpret_cast<unsigned *>(vt + 8 * pc * kTaStride) + tp;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                to[2 * j * (kTaStride / 2)] = __builtin_amdgcn_perm(b[j], a[j], 0x05040100u);
                to[(2 * j + 1) * (kTaStride / 2)] = __builtin_amdgcn_perm(b[j], a[j], 0x07060302u);
            }
        }
    }
};

// largest and sum over the four lanes that share lane % 16
__device__ __forceinline__ float ta_max4(float v)
{
    auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
    p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float ta_sum4(float v)
{
    auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

constexpr float kTaUp = 14.f;                              // weights are 2^14 times their size

// 32 bits of "sees position t .. t + 31" of a node: cached positions, then its words; t a multiple of 32, its request's last position behind it or not
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

// One wavefront, one query row: its sums over the wavefront's rows in fp32, position by position, unseen ones left out
template <int D>
__device__ __forceinline__ void ta_alone(const TreeAttention &P, const TreeItem &it, const TaPages &pages, const __half *K, const __half *V, const unsigned *mask,
                                         const __half *q, int row0, int lane, float *o_out, float *m_out, float *l_out)
{
    constexpr int NE = (D + 63) / 64;
    const float scale = 1.44269504088896340736f / sqrtf((float)D);
    const unsigned slab = (unsigned)P.pg.page * 16u;
    float qs[NE], o[NE], m = kTaLowest, l = 0.f;
    unsigned at[NE];
#pragma unroll
    for (int e = 0; e < NE; ++e) {
        const int dim = min(lane + 64 * e, D - 1);
        at[e] = (unsigned)(dim >> 4) * slab + (dim & 15);
        qs[e] = lane + 64 * e < D ? __half2float(q[dim]) : 0.f;
        o[e] = 0.f;
    }
    for (int row = row0; row * kTaRow < it.t1; row += kTaWaves) {
        for (int t = row * kTaRow; t < min(row * kTaRow + kTaRow, it.t1); ++t) {
            const int node = t - it.len;
            if (node >= 0 && !((mask[node >> 5] >> (node & 31)) & 1)) continue;        // (uniform)
            const TaPlace w = pages.place(t >> 4);
            const unsigned in = (unsigned)(t & 15) * 16u;
            float s = 0.f;
#pragma unroll
            for (int e = 0; e < NE; ++e) s = lane + 64 * e < D ? fmaf(qs[e], __half2float(K[w.at + at[e] + in]), s) : s;
            s = w.good ? wave_sum(s) * scale : NAN;
            const float mn = fmaxf(m, s), corr = __builtin_amdgcn_exp2f(m - mn), p = __builtin_amdgcn_exp2f(s - (mn - kTaUp));
            m = mn;
            l = l * corr + p;
#pragma unroll
            for (int e = 0; e < NE; ++e) o[e] = fmaf(p, w.good ? __half2float(V[w.at + at[e] + in]) : 0.f, o[e] * corr);
        }
    }
#pragma unroll
    for (int e = 0; e < NE; ++e)
        if (lane + 64 * e < D) o_out[lane + 64 * e] = o[e];
    if (lane == 0) { *m_out = m; *l_out = l; }
}

template <int D>
constexpr int ta_lds()                                     // V; then the wavefronts' sums of 16 query rows
{
    const int v = kTaWaves * D * kTaStride * 2, w = kTaWaves * 16 * (D + 2) * 4;
    return v > w ? v : w;
}

template <int D, int QT>
__global__ void __launch_bounds__(kTaThreads, 2) k_tree_attention(TreeAttention P, TreePlanLayout L, char *plan)
{
    constexpr int KS = TaRow<D>::KS, NT = D / 16, TQ = 16 * QT, W = kTaWaves;
    __shared__ __align__(16) char mem[ta_lds<D>()];
    constexpr bool LDS_Q = QT * KS > 8;
    __shared__ __align__(16) u32x4 sq[LDS_Q ? QT * KS : 1][LDS_Q ? 64 : 1];
    __shared__ unsigned smask[TQ][kTreeMaxNodes / 32];
    __shared__ int last_one;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, kg = lane >> 4;
    const int H = P.pg.heads, item = (int)blockIdx.x / H, head = (int)blockIdx.x - item * H;
    const TreePlanHead &plan_head = *reinterpret_cast<const TreePlanHead *>(plan);
    if (plan_head.key != L.key || item >= plan_head.items) return;     // (a plan that was made for other sizes, or never)
    const TreeItem it = reinterpret_cast<const TreeItem *>(plan + L.items)[item];
    const int G = P.group, words = tree_words(P.b.max_nodes), n_rows = it.nodes * G;
    const __half *K = P.pool, *V = P.pool + page_which_elems(P.pg);
    const unsigned slab = (unsigned)P.pg.page * 16u;
    TaPages pages;
    pages.table = P.b.table + (size_t)it.request * P.b.stride;
    pages.page16 = P.pg.page >> 4; pages.n_pages = P.pg.n_pages; pages.last = (it.t1 - 1) >> 4; pages.inv = P.page16_inv;
    pages.per_page = (size_t)H * page_head_elems(P.pg);
    pages.head = (size_t)head * page_head_elems(P.pg);
    TaRow<D> r;
    const int row0 = it.t0 / kTaRow + wave;
    r.request(K, V, pages, slab, row0, lane);
    // query rows: node (tile TQ + i) / G, query head (head G + the rest); those past the last are the last again
    const bool tail = it.t1 > it.len;
    if (tail) {
        for (int e = tid; e < TQ * words; e += kTaThreads) {
            const int i = e / words, node = min(it.tile * TQ + i, n_rows - 1) / G;
            smask[i][e - i * words] = P.b.masks[(size_t)(it.first + node) * words + (e - i * words)];
        }
    }
    auto query = [&](int i) {
        const int qr = min(it.tile * TQ + i, n_rows - 1), node = qr / G;
        return P.q + (size_t)(it.first + node) * P.q_stride + (size_t)(head * G + (qr - node * G)) * D;
    };
    // Q^T: dimensions 32 s + 8 kg .. + 7 of query row col; in registers, or, where these are short, in LDS
    auto fragment = [&](int j, int s) {
        const bool real = D % 32 == 0 || 32 * s + 8 * kg < D;
        u32x4 x = load16(query(16 * j + col) + (real ? 32 * s + 8 * kg : 0));
        if (!real) x = u32x4{0u, 0u, 0u, 0u};
        return x;
    };
    u32x4 Qr[LDS_Q ? 1 : QT][LDS_Q ? 1 : KS];
    if constexpr (LDS_Q) {
        for (int j = wave; j < QT; j += W)
#pragma unroll
            for (int s = 0; s < KS; ++s) sq[j * KS + s][lane] = fragment(j, s);
    } else {
#pragma unroll
        for (int j = 0; j < QT; ++j)
#pragma unroll
            for (int s = 0; s < KS; ++s) Qr[j][s] = fragment(j, s);
    }
    if (tail || LDS_Q) __syncthreads();                    // (uniform)
    auto Q = [&](int j, int s) -> ta_f16x8 {
        if constexpr (LDS_Q) return __builtin_bit_cast(ta_f16x8, sq[j * KS + s][lane]);
        else return __builtin_bit_cast(ta_f16x8, Qr[j][s]);
    };
    const float scale = 1.44269504088896340736f / sqrtf((float)D);
    f32x4 O[QT][NT];
    float m_run[QT], l_run[QT];                            // l_run: of this lane's positions
#pragma unroll
    for (int j = 0; j < QT; ++j) {
        m_run[j] = kTaLowest;
        l_run[j] = 0.f;
#pragma unroll
        for (int t = 0; t < NT; ++t) O[j][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    __half *vt = reinterpret_cast<__half *>(mem) + wave * D * kTaStride;
    for (int row = row0; row * kTaRow < it.t1; row += W) {
        r.store(vt, row, it.t1, lane);
        asm volatile("" ::: "memory");                     // (LDS takes a wavefront's accesses in order)
        f32x4 S[QT][2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int j = 0; j < QT; ++j) S[j][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                u32x4 k = r.k[t][s];
                if (D % 32 != 0 && s == KS - 1 && 32 * s + 8 * kg >= D) k = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
                for (int j = 0; j < QT; ++j) S[j][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(ta_f16x8, k), Q(j, s), S[j][t], 0, 0, 0);
            }
        }
        const bool good[2] = {r.good[0], r.good[1]};
        r.request(K, V, pages, slab, row + W, lane);
        const bool masked = row * kTaRow + kTaRow > it.len || !good[0] || !good[1];    // (uniform)
        ta_f16x8 ph[QT], pl[QT];
#pragma unroll
        for (int j = 0; j < QT; ++j) {
            unsigned window = ~0u;
            if (masked) window = ta_window(smask[16 * j + col], words, row * kTaRow, it.len, it.nodes);
            float most = -INFINITY;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float s = S[j][t][e] * scale;
                    if (masked) {
                        s = good[t] ? s : NAN;
                        s = (window >> (16 * t + 4 * kg + e)) & 1 ? s : -INFINITY;
                    }
                    S[j][t][e] = s;
                    most = fmaxf(most, s);
                }
            most = ta_max4(most);
            if (__any(most > m_run[j])) {
                const float mn = fmaxf(m_run[j], most), corr = __builtin_amdgcn_exp2f(m_run[j] - mn);
                m_run[j] = mn;
                l_run[j] *= corr;
#pragma unroll
                for (int t = 0; t < NT; ++t) O[j][t] *= corr;
            }
            const float base = m_run[j] - kTaUp;
            float sum = 0.f;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p = split_value(__builtin_amdgcn_exp2f(S[j][t][e] - base));
                    const _Float16 h = (_Float16)p;
                    sum += p;
                    ph[j][4 * t + e] = h;
                    pl[j][4 * t + e] = (_Float16)(p - (float)h);
                }
            l_run[j] += sum;
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const __half *at = vt + (16 * t + col) * kTaStride + 4 * kg;
            const ta_f16x4 v0 = *reinterpret_cast<const ta_f16x4 *>(at), v1 = *reinterpret_cast<const ta_f16x4 *>(at + 16);
            const ta_f16x8 v = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
            for (int j = 0; j < QT; ++j) {
                O[j][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, ph[j], O[j][t], 0, 0, 0);
                O[j][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pl[j], O[j][t], 0, 0, 0);
            }
        }
        asm volatile("" ::: "memory");
    }
    // The wavefronts' sums, 16 query rows at a time: maxima and weights [wave][row], sums [wave][row][D] in the place of V
    float *wp = reinterpret_cast<float *>(mem), *wm = wp + W * 16 * D, *wl = wm + W * 16;
    float *sums = reinterpret_cast<float *>(plan + L.sums);
    const size_t slot_size = (size_t)TQ * (D + 2);
    float *slot = sums + ((size_t)(it.slot + it.piece) * H + head) * slot_size;        // (single pieces: not used)
    auto deliver = [&](int i, int dim, float s, float l) {
        const int qr = it.tile * TQ + i;
        if (qr >= n_rows) return;
        const int node = qr / G, qh = head * G + (qr - node * G);
        float v = s / l;
        if (l == 0.f) {                                    // every score was minus infinity, or nothing is seen
            bool any = it.len > 0;
            for (int w = 0; w < words; ++w) {
                const int left = it.nodes - 32 * w;
                any = any || (left > 0 && (P.b.masks[(size_t)(it.first + node) * words + w] & (left < 32 ? (1u << left) - 1u : ~0u)));
            }
            v = any ? NAN : 0.f;
        }
        P.out[(size_t)(it.first + node) * P.out_stride + (size_t)qh * D + dim] = __float2half_rn(v);
    };
#pragma unroll
    for (int j = 0; j < QT; ++j) {
        const float l = ta_sum4(l_run[j]);
        bool finite = fabsf(l) < INFINITY;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) finite = finite && fabsf(O[j][t][e]) < INFINITY;
        const unsigned long long again = __ballot(!finite);            // (bit i: query row i % 16)
        __syncthreads();                                   // V, or the rows before these, have been read
#pragma unroll
        for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4 *>(wp + (wave * 16 + col) * D + 16 * t + 4 * kg) = O[j][t];
        if (kg == 0) { wm[wave * 16 + col] = m_run[j]; wl[wave * 16 + col] = l; }
        if (again) {                                       // (uniform)
            asm volatile("" ::: "memory");
            for (int i = 0; i < 16; ++i)
                if (again & (0x0001000100010001ull << i))
                    ta_alone<D>(P, it, pages, K, V, smask[16 * j + i], query(16 * j + i), row0, lane, wp + (wave * 16 + i) * D, wm + wave * 16 + i, wl + wave * 16 + i);
        }
        __syncthreads();
        for (int e = tid; e < 16 * D; e += kTaThreads) {
            const int i = e / D, dim = e - i * D;
            float M = wm[i], l = 0.f, s = 0.f;
#pragma unroll
            for (int w = 1; w < W; ++w) M = fmaxf(M, wm[w * 16 + i]);
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float ew = __builtin_amdgcn_exp2f(wm[w * 16 + i] - M);
                l += wl[w * 16 + i] * ew;
                s += wp[(w * 16 + i) * D + dim] * ew;
            }
            if (it.pieces == 1) {
                deliver(16 * j + i, dim, s, l);
            } else {
                xwg_store(slot + (16 * j + i) * D + dim, s);
                if (dim == 0) { xwg_store(slot + TQ * D + 16 * j + i, M); xwg_store(slot + TQ * D + TQ + 16 * j + i, l); }
            }
        }
    }
    if (it.pieces == 1) return;
    // the tile's last workgroup adds the pieces in order
    unsigned *counter = reinterpret_cast<unsigned *>(plan + L.counters) + (size_t)it.counter * H + head;
    xwg_wait_stores();
    __syncthreads();
    if (tid == 0) last_one = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (unsigned)it.pieces - 1;
    __syncthreads();
    if (!last_one) return;
    const float *from = sums + ((size_t)it.slot * H + head) * slot_size;
    const size_t step = (size_t)H * slot_size;             // from piece to piece
    const int rows = min(TQ, n_rows - it.tile * TQ);
    for (int e = tid; e < rows * D; e += kTaThreads) {
        const int i = e / D, dim = e - i * D;
        float M = kTaLowest, l = 0.f, s = 0.f;
        constexpr int AT = 8;                              // in flight together (past the last: the last again)
        for (int z = 0; z < it.pieces; z += AT) {
            float mj[AT], lj[AT], oj[AT];
#pragma unroll
            for (int u = 0; u < AT; ++u) {
                const float *f = from + (size_t)min(z + u, it.pieces - 1) * step;
                mj[u] = xwg_load(f + TQ * D + i);
                lj[u] = xwg_load(f + TQ * D + TQ + i);
                oj[u] = xwg_load(f + i * D + dim);
            }
#pragma unroll
            for (int u = 0; u < AT; ++u) {
                if (z + u >= it.pieces) continue;          // (uniform)
                const float mn = fmaxf(M, mj[u]), c0 = __builtin_amdgcn_exp2f(M - mn), c1 = __builtin_amdgcn_exp2f(mj[u] - mn);
                l = l * c0 + lj[u] * c1;
                s = s * c0 + oj[u] * c1;
                M = mn;
            }
        }
        deliver(i, dim, s, l);
    }
    if (tid == 0) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <int D>
static hipError_t launch_of(const TreeAttention &P, const TreePlanLayout &L, char *plan, hipStream_t s)
{
    const dim3 grid((unsigned)L.work * P.pg.heads), block(kTaThreads);
    switch (L.tile_rows) {
    case 16: hipLaunchKernelGGL((k_tree_attention<D, 1>), grid, block, 0, s, P, L, plan); break;
    case 32: hipLaunchKernelGGL((k_tree_attention<D, 2>), grid, block, 0, s, P, L, plan); break;
    default: hipLaunchKernelGGL((k_tree_attention<D, 4>), grid, block, 0, s, P, L, plan); break;
    }
    return hipGetLastError();
}

hipError_t launch_tree_attention(const TreeAttention &A, char *plan, hipStream_t s)
{
    TreeAttention P = A;
    const TreePlanLayout L = tree_plan_layout(P.pg, P.n_heads, P.b.requests, P.b.max_rows, P.b.max_nodes, P.b.stride);
    const unsigned page16 = (unsigned)P.pg.page >> 4;
    P.page16_inv = (unsigned)(((1ull << 32) + page16 - 1) / page16);
    switch (P.pg.d) {
    case 64: return launch_of<64>(P, L, plan, s);
    case 80: return launch_of<80>(P, L, plan, s);
    default: return launch_of<128>(P, L, plan, s);
    }
}

}  // namespace cfpp
