// Attention of drafted trees over a paged cache, the ancestor masks it reads and its launch plan.
//
// A node's output is softmax(q K^T / sqrt d) V over its request's cached positions, which every node sees, and the nodes of its
// own mask.  The query rows of a request that share a key head - its nodes, times the query heads to a key head - are the columns of
// both products (v_mfma_f32_16x16x32_f16), so a K and V row is read once for up to 128 of them:
//   S = K Q^T      (16 positions x 16 query rows): a lane holds row lane % 16 and positions 4 (lane / 16) .. + 3
//   O^T += V^T P^T (16 dimensions x 16 query rows): a lane's 8 K values are the positions of its own scores in two granules of 16, so
//                  that P needs no exchange.  V goes through LDS as it lies in the pool; ds_read_b64_tr_b16 gives a lane four positions of its
//                  dimension, 512 contiguous bytes to a wavefront.
// One pass over the positions with the running maximum and sum of the softmax.  A workgroup has a piece of a request's positions for one key
// head: up to 32 query rows, its four wavefronts take every fourth row of 32 positions, each with sums of its own that are joined in LDS in
// order (ta_narrow); more query rows, the wavefronts share the query rows and every position goes through LDS once (ta_wide).  Requests are
// cut into pieces until the CUs are full (k_tree_plan), and the pieces' sums are added in order, so a result does not depend on who comes first.
// Weights enter the matrix instruction as two fp16 values, head and remainder, 2^9 times their size: 2^-21 of each and 2^-33 of the largest, as near
// as the sums in 32 bits are.  Queries and keys are fp16 as they come.
//
// Bound and measured (calls in a captured graph, the join included; so are both sides of the rules below, each pair on one card): few query rows by the
// K and V that are read - one token of 8 requests behind 1000 to 8000 positions of hidden 4096 107 us, 5.5 TB/s; 64 requests of up to 9 nodes behind up to
// 3000, four query heads to a key head, 77 us, 4.8 TB/s; 16 of 30 behind 2500 of hidden 2560 70 us, 5.4 TB/s - by the launches and one piece's way through
// them where a single request is short (one token behind 128 positions 6.8 us, 26 behind 4096 18.7 us).  Many query rows are bound by issue: 8 requests
// of 200 to 256 nodes behind 6000 to 8200 of hidden 4096 take 403 - 410 us, 230 GFLOP of the formula's own, 413 issued with the remainders, the sums of the
// weights and the rows that fill tiles: 1.0 PFLOP/s, where a library product of 8192^3 reached 1.1.  Without the remainders an earlier build took 388 of
// 462 us, an error of 2^-11 to each weight: not taken.
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include "tree_params.h"
#include "device_utils.h"
#include "half_split.h"
#include "prefill_device.h"
#include "lds_dma.h"
#include "tree_blocks.h"

namespace cfpp {

// Positions that are not cut.  Of hidden 2560 and one token, whole / cut: behind 500 10.5 / 10.0 us, behind 900 12.0 / 9.7; a piece of 128 is one row to a
// wavefront, and joining pieces costs about what a second row does.
constexpr int kTaWhole = 256;
// Workgroups that the pieces aim at, two to a CU.  With 256 / 512 / 768 / 1024 / 1536: one token of 8 requests behind 8000 117 / 107 / 107 / 104 / 103 us, 64 requests of
// up to 9 nodes 84 / 77 / 85 / 83 / 91, 8 of 256 406 / 405 / 435 / 428 / 439, 64 nodes behind 8000 of hidden 4096 34.6 / 37.7 / 43.7 / 46.9 / 54, 4 requests of 60 nodes
// with four query heads to a key head 48.5 / 44.5 / 55 / 58 / 72.  Two wavefronts more to each SIMD in workgroups of eight instead, in an earlier build: 112 of 104, 20.5 of 18.4.
constexpr int kTaWgs = 512;
// Up to 32 query rows whose pieces would have half as many positions or fewer are given half the workgroups: 26 nodes behind 4096 22.6 / 18.5 us, one token
// there 15.9 / 14.5; tiles of 128 rows are left at kTaWgs, where half of them costs 48.5 us instead of 44.5 (the 4 requests above).
constexpr int kTaShort = 1024;

// ---- the plan --------------------------------------------------------------------------------------
TreePlanLayout tree_plan_layout(const PageDims &pg, int n_heads, int requests, int max_rows, int max_nodes, int stride)
{
    TreePlanLayout L;
    const long long group = n_heads / pg.heads;
    L.tile_rows = tree_tile_rows((int)(group * max_nodes));
    const long long each = (group * max_nodes + L.tile_rows - 1) / L.tile_rows * requests, all = group * max_rows / L.tile_rows + requests;
    L.tiles = (int)(each < all ? each : all);
    L.want = (kTaWgs + pg.heads - 1) / pg.heads;
    L.work = L.want + L.tiles;                             // (pieces of a tile: its share of `want`, to the nearest whole number, and one at least)
    L.piece_step = L.tile_rows <= 32 ? kTaStep : kTaRow;
    size_t o = align_up(sizeof(TreePlanHead), 256);
    L.items = o; o = align_up(o + (size_t)L.work * sizeof(TreeItem), 256);
    L.cut = o; o = align_up(o + (size_t)L.want * sizeof(int), 256);
    // tiles of more than one piece have less than twice `want` of them in all; the first one's number names the tile
    L.counters = o; o = align_up(o + (size_t)2 * L.want * pg.heads * 4, 256);
    L.sums = o; o = align_up(o + (size_t)2 * L.want * pg.heads * L.tile_rows * (pg.d + 2) * 4, 256);
    L.total = o;
    // what the plan depends on, as one number
    unsigned k = 0x7ee5u;
    for (int v : {pg.heads, pg.d, pg.page, pg.n_pages, n_heads, requests, max_rows, max_nodes, stride}) k = (k ^ (unsigned)v) * 0x9e3779b1u;
    L.key = (int)(k | 1u);
    return L;
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

// The work list, by one workgroup: with tiles_r tiles of query rows, a request's positions are cut into equal pieces of about C, multiples of what the
// wavefronts take at a time, so that all pieces come to about `want`.  The requests of the longest pieces come first, in classes of an eighth of C, so that
// short ones fill the end: 64 requests of up to 9 nodes, lengths from 33 to 3000, 87 us in the requests' order and 78 so, of 16 nodes each 109 and 96 (but one
// token of 8 requests 104 and 107).
// L.tiles bounds the tiles of rows that are one request's each.  Where row_start falls, rows can be several requests', whose tiles may be more than the list
// holds: such a batch has no items.
__device__ __forceinline__ void tree_work(const PageDims &pg, const TreeBatch &b, int group, const TreePlanLayout &L, char *plan)
{
    extern __shared__ int tp_sums[];                       // [3][requests]: running sums of the items and of those of cut tiles; tiles, class, first place
    int *items = tp_sums, *multi = tp_sums + b.requests, *place = tp_sums + 2 * b.requests;
    constexpr int CLASSES = 16;
    __shared__ int wave_part[2][kTaWaves], cuts, classes[CLASSES];
    if (threadIdx.x == 0) cuts = 0;
    if (threadIdx.x < CLASSES) classes[threadIdx.x] = 0;
    __shared__ long long wave_total[kTaWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, R = b.requests, each = (R + kTaThreads - 1) / kTaThreads;
    const int lo = min(tid * each, R), hi = min(lo + each, R);
    int first;
    long long total = 0;
    constexpr long long FALLS = 1ll << 53;                 // (512 tiles of 2^30 positions for 4096 requests are less than half of it, it times 256 threads fits)
    bool falls = false;
    for (int r = lo; r < hi; ++r) {
        const int n = tree_rows(pg, b, r, first), t = (n * group + L.tile_rows - 1) / L.tile_rows;
        falls = falls || b.row_start[r + 1] < first;
        place[r] = t;
        items[r] = n > 0 ? b.lens[r] + n : 0;              // (positions, for the moment)
        total += (long long)t * items[r];
    }
    if (falls) total += FALLS;
    for (int m = 1; m < 64; m <<= 1) total += __shfl_xor(total, m, 64);
    if (lane == 0) wave_total[wave] = total;
    __syncthreads();
    total = 0;
    for (int w = 0; w < kTaWaves; ++w) total += wave_total[w];
    falls = total >= FALLS;
    const int want = L.tile_rows <= 32 && total * 2 <= (long long)kTaShort * L.want ? (L.want + 1) / 2 : L.want;
    const long long C = max((total + want - 1) / want, (long long)kTaStep);
    // the nearest number of pieces: they come to 4 / 3 of `want` at most beside those of the tiles that stay whole
    auto piece_size = [&](int x, int pieces) { return ((x + pieces - 1) / pieces + L.piece_step - 1) / L.piece_step * L.piece_step; };
    auto pieces_of = [&](int x) { return x <= kTaWhole ? 1 : max(1, (int)((2 * (long long)x + C) / (2 * C))); };
    int sum[2] = {0, 0};
    for (int r = lo; r < hi; ++r) {
        const int t = falls ? 0 : place[r], x = items[r], n = pieces_of(x), size = piece_size(x, n), pieces = t <= 0 ? 0 : (x + size - 1) / size;
        sum[0] += t * pieces;
        sum[1] += pieces > 1 ? t * pieces : 0;
        items[r] = sum[0]; multi[r] = sum[1];
        const int c = CLASSES - 1 - (int)min(CLASSES - 1LL, 8LL * size / C);
        place[r] = c;
        if (t > 0) atomicAdd(&classes[c], t * pieces);
    }
    int before[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        int s = sum[k];
        for (int m = 1; m < 64; m <<= 1) {
            const int o = __shfl_up(s, m, 64);
            if (lane >= m) s += o;
        }
        if (lane == 63) wave_part[k][wave] = s;
        before[k] = s - sum[k];
    }
    __syncthreads();
    for (int k = 0; k < 2; ++k)
        for (int w = 0; w < wave; ++w) before[k] += wave_part[k][w];
    if (wave == 0) {                                       // where the classes begin
        int s = lane < CLASSES ? classes[lane] : 0;
        const int own = s;
        for (int m = 1; m < CLASSES; m <<= 1) {
            const int o = __shfl_up(s, m, 64);
            if (lane >= m) s += o;
        }
        if (lane < CLASSES) classes[lane] = s - own;
    }
    __syncthreads();
    int last = 0;
    for (int r = lo; r < hi; ++r) {
        const int sums = items[r];
        if (sums > last) place[r] = atomicAdd(&classes[place[r]], sums - last);
        last = sums;
        items[r] = sums + before[0]; multi[r] += before[1];
    }
    __syncthreads();
    const int n_items = R > 0 ? items[R - 1] : 0;
    if (tid == 0) {
        reinterpret_cast<TreePlanHead *>(plan)->items = n_items;
        reinterpret_cast<TreePlanHead *>(plan)->key = L.key;
    }
    TreeItem *list = reinterpret_cast<TreeItem *>(plan + L.items);
    int *cut = reinterpret_cast<int *>(plan + L.cut);
    for (int i = tid; i < n_items; i += kTaThreads) {
        int a = 0, z = R - 1;                              // the first request whose sum is above i
        while (a < z) {
            const int mid = (a + z) >> 1;
            if (items[mid] > i) z = mid;
            else a = mid + 1;
        }
        const int r = a, before = r > 0 ? items[r - 1] : 0, at = i - before;
        TreeItem it;
        it.request = r;                                    // (one that takes part: it has items)
        it.first = b.row_start[r];
        it.nodes = b.row_start[r + 1] - it.first;
        it.len = b.lens[r];
        const int n_tiles = (it.nodes * group + L.tile_rows - 1) / L.tile_rows, to = place[r] + at;
        it.pieces = (items[r] - before) / n_tiles;
        it.piece = at / n_tiles;                           // (the tiles of a piece follow one another: they read the same rows)
        it.tile = at - it.piece * n_tiles;
        it.slot = it.pieces > 1 ? (r > 0 ? multi[r - 1] : 0) + it.tile * it.pieces : -1;
        const int x = it.len + it.nodes, size = piece_size(x, pieces_of(x));
        it.t0 = it.piece * size;
        it.t1 = min(x, it.t0 + size);
        if (it.pieces > 1 && it.piece == 0) cut[atomicAdd(&cuts, 1)] = to;             // (at most want / 1.5; in any order)
        it.pad[0] = it.pad[1] = 0;
        list[to] = it;
    }
    __syncthreads();
    if (tid == 0) reinterpret_cast<TreePlanHead *>(plan)->cuts = cuts;
    unsigned *counters = reinterpret_cast<unsigned *>(plan + L.counters);
    for (int i = tid; i < 2 * L.want * pg.heads; i += kTaThreads) counters[i] = 0u;
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
    hipLaunchKernelGGL(k_tree_plan, dim3(b.requests + 1), dim3(kTaThreads), 3 * b.requests * sizeof(int), s, pg, b, n_heads / pg.heads, L, plan);
    return hipGetLastError();
}

// ---- the attention -----------------------------------------------------------------------------------
constexpr int ta_granule(int D) { return D * 32; }         // bytes of 16 positions of K or V: [d / 16][16][16] fp16

// V of 16 dimensions and a granule, transposed: this lane's dimension lane % 16, positions 4 (lane / 16) .. + 3
__device__ __forceinline__ ta_u32x2 ta_transposed(const char *at, int lane)
{
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 *lds;
    return __builtin_bit_cast(ta_u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(at + lane * 8)));
}

// what a wavefront holds of a row of 32 positions
template <int D>
struct TaRow {
    static constexpr int KS = (D + 31) / 32, PG = 2 * D, UN = 2 * PG / 64;             // PG: pieces of 16 bytes to a granule
    u32x4 k[2][KS], v[UN];
    __device__ __forceinline__ void request(const __half *K, const __half *V, const TaPages &pages, unsigned slab, const TaPick (&pick)[2], int lane)
    {
        const int n = lane & 15, kg = lane >> 4;
        const size_t w[2] = {pages.place(pick[0]), pages.place(pick[1])};
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int s = 0; s < KS; ++s) k[t][s] = load16_stream(K + w[t] + (unsigned)min(2 * s + (kg >> 1), D / 16 - 1) * slab + n * 16u + (kg & 1) * 8u);
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            const int e = lane + 64 * u, t = PG % 64 == 0 ? (64 * u) / PG : e >= PG, i = e - t * PG;
            v[u] = load16_stream(V + (t ? w[1] : w[0]) + (unsigned)(i >> 5) * slab + (i & 31) * 8u);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    // V to LDS as it is: [granule][d / 16][16][16]; positions from `end` on as zeros
    __device__ __forceinline__ void store(char *vt, int row, int end, int lane) const
    {
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            const int e = lane + 64 * u, t = PG % 64 == 0 ? (64 * u) / PG : e >= PG, i = e - t * PG;
            const bool ok = row * kTaRow + 16 * t + ((i >> 1) & 15) < end;
            *reinterpret_cast<u32x4 *>(vt + e * 16) = ok ? v[u] : u32x4{0u, 0u, 0u, 0u};
        }
    }
};

// One wavefront, one query row: its sums over rows row0, row0 + STEP .. of the piece in fp32, unseen positions left out: a lane has a position and half
// of the dimensions for the scores, then the lanes have the dimensions
template <int D, int STEP, class T>
__device__ __forceinline__ void ta_alone(const TreeAttention &P, const TreeItem &it, const TaPages &pages, const __half *K, const __half *V, const unsigned *mask,
                                         const T *q, int row0, int lane, float *o_out, float *m_out, float *l_out)
{
    constexpr int NE = (D + 63) / 64, NS = D / 16, AT = 8;
    const float scale = 1.44269504088896340736f / sqrtf((float)D);
    const unsigned slab = (unsigned)P.pg.page * 16u;
    const int n = lane & 15, t1 = (lane >> 4) & 1, upper = lane >> 5;      // position 16 t1 + n of the row; slabs of the upper half
    float o[NE], m = kTaLowest, l = 0.f;
    unsigned at[NE];
#pragma unroll
    for (int e = 0; e < NE; ++e) {
        const int dim = min(lane + 64 * e, D - 1);
        at[e] = (unsigned)(dim >> 4) * slab + (dim & 15);
        o[e] = 0.f;
    }
    for (int row = row0; row * kTaRow < it.t1; row += STEP) {
        const int t = row * kTaRow + (lane & 31), node = t - it.len;
        const bool sees = t < it.t1 && (node < 0 || ((mask[max(node, 0) >> 5] >> (node & 31)) & 1));
        const unsigned long long seen = __ballot(sees);
        if (!seen) continue;                               // (uniform)
        const TaPick pick[2] = {pages.pick(2 * row), pages.pick(2 * row + 1)};
        const size_t w[2] = {pages.place(pick[0]), pages.place(pick[1])};
        const bool good[2] = {(unsigned)pick[0].page < (unsigned)pages.n_pages, (unsigned)pick[1].page < (unsigned)pages.n_pages};
        const __half *k = K + (t1 ? w[1] : w[0]) + n * 16;
        float s = 0.f;
        for (int sl = upper * ((NS + 1) / 2); sl < (upper ? NS : (NS + 1) / 2); ++sl)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const u32x4 x = load16(k + (unsigned)sl * slab + h * 8);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 f = unpack_h2(x[e]);
                    s = fmaf((float)q[sl * 16 + h * 8 + 2 * e], f.x, s);
                    s = fmaf((float)q[sl * 16 + h * 8 + 2 * e + 1], f.y, s);
                }
            }
        s += __shfl_xor(s, 32, 64);
        s = !sees ? -INFINITY : (t1 ? good[1] : good[0]) ? s * scale : NAN;
        const float mn = fmaxf(m, wave_max(s)), corr = __builtin_amdgcn_exp2f(m - mn), p = sees ? __builtin_amdgcn_exp2f(s - (mn - kTaUp)) : 0.f;
        m = mn;
        l = l * corr + wave_sum(upper ? 0.f : p);
#pragma unroll
        for (int e = 0; e < NE; ++e) o[e] *= corr;
#pragma unroll 1
        for (int i0 = 0; i0 < kTaRow; i0 += AT) {
            const __half *v = V + (i0 < 16 ? w[0] : w[1]) + (i0 & 15) * 16;
            const bool ok = i0 < 16 ? good[0] : good[1];
            float x[AT][NE];
#pragma unroll
            for (int i = 0; i < AT; ++i)
#pragma unroll
                for (int e = 0; e < NE; ++e) x[i][e] = __half2float(v[at[e] + i * 16u]);
#pragma unroll
            for (int i = 0; i < AT; ++i) {
                const float pi = readlane_f(p, i0 + i);
                if ((seen >> (i0 + i)) & 1)                // (uniform)
#pragma unroll
                    for (int e = 0; e < NE; ++e) o[e] = fmaf(pi, ok ? x[i][e] : 0.f, o[e]);
            }
        }
    }
#pragma unroll
    for (int e = 0; e < NE; ++e)
        if (lane + 64 * e < D) o_out[lane + 64 * e] = o[e];
    if (lane == 0) { *m_out = m; *l_out = l; }
}

// What the workgroups of both kernels begin with
template <int D, int TQ, bool STACK>
struct TaStart {
    using Query = std::conditional_t<STACK, float, __half>;
    TreeItem it;
    int head, rows, n_rows;            // key head; query rows of the tile, of the request
    const __half *K, *V;
    unsigned slab;
    TaPages pages;
    __device__ __forceinline__ bool of(const TreeAttention &P, const TreePlanLayout &L, const char *plan)
    {
        const int H = P.pg.heads, item = (int)blockIdx.x / H;
        head = (int)blockIdx.x - item * H;
        const TreePlanHead &plan_head = *reinterpret_cast<const TreePlanHead *>(plan);
        it = reinterpret_cast<const TreeItem *>(plan + L.items)[item];
        if (plan_head.key != L.key || item >= plan_head.items) return false;           // (a plan that was made for other sizes, or never)
        n_rows = it.nodes * P.group;
        rows = min(TQ, n_rows - it.tile * TQ);
        K = P.pool; V = P.pool + page_which_elems(P.pg);
        slab = (unsigned)P.pg.page * 16u;
        pages.table = P.b.table + (size_t)it.request * P.b.stride;
        pages.page16 = P.pg.page >> 4; pages.n_pages = P.pg.n_pages; pages.last = (it.t1 - 1) >> 4; pages.inv = P.page16_inv;
        pages.per_page = (size_t)H * page_head_elems(P.pg);
        pages.head = (size_t)head * page_head_elems(P.pg);
        return true;
    }
    // masks of the tile's query rows; those past the last are the last again (a barrier behind it)
    __device__ __forceinline__ void masks(const TreeAttention &P, unsigned (*smask)[kTreeMaxNodes / 32]) const
    {
        const int words = tree_words(P.b.max_nodes);
        for (int e = threadIdx.x; e < TQ * words; e += kTaThreads) {
            const int i = e / words, node = min(it.tile * TQ + i, n_rows - 1) / P.group;
            smask[i][e - i * words] = P.b.masks[(size_t)(it.first + node) * words + (e - i * words)];
        }
    }
    // query row i of the tile: node (tile TQ + i) / G, query head (head G + the rest)
    __device__ __forceinline__ const Query *query(const TreeAttention &P, int i) const
    {
        const int G = P.group, qr = min(it.tile * TQ + i, n_rows - 1), node = qr / G;
        const Query *q;
        if constexpr (STACK) q = P.q32;
        else q = P.q;
        return q + (size_t)(it.first + node) * P.q_stride + (size_t)(head * G + (qr - node * G)) * D;
    }
};

// Q^T of a query row: dimensions 32 s + 8 kg .. + 7; a stack's queries, in 32 bits, are head and remainder (half_split.h)
template <int D, bool STACK>
struct TaQuery {
    static constexpr int KS = (D + 31) / 32;
    ta_f16x8 hi[KS], lo[STACK ? KS : 1];
    template <class T>
    __device__ __forceinline__ void load(const T *q, int kg)
    {
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const bool real = D % 32 == 0 || 32 * s + 8 * kg < D;
            const T *at = q + (real ? 32 * s + 8 * kg : 0);
            if constexpr (STACK) {
                const f32x4 a = *as_global(reinterpret_cast<const f32x4 *>(at)), b = *as_global(reinterpret_cast<const f32x4 *>(at + 4));
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float v = split_value(real ? (e < 4 ? a[e & 3] : b[e & 3]) : 0.f);
                    hi[s][e] = (_Float16)v;
                    lo[s][e] = (_Float16)(v - (float)hi[s][e]);
                }
            } else {
                u32x4 x = load16(at);
                if (!real) x = u32x4{0u, 0u, 0u, 0u};
                hi[s] = __builtin_bit_cast(ta_f16x8, x);
            }
        }
    }
    __device__ __forceinline__ f32x4 score(u32x4 k, int s, f32x4 S) const
    {
        S = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(ta_f16x8, k), hi[s], S, 0, 0, 0);
        if constexpr (STACK) S = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(ta_f16x8, k), lo[s], S, 0, 0, 0);
        return S;
    }
};

// A query tile's 16 rows and 32 positions, scores of this lane: row lane % 16, positions 4 (lane / 16) .. + 3 of both granules.
// What a row does not see is minus infinity.  window: which positions the row sees
__device__ __forceinline__ void ta_mask(f32x4 (&S)[2], unsigned window, int kg)
{
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) S[t][e] = (window >> (16 * t + 4 * kg + e)) & 1 ? S[t][e] : -INFINITY;
}
// The sums so far to a new reference, where a score is 2^kTaSlack above the one that the weights are relative to; the reference is the same in the four
// lanes of a row.  L: sums of the weights, in every element.
template <int NT>
__device__ __forceinline__ void ta_rise(const f32x4 (&S)[2], float scale, float &m_run, f32x4 &L, f32x4 (&O)[NT])
{
    float most = fmaxf(S[0][0], S[0][1]);
    most = fmaxf(fmaxf(most, S[0][2]), S[0][3]);
    most = fmaxf(fmaxf(most, S[1][0]), S[1][1]);
    most = fmaxf(fmaxf(most, S[1][2]), S[1][3]) * scale;
    if (__any(most > m_run + kTaSlack)) {
        const float mn = fmaxf(m_run, ta_max4(most)), corr = __builtin_amdgcn_exp2f(m_run - mn);
        m_run = mn;
        L *= corr;
#pragma unroll
        for (int t = 0; t < NT; ++t) O[t] *= corr;
    }
}
// Weights, 2^kTaUp times their size.  One's head is cut off, not rounded, and its remainder, which is exact, is cut off in turn: together 2^-21 of it.
__device__ __forceinline__ void ta_weights(const f32x4 (&S)[2], float scale, float m_run, ta_f16x8 &ph, ta_f16x8 &pl)
{
    const float base = kTaUp - m_run;
    float minus = -1.f;                                    // (as a number that the compiler does not know: one instruction from a half to a remainder)
    asm("" : "+v"(minus));
    u32x4 hi, lo;
#pragma unroll
    for (int e = 0; e < 4; ++e) {                          // words: positions 4 kg + 0, 1; + 2, 3; the same of the second granule
        const int t = e >> 1, i = 2 * (e & 1);
        const float p0 = split_value(__builtin_amdgcn_exp2f(fmaf(S[t][i], scale, base))), p1 = split_value(__builtin_amdgcn_exp2f(fmaf(S[t][i + 1], scale, base)));
        const auto h = __builtin_amdgcn_cvt_pkrtz(p0, p1);
        const auto l = __builtin_amdgcn_cvt_pkrtz(fmaf((float)h[0], minus, p0), fmaf((float)h[1], minus, p1));
        hi[e] = __builtin_bit_cast(unsigned, h);
        lo[e] = __builtin_bit_cast(unsigned, l);
    }
    ph = __builtin_bit_cast(ta_f16x8, hi);
    pl = __builtin_bit_cast(ta_f16x8, lo);
}
// a row's weights, added up by the matrix instruction too: every element of the sum is the total over the 32 positions
__device__ __forceinline__ f32x4 ta_total(ta_f16x8 ph, ta_f16x8 pl, f32x4 L)
{
    const _Float16 one = (_Float16)1.f;
    const ta_f16x8 ones = {one, one, one, one, one, one, one, one};
    L = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, ph, L, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, pl, L, 0, 0, 0);
}

// ---- up to 32 query rows of a tile: the wavefronts share the positions --------------------------------------------
template <int D, int QT>
constexpr int ta_lds()                                     // V, or the wavefronts' sums
{
    const int v = kTaWaves * 2 * ta_granule(D), w = kTaWaves * 16 * QT * (D + 2) * 4;
    return v > w ? v : w;
}

template <int D, int TQ, int QT, bool STACK>
__device__ __forceinline__ void ta_narrow(const TreeAttention &P, const TreePlanLayout &L, char *plan, const TaStart<D, TQ, STACK> &w, char *mem,
                                          unsigned (*smask)[kTreeMaxNodes / 32])
{
    constexpr int KS = TaRow<D>::KS, NT = D / 16, TR = 16 * QT, W = kTaWaves, D4 = D / 4;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, kg = lane >> 4;
    const TreeItem &it = w.it;
    const int words = tree_words(P.b.max_nodes);
    // rows on their way in registers: as many as fit beside the sums (two of head_dim 128 with 32 query rows go to memory).  Bypassing the caches pays: no
    // row is read again but by the tiles of its own request (loads kept there: the 64 requests 86 of 77 us, one token of 8 behind 8000 117 of 107).
    constexpr int AHEAD = QT == 1 || D <= 80 ? 2 : 1;
    TaRow<D> r[AHEAD];
    const int row0 = it.t0 / kTaRow + wave;
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
        const TaPick at[2] = {w.pages.pick(2 * (row0 + a * W)), w.pages.pick(2 * (row0 + a * W) + 1)};
        r[a].request(w.K, w.V, w.pages, w.slab, at, lane);
    }
    TaPick next[2] = {w.pages.pick(2 * (row0 + AHEAD * W)), w.pages.pick(2 * (row0 + AHEAD * W) + 1)};
    const unsigned entries = w.pages.largest(it.t0 >> 4, lane);
    const bool tail = it.t1 > it.len;
    if (tail) w.masks(P, smask);
    TaQuery<D, STACK> Q[QT];
#pragma unroll
    for (int j = 0; j < QT; ++j) Q[j].load(w.query(P, 16 * j + col), kg);
    if (tail) __syncthreads();                             // (uniform)
    const float scale = 1.44269504088896340736f / sqrtf((float)D);
    f32x4 O[QT][NT];
    f32x4 sum[QT];
    float m_run[QT];
#pragma unroll
    for (int j = 0; j < QT; ++j) {
        m_run[j] = kTaLowest;
        sum[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < NT; ++t) O[j][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    char *vt = mem + wave * 2 * ta_granule(D);
    auto step = [&](TaRow<D> &r, int row) {
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
                for (int j = 0; j < QT; ++j) S[j][t] = Q[j].score(k, s, S[j][t]);
            }
        }
        r.request(w.K, w.V, w.pages, w.slab, next, lane);
        next[0] = w.pages.pick(2 * (row + (AHEAD + 1) * W));
        next[1] = w.pages.pick(2 * (row + (AHEAD + 1) * W) + 1);
        const bool masked = row * kTaRow + kTaRow > it.len;                // (uniform)
        ta_f16x8 ph[QT], pl[QT];                           // element 4 t + e: position 16 t + 4 kg + e
#pragma unroll
        for (int j = 0; j < QT; ++j) {
            if (masked) ta_mask(S[j], ta_window(smask[16 * j + col], words, row * kTaRow, it.len, it.nodes), kg);
            ta_rise(S[j], scale, m_run[j], sum[j], O[j]);
            ta_weights(S[j], scale, m_run[j], ph[j], pl[j]);
            sum[j] = ta_total(ph[j], pl[j], sum[j]);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const ta_u32x2 v0 = ta_transposed(vt + t * 512, lane), v1 = ta_transposed(vt + ta_granule(D) + t * 512, lane);
            const ta_f16x8 v = __builtin_bit_cast(ta_f16x8, u32x4{v0[0], v0[1], v1[0], v1[1]});
#pragma unroll
            for (int j = 0; j < QT; ++j) {
                O[j][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, ph[j], O[j][t], 0, 0, 0);
                O[j][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pl[j], O[j][t], 0, 0, 0);
            }
        }
        asm volatile("" ::: "memory");
    };
    for (int row = row0; row * kTaRow < it.t1; row += AHEAD * W)
#pragma unroll
        for (int a = 0; a < AHEAD; ++a)
            if ((row + a * W) * kTaRow < it.t1) step(r[a], row + a * W);               // (uniform)
    // The wavefronts' sums: [wave][row][D], maxima and weights [wave][row], in the place of V
    float *wp = reinterpret_cast<float *>(mem), *wm = wp + W * TR * D, *wl = wm + W * TR;
    const bool bad = __any(entries >= (unsigned)w.pages.n_pages);
    __syncthreads();                                       // V has been read
#pragma unroll
    for (int j = 0; j < QT; ++j) {
        const int at = wave * TR + 16 * j;
        const float l = sum[j][0];
        // A sum of weights that is no number is the answer: a score that the row sees is none, or plus infinity.  (But queries in 32 bits meet an infinite
        // key in two parts, of which one may be zero.)
        const bool none = !STACK && l != l;
        bool finite = (STACK ? fabsf(l) < INFINITY : true) && !bad;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int e = 0; e < 4; ++e) finite = finite && (none || fabsf(O[j][t][e]) < INFINITY);
            *reinterpret_cast<f32x4 *>(wp + (at + col) * D + 16 * t + 4 * kg) = O[j][t];
        }
        if (kg == 0) { wm[at + col] = m_run[j]; wl[at + col] = l; }
        const unsigned long long again = __ballot(!finite);            // (bit i: query row i % 16)
        if (again) {                                       // (uniform)
            asm volatile("" ::: "memory");
            for (int i = 0; i < 16; ++i)
                if (again & (0x0001000100010001ull << i))
                    ta_alone<D, W>(P, it, w.pages, w.K, w.V, smask[16 * j + i], w.query(P, 16 * j + i), row0, lane, wp + (at + i) * D, wm + at + i, wl + at + i);
        }
    }
    __syncthreads();
    const TaSlot<D> slot(L, plan, it, P.pg.heads, w.head, it.piece);
    for (int e = tid; e < w.rows * D4; e += kTaThreads) {
        const int i = e / D4, dim = 4 * (e - i * D4);
        float M = wm[i], l = 0.f;
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 1; v < W; ++v) M = fmaxf(M, wm[v * TR + i]);
#pragma unroll
        for (int v = 0; v < W; ++v) {
            const float ew = __builtin_amdgcn_exp2f(wm[v * TR + i] - M);
            l += wl[v * TR + i] * ew;
            s += *reinterpret_cast<const f32x4 *>(wp + (v * TR + i) * D + dim) * ew;
        }
        if (it.pieces == 1) {
            ta_deliver<D, STACK>(P, it, w.head, it.tile * TQ + i, dim, s, l);
        } else {
            slot.put(i, dim, s);
            if (dim == 0) slot.put_ml(i, M, l);
        }
    }
}

// ---- more query rows: the wavefronts share the rows -------------------------------------------------------
// A row of 32 positions goes through LDS for all four wavefronts, K and V as they lie in the pool, straight from memory: a ring of kTwRing
// rows, one granule of K or V of each to a wavefront, waited for by count, and one barrier a row.  A wavefront has 16 QT query rows and all positions
// of the piece, so nothing is joined but the pieces.  Positions past the piece's end read its last one again: their weights are zero.
// A workgroup's rows come through LDS, not registers, because four wavefronts read each of them: 607 -> 576 us (8 requests of 256 nodes; builds of then).  A K value is
// then used by 32 query rows and a V value by as many, so the LDS reads stay below the matrix instructions' time; scores a row ahead took 495 to 475,
// sums side by side 444 to 420.  (With every load of one row that the L2 holds: 446 to 404, so waiting for memory is a tenth at most.)
constexpr int kTwRing = 4;
template <int D>
struct TwLds {
    // (an odd slab's second half is left free, so that a load's 64 lanes always fill two)
    static constexpr int slabs = D / 16, loads = (slabs + 1) / 2, granule = loads * 1024, row = 4 * granule, bytes = kTwRing * row;
};
template <int N>
__device__ __forceinline__ void tw_arrive()                // all but the N newest loads of this wavefront have landed, and every wavefront is here
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(N) : "memory");
}

template <int D, int TQ, int QT, bool STACK>
__device__ __forceinline__ void ta_wide(const TreeAttention &P, const TreePlanLayout &L, char *plan, const TaStart<D, TQ, STACK> &w, char *mem,
                                        unsigned (*smask)[kTreeMaxNodes / 32])
{
    using Lds = TwLds<D>;
    constexpr int KS = TaRow<D>::KS, NT = D / 16, RW = 16 * QT;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, kg = lane >> 4;
    const TreeItem &it = w.it;
    const int words = tree_words(P.b.max_nodes);
    // this wavefront's granule of a row: K (0, 1) or V (2, 3)
    const __half *half = wave < 2 ? w.K : w.V;
    const int mine = wave & 1, last_n = (it.t1 - 1) & 15;
    const unsigned base = lds_address(mem);
    auto request = [&](int row, int at, const TaPick &pick) {
        const int n = min((lane & 31) >> 1, 2 * row + mine < w.pages.last ? 15 : last_n);
        const i32x4 rsrc = dma_rsrc(half + w.pages.place(pick), 0x7fffffffu);
        const unsigned to = base + at * Lds::row + wave * Lds::granule;
#pragma unroll
        for (int u = 0; u < Lds::loads; ++u) {
            const unsigned off = ((lane >> 5) * w.slab + n * 16u + (lane & 1) * 8u) * 2u;
            if (Lds::slabs % 2 == 0 || u < Lds::loads - 1 || lane < 32) lds_dma16(rsrc, to + u * 1024, off, 2 * u * w.slab * 2u);
        }
    };
    const int first = it.t0 / kTaRow;
    const bool bad = __any(w.pages.largest(it.t0 >> 4, lane) >= (unsigned)w.pages.n_pages);
#pragma unroll
    for (int a = 0; a < kTwRing - 1; ++a) request(first + a, a, w.pages.pick(2 * (first + a) + mine));
    TaPick next = w.pages.pick(2 * (first + kTwRing - 1) + mine);
    if (it.t1 > it.len) w.masks(P, smask);
    TaQuery<D, STACK> Q[QT];
#pragma unroll
    for (int j = 0; j < QT; ++j) Q[j].load(w.query(P, wave * RW + 16 * j + col), kg);
    const float scale = 1.44269504088896340736f / sqrtf((float)D);
    f32x4 O[QT][NT];
    f32x4 sum[QT];
    float m_run[QT];
#pragma unroll
    for (int j = 0; j < QT; ++j) {
        m_run[j] = kTaLowest;
        sum[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < NT; ++t) O[j][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // Scores are a row ahead of the weights: the matrix instructions of one run beside the vector instructions of the other.
    f32x4 S[QT][2];
    u32x4 k[2][KS];
    auto keys = [&](int at) {
        const char *kb = mem + at * Lds::row;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const bool real = D % 32 == 0 || 32 * s + 8 * kg < D;
                k[t][s] = *reinterpret_cast<const u32x4 *>(kb + t * Lds::granule + (real ? 2 * s + (kg >> 1) : 0) * 512 + col * 32 + (kg & 1) * 16);
            }
    };
    auto scores = [&](f32x4 (&S)[QT][2]) {                 // (the sums side by side: a matrix instruction does not wait for the one before)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int j = 0; j < QT; ++j) S[j][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const bool real = D % 32 == 0 || 32 * s + 8 * kg < D;
                const u32x4 x = real ? k[t][s] : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
                for (int j = 0; j < QT; ++j) S[j][t] = Q[j].score(x, s, S[j][t]);
            }
    };
    int at = 0;
    tw_arrive<(kTwRing - 2) * Lds::loads>();
    // A wavefront without a query row of its own only loads and waits with the others (64 requests of 36 query rows: 91.6 -> 88.8 us).
    if (wave * RW >= w.rows) {
        for (int row = first; row * kTaRow < it.t1; ++row) {
            tw_arrive<(kTwRing - 3) * Lds::loads>();
            request(row + kTwRing - 1, (at + kTwRing - 1) % kTwRing, next);
            next = w.pages.pick(2 * (row + kTwRing) + mine);
            at = (at + 1) % kTwRing;
        }
        tw_arrive<0>();
        return;
    }
    keys(0);
    scores(S);
    for (int row = first; row * kTaRow < it.t1; ++row) {
        const int ahead = (at + 1) % kTwRing;
        tw_arrive<(kTwRing - 3) * Lds::loads>();           // (the next row is here)
        keys(ahead);
        request(row + kTwRing - 1, (at + kTwRing - 1) % kTwRing, next);    // (the place of the row before this one, which everyone has read)
        next = w.pages.pick(2 * (row + kTwRing) + mine);
        const char *vb = mem + at * Lds::row + 2 * Lds::granule;
        const bool masked = row * kTaRow + kTaRow > it.len;                // (uniform)
#pragma unroll
        for (int j = 0; j < QT; ++j) {
            if (masked) ta_mask(S[j], ta_window(smask[wave * RW + 16 * j + col], words, row * kTaRow, it.len, it.nodes), kg);
            ta_rise(S[j], scale, m_run[j], sum[j], O[j]);
        }
        f32x4 ahead_S[QT][2];
        scores(ahead_S);
        ta_f16x8 ph[QT], pl[QT];
#pragma unroll
        for (int j = 0; j < QT; ++j) {
            ta_weights(S[j], scale, m_run[j], ph[j], pl[j]);
            sum[j] = ta_total(ph[j], pl[j], sum[j]);
        }
#pragma unroll
        for (int t = 0; t < NT; t += 2) {                  // (NT is 4, 5 or 8)
            ta_f16x8 v[2];
#pragma unroll
            for (int u = 0; u < 2 && t + u < NT; ++u) {
                const ta_u32x2 v0 = ta_transposed(vb + (t + u) * 512, lane), v1 = ta_transposed(vb + Lds::granule + (t + u) * 512, lane);
                v[u] = __builtin_bit_cast(ta_f16x8, u32x4{v0[0], v0[1], v1[0], v1[1]});
            }
#pragma unroll
            for (int part = 0; part < 2; ++part)
#pragma unroll
                for (int u = 0; u < 2 && t + u < NT; ++u)
#pragma unroll
                    for (int j = 0; j < QT; ++j) O[j][t + u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v[u], part ? pl[j] : ph[j], O[j][t + u], 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < QT; ++j)
#pragma unroll
            for (int t = 0; t < 2; ++t) S[j][t] = ahead_S[j][t];
        at = ahead;
    }
    tw_arrive<0>();                                        // nothing is on its way to LDS any more
    const TaSlot<D> slot(L, plan, it, P.pg.heads, w.head, it.piece);
#pragma unroll
    for (int j = 0; j < QT; ++j) {
        const int i = wave * RW + 16 * j + col;
        float l = sum[j][0];
        // A sum of weights that is no number is the answer: a score that the row sees is none, or plus infinity.  (But queries in 32 bits meet an infinite
        // key in two parts, of which one may be zero.)
        const bool none = !STACK && l != l;
        bool finite = (STACK ? fabsf(l) < INFINITY : true) && !bad;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) finite = finite && (none || fabsf(O[j][t][e]) < INFINITY);
        const unsigned long long again = __ballot(!finite);
        if (again) {                                       // (uniform) rows worked out once more, through LDS that no one needs now
            float *o = reinterpret_cast<float *>(mem) + wave * 16 * (D + 2);
            for (int q = 0; q < 16; ++q)
                if (again & (0x0001000100010001ull << q))
                    ta_alone<D, 1>(P, it, w.pages, w.K, w.V, smask[wave * RW + 16 * j + q], w.query(P, wave * RW + 16 * j + q), it.t0 / kTaRow, lane, o + q * (D + 2),
                                   o + q * (D + 2) + D, o + q * (D + 2) + D + 1);
            asm volatile("" ::: "memory");
            if (again & (0x0001000100010001ull << col)) {
                const float *mine = o + col * (D + 2);
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) O[j][t][e] = mine[16 * t + 4 * kg + e];
                m_run[j] = mine[D];
                l = mine[D + 1];
            }
        }
        if (i >= w.rows) continue;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if (it.pieces == 1) ta_deliver<D, STACK>(P, it, w.head, it.tile * TQ + i, 16 * t + 4 * kg, O[j][t], l);
            else slot.put(i, 16 * t + 4 * kg, O[j][t]);
        }
        if (it.pieces > 1 && kg == 0) slot.put_ml(i, m_run[j], l);
    }
}

// A tile runs by the query rows that it has: requests of one step may differ in size.
template <int D, int TQ>
constexpr int ta_lds_of()
{
    return TQ <= 32 ? ta_lds<D, TQ / 16>() : TwLds<D>::bytes > ta_lds<D, 2>() ? TwLds<D>::bytes : ta_lds<D, 2>();
}
// STACK: the rows of a stack's step, queries in 32 bits and outputs as its products take them
template <int D, int TQ, bool STACK>
__global__ void __launch_bounds__(kTaThreads, 2) k_tree_attention(TreeAttention P, TreePlanLayout L, char *plan)
{
    extern __shared__ __align__(16) char ta_mem[];
    __shared__ unsigned smask[TQ][kTreeMaxNodes / 32];
    __shared__ int last_one;
    TaStart<D, TQ, STACK> w;
    if (!w.of(P, L, plan)) return;
    if (TQ == 16 || w.rows <= 16) {
        ta_narrow<D, TQ, 1, STACK>(P, L, plan, w, ta_mem, smask);
    } else if (TQ == 32 || w.rows <= 32) {
        if constexpr (TQ >= 32) ta_narrow<D, TQ, 2, STACK>(P, L, plan, w, ta_mem, smask);
    } else if (TQ == 64 || w.rows <= 64) {
        if constexpr (TQ >= 64) ta_wide<D, TQ, 1, STACK>(P, L, plan, w, ta_mem, smask);
    } else {
        if constexpr (TQ >= 128) ta_wide<D, TQ, 2, STACK>(P, L, plan, w, ta_mem, smask);
    }
    if constexpr (TQ <= kTaLastJoins)
        if (w.it.pieces > 1) ta_join<D, STACK>(P, L, plan, w.it, P.pg.heads, w.head, w.rows, &last_one);
}

// The pieces of many query rows are added by a launch of its own, 1024 sums to a workgroup at a time: for one workgroup they are up to 16384.
constexpr int kTaJoinWgs = 1024;                          // (256 / 512 / 1024: 4 requests of 60 nodes 50 / 47 / 46 us, 64 of 9 81 / 79 / 78)
template <int D, int TQ, bool STACK>
__global__ void __launch_bounds__(kTaThreads) k_tree_join(TreeAttention P, TreePlanLayout L, const char *plan)
{
    constexpr int D4 = D / 4, CHUNKS = (TQ * D4 + kTaThreads - 1) / kTaThreads;
    const int H = P.pg.heads;
    const TreePlanHead &plan_head = *reinterpret_cast<const TreePlanHead *>(plan);
    if (plan_head.key != L.key) return;
    const size_t step = (size_t)H * TQ * (D + 2);          // from piece to piece
    for (int unit = blockIdx.x; unit < plan_head.cuts * H * CHUNKS; unit += gridDim.x) {
        const int b = unit / CHUNKS, chunk = unit - b * CHUNKS, k = b / H, head = b - k * H;
        const TreeItem it = reinterpret_cast<const TreeItem *>(plan + L.items)[reinterpret_cast<const int *>(plan + L.cut)[k]];
        const int e = chunk * kTaThreads + (int)threadIdx.x, i = e / D4, dim = 4 * (e - i * D4);
        if (i >= min(TQ, it.nodes * P.group - it.tile * TQ)) continue;
        const float *at = reinterpret_cast<const float *>(plan + L.sums) + ((size_t)it.slot * H + head) * (TQ * (D + 2));
        float M = kTaLowest, l = 0.f;
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
        constexpr int AT = 8;                              // in flight together (past the last: the last again)
        for (int z = 0; z < it.pieces; z += AT) {
            float2 ml[AT];
            f32x4 a[AT];
#pragma unroll
            for (int u = 0; u < AT; ++u) {
                const float *f = at + (size_t)min(z + u, it.pieces - 1) * step;
                ml[u] = *reinterpret_cast<const float2 *>(f + TQ * D + 2 * i);
                a[u] = *as_global(reinterpret_cast<const f32x4 *>(f + i * D + dim));
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
        ta_deliver<D, STACK>(P, it, head, it.tile * TQ + i, dim, s, l);
    }
}

template <int D, int TQ, bool STACK>
static hipError_t launch_tile(const TreeAttention &P, const TreePlanLayout &L, char *plan, hipStream_t s)
{
    constexpr int lds = ta_lds_of<D, TQ>();
    if constexpr (lds > 64 * 1024 - 8192) {                // (more than the default limit, with the masks)
        const hipError_t e = hipFuncSetAttribute((const void *)k_tree_attention<D, TQ, STACK>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((k_tree_attention<D, TQ, STACK>), dim3((unsigned)L.work * P.pg.heads), dim3(kTaThreads), lds, s, P, L, plan);
    if constexpr (TQ > kTaLastJoins) {
        hipLaunchKernelGGL((k_tree_join<D, TQ, STACK>), dim3(kTaJoinWgs), dim3(kTaThreads), 0, s, P, L, plan);
    }
    return hipGetLastError();
}
template <int D, bool STACK>
static hipError_t launch_of(const TreeAttention &P, const TreePlanLayout &L, char *plan, hipStream_t s)
{
    switch (L.tile_rows) {
    case 16: return launch_tile<D, 16, STACK>(P, L, plan, s);
    case 32: return launch_tile<D, 32, STACK>(P, L, plan, s);
    case 64: return launch_tile<D, 64, STACK>(P, L, plan, s);
    default: return launch_tile<D, 128, STACK>(P, L, plan, s);
    }
}

template <bool STACK>
static hipError_t launch_attention(const TreeAttention &A, char *plan, hipStream_t s)
{
    TreeAttention P = A;
    const TreePlanLayout L = tree_plan_layout(P.pg, P.n_heads, P.b.requests, P.b.max_rows, P.b.max_nodes, P.b.stride);
    const unsigned page16 = (unsigned)P.pg.page >> 4;
    P.page16_inv = (unsigned)(((1ull << 32) + page16 - 1) / page16);
    switch (P.pg.d) {
    case 64: return launch_of<64, STACK>(P, L, plan, s);
    case 80: return launch_of<80, STACK>(P, L, plan, s);
    default: return launch_of<128, STACK>(P, L, plan, s);
    }
}

hipError_t launch_tree_attention(const TreeAttention &P, char *plan, hipStream_t s) { return launch_attention<false>(P, plan, s); }

template <int D>
static hipError_t launch_join(const TreeAttention &P, const TreePlanLayout &L, const char *plan, hipStream_t s)
{
    if (L.tile_rows == 32) hipLaunchKernelGGL((k_tree_join<D, 32, false>), dim3(kTaJoinWgs), dim3(kTaThreads), 0, s, P, L, plan);
    else if (L.tile_rows == 64) hipLaunchKernelGGL((k_tree_join<D, 64, false>), dim3(kTaJoinWgs), dim3(kTaThreads), 0, s, P, L, plan);
    else if (L.tile_rows == 128) hipLaunchKernelGGL((k_tree_join<D, 128, false>), dim3(kTaJoinWgs), dim3(kTaThreads), 0, s, P, L, plan);
    return hipGetLastError();
}
hipError_t launch_tree_join(const TreeAttention &P, const TreePlanLayout &L, const char *plan, hipStream_t s)
{
    return P.pg.d == 64 ? launch_join<64>(P, L, plan, s) : P.pg.d == 80 ? launch_join<80>(P, L, plan, s) : launch_join<128>(P, L, plan, s);
}

// ---- a stack's rows ------------------------------------------------------------------------------------
// Its first product leaves K and V rows in slabs of its own scratch, [2][head][d / 16][row][16], and queries in 32 bits; the K and V rows go
// to their slots, then every node attends.
hipError_t launch_tree_rows(const PfParams &F, hipStream_t s)
{
    const TreePass &T = *F.tree;
    hipError_t e = launch_page_append_slabs(T.pg, T.pool, F.kv, F.dm.max_seq, T.b.slots, F.n_rows, s);
    if (e != hipSuccess) return e;
    TreeAttention P;
    P.pg = T.pg; P.b = T.b;
    P.n_heads = F.dm.H; P.group = 1;
    P.pool = T.pool;
    P.q = nullptr; P.out = nullptr;
    P.q32 = F.q; P.planes = F.o; P.narrow = F.nrw.on;
    P.q_stride = F.dm.h; P.out_stride = 0;
    return launch_attention<true>(P, T.plan, s);
}

}  // namespace cfpp
