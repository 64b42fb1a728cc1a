// Attention of drafted trees over a paged cache, the ancestor masks it reads and its launch plan.
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include "tree_params.h"
#include "device_utils.h"

namespace cfpp {

// ---- the plan --------------------------------------------------------------------------------------
TreePlanLayout tree_plan_layout(const PageDims &, int, int requests, int, int)
{
    TreePlanLayout L;
    L.total = align_up((size_t)requests * 4, 256);         // rows of each request that take part
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
__global__ void __launch_bounds__(kTreeMaxNodes) k_tree_plan(PageDims pg, TreeBatch b, int *rows)
{
    constexpr int W = kTreeMaxNodes / 32;
    __shared__ unsigned m[kTreeMaxNodes][W + 1];
    __shared__ int up[kTreeMaxNodes];
    const int r = blockIdx.x, i = threadIdx.x, words = tree_words(b.max_nodes);
    int first;
    const int n = tree_rows(pg, b, r, first);
    if (i == 0) rows[r] = n;
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

hipError_t launch_tree_plan(const PageDims &pg, const TreeBatch &b, int, char *plan, hipStream_t s)
{
    hipLaunchKernelGGL(k_tree_plan, dim3(b.requests), dim3(kTreeMaxNodes), 0, s, pg, b, reinterpret_cast<int *>(plan));
    return hipGetLastError();
}

// ---- the attention -----------------------------------------------------------------------------------
// One wavefront to a row and head: 64 positions at a time, one to a lane for the scores, then the lanes have the dimensions.
__global__ void __launch_bounds__(64) k_tree_attention(TreeAttention P, const int *rows)
{
    __shared__ float q[128], weight[64];
    __shared__ long long base[64];
    const int lane = threadIdx.x, D = P.pg.d, head = blockIdx.y, kvh = head / P.group, words = tree_words(P.b.max_nodes);
    const int row = blockIdx.x;
    // the request: the first one whose rows end behind this row
    int lo = 0, hi = P.b.requests;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (P.b.row_start[mid + 1] > row) hi = mid;
        else lo = mid + 1;
    }
    const int r = lo;
    if (r >= P.b.requests || row < P.b.row_start[r] || rows[r] == 0) return;
    const int len = P.b.lens[r], n = rows[r], ends = len + n;
    const unsigned *mask = P.b.masks + (size_t)row * words;
    const size_t which = page_which_elems(P.pg);
    for (int i = lane; i < D; i += 64) q[i] = __half2float(P.q[(size_t)row * P.q_stride + head * D + i]) * (1.44269504088896340736f / sqrtf((float)D));
    __syncthreads();
    float m = -3.0e38f, l = 0.f, o[2] = {0.f, 0.f};
    bool any = len > 0;
    for (int t0 = 0; t0 < ends; t0 += 64) {
        const int t = t0 + lane;
        bool sees = t < len;
        if (t >= len && t < ends) sees = (mask[(t - len) >> 5] >> ((t - len) & 31)) & 1;
        any = any || __any(sees);
        float s = -INFINITY;
        long long at = -1;
        if (sees) {
            const int page = P.b.table[(size_t)r * P.b.stride + t / P.pg.page];
            if (page < 0 || page >= P.pg.n_pages) {
                s = NAN;
            } else {
                at = (long long)(((size_t)page * P.pg.heads + kvh) * page_head_elems(P.pg) + (size_t)(t % P.pg.page) * 16);
                s = 0.f;
                for (int pc = 0; pc < D / 8; ++pc) {
                    const u32x4 k = load16(P.pool + at + (size_t)(pc >> 1) * P.pg.page * 16 + (pc & 1) * 8);
                    s = dot8(k, *reinterpret_cast<const float4 *>(q + 8 * pc), *reinterpret_cast<const float4 *>(q + 8 * pc + 4), s);
                }
            }
        }
        const float mn = fmaxf(m, wave_max(s)), corr = __builtin_amdgcn_exp2f(m - mn), p = sees ? __builtin_amdgcn_exp2f(s - mn) : 0.f;
        m = mn;
        l = l * corr + wave_sum(p);
        weight[lane] = p;
        base[lane] = at;
        __syncthreads();
        o[0] *= corr; o[1] *= corr;
        for (int j = 0; j < 64; ++j) {
            if (base[j] < 0) {
                if (weight[j] != weight[j]) o[0] = o[1] = NAN;
                continue;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int dim = lane + 64 * e;
                if (dim < D) o[e] = fmaf(weight[j], __half2float(P.pool[which + base[j] + (size_t)(dim >> 4) * P.pg.page * 16 + (dim & 15)]), o[e]);
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int dim = lane + 64 * e;
        if (dim < D) P.out[(size_t)row * P.out_stride + head * D + dim] = __float2half_rn(any ? o[e] / l : 0.f);
    }
}

hipError_t launch_tree_attention(const TreeAttention &P, char *plan, hipStream_t s)
{
    hipLaunchKernelGGL(k_tree_attention, dim3(P.b.max_rows, P.n_heads), dim3(64), 0, s, P, reinterpret_cast<const int *>(plan));
    return hipGetLastError();
}

}  // namespace cfpp
