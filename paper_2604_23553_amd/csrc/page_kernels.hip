// Pages of a cache that requests share, and the trees of drafted tokens on it: block tables and slots, ancestor masks, the append
// of new rows, the accepted path.  Whole numbers and copies; the attention is tree_attention.hip.
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include "tree_params.h"
#include "device_utils.h"

namespace cfpp {

// ---- block tables and slots --------------------------------------------------------------------
// target_r = ceil((len_r + count_r) / page); a request takes target - held pages from the end of the free list or gives back
// held - target.  Three running sums over the requests (pages taken, pages given back, rows) say which entry of the free list and
// which rows are whose.  One workgroup has all requests: every sum needs all of the ones before it, and 4096 requests are four to a thread.
// A chain of dependent reads, not bytes, bounds it: lengths, sums, and for the pages that move a search of their request, the list, the table.  One request
// 3.7 us, 4.0 where it takes a page; 4096 requests 9.8 us where no page moves, 18.1 where 8428 are taken, 20.4 where they are given back (160 KB of lists
// and tables); the launch of their slots 4.1, and 15.3 where all of 131 thousand rows are nobody's, which one workgroup writes.
constexpr int kTablesEach = 4;           // requests of a thread
// Rows whose slots it writes itself, in a launch less (a launch is about 4 us): 4096 are four to a thread of 1024 or sixteen to one of 256
constexpr int kTablesRows = 4096;
constexpr int kSumMost = 1 << 28;      // sums stop here: more than any pool's pages or batch's rows, and two of them still fit 32 bits

__device__ __forceinline__ int add_most(int a, int b) { return min(a + b, kSumMost); }

// Running sums of three values a thread over the workgroup; v: this thread's, on return the sums of the threads before it.
template <int WAVES>
__device__ __forceinline__ void block_sums(int (&v)[3], int (*part)[WAVES], int tid)
{
    const int lane = tid & 63, wave = tid >> 6;
    int own[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        int s = v[k];
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const int t = __shfl_up(s, m, 64);
            if (lane >= m) s = add_most(s, t);
        }
        own[k] = s;
        if (lane == 63) part[k][wave] = s;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        int before = 0;
        for (int w = 0; w < wave; ++w) before = add_most(before, part[k][w]);
        const int left = __shfl_up(own[k], 1, 64);
        v[k] = lane ? add_most(before, left) : before;
    }
}

// the first index in [0, n) whose running sum is above v (sum[n - 1] > v)
__device__ __forceinline__ int find_above(const int *sum, int n, int v)
{
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (sum[mid] > v) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// -1 where the block table's entry lies outside the pool (its product with the page's length could come back to a slot of another page)
__device__ __forceinline__ int slot_of(const TablesParams &P, int r, int at)
{
    const int page = P.b.table[(size_t)r * P.b.stride + at / P.pg.page];
    return (unsigned)page < (unsigned)P.pg.n_pages ? page * P.pg.page + at % P.pg.page : -1;
}

template <int THREADS, bool SLOTS>
__global__ void __launch_bounds__(THREADS) k_page_tables(TablesParams P)
{
    constexpr int MOST = THREADS * kTablesEach;
    __shared__ int taken[MOST], given[MOST], rows[MOST], part[3][THREADS / 64];
    const int R = P.b.requests, tid = threadIdx.x;
    const int F = max(0, min(*P.free_count, P.pg.n_pages));
    int target[kTablesEach], held[kTablesEach], sum[3] = {0, 0, 0};
    bool fits[kTablesEach];
    // this thread's requests, their own sums first
    int need[kTablesEach], surplus[kTablesEach], count[kTablesEach];
#pragma unroll
    for (int k = 0; k < kTablesEach; ++k) {
        const int r = tid * kTablesEach + k;
        need[k] = surplus[k] = count[k] = target[k] = held[k] = 0;
        fits[k] = false;
        if (r < R) {
            const int len = P.b.lens[r], n = P.counts[r];
            held[k] = max(0, min(P.held[r], P.b.stride));
            count[k] = max(0, min(n, kTreeMaxRows));
            const long long pages = ((long long)len + n + P.pg.page - 1) / P.pg.page;
            fits[k] = len >= 0 && n >= 0 && n <= P.b.max_rows && pages <= P.b.stride;
            target[k] = fits[k] ? (int)pages : held[k];
        }
        sum[2] = add_most(sum[2], count[k]);
    }
    block_sums<THREADS / 64>(sum, part, tid);
    int row = sum[2];
    sum[0] = sum[1] = sum[2] = 0;
#pragma unroll
    for (int k = 0; k < kTablesEach; ++k) {
        row = add_most(row, count[k]);
        fits[k] = fits[k] && row <= P.b.max_rows;
        if (!fits[k]) target[k] = held[k];
        need[k] = min(max(target[k] - held[k], 0), kSumMost);
        surplus[k] = max(held[k] - target[k], 0);
        const int r = tid * kTablesEach + k;
        if (r < R) rows[r] = min(row, P.b.max_rows);
        sum[0] = add_most(sum[0], need[k]);
        sum[1] = add_most(sum[1], surplus[k]);
    }
    __syncthreads();                                       // part has been read
    block_sums<THREADS / 64>(sum, part, tid);
    int before = sum[0], back = sum[1];
#pragma unroll
    for (int k = 0; k < kTablesEach; ++k) {
        const int r = tid * kTablesEach + k;
        before = add_most(before, need[k]);
        back = add_most(back, surplus[k]);
        if (r >= R) continue;
        const bool granted = fits[k] && (need[k] == 0 || before <= F);
        // (the ones that are granted pages are the first that need any: their sums are whole)
        taken[r] = min(before, kSumMost) <= F ? before : -1;
        given[r] = back;
        P.granted[r] = granted;
        P.b.row_start[r + 1] = rows[r];
        if (!granted && fits[k]) target[k] = held[k];
        fits[k] = granted;
    }
    if (tid == 0) P.b.row_start[0] = 0;
    __syncthreads();
    // taken[]: where a request's sum passes the free pages nothing more is taken
    int T = 0;
    {
        int lo = 0, hi = R;                                // first request whose sum passes F
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (taken[mid] < 0) hi = mid;
            else lo = mid + 1;
        }
        T = lo > 0 ? taken[lo - 1] : 0;
        for (int i = tid; i < T; i += THREADS) {
            const int r = find_above(taken, lo, i), k = i - (r > 0 ? taken[r - 1] : 0);
            P.b.table[(size_t)r * P.b.stride + max(0, min(P.held[r], P.b.stride)) + k] = P.free_pages[F - 1 - i];
        }
    }
    __syncthreads();                                       // every taken entry of the list has been read
    const int G = R > 0 ? given[R - 1] : 0;
    for (int i = tid; i < G; i += THREADS) {
        const int r = find_above(given, R, i), first = r > 0 ? given[r - 1] : 0, n = given[r] - first;
        int *entry = P.b.table + (size_t)r * P.b.stride + max(0, min(P.held[r], P.b.stride)) - n + (i - first);
        if (F - T + i < P.pg.n_pages) P.free_pages[F - T + i] = *entry;
        *entry = -1;
    }
    __syncthreads();                                       // held has been read, the block tables are written
    if constexpr (SLOTS) {
        for (int i = tid; i < P.b.max_rows; i += THREADS) {
            int slot = -1;
            if (i < rows[R - 1]) {
                const int r = find_above(rows, R, i);
                // (a request is granted what it asks for or nothing)
                if (P.granted[r]) slot = slot_of(P, r, P.b.lens[r] + i - (r > 0 ? rows[r - 1] : 0));
            }
            P.b.slots[i] = slot;
        }
    }
#pragma unroll
    for (int k = 0; k < kTablesEach; ++k) {
        const int r = tid * kTablesEach + k;
        if (r < R && fits[k]) P.held[r] = target[k];
    }
    if (tid == 0) *P.free_count = min(F - T + G, P.pg.n_pages);
}

// slots: a workgroup for each request, and one for the rows behind the last one
__global__ void __launch_bounds__(256) k_page_slots(TablesParams P)
{
    const int r = blockIdx.x, R = P.b.requests;
    if (r == R) {
        for (int i = P.b.row_start[R] + (int)threadIdx.x; i < P.b.max_rows; i += 256) P.b.slots[i] = -1;
        return;
    }
    const int first = P.b.row_start[r], n = P.b.row_start[r + 1] - first, len = P.b.lens[r];
    const bool granted = P.granted[r] != 0;
    for (int i = threadIdx.x; i < n; i += 256) P.b.slots[first + i] = granted ? slot_of(P, r, len + i) : -1;
}

hipError_t launch_page_tables(const TablesParams &P, hipStream_t s)
{
    const bool few = P.b.requests <= 256 * kTablesEach;
    if (P.b.max_rows <= kTablesRows) {
        if (few) hipLaunchKernelGGL((k_page_tables<256, true>), dim3(1), dim3(256), 0, s, P);
        else hipLaunchKernelGGL((k_page_tables<1024, true>), dim3(1), dim3(1024), 0, s, P);
        return hipGetLastError();
    }
    if (few) hipLaunchKernelGGL((k_page_tables<256, false>), dim3(1), dim3(256), 0, s, P);
    else hipLaunchKernelGGL((k_page_tables<1024, false>), dim3(1), dim3(1024), 0, s, P);
    hipLaunchKernelGGL(k_page_slots, dim3(P.b.requests + 1), dim3(256), 0, s, P);
    return hipGetLastError();
}

// ---- append ------------------------------------------------------------------------------------
// A wavefront has 8 rows and 128 bytes of each, 16 to a lane: whole lines are read, and where the rows' slots follow one another 256 bytes in a
// run are written.  Bound by the bytes: 4096 rows of hidden 4096, 134 MB read and written, 27.4 us, 4.9 TB/s, where a large copy reaches 5.14.  `from`: where the
// pieces of K and V rows lie.
struct AppendFrom {
    const __half *k, *v;
    long long row, head;       // halves from row to row, from head to head
    int slab;                  // from 16 dimensions to the next
};
__global__ void __launch_bounds__(256) k_page_append(PageDims pg, __half *pool, AppendFrom from, const int *slots, int n_rows)
{
    const int d8 = pg.d / 8, per = pg.heads * d8, groups = (per + 7) / 8, lane = threadIdx.x & 63;
    const long long unit = blockIdx.x * 4LL + (threadIdx.x >> 6);
    const int set = (int)(unit / (2 * groups)), g = (int)(unit - (long long)set * (2 * groups)), w = g >= groups;
    const int row = set * 8 + (lane >> 3), piece = (g - w * groups) * 8 + (lane & 7);
    if (row >= n_rows || piece >= per) return;
    const int slot = slots[row];
    const int page = slot / pg.page, at = slot - page * pg.page, head = piece / d8, pc = piece - head * d8;
    const u32x4 x = load16((w ? from.v : from.k) + row * from.row + head * from.head + (long long)(pc >> 1) * from.slab + (pc & 1) * 8);
    if (slot < 0 || slot >= pg.n_pages * pg.page) return;
    __half *to = pool + w * page_which_elems(pg) + ((size_t)page * pg.heads + head) * page_head_elems(pg) + ((size_t)(pc >> 1) * pg.page + at) * 16 + (pc & 1) * 8;
    *as_global(reinterpret_cast<u32x4 *>(to)) = x;
}

static hipError_t append(const PageDims &pg, __half *pool, const AppendFrom &from, const int *slots, int n_rows, hipStream_t s)
{
    const long long units = (long long)((n_rows + 7) / 8) * 2 * ((pg.heads * (pg.d / 8) + 7) / 8);
    hipLaunchKernelGGL(k_page_append, dim3((unsigned)((units + 3) / 4)), dim3(256), 0, s, pg, pool, from, slots, n_rows);
    return hipGetLastError();
}
hipError_t launch_page_append(const PageDims &pg, __half *pool, const __half *k, const __half *v, long long row_stride, const int *slots,
                              int n_rows, hipStream_t s)
{
    return append(pg, pool, AppendFrom{k, v, row_stride, pg.d, 16}, slots, n_rows, s);
}
hipError_t launch_page_append_slabs(const PageDims &pg, __half *pool, const __half *kv, int rows, const int *slots, int n_rows, hipStream_t s)
{
    return append(pg, pool, AppendFrom{kv, kv + (size_t)pg.heads * pg.d * rows, 16, (long long)pg.d * rows, 16 * rows}, slots, n_rows, s);
}

// ---- either side of a stack's step ---------------------------------------------------------------
__global__ void __launch_bounds__(256) k_tree_rope(PageDims pg, TreeBatch b, TreeRows R)
{
    const int i = blockIdx.x * 256 + threadIdx.x, per = max(R.half, 1), row = i / per, j = i - row * per;
    if (row >= b.max_rows) return;
    int lo = 0, hi = b.requests - 1;                       // the last request that begins at this row or before it
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (b.row_start[mid] <= row) lo = mid;
        else hi = mid - 1;
    }
    int first;
    const int n = tree_rows(pg, b, lo, first);
    const TreePlanHead &plan = *reinterpret_cast<const TreePlanHead *>(R.plan);
    const bool served = plan.key == R.key && plan.items > 0 && row >= first && row < first + n;
    const int slot = served ? b.slots[row] : -1;
    if (j == 0) R.slots[row] = slot;
    int pos = slot >= 0 ? b.positions[row] : 0;
    if (pos < 0 || pos >= R.max_seq) {
        *R.err = kErrBadPos;
        pos = 0;
    }
    if (R.half > 0) R.rope_rows[i] = R.rope[(size_t)pos * R.half + j];     // (positions count where nothing is rotated too)
}
hipError_t launch_tree_rope(const PageDims &pg, const TreeBatch &b, const TreeRows &R, hipStream_t s)
{
    hipLaunchKernelGGL(k_tree_rope, dim3((unsigned)(((long long)b.max_rows * (R.half > 0 ? R.half : 1) + 255) / 256)), dim3(256), 0, s, pg, b, R);
    return hipGetLastError();
}

__global__ void __launch_bounds__(256) k_tree_out(const int *slots, const __half *from, __half *to, int h)
{
    const int row = blockIdx.x;
    if (slots[row] < 0) return;
    for (int i = threadIdx.x * 8; i < h; i += 256 * 8)
        *as_global(reinterpret_cast<u32x4 *>(to + (size_t)row * h + i)) = load16(from + (size_t)row * h + i);
}
hipError_t launch_tree_out(const int *slots, int n_rows, const __half *from, __half *to, int h, hipStream_t s)
{
    hipLaunchKernelGGL(k_tree_out, dim3(n_rows), dim3(256), 0, s, slots, from, to, h);
    return hipGetLastError();
}

// ---- the accepted path ---------------------------------------------------------------------------
// A workgroup has one request and one of the K and V arrays of the layers; each walks the tree by itself (a step: every thread
// looks whether its node is a child that agrees, the lowest one goes on).  Node path[j] >= j moves to index j: rows are moved in
// ascending order, a block of pieces at a time, read before written: 8 loads to a thread are in flight, and the walk is done again by each workgroup
// because a launch in between would cost more than its few steps in LDS.  48 requests of up to 63 nodes, 16 layers of hidden 4096, of which
// some 100 nodes move, take 35 - 40 us for 27 MB read and as many written: a row lies in runs of 32 bytes, and the lines of 128 that hold them are 99 MB
// (counted; 30 MB written), so that 3.3 - 3.7 TB/s flow.  26 nodes of one request are bound by the walk's steps (6.1 us).
__global__ void __launch_bounds__(256) k_tree_accept(AcceptParams P, int n_layers)
{
    __shared__ int parent[kTreeMaxNodes], token[kTreeMaxNodes], pick[kTreeMaxNodes], slot[kTreeMaxNodes], path[kTreeMaxNodes], child[2];
    const int r = blockIdx.x, array = blockIdx.y, tid = threadIdx.x;
    const int first = P.b.row_start[r], rows = P.b.row_start[r + 1] - first;
    bool serve = rows > 0 && rows <= P.b.max_nodes && first >= 0 && first + rows <= P.b.max_rows;
    const int n = serve ? rows : 0;
    serve = serve && P.b.slots[first] >= 0;
    if (tid < n) {
        parent[tid] = P.b.parents[first + tid];
        token[tid] = P.tokens[first + tid];
        pick[tid] = P.picks[first + tid];
        slot[tid] = P.b.slots[first + tid];
    }
    if (tid < 2) child[tid] = kTreeMaxNodes;
    __syncthreads();
    int count = 0, cur = 0;
    if (serve) {
        for (int step = 0;; ++step) {
            if (tid == 0) { path[step] = cur; child[(step + 1) & 1] = kTreeMaxNodes; }
            ++count;
            if (tid < n && tid > cur && parent[tid] == cur && token[tid] == pick[cur]) atomicMin(&child[step & 1], tid);
            __syncthreads();
            const int next = child[step & 1];
            if (next >= n) break;                          // (node numbers rise: at most n steps)
            cur = next;
            __syncthreads();
        }
    }
    __syncthreads();
    if (array == 0) {
        for (int j = tid; j < P.b.max_nodes; j += 256) P.path[(size_t)r * P.b.max_nodes + j] = j < count ? path[j] : -1;
        if (tid == 0) {
            P.accepted[r] = count;
            P.next[r] = count > 0 ? pick[cur] : -1;
            P.lens_out[r] = P.b.lens[r] + count;
        }
    }
    if (n_layers == 0) return;
    __half *pool = P.pool[array >> 1] + (array & 1) * page_which_elems(P.pg);
    const int per = P.pg.heads * (P.pg.d / 8), total = count * per, limit = P.pg.n_pages * P.pg.page;
    auto at = [&](int sl, int piece) {
        const int page = sl / P.pg.page, off = sl - page * P.pg.page, head = piece / (P.pg.d / 8), pc = piece - head * (P.pg.d / 8);
        return as_global(reinterpret_cast<u32x4 *>(pool + ((size_t)page * P.pg.heads + head) * page_head_elems(P.pg) + ((size_t)(pc >> 1) * P.pg.page + off) * 16 + (pc & 1) * 8));
    };
    constexpr int EACH = 8;
    for (int i0 = 0; i0 < total; i0 += 256 * EACH) {
        u32x4 x[EACH];
        bool moves[EACH];
        int to[EACH], piece[EACH];
#pragma unroll
        for (int u = 0; u < EACH; ++u) {
            const int i = i0 + u * 256 + tid, j = min(i / per, count - 1);
            piece[u] = min(i, total - 1) - j * per;
            const int from = slot[path[j]];
            to[u] = slot[j];
            moves[u] = i < total && path[j] != j && from >= 0 && from < limit && to[u] >= 0 && to[u] < limit;
            if (moves[u]) x[u] = *at(from, piece[u]);
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < EACH; ++u)
            if (moves[u]) *at(to[u], piece[u]) = x[u];
        __syncthreads();
    }
}

hipError_t launch_tree_accept(const AcceptParams &P, int n_layers, hipStream_t s)
{
    hipLaunchKernelGGL(k_tree_accept, dim3(P.b.requests, n_layers > 0 ? 2 * n_layers : 1), dim3(256), 0, s, P, n_layers);
    return hipGetLastError();
}

}  // namespace cfpp
