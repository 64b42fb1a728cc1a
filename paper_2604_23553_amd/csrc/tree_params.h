// Arguments of the kernels for drafted trees over a paged cache (page_kernels.hip, tree_attention.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include "layout.h"

namespace cfpp {

constexpr int kTreeMaxRequests = 4096, kTreeMaxNodes = 256, kTreeMaxGroup = 256, kTreeMaxRows = 1 << 20;

// a pool of pages: fp16 [2][n_pages][heads][d / 16][page][16], and the requests of a step
struct PageDims { int n_pages, page, heads, d; };
struct TreeBatch {
    int requests, max_rows, max_nodes, stride;     // stride: entries of a block table
    const int *lens;
    int *row_start, *table, *slots;
    const int *parents;
    unsigned *masks;
    int *positions;
};

CFPP_HD size_t page_head_elems(const PageDims &p) { return (size_t)p.d * p.page; }
CFPP_HD size_t page_which_elems(const PageDims &p) { return (size_t)p.n_pages * p.heads * page_head_elems(p); }
CFPP_HD int tree_words(int max_nodes) { return (max_nodes + 31) / 32; }

struct TablesParams {
    PageDims pg;
    TreeBatch b;
    const int *counts;
    int *held, *free_pages, *free_count, *granted;
};
hipError_t launch_page_tables(const TablesParams &P, hipStream_t s);

hipError_t launch_page_append(const PageDims &pg, __half *pool, const __half *k, const __half *v, long long row_stride, const int *slots,
                              int n_rows, hipStream_t s);

struct AcceptParams {
    PageDims pg;
    TreeBatch b;
    const int *tokens, *picks;
    int *accepted, *path, *next, *lens_out;
    __half *pool[kMaxLayers];
};
hipError_t launch_tree_accept(const AcceptParams &P, int n_layers, hipStream_t s);

// Rows of a request that take part, in the plan and so in all that follows it: all or none
__device__ __forceinline__ int tree_rows(const PageDims &pg, const TreeBatch &b, int r, int &first)
{
    first = b.row_start[r];
    const int n = b.row_start[r + 1] - first, len = b.lens[r];
    if (n <= 0 || n > b.max_nodes || first < 0 || first + n > b.max_rows || len < 0 || (long long)len + n > (long long)b.stride * pg.page) return 0;
    return b.slots && b.slots[first] < 0 ? 0 : n;
}

// ---- the attention and its plan --------------------------------------------------------------
// Query rows (a node's heads that share a key head, nodes one after the other) go to workgroups in tiles of 16, 32, 64 or 128, positions in pieces.
// A plan: the work list of a key head (TreeItem), arrival counters and the sums of the tiles that are cut into pieces.
struct TreeItem {
    int request, first, nodes, len;    // rows first .. first + nodes - 1 behind len cached positions
    int tile, piece, pieces, slot;     // slot: the tile's first place among the sums, one for each piece; -1 with a single piece
    int t0, t1, pad[2];                // positions
};
struct TreePlanHead { int items, key, cuts, pad[13]; };       // cuts: tiles that have several pieces, listed behind the items
struct TreePlanLayout {
    int tile_rows, want, tiles, work;  // rows of a tile; items aimed at; most tiles; most items
    int piece_step;                    // positions that pieces are multiples of
    int key;                           // of the sizes that a plan is made for
    size_t items, cut, counters, sums, total;   // byte offsets
};
// The smallest tile that has a request's query rows, or 128.  Tiles of 64 and 128 rows read K and V once where tiles of 32 read them twice or more: 64
// requests of 16 nodes, four query heads to a key head, 98 us with tiles of 64 and 118 with 32, 36 rows to a request 88 and 107, 8 requests of up to 256 rows 405
// with 128, 480 with 64 and 758 with 32.  Requests of fewer rows than the tile run as if it were smaller, so a ragged batch loses nothing: up to 36 rows, of
// which most have fewer, 78 and 79.
CFPP_HD int tree_tile_rows(int max_rows_of_request) { return max_rows_of_request <= 16 ? 16 : max_rows_of_request <= 32 ? 32 : max_rows_of_request <= 64 ? 64 : 128; }
TreePlanLayout tree_plan_layout(const PageDims &pg, int n_heads, int requests, int max_rows, int max_nodes, int stride);

struct TreeAttention {
    PageDims pg;
    TreeBatch b;
    int n_heads, group;
    const __half *pool;
    const __half *q;
    __half *out;
    long long q_stride, out_stride;
    unsigned page16_inv;               // ceil(2^32 / (page / 16)), set by the launcher
    // of a stack's rows instead of q and out: queries in 32 bits, outputs as heads and remainders in the order of its products
    const float *q32;
    __half *planes;
    bool narrow;
};
hipError_t launch_tree_plan(const PageDims &pg, const TreeBatch &b, int n_heads, char *plan, hipStream_t s);
hipError_t launch_tree_attention(const TreeAttention &P, char *plan, hipStream_t s);
// adds the pieces of tiles of more than kTaLastJoins query rows
hipError_t launch_tree_join(const TreeAttention &P, const TreePlanLayout &L, const char *plan, hipStream_t s);

// ---- a cache in 8 bits (page8_kernels.hip, page8_attention.hip) -------------------------------
// A pool: bytes [n_pages][heads][page / 16][page8_granule(d)].  A granule, 16 positions t = 4 T + i of a head: K codes [T][d / 16][i][16], V codes
// [d][16 positions], then the largest absolute values of its K rows and of its V rows, fp16 [16] each.
enum { kPage8Int8 = 3, kPage8E4m3 = 4 };
CFPP_HD int page8_granule(int d) { return 32 * d + 64; }
CFPP_HD size_t page8_pool_bytes(const PageDims &p) { return (size_t)p.n_pages * p.heads * (p.page / 16) * page8_granule(p.d); }
struct Page8Rows {
    PageDims pg;
    unsigned char *pool;
    __half *k, *v;                     // [n_rows][stride]: read by the append, written by the other one
    long long stride;
    const int *slots;
    int n_rows;
};
hipError_t launch_page8_append(const Page8Rows &P, int type, hipStream_t s);
hipError_t launch_page8_read(const Page8Rows &P, int type, hipStream_t s);
// P: as for launch_tree_attention, without its pool
hipError_t launch_page8_attention(const TreeAttention &P, const unsigned char *pool, int type, char *plan, hipStream_t s);
// workgroups that the attention launches for each item of the plan's list and key head
CFPP_HD int page8_subtiles(const TreePlanLayout &L) { return L.tile_rows / 16; }

// ---- the rows of a stack's step (PfParams::tree) ---------------------------------------------
struct TreePass {
    PageDims pg;
    TreeBatch b;
    __half *pool;                      // the layer's
    char *plan;
};
hipError_t launch_page_append_slabs(const PageDims &pg, __half *pool, const __half *kv, int rows, const int *slots, int n_rows, hipStream_t s);
// What a step needs of each row: its slot, -1 where its request takes no part in the plan, and its line of the rotary table, rope[positions[row]]; rows
// without a slot take position 0, positions outside the table raise the error flag
struct TreeRows {
    const char *plan;
    int key;                           // of the plan that belongs to the batch
    const float2 *rope;
    int half, max_seq;
    float2 *rope_rows;
    int *slots;
    unsigned *err;
};
hipError_t launch_tree_rope(const PageDims &pg, const TreeBatch &b, const TreeRows &R, hipStream_t s);
// rows that have a slot
hipError_t launch_tree_out(const int *slots, int n_rows, const __half *from, __half *to, int h, hipStream_t s);
struct PfParams;
hipError_t launch_tree_rows(const PfParams &P, hipStream_t s);

}  // namespace cfpp
