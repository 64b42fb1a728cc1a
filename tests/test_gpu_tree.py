"""Drafted trees over a paged cache on the GPU: every operator against its plain form in 64 bits, and a run of them together."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2604_23553_amd as cf
from tests import tree_ref

pytestmark = pytest.mark.gpu

NAN16 = np.uint16(0x7E01)


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def i32(a):
    return dev(np.asarray(a, dtype=np.int32))


def stream():
    return torch.cuda.current_stream().cuda_stream


def half_steps(e):
    """The most that a rounding to fp16 is off: 2^-11 of a value, or half of the subnormals' step, 2^-24 / 2."""
    return np.maximum(np.abs(e) * 2.0 ** -11, 2.0 ** -25)


class Step:
    """Requests with their trees on a pool of pages; every slot that nothing was put into holds NaN."""

    def __init__(self, lens, trees, heads, page=16, seed=0, max_rows=None, max_nodes=None, spare=2, layers=1, scale=1.0, q_pad=0, out_pad=0):
        rng = self.rng = np.random.default_rng([seed, 77])
        self.lens, self.trees, self.page, self.layers = list(lens), trees, page, layers
        self.H, self.kv, self.d = heads
        counts = [len(t) for t in trees]
        self.counts, self.R = counts, len(lens)
        self.rows = sum(counts)
        self.max_rows = self.rows + spare if max_rows is None else max_rows
        self.max_nodes = max(counts + [1]) if max_nodes is None else max_nodes
        self.words = (self.max_nodes + 31) // 32
        self.stride = max(max(tree_ref.pages_for(a + b, page) for a, b in zip(lens, counts)), 1) + 1
        need = sum(tree_ref.pages_for(a + b, page) for a, b in zip(lens, counts))
        self.n_pages = need + 3
        self.alloc = tree_ref.Allocator(self.n_pages, page, self.R, self.stride, rng)
        self.granted, self.starts, self.slots = self.alloc.step(self.lens, counts, self.max_rows)
        assert all(self.granted)
        self.table = np.full((self.R, self.stride), -1, dtype=np.int32)
        for r, t in enumerate(self.alloc.tables):
            self.table[r, :len(t)] = t
        pool = np.full((layers, 2, self.n_pages, self.kv, self.d // 16, page, 16), NAN16, dtype=np.uint16).view(np.float16)
        self.pool = pool
        for r in range(self.R):
            for t in range(self.lens[r] + counts[r]):
                p = self.table[r, t // page]
                pool[:, :, p, :, :, t % page] = rng.standard_normal((layers, 2, self.kv, self.d // 16, 16)).astype(np.float16)
        self.q_stride, self.out_stride = self.H * self.d + q_pad, self.H * self.d + out_pad
        self.q = np.full((self.max_rows, self.q_stride), NAN16, dtype=np.uint16).view(np.float16)
        self.q[:self.rows, :self.H * self.d] = (scale * rng.standard_normal((self.rows, self.H * self.d))).astype(np.float16)
        self.parents = np.full(self.max_rows, 12345, dtype=np.int32)
        self.parents[:self.rows] = sum((list(t) for t in trees), [])
        self.up = [tree_ref.ancestors(t) for t in trees]

    def to_gpu(self):
        self.g = {n: i32(getattr(self, n)) for n in ("lens", "starts", "table", "slots", "parents")}
        self.g_pool, self.g_q = dev(self.pool), dev(self.q)
        self.g_masks = torch.full((self.max_rows, self.words), -7, dtype=torch.int32, device="cuda")
        self.g_positions = torch.full((self.max_rows,), -9, dtype=torch.int32, device="cuda")
        self.g_out = torch.full((self.max_rows, self.out_stride), 7.0, dtype=torch.float16, device="cuda")
        self.pages = cf.Pages(self.n_pages, self.page, self.kv, self.d)
        n = cf.cfpp_tree_plan_bytes(self.pages, self.H, self.R, self.max_rows, self.max_nodes)
        self.plan = torch.full((n,), 0xA5, dtype=torch.uint8, device="cuda")
        self.batch = cf.TreeBatch.of(self.max_nodes, self.g["lens"], self.g["starts"], self.g["table"], self.g["slots"], self.g["parents"],
                                     self.g_masks, self.g_positions, self.plan)
        torch.cuda.synchronize()
        return self

    def run_plan(self):
        cf.cfpp_tree_plan(self.pages, self.batch, self.H, stream())
        return self

    def attention(self, layer=0):
        cf.cfpp_tree_attention(self.pages, self.g_pool[layer], self.batch, self.g_q, self.H, self.g_out, self.q_stride, self.out_stride, stream())
        torch.cuda.synchronize()
        return self.g_out.cpu().numpy()

    def seen(self, r, up):
        n, S = self.counts[r], self.lens[r] + self.counts[r]
        s = np.ones((n, S), dtype=bool)
        s[:, self.lens[r]:] = up[:n, :n]
        return s

    def plain(self, r, up, layer=0):
        S = self.lens[r] + self.counts[r]
        kv = np.zeros((2, S, self.kv, self.d))
        for t in range(S):
            kv[:, t] = tree_ref.slot_row(self.pool[layer], int(self.table[r, t // self.page]) * self.page + t % self.page, self.page)
        a = self.starts[r]
        q = self.q[a:a + self.counts[r], :self.H * self.d].astype(np.float64).reshape(-1, self.H, self.d)
        return tree_ref.attend(q, kv[0], kv[1], self.seen(r, up))

    def check(self, got, up=None, requests=None, layer=0):
        up = self.up if up is None else up
        width = self.H * self.d
        assert (got[:, width:] == 7.0).all(), "columns behind the heads were written"
        assert (got[self.rows:] == 7.0).all(), "rows behind the last request were written"
        err = ref = 0.0
        for r in range(self.R) if requests is None else requests:
            if not self.counts[r]:
                continue
            e, off = self.plain(r, up[r], layer)
            a = self.starts[r]
            g = got[a:a + self.counts[r], :width].astype(np.float64).reshape(e.shape)
            fine = np.isfinite(e)
            assert np.array_equal(np.isnan(g), np.isnan(e)), f"request {r}: NaN in other places"
            assert np.array_equal(g[~fine & ~np.isnan(e)], e[~fine & ~np.isnan(e)])
            limit = np.abs(e) * 2.0 ** -11 + 2.0 ** -25 + off * (1 + 2.0 ** -11)
            far = np.abs(g[fine] - e[fine])
            assert (far <= limit[fine]).all(), f"request {r}: {(far / limit[fine]).max()} of the limit"
            err += (far ** 2).sum()
            ref += (half_steps(e[fine]) ** 2).sum()
        # all roundings together, and 5 % for the evaluation
        assert err <= 1.05 ** 2 * ref, f"2-norm {np.sqrt(err / ref)} of the roundings'"


def trees_of(rng, sizes):
    return [tree_ref.random_tree(rng, n, wide=bool(rng.integers(2))) if n else [] for n in sizes]


# ---- pages and slots ------------------------------------------------------------------------------
def tables_on_gpu(alloc, lens, counts, max_rows, table=None):
    """One call of cfpp_page_tables from an Allocator's state, and everything it wrote."""
    R, page = len(lens), alloc.page
    t = np.full((R, alloc.stride), -77, dtype=np.int32)
    for r, p in enumerate(alloc.tables):
        t[r, :len(p)] = p
    free = np.full(alloc.n_pages, -55, dtype=np.int32)
    free[:len(alloc.free)] = alloc.free
    g = dict(lens=i32(lens), counts=i32(counts), table=i32(t), held=i32([len(p) for p in alloc.tables]), free=i32(free),
             free_count=i32([len(alloc.free)]), granted=i32([-5] * R), row_start=i32([-5] * (R + 1)), slots=i32([-5] * max_rows))
    pages = cf.Pages(alloc.n_pages, page, 1, 64)
    batch = cf.TreeBatch.of(1, g["lens"], g["row_start"], g["table"], g["slots"])
    cf.cfpp_page_tables(pages, batch, g["counts"], g["held"], g["free"], g["free_count"], g["granted"], stream())
    torch.cuda.synchronize()
    return {n: v.cpu().numpy() for n, v in g.items()}, t


def check_tables(alloc, lens, counts, max_rows):
    before = [list(t) for t in alloc.tables]
    got, table = tables_on_gpu(alloc, lens, counts, max_rows)
    granted, starts, slots = alloc.step(lens, counts, max_rows)
    assert list(got["granted"]) == granted
    assert list(got["row_start"]) == starts
    assert np.array_equal(got["slots"], slots)
    assert list(got["held"]) == [len(t) for t in alloc.tables]
    assert got["free_count"][0] == len(alloc.free) and list(got["free"][:len(alloc.free)]) == alloc.free
    for r, t in enumerate(alloc.tables):
        want = table[r].copy()
        want[:len(t)] = t
        want[len(t):len(before[r])] = -1
        assert np.array_equal(got["table"][r], want), f"block table of request {r}"
    return granted


@pytest.mark.parametrize("requests,page,most,stride,share", [(1, 16, 40, 12, 3), (7, 48, 100, 9, 3), (64, 16, 64, 20, 3), (1000, 32, 5, 8, 3), (1025, 16, 70, 12, 3),
                                                             (4096, 16, 9, 30, 3), (40, 16, 60, 12, 6), (300, 32, 100, 12, 5), (4096, 16, 20, 30, 20)])
def test_page_tables_over_steps(requests, page, most, stride, share):
    """Requests grow, shrink, end and begin; in the last three the pages do not reach for all of them."""
    rng = np.random.default_rng([requests, page])
    alloc = tree_ref.Allocator(max(2, requests * stride // share), page, requests, stride, rng)
    lens = rng.integers(0, page * 2, requests)
    refused = 0
    for step in range(6):
        counts = rng.integers(0, most + 1, requests)
        ended = rng.random(requests) < 0.2
        lens[ended], counts[ended] = 0, 0
        granted = check_tables(alloc, [int(v) for v in lens], [int(v) for v in counts], int(counts.sum()) + 5)
        refused += granted.count(0)
        kept = np.array(granted, dtype=bool)
        lens[kept] += rng.integers(0, counts[kept] + 1)
        assert len(set(sum(alloc.tables, []) + alloc.free)) == alloc.n_pages
    assert refused or share == 3


def test_page_tables_refuse_single_requests():
    """A negative length or count, a table that is too short, rows that pass the batch's: only that request goes without."""
    alloc = tree_ref.Allocator(40, 16, 6, 4, np.random.default_rng(5))
    assert check_tables(alloc, [0, -1, 5, 0, 40, 3], [10, 5, -3, 70, 20, 10], 120) == [1, 0, 0, 0, 1, 1]
    assert check_tables(alloc, [10, 0, 5, 0, 60, 13], [10, 5, 2 ** 31 - 1, 4, 2, 10], 25) == [1, 1, 0, 0, 0, 0]
    assert check_tables(alloc, [2 ** 31 - 1, 0, 5, 0, 60, 13], [2 ** 31 - 1, 0, 0, 0, 0, 0], 25) == [0] * 6
    assert check_tables(alloc, [0] * 6, [0] * 6, 1) == [1] * 6
    assert sorted(alloc.free) == list(range(40))


@pytest.mark.parametrize("max_rows", [80, 5000])
def test_slots_of_block_table_entries_outside_the_pool(max_rows):
    """Held pages that are none: their positions have a slot of -1, also where page * page_len comes back to a slot of the pool in 32 bits."""
    page, n_pages, stride = 16, 9, 4
    odd = [2 ** 28 + 3, -3, n_pages, -2 ** 31, 2]          # (the first: slot 48 of 2^32 + 48)
    lens, counts = [5] * 5, [14] * 5
    table = np.full((5, stride), -1, dtype=np.int32)
    table[:, 0] = odd
    g = dict(lens=i32(lens), row_start=i32([0] * 6), table=i32(table), slots=i32([-5] * max_rows), counts=i32(counts), held=i32([1] * 5),
             free=i32([0, 1, 3, 4, 5, 6, 7, 8, -1]), free_count=i32([8]), granted=i32([-5] * 5))
    cf.cfpp_page_tables(cf.Pages(n_pages, page, 1, 64), cf.TreeBatch.of(14, g["lens"], g["row_start"], g["table"], g["slots"]), g["counts"], g["held"],
                        g["free"], g["free_count"], g["granted"], stream())
    torch.cuda.synchronize()
    slots, table = g["slots"].cpu().numpy(), g["table"].cpu().numpy()
    assert list(g["granted"].cpu().numpy()) == [1] * 5 and list(table[:, 0]) == odd and list(table[:, 1]) == [8, 7, 6, 5, 4]
    for r in range(5):
        first = [2 * page + 5 + i if r == 4 else -1 for i in range(11)]
        assert list(slots[14 * r:14 * r + 14]) == first + [(8 - r) * page + i for i in range(3)], f"request {r}"
    assert (slots[70:] == -1).all()


# ---- masks and positions ---------------------------------------------------------------------------
@pytest.mark.parametrize("sizes", [[1], [26], [33, 1, 0, 32, 64, 31], [256, 255, 129], [0, 0, 3]])
def test_tree_plan(sizes):
    rng = np.random.default_rng(sum(sizes))
    s = Step([int(rng.integers(0, 50)) for _ in sizes], trees_of(rng, sizes), (4, 2, 64)).to_gpu().run_plan()
    torch.cuda.synchronize()
    masks, positions = s.g_masks.cpu().numpy(), s.g_positions.cpu().numpy()
    for r, n in enumerate(sizes):
        a = s.starts[r]
        assert np.array_equal(masks[a:a + n], tree_ref.mask_words(s.up[r], s.words))
        assert np.array_equal(positions[a:a + n], s.lens[r] + s.up[r].sum(1) - 1)
    assert (masks[s.rows:] == -7).all() and (positions[s.rows:] == -9).all()


def test_tree_plan_chains_and_odd_parents():
    """A chain of 256 nodes; parents that are no earlier node's make roots."""
    chain = [i - 1 for i in range(256)]
    odd = [5, 1, 7, 2, -3, 2 ** 31 - 1, -(2 ** 31), 0, 7]
    s = Step([3, 9], [chain, odd], (4, 4, 64)).to_gpu().run_plan()
    torch.cuda.synchronize()
    up = tree_ref.ancestors(odd)
    assert up.sum() == 9 + 1 + 1 + 2 and np.array_equal(s.g_masks.cpu().numpy()[256:265], tree_ref.mask_words(up, 8))
    assert list(s.g_positions.cpu().numpy()[:256]) == list(range(3, 259))


def test_requests_that_the_plan_leaves_out():
    """More nodes than max_nodes, no slots, lengths that are negative or past the block table: masks, positions and outputs stay as they were."""
    rng = np.random.default_rng(8)
    s = Step([20, 20, 20, 20, 20], trees_of(rng, [6, 9, 5, 7, 4]), (4, 2, 64), max_nodes=8)
    s.slots[s.starts[2]:s.starts[3]] = -1
    real = list(s.lens)
    s.lens[3], s.lens[4] = -1, s.stride * s.page - 3
    s.to_gpu().run_plan()
    got = s.attention()
    masks = s.g_masks.cpu().numpy()
    assert (masks[6:s.rows] == -7).all() and (s.g_positions.cpu().numpy()[6:s.rows] == -9).all()
    assert (got[6:] == 7.0).all()
    s.lens = real
    s.check(got, requests=[0])


def test_a_plan_without_slots_counts_every_request_and_one_of_other_sizes_writes_nothing():
    rng = np.random.default_rng(18)
    s = Step([30, 7], trees_of(rng, [5, 40]), (4, 2, 64)).to_gpu()
    s.g["slots"].fill_(-1)
    s.batch.slots = 0
    s.run_plan()
    s.check(s.attention())
    s.g_out.fill_(7.0)
    cf.cfpp_tree_attention(s.pages, s.g_pool[0], s.batch, s.g_q, s.H // 2 * 1, s.g_out, s.q_stride, s.out_stride, stream())   # (2 query heads)
    s.batch.max_nodes -= 1
    cf.cfpp_tree_attention(s.pages, s.g_pool[0], s.batch, s.g_q, s.H, s.g_out, s.q_stride, s.out_stride, stream())
    torch.cuda.synchronize()
    assert (s.g_out == 7.0).all()


def test_a_row_start_that_falls_leaves_every_request_out():
    """Rows that are several requests', of which the work list's room knows nothing: no output is written, nor anything behind the plan.  2048 tiles of
    query rows where the plan's sizes are made for 272."""
    R, rows = 256, 256
    s = Step([1], [[-1] + [0] * (rows - 1)], (8, 1, 64), max_nodes=rows, max_rows=rows)
    s.R = R                                                # (sizes of R requests; the arrays below take the place of the one request's)
    s.to_gpu()
    n = s.plan.numel()
    guarded = torch.full((n + (1 << 20),), 0x5A, dtype=torch.uint8, device="cuda")
    starts, lens = i32([0, rows] * (R // 2) + [0]), i32([1] * R)
    table, slots = i32(np.repeat(s.table, R, 0)), i32(s.slots)
    s.batch = cf.TreeBatch.of(rows, lens, starts, table, slots, s.g["parents"], s.g_masks, s.g_positions, guarded[:n])
    s.run_plan()
    got = s.attention()
    assert (got == 7.0).all()
    assert bool((guarded[n:] == 0x5A).all())
    starts.copy_(i32([0] + [rows] * R))                    # (one request has them all)
    s.run_plan()
    s.R, s.starts = 1, [0]
    s.check(s.attention())


# ---- append ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("heads,d,page,rows,pad", [(1, 64, 16, 1, 0), (3, 80, 48, 37, 8), (8, 128, 64, 300, 0), (32, 80, 16, 5, 5120)])
def test_page_append(heads, d, page, rows, pad):
    rng = np.random.default_rng(rows)
    n_pages = rows // page + 5
    slots = rng.permutation(n_pages * page)[:rows].astype(np.int32)
    if rows > 4:
        slots[1], slots[2], slots[3] = -1, n_pages * page, 2 ** 31 - 1
    width = heads * d + pad
    k, v = rng.standard_normal((rows, width)).astype(np.float16), rng.standard_normal((rows, width)).astype(np.float16)
    pool = rng.standard_normal((2, n_pages, heads, d // 16, page, 16)).astype(np.float16)
    g = dev(pool)
    cf.cfpp_page_append(cf.Pages(n_pages, page, heads, d), g, dev(k), dev(v), i32(slots), rows, width, stream())
    torch.cuda.synchronize()
    for i, slot in enumerate(slots):
        if 0 <= slot < n_pages * page:
            pool[0, slot // page, :, :, slot % page] = k[i, :heads * d].reshape(heads, d // 16, 16)
            pool[1, slot // page, :, :, slot % page] = v[i, :heads * d].reshape(heads, d // 16, 16)
    assert np.array_equal(g.cpu().numpy().view(np.uint16), pool.view(np.uint16))


# ---- attention -------------------------------------------------------------------------------------------
@pytest.mark.parametrize("heads", [(8, 8, 64), (4, 1, 64), (6, 2, 80), (16, 16, 80), (5, 5, 128), (12, 4, 128), (34, 2, 64)])
@pytest.mark.parametrize("lens,sizes,page", [
    ([0], [1], 16), ([1], [1], 16), ([300], [1], 64), ([31, 32, 33], [1, 2, 3], 16), ([0, 5, 0], [17, 0, 33], 48), ([100, 0, 257, 640], [16, 1, 7, 15], 32),
    ([1000, 47], [26, 64], 64), ([130], [100], 16),
])
def test_tree_attention(heads, lens, sizes, page):
    rng = np.random.default_rng([*heads, sum(lens), sum(sizes)])
    s = Step(lens, trees_of(rng, sizes), heads, page, seed=sum(lens)).to_gpu().run_plan()
    s.check(s.attention())


@pytest.mark.parametrize("heads,lens,sizes,page", [
    ((2, 2, 128), [3000], [256], 128), ((8, 2, 80), [5000, 17], [70, 3], 16), ((1, 1, 64), [8191], [1], 256), ((16, 1, 64), [2049], [31], 48),
])
def test_tree_attention_behind_long_contexts(heads, lens, sizes, page):
    rng = np.random.default_rng([*heads, sum(lens), sum(sizes)])
    s = Step(lens, trees_of(rng, sizes), heads, page).to_gpu().run_plan()
    first = s.attention()
    s.check(first)
    assert np.array_equal(first.view(np.uint16), s.attention().view(np.uint16)), "the bits change from call to call"


def test_a_page_outside_the_pool_that_only_some_nodes_see():
    """A drafted node in a page outside the pool: its descendants and itself are NaN, the others as ever."""
    s = Step([16], [[-1] + [0] * 30 + [30, 31]], (4, 2, 64), page=16)       # nodes 16 .. 31 stand in the third page
    good = s.table.copy()
    s.table[0, 2] = -1
    s.to_gpu().run_plan()
    got = s.attention()
    s.table = good
    assert np.isnan(got[16:33, :256]).all() and np.isfinite(got[:16]).all()
    e, off = s.plain(0, s.up[0])
    g = got[:16, :256].astype(np.float64).reshape(16, 4, 64)
    assert (np.abs(g - e[:16]) <= np.abs(e[:16]) * 2.0 ** -11 + 2.0 ** -25 + off[:16] * (1 + 2.0 ** -11)).all()


def test_tree_attention_many_requests():
    rng = np.random.default_rng(4)
    sizes = [int(v) for v in rng.integers(0, 6, 300)]
    s = Step([int(v) for v in rng.integers(0, 90, 300)], trees_of(rng, sizes), (4, 2, 64)).to_gpu().run_plan()
    s.check(s.attention())


def test_tree_attention_of_4096_requests():
    """All that a step may have, most of them short or without rows: the plan's classes by length, several requests to a thread."""
    rng = np.random.default_rng(8)
    sizes, lens = [int(v) for v in rng.integers(0, 3, 4096)], [int(v) for v in rng.integers(0, 20, 4096)]
    for r, n in ((0, 700), (17, 1500), (2048, 333), (4095, 900)):
        sizes[r], lens[r] = 2, n
    s = Step(lens, trees_of(rng, sizes), (2, 1, 64), 16).to_gpu().run_plan()
    s.check(s.attention())


@pytest.mark.parametrize("heads", [(4, 1, 64), (8, 2, 80), (4, 1, 128)])
def test_tiles_that_some_wavefronts_have_no_rows_of(heads):
    rng = np.random.default_rng(sum(heads))
    sizes = [9, 16, 24, 13, 17, 1]                         # query rows: 36, 64, 96, 52, 68, 4
    s = Step([900, 40, 2000, 5, 33, 4000], trees_of(rng, sizes), heads, 48).to_gpu().run_plan()
    first = s.attention()
    s.check(first)
    assert np.array_equal(first.view(np.uint16), s.run_plan().attention().view(np.uint16)), "the bits change from plan to plan"


@pytest.mark.parametrize("lens,sizes", [([0, 40], [9, 40]), ([70], [33])])
def test_masks_of_the_callers_own(lens, sizes):
    """Any set of nodes; rows that see nothing (zeros where nothing is cached), all, a later node, and bits behind the last node."""
    rng = np.random.default_rng(sum(sizes))
    s = Step(lens, trees_of(rng, sizes), (4, 2, 80)).to_gpu().run_plan()
    up = [rng.random((n, n)) < 0.5 for n in sizes]
    for u in up:
        u[0], u[1], u[-1] = False, True, False
        u[2, :], u[2, -1] = False, True
    words = [tree_ref.mask_words(u, s.words) for u in up]
    for w in words:
        w[3] |= np.int32(-2 ** 31) if s.words == 1 else 0
    g = np.concatenate(words + [np.full((s.max_rows - s.rows, s.words), -1, dtype=np.int32)])
    for u in up:
        u[3, 31:32] |= s.words == 1
    s.g_masks.copy_(dev(g))
    s.check(s.attention(), up)


def test_strides_and_columns_between():
    rng = np.random.default_rng(2)
    s = Step([50, 3], trees_of(rng, [20, 5]), (6, 3, 80), q_pad=488, out_pad=24).to_gpu().run_plan()
    s.check(s.attention())


def test_unseen_positions_that_are_not_finite():
    """Siblings whose K and V are infinite or NaN change nothing for the nodes that do not see them, and the nodes that do are as the formula has it."""
    rng = np.random.default_rng(6)
    s = Step([45, 0], [tree_ref.random_tree(rng, 40), tree_ref.random_tree(rng, 20)], (4, 2, 64))
    for r, node, which, value in ((0, 7, 0, np.nan), (0, 9, 1, np.nan), (0, 12, 1, np.inf), (0, 13, 0, np.inf), (1, 3, 1, -np.inf), (1, 5, 0, -np.inf)):
        at = s.lens[r] + node
        s.pool[0, which, s.table[r, at // 16], :, :, at % 16, 3:5] = value
    s.to_gpu().run_plan()
    s.check(s.attention())


def test_cached_positions_that_are_not_finite():
    """A cached V of infinity is everybody's infinity of its sign; a cached NaN is everybody's NaN; a key of minus infinity weighs nothing."""
    rng = np.random.default_rng(7)
    s = Step([45, 100, 64], trees_of(rng, [5, 40, 3]), (4, 4, 64))
    s.pool[0, 1, s.table[0, 20 // 16], 1, 2, 20 % 16, 5] = np.inf
    s.pool[0, 1, s.table[0, 30 // 16], 1, 2, 30 % 16, 9] = -np.inf
    s.pool[0, 1, s.table[1, 99 // 16], 2, 0, 99 % 16, 0] = np.nan
    s.pool[0, 0, s.table[2, 10 // 16], 3, 0, 10 % 16, 0] = np.inf       # a score of plus or minus infinity by the sign of q
    s.to_gpu().run_plan()
    s.check(s.attention())


def test_values_that_are_large_and_small():
    """Scores far apart (a single position takes all the weight), and outputs near both ends of the type."""
    rng = np.random.default_rng(9)
    for scale in (60.0, 1e-3):
        s = Step([500], trees_of(rng, [30]), (2, 1, 128), page=64, scale=scale)
        s.pool[0, 1][np.isfinite(s.pool[0, 1])] *= np.float16(8000.0 if scale > 1 else 1e-4)
        s.to_gpu().run_plan()
        s.check(s.attention())


def test_light_positions_behind_a_heavy_one_without_value():
    """The output is what positions of 2^-16 of the largest weight leave: their own digits count."""
    rng = np.random.default_rng(10)
    s = Step([400], trees_of(rng, [20]), (2, 2, 64))
    q = np.zeros((s.rows, s.H, s.d))
    q[:, :, 0], q[:, :, 1:] = 4.0, rng.standard_normal((s.rows, s.H, s.d - 1)) * 0.25
    s.q[:s.rows, :s.H * s.d] = q.reshape(s.rows, -1)
    s.pool[0, 0][:, :, 0, :, 0] = np.where(np.isfinite(s.pool[0, 0][:, :, 0, :, 0]), np.float16(0), s.pool[0, 0][:, :, 0, :, 0])
    s.pool[0, 0, s.table[0, 0], :, 0, 5, 0] = 22.0                      # 4 * 22 / 8 = 11 above the others: e^11 is 2^16 times their weight
    s.pool[0, 1, s.table[0, 0], :, :, 5] = 0
    s.to_gpu().run_plan()
    s.check(s.attention())


@pytest.mark.parametrize("sizes", [[10, 6, 4], [3, 40, 33]])
def test_pages_outside_the_pool_make_their_readers_nan(sizes):
    rng = np.random.default_rng(11)
    s = Step([40, 70, 20], trees_of(rng, sizes), (4, 2, 80))
    good = s.table.copy()
    s.table[1, 2] = s.n_pages
    s.table[2, 0] = -5
    s.to_gpu().run_plan()
    got = s.attention()
    a = s.starts
    assert np.isnan(got[a[1]:a[3], :s.H * s.d]).all()
    s.table = good
    s.check(got, requests=[0])


def test_a_contiguous_cache_is_a_pool():
    """The library's own layer of two sequences, filled by cfpp_kv_import, as two pages."""
    H, d, cap, lens = 4, 80, 64, [40, 9]
    rng = np.random.default_rng(12)
    cfg = cf.Config(H * d, H, d, 20, 4 * H * d, 1, cap, 2, 10000.0, 1e-5, 0)
    kv = torch.full((cf.cfpp_kv_layer_bytes(cfg),), 0xFF, dtype=torch.uint8, device="cuda")
    k, v = (rng.standard_normal((2, H, cap, d)).astype(np.float16) for _ in range(2))
    for b in range(2):
        cf.cfpp_kv_import(cfg, dev(k[b]), dev(v[b]), cap, lens[b] + 2, b, kv, stream())
    q = rng.standard_normal((4, H, d)).astype(np.float16)
    pages = cf.Pages(2, cap, H, d)
    plan = torch.empty(cf.cfpp_tree_plan_bytes(pages, H, 2, 4, 2), dtype=torch.uint8, device="cuda")
    t = [i32(lens), i32([0, 2, 4]), i32([[0], [1]]), i32([lens[0], lens[0] + 1, cap + lens[1], cap + lens[1] + 1]), i32([-1, 0, -1, 0])]
    masks, positions, out = (torch.zeros(n, dtype=ty, device="cuda") for n, ty in (((4, 1), torch.int32), (4, torch.int32), ((4, H * d), torch.float16)))
    batch = cf.TreeBatch.of(2, *t, masks, positions, plan)
    cf.cfpp_tree_plan(pages, batch, H, stream())
    gq = dev(q)
    cf.cfpp_tree_attention(pages, kv, batch, gq, H, out, stream=stream())
    torch.cuda.synchronize()
    for b in range(2):
        S = lens[b] + 2
        seen = np.ones((2, S), dtype=bool)
        seen[0, -1] = False
        e, off = tree_ref.attend(q[2 * b:2 * b + 2].astype(np.float64), *(x[b].astype(np.float64).transpose(1, 0, 2)[:S] for x in (k, v)), seen)
        g = out[2 * b:2 * b + 2].cpu().numpy().astype(np.float64).reshape(e.shape)
        assert (np.abs(g - e) <= np.abs(e) * 2.0 ** -11 + 2.0 ** -25 + off * (1 + 2.0 ** -11)).all()


def test_offsets_past_32_bits():
    """Pages whose values lie past 2^31 elements of the pool."""
    pages = cf.Pages(560, 256, 128, 128)                    # 2 * 560 * 256 * 128 * 128 elements: 4.7 G
    n = cf.cfpp_page_pool_bytes(pages)
    if torch.cuda.mem_get_info()[0] < n + (4 << 30):
        pytest.skip("not enough memory")
    pool = torch.empty((2, 560, 128, 8, 256, 16), dtype=torch.float16, device="cuda")
    rng = np.random.default_rng(13)
    k, v, q = (rng.standard_normal((3, 128, 128)).astype(np.float16) for _ in range(3))
    slots = i32([559 * 256 + 255, 300 * 256, 300 * 256 + 1])
    cf.cfpp_page_append(pages, pool, dev(k), dev(v), slots, 3, None, stream())
    plan = torch.empty(cf.cfpp_tree_plan_bytes(pages, 128, 1, 2, 2), dtype=torch.uint8, device="cuda")
    table = i32([[559, 300]])
    # positions 0 .. 255 of page 559 are cached; all but the last weigh nothing (their keys are minus infinity in q's direction)
    pool[0, 559, :, :, :255] = 0
    pool[0, 559, :, 0, :255, 0] = float("-inf")
    pool[1, 559, :, :, :255] = 0
    q[:, :, 0] = np.abs(q[:, :, 0]) + 0.5
    gq, out = dev(q[:2]), torch.zeros((2, 128 * 128), dtype=torch.float16, device="cuda")
    masks, positions = torch.zeros((2, 1), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    lens, starts, parents, two = i32([256]), i32([0, 2]), i32([-1, 0]), i32([300 * 256, 300 * 256 + 1])
    batch = cf.TreeBatch.of(2, lens, starts, table, two, parents, masks, positions, plan)
    cf.cfpp_tree_plan(pages, batch, 128, stream())
    cf.cfpp_tree_attention(pages, pool, batch, gq, 128, out, stream=stream())
    torch.cuda.synchronize()
    seen = np.array([[1, 1, 0], [1, 1, 1]], dtype=bool)
    e, off = tree_ref.attend(q[:2].astype(np.float64), k.astype(np.float64), v.astype(np.float64), seen)
    g = out.cpu().numpy().astype(np.float64).reshape(e.shape)
    assert (np.abs(g - e) <= np.abs(e) * 2.0 ** -11 + 2.0 ** -25 + off * (1 + 2.0 ** -11)).all()


# (query rows of 16, 32, 64 and 128 to a tile; more than 256 positions are cut into pieces)
@pytest.mark.parametrize("heads,sizes", [((4, 4, 64), [7, 2]), ((5, 5, 80), [26, 3]), ((4, 2, 128), [30, 20]), ((4, 1, 64), [33, 9])])
def test_values_that_are_not_finite_in_pieces(heads, sizes):
    """Infinite and NaN K and V in the middle of a request that is cut into pieces, cached (everybody's) and drafted (its descendants')."""
    rng = np.random.default_rng(sum(sizes))
    s = Step([1500, 700, 400], trees_of(rng, sizes + [5]), heads, 16)
    H = heads[1]
    for r, at, which, head, value in ((0, 620, 1, 0, np.inf), (0, 700, 1, 1 % H, -np.inf), (0, 1001, 0, H - 1, np.inf), (1, 333, 1, 0, np.nan), (1, 420, 0, H - 1, -np.inf),
                                      (2, 402, 1, 0, np.nan), (2, 403, 0, 0, np.inf)):
        s.pool[0, which, s.table[r, at // 16], head, 1, at % 16, 5] = value
    s.to_gpu().run_plan()
    first = s.attention()
    # (the 2-norm of all roundings needs many finite values: each by itself here)
    for r in range(3):
        e, off = s.plain(r, s.up[r])
        g = first[s.starts[r]:s.starts[r] + s.counts[r], :s.H * s.d].astype(np.float64).reshape(e.shape)
        fine = np.isfinite(e)
        assert np.array_equal(np.isnan(g), np.isnan(e)), f"request {r}: NaN in other places"
        assert np.array_equal(g[~fine & ~np.isnan(e)], e[~fine & ~np.isnan(e)])
        assert (np.abs(g[fine] - e[fine]) <= np.abs(e[fine]) * 2.0 ** -11 + 2.0 ** -25 + off[fine] * (1 + 2.0 ** -11)).all(), f"request {r}"
    assert np.isfinite(first[:s.rows]).any() and np.isnan(first[:s.rows, :s.H * s.d]).any()
    assert np.array_equal(first.view(np.uint16), s.attention().view(np.uint16)), "the bits change from call to call"


@pytest.mark.parametrize("heads", [(2, 2, 64), (4, 2, 80), (8, 2, 64)])
def test_pages_outside_the_pool_in_pieces(heads):
    """A cached page outside the pool in a middle piece makes all of its request NaN; one that only some nodes see, in the last piece, makes these NaN."""
    rng = np.random.default_rng(sum(heads))
    s = Step([1500, 1500, 600], [tree_ref.random_tree(rng, 6), [-1] + [0] * 12 + [12, 13], tree_ref.random_tree(rng, 11)], heads, 16)
    good = s.table.copy()
    s.table[0, 40] = s.n_pages + 7
    s.table[1, 94] = -1                                    # (positions 1504 on: the second request's nodes 4 .. 14)
    s.to_gpu().run_plan()
    got = s.attention()
    width = s.H * s.d
    assert np.isnan(got[:6, :width]).all() and np.isnan(got[10:21, :width]).all()
    s.table = good
    e, off = s.plain(1, s.up[1])
    g = got[6:10, :width].astype(np.float64).reshape(4, s.H, s.d)
    assert (np.abs(g - e[:4]) <= np.abs(e[:4]) * 2.0 ** -11 + 2.0 ** -25 + off[:4] * (1 + 2.0 ** -11)).all()
    s.check(got, requests=[2])


# ---- the accepted path -------------------------------------------------------------------------------------
def check_accept(s, tokens, picks, layers, inplace=False, limit=None):
    s.to_gpu()
    g = dict(tokens=i32(tokens), picks=i32(picks), accepted=i32([-5] * s.R), path=i32(np.full((s.R, s.max_nodes), -5)), next=i32([-5] * s.R),
             lens_out=s.g["lens"] if inplace else i32([-5] * s.R))
    cf.cfpp_tree_accept(s.pages, list(s.g_pool[:layers]), s.batch, g["tokens"], g["picks"], g["accepted"], g["path"], g["next"], g["lens_out"], stream())
    torch.cuda.synchronize()
    got = {n: v.cpu().numpy() for n, v in g.items()}
    pool = s.g_pool.cpu().numpy()
    want = s.pool.copy()
    free = np.zeros(s.n_pages * s.page, dtype=bool)        # slots of rows that are not on a path: anything may be left there
    for r, t in enumerate(s.trees):
        a, n = s.starts[r], len(t)
        served = 0 < n <= s.max_nodes and s.slots[a] >= 0
        path = tree_ref.accept(t, tokens[a:a + n], picks[a:a + n]) if served else []
        assert got["accepted"][r] == len(path) and list(got["path"][r]) == path + [-1] * (s.max_nodes - len(path)), f"request {r}"
        assert got["next"][r] == (picks[a + path[-1]] if path else -1) and got["lens_out"][r] == s.lens[r] + len(path)
        for j, i in enumerate(path):
            to, at = int(s.slots[a + j]), int(s.slots[a + i])
            want[:layers, :, to // s.page, :, :, to % s.page] = s.pool[:layers, :, at // s.page, :, :, at % s.page]
        for i in range(len(path), n):
            if s.slots[a + i] >= 0:
                free[s.slots[a + i]] = True
    same = (pool.view(np.uint16) == want.view(np.uint16)).transpose(2, 5, 0, 1, 3, 4, 6).reshape(s.n_pages * s.page, -1).all(1)
    assert (same | free).all()
    return got


def drafted(rng, trees, rows, agree):
    """Tokens and picks; a node agrees with the pick behind its parent with that probability."""
    tokens, picks = rng.integers(0, 50, rows).astype(np.int32), rng.integers(0, 50, rows).astype(np.int32)
    a = 0
    for t in trees:
        for i, p in enumerate(t):
            if p >= 0 and rng.random() < agree:
                tokens[a + i] = picks[a + p]
        a += len(t)
    return tokens, picks


@pytest.mark.parametrize("sizes,heads,page,layers,agree", [
    ([1], (2, 2, 64), 16, 1, 1.0), ([26], (4, 4, 80), 16, 3, 0.7), ([5, 0, 33, 1, 64], (2, 2, 128), 48, 2, 0.8), ([256], (1, 1, 64), 16, 2, 1.0),
    ([256, 200], (3, 3, 80), 64, 1, 0.95), ([17] * 40, (2, 2, 64), 16, 2, 0.5),
])
def test_tree_accept(sizes, heads, page, layers, agree):
    rng = np.random.default_rng(sum(sizes))
    trees = trees_of(rng, sizes)
    if len(sizes) == 2:
        trees[0] = [max(i - 2, -1) for i in range(256)]     # two chains: a path far from its place
        trees[0][1] = 0
    s = Step([int(rng.integers(0, 40)) for _ in sizes], trees, heads, page, layers=layers)
    tokens, picks = drafted(rng, trees, s.max_rows, agree)
    check_accept(s, tokens, picks, layers)


def test_tree_accept_in_place_without_layers_and_left_out():
    rng = np.random.default_rng(21)
    trees = trees_of(rng, [6, 12, 7])
    s = Step([10, 20, 30], trees, (2, 2, 64), max_nodes=8)
    s.slots[s.starts[2]:s.starts[3]] = -1
    tokens, picks = drafted(rng, trees, s.max_rows, 1.0)
    got = check_accept(s, tokens, picks, 0, inplace=True)
    assert got["accepted"][0] > 1 and list(got["accepted"][1:]) == [0, 0]


def test_tree_accept_roots_other_than_node_0():
    """A second node without parent is never taken, nor a child whose number is not above its parent's."""
    s = Step([4], [[-1, -1, 1, 0, 3]], (2, 2, 64))
    got = check_accept(s, np.array([1, 7, 7, 7, 9, 0, 0], dtype=np.int32), np.array([7, 7, 7, 9, 2, 0, 0], dtype=np.int32), 1)
    assert list(got["path"][0][:4]) == [0, 3, 4, -1]


# ---- together ------------------------------------------------------------------------------------------------
class Server:
    """Steps of tables, plan, append, attention and accept over a pool, beside a plain cache for each request."""

    def __init__(self, R, heads, page, layers, max_rows, max_nodes, n_pages, stride, seed):
        self.rng = np.random.default_rng(seed)
        self.R, (self.H, self.kv, self.d), self.page, self.layers, self.max_rows, self.max_nodes = R, heads, page, layers, max_rows, max_nodes
        z = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
        self.pages = cf.Pages(n_pages, page, self.kv, self.d)
        words = (max_nodes + 31) // 32
        self.lens, self.counts, self.row_start, self.table, self.held = z(R), z(R), z(R + 1), z(R, stride), z(R)
        self.free, self.free_count = torch.randperm(n_pages, dtype=torch.int32, device="cuda"), i32([n_pages])
        self.granted, self.slots, self.parents, self.masks, self.positions = z(R), z(max_rows), z(max_rows), z(max_rows, words), z(max_rows)
        self.tokens, self.picks, self.accepted, self.path, self.next = z(max_rows), z(max_rows), z(R), z(R, max_nodes), z(R)
        self.plan = torch.empty(cf.cfpp_tree_plan_bytes(self.pages, self.H, R, max_rows, max_nodes), dtype=torch.uint8, device="cuda")
        self.batch = cf.TreeBatch.of(max_nodes, self.lens, self.row_start, self.table, self.slots, self.parents, self.masks, self.positions, self.plan)
        self.pool = torch.full((layers, 2, n_pages, self.kv, self.d // 16, page, 16), float("nan"), dtype=torch.float16, device="cuda")
        h = lambda heads: torch.zeros((layers, max_rows, heads, self.d), dtype=torch.float16, device="cuda")  # noqa: E731
        self.q, self.k, self.v, self.out = h(self.H), h(self.kv), h(self.kv), h(self.H)
        self.cache = [np.zeros((layers, 2, 0, self.kv, self.d)) for _ in range(R)]

    def enqueue(self):
        s = stream()
        cf.cfpp_page_tables(self.pages, self.batch, self.counts, self.held, self.free, self.free_count, self.granted, s)
        cf.cfpp_tree_plan(self.pages, self.batch, self.H, s)
        for l in range(self.layers):
            cf.cfpp_page_append(self.pages, self.pool[l], self.k[l], self.v[l], self.slots, self.max_rows, None, s)
            cf.cfpp_tree_attention(self.pages, self.pool[l], self.batch, self.q[l], self.H, self.out[l], stream=s)
        cf.cfpp_tree_accept(self.pages, list(self.pool), self.batch, self.tokens, self.picks, self.accepted, self.path, self.next, self.lens, s)

    def new_inputs(self, sizes):
        self.trees = trees_of(self.rng, sizes)
        self.sizes = sizes
        f = lambda t: t.copy_(dev(self.rng.standard_normal(tuple(t.shape)).astype(np.float16)))  # noqa: E731
        self.host = [f(t).cpu().numpy().astype(np.float64) for t in (self.q, self.k, self.v)]
        tokens, picks = drafted(self.rng, self.trees, self.max_rows, 0.7)
        self.host_tokens, self.host_picks = tokens, picks
        parents = np.full(self.max_rows, -1, dtype=np.int32)
        parents[:sum(sizes)] = sum(self.trees, [])
        for t, a in ((self.tokens, tokens), (self.picks, picks), (self.parents, parents), (self.counts, np.array(sizes, dtype=np.int32))):
            t.copy_(dev(a))
        self.out.fill_(7.0)
        torch.cuda.synchronize()

    def check(self):
        torch.cuda.synchronize()
        assert (self.granted.cpu().numpy() == 1).all()
        out, accepted = self.out.cpu().numpy().astype(np.float64), self.accepted.cpu().numpy()
        a = 0
        for r, n in enumerate(self.sizes):
            path = tree_ref.accept(self.trees[r], self.host_tokens[a:a + n], self.host_picks[a:a + n]) if n else []
            assert accepted[r] == len(path)
            S = self.cache[r].shape[2]
            q, k, v = (x[:, a:a + n] for x in self.host)
            new = np.stack([k, v], 1)
            both = np.concatenate([self.cache[r], new], 2)
            seen = np.ones((n, S + n), dtype=bool)
            if n:
                seen[:, S:] = tree_ref.ancestors(self.trees[r])
            for l in range(self.layers):
                e, off = tree_ref.attend(q[l], both[l, 0], both[l, 1], seen)
                g = out[l, a:a + n]
                assert (np.abs(g - e) <= np.abs(e) * 2.0 ** -11 + 2.0 ** -25 + off * (1 + 2.0 ** -11)).all(), f"request {r}, layer {l}"
            self.cache[r] = np.concatenate([self.cache[r], new[:, :, path]], 2)
            a += n
        assert list(self.lens.cpu().numpy()) == [c.shape[2] for c in self.cache]
        assert (out[:, a:] == 7.0).all()


def test_steps_together():
    s = Server(4, (4, 2, 64), 16, 2, 70, 20, 60, 12, 31)
    for step, sizes in enumerate([[20, 1, 7, 0], [3, 20, 0, 12], [1, 1, 1, 1], [20, 20, 20, 9], [0, 0, 1, 0], [5, 6, 7, 8]]):
        s.new_inputs(sizes)
        s.enqueue()
        s.check()


def test_steps_replayed_from_a_graph_on_another_stream():
    """One captured step, replayed with new trees, lengths and counts; eager work of the program in between."""
    s = Server(3, (4, 4, 80), 16, 2, 50, 26, 60, 12, 32)
    side = torch.cuda.Stream()
    s.new_inputs([4, 0, 9])
    with torch.cuda.stream(side):
        s.enqueue()
    side.synchronize()
    s.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        s.enqueue()
    for sizes in ([26, 1, 3], [1, 1, 1], [2, 26, 20], [0, 0, 0], [7, 8, 9]):
        s.new_inputs(sizes)
        graph.replay()
        torch.randn(1000, device="cuda").sum().item()
        s.check()
