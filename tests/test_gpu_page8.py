"""A paged cache in 8 bits on the GPU: rows into it and back, and the attention over it, against plain forms in 64 bits."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2604_23553_amd as cf
from tests import page8_ref, tree_ref
from tests.test_gpu_tree import NAN16, Step, dev, half_steps, i32, stream, trees_of

pytestmark = pytest.mark.gpu

TYPES = [page8_ref.INT8, page8_ref.E4M3]


def bits(a):
    return np.ascontiguousarray(a).view(np.uint16)


# ---- rows in and out ----------------------------------------------------------------------------------
def same_bytes(got, want):
    """Two pools' bytes: e4m3's zeros of either sign are equal, and NaN of any bits"""
    d = want.d
    far = got != want.bytes
    if want.type == page8_ref.E4M3:
        far[..., :32 * d] &= ((got | want.bytes)[..., :32 * d] & 0x7F) != 0
    nan = [np.isnan(np.ascontiguousarray(b[..., 32 * d:]).view(np.float16)) for b in (got, want.bytes)]
    far[..., 32 * d:] &= ~np.repeat(nan[0] & nan[1], 2, -1)
    return not far.any()


def append(pool, k, v, slots, pad=0):
    """pool: a page8_ref.Pool, whose bytes are those before; the bytes behind"""
    n = len(slots)
    width = pool.heads * pool.d
    rows = np.full((2, n, width + pad), NAN16, dtype=np.uint16).view(np.float16)
    rows[0, :, :width], rows[1, :, :width] = k.reshape(n, width), v.reshape(n, width)
    g, gk, gv, gs = dev(pool.bytes), dev(rows[0]), dev(rows[1]), i32(slots)
    cf.cfpp_page8_append(cf.Pages(pool.n_pages, pool.page, pool.heads, pool.d), pool.type, g, gk, gv, gs, n, width + pad, stream())
    torch.cuda.synchronize()
    return g.cpu().numpy()


def read(pool, slots, pad=0):
    n, width = len(slots), pool.heads * pool.d
    out = [torch.full((n, width + pad), 7.0, dtype=torch.float16, device="cuda") for _ in range(2)]
    cf.cfpp_page8_read(cf.Pages(pool.n_pages, pool.page, pool.heads, pool.d), pool.type, dev(pool.bytes), i32(slots), n, out[0], out[1], width + pad, stream())
    torch.cuda.synchronize()
    got = np.stack([x.cpu().numpy() for x in out])
    assert (got[:, :, width:] == 7.0).all(), "columns behind the heads were written"
    return got[:, :, :width].reshape(2, n, pool.heads, pool.d)


def slots_of(kind, n, positions, page, rng):
    """Slots of n rows in a pool of so many positions"""
    if kind == "scattered":
        return rng.permutation(positions)[:n]
    if kind == "in order":
        return np.arange(n) + 5
    if kind == "pieces":                                   # runs of all lengths, holes and slots that are none between them
        out, at = [], 0
        while len(out) < n:
            k = int(rng.integers(1, 40))
            out += list(range(at, at + k))
            at += k + int(rng.integers(0, 3))
            if rng.random() < 0.3:
                out.append([-1, positions, 2 ** 31 - 1, -2 ** 31][int(rng.integers(4))])
        return np.array(out[:n])
    return (np.arange(n) + 3)[::-1]                        # backwards


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("heads,d,page,n,kind", [
    (1, 64, 16, 1, "scattered"), (8, 64, 16, 33, "pieces"), (3, 80, 48, 100, "pieces"), (32, 80, 64, 64, "scattered"), (5, 128, 32, 300, "pieces"),
    (2, 128, 256, 17, "in order"), (7, 80, 16, 160, "backwards"), (9, 64, 128, 1000, "in order"), (4, 128, 64, 16, "in order"), (6, 64, 16, 257, "scattered"),
    (33, 80, 16, 31, "pieces"), (1, 128, 16, 15, "pieces")])
def test_rows_in_and_out(type, heads, d, page, n, kind):
    rng = np.random.default_rng([heads, d, n])
    n_pages = (3 * n + 80) // page + 2
    slots = slots_of(kind, n, n_pages * page, page, rng).astype(np.int64)
    assert len(np.unique(slots[(slots >= 0) & (slots < n_pages * page)])) == ((slots >= 0) & (slots < n_pages * page)).sum()
    rows = (rng.standard_normal((2, n, heads, d)) * 2.0 ** rng.integers(-12, 10, (2, n, heads, 1))).astype(np.float16)
    pad = [0, 8, 24][n % 3]
    want = page8_ref.Pool(n_pages, page, heads, d, type)
    got = append(want, rows[0], rows[1], slots, pad)
    for s, k, v in zip(slots, rows[0], rows[1]):
        want.put(int(s), k, v)
    assert same_bytes(got, want)
    # and back, the same slot twice among them
    back = np.concatenate([slots, slots[:1], slots[-3:]])
    out = read(want, back, pad)
    for i, s in enumerate(back):
        if 0 <= s < n_pages * page:
            assert np.array_equal(out[:, i], want.get(int(s)).astype(np.float16)), f"row {i}"
        else:
            assert (out[:, i] == 7.0).all(), f"row {i} has no slot"


@pytest.mark.parametrize("type", TYPES)
def test_codes_next_to_ties_and_values_out_of_the_way(type):
    """Ties between codes, the smallest and largest numbers, rows of zeros, infinities and NaN; d = 80 has them in all places."""
    rng = np.random.default_rng(4)
    d, heads, n = 80, 2, 400
    rows = rng.standard_normal((2, n, heads, d)).astype(np.float16)
    whole = rng.integers(-254, 255, (n, heads, d))
    whole[..., 3] = 254                                    # 127 x / 254: every odd number is a tie
    rows[0] = whole
    rows[1] = rng.choice(np.concatenate([page8_ref.E4M3_VALUES[:126] / 2 + page8_ref.E4M3_VALUES[1:127] / 2, page8_ref.E4M3_VALUES[:127]]), (n, heads, d))
    rows[1][..., 7] = -448
    rows[:, 100:150] *= np.float16(2.0 ** -8)
    rows[0, 150:200] = (rng.integers(-40, 41, (50, heads, d)) * 2.0 ** -24).astype(np.float16)
    rows[1, 150:200] = (rng.integers(-2047, 2048, (50, heads, d)) * 32.0).astype(np.float16)
    rows[:, 200:210] = 0.0
    rows[:, 210:215] = -0.0
    for i, bad in enumerate((np.inf, -np.inf, np.nan)):
        rows[i % 2, 220 + i, 1, 11 * i] = bad
    want = page8_ref.Pool(n // 16 + 2, 16, heads, d, type)
    slots = np.arange(n) + 7
    got = append(want, rows[0], rows[1], slots)
    for s, k, v in zip(slots, rows[0], rows[1]):
        want.put(int(s), k, v)
    assert same_bytes(got, want)
    out = read(want, slots)
    for i, s in enumerate(slots):
        w = want.get(int(s)).astype(np.float16)
        assert np.array_equal(out[:, i], w, equal_nan=True)
    assert np.isnan(out[0, 220, 1]).all() and np.isfinite(out[0, 220, 0]).all() and np.isfinite(out[1, 220]).all()


def test_rows_interleaved_with_others():
    """K and V as two halves of one array's rows, in and out"""
    rng = np.random.default_rng(8)
    heads, d, n = 4, 64, 50
    both = rng.standard_normal((n, 2, heads * d)).astype(np.float16)
    pool = page8_ref.Pool(8, 16, heads, d, page8_ref.INT8)
    pages, g, x, s = cf.Pages(8, 16, heads, d), dev(pool.bytes), dev(both), i32(np.arange(n) + 30)
    back = torch.zeros_like(x)
    cf.cfpp_page8_append(pages, pool.type, g, x.data_ptr(), x.data_ptr() + 2 * heads * d, s, n, 2 * heads * d, stream())
    cf.cfpp_page8_read(pages, pool.type, g, s, n, back.data_ptr(), back.data_ptr() + 2 * heads * d, 2 * heads * d, stream())
    torch.cuda.synchronize()
    for i in range(n):
        pool.put(30 + i, *both[i].reshape(2, heads, d))
        assert np.array_equal(back[i].cpu().numpy(), pool.get(30 + i).astype(np.float16).reshape(2, -1))


# ---- the attention -------------------------------------------------------------------------------------
class Step8(Step):
    """Step with a pool of codes: what its fp16 pool holds, quantised; what it does not hold is no number in any part."""

    def __init__(self, *args, type=page8_ref.INT8, change=None, **more):
        super().__init__(*args, **more)
        self.type = type
        if change:
            change(self)

    def to_gpu(self):
        x = self.pool[0].transpose(1, 4, 0, 2, 3, 5).reshape(self.n_pages, self.page, 2, self.kv, self.d)
        self.pool8 = page8_ref.Pool(self.n_pages, self.page, self.kv, self.d, self.type)
        unwritten = bits(x[:, :, 0, 0, 0]).reshape(self.n_pages, self.page) == NAN16
        for p, t in zip(*np.nonzero(~unwritten)):
            self.pool8.put(int(p) * self.page + int(t), x[p, t, 0], x[p, t, 1])
        self.g_pool8 = dev(self.pool8.bytes)
        return super().to_gpu()

    def attention8(self, on=None):
        cf.cfpp_page8_attention(self.pages, self.type, self.g_pool8, self.batch, self.g_q, self.H, self.g_out, self.q_stride, self.out_stride,
                                stream() if on is None else on)
        return self

    def result(self):
        torch.cuda.synchronize()
        return self.g_out.cpu().numpy()

    def plain(self, r, up, layer=0):
        S = self.lens[r] + self.counts[r]
        kv = np.stack([self.pool8.get(int(self.table[r, t // self.page]) * self.page + t % self.page) for t in range(S)], 1)
        a = self.starts[r]
        q = self.q[a:a + self.counts[r], :self.H * self.d].astype(np.float64).reshape(-1, self.H, self.d)
        return page8_ref.attend(q, kv[0], kv[1], self.seen(r, up))


def ones(n):
    return [[-1]] * n


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("lens,heads,page,more", [
    ([0], (8, 8, 64), 16, {}),
    ([1, 0, 14, 15, 16, 17], (4, 4, 80), 16, {}),
    ([62, 63, 64, 65, 126, 127, 128, 129], (8, 2, 128), 48, dict(q_pad=8, out_pad=16)),
    ([254, 255, 256, 257, 300], (16, 1, 64), 64, {}),
    ([700, 3, 1023, 40], (3, 3, 80), 256, dict(out_pad=8)),
    ([2500], (4, 2, 128), 32, {}),
    ([4095], (2, 2, 80), 64, {}),
    ([90, 513, 0], (20, 1, 80), 16, {}),                     # more than 16 query heads to a key head
    ([400, 33], (34, 2, 64), 32, {}),
    ([129], (256, 1, 64), 16, {}),
    ([6000], (5, 1, 64), 128, {}),
])
def test_single_tokens(type, lens, heads, page, more):
    s = Step8(lens, ones(len(lens)), heads, page=page, seed=len(lens) + heads[0], type=type, **more).to_gpu()
    s.run_plan().attention8()
    s.check(s.result())


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("sizes,lens,heads,page", [
    ([5, 0, 16, 1], [100, 7, 0, 333], (2, 2, 80), 16),       # 16 query rows at most
    ([9, 3, 32], [70, 600, 0], (4, 2, 64), 32),              # 64
    ([40, 64, 2], [500, 31, 1], (4, 4, 128), 16),            # 64, with masks of several words
    ([100, 7], [400, 900], (4, 2, 80), 64),                  # 128 and more tiles
])
def test_trees(type, sizes, lens, heads, page):
    rng = np.random.default_rng(len(sizes))
    s = Step8(lens, trees_of(rng, sizes), heads, page=page, seed=9, type=type).to_gpu()
    s.run_plan().attention8()
    s.check(s.result())


@pytest.mark.parametrize("type", TYPES)
def test_masks_of_the_callers(type):
    """Any set of the request's nodes, none among them, over no cached positions too"""
    rng = np.random.default_rng(2)
    sizes = [6, 10, 3]
    s = Step8([0, 90, 0], trees_of(rng, sizes), (4, 4, 64), seed=5, type=type).to_gpu()
    s.run_plan()
    up = [rng.random((n, n)) < 0.5 for n in sizes]
    up[0][2] = False
    up[2][:] = False
    words = np.concatenate([tree_ref.mask_words(u, s.words) for u in up] + [np.zeros((s.max_rows - s.rows, s.words), np.int32)])
    s.g_masks.copy_(dev(words.astype(np.int32)))
    s.attention8()
    s.check(s.result(), up=up)


@pytest.mark.parametrize("type", TYPES)
def test_scales_of_all_sizes(type):
    """Rows of V from fp16's smallest numbers to its largest in one request, rows of zeros, keys that dominate"""
    def change(s):
        for r in range(s.R):
            for t in range(s.lens[r] + 1):
                at = s.pool[0][:, s.table[r, t // s.page], :, :, t % s.page]
                at[1] *= np.float16(2.0) ** np.float16(s.rng.integers(-22, 13) if r else -14)
                if t % 7 == 3:
                    at[t % 2] = 0.0
                if t % 50 == 9:
                    at[0] *= np.float16(8.0)
    s = Step8([200, 200, 1000], ones(3), (4, 2, 80), seed=3, type=type, change=change).to_gpu()
    s.run_plan().attention8()
    s.check(s.result())


@pytest.mark.parametrize("type", TYPES)
def test_rows_that_are_no_numbers(type):
    """An infinite value in a row of K or of V makes the heads that see it NaN, and no others"""
    def change(s):
        s.pool[0][0, s.table[0, 2], 1, 0, 5, 3] = np.inf
        s.pool[0][1, s.table[1, 0], 0, 2, 15, 0] = np.nan
        s.pool[0][1, s.table[2, 1], 1, 3, 1, 1] = -np.inf
    s = Step8([130, 40, 300, 77], ones(4), (4, 2, 64), seed=6, type=type, change=change).to_gpu()
    s.run_plan().attention8()
    got = s.result()
    s.check(got)
    nan = np.isnan(got[:4].astype(np.float32)).reshape(4, 4, 64).all(-1)
    assert nan.tolist() == [[False, False, True, True], [True, True, False, False], [False, False, True, True], [False] * 4]


def test_a_query_that_is_infinite():
    s = Step8([20, 200], ones(2), (2, 2, 64), seed=6)
    s.q[0, 5], s.q[1, 64 + 9] = np.inf, -np.inf
    s.to_gpu().run_plan().attention8()
    got = s.result()[:2].astype(np.float32).reshape(2, 2, 64)
    assert np.isnan(got[0, 0]).all() and np.isnan(got[1, 1]).all() and np.isfinite(got[0, 1]).all() and np.isfinite(got[1, 0]).all()


@pytest.mark.parametrize("bad", [-1, 10 ** 6, -2 ** 31])
def test_block_table_entries_outside_the_pool(bad):
    s = Step8([200, 60, 90], ones(3), (4, 2, 64), seed=7).to_gpu()
    s.g["table"][0, 3] = bad
    s.g["table"][1, 1:] = bad                               # the request's second page on
    s.g["table"][2, 6:] = bad                               # behind its last position
    s.run_plan().attention8()
    got = s.result()
    s.check(got, requests=[2])
    assert np.isnan(got[:2, :256]).all()


def test_requests_that_are_left_out():
    """No row, no slot, lengths that are none: their rows stay as they were"""
    s = Step8([50, 60, 70, 80], ones(4), (4, 4, 64), seed=8).to_gpu()
    s.g["slots"][1] = -1
    s.g["lens"][2] = -5
    s.run_plan().attention8()
    got = s.result()
    s.check(got, requests=[0, 3])
    assert (got[1:3] == 7.0).all()


def test_a_plan_of_other_sizes_writes_nothing():
    s = Step8([50], ones(1), (4, 4, 64), seed=8).to_gpu()
    s.attention8()
    assert (s.result() == 7.0).all()


def test_the_same_bits_every_time_and_from_a_graph():
    """Replays follow what is in memory: lengths, tables and masks of other steps, with eager work in between"""
    s = Step8([900, 64, 2000, 0], ones(4), (8, 2, 128), page=16, seed=11, type=page8_ref.E4M3).to_gpu()
    first = s.run_plan().attention8().result().copy()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        cf.cfpp_tree_plan(s.pages, s.batch, s.H, stream())
        s.attention8()
    lens = s.g["lens"].clone()
    for k in range(4):
        s.g_out.fill_(7.0)
        graph.replay()
        assert np.array_equal(bits(s.result()), bits(first))
        s.g["lens"].copy_(torch.clamp(lens - 31 * (k + 1), min=0))
        s.g_out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        shorter = s.g_out.cpu().numpy()
        s.g_out.fill_(7.0)
        s.run_plan().attention8()
        assert np.array_equal(bits(s.result()), bits(shorter)) and not np.array_equal(bits(shorter), bits(first))
        s.g["lens"].copy_(lens)


def test_long_contexts_and_offsets_past_32_bits():
    """A pool of more than 4 GB; 70000 positions of one request, cut into many pieces"""
    heads, d, page, n = 32, 128, 64, 70000
    pages = n // page + 1
    n_pages = 9000                                          # 4.8 GB
    pool = torch.zeros((n_pages, heads, page // 16, 32 * d + 64), dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    order = torch.randperm(n_pages, generator=g, device="cuda")[:pages]
    order[-1] = n_pages - 1                                 # (its last positions lie past 2^32 bytes)
    order = torch.unique(order).flip(0)
    table = order[None].to(torch.int32).contiguous()
    have = table.shape[1] * page
    pos = torch.arange(have, device="cuda")
    slots = (table[0, pos // page] * page + pos % page).to(torch.int32)
    P = cf.Pages(n_pages, page, heads, d)
    k = torch.randn((have, heads, d), generator=g, device="cuda", dtype=torch.float16)
    v = torch.randn((have, heads, d), generator=g, device="cuda", dtype=torch.float16)
    cf.cfpp_page8_append(P, cf.TYPE_INT8, pool, k, v, slots, have, stream=stream())
    kk, vv = torch.zeros_like(k), torch.zeros_like(v)
    cf.cfpp_page8_read(P, cf.TYPE_INT8, pool, slots, have, kk, vv, stream=stream())
    for x, y in ((k, kk), (v, vv)):
        a = x.abs().amax(-1, keepdim=True).double()
        codes = torch.round(x.double() * 127 / a)
        assert torch.equal(y, (codes * a / 127).half())
    q = torch.randn((1, heads, d), generator=g, device="cuda", dtype=torch.float16)
    out = torch.zeros_like(q)
    L = have - 1
    lens, starts, one = i32([L]), i32([0, 1]), i32([int(slots[L])])
    plan = torch.empty(cf.cfpp_tree_plan_bytes(P, heads, 1, 1, 1), dtype=torch.uint8, device="cuda")
    parents, masks, positions = i32([-1]), i32([[0]]), i32([0])
    batch = cf.TreeBatch.of(1, lens, starts, table, one, parents, masks, positions, plan)
    cf.cfpp_tree_plan(P, batch, heads, stream())
    cf.cfpp_page8_attention(P, cf.TYPE_INT8, pool, batch, q, heads, out, stream=stream())
    torch.cuda.synchronize()
    for h in (0, 13, 31):
        x, y = (t[:, h].double() for t in (k, v))
        x, y = (torch.round(t * 127 / t.abs().amax(-1, keepdim=True)) * t.abs().amax(-1, keepdim=True) / 127 for t in (x, y))
        p = torch.softmax(torch.mv(x, q[0, h].double()) / np.sqrt(d), 0)
        want = torch.mv(y.t().contiguous(), p)
        # half a step of fp16; weights off by 2^-18 at most, of sums of |p v|
        limit = want.abs() * 2.0 ** -11 + 2.0 ** -25 + 2.0 ** -17 * torch.mv(y.abs().t().contiguous(), p)
        assert ((out[0, h].double() - want).abs() <= limit).all()


def test_two_batches_on_two_streams():
    """Each with a plan of its own, over one pool"""
    a = Step8([1500, 90], ones(2), (8, 8, 64), seed=21).to_gpu()
    b = Step8([700, 2100], ones(2), (4, 4, 80), seed=22, type=page8_ref.E4M3).to_gpu()
    a.run_plan()
    b.run_plan()
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        a.attention8(one.cuda_stream)
        b.attention8(two.cuda_stream)
    a.check(a.result())
    b.check(b.result())


@pytest.mark.parametrize("type", TYPES)
def test_many_pieces_behind_one_plan(type):
    """Requests of 31 and 20 pieces, whose sums are joined in two steps: every layer's call finds the plan as the one before it did, one over an fp16 pool among them"""
    s = Step8([3950, 900, 2500], ones(3), (4, 2, 80), seed=41, type=type).to_gpu()
    s.run_plan()
    first = s.attention8().result().copy()
    s.check(first)
    half = s.attention().copy()
    for _ in range(3):
        s.g_out.fill_(7.0)
        assert np.array_equal(bits(s.attention8().result()), bits(first))
        s.g_out.fill_(7.0)
        assert np.array_equal(bits(s.attention()), bits(half))
    s.q = -s.q                                              # other queries: no sum is that of the call before
    s.g_q.copy_(dev(s.q))
    s.check(s.attention8().result())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    one = torch.zeros_like(s.g_out)
    with torch.cuda.graph(graph, stream=side):
        cf.cfpp_tree_plan(s.pages, s.batch, s.H, stream())
        s.attention8()
        one.copy_(s.g_out)
        s.attention8()
    for r, n in ((0, 3950), (1, 3000), (0, 2049), (2, 64)):
        s.g["lens"][r] = s.lens[r] = min(n, s.lens[r])
        s.g_out.fill_(7.0)
        graph.replay()
        replayed = s.result().copy()
        assert np.array_equal(bits(replayed), bits(one.cpu().numpy()))
        s.g_out.fill_(7.0)
        s.run_plan().attention8()
        assert np.array_equal(bits(s.result()), bits(replayed))
        s.check(replayed)


def test_many_pieces_on_two_streams():
    """Each batch with a plan of its own, over and over"""
    a = Step8([3950, 90], ones(2), (8, 2, 64), seed=42).to_gpu()
    b = Step8([3500, 90], ones(2), (4, 2, 128), seed=43, type=page8_ref.E4M3).to_gpu()
    a.run_plan()
    b.run_plan()
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        a.attention8(one.cuda_stream)
        b.attention8(two.cuda_stream)
    a.check(a.result())
    b.check(b.result())


# ---- what lies in positions that a row does not see ------------------------------------------------------
def unwritten(s, r, node):
    """A node's slot holds what a pool begins with"""
    t = s.lens[r] + node
    s.pool[0][:, s.table[r, t // s.page], :, :, t % s.page] = np.full(1, NAN16, dtype=np.uint16).view(np.float16)


@pytest.mark.parametrize("poison", [0x7F, 0xFF])
@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("sizes,lens,heads,page", [
    ([4, 1, 6], [0, 33, 100], (2, 2, 64), 16),               # 16 query rows at most
    ([11, 3, 9], [70, 250, 16], (4, 2, 80), 16),             # 64
    ([6, 16], [45, 300], (4, 4, 128), 32),
    ([64, 40], [500, 31], (2, 1, 128), 48),                  # 128, masks of several words
])
def test_unseen_positions_that_were_never_written(type, poison, sizes, lens, heads, page):
    """Nodes that no mask shows need no K and V: codes and scales that are no numbers change nothing for the rows of their tile"""
    rng = np.random.default_rng(len(sizes) + page)
    hidden = [rng.random(n) < 0.4 for n in sizes]
    hidden[0][0] = hidden[-1][-1] = True

    def change(s):
        for r, h in enumerate(hidden):
            for node in np.nonzero(h)[0]:
                unwritten(s, r, int(node))
    s = Step8(lens, trees_of(rng, sizes), heads, page=page, seed=31, type=type, change=change).to_gpu()
    s.pool8.bytes[s.pool8.bytes == 0x7F] = poison
    s.g_pool8.copy_(dev(s.pool8.bytes))
    s.run_plan()
    up = [(rng.random((n, n)) < 0.6) & ~h for n, h in zip(sizes, hidden)]
    words = np.concatenate([tree_ref.mask_words(u, s.words) for u in up] + [np.zeros((s.max_rows - s.rows, s.words), np.int32)])
    s.g_masks.copy_(dev(words.astype(np.int32)))
    s.attention8()
    s.check(s.result(), up=up)


@pytest.mark.parametrize("bad", [-1, 10 ** 6])
@pytest.mark.parametrize("type", TYPES)
def test_a_bad_entry_that_some_rows_see(type, bad):
    """The rows that see one of its positions are NaN, the others have their answer, whatever the pool's last page holds"""
    tree = [-1, 0, 1, 0, 3, 4, 1]                           # nodes 2 .. 6 lie in the second page; 0 and 1 see nothing of it
    def change(s):
        last = np.full((1, 2, 1) + s.pool.shape[3:], NAN16, dtype=np.uint16).view(np.float16)
        s.pool = np.concatenate([s.pool, last], axis=2)
        s.n_pages += 1
    s = Step8([14, 62, 30], [tree, tree, tree], (4, 2, 64), seed=32, type=type, change=change).to_gpu()
    for r in range(2):
        s.g["table"][r, (s.lens[r] + 2) // s.page] = bad
    s.run_plan().attention8()
    got = s.result()
    s.check(got, requests=[2])
    for r in range(2):
        e, off = s.plain(r, s.up[r])
        g = got[s.starts[r]:s.starts[r] + 7, :256].astype(np.float64).reshape(e.shape)
        sees = s.up[r][:7, 2:7].any(-1)
        assert sees.tolist() == [False, False, True, True, True, True, True]
        assert np.isnan(g[sees]).all()
        assert (np.abs(g[~sees] - e[~sees]) <= np.abs(e[~sees]) * 2.0 ** -11 + 2.0 ** -25 + off[~sees] * (1 + 2.0 ** -11)).all()
