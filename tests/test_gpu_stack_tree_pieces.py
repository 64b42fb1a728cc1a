"""cfpp_stack_tree behind contexts that are cut into pieces and with values that are not finite, against the CPU oracle, one decode step per node along
every path; requests and positions that it does not serve."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2604_23553_amd as cf
import synth
from tests import tree_ref
from tests.parity import assert_block_close
from tests.test_gpu_stack_tree import H512, H1024, H1280, Model, check_step, dev, i32

pytestmark = pytest.mark.gpu


def fill_cache(m, lens, seed, change):
    """Model.fill_cache, then change(layer, request, K, V) of every layer's and request's rows, K and V [H, len, d]; the rows go to their slots once more."""
    kvs, table, H, d = m.fill_cache(lens, seed), m.table.cpu().numpy(), m.shape.n_heads, m.shape.head_dim
    for l, pool in enumerate(m.pools):
        for r, (K, V) in enumerate(kvs[l]):
            change(l, r, K, V)
            t = np.arange(lens[r])
            k, v = (dev(x.transpose(1, 0, 2)) for x in (K, V))
            cf.cfpp_page_append(m.pages, pool, k, v, i32(table[r, t // m.page] * m.page + t % m.page), lens[r], H * d, torch.cuda.current_stream().cuda_stream)
            torch.cuda.synchronize()
    return kvs


def steps_along_paths(orc, m, kvs, lens, X):
    """{(request, node): the oracle's output}, X: a row for each node in the requests' order."""
    H, d, L = m.shape.n_heads, m.shape.head_dim, m.shape.n_layers
    want, a = {}, 0
    for r, parents in enumerate(m.trees):
        for leaf in sorted(range(len(parents)), key=lambda i: -i):
            if (r, leaf) in want:
                continue
            path = [leaf]
            while 0 <= parents[path[-1]] < path[-1]:
                path.append(parents[path[-1]])
            path.reverse()
            Ks, Vs = [], []
            for l in range(L):
                K, V = (np.zeros((H, lens[r] + len(path), d), dtype=np.float16) for _ in range(2))
                K[:, :lens[r]], V[:, :lens[r]] = kvs[l][r]
                Ks.append(K)
                Vs.append(V)
            out, _ = orc.prefill(m.shape, m.ws, Ks, Vs, lens[r], X[a + np.array(path)])
            for j, i in enumerate(path):
                want[r, i] = out[j]
        a += len(parents)
    return want


def levels(layer, r, K, V):
    """Every 32 cached positions' V have a level of their own in all dimensions: a piece of 128 positions that is left out moves the outputs by ten times the
    tolerance at least."""
    rng = np.random.default_rng([layer, r])
    V += (6.0 * rng.standard_normal((V.shape[1] + 31) // 32)).repeat(32)[:V.shape[1], None].astype(np.float16)


# (more than 256 positions are cut into pieces; tiles of 16, 32, 64 and 128 query rows, each with the products of few rows and of many)
@pytest.mark.parametrize("shape,lens,sizes,spare", [
    (H512, [700], [1], 2), (H512, [1300, 30, 600], [9, 2, 16], 3), (H1280, [1100], [26], 1), (H512, [900, 1500], [26, 5], 200), (H1024, [1000], [40], 2),
    (H512, [700, 900], [12, 64], 100), (H1024, [500], [70], 1), (H512, [1200, 10], [100, 30], 2), (H1280, [800], [1], 300),
])
def test_stack_tree_in_pieces(orc, shape, lens, sizes, spare):
    rng = np.random.default_rng([shape.hidden, sum(sizes), 1])
    n_pages = sum(tree_ref.pages_for(a + b, 16) for a, b in zip(lens, sizes)) + 2
    print(f"[case] {shape.name} lens={lens} sizes={sizes} spare={spare}", flush=True)
    m = Model(shape, len(lens), 16, n_pages, sum(sizes) + spare, max(sizes), 3, max_seq=2048)
    try:
        kvs = fill_cache(m, lens, 5, levels)
        m.set_trees([tree_ref.random_tree(rng, n) for n in sizes])
        X = synth.x_input(shape, 11, batch=sum(sizes))
        m.x[:sum(sizes)] = dev(X)
        m.enqueue_tables()
        m.enqueue_stack()
        torch.cuda.synchronize()
        cf.cfpp_device_error(m.ctx)
        first = m.out.cpu().numpy()
        check_step(orc, m, kvs, lens, X, first)
        m.enqueue_tables()
        m.enqueue_stack()
        torch.cuda.synchronize()
        assert np.array_equal(first.view(np.uint16), m.out.cpu().numpy().view(np.uint16)), "the bits change from call to call"
    finally:
        m.close()


@pytest.mark.parametrize("lens,sizes", [([500, 40], [13, 5]), ([300, 700], [8, 30]), ([900], [60]), ([400], [100])])
def test_stack_tree_of_values_that_are_not_finite(orc, lens, sizes):
    """A cached key that is infinite (no number for the nodes whose query is positive there, no weight for the others), and a node whose input is no number:
    its descendants have none either, nodes that do not see it are as ever."""
    shape, L = H512, H512.n_layers
    rng = np.random.default_rng(sum(sizes))
    n_pages = sum(tree_ref.pages_for(a + b, 16) for a, b in zip(lens, sizes)) + 2
    m = Model(shape, len(lens), 16, n_pages, sum(sizes) + 3, max(sizes), 3, max_seq=2048)
    try:
        def change(layer, r, K, V):
            if layer == L - 1 and r == 0:                  # (the last layer's: no other node's K and V come from what it leaves)
                K[1, lens[0] * 2 // 3, 40] = np.inf
        kvs = fill_cache(m, lens, 5, change)
        m.set_trees([tree_ref.random_tree(rng, n) for n in sizes])
        X = synth.x_input(shape, 11, batch=sum(sizes))
        X[sizes[0] // 2] = np.nan
        m.x[:sum(sizes)] = dev(X)
        m.enqueue_tables()
        m.enqueue_stack()
        torch.cuda.synchronize()
        cf.cfpp_device_error(m.ctx)
        want, got, starts = steps_along_paths(orc, m, kvs, lens, X), m.out.cpu().numpy(), m.row_start.cpu().numpy()
        kinds = [0, 0]
        for (r, i), w in want.items():
            g = got[starts[r] + i]
            if np.isfinite(w).all():
                assert_block_close(g, w, f"request {r}, node {i}")
                kinds[r == 0] += 1
            else:
                assert np.isnan(w).all() and np.isnan(g).all(), f"request {r}, node {i}"
        assert 1 < kinds[1] < sizes[0] - 1
    finally:
        m.close()


@pytest.mark.parametrize("max_rows", [8, 300])
def test_far_positions_without_rotary_dimensions(orc, max_rows):
    """A position outside [0, max_seq) raises the flag whatever the rotation."""
    shape = synth.ModelShape(512, 8, 64, 0, 2048, n_layers=2, name="neox-h512-r0")
    m = Model(shape, 1, 16, 5, max_rows, 4, 3, max_seq=64)
    try:
        kvs = m.fill_cache([30], 6)
        m.set_trees([[-1, 0, 0, 2]])
        X = synth.x_input(shape, 13, batch=4)
        m.x[:4] = dev(X)
        m.enqueue_tables()
        m.enqueue_stack()
        torch.cuda.synchronize()
        cf.cfpp_device_error(m.ctx)
        check_step(orc, m, kvs, [30], X, m.out.cpu().numpy())
        for position in (64, -1):
            m.positions[3] = position
            m.enqueue_stack()
            with pytest.raises(cf.CfppError) as e:
                cf.cfpp_device_error(m.ctx)
            assert e.value.status == -6
        m.positions[3] = 63
        m.enqueue_stack()
        cf.cfpp_device_error(m.ctx)
    finally:
        m.close()


@pytest.mark.parametrize("max_rows", [40, 300])
def test_requests_that_the_plan_leaves_out(orc, max_rows):
    """A request of more than max_nodes nodes has pages and slots, but no masks and positions: its outputs and its slots stay as they were, its positions, of
    whatever step, raise no flag, and the others are served.  A plan of other sizes serves nobody."""
    shape, lens = H512, [20, 5, 10]
    m = Model(shape, 3, 16, 6, max_rows, 12, 3, max_seq=64)
    try:
        kvs = m.fill_cache(lens, 6)
        rng = np.random.default_rng(9)
        m.set_trees([tree_ref.random_tree(rng, n) for n in (12, 14, 5)])
        X = synth.x_input(shape, 13, batch=31)
        m.x[:31] = dev(X)
        m.positions.fill_(10 ** 6)
        m.enqueue_tables()
        m.enqueue_stack()
        torch.cuda.synchronize()
        assert (m.granted == 1).all() and (m.slots[:31] >= 0).all()
        cf.cfpp_device_error(m.ctx)
        got, slots = m.out.cpu().numpy(), m.slots.cpu().numpy()
        assert (got[12:26] == 7.0).all()
        for l in range(shape.n_layers):
            assert all(np.isnan(m.row(l, int(slot))).all() for slot in slots[12:26])
        m.trees[1] = []
        check_step(orc, m, kvs, lens, X, got)
        before = [p.clone() for p in m.pools]
        m.batch.max_nodes = 11
        m.out.fill_(7.0)
        m.enqueue_stack()
        torch.cuda.synchronize()
        cf.cfpp_device_error(m.ctx)
        assert (m.out == 7.0).all()
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(before, m.pools))
    finally:
        m.close()
