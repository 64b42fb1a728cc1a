"""Drafted trees over a paged cache: sizes and refusals, host only (no GPU), and the plain forms that the GPU tests compare with."""
import ctypes as C

import numpy as np
import pytest

import paper_2604_23553_amd as cf
from tests import tree_ref

PAGES = (16, 64, 4, 80)                                    # pages, positions to one, heads, head size


def a_batch(**change):
    """A batch whose pointers are stand-ins: no call below gets as far as using one."""
    fields = dict(n_requests=3, max_rows=20, max_nodes=8, table_stride=4, lens=4096, row_start=8192, block_table=12288, slots=16384,
                  parents=20480, masks=24576, positions=28672, plan=32768, plan_bytes=1 << 40)
    fields.update(change)
    b = cf.TreeBatch()
    for n, v in fields.items():
        setattr(b, n, v)
    return b


def refused(call, *args, **more):
    with pytest.raises(cf.CfppError) as e:
        call(*args, **more)
    return e.value.status


@pytest.mark.parametrize("pages,status", [
    (PAGES, 0), ((1, 16, 1, 64), 0), ((1 << 20, 16, 32, 128), 0), ((0, 64, 4, 80), -1), ((4, 0, 4, 80), -1), ((4, 64, 0, 80), -1),
    ((4, 64, 4, 0), -1), ((1 << 27, 16, 1, 64), -1), ((4, 40, 4, 80), -2), ((4, 8, 4, 80), -2), ((4, 64, 4, 96), -2), ((4, 64, 1025, 64), -2),
    ((2, (1 << 20) + 16, 1, 64), -2), ((2, 1 << 20, 1, 64), 0),
])
def test_pages(pages, status):
    p = cf.Pages(*pages)
    assert cf.cfpp_validate_pages(p) == status
    assert cf.cfpp_page_pool_bytes(p) == (2 * 2 * np.prod(np.array(pages, dtype=np.int64)) if status == 0 else 0)


def test_pool_is_a_kv_layer_whose_sequences_are_pages():
    cfg = cf.Config(2560, 32, 80, 20, 10240, 1, 64, 7, 10000.0, 1e-5, 0)
    assert cf.cfpp_page_pool_bytes(cf.Pages(7, 64, 32, 80)) == cf.cfpp_kv_layer_bytes(cfg)


def test_plan_bytes():
    p = cf.Pages(*PAGES)
    assert cf.cfpp_tree_plan_bytes(p, 8, 3, 20, 8) > 0
    assert cf.cfpp_tree_plan_bytes(p, 4, 4096, 1 << 20, 256) > 0
    for heads, requests, rows, nodes in ((6, 3, 20, 8), (0, 3, 20, 8), (4 * 257, 3, 20, 8), (8, 0, 20, 8), (8, 4097, 20, 8), (8, 3, 0, 8),
                                         (8, 3, (1 << 20) + 1, 8), (8, 3, 20, 0), (8, 3, 20, 257)):
        assert cf.cfpp_tree_plan_bytes(p, heads, requests, rows, nodes) == 0
    assert cf.cfpp_tree_plan_bytes(cf.Pages(4, 40, 4, 80), 8, 3, 20, 8) == 0


@pytest.mark.parametrize("change", [dict(n_requests=0), dict(n_requests=4097), dict(max_rows=0), dict(max_rows=(1 << 20) + 1), dict(max_nodes=0),
                                    dict(max_nodes=257), dict(table_stride=0), dict(table_stride=1 << 26), dict(table_stride=(1 << 24) + 1), dict(lens=0), dict(lens=4098),
                                    dict(row_start=0)])
def test_batches_that_no_call_takes(change):
    p, b, x = cf.Pages(*PAGES), a_batch(**change), 65536
    assert refused(cf.cfpp_page_tables, p, b, x, x, x, x, x) == -1
    assert refused(cf.cfpp_tree_plan, p, b, 8) == -1
    assert refused(cf.cfpp_tree_attention, p, x, b, x, 8, 2 * x) == -1
    assert refused(cf.cfpp_tree_accept, p, [x], b, x, x, x, x, x, x) == -1


def test_refusals_of_each_call():
    p, b, x = cf.Pages(*PAGES), a_batch(), 65536
    bad = cf.Pages(4, 64, 4, 96)
    for k in range(5):
        args = [x] * 5
        args[k] = 0 if k % 2 else 65538
        assert refused(cf.cfpp_page_tables, p, b, *args) == -1
    for name in ("block_table", "slots"):
        assert refused(cf.cfpp_page_tables, p, a_batch(**{name: 0}), x, x, x, x, x) == -1
    for name in ("masks", "parents", "positions", "plan"):
        assert refused(cf.cfpp_tree_plan, p, a_batch(**{name: 0}), 8) == -1
    assert refused(cf.cfpp_tree_plan, p, a_batch(slots=2), 8) == -1
    assert refused(cf.cfpp_tree_plan, p, a_batch(plan=32768 + 16), 8) == -1
    assert refused(cf.cfpp_tree_plan, p, a_batch(plan_bytes=cf.cfpp_tree_plan_bytes(p, 8, 3, 20, 8) - 1), 8) == -3
    assert refused(cf.cfpp_tree_plan, p, b, 6) == -1
    assert refused(cf.cfpp_tree_plan, p, b, 4 * 257) == -2
    assert refused(cf.cfpp_tree_plan, bad, b, 8) == -2
    for pool, q, out in ((0, x, 2 * x), (x, 0, 2 * x), (x, x, 0), (x + 8, x, 2 * x), (x, x + 8, 2 * x), (x, x, 2 * x + 8), (x, x, x), (x, x, x + 16)):
        assert refused(cf.cfpp_tree_attention, p, pool, b, q, 8, out) == -1
    for strides in (dict(q_stride=644), dict(q_stride=632), dict(out_stride=632), dict(out_stride=-640), dict(q_stride=1 << 33)):
        assert refused(cf.cfpp_tree_attention, p, x, b, x, 8, 1 << 40, **strides) == -1
    for name in ("masks", "block_table", "plan"):
        assert refused(cf.cfpp_tree_attention, p, x, a_batch(**{name: 0}), x, 8, 2 * x) == -1
    assert refused(cf.cfpp_tree_attention, p, x, a_batch(plan_bytes=64), x, 8, 2 * x) == -3
    for pool, k, v, slots, n, stride in ((0, x, x, x, 3, None), (x, 0, x, x, 3, None), (x, x, x + 2, x, 3, None), (x, x, x, 0, 3, None),
                                         (x, x, x, x, -1, None), (x, x, x, x, 3, 312), (x, x, x, x, 3, 324), (x, x, x, x, 3, -320)):
        assert refused(cf.cfpp_page_append, p, pool, k, v, slots, n, stride) == -1
    assert refused(cf.cfpp_page_append, bad, x, x, x, x, 3) == -2
    for k in range(6):
        args = [x] * 6
        args[k] = 65538 if k % 2 else 0
        assert refused(cf.cfpp_tree_accept, p, [x], b, *args) == -1
    assert refused(cf.cfpp_tree_accept, p, [x, 0], b, *[x] * 6) == -1
    assert refused(cf.cfpp_tree_accept, p, [x] * 65, b, *[x] * 6) == -1
    for name in ("slots", "parents"):
        assert refused(cf.cfpp_tree_accept, p, [x], a_batch(**{name: 0}), *[x] * 6) == -1
    assert cf.lib().cfpp_page_append(None, C.c_void_p(x), C.c_void_p(x), C.c_void_p(x), C.c_int64(320), C.c_void_p(x), 3, None) == -1
    assert cf.lib().cfpp_tree_plan(C.byref(p), None, 8, None) == -1


def test_the_stack_without_a_context():
    cfg = cf.Config(512, 8, 64, 16, 2048, 1, 64, 1, 10000.0, 1e-5, 0)
    assert refused(cf.cfpp_stack_tree, 0, [65536], [65536], cf.Pages(4, 16, 8, 64), a_batch(), 65536, 1 << 20, 1 << 21, 1 << 30) == -1
    assert cf.cfpp_tree_scratch_bytes(cfg, 0) == 0 and cf.cfpp_tree_scratch_bytes(cfg, 4097) == 0
    assert cf.cfpp_tree_scratch_bytes(cfg, 1) == cf.cfpp_tree_scratch_bytes(cfg, 128) > cf.cfpp_prefill_scratch_bytes(cfg, 128)


def test_nothing_to_append_is_no_error():
    cf.cfpp_page_append(cf.Pages(*PAGES), 65536, 65536, 65536, 65536, 0)


# ---- the plain forms -------------------------------------------------------------------------
def test_plain_attention_against_a_softmax():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((2, 4, 64)), rng.standard_normal((9, 2, 64)), rng.standard_normal((9, 2, 64))
    seen = np.ones((2, 9), dtype=bool)
    seen[1, 4:] = False
    got, off = tree_ref.attend(q, k, v, seen)
    for i, S in ((0, 9), (1, 4)):
        for h in range(4):
            e = np.exp(k[:S, h // 2] @ q[i, h] / 8.0)
            assert np.allclose(got[i, h], (e / e.sum()) @ v[:S, h // 2], atol=1e-13)
    assert (off > 0).all() and off.max() < 1e-3
    assert not tree_ref.attend(q, k, v, np.zeros((2, 9), dtype=bool))[0].any()


def test_plain_tree_by_hand():
    up = tree_ref.ancestors([-1, 0, 0, 1, 3, 2, -1])
    assert [list(np.nonzero(u)[0]) for u in up] == [[0], [0, 1], [0, 2], [0, 1, 3], [0, 1, 3, 4], [0, 2, 5], [6]]
    assert list(tree_ref.mask_words(up, 1)[:, 0]) == [1, 3, 5, 11, 27, 37, 64]
    assert tree_ref.accept([-1, 0, 0, 1, 3, 2, -1], [5, 9, 7, 4, 3, 8, 9], [7, 4, 8, 3, 1, 2, 0]) == [0, 2, 5]
    assert tree_ref.accept([-1, 0, 0, 0], [5, 9, 7, 7], [7, 1, 1, 1]) == [0, 2]


def test_plain_allocator_by_hand():
    a = tree_ref.Allocator(4, 16, 2, 3, np.random.default_rng(0))
    a.free = [10, 11, 12, 13]
    granted, starts, slots = a.step([0, 0], [17, 3], 24)
    assert granted == [1, 1] and starts == [0, 17, 20] and a.tables == [[13, 12], [11]] and a.free == [10]
    assert slots[16] == 12 * 16 and slots[17] == 11 * 16 and list(slots[20:]) == [-1] * 4
    granted, starts, slots = a.step([0, 20], [0, 30], 24)            # 50 positions are four pages: the table is too short
    assert granted == [1, 0] and a.tables == [[], [11]] and a.free == [10, 13, 12]


def test_launches_of_2_32_threads_are_refused():
    p, x = cf.Pages(64, 16, 256, 64), 65536
    b = a_batch(n_requests=4096, max_rows=1 << 20, max_nodes=256)
    assert cf.cfpp_tree_plan_bytes(p, 256, 4096, 1 << 20, 256) > 0                     # 16384 tiles, 256 key heads
    for heads, rows in ((256 * 16, 1 << 20), (256 * 256, 1 << 20), (256 * 256, 1 << 16)):
        assert cf.cfpp_tree_plan_bytes(p, heads, 4096, rows, 256) == 0
        b.max_rows = rows
        assert refused(cf.cfpp_tree_plan, p, b, heads) == -2
        assert refused(cf.cfpp_tree_attention, p, x, b, x, heads, 1 << 50) == -2
    wide = cf.Pages(64, 16, 64, 128)
    assert refused(cf.cfpp_page_append, wide, x, x, x, x, 1 << 20) == -2
