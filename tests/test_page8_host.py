"""A paged cache in 8 bits and sampling: sizes and refusals, host only (no GPU), and the plain forms that the GPU tests compare with."""
import ctypes as C

import numpy as np
import pytest

import paper_2604_23553_amd as cf
from tests import page8_ref
from tests.test_tree_host import PAGES, a_batch, refused


@pytest.mark.parametrize("pages", [PAGES, (1, 16, 1, 64), (1 << 20, 16, 32, 128), (3, 48, 5, 80)])
def test_pool_bytes(pages):
    n, page, heads, d = pages
    assert cf.cfpp_page8_pool_bytes(cf.Pages(*pages)) == 2 * n * page * heads * (d + 2)


@pytest.mark.parametrize("pages", [(0, 64, 4, 80), (4, 40, 4, 80), (4, 64, 4, 96), (4, 64, 1025, 64)])
def test_pool_bytes_of_pages_that_are_none(pages):
    assert cf.cfpp_page8_pool_bytes(cf.Pages(*pages)) == 0


@pytest.mark.parametrize("type", [0, 1, 2, 5, -1])
def test_types_that_are_no_cache(type):
    p, x = cf.Pages(*PAGES), 65536
    assert refused(cf.cfpp_page8_append, p, type, x, x, x, x, 3) == -1
    assert refused(cf.cfpp_page8_read, p, type, x, x, 3, x, x) == -1
    assert refused(cf.cfpp_page8_attention, p, type, x, a_batch(), x, 8, 2 * x) == -1


@pytest.mark.parametrize("type", [cf.TYPE_INT8, cf.TYPE_E4M3])
def test_refusals_of_rows(type):
    p, x = cf.Pages(*PAGES), 65536
    for pool, k, v, slots, n, stride in ((0, x, x, x, 3, None), (x, 0, x, x, 3, None), (x, x, x + 2, x, 3, None), (x + 8, x, x, x, 3, None), (x, x, x, 0, 3, None),
                                         (x, x, x, x + 2, 3, None), (x, x, x, x, -1, None), (x, x, x, x, (1 << 20) + 1, None), (x, x, x, x, 3, 312),
                                         (x, x, x, x, 3, 324), (x, x, x, x, 3, -320), (x, x, x, x, 3, 1 << 33)):
        assert refused(cf.cfpp_page8_append, p, type, pool, k, v, slots, n, stride) == -1
        assert refused(cf.cfpp_page8_read, p, type, pool, slots, n, k, v, stride) == -1
    bad, wide = cf.Pages(4, 64, 4, 96), cf.Pages(64, 16, 64, 128)
    assert refused(cf.cfpp_page8_append, bad, type, x, x, x, x, 3) == -2
    assert refused(cf.cfpp_page8_read, bad, type, x, x, 3, x, x) == -2
    assert refused(cf.cfpp_page8_append, wide, type, x, x, x, x, 1 << 20) == -2
    assert refused(cf.cfpp_page8_read, wide, type, x, x, 1 << 20, x, x) == -2
    cf.cfpp_page8_append(p, type, x, x, x, x, 0)             # nothing to do is no error
    cf.cfpp_page8_read(p, type, x, x, 0, x, x)
    assert cf.lib().cfpp_page8_append(None, type, x, x, x, 320, x, 3, None) == -1


def test_refusals_of_the_attention():
    p, b, x, t = cf.Pages(*PAGES), a_batch(), 65536, cf.TYPE_INT8
    for pool, q, out in ((0, x, 2 * x), (x, 0, 2 * x), (x, x, 0), (x + 8, x, 2 * x), (x, x + 8, 2 * x), (x, x, 2 * x + 8), (x, x, x), (x, x, x + 16)):
        assert refused(cf.cfpp_page8_attention, p, t, pool, b, q, 8, out) == -1
    for strides in (dict(q_stride=644), dict(q_stride=632), dict(out_stride=632), dict(out_stride=-640), dict(q_stride=1 << 33)):
        assert refused(cf.cfpp_page8_attention, p, t, x, b, x, 8, 1 << 40, **strides) == -1
    for change in (dict(masks=0), dict(block_table=0), dict(plan=0), dict(plan=32768 + 16), dict(n_requests=0), dict(max_nodes=257), dict(table_stride=0),
                   dict(lens=0), dict(row_start=2)):
        assert refused(cf.cfpp_page8_attention, p, t, x, a_batch(**change), x, 8, 2 * x) == -1
    assert refused(cf.cfpp_page8_attention, p, t, x, a_batch(plan_bytes=64), x, 8, 2 * x) == -3
    assert refused(cf.cfpp_page8_attention, p, t, x, b, x, 6, 2 * x) == -1
    assert refused(cf.cfpp_page8_attention, p, t, x, b, x, 4 * 257, 2 * x) == -2
    # tiles of 128 query rows are eight sets of 16 to a launch
    big = cf.Pages(64, 16, 256, 64)
    many = a_batch(n_requests=4096, max_rows=1 << 20, max_nodes=256)
    assert cf.cfpp_tree_plan_bytes(big, 256, 4096, 1 << 20, 256) > 0
    assert refused(cf.cfpp_page8_attention, big, t, x, many, x, 256, 1 << 50) == -2


def test_refusals_of_sampling():
    x = 65536
    how = cf.Sampling.of(uniform=x, temperature=x, top_k=x, top_p=x, min_p=x)
    f32 = cf.TYPE_F32
    for args in ((0, f32, 3, 100), (x + 2, f32, 3, 100), (x + 1, cf.TYPE_F16, 3, 100), (x, 0, 3, 100), (x, cf.TYPE_INT8, 3, 100), (x, f32, -1, 100),
                 (x, f32, (1 << 20) + 1, 100), (x, f32, 3, 0)):
        assert refused(cf.cfpp_sample, *args, how, x, x, x) == -1
    assert refused(cf.cfpp_sample, x, f32, 3, (1 << 18) + 1, how, x, x, x) == -2
    for stride in (99, 0, -100, (1 << 32) + 1):
        assert refused(cf.cfpp_sample, x, f32, 3, 100, how, x, x, x, row_stride=stride) == -1
    for name in ("temperature", "top_k", "top_p", "min_p", "uniform"):
        assert refused(cf.cfpp_sample, x, f32, 3, 100, cf.Sampling.of(**{"uniform": x, name: x + 2}), x) == -1
    assert refused(cf.cfpp_sample, x, f32, 3, 100, cf.Sampling.of(uniform=0), x) == -1
    for tokens, probs, kept in ((0, x, x), (x + 2, x, x), (x, x + 2, x), (x, x, x + 2)):
        assert refused(cf.cfpp_sample, x, f32, 3, 100, how, tokens, probs, kept) == -1
    assert cf.lib().cfpp_sample(x, f32, 100, 3, 100, None, x, x, x, None) == -1
    cf.cfpp_sample(x, f32, 0, 100, how, x)                   # no rows
    cf.cfpp_sample(x + 2, cf.TYPE_F16, 0, 100, cf.Sampling.of(uniform=x), x)


def test_the_loop_without_a_context():
    x, how = 65536, cf.Sampling.of(uniform=65536)
    lm = cf.Lm.of(x, x, x, x, 100)
    assert refused(cf.cfpp_lm_sample, 0, lm, x, how, x, x, x) == -1
    assert refused(cf.cfpp_generate_sample_capture, 0, [x], [x], lm, how, x, x, x, x, x, x) == -1
    assert cf.lib().cfpp_generate_sample_capture(None, None, None, None, None, None, None, None, None, None, None) == -1


# ---- the plain forms -------------------------------------------------------------------------
def test_e4m3_by_hand():
    v = page8_ref.E4M3_VALUES
    assert v[0x7E] == 448 and v[0x38] == 1 and v[0x39] == 1.125 and v[0x01] == 2.0 ** -9 and v[0x08] == 2.0 ** -6 and v[0xB8] == -1
    assert np.isnan(v[[0x7F, 0xFF]]).all() and np.isfinite(np.delete(v, [0x7F, 0xFF])).all()


@pytest.mark.parametrize("type", [page8_ref.INT8, page8_ref.E4M3])
def test_codes_are_the_nearest(type):
    rng = np.random.default_rng(type)
    x = (rng.standard_normal((200, 64)) * 10.0 ** rng.integers(-6, 4, (200, 1))).astype(np.float16)
    codes, a = page8_ref.quantise(x, type)
    every = page8_ref.code_values(np.arange(256, dtype=np.uint8), type)
    every = every[np.abs(every) <= page8_ref.MOST[type]]       # (no NaN, and whole numbers of -128 are not used)
    y = page8_ref.MOST[type] * x.astype(np.float64) / a.astype(np.float64)[:, None]
    best = np.abs(y[..., None] - every).min(-1)
    assert np.array_equal(np.abs(y - page8_ref.code_values(codes, type)), best)


def test_codes_by_hand():
    # a = 254: 127 x / 254 = x / 2, so odd x are ties
    codes, a = page8_ref.quantise(np.array([[254, 1, 3, 5, -1, -3, -254, 0]], dtype=np.float16), page8_ref.INT8)
    assert list(codes.view(np.int8)[0]) == [127, 0, 2, 2, 0, -2, -127, 0] and a[0] == 254
    codes, a = page8_ref.quantise(np.array([[448, 17, 19, -17, 2.0 ** -10, 3 * 2.0 ** -10, 0, 1]], dtype=np.float16), page8_ref.E4M3)
    assert list(page8_ref.code_values(codes, page8_ref.E4M3)[0]) == [448, 16, 20, -16, 0, 2.0 ** -8, 0, 1] and a[0] == 448
    for bad in (np.inf, np.nan):
        codes, a = page8_ref.quantise(np.array([[1, bad]], dtype=np.float16), page8_ref.INT8)
        assert np.isnan(a[0]) and not codes.any()
    codes, a = page8_ref.quantise(np.zeros((1, 4), dtype=np.float16), page8_ref.E4M3)
    assert a[0] == 0 and not codes.any()


@pytest.mark.parametrize("type", [page8_ref.INT8, page8_ref.E4M3])
def test_pool_gives_back_what_was_put(type):
    rng = np.random.default_rng(1)
    pool = page8_ref.Pool(3, 32, 2, 80, type)
    rows = rng.standard_normal((2, 96, 2, 80)).astype(np.float16)
    for s in rng.permutation(96):
        pool.put(int(s), rows[0, s], rows[1, s])
    step = {page8_ref.INT8: 1 / 254, page8_ref.E4M3: 2.0 ** -4}[type]
    for s in range(96):
        want = rows[:, s].astype(np.float64)
        assert (np.abs(pool.get(s) - want) <= step * np.abs(want).max(-1, keepdims=True) * (1 + 1e-12)).all()


def test_plain_sampling_by_hand():
    x = np.log(np.array([1.0, 4.0, 2.0, 2.0, 1.0]))
    # the order: 1, 2, 3, 0, 4 with 4, 2, 2, 1, 1 of 10
    for u, token, p in ((0.0, 1, 0.4), (0.39, 1, 0.4), (0.41, 2, 0.2), (0.61, 3, 0.2), (0.81, 0, 0.1), (0.95, 4, 0.1)):
        r = page8_ref.sample(x, uniform=u)
        assert r["token"] == token and abs(r["prob"] - p) < 1e-9 and r["kept"] == 5
    assert page8_ref.sample(x, top_k=2, uniform=0.9)["token"] == 2
    assert page8_ref.sample(x, top_p=0.5, uniform=0.0)["kept"] == 2
    assert page8_ref.sample(x, top_k=2, top_p=0.5, uniform=0.0)["kept"] == 1     # 4 of 6
    assert page8_ref.sample(x, min_p=0.45, uniform=0.99)["kept"] == 3
    assert page8_ref.sample(x, temperature=0.0, uniform=0.9)["token"] == 1
    assert page8_ref.sample(np.array([np.nan, -np.inf]), uniform=0.5)["token"] == -1
    r = page8_ref.sample(np.array([1.0, np.inf, 3.0, np.inf]), uniform=0.75)
    assert r["token"] == 3 and r["kept"] == 2 and r["prob"] == 0.5
