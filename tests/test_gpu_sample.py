"""Sampling on the GPU against its plain form in 64 bits, and a server's step on a cache in 8 bits."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2604_23553_amd as cf
from tests import page8_ref
from tests.test_gpu_tree import dev, i32, stream

pytestmark = pytest.mark.gpu


def f32(a):
    return dev(np.asarray(a, dtype=np.float32))


def draw(logits, temperature=None, top_k=None, top_p=None, min_p=None, uniform=None, stride=None, offset=0):
    """[(token, prob, kept)] of each row; offset: logits in front of the first row"""
    n, vocab = logits.shape
    stride = vocab if stride is None else stride
    flat = np.full(offset + n * stride, np.nan, dtype=logits.dtype)
    for r in range(n):
        flat[offset + r * stride:offset + r * stride + vocab] = logits[r]
    x = dev(flat)
    how = {k: v for k, v in dict(temperature=temperature, top_p=top_p, min_p=min_p, uniform=uniform).items() if v is not None}
    g = {k: f32(np.broadcast_to(v, n)) for k, v in how.items()}
    if top_k is not None:
        g["top_k"] = i32(np.broadcast_to(top_k, n))
    tokens, kept, probs = i32([-7] * n), i32([-7] * n), f32([-7] * n)
    type = cf.TYPE_F16 if logits.dtype == np.float16 else cf.TYPE_F32
    cf.cfpp_sample(x.data_ptr() + offset * logits.itemsize, type, n, vocab, cf.Sampling.of(**g), tokens, probs, kept, stride, stream())
    torch.cuda.synchronize()
    return list(zip(tokens.cpu().numpy().tolist(), probs.cpu().numpy().tolist(), kept.cpu().numpy().tolist()))


def check(logits, **how):
    got = draw(logits, **how)
    for n in ("stride", "offset"):
        how.pop(n, None)
    for r in range(len(logits)):
        one = {k: (int if k == "top_k" else float)(np.broadcast_to(v, len(logits))[r]) for k, v in how.items()}
        page8_ref.check_sample(logits[r], got[r], **one)
    return got


def model_logits(rng, n, vocab, dtype=np.float32):
    x = 2.5 * rng.standard_normal((n, vocab))
    for r in range(n):
        x[r, rng.integers(0, vocab, 12)] += 9.0
    return x.astype(dtype)


@pytest.mark.parametrize("dtype", [np.float32, np.float16])
@pytest.mark.parametrize("vocab", [1, 2, 3, 5, 63, 64, 65, 255, 1023, 4095, 4096, 4097, 12289, 50304, 131071])
def test_sizes(vocab, dtype):
    rng = np.random.default_rng(vocab)
    n = 24
    x = model_logits(rng, n, vocab, dtype)
    check(x, temperature=rng.choice([0.0, 0.3, 0.8, 1.0, 2.0], n), top_k=rng.choice([0, 1, 2, 5, 50, 400, vocab - 1, vocab, vocab + 1], n),
          top_p=rng.choice([0.1, 0.5, 0.9, 0.99, 1.0], n), min_p=rng.choice([0.0, 0.01, 0.1, 0.5], n), uniform=rng.random(n, dtype=np.float32),
          stride=vocab + 3, offset=1)


@pytest.mark.parametrize("how", [dict(), dict(temperature=0.7), dict(top_k=40), dict(top_p=0.9), dict(min_p=0.05), dict(top_k=1000, top_p=0.95), dict(top_k=7, min_p=0.2),
                                 dict(top_p=0.8, min_p=0.02), dict(top_k=300, top_p=0.7, min_p=0.001, temperature=1.5), dict(top_k=30000), dict(top_p=0.999, temperature=3.0)])
def test_filters(how):
    rng = np.random.default_rng(17)
    u = np.concatenate([[0.0, 2.0 ** -24, 0.5, 1 - 2.0 ** -24], rng.random(36, dtype=np.float32)])
    check(model_logits(rng, 40, 50304), uniform=u, **how)


def test_filters_that_are_not_given_or_keep_all():
    rng = np.random.default_rng(3)
    x, u = model_logits(rng, 30, 3000), rng.random(30, dtype=np.float32)
    plain = draw(x, uniform=u)
    for how in (dict(temperature=1.0), dict(top_k=0), dict(top_k=-5), dict(top_k=3000), dict(top_k=2 ** 31 - 1), dict(top_p=1.0), dict(top_p=7.0), dict(top_p=np.nan),
                dict(min_p=0.0), dict(min_p=-1.0), dict(min_p=np.nan)):
        assert draw(x, uniform=u, **how) == plain, how


def test_filters_that_leave_the_first():
    rng = np.random.default_rng(4)
    x, u = model_logits(rng, 30, 3000), rng.random(30, dtype=np.float32)
    first = [(int(i), 1.0, 1) for i in x.argmax(-1)]
    for how in (dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=np.nan), dict(top_k=1), dict(top_p=0.0), dict(top_p=-2.0), dict(min_p=1.0),
                dict(min_p=5.0), dict(top_p=1e-30), dict(temperature=1e-30)):
        got = draw(x, uniform=u, **how)
        if "temperature" in how and how["temperature"] > 0:
            got = [(t, p, 1) for t, p, _ in got]
        assert got == first, how


@pytest.mark.parametrize("dtype", [np.float32, np.float16])
def test_equal_logits(dtype):
    """Ties go by the index: whole rows of one value, a few values, and ties in the place where a filter ends"""
    rng = np.random.default_rng(5)
    n, vocab = 20, 9000
    u = rng.random(n, dtype=np.float32)
    x = np.full((n, vocab), -1.25, dtype=dtype)
    got = check(x, uniform=u)
    assert [t for t, _, _ in got] == [int(np.floor(float(v) * vocab)) for v in u]
    got = check(x, uniform=u, top_k=4321)
    assert [t for t, _, _ in got] == [int(np.floor(float(v) * 4321)) for v in u]
    check(x, uniform=u, top_p=0.37)
    x = rng.choice(np.array([0.0, 1.0, 1.5, -0.0], dtype=dtype), (n, vocab))
    check(x, uniform=u)
    check(x, uniform=u, top_k=rng.integers(2, vocab, n))
    check(x, uniform=u, top_p=rng.random(n, dtype=np.float32) * np.float32(0.98) + np.float32(0.01), top_k=rng.integers(2, vocab, n))


def test_logits_of_all_sizes():
    """Values that stand apart by more than the histogram reaches, so that most of a row falls into one bin"""
    rng = np.random.default_rng(6)
    n, vocab = 30, 20000
    u = rng.random(n, dtype=np.float32)
    x = rng.standard_normal((n, vocab)).astype(np.float32)
    x[:10, 77] = 1e30
    x[10:20] *= 1e4
    x[20:] *= 1e-30
    for how in (dict(), dict(top_k=3000), dict(top_k=15000, top_p=0.5), dict(top_p=0.9), dict(temperature=1e-6), dict(temperature=1e30), dict(temperature=np.inf),
                dict(temperature=1e-40), dict(min_p=0.3), dict(top_k=5000, temperature=1e4)):
        check(x, uniform=u, **how)


@pytest.mark.parametrize("dtype", [np.float32, np.float16])
def test_logits_that_are_no_numbers_or_infinite(dtype):
    rng = np.random.default_rng(7)
    n, vocab = 12, 5000
    x = model_logits(rng, n, vocab, dtype)
    x[0, ::2] = np.nan
    x[1, 10:] = -np.inf
    x[2] = -np.inf
    x[3] = np.nan
    x[4, [5, 4000, 4999]] = np.inf
    x[5, 17] = np.inf
    x[5, 3:9] = np.nan
    x[6, :-1] = -np.inf
    x[7] = np.finfo(dtype).min
    x[8, 1:] = np.finfo(dtype).min
    x[9, ::3] = np.finfo(dtype).max
    u = rng.random(n, dtype=np.float32)
    for how in (dict(), dict(top_k=3), dict(top_p=0.6), dict(temperature=0.0), dict(top_k=100, top_p=0.9, min_p=0.1), dict(temperature=0.5)):
        got = check(x, uniform=u, **how)
        assert got[2] == got[3] == (-1, 0.0, 0) and got[6][0] == vocab - 1


@pytest.mark.parametrize("dtype", [np.float32, np.float16])
@pytest.mark.parametrize("vocab", [1, 2, 3, 4, 5])
def test_few_logits_far_from_zero(vocab, dtype):
    rng = np.random.default_rng(vocab)
    n = 24
    x = (np.repeat([-1e4, -100.0, -30.0, 30.0, 100.0, 1e4], 4)[:, None] + np.round(2 * rng.standard_normal((n, vocab)), 1)).astype(dtype)
    u = rng.random(n, dtype=np.float32)
    for how in (dict(), dict(temperature=3.0), dict(top_k=2), dict(top_p=0.7), dict(min_p=0.2), dict(top_k=2, top_p=0.9, min_p=0.01)):
        check(x, uniform=u, **how)


@pytest.mark.parametrize("dtype", [np.float32, np.float16])
@pytest.mark.parametrize("first", [-np.inf, np.nan, -3e4, -60.0])
def test_a_beginning_that_is_masked_or_far_below(first, dtype):
    """The first 17000 logits, and all but the last 300, in rows whose others stand about a value from far below zero to far above it"""
    rng = np.random.default_rng(31)
    n, vocab = 24, 20000
    about = np.repeat([-2000.0, -100.0, -18.0, -0.5, 25.0, 1000.0], 4)
    x = (about[:, None] + 2.0 * rng.standard_normal((n, vocab))).astype(dtype)
    for r in range(n):
        x[r, :17000 if r % 2 else vocab - 300] = first
    u = rng.random(n, dtype=np.float32)
    for how in (dict(), dict(top_k=40), dict(top_k=600), dict(top_p=0.9), dict(min_p=0.05), dict(top_k=600, top_p=0.8, min_p=0.01), dict(temperature=0.3), dict(temperature=4.0)):
        check(x, uniform=u, **how)


@pytest.mark.parametrize("min_p", [1e-40, 2.0 ** -70, 1e-15, 2.0 ** -47.5, 1e-6, 0.01, 0.3, 0.9])
def test_min_p_with_the_others(min_p):
    """Least weights from below what a sum notices to near the largest, before and behind the place where top-k or top-p ends"""
    rng = np.random.default_rng(41)
    n, vocab = 24, 30000
    x = model_logits(rng, n, vocab)
    x[8:16] *= 12.0                                        # weights down to 2^-150 of the largest
    x[16:] = np.round(x[16:])
    u = rng.random(n, dtype=np.float32)
    for how in (dict(), dict(top_k=600), dict(top_k=25000), dict(top_p=0.6), dict(top_p=1 - 2.0 ** -24), dict(top_k=600, top_p=0.99), dict(top_k=100), dict(temperature=0.2)):
        check(x, uniform=u, min_p=min_p, **how)


@pytest.mark.parametrize("left", [100, 511, 600, 5000])
def test_top_k_of_about_as_many_as_there_are(left):
    """k below, at and above the number of logits that are numbers; ties where it ends"""
    rng = np.random.default_rng(left)
    n, vocab = 16, 9000
    x = np.full((n, vocab), -np.inf, dtype=np.float32)
    for r in range(n):
        at = rng.permutation(vocab)[:left]
        x[r, at] = np.round(3.0 * rng.standard_normal(left), 1 if r % 2 else 4)
        x[r, rng.permutation(vocab)[:50]] = np.nan
    u = rng.random(n, dtype=np.float32)
    for k in (left - 80, left - 51, left, left + 1, 448, 449, 512, 513):
        for how in (dict(), dict(top_p=0.8), dict(min_p=0.01), dict(top_p=0.999, min_p=1e-4)):
            check(x, uniform=u, top_k=k, **how)


@pytest.mark.parametrize("how", [dict(), dict(top_k=300), dict(top_k=4000), dict(top_p=1 - 2.0 ** -24)])
def test_probabilities_of_rare_tokens(how):
    """Drawn by random numbers next to 1 behind a few tokens that have nearly all of the weight: they are as precise as those of the likely ones"""
    rng = np.random.default_rng(61)
    n, vocab = 30, 19253
    x = (2.0 * rng.standard_normal((n, vocab))).astype(np.float32)
    x[:, 5000] = np.linspace(10, 25, n)
    got = check(x, uniform=1 - 2.0 ** -24, **how)
    for r, (token, prob, kept) in enumerate(got):
        p = page8_ref.sample(x[r], **how)
        at = int(np.nonzero(p["order"] == token)[0][0])
        # the weight 2^-41 off, the sum 2^-39, the quotient rounded to fp32
        want = p["w"][at] / p["sums"][kept - 1]
        assert abs(prob - want) <= want * (2.0 ** -24 + 2.0 ** -38), (r, prob, want)
    # (that the inputs are what the test is about: the 300th of so many is near 2 * 2.16, and exp(4.3 - 25) is 2^-29.9)
    assert min(g[1] for g in got) < 2.0 ** -29


FILTERS = [dict(), dict(top_k=30), dict(top_k=600), dict(top_p=0.8), dict(min_p=0.03), dict(top_k=600, top_p=0.9, min_p=0.01)]


@pytest.mark.parametrize("temperature", [4e-36, 1e-37, 1e-40, 2.0 ** -149])
@pytest.mark.parametrize("vocab", [3, 300, 20000])
def test_temperatures_next_to_zero(vocab, temperature):
    """Logits as far apart as the temperature is large, down to the smallest positive number, alone and behind others that are far below"""
    rng = np.random.default_rng(vocab)
    n = 24
    t = np.float32(temperature)
    x = (3.0 * rng.standard_normal((n, vocab)) * np.float64(t)).astype(np.float32)
    x[8:] -= x[8:].max(-1, keepdims=True)                   # the largest is 0
    x[12:16, :vocab * 4 // 5] = -1e30
    x[16:20, :vocab * 4 // 5] = np.finfo(np.float32).min
    x[20:, ::2] = -np.inf
    u = rng.random(n, dtype=np.float32)
    for how in FILTERS:
        check(x, uniform=u, temperature=t, **how)


@pytest.mark.parametrize("temperature", [1e37, 1e38, np.finfo(np.float32).max])
@pytest.mark.parametrize("vocab", [2, 300, 20000])
def test_logits_further_apart_than_their_largest(vocab, temperature):
    """Finite logits whose difference is beyond the type's range weigh what the temperature says"""
    rng = np.random.default_rng(vocab)
    n, most = 24, np.finfo(np.float32).max
    x = (np.float64(most) * rng.uniform(-1, 1, (n, vocab))).astype(np.float32)
    x[:8] = np.where(rng.random((8, vocab)) < 0.5, most, -most)
    x[8:12, :vocab * 4 // 5] = -most
    x[12:16, ::2] = -np.inf
    x[16] = [most, -most] * (vocab // 2)
    u = rng.random(n, dtype=np.float32)
    for how in FILTERS:
        check(x, uniform=u, temperature=np.float32(temperature), **how)


@pytest.mark.parametrize("vocab", [2, 300, 20000])
def test_an_infinite_temperature(vocab):
    """All finite logits weigh one, however far apart they are; min-p of 1 keeps them all"""
    rng = np.random.default_rng(vocab)
    n, most = 24, np.finfo(np.float32).max
    x = (np.float64(most) * rng.uniform(-1, 1, (n, vocab))).astype(np.float32)
    x[:8] = rng.standard_normal((8, vocab)).astype(np.float32)
    x[8:12, :vocab * 4 // 5] = -most
    x[12:16, 1::2] = -np.inf
    u = rng.random(n, dtype=np.float32)
    for how in FILTERS + [dict(min_p=1.0), dict(top_k=600, min_p=1.0)]:
        check(x, uniform=u, temperature=np.float32(np.inf), **how)


def test_random_numbers_out_of_range():
    rng = np.random.default_rng(8)
    x = model_logits(rng, 6, 700)
    zero, last = draw(x, uniform=0.0), draw(x, uniform=np.float32(1 - 2.0 ** -24))
    assert [g[0] for g in zero] == list(x.argmax(-1))
    for u in (-1.0, -np.inf, np.nan):
        assert draw(x, uniform=u) == zero
    for u in (1.0, 3.0, np.inf):
        check(x, uniform=u)
    assert draw(x, uniform=1.0) == draw(x, uniform=np.inf) and len(last) == 6


def test_draws_follow_the_weights():
    """Over random numbers that are evenly spaced a token comes up as often as its probability says, to one"""
    rng = np.random.default_rng(9)
    x = rng.standard_normal(40).astype(np.float32)
    n = 1 << 14
    got = draw(np.broadcast_to(x, (n, 40)), uniform=np.arange(n) / n, top_p=0.9, temperature=0.8)
    r = page8_ref.sample(x, uniform=0.0, top_p=0.9, temperature=0.8)
    times = np.bincount([t for t, _, _ in got], minlength=40)
    want = np.zeros(40)
    want[r["order"][:r["kept"]]] = r["w"][:r["kept"]] / r["sums"][r["kept"] - 1]
    assert (np.abs(times - want * n) <= 1.0 + 1e-6).all()


def test_outputs_that_are_not_wanted_and_replays():
    rng = np.random.default_rng(10)
    n, vocab = 300, 50304
    x, u = model_logits(rng, n, vocab), rng.random(n, dtype=np.float32)
    gx, gu, tokens = dev(x), f32(u), i32([-7] * n)
    p = f32(rng.choice([0.5, 0.9, 1.0], n))
    how = cf.Sampling.of(uniform=gu, top_p=p)
    cf.cfpp_sample(gx, cf.TYPE_F32, n, vocab, how, tokens, stream=stream())
    first = tokens.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        cf.cfpp_sample(gx, cf.TYPE_F32, n, vocab, how, tokens, stream=stream())
    for k in range(3):
        tokens.fill_(-7)
        graph.replay()
        assert torch.equal(tokens, first)
        gu.copy_(f32(rng.random(n, dtype=np.float32)))
        graph.replay()
        again = tokens.clone()
        cf.cfpp_sample(gx, cf.TYPE_F32, n, vocab, how, tokens, stream=stream())
        assert torch.equal(tokens, again) and not torch.equal(tokens, first)
        gu.copy_(f32(u))


@pytest.mark.parametrize("dtype", [np.float32, np.float16])
def test_rows_that_lie_far_apart(dtype):
    """row_stride of 2^32 values, its most"""
    rng = np.random.default_rng(51)
    vocab, stride = 1001, 1 << 32
    x, u = model_logits(rng, 2, vocab, dtype), rng.random(2, dtype=np.float32)
    g = torch.empty(stride + vocab, dtype=torch.float16 if dtype == np.float16 else torch.float32, device="cuda")
    g[:vocab].copy_(dev(x[0]))
    g[stride:].copy_(dev(x[1]))
    tokens, kept, probs = i32([-7] * 2), i32([-7] * 2), f32([-7] * 2)
    gu = f32(u)
    cf.cfpp_sample(g, cf.TYPE_F16 if dtype == np.float16 else cf.TYPE_F32, 2, vocab, cf.Sampling.of(uniform=gu), tokens, probs, kept, stride, stream())
    torch.cuda.synchronize()
    for r in range(2):
        page8_ref.check_sample(x[r], (int(tokens[r]), float(probs[r]), int(kept[r])), uniform=float(u[r]))


@pytest.mark.parametrize("dtype", [np.float32, np.float16])
def test_as_many_logits_as_there_may_be(dtype):
    """2^18 of them: equal ones, whose sum is the largest there is, and such as a model has"""
    rng = np.random.default_rng(53)
    n, vocab = 6, 1 << 18
    x = model_logits(rng, n, vocab, dtype)
    x[:2] = [[-1.25], [3.5]]
    x[4] = np.round(x[4])
    x[5, :-200] = -np.inf
    u = rng.random(n, dtype=np.float32)
    for how in (dict(), dict(top_k=200000), dict(top_p=0.37), dict(min_p=0.5), dict(top_k=600, top_p=0.9), dict(temperature=1e-3), dict(temperature=50.0, top_p=0.999)):
        got = check(x, uniform=u, **how)
        kept = 200000 if "top_k" in how and "top_p" not in how else vocab
        if "top_p" not in how:
            assert [t for t, _, _ in got[:2]] == [int(np.floor(float(v) * kept)) for v in u[:2]]


def test_two_streams_at_once():
    rng = np.random.default_rng(52)
    x, u = [model_logits(rng, 40, 50304) for _ in range(2)], rng.random(40, dtype=np.float32)
    want = [[t for t, _, _ in draw(a, uniform=u, top_p=0.9)] for a in x]
    g, gu, p = [dev(a) for a in x], f32(u), f32([0.9] * 40)
    how = cf.Sampling.of(uniform=gu, top_p=p)
    tokens, streams = [i32([-7] * 40) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for i in range(2):
            cf.cfpp_sample(g[i], cf.TYPE_F32, 40, 50304, how, tokens[i], stream=streams[i].cuda_stream)
    torch.cuda.synchronize()
    assert [t.cpu().numpy().tolist() for t in tokens] == want


# ---- the generation loop -----------------------------------------------------------------------------
def test_generation_with_sampling():
    """The captured loop against its calls one by one, and every token against the plain form on the logits that the step left"""
    import synth
    from tests.test_gpu_generate import SHAPE, VOCAB, _device, _world
    S, steps = 21, 24
    cap, layers, kv, head, embed, tokens = _world(99, S, steps)
    rng = np.random.default_rng(12)
    u = rng.random(cap, dtype=np.float32)
    g = dict(uniform=f32(u), temperature=f32([0.8]), top_k=i32([200]), top_p=f32([0.9]), min_p=f32([0.001]))
    how = cf.Sampling.of(**g)
    runs = []
    for graph in (True, False):
        ds = _device(cap, layers, kv, head, embed, S, 2 if graph else 0)
        try:
            ds.set_tokens(tokens, S)
            if graph:
                cf.cfpp_generate_sample_capture(ds.ctx, ds.packed, ds.kv, ds.lm, how, ds.tokens, ds.pos, ds.x, ds.out, ds.logits, ds.s)
            out = []
            for step in range(steps):
                if graph:
                    ds.replay()
                else:
                    cf.cfpp_lm_embed(ds.ctx, ds.lm, ds.tokens, ds.pos, ds.x, ds.s)
                    cf.cfpp_stack_decode(ds.ctx, ds.packed, ds.kv, ds.x, ds.pos, 1, ds.out, ds.s)
                    cf.cfpp_lm_sample(ds.ctx, ds.lm, ds.out, how, ds.tokens, ds.pos, ds.logits, ds.s)
                ds.stream.synchronize()
                assert int(ds.pos[0].item()) == S + step + 1
                token, logits = int(ds.tokens[S + step + 1].item()), ds.logits.cpu().numpy().copy()
                r = page8_ref.sample(logits, temperature=0.8, top_k=200, top_p=0.9, min_p=0.001, uniform=u[S + step])
                at = int(np.nonzero(r["order"] == token)[0][0])
                before, off = r["sums"][at - 1] if at else 0.0, page8_ref.sample_off(r)
                assert at < r["kept"] and before <= r["target"] + off and r["sums"][at] >= r["target"] - off
                out.append((token, logits))
            ds.check()
            runs.append(out)
            # past the end nothing is drawn
            ds.pos[:1].fill_(cap)
            torch.cuda.synchronize()
            was = ds.tokens.clone()
            cf.cfpp_lm_sample(ds.ctx, ds.lm, ds.out, how, ds.tokens, ds.pos, ds.logits, ds.s)
            ds.stream.synchronize()
            assert torch.equal(was, ds.tokens) and int(ds.pos[0].item()) == cap
        finally:
            ds.close()
    assert len({t for t, _ in runs[0]}) > 3
    # the head alone leaves the same logits whether the token is drawn or picked
    ds = _device(cap, layers, kv, head, embed, S, 0)
    try:
        ds.set_tokens(tokens, S)
        ds.generate_step(want_logits=True)
        ds.stream.synchronize()
        assert np.array_equal(ds.logits.cpu().numpy(), runs[1][0][1])
        greedy = int(ds.tokens[S + 1].item())
        ds.set_tokens(tokens, S)
        cold = cf.Sampling.of(uniform=g["uniform"], temperature=f32([0.0]))
        cf.cfpp_lm_sample(ds.ctx, ds.lm, ds.out, cold, ds.tokens, ds.pos, ds.logits, ds.s)
        ds.stream.synchronize()
        assert int(ds.tokens[S + 1].item()) == greedy
        for bad in (dict(logits_dev=0), dict(how=cf.Sampling.of(uniform=0))):
            with pytest.raises(cf.CfppError) as e:
                cf.cfpp_lm_sample(ds.ctx, ds.lm, ds.out, bad.get("how", cold), ds.tokens, ds.pos, bad.get("logits_dev", ds.logits), ds.s)
            assert e.value.status == -1
    finally:
        ds.close()


@pytest.mark.parametrize("heads,d,vocab,threads", [(2, 64, 300, 512), (1, 80, 500, 512), (8, 64, 900, 256), (2, 64, 3, 512)])
def test_a_token_behind_both_kernels_of_the_head(heads, d, vocab, threads):
    """Twice from the same position: nothing is left behind for the pick of cfpp_lm_next, which follows"""
    import synth
    from paper_2604_23553_amd.harness import DeviceStack
    shape = synth.ModelShape(heads * d, heads, d, 16, 512, n_layers=1, name=f"lm-h{heads * d}")
    ds = DeviceStack(shape, 8, 1, 1)
    try:
        ds.set_options(threads=threads)
        ds.load_lm(synth.lm_head(shape, 15, vocab=vocab), synth.embedding(shape, 15, vocab=vocab))
        ds.out[:1].copy_(torch.from_numpy(synth.x_input(shape, 15)))
        u = np.float32([0.9, 0.37, 0.2, 0.1, 0.0, 0.0, 0.0, 0.0])
        g = dict(uniform=f32(u), temperature=f32([0.5]))
        for step in range(2):
            ds.set_tokens([0, 0], 1)
            cf.cfpp_lm_sample(ds.ctx, ds.lm, ds.out, cf.Sampling.of(**g), ds.tokens, ds.pos, ds.logits, ds.s)
            ds.check()
            logits = ds.logits.cpu().numpy()
            r = page8_ref.sample(logits, temperature=0.5, uniform=float(u[1]))
            at = int(np.nonzero(r["order"] == int(ds.tokens[2].item()))[0][0])
            off = page8_ref.sample_off(r)
            assert (r["sums"][at - 1] if at else 0.0) <= r["target"] + off and r["sums"][at] >= r["target"] - off
            assert int(ds.pos[0].item()) == 2
        ds.set_tokens([0, 0], 1)
        cf.cfpp_lm_next(ds.ctx, ds.lm, ds.out, ds.tokens, ds.pos, ds.logits, ds.s)
        ds.check()
        assert np.array_equal(ds.logits.cpu().numpy(), logits) and int(ds.tokens[2].item()) == int(np.argmax(logits))
    finally:
        ds.close()


# ---- a server's step ----------------------------------------------------------------------------------
@pytest.mark.parametrize("type", [page8_ref.INT8, page8_ref.E4M3])
def test_a_servers_steps(type):
    """Tables, plan, append and attention of two layers, logits and sampling, captured once and replayed: requests grow over page borders, one ends and begins
    anew, one has no row.  Every operator's result against the plain form on what the step before it left."""
    from tests import tree_ref
    rng = np.random.default_rng(type)
    R, H, kv, d, page, vocab, layers, stride = 5, 4, 2, 64, 16, 999, 2, 6
    h, n_pages = H * d, 24
    lens = [14, 0, 31, 60, 7]
    alloc = tree_ref.Allocator(n_pages, page, R, stride, rng)
    pools = [page8_ref.Pool(n_pages, page, kv, d, type) for _ in range(layers)]
    # what the requests have cached before
    alloc.step([0] * R, lens, sum(lens))
    for pool in pools:
        for r in range(R):
            for t in range(lens[r]):
                pool.put(alloc.tables[r][t // page] * page + t % page, *rng.standard_normal((2, kv, d)).astype(np.float16))
    half = lambda *n: dev((rng.standard_normal(n) / np.sqrt(n[0])).astype(np.float16))  # noqa: E731
    embed, w_out = dev(rng.standard_normal((vocab, h)).astype(np.float16)), half(h, vocab)
    w = [(half(h, h), half(h, kv * d), half(h, kv * d), half(h, h)) for _ in range(layers)]
    table = np.full((R, stride), -1, dtype=np.int32)
    for r, t in enumerate(alloc.tables):
        table[r, :len(t)] = t
    free = np.full(n_pages, -1, dtype=np.int32)
    free[:len(alloc.free)] = alloc.free
    g = dict(lens=i32(lens), counts=i32([1] * R), table=i32(table), held=i32([len(t) for t in alloc.tables]), free=i32(free), free_count=i32([len(alloc.free)]),
             granted=i32([0] * R), row_start=i32([0] * (R + 1)), slots=i32([0] * R), parents=i32([-1] * R), masks=i32([[0]] * R), positions=i32([0] * R),
             tokens=i32(rng.integers(0, vocab, R)), kept=i32([0] * R), uniform=f32(np.zeros(R)), top_p=f32([0.9] * R), top_k=i32([0, 40, 0, 40, 0]),
             temperature=f32([1.0, 0.7, 0.0, 1.5, 1.0]), probs=f32([0] * R))
    P = cf.Pages(n_pages, page, kv, d)
    plan = torch.empty(cf.cfpp_tree_plan_bytes(P, H, R, R, 1), dtype=torch.uint8, device="cuda")
    batch = cf.TreeBatch.of(1, g["lens"], g["row_start"], g["table"], g["slots"], g["parents"], g["masks"], g["positions"], plan)
    how = cf.Sampling.of(uniform=g["uniform"], temperature=g["temperature"], top_k=g["top_k"], top_p=g["top_p"])
    g_pools = [dev(p.bytes) for p in pools]
    q, k, v, o = (torch.zeros((layers, R, n), dtype=torch.float16, device="cuda") for n in (h, kv * d, kv * d, h))
    logits = torch.zeros((R, vocab), dtype=torch.float32, device="cuda")

    def step():
        s = stream()
        cf.cfpp_page_tables(P, batch, g["counts"], g["held"], g["free"], g["free_count"], g["granted"], s)
        cf.cfpp_tree_plan(P, batch, H, s)
        x = embed[g["tokens"].long()]
        for l in range(layers):
            for to, by in zip((q, k, v), w[l]):
                torch.matmul(x, by, out=to[l])
            cf.cfpp_page8_append(P, type, g_pools[l], k[l], v[l], g["slots"], R, stream=s)
            cf.cfpp_page8_attention(P, type, g_pools[l], batch, q[l], H, o[l], stream=s)
            x = x + torch.matmul(o[l], w[l][3])
        logits.copy_(torch.matmul(x, w_out))
        cf.cfpp_sample(logits, cf.TYPE_F32, R, vocab, how, g["tokens"], g["probs"], g["kept"], stream=s)

    # (the first call of a library product may not be captured)
    torch.matmul(embed[:R], w[0][0])
    torch.matmul(embed[:R], w[0][1])
    torch.matmul(embed[:R], w_out)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    counts = [1] * R
    for n in range(12):
        if n == 5:
            lens[2] = 0                                     # a request ends, another begins in its place
        counts[4] = 0 if n in (3, 4) else 1                # the last one pauses
        u = rng.random(R, dtype=np.float32)
        g["lens"].copy_(i32(lens))
        g["counts"].copy_(i32(counts))
        g["uniform"].copy_(f32(u))
        o.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        granted, starts, slots = alloc.step(lens, counts, R)
        assert granted == [1] * R and np.array_equal(g["slots"].cpu().numpy(), slots) and g["row_start"].cpu().tolist() == starts
        for l in range(layers):
            kk, vv, qq, got = (t[l].cpu().numpy() for t in (k, v, q, o))
            for r in range(R):
                if not counts[r]:
                    assert (got[r] == 7.0).all()           # (the last row is nobody's then)
                    continue
                pools[l].put(int(slots[r]), kk[r].reshape(kv, d), vv[r].reshape(kv, d))
                rows = np.stack([pools[l].get(alloc.tables[r][t // page] * page + t % page) for t in range(lens[r] + 1)], 1)
                want, off = page8_ref.attend(qq[r].astype(np.float64).reshape(1, H, d), rows[0], rows[1], np.ones((1, lens[r] + 1), dtype=bool))
                limit = np.abs(want) * 2.0 ** -11 + 2.0 ** -25 + off * (1 + 2.0 ** -11)
                assert (np.abs(got[r].astype(np.float64).reshape(1, H, d) - want) <= limit).all(), f"step {n}, layer {l}, request {r}"
        x, tokens, probs, kept = (t.cpu().numpy() for t in (logits, g["tokens"], g["probs"], g["kept"]))
        for r in range(R):
            page8_ref.check_sample(x[r], (int(tokens[r]), float(probs[r]), int(kept[r])), uniform=float(u[r]), temperature=[1.0, 0.7, 0.0, 1.5, 1.0][r],
                                   top_k=[0, 40, 0, 40, 0][r], top_p=0.9)
        for r in range(R):
            lens[r] += counts[r]
