"""What a server does for every new token on a cache in 8 bits: the operators that a step takes, as cases that can be timed and checked.

    append     the new K and V rows of a layer, quantised into their slots               cfpp_page8_append
    read       rows read back out of their slots                                         cfpp_page8_read
    attention  every request's new token over its cached positions and itself            cfpp_page8_attention
    sample     the next token from logits: temperature, top-k, top-p, min-p              cfpp_sample

Where `own` is false, run() computes them with elementary torch operations; where it is true it makes the package's calls.
A row of K or V of one head is held as d codes of 8 bits and its largest absolute value a: a code c stands for c * a / 127
(int8) or c * a / 448 (e4m3).  A pool of pages is bytes [pages][key heads][page length / 16][32 d + 64]; the last axis, 16 positions
t = 4 T + i of a head: K codes [T][d / 16][i][16], V codes [d][16 positions], a of K [16], a of V [16] (fp16).
"""
import math
import random

import numpy as np
import torch

own = False

# name: query heads, key heads, head size
HEADS = {
    "h512": (8, 8, 64),
    "h1280": (16, 16, 80),
    "h2560": (32, 32, 80),       # the Pythia-2.8B shape
    "h4096": (32, 32, 128),      # the Pythia-6.9B shape
    "g4": (32, 8, 128),          # four query heads to a key head
    "g8": (16, 2, 64),
}
TOP = {"int8": 127.0, "e4m3": 448.0}
TYPE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
MOST_BYTES = 1.5e9                                         # a pass of the largest listed case


def _rows(op, rows=1, page=64, heads="h2560", type="int8", **more):
    """rows: rows that are written or read back; first: the first one's position of those that follow one another, -1: one row to a request."""
    return dict(more, op=op, rows=rows, page=page, heads=heads, type=type)


def _attention(requests=1, lo=0, hi=0, page=64, heads="h2560", type="int8", **more):
    """lo .. hi: cached positions of a request."""
    return dict(more, op="attention", requests=requests, lo=lo, hi=hi, page=page, heads=heads, type=type)


def _sample(rows=1, vocab=50304, filters="p", type="f32", **more):
    """filters: which of k, p and m (min-p) every row has; "mixed": each row draws its own."""
    return dict(more, op="sample", rows=rows, vocab=vocab, filters=filters, type=type)


def listed():
    return [
        # a decode step of a serving batch: one new row to a request, anywhere in the pool
        _rows("append", rows=64, first=-1, name="append_r64_h2560"),
        # the rows of a long prompt pass
        _rows("append", rows=4096, first=0, heads="h4096", type="e4m3", name="append_n4096_h4096_e4m3"),
        # a short conversation's rows read back, from the middle of a page on
        _rows("read", rows=77, first=1003, name="read_n77_h2560"),
        # a long context read back into an fp16 cache
        _rows("read", rows=16384, first=0, page=128, heads="g4", type="e4m3", name="read_n16384_g4_e4m3"),
        # a single token of a small model behind a short context
        _attention(lo=127, hi=127, heads="h512", name="attention_r1_s128_h512"),
        # one conversation behind a long context
        _attention(lo=4095, hi=4095, type="e4m3", name="attention_r1_s4096_h2560_e4m3"),
        # one request with a very long document, two key heads
        _attention(lo=131071, hi=131071, page=128, heads="g8", name="attention_r1_s131072_g8"),
        # a serving batch, ragged lengths, shared key heads, small pages
        _attention(requests=64, lo=33, hi=3001, page=16, heads="g4", type="e4m3", name="attention_r64_g4_e4m3"),
        # a serving batch behind long contexts
        _attention(requests=32, lo=3000, hi=8191, heads="h4096", name="attention_r32_s8192_h4096"),
        # the next token of one conversation
        _sample(name="sample_r1_p"),
        # a serving batch with a usual set of filters
        _sample(rows=64, filters="kpm", name="sample_r64_kpm"),
        # the rows of a large batch of drafted trees, each request with filters of its own
        _sample(rows=512, filters="mixed", name="sample_r512_mixed"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "read", "attention", "attention", "attention", "sample", "sample"])
    page, heads, type = rng.choice([16, 32, 48, 64, 128, 256]), rng.choice(sorted(HEADS)), rng.choice(sorted(TOP))
    if op == "sample":
        c = _sample(rows=_log_int(rng, 1, 512), vocab=_log_int(rng, 1000, 131072), filters=rng.choice(["", "k", "p", "m", "kp", "kpm", "mixed"]),
                    type=rng.choice(["f32", "f32", "f16"]))
        while c["rows"] > 1 and c["rows"] * c["vocab"] > 512 * 50304:
            c["rows"] = (c["rows"] * 3) // 4
        return c
    if op != "attention":
        return _rows(op, rows=_log_int(rng, 1, 4096), page=page, heads=heads, type=type, first=rng.choice([-1, rng.randint(0, 2000)]))
    hi = _log_int(rng, 1, 131072)
    c = _attention(requests=_log_int(rng, 1, 64), lo=rng.choice([hi, rng.randint(0, hi)]), hi=hi, page=page, heads=heads, type=type)
    while c["requests"] > 1 and work(c)["bytes"] > MOST_BYTES:
        c["requests"] = (c["requests"] * 3) // 4
    while work(c)["bytes"] > MOST_BYTES:
        c["hi"], c["lo"] = c["hi"] // 2, c["lo"] // 2
    return c


# ---- sizes that follow from a case ---------------------------------------------------------
def _lens(case):
    """Cached positions of each request; the first has the most."""
    r = random.Random(case["lo"] * 8209 + case["hi"] * 17 + case["requests"] * 5)
    return [case["hi"]] + [r.randint(case["lo"], case["hi"]) for _ in range(case["requests"] - 1)]


def _pages_of(n, page):
    return -(-n // page)


def work(case):
    """Every input and every cached position read once, every output written once; two operations a multiplication."""
    if case["op"] == "sample":
        size = 4 if case["type"] == "f32" else 2
        # a weight and its sum for every logit
        return {"bytes": case["rows"] * (case["vocab"] * size + 5 * 4 + 3 * 4), "flops": 4 * case["rows"] * case["vocab"]}
    q, kv, d = HEADS[case["heads"]]
    if case["op"] != "attention":
        return {"bytes": case["rows"] * (2 * kv * (2 * d + d + 2) + 4), "flops": 4 * case["rows"] * kv * d}
    lens = _lens(case)
    seen = sum(lens) + len(lens)
    return {"bytes": seen * 2 * kv * (d + 2) + 2 * 2 * len(lens) * q * d + 4 * sum(_pages_of(n + 1, case["page"]) for n in lens), "flops": 4 * q * d * seen}


# ---- the pool ---------------------------------------------------------------------------------
def _parts(pool, d, type):
    """Views of a pool: K codes [pages][heads][granules][T][d / 16][i][16], V codes [pages][heads][granules][d][16], a of K and V [pages][heads][granules][16]"""
    k = pool[..., :16 * d].view(TYPE[type]).unflatten(-1, (4, d // 16, 4, 16))
    v = pool[..., 16 * d:32 * d].view(TYPE[type]).unflatten(-1, (d, 16))
    return k, v, pool[..., 32 * d:32 * d + 32].view(torch.float16), pool[..., 32 * d + 32:].view(torch.float16)


def _codes(x, type):
    """(codes, a) of rows [..., d]"""
    a = x.abs().amax(-1, keepdim=True)
    # (the product is exact in 32 bits, the quotient is rounded once and never next to the middle of two codes unless it is the middle)
    y = x.float() * TOP[type] / a.float()
    y = y.round() if type == "int8" else y
    return y.nan_to_num(0.0).to(TYPE[type]), a.squeeze(-1)


def _some_pool(n_pages, page, kv, d, type, g):
    """A pool whose every position holds a row of N(0, 1)"""
    pool = torch.zeros((n_pages, kv, page // 16, 32 * d + 64), dtype=torch.uint8, device="cuda")
    at = max(1, (1 << 26) // (kv * page * d))
    for p in range(0, n_pages, at):
        part = pool[p:p + at]
        k, v, ka, va = _parts(part, d, type)
        n = part.shape[0]
        x, a = _codes(torch.randn((n, kv, page // 16, 4, 4, d), generator=g, dtype=torch.float16, device="cuda"), type)
        k.copy_(x.unflatten(-1, (d // 16, 16)).transpose(4, 5))
        ka.copy_(a.flatten(-2))
        x, a = _codes(torch.randn((n, kv, page // 16, 16, d), generator=g, dtype=torch.float16, device="cuda"), type)
        v.copy_(x.transpose(-1, -2))
        va.copy_(a)
    return pool


# ---- inputs -----------------------------------------------------------------------------------
class _State:
    pass


def prepare(case, seed):
    s = _State()
    s.case = case
    rng = np.random.default_rng([seed, 3])
    dev = dict(device="cuda")
    i32 = lambda v: torch.tensor(np.asarray(v, dtype=np.int32), **dev)  # noqa: E731
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + 29)
    if case["op"] == "sample":
        R, V = case["rows"], case["vocab"]
        # a language model's logits: a broad field and a few tokens that stand out of it
        x = 2.5 * torch.randn((R, V), generator=g, **dev)
        x.scatter_add_(1, torch.randint(0, V, (R, 12), generator=g, **dev), 9.0 + 2.0 * torch.randn((R, 12), generator=g, **dev))
        s.logits = x.half() if case["type"] == "f16" else x
        on = {n: rng.random(R) < 0.5 if case["filters"] == "mixed" else np.full(R, n in case["filters"]) for n in "kpm"}
        f32 = lambda v: torch.tensor(np.asarray(v, dtype=np.float32), **dev)  # noqa: E731
        s.temperature = f32(np.where(rng.random(R) < 0.1, 0.0, rng.choice([0.6, 0.8, 1.0, 1.0, 1.3], R)) if case["filters"] == "mixed" else np.full(R, 0.8))
        s.top_k = i32(np.where(on["k"], rng.choice([1, 20, 40, 50, 100, 1000], R) if case["filters"] == "mixed" else 50, 0))
        s.top_p = f32(np.where(on["p"], rng.choice([0.5, 0.8, 0.9, 0.95, 0.99], R) if case["filters"] == "mixed" else 0.95, 1.0))
        s.min_p = f32(np.where(on["m"], rng.choice([0.01, 0.05, 0.1], R) if case["filters"] == "mixed" else 0.02, 0.0))
        s.uniform = f32(rng.integers(0, 1 << 24, R) / float(1 << 24))
        s.tokens, s.kept, s.probs = i32(np.zeros(R)), i32(np.zeros(R)), f32(np.zeros(R))
        if own:
            import paper_2604_23553_amd as cf
            s.type = {"f32": cf.TYPE_F32, "f16": cf.TYPE_F16}[case["type"]]
            s.how = cf.Sampling.of(temperature=s.temperature, top_k=s.top_k, top_p=s.top_p, min_p=s.min_p, uniform=s.uniform)
        return s
    q, kv, d = HEADS[case["heads"]]
    page, type = case["page"], case["type"]
    if case["op"] != "attention":
        n, first = case["rows"], case["first"]
        n_pages = (n if first < 0 else _pages_of(first + n, page)) + 3
        order = rng.permutation(n_pages)
        at = np.arange(n) * page + rng.integers(0, page, n) if first < 0 else first + np.arange(n)
        s.slots = i32(order[at // page] * page + at % page)
        s.pool = _some_pool(n_pages, page, kv, d, type, g)
        s.k, s.v = (torch.randn((n, kv, d), generator=g, dtype=torch.float16, **dev) for _ in range(2))
    else:
        lens = _lens(case)
        R, stride = case["requests"], _pages_of(case["hi"] + 1, page)
        need = np.array([_pages_of(a + 1, page) for a in lens])
        n_pages = int(need.sum()) + 3
        table = np.full((R, stride), -1, dtype=np.int32)
        table[np.arange(stride)[None, :] < need[:, None]] = rng.permutation(n_pages)[:need.sum()]
        s.lens, s.table, s.row_start = i32(lens), i32(table), i32(np.arange(R + 1))
        at = np.array(lens)
        s.slots = i32(table[np.arange(R), at // page] * page + at % page)
        s.pool = _some_pool(n_pages, page, kv, d, type, g)
        s.q = torch.randn((R, q, d), generator=g, dtype=torch.float16, **dev)
        s.out = torch.zeros_like(s.q)
    if own:
        import paper_2604_23553_amd as cf
        s.type = {"int8": cf.TYPE_INT8, "e4m3": cf.TYPE_E4M3}[type]
        s.pages = cf.Pages(n_pages, page, kv, d)
        if case["op"] == "attention":                      # once a step; its layers then share it
            s.parents, s.masks, s.positions = i32(np.full(R, -1)), i32(np.zeros((R, 1))), i32(np.zeros(R))
            s.plan = torch.empty(cf.cfpp_tree_plan_bytes(s.pages, q, R, R, 1), dtype=torch.uint8, **dev)
            s.batch = cf.TreeBatch.of(max_nodes=1, lens=s.lens, row_start=s.row_start, block_table=s.table, slots=s.slots,
                                      parents=s.parents, masks=s.masks, positions=s.positions, plan=s.plan)
            cf.cfpp_tree_plan(s.pages, s.batch, q, torch.cuda.current_stream().cuda_stream)
    return s


# ---- the plain forms ------------------------------------------------------------------------------
def _at(s):
    """page, granule, T, i of each slot"""
    slot, page = s.slots.long(), s.case["page"]
    t = slot % page
    return slot // page, t // 16, t % 16 // 4, t % 4


def _plain_append(s):
    d, type = HEADS[s.case["heads"]][2], s.case["type"]
    k, v, ka, va = _parts(s.pool, d, type)
    page, granule, T, i = _at(s)
    x, a = _codes(s.k, type)
    k.view(torch.uint8)[page, :, granule, T, :, i] = x.view(torch.uint8).unflatten(-1, (d // 16, 16))
    ka[page, :, granule, 4 * T + i] = a
    x, a = _codes(s.v, type)
    v.view(torch.uint8)[page, :, granule, :, 4 * T + i] = x.view(torch.uint8)
    va[page, :, granule, 4 * T + i] = a


def _plain_read(s):
    d, type = HEADS[s.case["heads"]][2], s.case["type"]
    k, v, ka, va = _parts(s.pool, d, type)
    page, granule, T, i = _at(s)
    x = k.view(torch.uint8)[page, :, granule, T, :, i].flatten(-2).view(TYPE[type]).float()
    s.k.copy_(x * ka[page, :, granule, 4 * T + i].float()[..., None] / TOP[type])
    x = v.view(torch.uint8)[page, :, granule, :, 4 * T + i].view(TYPE[type]).float()
    s.v.copy_(x * va[page, :, granule, 4 * T + i].float()[..., None] / TOP[type])


def _plain_attention(s):
    (q, kv, d), type = HEADS[s.case["heads"]], s.case["type"]
    R = s.case["requests"]
    k, v, ka, va = _parts(s.pool[s.table.long().clamp(min=0)], d, type)                # [R][pages][kv][granules]...
    k = k.float().transpose(-2, -3).flatten(-2).flatten(-3, -2) * (ka.float() / TOP[type])[..., None]
    v = v.float().transpose(-1, -2) * (va.float() / TOP[type])[..., None]
    k, v = (x.transpose(1, 2).flatten(2, 4) for x in (k, v))                           # [R][kv][positions][d]
    late = torch.arange(k.shape[2], device="cuda")[None, :] > s.lens[:, None]
    qq = s.q.float().view(R, kv, q // kv, d)
    score = torch.matmul(qq, k.transpose(2, 3).contiguous()) / math.sqrt(d)
    score.masked_fill_(late[:, None, None, :], -math.inf)
    score = (score - score.amax(-1, keepdim=True)).exp_()
    s.out.copy_((torch.matmul(score, v) / score.sum(-1, keepdim=True)).view(R, q, d))


def _plain_sample(s):
    x = s.logits.double()
    V = x.shape[1]
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices
    tau = s.temperature.double()[:, None]
    w = torch.exp((x - x.amax(-1, keepdim=True)) / torch.where(tau > 0, tau, 1.0))
    ws = w.gather(1, order)
    rank = torch.arange(V, device="cuda")[None, :]
    keep = rank < torch.where(s.top_k > 0, s.top_k, V)[:, None]
    sums = (ws * keep).cumsum(-1)
    before = torch.cat([torch.zeros_like(sums[:, :1]), sums[:, :-1]], 1)
    p = s.top_p.double()[:, None]
    keep &= (before < p * sums[:, -1:]) | (p >= 1)
    keep &= ws >= s.min_p.double()[:, None]
    keep = (keep & (tau > 0)) | (rank == 0)
    s.kept.copy_(keep.sum(-1))
    ws = ws * keep
    sums = ws.cumsum(-1)
    at = (sums <= s.uniform.double()[:, None] * sums[:, -1:]).sum(-1, keepdim=True).clamp(max=V - 1)
    s.tokens.copy_(order.gather(1, at)[:, 0])
    s.probs.copy_((ws.gather(1, at) / sums[:, -1:])[:, 0])


def run(s):
    op = s.case["op"]
    if own:
        import paper_2604_23553_amd as cf
        stream = torch.cuda.current_stream().cuda_stream
        if op == "append":
            cf.cfpp_page8_append(s.pages, s.type, s.pool, s.k, s.v, s.slots, s.case["rows"], stream=stream)
        elif op == "read":
            cf.cfpp_page8_read(s.pages, s.type, s.pool, s.slots, s.case["rows"], s.k, s.v, stream=stream)
        elif op == "attention":
            cf.cfpp_page8_attention(s.pages, s.type, s.pool, s.batch, s.q, HEADS[s.case["heads"]][0], s.out, stream=stream)
        else:
            cf.cfpp_sample(s.logits, s.type, s.case["rows"], s.case["vocab"], s.how, s.tokens, s.probs, s.kept, stream=stream)
    elif op == "append":
        _plain_append(s)
    elif op == "read":
        _plain_read(s)
    elif op == "attention":
        _plain_attention(s)
    else:
        _plain_sample(s)
    if op == "append":
        return dict(zip(("k", "v", "k_most", "v_most"), _parts(s.pool, HEADS[s.case["heads"]][2], s.case["type"])))
    if op == "read":
        return {"k": s.k, "v": s.v}
    if op == "attention":
        return {"out": s.out}
    return {"tokens": s.tokens, "probs": s.probs, "kept": s.kept}


# ---- the same in 64 bits, row after row or request after request ------------------------------------
def _to_e4m3(y):
    """The nearest value of three fraction bits, ties to even: steps of 2^(e - 3) from 2^e to 2^(e + 1), of 2^-9 below 2^-6"""
    e = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return torch.round(y / step) * step


def _value(pool, slots, page, d, type):
    """([rows][heads][d] of K, of V) in 64 bits: byte after byte from where the layout has it"""
    p, t = torch.div(slots, page, rounding_mode="floor"), slots % page
    one = pool[p, :, torch.div(t, 16, rounding_mode="floor")]                          # [rows][heads][32 d + 64]
    t = t % 16
    dim = torch.arange(d, device=pool.device)
    where = {"k": torch.div(t, 4, rounding_mode="floor")[:, None] * 4 * d + torch.div(dim, 16, rounding_mode="floor") * 64 + (t % 4)[:, None] * 16 + dim % 16,
             "v": 16 * d + dim[None, :] * 16 + t[:, None]}
    out = []
    for n, (which, at) in enumerate(where.items()):
        code = one.gather(2, at[:, None, :].expand(-1, one.shape[1], -1)).view(TYPE[type]).double()
        most = one[..., 32 * d + 32 * n:32 * d + 32 * n + 32].contiguous().view(torch.float16).double()
        out.append(code * most.gather(2, t[:, None, None].expand(-1, one.shape[1], 1)) / TOP[type])
    return out


def exact(case, seed):
    global own
    before, own = own, False
    s = prepare(case, seed)
    own = before
    if case["op"] == "sample":
        x, probs = s.logits.cpu().numpy().astype(np.float64), np.zeros(case["rows"])
        how = [v.cpu().numpy().astype(np.float64) for v in (s.temperature, s.top_k, s.top_p, s.min_p, s.uniform)]
        for r, (tau, k, p, m, u) in enumerate(zip(*how)):
            if tau <= 0:
                probs[r] = 1.0
                continue
            w = np.exp((x[r] - x[r].max()) / tau)
            first = np.argsort(-x[r], kind="stable")
            first = first[:int(k)] if k > 0 else first
            if p < 1:
                first = first[:1 + np.searchsorted(np.cumsum(w[first]), p * w[first].sum())]
            first = first[w[first] >= m]
            sums = np.cumsum(w[first])
            probs[r] = w[first[np.searchsorted(sums, u * sums[-1], side="right")]] / sums[-1]
        return {"tokens": None, "probs": torch.from_numpy(probs), "kept": None}
    (q, kv, d), page, type = HEADS[case["heads"]], case["page"], case["type"]
    if case["op"] == "read":
        k, v = _value(s.pool, s.slots.long(), page, d, type)
        return {"k": k, "v": v}
    if case["op"] == "append":
        k, v, ka, va = (x.double() if x.is_floating_point() or type == "e4m3" else None for x in _parts(s.pool, d, type))
        slots = s.slots.long()
        p, t = torch.div(slots, page, rounding_mode="floor"), slots % page
        gr, t = torch.div(t, 16, rounding_mode="floor"), t % 16
        for x, codes, most in ((s.k, k, ka), (s.v, v, va)):
            a = x.double().abs().max(-1).values
            most[p, :, gr, t] = a
            if codes is not None:
                y = _to_e4m3(x.double() * 448.0 / a[..., None].clamp(min=1e-30))
                if codes is k:
                    codes[p, :, gr, torch.div(t, 4, rounding_mode="floor"), :, t % 4] = y.unflatten(-1, (d // 16, 16))
                else:
                    codes[p, :, gr, :, t] = y
        return {"k": k, "v": v, "k_most": ka, "v_most": va}
    out = torch.zeros((case["requests"], q, d), dtype=torch.float64, device="cuda")
    for r, n in enumerate(_lens(case)):
        at = torch.arange(n + 1, device="cuda")
        k, v = _value(s.pool, s.table[r, torch.div(at, page, rounding_mode="floor")].long() * page + at % page, page, d, type)
        for h in range(q):
            score = torch.mv(k[:, h // (q // kv)], s.q[r, h].double()) / math.sqrt(d)
            out[r, h] = torch.mv(v[:, h // (q // kv)].t().contiguous(), torch.softmax(score, 0))
    return {"out": out}
