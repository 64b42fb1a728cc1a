"""Verifying trees of drafted tokens over a paged cache: the five operators that a step takes, as cases that can be timed and checked.

    tables     pages taken and given back, block tables, slots of the new rows      cfpp_page_tables
    plan       ancestor masks and positions of the nodes from their parents         cfpp_tree_plan
    append     the new K and V rows of a layer into their slots                     cfpp_page_append
    attention  every node over its request's cached positions and its ancestors     cfpp_tree_attention
    accept     the path that agrees with the model's picks, its rows moved forward  cfpp_tree_accept

Where `own` is false, run() computes them with elementary torch operations, in 32 bits; where it is true it makes the package's
calls.  A pool of pages is fp16 [2 (K, V)][pages][key heads][head size / 16][page length][16].  Request r has lens[r] cached
positions and the rows row_start[r] .. row_start[r + 1] - 1; node i of it stands at cache index lens[r] + i.
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
MOST_BYTES, MOST_FLOPS = 1.2e9, 3e11                       # a pass of the largest listed case


def _case(op, requests=1, nodes=1, least=None, lo=0, hi=0, page=64, heads="", layers=1, **more):
    """least .. nodes: rows of a request; lo .. hi: cached positions of a request; page: positions to a page."""
    return dict(more, op=op, requests=requests, nodes=nodes, least=nodes if least is None else least, lo=lo, hi=hi, page=page,
                heads=heads, layers=layers)


def listed():
    return [
        # one request, one token: what a step of a single conversation costs at least
        _case("tables", lo=1000, hi=1000, name="tables_r1"),
        # a full server: thousands of requests of all lengths, small pages
        _case("tables", requests=4096, nodes=64, least=1, lo=1, hi=8192, page=16, name="tables_r4096"),
        # eight conversations with a usual tree each
        _case("plan", requests=8, nodes=26, lo=100, hi=4000, heads="h2560", name="plan_r8_n26"),
        # many requests, larger trees of odd sizes
        _case("plan", requests=512, nodes=63, least=1, lo=1, hi=8192, heads="h4096", name="plan_r512_n63"),
        # one tree's rows of a layer
        _case("append", nodes=26, lo=1000, hi=1000, heads="h2560", name="append_n26_h2560"),
        # the rows of a long prompt pass, or of a large batch of trees
        _case("append", requests=64, nodes=64, lo=17, hi=2000, page=16, heads="h4096", name="append_n4096_h4096"),
        # a single token of a small model behind a short context
        _case("attention", nodes=1, lo=128, hi=128, heads="h512", name="attention_n1_s128_h512"),
        # one conversation's tree behind a long context
        _case("attention", nodes=26, lo=4096, hi=4096, heads="h2560", name="attention_n26_s4096_h2560"),
        # a serving batch of small trees, ragged lengths, shared key heads, small pages
        _case("attention", requests=64, nodes=9, least=1, lo=33, hi=3001, page=16, heads="g4", name="attention_r64_n9_g4"),
        # the largest trees behind long contexts
        _case("attention", requests=8, nodes=256, least=200, lo=6000, hi=8192, page=128, heads="h4096", name="attention_r8_n256_h4096"),
        # one conversation: the verdict and the move through 32 layers
        _case("accept", nodes=26, lo=700, hi=700, heads="h2560", layers=32, name="accept_n26_h2560"),
        # a serving batch
        _case("accept", requests=48, nodes=63, least=2, lo=20, hi=200, page=16, heads="h4096", layers=16, name="accept_r48_n63_h4096"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["tables", "plan", "append", "attention", "attention", "attention", "attention", "accept"])
    page = rng.choice([16, 32, 48, 64, 128, 256])
    heads = rng.choice(sorted(HEADS))
    if op in ("tables", "plan"):
        requests, nodes, hi, layers = _log_int(rng, 1, 4096 if op == "tables" else 512), _log_int(rng, 1, 64) if op == "tables" else _log_int(rng, 8, 256), _log_int(rng, 1, 8192), 1
    elif op == "append":
        requests, nodes, hi, layers = _log_int(rng, 1, 64), _log_int(rng, 1, 64), _log_int(rng, 1, 2048), 1
    elif op == "accept":
        requests, nodes, hi, layers = _log_int(rng, 1, 48), _log_int(rng, 2, 64), _log_int(rng, 1, 200), _log_int(rng, 1, 32)
    else:
        requests, nodes, hi, layers = _log_int(rng, 1, 64), _log_int(rng, 1, 256), _log_int(rng, 1, 8192), 1
    c = _case(op, requests=requests, nodes=nodes, least=rng.choice([nodes, rng.randint(1, nodes)]), lo=rng.choice([hi, rng.randint(0, hi)]), hi=hi,
              page=page, heads=heads, layers=layers)
    while c["requests"] > 1 and (work(c)["bytes"] > MOST_BYTES or work(c)["flops"] > MOST_FLOPS or _pool_bytes(c) > 4e9):
        c["requests"] = (c["requests"] * 3) // 4
    return c


# ---- sizes that follow from a case ---------------------------------------------------------
def _sizes(case):
    """Cached positions and rows of each request; the first has the most of both."""
    r = random.Random(case["lo"] * 8209 + case["hi"] * 17 + case["requests"] * 5 + case["nodes"])
    lens = [case["hi"]] + [r.randint(case["lo"], case["hi"]) for _ in range(case["requests"] - 1)]
    counts = [case["nodes"]] + [r.randint(case["least"], case["nodes"]) for _ in range(case["requests"] - 1)]
    return lens, counts


def _pages_of(n, page):
    return -(-n // page)


def _stride(case):
    return _pages_of(case["hi"] + case["nodes"], case["page"])


def _n_pages(case):
    lens, counts = _sizes(case)
    return sum(_pages_of(a + b, case["page"]) for a, b in zip(lens, counts)) + (61 if case["op"] == "tables" else 3)


def _pool_bytes(case):
    if case["op"] in ("tables", "plan"):
        return 0
    _, kv, d = HEADS[case["heads"]]
    return case["layers"] * 4 * kv * d * _n_pages(case) * case["page"]


def work(case):
    """Every input and every cached row that counts read once, every output written once; two operations a multiplication."""
    lens, counts = _sizes(case)
    R, n = case["requests"], sum(counts)
    words = (case["nodes"] + 31) // 32
    if case["op"] == "tables":
        # lens, counts, held; row_start, granted; a slot and the page behind it for each row
        return {"bytes": 4 * (5 * R + n + sum(_pages_of(a + b, case["page"]) - a // case["page"] for a, b in zip(lens, counts))), "flops": 0}
    if case["op"] == "plan":
        return {"bytes": 4 * (2 * R + n * (2 + words)), "flops": 0}
    q, kv, d = HEADS[case["heads"]]
    row = 2 * 2 * kv * d                                   # bytes of a position's K and V in one layer
    if case["op"] == "append":
        return {"bytes": n * (2 * row + 4), "flops": 0}
    if case["op"] == "accept":
        # (a path is some 3 + log2(nodes) long; all but its first node move)
        moved = sum(int(2 + math.log2(c)) if c > 1 else 0 for c in counts)
        return {"bytes": 4 * (3 * n + 3 * R + R * case["nodes"]) + 2 * moved * case["layers"] * row, "flops": 0}
    seen = sum(a + b for a, b in zip(lens, counts))
    return {"bytes": seen * row + 2 * 2 * n * q * d + 4 * n * words + 4 * R, "flops": 4 * q * d * sum(c * (a + c) for a, c in zip(lens, counts))}


# ---- inputs -----------------------------------------------------------------------------------
class _State:
    pass


def _tree(r, n):
    """Parents of n nodes, each behind its parent; node 0 is the token that the last step picked."""
    wide = r.random() < 0.5
    return [-1] + [r.randint(0, i - 1) if wide else r.randint(max(0, i - 3), i - 1) for i in range(1, n)]


def _path(parents, r):
    """A path from node 0 whose move can be made twice: no node of it stands where another one goes."""
    best = [0]
    for leaf in r.sample(range(len(parents)), len(parents)):
        p = [leaf]
        while p[-1] > 0:
            p.append(parents[p[-1]])
        p.reverse()
        want = int(3 + math.log2(len(parents)))
        p = p[:want]
        while any(at != j and at < len(p) for j, at in enumerate(p)):
            p.pop()
        if len(p) > len(best):
            best = p
    return best


def prepare(case, seed):
    s = _State()
    s.case = case
    lens, counts = _sizes(case)
    R, page, n_pages, stride = case["requests"], case["page"], _n_pages(case), _stride(case)
    r = random.Random(seed * 7919 + 1)
    rng = np.random.default_rng([seed, 2])
    dev = dict(device="cuda")
    i32 = lambda v: torch.tensor(np.asarray(v, dtype=np.int32), **dev)  # noqa: E731
    s.lens, s.counts, s.n_pages, s.stride = i32(lens), i32(counts), n_pages, stride
    starts = np.concatenate([[0], np.cumsum(counts)])
    s.rows = int(starts[-1])
    order = rng.permutation(n_pages)
    if case["op"] == "tables":
        # what the requests hold: the pages of their cached positions; every eighth has one more left of an earlier step
        held = np.array([min(_pages_of(a, page) + (k % 8 == 5), stride) for k, a in enumerate(lens)])
        need = np.array([_pages_of(a + b, page) for a, b in zip(lens, counts)])
        extra = int(np.maximum(held - need, 0).sum())
        order = rng.permutation(n_pages + extra)
        s.n_pages = n_pages + extra
        table = np.full((R, stride), -1, dtype=np.int32)
        cols = np.arange(stride)[None, :] < held[:, None]
        table[cols] = order[:held.sum()]
        s.held, s.table = i32(held), i32(table)
        free = np.full(s.n_pages, -1, dtype=np.int32)
        left = order[held.sum():]
        free[:len(left)] = left
        s.free, s.free_count = i32(free), i32([len(left)])
        s.row_start, s.slots, s.granted = i32(np.zeros(R + 1)), i32(np.zeros(s.rows + 7)), i32(np.zeros(R))
        if own:
            import paper_2604_23553_amd as cf
            s.pages = cf.Pages(s.n_pages, page, 1, 64)
            s.batch = cf.TreeBatch.of(max_nodes=case["nodes"], lens=s.lens, row_start=s.row_start, block_table=s.table, slots=s.slots)
        return s
    q, kv, d = HEADS[case["heads"]]
    s.row_start = i32(starts)
    need = np.array([_pages_of(a + b, page) for a, b in zip(lens, counts)])
    table = np.full((R, stride), -1, dtype=np.int32)
    cols = np.arange(stride)[None, :] < need[:, None]
    table[cols] = order[:need.sum()]
    s.table = i32(table)
    at = np.concatenate([a + np.arange(b) for a, b in zip(lens, counts)])
    req = np.repeat(np.arange(R), counts)
    s.slots = i32(table[req, at // page] * page + at % page)
    parents = [_tree(r, n) for n in counts]
    s.parents = i32(sum(parents, []))
    words = (case["nodes"] + 31) // 32
    s.masks = torch.zeros((s.rows, words), dtype=torch.int32, **dev)
    s.positions = torch.zeros(s.rows, dtype=torch.int32, **dev)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + 11)
    normal = lambda *dims: torch.randn(dims, generator=g, dtype=torch.float16, **dev)  # noqa: E731
    if case["op"] in ("append", "attention", "accept"):
        s.pool = normal(case["layers"], 2, n_pages, kv, d // 16, page, 16)
    if case["op"] == "append":
        s.k, s.v = normal(s.rows, kv, d), normal(s.rows, kv, d)
    if case["op"] == "attention":
        s.q = normal(s.rows, q, d)
        s.out = torch.zeros_like(s.q)
    if case["op"] == "accept":
        tokens, picks = rng.integers(0, 50304, s.rows), rng.integers(0, 50304, s.rows)
        for k, p in enumerate(parents):
            path, a = _path(p, r), starts[k]
            for i in range(1, len(p)):                     # (no other child agrees with the pick behind its parent)
                tokens[a + i] = (picks[a + p[i]] + 1 + i) % 50304
            for i in path[1:]:
                tokens[a + i] = picks[a + p[i]]
        s.tokens, s.picks = i32(tokens), i32(picks)
        s.accepted, s.next, s.lens_out = i32(np.zeros(R)), i32(np.zeros(R)), i32(np.zeros(R))
        s.path = torch.zeros((R, case["nodes"]), dtype=torch.int32, **dev)
    # what every operator behind the plan reads
    bits = np.zeros((s.rows, words), dtype=np.uint32)
    pos = np.zeros(s.rows, dtype=np.int32)
    for k, p in enumerate(parents):
        for i, up in enumerate(p):
            row = starts[k] + i
            if up >= 0:
                bits[row] = bits[starts[k] + up]
            pos[row] = lens[k] if up < 0 else pos[starts[k] + up] + 1
            bits[row, i // 32] |= np.uint32(1 << (i % 32))
    if case["op"] != "plan":
        s.masks, s.positions = torch.from_numpy(bits.view(np.int32)).cuda(), i32(pos)
    if own:
        import paper_2604_23553_amd as cf
        s.pages = cf.Pages(n_pages, page, kv, d)
        nbytes = cf.cfpp_tree_plan_bytes(s.pages, q, R, s.rows, case["nodes"])
        s.plan = torch.empty(nbytes, dtype=torch.uint8, **dev)
        s.batch = cf.TreeBatch.of(max_nodes=case["nodes"], lens=s.lens, row_start=s.row_start, block_table=s.table, slots=s.slots,
                                  parents=s.parents, masks=s.masks, positions=s.positions, plan=s.plan)
        if case["op"] == "accept":
            s.pools = list(s.pool)                         # a program has its layers' pools at hand
        if case["op"] == "attention":                      # once a step; its layers then share it
            cf.cfpp_tree_plan(s.pages, s.batch, q, torch.cuda.current_stream().cuda_stream)
    return s


# ---- the plain forms ------------------------------------------------------------------------------
def _place(s, rows):
    """Request and node of rows 0 .. rows - 1 (past the last row: of the last request)."""
    row = torch.arange(rows, device="cuda")
    req = torch.searchsorted(s.row_start[1:].long(), row, right=True).clamp_(max=s.case["requests"] - 1)
    return row, req, row - s.row_start.long()[req]


def _plain_tables(s):
    page, stride, P = s.case["page"], s.stride, s.n_pages
    lens, counts, held, F = s.lens.long(), s.counts.long(), s.held.long(), s.free_count.long()
    target = (lens + counts + page - 1) // page
    need, surplus = (target - held).clamp(min=0), (held - target).clamp(min=0)
    sums = need.cumsum(0)
    granted = (need == 0) | (sums <= F)
    need = need * granted
    taken = need.sum()
    col = torch.arange(stride, device="cuda")[None, :]
    take = granted[:, None] & (col >= held[:, None]) & (col < target[:, None])
    which = F - 1 - (need.cumsum(0) - need)[:, None] - (col - held[:, None])
    given = (col >= target[:, None]) & (col < held[:, None])
    to = torch.where(given, F - taken + (surplus.cumsum(0) - surplus)[:, None] + col - target[:, None], P)
    free = torch.cat([s.free, s.free[:1]])
    table = torch.where(take, s.free[which.clamp(0, P - 1)], s.table)
    free[to.reshape(-1)] = table.reshape(-1)
    s.free.copy_(free[:P])
    s.table.copy_(torch.where(given, -1, table))
    s.held.copy_(torch.where(granted, target, held))
    s.free_count.copy_(F - taken + surplus.sum())
    s.row_start[1:] = counts.cumsum(0)
    s.granted.copy_(granted)
    row, req, node = _place(s, s.slots.numel())
    at = lens[req] + node
    slot = s.table.reshape(-1)[req * stride + (at // page).clamp(max=stride - 1)] * page + at % page
    s.slots.copy_(torch.where((row < s.row_start[-1]) & granted[req], slot, -1))


def _padded(s, packed, fill):
    """[rows] -> [requests][nodes]"""
    node = torch.arange(s.case["nodes"], device="cuda")[None, :]
    row = s.row_start[:-1].long()[:, None] + node
    real = row < s.row_start[1:].long()[:, None]
    return torch.where(real, packed[row.clamp(max=s.rows - 1)], fill), real


def _plain_plan(s):
    n = s.case["nodes"]
    parents, real = _padded(s, s.parents, -1)
    node = torch.arange(n, device="cuda")
    # I + A, halved; its n-th power is positive exactly where a way of less than n steps leads upwards
    step = ((parents[:, :, None] == node) | (node[:, None] == node)[None]).double() * 0.5
    up = torch.linalg.matrix_power(step, max(1, n)) > 0
    words = s.masks.shape[1]
    bits = torch.zeros((*up.shape[:2], 32 * words), dtype=torch.int64, device="cuda")
    bits[:, :, :n] = up
    packed = (bits.view(*up.shape[:2], words, 32) << torch.arange(32, device="cuda")).sum(-1)
    row, req, at = _place(s, s.rows)
    s.masks.copy_((packed - ((packed >> 31) << 32))[req, at])
    s.positions.copy_(s.lens[req] + up.sum(-1)[req, at] - 1)


def _pool_rows(pool):
    """A view with page and offset in front of what a position holds: [pages][offset][...]"""
    return pool.permute(2, 5, 0, 1, 3, 4, 6)


def _plain_append(s):
    page, kv, d = s.case["page"], *HEADS[s.case["heads"]][1:]
    rows = torch.stack([s.k, s.v], 1).view(s.rows, 1, 2, kv, d // 16, 16)
    slot = s.slots.long()
    _pool_rows(s.pool)[slot // page, slot % page] = rows


def _seen(s, S):
    """[requests][nodes][S]: whether a node sees a position"""
    words = _padded_words(s)
    t = torch.arange(S, device="cuda")[None, :] - s.lens.long()[:, None]
    j = t.clamp(0, 32 * s.masks.shape[1] - 1)
    word = torch.gather(words, 2, (j // 32)[:, None, :].expand(-1, words.shape[1], -1))
    bit = ((word >> (j % 32)[:, None, :]) & 1) == 1
    count = (s.row_start[1:] - s.row_start[:-1]).long()
    return (t < 0)[:, None, :] | ((t >= 0) & (t < count[:, None]))[:, None, :] & bit


def _padded_words(s):
    node = torch.arange(s.case["nodes"], device="cuda")[None, :]
    row = (s.row_start[:-1].long()[:, None] + node).clamp(max=s.rows - 1)
    return s.masks[row].long()


def _plain_attention(s):
    page, (q, kv, d) = s.case["page"], HEADS[s.case["heads"]]
    R, n, S, G = s.case["requests"], s.case["nodes"], s.stride * page, q // kv
    got = s.pool[0][:, s.table.long().clamp(min=0)]        # [2][R][pages][kv][d / 16][page][16]
    got = got.permute(0, 1, 3, 2, 5, 4, 6).reshape(2, R, kv, S, d).float()
    ends = s.lens.long() + s.row_start[1:].long() - s.row_start[:-1].long()
    late = torch.arange(S, device="cuda")[None, :] >= ends[:, None]
    got.masked_fill_(late[None, :, None, :, None], 0.0)
    row = (s.row_start[:-1].long()[:, None] + torch.arange(n, device="cuda")[None, :]).clamp(max=s.rows - 1)
    qq = s.q[row].view(R, n, kv, G, d).permute(0, 2, 1, 3, 4).reshape(R, kv, n * G, d).float()
    seen = _seen(s, S).repeat_interleave(G, 1)[:, None]
    score = torch.matmul(qq, got[0].transpose(2, 3).contiguous()) / math.sqrt(d)
    score.masked_fill_(~seen, -math.inf)
    score = score.sub_(score.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    o = torch.matmul(score, got[1]) / score.sum(-1, keepdim=True).clamp(min=1e-30)
    o = o.view(R, kv, n, G, d).permute(0, 2, 1, 3, 4).reshape(R, n, q, d)
    _, req, at = _place(s, s.rows)
    s.out.copy_(o[req, at])


def _plain_accept(s):
    n, page = s.case["nodes"], s.case["page"]
    parents, real = _padded(s, s.parents, -1)
    tokens, _ = _padded(s, s.tokens, -1)
    picks, _ = _padded(s, s.picks, -1)
    words = _padded_words(s)
    node = torch.arange(n, device="cuda")
    up = ((words[:, :, node // 32] >> (node % 32)) & 1).bool() & real[:, :, None]          # [request][node][ancestor]
    depth = up.sum(-1) - 1
    fits = real & (parents >= 0) & (tokens == torch.gather(picks, 1, parents.long().clamp(min=0)))
    # an earlier child of the same parent that fits too goes first
    twin = (parents[:, :, None] == parents[:, None, :]) & fits[:, None, :] & (node[None, :] < node[:, None])[None]
    fits = (fits & ~twin.any(-1)) | (real & (node == 0)[None])
    good = real & ((up & ~fits[:, None, :]).sum(-1) == 0)
    count = good.sum(-1)
    path = torch.full((good.shape[0], n + 1), -1, dtype=torch.int64, device="cuda")
    path.scatter_(1, torch.where(good, depth, n), node[None, :].expand_as(depth))
    path = path[:, :n]
    last = path.gather(1, (count - 1).clamp(min=0)[:, None])
    s.accepted.copy_(count)
    s.path.copy_(torch.where(node[None] < count[:, None], path, -1))
    s.next.copy_(torch.where(count > 0, picks.gather(1, last.clamp(min=0))[:, 0], -1))
    s.lens_out.copy_(s.lens + count)
    row = (s.row_start[:-1].long()[:, None] + node[None]).clamp(max=s.rows - 1)
    from_row = torch.where(node[None] < count[:, None], s.row_start[:-1].long()[:, None] + path.clamp(min=0), row)
    # (rows past a request's last are another's: they are left to that one)
    row, from_row = torch.where(real, row, row[:, :1]), torch.where(real, from_row, from_row[:, :1])
    to, at = s.slots[row].long().view(-1), s.slots[from_row].long().view(-1)
    view = _pool_rows(s.pool)
    view[to // page, to % page] = view[at // page, at % page]


def run(s):
    op = s.case["op"]
    if own:
        import paper_2604_23553_amd as cf
        stream = torch.cuda.current_stream().cuda_stream
        if op == "tables":
            cf.cfpp_page_tables(s.pages, s.batch, s.counts, s.held, s.free, s.free_count, s.granted, stream)
        elif op == "plan":
            cf.cfpp_tree_plan(s.pages, s.batch, HEADS[s.case["heads"]][0], stream)
        elif op == "append":
            cf.cfpp_page_append(s.pages, s.pool[0], s.k, s.v, s.slots, s.rows, stream=stream)
        elif op == "attention":
            cf.cfpp_tree_attention(s.pages, s.pool[0], s.batch, s.q, HEADS[s.case["heads"]][0], s.out, stream=stream)
        else:
            cf.cfpp_tree_accept(s.pages, s.pools, s.batch, s.tokens, s.picks, s.accepted, s.path, s.next, s.lens_out, stream)
    elif op == "tables":
        _plain_tables(s)
    elif op == "plan":
        _plain_plan(s)
    elif op == "append":
        _plain_append(s)
    elif op == "attention":
        _plain_attention(s)
    else:
        _plain_accept(s)
    if op == "tables":
        return {"table": s.table, "held": s.held, "free": s.free, "free_count": s.free_count, "row_start": s.row_start, "slots": s.slots, "granted": s.granted}
    if op == "plan":
        return {"masks": s.masks, "positions": s.positions}
    if op == "append":
        return {"pool": s.pool}
    if op == "attention":
        return {"out": s.out}
    return {"accepted": s.accepted, "path": s.path, "next": s.next, "lens": s.lens_out, "pool": s.pool}


# ---- the same in 64 bits, one request after the other ------------------------------------------------
def exact(case, seed):
    if case["op"] in ("tables", "plan"):
        return None                                        # (whole numbers)
    global own
    before, own = own, False
    s = prepare(case, seed)
    own = before
    lens, counts = _sizes(case)
    page, (q, kv, d) = case["page"], HEADS[case["heads"]]
    slots, starts = s.slots.tolist(), s.row_start.tolist()
    if case["op"] == "append":
        pool = s.pool.double()
        for row, slot in enumerate(slots):
            pool[0, 0, slot // page, :, :, slot % page] = s.k[row].view(kv, d // 16, 16).double()
            pool[0, 1, slot // page, :, :, slot % page] = s.v[row].view(kv, d // 16, 16).double()
        return {"pool": pool}
    if case["op"] == "accept":
        pool, parents, tokens, picks = s.pool.double(), s.parents.tolist(), s.tokens.tolist(), s.picks.tolist()
        for r in range(case["requests"]):
            a, cur, path = starts[r], 0, [0]
            while True:
                child = [i for i in range(cur + 1, counts[r]) if parents[a + i] == cur and tokens[a + i] == picks[a + cur]]
                if not child:
                    break
                cur = child[0]
                path.append(cur)
            for j, i in enumerate(path):
                to, at = slots[a + j], slots[a + i]
                pool[:, :, to // page, :, :, to % page] = pool[:, :, at // page, :, :, at % page]
        return {"accepted": None, "path": None, "next": None, "lens": None, "pool": pool}
    out = torch.zeros((s.rows, q, d), dtype=torch.float64, device="cuda")
    for r in range(case["requests"]):
        a, n, S = starts[r], counts[r], lens[r] + counts[r]
        got = s.pool[0][:, s.table[r, :_pages_of(S, page)].long()].permute(0, 2, 1, 4, 3, 5).reshape(2, kv, -1, d)[:, :, :S].double()
        bits = torch.zeros((n, n), dtype=torch.bool, device="cuda")
        for j in range(n):
            bits[:, j] = (s.masks[a:a + n, j // 32] >> (j % 32)) & 1 != 0
        qq = s.q[a:a + n].double().view(n, kv, q // kv, d)
        for h in range(kv):
            score = (qq[:, h].reshape(-1, d) @ got[0, h].t().contiguous() / math.sqrt(d)).view(n, q // kv, S)
            score[:, :, lens[r]:].masked_fill_(~bits[:, None, :], -math.inf)
            out[a:a + n].view(n, kv, q // kv, d)[:, h] = torch.softmax(score, -1) @ got[1, h]
    return {"out": out}
