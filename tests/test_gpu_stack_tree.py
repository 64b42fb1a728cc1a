"""A stack's pass over drafted trees on a paged cache (cfpp_stack_tree) against the CPU oracle, which takes one decode step per node
along every path, and the loop of drafting and checking against plain generation."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2604_23553_amd as cf
import synth
from tests import tree_ref
from tests.parity import assert_block_close, errors

pytestmark = pytest.mark.gpu

H512 = synth.ModelShape(512, 8, 64, 16, 2048, n_layers=3, name="neox-h512-x3")
H1280 = synth.ModelShape(1280, 16, 80, 20, 5120, n_layers=2, name="neox-h1280-x2")
H1024 = synth.ModelShape(1024, 8, 128, 32, 4096, n_layers=2, name="neox-h1024-x2")


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def i32(a):
    return dev(np.asarray(a, dtype=np.int32))


class Model:
    """A context with its packed layers, and pools of pages with everything a step needs."""

    def __init__(self, shape, requests, page, n_pages, max_rows, max_nodes, seed, max_seq=512):
        self.shape, self.page, self.n_pages, self.R, self.max_rows, self.max_nodes = shape, page, n_pages, requests, max_rows, max_nodes
        L, H, d = shape.n_layers, shape.n_heads, shape.head_dim
        self.cfg = cf.Config.from_shape(shape, max_seq, 1, L)
        self.ws = [synth.layer_weights(shape, seed, l) for l in range(L)]
        u8 = dict(dtype=torch.uint8, device="cuda")
        self.packed, self.keep = [], []
        for w in self.ws:
            t = {n: dev(w[n]) for n in cf.binding.LAYER_TENSORS}
            p = torch.empty(cf.cfpp_packed_layer_bytes(self.cfg), **u8)
            cf.cfpp_pack_layer(self.cfg, t, p, torch.cuda.current_stream().cuda_stream)
            torch.cuda.synchronize()
            self.packed.append(p)
        self.workspace = torch.empty(cf.cfpp_workspace_bytes(self.cfg), **u8)
        self.ctx = cf.cfpp_create(self.cfg, self.workspace, self.workspace.numel())
        self.pages = cf.Pages(n_pages, page, H, d)
        self.pools = [torch.full((2, n_pages, H, d // 16, page, 16), float("nan"), dtype=torch.float16, device="cuda") for _ in range(L)]
        self.stride = n_pages
        z = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
        R, words = requests, (max_nodes + 31) // 32
        self.lens, self.counts, self.row_start, self.table, self.held = z(R), z(R), z(R + 1), z(R, self.stride), z(R)
        self.free, self.free_count, self.granted = torch.randperm(n_pages, dtype=torch.int32, device="cuda"), i32([n_pages]), z(R)
        self.slots, self.parents, self.masks, self.positions = z(max_rows), z(max_rows), z(max_rows, words), z(max_rows)
        self.tokens, self.picks, self.accepted, self.path, self.next = z(max_rows), z(max_rows), z(R), z(R, max_nodes), z(R)
        self.plan = torch.empty(cf.cfpp_tree_plan_bytes(self.pages, H, R, max_rows, max_nodes), **u8)
        self.scratch = torch.full((cf.cfpp_tree_scratch_bytes(self.cfg, max_rows),), 0xFF, **u8)
        self.x = torch.full((max_rows, shape.hidden), float("nan"), dtype=torch.float16, device="cuda")
        self.out = torch.full_like(self.x, 7.0)
        self.batch = cf.TreeBatch.of(max_nodes, self.lens, self.row_start, self.table, self.slots, self.parents, self.masks, self.positions, self.plan)
        torch.cuda.synchronize()

    def close(self):
        torch.cuda.synchronize()
        cf.cfpp_destroy(self.ctx)

    def enqueue_tables(self):
        s = torch.cuda.current_stream().cuda_stream
        cf.cfpp_page_tables(self.pages, self.batch, self.counts, self.held, self.free, self.free_count, self.granted, s)
        cf.cfpp_tree_plan(self.pages, self.batch, self.shape.n_heads, s)

    def enqueue_stack(self):
        cf.cfpp_stack_tree(self.ctx, self.packed, self.pools, self.pages, self.batch, self.x, self.out, self.scratch, self.scratch.numel(),
                           torch.cuda.current_stream().cuda_stream)

    def enqueue_accept(self):
        cf.cfpp_tree_accept(self.pages, self.pools, self.batch, self.tokens, self.picks, self.accepted, self.path, self.next, self.lens,
                            torch.cuda.current_stream().cuda_stream)

    def set_trees(self, trees):
        self.trees = trees
        self.counts.copy_(i32([len(t) for t in trees]))
        p = np.full(self.max_rows, -1, dtype=np.int32)
        p[:sum(len(t) for t in trees)] = sum(trees, [])
        self.parents.copy_(i32(p))

    def fill_cache(self, lens, seed):
        """Cached rows of every request, by cfpp_page_append; as [layer][request] arrays K, V [H, len, d] too."""
        H, d = self.shape.n_heads, self.shape.head_dim
        self.lens.zero_()
        self.counts.copy_(i32(lens))
        s = torch.cuda.current_stream().cuda_stream
        rows = sum(lens)
        slots, start = torch.empty(max(rows, 1), dtype=torch.int32, device="cuda"), torch.zeros(self.R + 1, dtype=torch.int32, device="cuda")
        first = cf.TreeBatch.of(1, self.lens, start, self.table, slots)
        cf.cfpp_page_tables(self.pages, first, self.counts, self.held, self.free, self.free_count, self.granted, s)
        torch.cuda.synchronize()
        assert (self.granted.cpu().numpy() == 1).all()
        rng = np.random.default_rng(seed)
        kvs = []
        for pool in self.pools:
            k, v = (rng.standard_normal((max(rows, 1), H, d)).astype(np.float16) for _ in range(2))
            cf.cfpp_page_append(self.pages, pool, dev(k), dev(v), slots, rows, None, s)
            ends = np.cumsum([0] + list(lens))
            kvs.append([tuple(np.ascontiguousarray(x[ends[r]:ends[r + 1]].transpose(1, 0, 2)) for x in (k, v)) for r in range(self.R)])
        torch.cuda.synchronize()
        self.lens.copy_(i32(lens))
        return kvs

    def row(self, layer, slot):
        """K and V, [2][H][d], in a slot"""
        return self.pools[layer][:, slot // self.page, :, :, slot % self.page].reshape(2, self.shape.n_heads, self.shape.head_dim).cpu().numpy()


def check_step(orc, m, kvs, lens, X, got):
    """Every node of every request against the oracle's steps along its path; the rows in its slots; rows without a slot."""
    starts, slots = m.row_start.cpu().numpy(), m.slots.cpu().numpy()
    H, d, L = m.shape.n_heads, m.shape.head_dim, m.shape.n_layers
    for r, parents in enumerate(m.trees):
        done = set()
        for leaf in sorted(range(len(parents)), key=lambda i: -i):
            if leaf in done:
                continue
            path = [leaf]
            while 0 <= parents[path[-1]] < path[-1]:
                path.append(parents[path[-1]])
            path.reverse()
            cap = lens[r] + len(path)
            Ks, Vs = [], []
            for l in range(L):
                K, V = (np.zeros((H, cap, d), dtype=np.float16) for _ in range(2))
                K[:, :lens[r]], V[:, :lens[r]] = kvs[l][r]
                Ks.append(K)
                Vs.append(V)
            want, _ = orc.prefill(m.shape, m.ws, Ks, Vs, lens[r], X[starts[r] + np.array(path)])
            for j, i in enumerate(path):
                assert_block_close(got[starts[r] + i], want[j], f"request {r}, node {i}")
                if i not in done:
                    for l in range(L):
                        e = errors(m.row(l, int(slots[starts[r] + i])), np.stack([Ks[l][:, lens[r] + j], Vs[l][:, lens[r] + j]]))
                        assert e[0] <= 2e-2 and e[1] <= 5e-3, f"K and V of request {r}, node {i}, layer {l}: {e}"
                done.add(i)
    total = int(starts[-1])
    assert (got[total:] == 7.0).all()


@pytest.mark.parametrize("shape,lens,sizes,page", [
    (H512, [37], [1], 16), (H512, [0], [9], 16), (H512, [20, 0, 65], [7, 3, 12], 48), (H1280, [33, 5], [11, 6], 16), (H1024, [10, 40], [20, 9], 32),
    (H512, [15, 70, 3], [40, 33, 1], 16), (H1280, [64], [70], 64), (H1024, [12, 3], [100, 2], 16),
])
def test_stack_tree(orc, shape, lens, sizes, page):
    rng = np.random.default_rng([shape.hidden, sum(sizes)])
    n_pages = sum(tree_ref.pages_for(a + b, page) for a, b in zip(lens, sizes)) + 2
    print(f"[case] {shape.name} lens={lens} sizes={sizes} page={page}", flush=True)
    m = Model(shape, len(lens), page, n_pages, sum(sizes) + 3, max(sizes), 3)
    try:
        kvs = m.fill_cache(lens, 5)
        m.set_trees([tree_ref.random_tree(rng, n, wide=n < 50) for n in sizes])
        X = synth.x_input(shape, 11, batch=sum(sizes))
        m.x[:sum(sizes)] = dev(X)
        m.enqueue_tables()
        m.enqueue_stack()
        torch.cuda.synchronize()
        cf.cfpp_device_error(m.ctx)
        check_step(orc, m, kvs, lens, X, m.out.cpu().numpy())
    finally:
        m.close()


def test_a_chain_is_a_prompt():
    """70 nodes in a chain behind an empty cache are a prompt of 70 tokens: outputs and K and V rows as cfpp_stack_prefill_gemm's."""
    shape, T = H1280, 70
    m = Model(shape, 1, 16, 6, T, T, 3)
    try:
        m.set_trees([[i - 1 for i in range(T)]])
        X = synth.x_input(shape, 12, batch=T)
        m.x.copy_(dev(X))
        m.enqueue_tables()
        m.enqueue_stack()
        u8 = dict(dtype=torch.uint8, device="cuda")
        kv = [torch.empty(cf.cfpp_kv_layer_bytes(m.cfg), **u8) for _ in range(shape.n_layers)]
        n = cf.cfpp_prefill_scratch_bytes(m.cfg, 128)
        out, scratch = torch.zeros_like(m.x), torch.empty(n, **u8)
        cf.cfpp_stack_prefill_gemm(m.ctx, m.packed, kv, m.x, 0, T, 0, out, scratch, n, 128, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        for t in range(T):
            assert_block_close(m.out[t].cpu().numpy(), out[t].cpu().numpy(), f"token {t}")
        slots = m.slots.cpu().numpy()
        for l in range(shape.n_layers):
            flat = kv[l].view(torch.float16).view(2, shape.n_heads, shape.head_dim // 16, m.cfg.max_seq, 16).cpu().numpy()
            for t in range(T):
                e = errors(m.row(l, int(slots[t])), flat[:, :, :, t].reshape(2, shape.n_heads, shape.head_dim))
                assert e[0] <= 2e-2 and e[1] <= 5e-3
    finally:
        m.close()


def test_refused_requests_and_far_positions(orc):
    """A request without pages keeps its rows' outputs as they were, the others are served; a position past the rotary table raises the flag."""
    shape = H512
    m = Model(shape, 3, 16, 4, 40, 12, 3, max_seq=64)
    try:
        kvs = m.fill_cache([20, 0, 10], 6)                  # 3 of 4 pages
        rng = np.random.default_rng(9)
        m.set_trees([tree_ref.random_tree(rng, 12), tree_ref.random_tree(rng, 12), tree_ref.random_tree(rng, 5)])
        m.counts.copy_(i32([12, 12, 5]))
        m.lens.copy_(i32([20, 10, 10]))                     # (the second one asks for two pages)
        X = synth.x_input(shape, 13, batch=29)
        m.x[:29] = dev(X)
        m.enqueue_tables()
        m.enqueue_stack()
        torch.cuda.synchronize()
        cf.cfpp_device_error(m.ctx)
        assert list(m.granted.cpu().numpy()) == [1, 0, 1]
        got = m.out.cpu().numpy()
        assert (got[12:24] == 7.0).all()
        m.trees[1] = []
        check_step(orc, m, kvs, [20, 10, 10], X, got)
        m.positions[3] = 64
        m.enqueue_stack()
        with pytest.raises(cf.CfppError) as e:
            cf.cfpp_device_error(m.ctx)
        assert e.value.status == -6
    finally:
        m.close()


def test_refusals_of_the_stack():
    shape = H512
    m = Model(shape, 2, 16, 4, 20, 8, 3)
    try:
        s = torch.cuda.current_stream().cuda_stream

        def status(**change):
            a = dict(packed=m.packed, pools=m.pools, pages=m.pages, batch=m.batch, x=m.x, out=m.out, scratch=m.scratch, n=m.scratch.numel())
            a.update(change)
            with pytest.raises(cf.CfppError) as e:
                cf.cfpp_stack_tree(m.ctx, a["packed"], a["pools"], a["pages"], a["batch"], a["x"], a["out"], a["scratch"], a["n"], s)
            return e.value.status

        assert status(n=m.scratch.numel() - 256) == -3
        assert status(scratch=m.scratch.data_ptr() + 16) == -1 and status(scratch=0) == -1
        assert status(out=m.x) == -1 and status(x=0) == -1 and status(out=m.out.data_ptr() + 2) == -1
        assert status(pools=[m.pools[0], 0, m.pools[2]]) == -1 and status(packed=[0] + m.packed[1:]) == -1
        assert status(pages=cf.Pages(4, 16, 4, 64)) == -1 and status(pages=cf.Pages(4, 24, 8, 64)) == -2
        for name in ("lens", "row_start", "block_table", "slots", "positions", "masks", "plan"):
            b = cf.TreeBatch.from_buffer_copy(m.batch)
            setattr(b, name, 0)
            assert status(batch=b) == -1, name
        b = cf.TreeBatch.from_buffer_copy(m.batch)
        b.max_rows, b.plan_bytes = 4097, 1 << 40
        assert status(batch=b) == -2
        assert cf.cfpp_tree_scratch_bytes(m.cfg, 0) == 0 and cf.cfpp_tree_scratch_bytes(m.cfg, 4097) == 0 < cf.cfpp_tree_scratch_bytes(m.cfg, 4096)
    finally:
        m.close()


def test_drafting_and_checking_generates_what_plain_steps_generate():
    """Greedy tokens from steps of one token on the library's own cache, then the same ones from trees that hold some of them among wrong drafts: tables,
    plan, stack, logits, acceptance, in a graph that is replayed with new trees."""
    from paper_2604_23553_amd.harness import DeviceStack
    shape, vocab, n_tokens, prompt = H512, 1000, 40, [5, 77, 900, 3, 410]
    rng = np.random.default_rng(17)
    ds = DeviceStack(shape, 128, 1, shape.n_layers)
    head, embed = synth.lm_head(shape, 3, vocab), synth.embedding(shape, 3, vocab)
    try:
        for l in range(shape.n_layers):
            ds.load_layer(l, synth.layer_weights(shape, 3, l))
        ds.load_lm(head, embed)
        ds.set_tokens(prompt, 0)
        known = list(prompt)
        for pos in range(len(prompt) + n_tokens):
            ds.set_tokens(known[:pos + 1], pos)
            ds.generate_step()
            ds.check()
            if pos + 1 >= len(known):
                known.append(int(ds.tokens[pos + 1]))
    finally:
        ds.close()
    m = Model(shape, 1, 16, 10, 12, 12, 3, max_seq=128)
    lm_t = {n: dev(a) for n, a in (("embed", embed), ("lnf_g", head["lnf_g"]), ("lnf_b", head["lnf_b"]), ("w_lm", head["w_lm"]))}
    lm = cf.Lm.of(lm_t["embed"], lm_t["lnf_g"], lm_t["lnf_b"], lm_t["w_lm"], vocab)
    side = torch.cuda.Stream()
    try:
        picked, at = torch.zeros(129, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")

        def step():
            s = torch.cuda.current_stream().cuda_stream
            m.x.copy_(lm_t["embed"][m.tokens.long()])
            m.enqueue_tables()
            m.enqueue_stack()
            at.zero_()
            for i in range(m.max_rows):                     # (the pick behind row i goes to picked[i + 1])
                cf.cfpp_lm_next(m.ctx, lm, m.out[i], picked, at, None, s)
            m.picks.copy_(picked[1:1 + m.max_rows])
            m.enqueue_accept()

        # the prompt but its last token, a chain: its rows are in their places, and nothing is left to be accepted
        first = prompt[:-1]
        t = np.zeros(m.max_rows, dtype=np.int32)
        t[:len(first)] = first
        m.tokens.copy_(i32(t))
        m.set_trees([[i - 1 for i in range(len(first))]])
        m.x.copy_(lm_t["embed"][m.tokens.long()])
        m.enqueue_tables()
        m.enqueue_stack()
        torch.cuda.synchronize()
        m.lens.fill_(len(first))
        got, graph = list(prompt), None
        while len(got) < len(prompt) + n_tokens:
            # the tree: the last token, which is not cached, then right and wrong drafts
            cached = int(m.lens[0])
            parents, tokens = [-1], [got[cached]]
            ahead, base = len(got), 0
            for k in range(int(rng.integers(0, 4))):        # right ones
                parents.append(base)
                tokens.append(known[ahead + k] if ahead + k < len(known) else 1)
                base = len(parents) - 1
            while len(parents) < m.max_rows - 1:            # wrong ones
                p = int(rng.integers(0, len(parents)))
                parents.append(p)
                tokens.append(int(rng.integers(0, vocab)))
            t = np.zeros(m.max_rows, dtype=np.int32)
            t[:len(tokens)] = tokens
            m.tokens.copy_(i32(t))
            m.set_trees([parents])
            m.out.fill_(0)
            torch.cuda.synchronize()
            if graph is None:
                with torch.cuda.stream(side):
                    step()
                side.synchronize()
            else:
                graph.replay()
                torch.cuda.synchronize()
            cf.cfpp_device_error(m.ctx)
            n, path = int(m.accepted[0]), m.path[0].cpu().numpy()
            assert n >= 1
            got = got[:cached] + [tokens[i] for i in path[:n]] + [int(m.next[0])]
            assert int(m.lens[0]) == len(got) - 1
            if graph is None:
                before = m.lens.clone(), m.held.clone(), m.free.clone(), m.free_count.clone()
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=side):
                    step()
                for t, b in zip((m.lens, m.held, m.free, m.free_count), before):
                    t.copy_(b)
        assert got[:len(prompt) + n_tokens] == known[:len(prompt) + n_tokens]
    finally:
        m.close()
