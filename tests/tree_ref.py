"""Plain implementations, in 64 bits and one request after the other, of the operators for drafted trees over a paged cache."""
import numpy as np


def pages_for(n, page):
    return -(-n // page)


class Allocator:
    """cfpp_page_tables: pages from the end of the free list, those given back behind what is left."""

    def __init__(self, n_pages, page, requests, stride, rng):
        self.page, self.n_pages, self.stride = page, n_pages, stride
        self.free = [int(p) for p in rng.permutation(n_pages)]
        self.tables = [[] for _ in range(requests)]

    def step(self, lens, counts, max_rows):
        """(granted, row_start, slots)"""
        F = len(self.free)
        ends, row = [], 0
        for n in counts:
            row += max(n, 0)
            ends.append(row)
        granted, asked, taken, back = [], 0, 0, []
        for r, (length, n) in enumerate(zip(lens, counts)):
            held = len(self.tables[r])
            fits = length >= 0 and n >= 0 and pages_for(length + n, self.page) <= self.stride and ends[r] <= max_rows
            target = pages_for(length + n, self.page) if fits else held
            need = max(target - held, 0)
            asked += need
            ok = fits and (need == 0 or asked <= F)
            granted.append(int(ok))
            if not ok:
                continue
            for _ in range(need):
                self.tables[r].append(self.free[F - 1 - taken])
                taken += 1
            back += self.tables[r][target:]
            del self.tables[r][target:]
        self.free = self.free[:F - taken] + back
        starts = [0] + [min(e, max_rows) for e in ends]
        slots = np.full(max_rows, -1, dtype=np.int32)
        for r, ok in enumerate(granted):
            if ok:
                for i in range(counts[r]):
                    at = lens[r] + i
                    slots[starts[r] + i] = self.tables[r][at // self.page] * self.page + at % self.page
        return granted, starts, slots


def ancestors(parents):
    """bool [n][n]: node i sees node j."""
    n = len(parents)
    up = np.zeros((n, n), dtype=bool)
    for i, p in enumerate(parents):
        if 0 <= p < i:
            up[i] = up[p]
        up[i, i] = True
    return up


def mask_words(up, words):
    n = up.shape[0]
    bits = np.zeros((n, 32 * words), dtype=np.uint64)
    bits[:, :up.shape[1]] = up
    packed = (bits.reshape(n, words, 32) << np.arange(32, dtype=np.uint64)).sum(-1)
    return packed.astype(np.uint32).view(np.int32)


def random_tree(rng, n, wide=True):
    return [-1] + [int(rng.integers(0, i) if wide else rng.integers(max(0, i - 3), i)) for i in range(1, n)]


def slot_row(pool, slot, page):
    """[2, heads, d] of a pool [2][pages][heads][d / 16][page][16]"""
    _, _, H, s, _, _ = pool.shape
    return pool[:, slot // page, :, :, slot % page].reshape(2, H, 16 * s)


def attend(q, k, v, seen):
    """q [n, H, d], k, v [S, Hkv, d], seen bool [n, S]: (outputs [n, H, d], bound on what an evaluation in 32 bits may be off).

    The bound: a score is a sum of d products in 32 bits, scaled, so off by at most ds = (d + 8) 2^-24 sum |q k| / sqrt(d); a weight
    by the factor exp(2 ds) (its own score's and the maximum's) and some steps of exp2 and of its two halves (8 * 2^-22 in all); an
    output, a ratio of sums of weights, by twice that and by the sums' own roundings, S 2^-23, times the largest |v| seen in its
    dimension.  Keys whose score is not finite have a weight of zero exactly, or make the output no number."""
    n, H, d = q.shape
    S, G = k.shape[0], H // k.shape[1]
    out, off = np.zeros((n, H, d)), np.zeros((n, H, d))
    with np.errstate(all="ignore"):
        for h in range(H):
            kk, vv = k[:, h // G], v[:, h // G]
            for i in range(n):
                at = np.nonzero(seen[i])[0]
                if not len(at):
                    continue
                s = kk[at] @ q[i, h] / np.sqrt(d)
                p = np.exp(s - (s.max() if not np.isnan(s).any() else np.nan))
                if s.max() == -np.inf:
                    p = np.full_like(s, np.nan)
                out[i, h] = (p[:, None] * vv[at]).sum(0) / p.sum()
                sizes = np.abs(kk[at]) @ np.abs(q[i, h])
                ds = (d + 8) * 2.0 ** -24 * sizes[np.isfinite(sizes)].max(initial=0.0) / np.sqrt(d)
                off[i, h] = np.abs(vv[at]).max(0) * (2 * (np.expm1(2 * ds) + 2.0 ** -19) + S * 2.0 ** -23)
    return out, off


def accept(parents, tokens, picks):
    path = [0]
    while True:
        child = [i for i in range(len(parents)) if i > path[-1] and parents[i] == path[-1] and tokens[i] == picks[path[-1]]]
        if not child:
            return path
        path.append(child[0])
