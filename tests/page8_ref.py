"""Plain implementations, in 64 bits, of a paged cache in 8 bits and of sampling."""
import numpy as np

from tests import tree_ref

INT8, E4M3 = 3, 4
MOST = {INT8: 127.0, E4M3: 448.0}


def e4m3_values():
    """What the 256 codes stand for: sign, four bits of exponent (bias 7), three of fraction; 0x7f and 0xff are no numbers."""
    v = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v[c] = np.nan if c & 127 == 127 else -x if c >= 128 else x
    return v


E4M3_VALUES = e4m3_values()


def code_values(codes, type):
    return codes.view(np.int8).astype(np.float64) if type == INT8 else E4M3_VALUES[codes]


def quantise(rows, type):
    """fp16 [..., d]: (codes uint8, a fp16 [...])"""
    x = rows.astype(np.float64)
    a = np.abs(x).max(-1)
    good = np.isfinite(a)
    with np.errstate(all="ignore"):
        y = np.where((good & (a > 0))[..., None], MOST[type] * x / a[..., None], 0.0)
    if type == INT8:
        codes = np.rint(y).astype(np.int8).view(np.uint8)
    else:
        e = np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6)))
        step = np.exp2(e - 3)
        z = np.rint(y / step) * step
        positive = E4M3_VALUES[:127]
        codes = (np.searchsorted(positive, np.abs(z)) + 128 * np.signbit(x)).astype(np.uint8)
        assert np.array_equal(np.abs(E4M3_VALUES[codes]), np.abs(z))
        codes[~good] = 0
    with np.errstate(over="ignore"):
        return codes, np.where(good, a, np.nan).astype(np.float16)


class Pool:
    """Bytes [pages][heads][page / 16][32 d + 64]; what was never written is `poison`"""

    def __init__(self, n_pages, page, heads, d, type, poison=0x7F):
        self.page, self.heads, self.d, self.type, self.n_pages = page, heads, d, type, n_pages
        self.bytes = np.full((n_pages, heads, page // 16, 32 * d + 64), poison, dtype=np.uint8)

    def where(self, t):
        """Places of a position's K codes, V codes, and of the first bytes of its two a, inside a granule"""
        dim = np.arange(self.d)
        k = (t // 4) * 4 * self.d + (dim // 16) * 64 + (t % 4) * 16 + dim % 16
        return k, 16 * self.d + dim * 16 + t, 32 * self.d + 2 * t, 32 * self.d + 32 + 2 * t

    def put(self, slot, k, v):
        """Rows fp16 [heads, d]"""
        if not 0 <= slot < self.n_pages * self.page:
            return
        g = self.bytes[slot // self.page, :, slot % self.page // 16]
        at = self.where(slot % 16)
        for rows, codes_at, most_at in ((k, at[0], at[2]), (v, at[1], at[3])):
            codes, a = quantise(rows, self.type)
            g[:, codes_at] = codes
            g[:, most_at:most_at + 2] = a.view(np.uint8).reshape(-1, 2)

    def get(self, slot):
        """Values in 64 bits, [2][heads][d]"""
        g = self.bytes[slot // self.page, :, slot % self.page // 16]
        at = self.where(slot % 16)
        out = []
        for codes_at, most_at in ((at[0], at[2]), (at[1], at[3])):
            a = np.ascontiguousarray(g[:, most_at:most_at + 2]).view(np.float16).astype(np.float64)
            out.append(code_values(np.ascontiguousarray(g[:, codes_at]), self.type) * a / MOST[self.type])
        return np.stack(out)


def attend(q, k, v, seen):
    """As tree_ref.attend, with the bound of an evaluation in 32 bits of scores that are scaled and shifted: s = S ks + e and
    its distance to a reference are rounded at numbers of up to |s| + |e| + 9 in steps of log 2, three roundings of 2^-24 beside those of
    the scale itself, three more of s; e is within 1 of the logarithm of the row's largest |v|."""
    out, off = tree_ref.attend(q, k, v, seen)
    n, H, d = q.shape
    S, G = k.shape[0], H // k.shape[1]
    with np.errstate(all="ignore"):
        for h in range(H):
            kk, vv = k[:, h // G], v[:, h // G]
            for i in range(n):
                at = np.nonzero(seen[i])[0]
                if not len(at):
                    continue
                s = np.abs(kk[at] @ q[i, h]) / np.sqrt(d) * np.log2(np.e)
                most = np.abs(vv[at]).max(-1)
                e = np.clip(np.abs(np.log2(np.where(most > 0, most, 1.0))) + 8.0, 0, 40)
                size = np.where(np.isfinite(s), s, 0).max() + np.where(np.isfinite(e), e, 0).max() + 9.0
                off[i, h] += np.abs(vv[at]).max(0) * 2 * np.expm1(2 * 6 * 2.0 ** -24 * size * np.log(2))
    return out, off


def sample(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, uniform=0.0):
    """One row: a dict with the order, the weights and running sums in it, how many tokens are kept and the place of the token in the order."""
    x = logits.astype(np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    order = np.argsort(-x, kind="stable")
    order = order[x[order] > -np.inf]
    if not len(order):
        return dict(order=order, token=-1, kept=0, prob=0.0)
    top = x[order[0]]
    if top == np.inf:
        x = np.where(x == np.inf, 0.0, -np.inf)
        order, top = order[x[order] == 0.0], 0.0
    if not temperature > 0 or top_k == 1 or top_p <= 0:
        return dict(order=order, token=int(order[0]), kept=1, prob=1.0)
    with np.errstate(over="ignore"):
        w = np.exp((x[order] - top) / np.float64(np.float32(temperature)))
    n = len(order) if top_k <= 0 else min(top_k, len(order))
    sums = np.cumsum(w[:n].astype(np.longdouble))          # (in 64 bits a sum of 2^17 weights may be 2^-37 of itself off)
    kept, target_p = n, None
    if top_p < 1:
        target_p = float(np.float32(top_p)) * sums[-1]
        kept = min(n, 1 + int(np.searchsorted(sums, target_p)))
    if min_p > 0:
        kept = min(kept, max(1, int((w[:n] >= min(float(np.float32(min_p)), 1.0)).sum())))
    u = float(np.float32(uniform))
    u = min(u, 1.0) if u > 0 else 0.0
    target = u * sums[kept - 1]
    at = min(int(np.searchsorted(sums[:kept], target, side="right")), kept - 1)
    while w[at] == 0.0 and at > 0:
        at -= 1
    return dict(order=order, token=int(order[at]), kept=kept, prob=w[at] / sums[kept - 1], w=w, sums=sums, target=target, target_p=target_p, n=n)


def sample_off(r):
    """How far a border and its target, each a running sum, may be apart.  A weight is a whole multiple of 2^-44 of its bin's middle, to the nearest, of a
    polynomial 2^-43.5 off: 2^-42 of itself.  The sum of a bin, 4096 at most, or of a token alone is cut off at a multiple of 2^-44 of the middle of the largest weight's bin, which is
    2^(1/64) of that weight at most; what lies behind the bins is less than 2^18 times 2^-64.  The plain form's exponents are 2^-46 off at most where a weight counts."""
    return 2 * (r["sums"][-1] * 2.0 ** -42 + min(len(r["order"]), 4098) * 2.0 ** (1 / 64 - 44))


def check_sample(logits, got, **how):
    """got: (token, prob, kept).  A token or a number of tokens that differs has to have its target next to a border."""
    r = sample(logits, **how)
    token, prob, kept = got
    if "w" not in r:
        assert (token, kept) == (r["token"], r["kept"]) and prob == r["prob"], (got, r["token"], r["kept"], r["prob"])
        return
    off = sample_off(r)
    if kept != r["kept"]:
        assert r["target_p"] is not None and 1 <= kept <= r["n"], (kept, r["kept"])
        before = r["sums"][kept - 2] if kept > 1 else 0.0
        assert before < r["target_p"] + off and r["sums"][kept - 1] > r["target_p"] - off, (kept, r["kept"])
    at = np.nonzero(r["order"] == token)[0]
    assert len(at) == 1 and at[0] < kept, (token, r["token"])
    at = int(at[0])
    if token != r["token"]:
        target = r["target"] / r["sums"][r["kept"] - 1] * r["sums"][kept - 1]
        before = r["sums"][at - 1] if at else 0.0
        assert before <= target + off and r["sums"][at] >= target - off, (token, r["token"], at, kept)
    want = r["w"][at] / r["sums"][kept - 1]
    # the weight, the sum and the quotient, which is rounded to fp32; 2^-149 is the smallest there is
    assert abs(prob - want) <= want * (2.0 ** -24 + 2.0 ** -42 + off / r["sums"][kept - 1]) + 2.0 ** -149, (prob, want)
