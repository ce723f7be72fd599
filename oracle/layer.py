"""Float64 definitions of the attention half of a serving iteration's layer (a
cache's pages, the attention of one new token over them, the norms around a block
and their gradient), written from their formulas with NumPy and plain loops.

Bounds: an ``Err`` carries a value and what a float32 computation of it may be off
by, step by step: each operation adds half a unit of its result (2^-24 relative),
sums of n terms n units of the sum of magnitudes, whatever their order.  Fused
operations round less often than that.
"""
from __future__ import annotations

import numpy as np

from .operators import EPS16, EPS32


# ---------------------------------------------------------------- pages

class Pages:
    """A cache's tables and the contents of its pages, one call at a time, one slot after the other."""

    def __init__(self, table, length, refs, content, page):
        self.table, self.length, self.refs = (np.array(a, np.int64) for a in (table, length, refs))
        self.content = np.array(content)
        self.page = page

    def pages_of(self, n):
        return -(-int(n) // self.page)

    def held(self, s):
        return [int(p) for p in self.table[s, : self.pages_of(self.length[s])]]

    def resize(self, delta):
        """-> (granted, whether a slot was refused)."""
        W = self.table.shape[1]
        for s, by in enumerate(int(x) for x in delta):
            if by < 0:
                left = max(0, int(self.length[s]) + by)
                for i in range(self.pages_of(left), self.pages_of(self.length[s])):
                    self.refs[self.table[s, i]] -= 1
                    self.table[s, i] = -1
                self.length[s] = left
        free = [p for p in range(len(self.refs)) if self.refs[p] == 0]
        shared = self.refs > 1
        granted, refused, full = np.zeros(len(delta), np.uint8), False, False
        for s, by in enumerate(int(x) for x in delta):
            if by <= 0:
                continue
            n, end = int(self.length[s]), int(self.length[s]) + by
            if end > W * self.page:
                refused = True
                continue
            first = self.pages_of(n)
            copies = n % self.page != 0 and shared[self.table[s, first - 1]]
            need = self.pages_of(end) - first + int(copies)
            if need and (full or need > len(free)):
                refused = full = True
                continue
            taken, free = free[:need], free[need:]
            if copies:
                old = self.table[s, first - 1]
                self.content[taken[0]] = self.content[old]
                self.refs[old] -= 1
                first -= 1
            for i, p in enumerate(taken):
                self.table[s, first + i] = p
                self.refs[p] += 1
            self.length[s] = end
            granted[s] = 1
        return granted, refused

    def fork(self, parent):
        """-> whether a parent was out of range."""
        rows, lengths = self.table.copy(), self.length.copy()
        bad = False
        for s, p in enumerate(int(x) for x in parent):
            if p < 0 or p == s:
                continue
            if p >= len(rows):
                bad = True
                continue
            for e in rows[s, : self.pages_of(lengths[s])]:
                self.refs[e] -= 1
            n = self.pages_of(lengths[p])
            self.table[s, : max(n, self.pages_of(lengths[s]))] = -1
            self.table[s, :n] = rows[p, :n]
            for e in rows[p, :n]:
                self.refs[e] += 1
            self.length[s] = lengths[p]
        return bad

    def compact(self):
        live = [p for p in range(len(self.refs)) if self.refs[p] > 0]
        n = len(live)
        holes = [p for p in range(n) if self.refs[p] == 0]
        for src, dst in zip([p for p in live if p >= n], holes):
            self.content[dst] = self.content[src]
            self.refs[dst], self.refs[src] = self.refs[src], 0
            self.table[self.table == src] = dst
        return n

    def copy(self, src, dst):
        """-> whether a pair was left out."""
        names = [int(x) for x in src] + [int(x) for x in dst]
        before, bad = self.content.copy(), False
        for a, b in zip(src, dst):
            if not (0 <= a < len(self.refs) and 0 <= b < len(self.refs)) or names.count(int(b)) != 1:
                bad = True
                continue
            self.content[b] = before[a]
        return bad

    def check(self):
        """Tables and counts agree."""
        refs = np.zeros_like(self.refs)
        for s in range(len(self.length)):
            n = self.pages_of(self.length[s])
            for p in self.table[s, :n]:
                refs[p] += 1
            assert (self.table[s, n:] == -1).all()
        assert (refs == self.refs).all()


def place(c, layer, values, head, token, dim):
    """Element of a page that holds a dimension of a token's key (or value) of a head.  c: page, layers, heads, head_dim,
    size (bytes of an element)."""
    n = 16 // c["size"]
    pieces = -(-c["head_dim"] * c["size"] // 64)
    row = pieces * 4 * n
    at = ((layer * 2 + int(values)) * c["heads"] + head) * c["page"] * row
    at += token // 16 * 16 * row + dim // (4 * n) * 64 * n
    r, d = token % 16, dim % (4 * n)
    if not values:
        return at + (16 * (d // n) + r) * n + d % n
    return at + (16 * (r // 4) + d % 16) * n + 4 * (d // 16) + r % 4


# ---------------------------------------------------------------- attention

def attention(q, k, v, scale, dtype):
    """One slot, one query head: q [D], k and v [n][D] of the tokens it sees -> (out, bound, lse, its bound)."""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    n, D = k.shape
    if n == 0:
        return np.zeros(D), np.zeros(D), -np.inf, 0.0
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        s = scale * (k @ q)
        if (s == -np.inf).all():
            return np.zeros(D), np.zeros(D), -np.inf, 0.0
        top = s.max()
        p = np.exp(s - top)
        out, total = p @ v / p.sum(), p.sum()
        # the exponent: an n-term product sum, the scale's and the base's roundings, a subtraction of values up to
        # the largest score
        size = np.abs(s).max()
        exponent = abs(scale) * (D + 4) * EPS32 * (np.abs(k) @ np.abs(q)).max() + 8 * EPS32 * size
        # the exponential (two units), p's two parts, the sums above and below, and a scaling of two units whenever a
        # maximum grows (once per 16 tokens at most) or parts are joined
        rel = exponent + 4 * EPS32 + (2 * EPS16 * EPS16 if dtype == "bf16" else 0.0) + (n + n / 4 + 512) * EPS32
        bound = 2 * rel * (p @ np.abs(v)) / total + 2 * EPS32 * np.abs(out)
        lse = top + np.log(total)
        return out, bound, lse, rel + 4 * EPS32 * (size + abs(lse) + 1)


# ---------------------------------------------------------------- norms

class Err:
    """A value and a bound on the error of its float32 computation."""

    def __init__(self, v, e=0.0):
        self.v = np.asarray(v, np.float64)
        self.e = np.broadcast_to(np.asarray(e, np.float64), self.v.shape)

    def __add__(self, o):
        v = self.v + o.v
        return Err(v, self.e + o.e + EPS32 * (np.abs(v) + self.e + o.e))

    def __sub__(self, o):
        return self + Err(-o.v, o.e)

    def __mul__(self, o):
        v = self.v * o.v
        e = np.abs(self.v) * o.e + np.abs(o.v) * self.e + self.e * o.e
        return Err(v, e + EPS32 * (np.abs(v) + e))

    def sum(self, axis):
        n = self.v.shape[axis]
        size = (np.abs(self.v) + self.e).sum(axis=axis, keepdims=True)
        return Err(self.v.sum(axis=axis, keepdims=True), self.e.sum(axis=axis, keepdims=True) + (n + 8) * EPS32 * size)

    def mean(self):
        n = self.v.shape[1]
        return self.sum(1) * Err(1.0 / n, EPS32 / n)

    def rsqrt(self):
        """Of a value above its bound: 1 / sqrt, two units of its own."""
        v = 1.0 / np.sqrt(self.v)
        low = np.maximum(self.v - self.e, self.v * 1e-3)
        return Err(v, 1.0 / np.sqrt(low) - v + 4 * EPS32 / np.sqrt(low))


def _normed(z, eps):
    """-> (1 / |z|, z / |z|)."""
    inv = ((z * z).mean() + Err(eps, EPS32 * eps)).rsqrt()
    return inv, z * inv


def _inputs(x, y, post, gate, pre):
    return [None if a is None else Err(np.atleast_2d(np.asarray(a, np.float64))) for a in (x, y, post, gate, pre)]


def _joined(x, y, post, gate, scale, eps):
    """-> (1 / |y|, y^, n, r)."""
    if y is None:
        return None, None, None, x
    inv, hat = (Err(np.ones((len(y.v), 1))), y) if post is None else _normed(y, eps)
    n = hat if post is None else hat * post
    step = n if gate is None else n * gate
    return inv, hat, n, x + Err(scale, EPS32 * abs(scale)) * step


def block_norm(x, y, post, gate, scale, pre, eps):
    """-> (r, h) as Err; h None without pre."""
    x, y, post, gate, pre = _inputs(x, y, post, gate, pre)
    _, _, _, r = _joined(x, y, post, gate, scale, eps)
    return r, None if pre is None else _normed(r, eps)[1] * pre


def block_norm_grad(dr, dh, x, y, post, gate, scale, pre, eps, kind):
    """-> (dx, dy, dpost, dgate, dpre) as Err, None where the input is; kind of the gate: None, channel, token, each."""
    x, y, post, gate, pre = _inputs(x, y, post, gate, pre)
    inv, hat, n, r = _joined(x, y, post, gate, scale, eps)
    total = Err(np.zeros_like(x.v)) if dr is None else Err(dr)
    dpre = dpost = dgate = dy = None
    if pre is not None:
        dh = Err(dh)
        inv_r, r_hat = _normed(r, eps)
        dpre = (dh * r_hat).sum(0)
        dz = dh * pre
        total = total + inv_r * (dz - r_hat * (dz * r_hat).mean())
    if y is not None:
        dn = Err(scale, EPS32 * abs(scale)) * total
        if gate is not None:
            each = dn * n
            dgate = {"channel": lambda: each.sum(0), "token": lambda: each.sum(1), "each": lambda: each}[kind]()
            dn = dn * gate
        dy = dn
        if post is not None:
            dpost = (dn * hat).sum(0)
            dz = dn * post
            dy = inv * (dz - hat * (dz * hat).mean())
    return total, dy, dpost, dgate, dpre
