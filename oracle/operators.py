"""Float64 definitions of the model operators around the search (embedding
lookup, pooling and gradient, the gate of an MoE layer, the chosen experts'
products), written from their formulas with NumPy and plain loops.

Next to each result stands a bound on what a float32 computation of it may be
off by, from the standard bound of an n-term sum (n units of 2^-24 of the sum of
the magnitudes, whatever the order) and the roundings named at each step.
"""
from __future__ import annotations

import numpy as np

EPS32 = 2.0 ** -24           # half a unit of float32, relative
EPS16 = 2.0 ** -8            # half a unit of bfloat16 (8 significant bits), relative
TINY = 2.0 ** -126           # below this, units are absolute


def rounding(dtype: str) -> float:
    return EPS16 if dtype == "bf16" else EPS32


def embed_lookup(table, tokens, scale):
    out = np.zeros((len(tokens), table.shape[1]))
    for t, v in enumerate(tokens):
        if 0 <= v < len(table):
            out[t] = table[v].astype(np.float64) * scale
    return out


def embed_pool(table, tokens, offsets, scale):
    """-> (mean rows, bound of the float32 sum and mean)."""
    B, d = len(offsets) - 1, table.shape[1]
    out, bound = np.zeros((B, d)), np.zeros((B, d))
    for b in range(B):
        lo, hi = (min(max(int(o), 0), len(tokens)) for o in offsets[b:b + 2])
        rows = [int(v) for v in tokens[lo:hi] if 0 <= v < len(table)]
        if rows:
            x = table[rows].astype(np.float64)
            out[b] = x.sum(axis=0) / len(rows) * scale
            bound[b] = (len(rows) + 4) * EPS32 * np.abs(x).sum(axis=0) / len(rows) * abs(scale)
    return out, bound


def embed_grad(dout, tokens, V, scale, base=None):
    """-> (gradient of the table, bound of the float32 sum); base: what it is added to."""
    out = np.zeros((V, dout.shape[1]))
    size, n = np.zeros_like(out), np.zeros(V)
    for t, v in enumerate(tokens):
        if 0 <= v < V:
            out[v] += dout[t].astype(np.float64)
            size[v] += np.abs(dout[t].astype(np.float64))
            n[v] += 1
    out, bound = out * scale, (n[:, None] + 4) * EPS32 * size * abs(scale)
    if base is not None:
        out = out + base
        bound += EPS32 * np.abs(out)
    return out, bound


def moe_route(x, gate, K, renorm, active=None):
    """-> (probs, ids, weight, mask): logits in float64, ranked by (logit
    descending, index ascending), NaN last."""
    T, E = len(x), len(gate)
    logits = x.astype(np.float64) @ gate.astype(np.float64).T
    probs, ids = np.zeros((T, E)), np.full((T, K), -1, np.int32)
    weight, mask = np.zeros((T, K)), np.zeros(T, np.uint64)
    for t in range(T):
        if active is not None and not active[t]:
            continue
        l = logits[t]
        with np.errstate(invalid="ignore", over="ignore"):
            e = np.exp(l - np.max(l)) if not np.isnan(l).any() else np.full(E, np.nan)
            probs[t] = e / e.sum()
        order = sorted(range(E), key=lambda j: (np.isnan(l[j]), -l[j] if not np.isnan(l[j]) else 0.0, j))[:K]
        ids[t] = order
        weight[t] = probs[t, order]
        if renorm:
            weight[t] /= weight[t].sum()
        for j in order:
            mask[t] |= np.uint64(1 << j)
    return probs, ids, weight, mask


def silu(z):
    with np.errstate(over="ignore"):
        return z / (1.0 + np.exp(-z))


def moe_experts(x, ids, weight, slots, slot_of, d, f, residual=None, dtype="f32"):
    """-> (out before its rounding, bound).  slots [n][3 d f] as float arrays."""
    T, K = ids.shape
    E = len(slot_of)
    out = np.zeros((T, d)) if residual is None else residual.astype(np.float64).copy()
    bound = np.zeros((T, d))
    magnitude = np.abs(out)
    rest = EPS16 ** 2 if dtype == "bf16" else EPS32   # what h is rounded to: a bf16 and the rest's bf16
    for e in range(E):
        s = int(slot_of[e])
        if not 0 <= s < len(slots):
            continue
        block = slots[s].astype(np.float64)
        wg, wu, wd = block[:d * f].reshape(f, d), block[d * f:2 * d * f].reshape(f, d), block[2 * d * f:].reshape(d, f)
        for t in range(T):
            w = float(sum(float(weight[t, k]) for k in range(K) if ids[t, k] == e))
            if not (ids[t] == e).any():
                continue
            xt = x[t].astype(np.float64)
            g, u = wg @ xt, wu @ xt
            eg = (d + 8) * EPS32 * (np.abs(wg) @ np.abs(xt))
            eu = (d + 8) * EPS32 * (np.abs(wu) @ np.abs(xt))
            h = w * silu(g) * u
            # |silu'| < 1.1; the exponential, quotient and products add a few units
            eh = abs(w) * (1.1 * eg * (np.abs(u) + eu) + np.abs(silu(g)) * eu) + (16 * EPS32 + rest) * np.abs(h)
            eh += abs(w) * 16 * EPS32 * np.abs(u) * np.abs(silu(g))
            out[t] += wd @ h
            bound[t] += np.abs(wd) @ eh
            magnitude[t] += np.abs(wd) @ np.abs(h)
    terms = 2 * f * min(K, E) + 64
    return out, bound + terms * EPS32 * magnitude
