"""The serving operators from their definitions, in 64 bits on the host: token by token through the block table, one
head at a time.  Shares no code with the library; tests compare with tolerances derived in `tolerance_*`."""
from __future__ import annotations

import math

import numpy as np
import torch

DT = {"fp16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}  # a rounding is off by at most this share of the value
TINY = {"fp16": 2.0 ** -25, "bf16": 0.0}             # and by this much where the type runs out of exponents


class Cache:
    """Pools of one instance on the host, with element access by (layer, block, head, K/V, token)."""

    def __init__(self, model, tp, NB, T, order, dtype, seed=0, fill=None):
        self.model, self.tp, self.NB, self.T, self.order, self.dtype = model, tp, NB, T, order, dtype
        self.Hr = model["Hkv"] // tp
        L, D = model["L"], model["D"]
        shape = (L, NB, self.Hr, 2, T, D) if order == 0 else (L, 2, NB, T, self.Hr, D)
        g = torch.Generator().manual_seed(seed)
        self.pools = [torch.randn(*shape, generator=g).to(DT[dtype]) if fill is None else
                      torch.full(shape, fill, dtype=DT[dtype]) for _ in range(tp)]

    def at(self, layer, block, head, kv, t, pools=None):
        """View of one token's key (kv = 0) or value (1)."""
        p = (pools or self.pools)[head // self.Hr]
        h = head % self.Hr
        return p[layer, block, h, kv, t] if self.order == 0 else p[layer, kv, block, t, h]

    def head(self, layer, table, n, head, kv):
        """float64 [n, D]: the first n tokens of a sequence; blocks outside the pool give NaN rows."""
        out = np.full((n, self.model["D"]), np.nan)
        for i in range(n):
            b = int(table[i // self.T])
            if 0 <= b < self.NB:
                out[i] = self.at(layer, b, head, kv, i % self.T).double().numpy()
        return out

    def ok(self, table, n):
        return np.array([0 <= int(table[i // self.T]) < self.NB for i in range(n)], bool)


def tables(lens, T, NB, seed=0, extra=0):
    """A random block table for the lengths, -1 behind each sequence's blocks."""
    nblk = [-(-int(n) // T) for n in lens]
    ids = np.random.default_rng(seed).permutation(NB)
    assert sum(nblk) <= NB
    bt = np.full((len(lens), max(nblk + [1]) + extra), -1, np.int32)
    k = 0
    for s, n in enumerate(nblk):
        bt[s, :n] = ids[k:k + n]
        k += n
    return bt


def seen(n_rows, length, window):
    """bool [n_rows, length]: which cached tokens each new token sees."""
    pos = length - n_rows + np.arange(n_rows)[:, None]
    key = np.arange(length)[None]
    m = key <= pos
    if window:
        m &= key > pos - window
    return m


def attend(cache, layer, bt, lens, starts, q, scale, window):
    """(out, lse, weight on |v|, largest possible |logit|) per row and query head; None rows stay NaN."""
    m = cache.model
    G, D = m["Hq"] // m["Hkv"], m["D"]
    rows = q.shape[0]
    out = np.full((rows, m["Hq"], D), np.nan)
    lse = np.full((rows, m["Hq"]), np.nan)
    absv, size = np.zeros_like(out), np.zeros_like(lse)
    for s, n in enumerate(lens):
        lo, hi = starts[s], starts[s + 1]
        ok = cache.ok(bt[s], n)
        see = seen(hi - lo, n, window) & ok[None]
        for h in range(m["Hkv"]):
            K = np.where(ok[:, None], cache.head(layer, bt[s], n, h, 0), 0.0)
            V = np.where(ok[:, None], cache.head(layer, bt[s], n, h, 1), 0.0)
            for r in range(hi - lo):
                use = see[r]
                for g in range(G):
                    qq = q[lo + r, h * G + g]
                    if not use.any():
                        out[lo + r, h * G + g], lse[lo + r, h * G + g] = 0.0, -math.inf
                        continue
                    x = scale * (K[use] @ qq)
                    top = x.max()
                    p = np.exp(x - top)
                    l = p.sum()
                    out[lo + r, h * G + g] = p @ V[use] / l
                    absv[lo + r, h * G + g] = p @ np.abs(V[use]) / l
                    lse[lo + r, h * G + g] = top + math.log(l)
                    size[lo + r, h * G + g] = abs(scale) * (np.abs(K[use]) @ np.abs(qq)).max()
    return out, lse, absv, size


def logit_error(D, size):
    """Of a logit: the products of 16-bit values are exact in 32 bits, each of the D additions and the two scalings may
    be off by 2^-23 of the partial sums, which stay below `size` = scale * sum |q||k| (2^-23 rather than half a step:
    the matrix units may cut instead of rounding)."""
    return (D + 4) * 2.0 ** -23 * size


def tolerance_attend(dtype, D, n, out, absv, size, vmax):
    """The weights and the output are rounded to the type once each; a weight's relative error in 32 bits is its logit's
    absolute one twice (in the weight and in the sum), 2^-21 of the exponential's, and the sums add n steps of 2^-23.
    A weight below the type's smallest is off by up to TINY, n of them by n * TINY of the largest value (the sum of the
    weights is 1 at least)."""
    e32 = 2 * logit_error(D, size)[..., None] + 2.0 ** -20 + (n + 8) * 2.0 ** -23
    u = HALF_STEP[dtype]
    return (u + e32) * absv * (1 + u) + (u + e32) * np.abs(out) + TINY[dtype] * (n * vmax + 1) + 1e-30


def tolerance_lse(D, n, lse, size):
    """Its logits' error, the sum's n steps, the exponential's 2^-21 and the logarithm's and the scaling's few."""
    return logit_error(D, size) + (n + 16) * 2.0 ** -23 + 2.0 ** -20 + np.abs(np.where(np.isfinite(lse), lse, 0)) * 2.0 ** -21


def scores(cache, layer, bt, lens, starts, q, scale, window, lse, scored, old):
    """{(sequence, head): float64 [len]} sums and their tolerances; lse as given to the call."""
    m = cache.model
    G, D = m["Hq"] // m["Hkv"], m["D"]
    got, tol = {}, {}
    for s, n in enumerate(lens):
        lo, hi = starts[s], starts[s + 1]
        see = seen(hi - lo, n, window)
        for h in range(m["Hkv"]):
            K = cache.head(layer, bt[s], n, h, 0)
            total, bound = np.zeros(n), np.zeros(n)
            for i in range(n):
                if scored is not None and i < scored[s]:
                    total[i] = old(s, h, i)
            bound += np.abs(total) * 2.0 ** -23
            for r in range(hi - lo):
                for g in range(G):
                    L = lse[lo + r, h * G + g]
                    if L == -math.inf or not see[r].any():
                        continue
                    qq = q[lo + r, h * G + g]
                    x = scale * (K @ qq)
                    p = np.where(see[r], np.exp(x - L), 0.0)
                    # the difference's error: the logit's, and 2^-23 of each of the two scaled terms
                    e = logit_error(D, abs(scale) * (np.abs(K) @ np.abs(qq))) + 3 * 2.0 ** -23 * (np.abs(x) + abs(L)) + 2.0 ** -20
                    total += p
                    bound += p * (e + (G * (hi - lo) + 4) * 2.0 ** -23)
            got[s, h], tol[s, h] = total, bound + 1e-37
    return got, tol


def turned(x, weight, eps, inv_freq, pos, rot, interleaved):
    """[rows, heads, D] float64: normalised and rotated; and the sizes that errors scale with."""
    x = x.astype(np.float64)
    if weight is not None:
        x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps) * weight
    size = np.abs(x)
    if inv_freq is not None:
        a = np.arange(0, rot, 2) if interleaved else np.arange(rot // 2)
        b = a + (1 if interleaved else rot // 2)
        ang = pos.astype(np.float64)[:, None, None] * inv_freq
        c, s = np.cos(ang), np.sin(ang)
        y, z = x.copy(), size.copy()
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        z[..., a] = z[..., b] = size[..., a] + size[..., b]
        x, size = y, z
    return x, size


def tolerance_append(dtype, D, y, size):
    """One rounding to the type; in 32 bits the mean's D additions, the root, division and products of a norm and the
    angle's rounding (half a step of pi) and the sine's couple of steps."""
    return HALF_STEP[dtype] * np.abs(y) + (D / 2 + 16) * 2.0 ** -23 * size + TINY[dtype] + 1e-30


def kept(score, n, budget, recent):
    """Indices that stay of a sequence of n tokens, in order; ties to the lower index, NaN below everything."""
    if n <= budget:
        return np.arange(n)
    free = n - recent
    x = np.asarray(score[:free], np.float64).copy() if free and score is not None else np.zeros(free)
    nan = np.isnan(x)
    x[nan] = 0.0
    order = np.lexsort((np.arange(free), -x, nan))[:budget - recent]
    return np.concatenate([np.sort(order), np.arange(free, n)]).astype(np.int64)
