"""Plain 64-bit CPU forms of the operators of drafted decoding: norms with rotation,
tree attention over the paged 8-bit cache, verification of drafted tokens, append of
an accepted path.  Test infrastructure only; written with loops, from the definitions
in include/sbd.h, and independent of the kernels."""
from __future__ import annotations

import math
from fractions import Fraction

import numpy as np

from oracle import paged_oracle as po

# pi to 50 digits, for angles of far positions
PI = Fraction(314159265358979323846264338327950288419716939937510, 10 ** 50)


def turn(position: int, freq: float) -> float:
    """position * freq in turns, whole ones dropped, in [0, 1): rational arithmetic."""
    t = Fraction(int(position)) * Fraction(float(freq)) / (2 * PI)
    return float(t - math.floor(t))


def norm_rope(x, positions, inv_freq, weight, eps, interleaved):
    """x [T, H, D]; positions [T]; inv_freq [R / 2] (None: no rotation); weight [D] or None."""
    x = np.array(x, np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    half = 0 if inv_freq is None else len(inv_freq)
    for t in range(x.shape[0]):
        for j in range(half):
            a = 2 * math.pi * turn(positions[t], inv_freq[j])
            i, k = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
            y1, y2 = x[t, :, i].copy(), x[t, :, k].copy()
            x[t, :, i] = y1 * math.cos(a) - y2 * math.sin(a)
            x[t, :, k] = y2 * math.cos(a) + y1 * math.sin(a)
    return x


def ancestors(parent, i):
    """Node i and the nodes above it; a parent that is not below its node is none."""
    out = [i]
    while 0 <= parent[i] < i:
        i = int(parent[i])
        out.append(i)
    return out


def tree_attention(q, kc, vc, ks, vs, table, lens, kb, vb, parent, scale=None):
    """As paged_oracle.block_attention, row i of the block with itself and its ancestors."""
    q = np.asarray(q, np.float64)
    B, n, Hq, D = q.shape
    H, page = kc.shape[1], kc.shape[2]
    scale = D ** -0.5 if scale is None else scale
    out, spread, wobble = np.zeros_like(q), np.zeros_like(q), np.zeros((B, n, Hq))
    for b in range(B):
        L = int(lens[b])
        K, V = (np.concatenate([po.paged_keys(c, s, table[b], L, page), np.asarray(x[b], np.float64).transpose(1, 0, 2)], 1)
                for c, s, x in ((kc, ks, kb), (vc, vs, vb)))
        for i in range(n):
            at = np.concatenate([np.arange(L), L + np.asarray(sorted(ancestors(parent[b], i)))]).astype(int)
            for h in range(Hq):
                Kh, Vh = K[h * H // Hq, at], V[h * H // Hq, at]
                z = scale * (Kh @ q[b, i, h])
                e = np.exp(z - z.max())
                p = e / e.sum()
                out[b, i, h] = p @ Vh
                spread[b, i, h] = p @ np.abs(Vh)
                a = np.abs(Kh)
                wobble[b, i, h] = scale * max((a @ np.abs(q[b, i, h])).max(), np.abs(q[b, i, h]).max() * a.sum(1).max())
    return out, spread, wobble


def _softmax(z, tau):
    """p, ln p (not ln of p: apart from a logit of 3e38 a sum of exponentials would vanish), and the logits."""
    z = np.asarray(z, np.float64)
    z = np.where(np.isnan(z), -np.inf, z)
    m = z.max()
    # (infinities: the largest of them are alike and leave nothing to the others)
    y = (z - m) / tau if np.isfinite(m) else np.where(z == m, 0.0, -np.inf)
    e = np.exp(y)
    return e / e.sum(), y - math.log(e.sum()), z


def verify(target, draft, parent, token, uniform, gumbel, tau):
    """One request: target, draft [n, V] (draft None: given tokens), the rest [n] and [V].
    Returns (path, tokens, logprob, margin): margin is how near to the border the nearest
    of its decisions is, relative to what is compared (of the argmax: the score's distance
    to the next one)."""
    n, V = target.shape
    node, path, tokens, logprob, margin = 0, [0], [], [], math.inf

    def say(x):
        tokens.append(int(x))
        logprob.append(float(_softmax(target[node], tau or 1.0)[1][x]))

    while True:
        p, _, z = _softmax(target[node], tau or 1.0)
        children = [c for c in range(1, n) if parent[c] == node and parent[c] < c and 0 <= token[c] < V]
        if tau == 0:
            best = int(np.argmax(z))
            hit = [c for c in children if token[c] == best]
            say(best)
            if not hit:
                return path, tokens, logprob, margin
            node = hit[0]
            path.append(node)
            continue
        q = None if draft is None else _softmax(draft[node], tau)[0]
        for c in children:
            x = int(token[c])
            lhs = float(uniform[c]) * (1.0 if q is None else q[x])
            margin = min(margin, abs(lhs - p[x]) / max(lhs, p[x], 1e-300))
            if lhs < p[x]:
                say(x)
                node = c
                path.append(c)
                break
            if q is None:
                left = p.copy()
                left[x] = 0.0
            else:
                left = np.maximum(p - q, 0.0)
            if left.sum() > 0:
                p = left / left.sum()
        else:
            with np.errstate(divide="ignore"):
                score = np.log(p) + np.asarray(gumbel, np.float64)
            x = int(np.argmax(score))
            if V > 1:
                margin = min(margin, float(score[x] - np.partition(score, -2)[-2]) if score[x] > -np.inf else math.inf)
            say(x)
            return path, tokens, logprob, margin


def append_path(x, path, start, slots, codes, scale, page):
    """x [B, n, Hkv, D] into codes and scale as paged_oracle.cache_append, request by request."""
    B, n = x.shape[:2]
    for b in range(B):
        m = min(max(int(start[b + 1]) - int(start[b]), 0), n)
        rows, to = [], []
        for j in range(m):
            t = int(start[b]) + j
            slot = int(slots[t]) if 0 <= t < len(slots) else -1
            node = int(path[b, j])
            if not 0 <= node < n:
                slot, node = -1, 0
            rows.append(x[b, node])
            to.append(slot)
        if rows:
            codes, scale = po.cache_append(np.stack(rows), to, codes, scale, page)
    return codes, np.asarray(scale, np.float32)
