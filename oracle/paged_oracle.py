"""Plain 64-bit CPU forms of the paged 8-bit KV cache operators: block tables,
quantising append, block attention.  Test infrastructure only; written with
loops, from the definitions in include/sbd.h, and independent of the kernels."""
from __future__ import annotations

import math

import numpy as np


def e4m3_values() -> np.ndarray:
    """The 256 values of the e4m3 codes (bias 7; 0x7f and 0xff are NaN)."""
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        if e == 15 and m == 7:
            x = math.nan
        out[c] = -x if c & 128 else x
    return out


E4M3 = e4m3_values()
_POS = E4M3[:127]                       # 0 .. 448, ascending


def e4m3_encode(x) -> np.ndarray:
    """Codes of x: nearest value, ties to the even code, saturating; NaN stays NaN."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.where(np.isnan(x), 0.0, np.abs(x)), 448.0)
    hi = np.clip(np.searchsorted(_POS, a), 1, 126)
    lo = hi - 1
    d_lo, d_hi = a - _POS[lo], _POS[hi] - a
    code = np.where((d_hi < d_lo) | ((d_hi == d_lo) & (hi % 2 == 0)), hi, lo)
    code = np.where(np.isnan(x), 127, code)
    return (code + np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def scale_for(amax: float) -> float:
    """The smallest power of two s >= 2^-126 with amax <= 448 s."""
    s = 2.0 ** -126
    while amax > 448.0 * s:
        s *= 2.0
    return s


def block_tables(cache_len, target_len, table, free, n_free, page, max_new):
    """Returns (table, length, new_start, slot_map, n_free, free) after the call."""
    B, cols = table.shape
    cap = cols * page
    table, free = table.copy(), free.copy()
    up = lambda x: -(-x // page)  # noqa: E731
    lens, target = [], []
    for l, t in zip(map(int, cache_len), map(int, target_len)):
        bad = not (0 <= l <= cap and 0 <= t <= cap)
        l = min(max(l, 0), cap)
        lens.append(l)
        target.append(l if bad else t)
    released = []
    for b in range(B):
        for p in range(up(target[b]), up(lens[b])):
            released.append(table[b, p])
            table[b, p] = -1
    stack = list(free[:n_free]) + released[::-1]
    free[n_free:len(stack)] = stack[n_free:]
    start, slots, length = [0], [], []
    need_sum = 0
    granted = 0
    avail = len(stack)
    for b in range(B):
        new, need = max(target[b] - lens[b], 0), max(up(target[b]) - up(lens[b]), 0)
        need_sum += need
        total = start[-1] + new
        ok = (need == 0 or need_sum <= avail) and (new == 0 or total <= max_new)
        length.append(target[b] if ok else lens[b])
        if ok:
            for p in range(up(lens[b]), up(target[b])):
                table[b, p] = stack[avail - 1 - granted]
                granted += 1
        slots += [int(table[b, i // page]) * page + i % page if ok else -1
                  for i in range(lens[b], lens[b] + new)]
        start.append(total)
    for b in range(B):
        table[b, up(length[b]):] = -1
    slots = (slots + [-1] * max_new)[:max_new]
    i32 = lambda x: np.asarray(x, np.int32)  # noqa: E731
    return i32(table), i32(length), i32(start), i32(slots), avail - granted, i32(free)


def cache_append(x, slots, codes, scale, page):
    """x [T, Hkv, D] into codes [n_pages, Hkv, P, D] uint8 and scale
    [n_pages, Hkv]; returns the updated copies."""
    codes, scale = codes.copy(), np.asarray(scale, np.float64).copy()
    x = np.asarray(x, np.float64)
    T, H, _ = x.shape
    t = 0
    while t < T:
        s = int(slots[t])
        if s < 0 or s >= codes.shape[0] * page:
            t += 1
            continue
        n = 1
        while t + n < T and slots[t + n] == s + n and (s + n) % page:
            n += 1
        pg, off = s // page, s % page
        for h in range(H):
            seg = x[t:t + n, h]
            fin = np.abs(seg[np.isfinite(seg)])
            new = scale_for(float(fin.max()) if fin.size else 0.0)
            old = scale[pg, h]
            if off:
                new = max(new, old)
                if new != old:
                    codes[pg, h, :off] = e4m3_encode(E4M3[codes[pg, h, :off]] * (old / new))
            scale[pg, h] = new
            codes[pg, h, off:off + n] = e4m3_encode(seg / new)
        t += n
    return codes, scale.astype(np.float32)


def paged_keys(codes, scale, table, length, page):
    """[Hkv, length, D] values of a request's cached tokens."""
    H, D = codes.shape[1], codes.shape[3]
    out = np.empty((H, length, D))
    for p in range(-(-length // page)):
        n = min(page, length - p * page)
        pg = int(table[p])
        out[:, p * page:p * page + n] = E4M3[codes[pg, :, :n]] * np.asarray(scale[pg], np.float64)[:, None, None]
    return out


def block_attention(q, kc, vc, ks, vs, table, lens, kb, vb, n_causal=0, scale=None, page=None):
    """Returns (out, spread, wobble), all [B, k, Hq, D] or [B, k, Hq]: spread =
    sum_j p_j |v_j| bounds what an error in the probabilities does to out, and
    wobble = scale * max_j max(sum_d |q_d k_jd|, max|q| sum_d |k_jd|) what a
    rounding of q or of the products does to a score."""
    q = np.asarray(q, np.float64)
    B, k, Hq, D = q.shape
    H = kc.shape[1]
    page = kc.shape[2] if page is None else page
    scale = D ** -0.5 if scale is None else scale
    out, spread = np.zeros_like(q), np.zeros_like(q)
    wobble = np.zeros((B, k, Hq))
    for b in range(B):
        K = np.concatenate([paged_keys(kc, ks, table[b], int(lens[b]), page),
                            np.asarray(kb[b], np.float64).transpose(1, 0, 2)], 1)
        V = np.concatenate([paged_keys(vc, vs, table[b], int(lens[b]), page),
                            np.asarray(vb[b], np.float64).transpose(1, 0, 2)], 1)
        for h in range(Hq):
            for i in range(k):
                seen = int(lens[b]) + (i + 1 if i < n_causal else k)
                Kh, Vh = K[h * H // Hq, :seen], V[h * H // Hq, :seen]
                z = scale * (Kh @ q[b, i, h])
                e = np.exp(z - z.max())
                p = e / e.sum()
                out[b, i, h] = p @ Vh
                spread[b, i, h] = p @ np.abs(Vh)
                a = np.abs(Kh)
                wobble[b, i, h] = scale * max((a @ np.abs(q[b, i, h])).max(),
                                              np.abs(q[b, i, h]).max() * a.sum(1).max())
    return out, spread, wobble
