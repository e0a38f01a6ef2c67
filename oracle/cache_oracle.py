"""Plain CPU oracle of the 8-bit key/value cache: append, attention, eviction, and of trees
of drafted tokens: their places, masks and other scores, and keeping an accepted path.

TEST INFRASTRUCTURE ONLY; it shares no code with the HIP library or its Python
binding.  All arithmetic is fp64; e4m3 codes go through a table of their 256
values.

The cache holds each group's keys (after their rotation) and values in pages of
64 tokens, as e4m3 codes in units of the page's scale: the smallest power of two
s >= 2^-100 with |x| <= 448 s.  A pool is a dict of arrays: ``k`` [P, H, 64, hd] and
``v`` [P, H, 4, hd, 16] (uint8 codes), ``kv_scale`` [P, H, 2], ``mass`` [P, H, 64].
"""

from __future__ import annotations

import numpy as np

from oracle.attention_oracle import apply_rope

__all__ = ["PAGE", "VALUES", "encode", "decode", "scale_for", "rotate", "append", "attend",
           "accept", "evict", "tokens", "MAX_DEPTH"]

PAGE = 64
MAX_DEPTH = 1 << 20  # places of a new row behind the context
TOO_LARGE = 1.9375 * 2.0 ** 127  # halfway from 240 * 2^120 to 2^128, which fp32 does not hold


def _values():
    out = np.empty(256)
    for c in range(256):
        s, e, m = (-1.0 if c & 128 else 1.0), (c >> 3) & 15, c & 7
        out[c] = s * (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
        if c & 127 == 127:
            out[c] = np.nan
    return out


VALUES = _values()
_STEPS = VALUES[:127]                      # ascending
_BORDERS = (_STEPS[1:] + _STEPS[:-1]) / 2  # halfway to the next


def decode(codes):
    return VALUES[np.asarray(codes, dtype=np.uint8)]


def encode(x):
    """Nearest e4m3 code of |x| <= 448 (ties to the even code), NaN -> 0x7f."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(np.where(np.isnan(x), 0.0, x))
    c = np.searchsorted(_BORDERS, a, side="left")
    tie = (c < len(_BORDERS)) & (a == _BORDERS[np.minimum(c, len(_BORDERS) - 1)]) & (c % 2 == 1)
    c = np.where(tie, c + 1, c).astype(np.uint8)
    c = np.where(np.signbit(x), c | 128, c)
    return np.where(np.isnan(x), 0x7F, c).astype(np.uint8)


def scale_for(amax):
    """Smallest power of two s >= 2^-100 with amax <= 448 s."""
    m, e = np.frexp(np.asarray(amax, dtype=np.float64))  # amax = m 2^e, m in [0.5, 1)
    s = np.ldexp(1.0, e - 9 + (m > 0.875))
    return np.maximum(np.where(np.asarray(amax) > 0, s, 0.0), 2.0 ** -100)


def rotate(x, pos, theta, scale):
    """Rows ``x`` [n, ..., hd] turned by their positions ``pos`` [n]."""
    hd = x.shape[-1]
    inv = float(theta) ** (-2.0 * np.arange(hd // 2) / hd)
    ang = (np.asarray(pos, dtype=np.float64) / scale)[:, None] * inv
    shape = (len(pos),) + (1,) * (x.ndim - 2) + (hd // 2,)
    return apply_rope(x, np.cos(ang).reshape(shape), np.sin(ang).reshape(shape))


def _v_rows(codes):
    """[4, hd, 16] -> [64, hd]"""
    return np.swapaxes(codes, 1, 2).reshape(PAGE, codes.shape[1])


def _v_put(page, rows, t0):
    """Writes rows [n, hd] as tokens t0.. of a page [4, hd, 16]."""
    for i, r in enumerate(rows):
        page[(t0 + i) // 16, :, (t0 + i) % 16] = r


def _page(pool, table, b, blk):
    if blk >= table.shape[1]:
        return -1
    p = int(table[b, blk])
    return p if 0 <= p < len(pool["k"]) else -1


def _depth(depth, r0, r1):
    return np.clip(np.asarray(depth[r0:r1], dtype=np.int64), 0, MAX_DEPTH)


def append(pool, qkv, table, ctx, row_start, theta, scale, pos=None, depth=None):
    """Stores the new rows in ``pool`` (in place), turned by their order or by their places
    ``depth`` [N] behind the context; returns the rotated queries
    [H, N, nq, hd] and ``raw``, the new keys and values before quantisation
    {(page, h, t): (k, v)}."""
    H, N, n2, hd = qkv.shape
    nq = n2 - 2
    q_out = np.full((H, N, nq, hd), np.nan)
    raw = {}
    for b in range(len(ctx)):
        r0, r1 = int(row_start[b]), int(row_start[b + 1])
        c, n = int(ctx[b]), r1 - r0
        if n <= 0:
            continue
        p0 = c if pos is None else int(pos[b])
        for h in range(H):
            x = np.asarray(qkv[h, r0:r1], dtype=np.float64)
            at = np.arange(n) if depth is None else _depth(depth, r0, r1)
            with np.errstate(invalid="ignore"):
                rot = rotate(x[:, :nq + 1], p0 + at, theta, scale)
            q_out[h, r0:r1] = rot[:, :nq]
            k, v = rot[:, nq], x[:, nq + 1]
            bad = ~((np.abs(k) < TOO_LARGE).all(-1) & (np.abs(v) < TOO_LARGE).all(-1))
            for blk in range(c // PAGE, (c + n - 1) // PAGE + 1):
                p = _page(pool, table, b, blk)
                if p < 0:
                    continue
                lo, hi = max(c, blk * PAGE), min(c + n, (blk + 1) * PAGE)
                rows, t0 = slice(lo - c, hi - c), lo - blk * PAGE
                ok = ~bad[rows]
                for i, (name, y) in enumerate((("k", k[rows]), ("v", v[rows]))):
                    s = float(scale_for(np.abs(y[ok]).max(initial=0.0)))
                    if t0 > 0:
                        old = float(pool["kv_scale"][p, h, i])
                        s = max(s, old)
                        if s != old:
                            if name == "k":
                                pool["k"][p, h] = encode(decode(pool["k"][p, h]) * (old / s))
                            else:
                                pool["v"][p, h] = encode(decode(pool["v"][p, h]) * (old / s))
                    pool["kv_scale"][p, h, i] = s
                    codes = encode(np.where(ok[:, None], y, 0.0) / s)
                    if name == "k":
                        codes[~ok] = 0x7F
                        pool["k"][p, h, t0:t0 + hi - lo] = codes
                    else:
                        _v_put(pool["v"][p, h], codes, t0)
                for i in range(hi - lo):
                    raw[(p, h, t0 + i)] = (k[lo - c + i], v[lo - c + i], bool(ok[i]))
    return q_out, raw


def tokens(pool, table, b, h, n):
    """Keys, values [n, hd] of a sequence's first n tokens and which of them are there."""
    hd = pool["k"].shape[-1]
    k, v, there = np.zeros((n, hd)), np.zeros((n, hd)), np.zeros(n, dtype=bool)
    for blk in range((n + PAGE - 1) // PAGE):
        p = _page(pool, table, b, blk)
        if p < 0:
            continue
        a, m = blk * PAGE, min(PAGE, n - blk * PAGE)
        k[a:a + m] = decode(pool["k"][p, h, :m]) * pool["kv_scale"][p, h, 0]
        v[a:a + m] = decode(_v_rows(pool["v"][p, h])[:m]) * pool["kv_scale"][p, h, 1]
        there[a:a + m] = True
    return k, v, there


def attend(pool, q, table, ctx, row_start, rows=None, mass=False, cap=0.0, slope=None,
           prefix=None, tree=None, depth=None):
    """Attention of the rows of ``q`` [H, N, nq, hd] (all, or those in ``rows``):
    o [N, H, nq, hd], ``spread`` = sum_t p_t |v_t| of the same shape, the largest
    sum |q_i k_i| / sqrt(hd) of a visible score, and with ``mass`` what the tokens
    receive, {(b, h): [tokens]}.  Scores may be capped, cap * tanh(s / cap), and biased by
    -slope [H, nq] * |distance| (``depth`` [N]: the rows' places behind the context); a row
    sees the first ``prefix`` [B] tokens besides, and with ``tree`` (row r sees new row i of
    its sequence where tree[r][i]) not those before it."""
    H, N, nq, hd = q.shape
    q = np.asarray(q, dtype=np.float64)
    o = np.full((N, H, nq, hd), np.nan)
    spread, got, big = np.full_like(o, np.nan), {}, 0.0
    top = table.shape[1] * PAGE
    for b in range(len(ctx)):
        r0, r1, c = int(row_start[b]), int(row_start[b + 1]), int(ctx[b])
        mine = [r for r in range(r0, r1) if rows is None or r in rows]
        if not mine:
            continue
        n = min(c + r1 - r0, top)
        place = c + (np.arange(r1 - r0) if depth is None else _depth(depth, r0, r1))
        spot = np.concatenate([np.arange(min(c, n)), place[:max(n - c, 0)]])
        for h in range(H):
            k, v, there = tokens(pool, table, b, h, n)
            total = np.zeros(n)
            for r in mine:
                if tree is None:
                    seen = np.arange(n) < min(c + r - r0 + 1, top)
                else:
                    seen = np.arange(n) < c
                    mask = np.zeros(max(n - c, 0), dtype=bool)
                    m = np.asarray(tree[r], dtype=bool)[:len(mask)]
                    mask[:len(m)] = m
                    seen[c:] = mask
                if prefix is not None:
                    seen |= np.arange(n) < int(prefix[b])
                seen &= there
                kk, vv = k[seen], v[seen]
                with np.errstate(invalid="ignore", over="ignore"):
                    s = q[h, r] @ kk.T / np.sqrt(hd)
                    if cap:
                        s = cap * np.tanh(s / cap)
                if slope is not None:
                    far = np.abs(place[r - r0] - spot[seen]).astype(np.float64)
                    s = s - np.asarray(slope, dtype=np.float64)[h][:, None] * far
                if s.shape[1] == 0:
                    o[r, h] = spread[r, h] = 0.0
                    continue
                with np.errstate(invalid="ignore"):
                    p = np.exp(s - s.max(-1, keepdims=True))
                    p /= p.sum(-1, keepdims=True)
                    o[r, h] = p @ vv
                    spread[r, h] = p @ np.abs(vv)
                    big = max(big, float(np.nanmax(np.abs(q[h, r]) @ np.abs(kk).T)) / np.sqrt(hd))
                total[seen] += p.sum(0)
            got[(b, h)] = total
    return (o, spread, big, got) if mass else (o, spread, big)


def accept(pool, table, ctx, row_start, path):
    """Keeps the rows of each sequence's path, moved together behind its context (in
    place); new_len.  ``pool["mass"]`` may be None."""
    H, hd = pool["k"].shape[1], pool["k"].shape[-1]
    new_len = np.array(ctx, dtype=np.int32)
    top = table.shape[1] * PAGE
    for b in range(len(ctx)):
        c = int(ctx[b])
        n = min(int(row_start[b + 1]) - int(row_start[b]), top - c)
        kept, last = [], -1
        for r in path[b]:
            if not last < r < n:
                break
            kept.append(int(r))
            last = int(r)
        new_len[b] = c + len(kept)
        if not kept:
            continue
        lo = c // PAGE * PAGE
        ids = np.concatenate([np.arange(lo, c), c + np.array(kept)]).astype(int)
        for h in range(H):
            k, v, there = tokens(pool, table, b, h, c + n)
            mass = [0.0 if pool["mass"] is None or not there[t] else
                    pool["mass"][_page(pool, table, b, t // PAGE), h, t % PAGE] for t in ids]
            for i in range(0, len(ids), PAGE):
                p = _page(pool, table, b, (lo + i) // PAGE)
                if p < 0:
                    continue
                t = ids[i:i + PAGE]
                sk = float(scale_for(np.nanmax(np.abs(k[t]), initial=0.0)))
                sv = float(scale_for(np.nanmax(np.abs(v[t]), initial=0.0)))
                # (a page's codes: a NaN code keeps its sign, as everywhere in the cache)
                old = pool["k"][p, h].copy()
                codes = encode(k[t] / sk)
                for j, x in enumerate(t):
                    src = _page(pool, table, b, x // PAGE)
                    if np.isnan(k[x]).all():
                        codes[j] = old[x % PAGE] if src == p else pool["k"][src, h, x % PAGE]
                pool["kv_scale"][p, h] = sk, sv
                pool["k"][p, h, :len(t)] = codes
                _v_put(pool["v"][p, h], encode(v[t] / sv), 0)
                if pool["mass"] is not None:
                    pool["mass"][p, h, :len(t)] = mass[i:i + PAGE]
    return new_len


def evict(pool, table, length, keep, recent, dst):
    """Moves the kept tokens to the pages of ``dst`` (in place); (kept, new_len)."""
    H, hd = pool["k"].shape[1], pool["k"].shape[-1]
    B = len(length)
    kept = np.full((B, H, keep), -1, dtype=np.int32)
    new_len = np.minimum(np.asarray(length), keep).astype(np.int32)
    out = []
    for b in range(B):
        n = int(length[b])
        for h in range(H):
            ids = np.arange(n)
            if n > keep:
                w = np.array([-np.inf if _page(pool, table, b, t // PAGE) < 0 else
                              pool["mass"][_page(pool, table, b, t // PAGE), h, t % PAGE]
                              for t in range(n - recent)], dtype=np.float64)
                nan = np.isnan(w)  # (above infinity; the earlier of equals first)
                top = np.lexsort((np.where(nan, 0.0, -w), ~nan))[:keep - recent]
                ids = np.concatenate([np.sort(top), np.arange(n - recent, n)])
            kept[b, h, :len(ids)] = ids
            k, v, there = tokens(pool, table, b, h, n)
            m = np.array([pool["mass"][_page(pool, table, b, t // PAGE), h, t % PAGE]
                          if there[t] else 0.0 for t in ids], dtype=np.float32)
            out.append((b, h, k[ids], v[ids], m))
    for b, h, k, v, m in out:
        for blk in range((len(m) + PAGE - 1) // PAGE):
            p = int(dst[b, blk])
            a = slice(blk * PAGE, min(len(m), (blk + 1) * PAGE))
            size = a.stop - a.start
            sk = float(scale_for(np.nanmax(np.abs(k[a]), initial=0.0)))
            sv = float(scale_for(np.nanmax(np.abs(v[a]), initial=0.0)))
            pool["kv_scale"][p, h] = sk, sv
            pool["k"][p, h, :size] = encode(k[a] / sk)
            _v_put(pool["v"][p, h], encode(v[a] / sv), 0)
            pool["mass"][p, h, :size] = m[a]
    return kept, new_len
