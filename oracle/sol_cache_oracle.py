"""Plain 64-bit reference of the serving operators (include/sol_cache.h), written from their definitions in numpy, row by
row.  Test infrastructure only; shares no code with the GPU path."""
from __future__ import annotations

import numpy as np

PAGE = 64
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
K_SCALES, V_SCALES = (-100, 125), (-23, 13)


def norm_rope(x, w, cos, sin, positions, eps, interleaved):
    """x [B,H,N,d]; w [d] or None; cos, sin [P, rot/2] or None; positions [B,N].  Returns (y, written [B,N])."""
    x = np.asarray(x, np.float64)
    B, H, N, d = x.shape
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    if w is not None:
        y = y * np.asarray(w, np.float64)
    out = y.copy()
    half = 0 if cos is None else cos.shape[1]
    written = positions >= 0
    if half:
        written = written & (positions < cos.shape[0])
        at = np.where(written, positions, 0)
        c, s = np.asarray(cos, np.float64)[at][:, None], np.asarray(sin, np.float64)[at][:, None]   # [B,1,N,half]
        ia = np.arange(half) * 2 if interleaved else np.arange(half)
        ib = ia + 1 if interleaved else ia + half
        out[..., ia] = y[..., ia] * c - y[..., ib] * s
        out[..., ib] = y[..., ib] * c + y[..., ia] * s
    return out, written


def tables(lens, add, table, ring, state, rows):
    """One step, request by request.  Returns (row_start, slots, positions, lens, state, table, ring)."""
    table, ring = np.array(table), np.array(ring)
    S, MP = table.shape
    P = len(ring)
    head, count = int(state[0]) % P, min(max(int(state[1]), 0), P)
    start, slots, positions, out = [0], [], [], []
    asked = taken = 0
    back = []
    for s in range(S):
        n, a = min(max(int(lens[s]), 0), MP * PAGE), int(add[s])
        start.append(start[-1] + max(a, 0))
        have = -(-n // PAGE)
        if a <= 0:
            left = max(0, n + a)
            back += [int(p) for p in table[s, -(-left // PAGE):have] if 0 <= p < P]
            out.append(left)
            continue
        good = n + a <= MP * PAGE
        if good:
            need = -(-(n + a) // PAGE) - have
            asked += need
            good = need == 0 or asked <= count
        if good:
            for p in range(have, have + need):
                table[s, p] = ring[(head + taken) % P]
                taken += 1
        out.append(n + a if good else n)
        for p in range(n, n + a):
            page = int(table[s, p // PAGE]) if good else -1
            slots.append(page * PAGE + p % PAGE if 0 <= page < P else -1)
            positions.append(p if good else -1)
    back = back[:P - count]
    for i, p in enumerate(back):
        ring[(head + count + i) % P] = p
    tail = [-1] * max(0, rows - len(slots))
    return (np.array(start), np.array((slots + tail)[:rows]), np.array((positions + tail)[:rows]), np.array(out),
            np.array([(head + taken) % P, count - taken + len(back)]), table, ring)


def quantise(x, limits):
    """x [..., d] -> (codes [..., d], exponents [..., d/32]); x finite."""
    x = np.asarray(x, np.float64)
    g = x.reshape(x.shape[:-1] + (-1, 32))
    top = np.abs(g).max(-1)
    safe = np.where(top > 0, top, 1.0)
    e = np.floor(np.log2(safe)).astype(int)
    e = np.where(2.0 ** e > safe, e - 1, e)          # log2 may round up at a power of two
    e = np.where(2.0 ** (e + 1) <= safe, e + 1, e) - 2
    e = np.where(top > 7 * 2.0 ** e, e + 1, e)
    e = np.where(top > 0, np.clip(e, *limits), limits[0])
    y = np.abs(g) / (2.0 ** e)[..., None]
    lower = np.clip(np.searchsorted(GRID, y, side="right") - 1, 0, 6)
    a, b = y - GRID[lower], GRID[lower + 1] - y
    up = (b < a) | ((b == a) & (lower % 2 == 1))     # ties to the even code
    code = np.where(y >= 6, 7, lower + up) + 8 * np.signbit(g)
    return code.reshape(x.shape), e


def values(code, e):
    grid = np.concatenate([GRID, -GRID])
    v = grid[code].reshape(code.shape[:-1] + (-1, 32)) * (2.0 ** e)[..., None]
    return v.reshape(code.shape)


def write_page_token(page, tok, d, k, v):
    """Puts one token's key and value (each (codes [d], exponents [d/32])) into a page of bytes [68 d]."""
    w = d // 64
    (kc, ke), (vc, ve) = k, v
    for b in range(d // 2):
        page[tok * (d // 2) + b] = kc[2 * b] | (kc[2 * b + 1] << 4)
    t = tok % 32
    t2 = (t & 0b10011) | (((t >> 2) & 1) << 3) | (((t >> 3) & 1) << 2)
    for g in range(d // 32):
        page[32 * d + (((g % 2) * 32 + t2) * w + g // 2) * 2 + tok // 32] = ke[g] + 127
        page[66 * d + ((tok // 8) * (d // 32) + g) * 8 + tok % 8] = ve[g] + 127
    per = d // 32
    for i in range(32):
        for b in range(w):
            c = per * i + 2 * b
            page[34 * d + (((tok // 8) * 32 + i) * 8 + tok % 8) * w + b] = vc[c] | (vc[c + 1] << 4)


def read_page(page, d):
    """(k, v) [64, d] of a page of bytes; tokens whose key scale is 255 are NaN."""
    w = d // 64
    page = np.asarray(page).astype(int)
    k, v = np.zeros((64, d)), np.zeros((64, d))
    grid = np.concatenate([GRID, -GRID])
    for tok in range(64):
        t = tok % 32
        t2 = (t & 0b10011) | (((t >> 2) & 1) << 3) | (((t >> 3) & 1) << 2)
        c = np.arange(d)
        g = c // 32
        kb = page[tok * (d // 2) + c // 2]
        ks = page[32 * d + (((g % 2) * 32 + t2) * w + g // 2) * 2 + tok // 32]
        per = d // 32
        vb = page[34 * d + (((tok // 8) * 32 + c // per) * 8 + tok % 8) * w + c % per // 2]
        vs = page[66 * d + ((tok // 8) * per + g) * 8 + tok % 8]
        nan = (ks == 255).any()
        k[tok] = np.nan if nan else grid[np.where(c % 2, kb >> 4, kb & 15)] * 2.0 ** (ks - 127.0)
        v[tok] = np.nan if nan else grid[np.where(c % 2, vb >> 4, vb & 15)] * 2.0 ** (vs - 127.0)
    return k, v


def attend(q, k, v, sees):
    """q [R,d], k, v [L,d], sees [R, L] bool.  Returns (out, spread, reach): the output rows, sum_j p_j |v_j - out| and
    sum_j p_j |v_j|, the measures that error bounds are made of.  Rows that see nothing are 0."""
    R, d = q.shape
    out, spread, reach = (np.zeros((R, d)) for _ in range(3))
    for r in range(R):
        at = np.nonzero(sees[r])[0]
        if not len(at):
            continue
        s = k[at] @ q[r] / np.sqrt(d)
        p = np.exp(s - s.max())
        p /= p.sum()
        out[r] = p @ v[at]
        spread[r] = p @ np.abs(v[at] - out[r])
        reach[r] = p @ np.abs(v[at])
    return out, spread, reach
