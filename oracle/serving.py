"""Oracle of the serving operators (float64 numpy, plain loops): page maps,
rotary positions, the 8-bit K/V pages and attention over them."""

from __future__ import annotations

import math

import numpy as np

PAGE = 64


# ------------------------------------------------------------------ page maps
def page_map(cached, added, table, free_pages, free_count, n_rows):
    """One sequence after another, a page at a time off the top of the stack."""
    B, width = table.shape
    table = table.copy()
    count = min(max(int(free_count), 0), len(free_pages))
    left, asked, row = count, 0, 0
    lens, status, start = np.zeros(B, np.int32), np.zeros(B, np.int32), [0]
    slot = np.full(n_rows, -1, np.int64)
    pos = np.full(n_rows, -1, np.int32)
    seq = np.full(n_rows, -1, np.int32)
    for b in range(B):
        c, a = int(cached[b]), int(added[b])
        rows = max(a, 0)
        seq[min(row, n_rows):min(row + rows, n_rows)] = b
        lens[b] = c
        first, last = -(-c // PAGE), -(-(c + a) // PAGE)
        if c < 0 or a < 0 or c + a > width * PAGE:
            status[b] = 2
        elif row + rows > n_rows:
            status[b] = 3
        else:
            asked += last - first
            if last > first and asked > count:
                status[b] = 1
            else:
                for p in range(first, last):
                    left -= 1
                    table[b, p] = free_pages[left]
                lens[b] = c + a
                for j in range(a):
                    pos[row + j] = c + j
                    slot[row + j] = int(table[b, (c + j) // PAGE]) * PAGE + (c + j) % PAGE
        row += rows
        start.append(min(row, n_rows))
    return dict(table=table, seq_lens=lens, row_start=np.array(start, np.int32), slot=slot, position=pos,
                seq_of_row=seq, status=status, free_left=left)


def page_release(finished, table, lens, free_pages, free_count):
    table, lens, stack = table.copy(), lens.copy(), list(free_pages[:min(max(int(free_count), 0), len(free_pages))])
    for b in range(len(finished)):
        if finished[b]:
            held = min(-(-max(int(lens[b]), 0) // PAGE), table.shape[1])
            stack += [p for p in table[b, :held] if p >= 0]
            table[b, :held] = -1
            lens[b] = 0
    stack = stack[:len(free_pages)]
    free_pages = free_pages.copy()
    free_pages[:len(stack)] = stack
    return table, lens, free_pages, len(stack)


# ------------------------------------------------------------ rotary positions
def angles(head_dim, rotary_dim, base=10000.0, scaling="none", factor=1.0, original=0.0, low=0.0, high=0.0):
    r, out = rotary_dim, []
    if scaling == "base":
        base = base * factor ** (r / (r - 2.0))
    for i in range(r // 2):
        th = base ** (-2.0 * i / r)
        if scaling == "linear":
            th /= factor
        elif scaling == "turns":
            n = original * th / (2 * math.pi)
            g = min(1.0, max(0.0, (n - low) / (high - low)))
            th = g * th + (1 - g) * th / factor
        elif scaling == "planes":
            plane = lambda n: r * math.log(original / (2 * math.pi * n)) / (2 * math.log(base))  # noqa: E731
            i0, i1 = max(0.0, math.floor(plane(high))), min(r - 1.0, math.ceil(plane(low)))
            g = min(1.0, max(0.0, (i - i0) / max(i1 - i0, 0.001)))
            th = (1 - g) * th + g * th / factor
        out.append(th)
    return np.array(out)


def turn(x, position, theta, layout="half", magnitude=1.0, inverse=False):
    """x [tokens, heads, d] by the complex product of every plane."""
    y = np.array(x, dtype=np.float64)
    n = len(theta)
    ang = np.asarray(position, np.float64)[:, None] * theta[None] * (-1 if inverse else 1)
    f = magnitude * np.exp(1j * ang)[:, None]
    a, b = ((slice(0, n), slice(n, 2 * n)) if layout == "half" else
            (slice(0, 2 * n, 2), slice(1, 2 * n, 2)))
    z = (y[..., a] + 1j * y[..., b]) * f
    y[..., a], y[..., b] = z.real, z.imag
    return y


# ----------------------------------------------------------------- 8-bit pages
def _e4m3_values():
    v = np.zeros(256)
    for i in range(256):
        s, e, m = (-1.0 if i & 0x80 else 1.0), (i >> 3) & 15, i & 7
        v[i] = s * (m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    v[0x7F] = v[0xFF] = np.nan
    return v


E4M3 = _e4m3_values()


def quantize(x):
    """Rows x [..., d] as (bytes, exponents): the nearest e4m3 value, ties to the
    even byte, under the least power of two in range."""
    x = np.asarray(x, np.float64)
    big = np.finfo(np.float32).max
    y = np.clip(np.where(np.isnan(x), 0, x), -big, big)
    amax = np.max(np.abs(y), axis=-1, keepdims=True)
    e = np.full(amax.shape, -112)
    while np.any(up := (amax > 448.0 * 2.0 ** e) & (e < 119)):
        e = e + up
    z = np.minimum(np.abs(y) / 2.0 ** e, 448.0)
    grid = E4M3[:0x7F]
    hi = np.clip(np.searchsorted(grid, z), 0, 0x7E)
    lo = np.maximum(hi - 1, 0)
    d_lo, d_hi = z - grid[lo], grid[hi] - z
    pick = np.where(d_lo < d_hi, lo, np.where(d_hi < d_lo, hi, np.where(lo % 2 == 0, lo, hi)))
    byte = pick | np.where(np.signbit(x), 0x80, 0)
    byte = np.where(np.isnan(x), 0x7F, byte)
    return byte.astype(np.uint8), e[..., 0]


def offsets(s, d, H, h):
    """Byte offsets in a page of slot s, head h: key columns, value columns,
    key scale, value scale."""
    n, q, v = s // 16, s % 16 // 4, s % 4
    base = h * (128 * d + 128)
    j = np.arange(d)
    key = base + n * 16 * d + (j // 16) * 256 + (s % 16) * 16 + j % 16
    val = base + 64 * d + (j // 16) * 1024 + q * 256 + (j % 16) * 16 + n * 4 + v
    sk = base + 128 * d + q * 16 + n * 4 + v
    return key, val, sk, sk + 64


def write(pool, slot, k, v):
    """Append rows k, v [tokens, H, d] (already turned) into pool [pages, bytes]."""
    n, H, d = k.shape
    kb, ke = quantize(k)
    vb, ve = quantize(v)
    for t in range(n):
        if 0 <= slot[t] < pool.shape[0] * PAGE:
            page = pool[slot[t] // PAGE]
            for h in range(H):
                key, val, sk, sv = offsets(int(slot[t] % PAGE), d, H, h)
                page[key], page[val] = kb[t, h], vb[t, h]
                page[sk], page[sv] = ke[t, h] + 127, ve[t, h] + 127


def read(pool, slot, H, d):
    k = np.zeros((len(slot), H, d))
    v = np.zeros((len(slot), H, d))
    for t, sl in enumerate(slot):
        if 0 <= sl < pool.shape[0] * PAGE:
            page = pool[sl // PAGE]
            for h in range(H):
                key, val, sk, sv = offsets(int(sl % PAGE), d, H, h)
                k[t, h] = E4M3[page[key]] * 2.0 ** (int(page[sk]) - 127)
                v[t, h] = E4M3[page[val]] * 2.0 ** (int(page[sv]) - 127)
    return k, v


def decode(q, pool, table, lens, H):
    """q [batch, Q, H_q, d]; returns the outputs and the scales of their rounding
    errors: per value sum_t p_t |v_t|, per row max_t sum_j |q_j k_tj| / sqrt(d)."""
    B, Q, Hq, d = q.shape
    per = Hq // H
    out, mag, dot = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:3])
    for b in range(B):
        T = min(max(int(lens[b]), 0), table.shape[1] * PAGE)
        pos = np.arange(T)
        page = table[b, pos // PAGE].astype(np.int64) if T else np.zeros(0, np.int64)
        ok = (page >= 0) & (page < pool.shape[0])
        k, v = read(pool, np.where(ok, page * PAGE + pos % PAGE, -1), H, d)
        for i in range(Q):
            see = ok & (pos <= T - Q + i)
            if not see.any():
                continue
            for h in range(Hq):
                s = k[see, h // per] @ q[b, i, h].astype(np.float64) / math.sqrt(d)
                dot[b, i, h] = np.max(np.abs(k[see, h // per]) @ np.abs(q[b, i, h].astype(np.float64))) / math.sqrt(d)
                with np.errstate(invalid="ignore", over="ignore"):
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    out[b, i, h] = p @ v[see, h // per]
                    mag[b, i, h] = p @ np.abs(v[see, h // per])
    return out, mag, dot
