"""The paged cache's two calls in float64, sequence by sequence and head by head (include/esa_paged.h is what they define)."""
from __future__ import annotations

import math

import numpy as np

F8_MAX = 448.0


def e4m3_table() -> np.ndarray:
    """The number of every e4m3 byte (OCP: no infinities, 0x7F and 0xFF are NaN)."""
    out = np.empty(256)
    for byte in range(256):
        e, m = byte >> 3 & 15, byte & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        if byte & 127 == 127:
            x = math.nan
        out[byte] = -x if byte >> 7 else x
    return out


def to_e4m3(x: np.ndarray) -> np.ndarray:
    """Nearest e4m3 numbers, ties to even; magnitudes over 448 become 448."""
    x = np.clip(np.asarray(x, dtype=np.float64), -F8_MAX, F8_MAX)
    _, e = np.frexp(x)                                          # |x| = m 2^e, m in [1/2, 1): a step is 2^(e-4), 2^-9 at least
    step = np.exp2(np.maximum(e - 4, -9).astype(np.float64))
    return np.rint(x / step) * step


def scale_byte(amax: float) -> int:
    """Exponent byte of the smallest power of two s in 2^-100 .. 2^112 with amax <= 448 s."""
    byte = 27
    while byte < 239 and amax > F8_MAX * 2.0 ** (byte - 127):
        byte += 1
    return byte


def turn(x: np.ndarray, pos: np.ndarray, base: float) -> np.ndarray:
    """Rows [n, heads, d] turned to positions pos [n] (rotate-half pairing)."""
    half = x.shape[-1] // 2
    angle = np.asarray(pos, dtype=np.float64)[:, None, None] * base ** (-2.0 * np.arange(half) / x.shape[-1])
    c, s = np.cos(angle), np.sin(angle)
    a, b = x[..., :half], x[..., half:]
    return np.concatenate((a * c - b * s, b * c + a * s), -1)


def append_blocks(values: np.ndarray, scale: np.ndarray, rows: np.ndarray, t0: int, pages, page_size: int) -> None:
    """8-bit pool [n_pages, h_kv, page_size, d] of e4m3 numbers and exponent bytes [n_pages, h_kv]: rows [n, h_kv, d] go to positions
    t0, t0 + 1, ... of the sequence that has `pages`."""
    n, h_kv, _ = rows.shape
    for p in range(t0 // page_size, -(-(t0 + n) // page_size)) if n else ():
        page, lo, hi = pages[p], max(t0 - p * page_size, 0), min(t0 + n - p * page_size, page_size)
        if not 0 <= page < values.shape[0]:
            continue
        for g in range(h_kv):
            new = rows[p * page_size + lo - t0:p * page_size + hi - t0, g]
            byte = scale_byte(float(np.max(np.abs(new))))
            if lo > 0:
                old = int(scale[page, g])
                byte = max(byte, old)
                values[page, g, :lo] = to_e4m3(values[page, g, :lo] * 2.0 ** (old - byte))
            values[page, g, lo:hi] = to_e4m3(new * 2.0 ** (127 - byte))
            scale[page, g] = byte


def visible(t0: int, n: int, l_i, l_l: int, idx) -> list:
    """Positions that the tokens t0 .. t0+n-1 choose from."""
    if l_i is None:
        return list(range(t0 + n))
    i_end = min(l_i, t0)
    l_start = max(t0 - l_l, i_end)
    chosen = [] if idx is None else [int(p) for p in idx if i_end <= p < l_start]
    return list(range(i_end)) + chosen + list(range(l_start, t0 + n))


def attend(q: np.ndarray, t0: int, K: np.ndarray, V: np.ndarray, positions, scale: float, cap: float = 0.0):
    """q [n, h, d]; K, V [len(positions), h_kv, d], the rows at `positions` -> out [n, h, d], lse [n, h], and per row what error bounds
    need: sum_j p_j |v_j| [n, h, d] and the largest sum |q||k_j| scale [n, h]."""
    n, h, d = q.shape
    group = h // K.shape[1]
    out, spread = np.zeros(q.shape), np.zeros(q.shape)
    lse, most = np.full((n, h), -math.inf), np.zeros((n, h))
    at = np.asarray(positions, dtype=np.int64)
    for i in range(h):
        k, v = K[:, i // group], V[:, i // group]
        x = q[:, i] @ k.T * scale
        if cap > 0:
            x = cap * np.tanh(x / cap)
        there = at[None, :] <= t0 + np.arange(n)[:, None]
        x = np.where(there, x, -math.inf)
        rows = there.any(1)
        if not rows.any():
            continue
        m = x[rows].max(1, keepdims=True)
        p = np.exp(x[rows] - m)
        l = p.sum(1, keepdims=True)
        lse[rows, i] = (m + np.log(l))[:, 0]
        out[rows, i] = p / l @ v
        spread[rows, i] = p / l @ np.abs(v)
        most[rows, i] = np.max(np.where(there, np.abs(q[:, i]) @ np.abs(k).T * scale, 0.0), axis=1)[rows]
    return out, lse, spread, most
