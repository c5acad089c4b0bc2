"""fp64 oracle of the paged key/value cache: E4M3 rows with power-of-two scales, rows into and out of
pages, attention over the cached rows.  Written from the definitions in include/eb.h."""
from __future__ import annotations

import numpy as np

from .eb_oracle import block_attention

E_MIN, E_MAX = -100, 120      # range of a row's exponent
NAN_CODE = 0x7F


def e4m3_values() -> np.ndarray:
    """The 256 values of E4M3 (sign, 4 exponent bits with bias 7, 3 mantissa bits; codes 0x7f and
    0xff are NaN)."""
    out = np.empty(256)
    for c in range(256):
        expo, frac = (c >> 3) & 15, c & 7
        mag = (8 + frac) * 2.0 ** (expo - 10) if expo else frac * 2.0 ** -9
        out[c] = np.nan if c & 0x7F == NAN_CODE else (-mag if c & 0x80 else mag)
    return out


def round_e4m3(y) -> np.ndarray:
    """Codes of the E4M3 values nearest to y (|y| <= 448; a tie goes to the even code; NaN and
    infinities to NaN).  The sign of a NaN is not defined and is cleared."""
    y = np.asarray(y, np.float64)
    mags = e4m3_values()[:NAN_CODE]                     # 0 .. 448, one per code
    mid = (mags[1:] + mags[:-1]) / 2
    a = np.where(np.isfinite(y), np.abs(y), 0.0)
    assert a.max(initial=0.0) <= 448.0
    code = np.searchsorted(mid, a, side="left")         # codes whose upper border lies below a
    code = np.where((code < len(mid)) & (a == mid[np.minimum(code, len(mid) - 1)]) & (code % 2 == 1),
                    code + 1, code)
    code = np.where(np.signbit(y), code | 0x80, code)
    return np.where(np.isfinite(y), code, NAN_CODE).astype(np.uint8)


def quantise(rows):
    """(codes, scale bytes) of rows [..., d], one scale per row."""
    x = np.asarray(rows, np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0).max(-1)
    e = np.full(a.shape, E_MIN)
    for c in range(E_MIN, E_MAX):                       # the smallest e with a <= 448 2^e
        e = np.where(a > 448.0 * 2.0 ** c, c + 1, e)
    with np.errstate(invalid="ignore"):
        codes = round_e4m3(x * 2.0 ** -e[..., None].astype(np.float64))
    return codes, (e + 127).astype(np.uint8)


def dequantise(codes, scale) -> np.ndarray:
    return e4m3_values()[codes] * 2.0 ** (np.asarray(scale, np.float64) - 127)[..., None]


def place(table, b, pos, page_size, n_pages):
    """(page, slot) of position pos of sequence b, or None: no such page."""
    j = pos // page_size
    if pos < 0 or j >= table.shape[1] or not 0 <= table[b, j] < n_pages:
        return None
    return int(table[b, j]), pos % page_size


def kv_write(pool, table, rows, cu_block, cached, pos=None) -> None:
    """rows [T, hkv, d] (anything the pool holds: values, codes, scale bytes) into
    pool [n_pages, hkv, page_size, ...] in place."""
    for b in range(len(cu_block) - 1):
        for i in range(cu_block[b], cu_block[b + 1]):
            p = int(pos[i]) if pos is not None else int(cached[b]) + i - cu_block[b]
            at = place(table, b, p, pool.shape[2], pool.shape[0])
            if at is not None:
                pool[at[0], :, at[1]] = rows[i]


def kv_read(values, table, cached) -> np.ndarray:
    """Packed rows [S, hkv, d] of the first cached[b] positions of every sequence; values
    [n_pages, hkv, page_size, d].  Rows without a page are zeros."""
    out = []
    for b, n in enumerate(cached):
        for p in range(n):
            at = place(table, b, p, values.shape[2], values.shape[0])
            out.append(np.zeros_like(values[0, :, 0]) if at is None else values[at[0], :, at[1]])
    return np.stack(out) if out else np.zeros((0, values.shape[1], values.shape[3]))


def paged_attention(q, k_blk, v_blk, k_values, v_values, table, cu_block, cached, hq, hkv,
                    scale=None):
    """Block attention whose prefix is the cached rows of every sequence."""
    cu = np.concatenate([[0], np.cumsum(cached)]).astype(np.int32)
    return block_attention(q, k_blk, v_blk, kv_read(k_values, table, cached),
                           kv_read(v_values, table, cached), cu_block, cu, hq, hkv, scale=scale)
