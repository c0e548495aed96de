"""Paged KV cache in float64: element order of a page, the append with rotation, attention over the pages.

Caches are arrays of numbers [pages, kv heads, page_size * d] (what the stored elements hold, scales not applied), a table is an
integer array [rows, pages per row] with -1 for a page that is not there."""
import numpy as np


def key_offset(pos, j, page_size, d, piece):
    """Place of (position, head dim) in a (page, head): blocks of 32 positions, pieces of 8 (bf16) or 16 (e4m3) head dims,
    piece by piece, position by position."""
    p = pos % page_size
    return (p // 32) * 32 * d + ((j // piece) * 32 + p % 32) * piece + j % piece


def value_offset(pos, j, page_size, d, piece):
    """The same for values: a position 16 t + 8 a + 4 h + b of its block is element 4 a + b of piece 2 t + h (bf16), or element
    8 t + 4 a + b of piece h (e4m3); a piece holds every head dim."""
    p = pos % page_size
    q = p % 32
    t, a, h, b = q // 16, q // 8 % 2, q // 4 % 2, q % 4
    if piece == 8:
        return (p // 32) * 32 * d + ((2 * t + h) * d + j) * 8 + 4 * a + b
    return (p // 32) * 32 * d + (h * d + j) * 16 + 8 * t + 4 * a + b


def places(table_row, pos, n_heads, page_size, d, piece):
    """Index arrays (page, head, key element), (page, head, value element), each broadcasting to [len(pos), heads, d];
    every page has to be there."""
    pos = np.asarray(pos)
    page = np.asarray(table_row)[pos // page_size][:, None, None]
    assert np.all(page >= 0)
    head = np.arange(n_heads)[None, :, None]
    j = np.arange(d)[None, None, :]
    p = pos[:, None, None]
    return (page, head, key_offset(p, j, page_size, d, piece)), (page, head, value_offset(p, j, page_size, d, piece))


def rotate(x, pos, table):
    """x [n, heads, d] at positions pos: element j turned with j + d/2 by the table's [pos, d/2, (cos, sin)]."""
    half = x.shape[-1] // 2
    c, s = table[pos][:, None, :, 0].astype(np.float64), table[pos][:, None, :, 1].astype(np.float64)
    lo, hi = x[..., :half], x[..., half:]
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], axis=-1)


def attention(q, k, v, positions, present, scale, window=0):
    """One sequence: q [n, Hq, d] at absolute positions `positions`, k and v [m, Hkv, d] of positions 0..m-1, present [m].
    Returns the output [n, Hq, d] and, element by element, how far it moves to first order where every q and every weight is
    off by the relative amounts (eps_q, eps_w): a function of the two."""
    n, hq, d = q.shape
    m, hkv, _ = k.shape
    g = hq // hkv
    out = np.zeros((n, hq, d))
    move_q = np.zeros((n, hq, d))
    move_w = np.zeros((n, hq, d))
    j = np.arange(m)
    seen = (j[None, :] <= positions[:, None]) & present[None, :]
    if window:
        seen &= j[None, :] > positions[:, None] - window
    for h in range(hq):
        kk, vv = k[:, h // g], v[:, h // g]
        kk, vv = np.where(present[:, None], kk, 0.0), np.where(present[:, None], vv, 0.0)
        s = scale * (q[:, h] @ kk.T)
        s = np.where(seen, s, -np.inf)
        top = np.max(s, axis=1, keepdims=True, initial=-np.inf)
        w = np.exp(s - np.where(np.isfinite(top), top, 0.0))
        total = w.sum(axis=1, keepdims=True)
        w = np.divide(w, total, out=np.zeros_like(w), where=total > 0)
        out[:, h] = w @ vv
        ds = scale * (np.abs(q[:, h]) @ np.abs(kk).T)         # how far a score can move per unit of eps_q
        mean = w @ np.abs(vv)
        move_q[:, h] = (w * ds) @ np.abs(vv) + (w * ds).sum(axis=1, keepdims=True) * mean
        move_w[:, h] = mean
    return out, lambda eps_q, eps_w: eps_q * move_q + eps_w * move_w
