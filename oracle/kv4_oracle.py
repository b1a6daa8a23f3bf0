"""CPU oracle for the 4-bit prefix cache and for the rows made from projections (fp64, numpy).

TEST INFRASTRUCTURE ONLY: the plain statement of what the library's entry points compute, sharing no code with them.
A page holds 32 rows of one head: key codes [D / 32][32][16 bytes], value codes [D][16 bytes], then bf16 key scale,
key offset, value scale and value offset of the 32 rows.  Value 8 w + 2 i + h of 16 bytes is the nibble at bits
4 i + 16 h of the little-endian 32-bit word w.
"""
from __future__ import annotations

import numpy as np

ROWS = 32


def to_bf16(x):
    """Nearest bf16 (ties to even) of fp32-rounded values, as float64, and its bit pattern."""
    bits = np.asarray(x, dtype=np.float64).astype(np.float32).view(np.uint32).astype(np.uint64)
    up = (bits + 0x7FFF + ((bits >> np.uint64(16)) & np.uint64(1))) >> np.uint64(16)
    up = up.astype(np.uint16)
    return (up.astype(np.uint32) << 16).view(np.float32).astype(np.float64), up


def quantise_row(x):
    """(codes, scale, offset, scale bits, offset bits) of one row."""
    x = np.asarray(x, dtype=np.float64)
    lo, hi = x.min() + 0.0, x.max() + 0.0                     # a zero is +0
    s, s_bits = to_bf16((hi - lo) / 15.0)
    o, o_bits = to_bf16(lo - 16.0 * s)
    if s > 0:
        codes = np.clip(np.rint((x - o) / s) - 16, 0, 15).astype(np.int64)
    else:
        codes = np.zeros(len(x), dtype=np.int64)
    return codes, float(s), float(o), int(s_bits), int(o_bits)


def stored_row(x):
    codes, s, o, _, _ = quantise_row(x)
    return s * (16.0 + codes) + o


def _place(e):
    """Byte and shift of value e (0..31) inside its 16 bytes."""
    w, i, h = e // 8, (e % 8) // 2, e % 2
    bit = 4 * i + 16 * h
    return 4 * w + bit // 8, bit % 8


def _key_place(D, r, d):
    byte, shift = _place(d % 32)
    return (d // 32) * ROWS * 16 + r * 16 + byte, shift


def _value_place(D, r, d):
    byte, shift = _place(r)
    return 16 * D + d * 16 + byte, shift


def _put(page, place, code):
    byte, shift = place
    page[byte] = (int(page[byte]) & ~(15 << shift) & 0xFF) | (int(code) << shift)


def write_row(cache, b, h, row, k, v):
    """Stores rows k, v [D] as row `row` of cache [B][H][pages][bytes] in place; rows outside the cache are dropped."""
    D = len(k)
    if row < 0 or row >= cache.shape[2] * ROWS:
        return
    page, r = cache[b, h, row // ROWS], row % ROWS
    scales = page[32 * D:].view(np.uint16)
    for which, (x, place) in enumerate(((k, _key_place), (v, _value_place))):
        codes, _, _, s_bits, o_bits = quantise_row(x)
        for d in range(D):
            _put(page, place(D, r, d), codes[d])
        scales[64 * which + r] = s_bits
        scales[64 * which + ROWS + r] = o_bits


def read_rows(cache, D):
    """Dense (k, v) [B][H][pages * 32][D] in fp64."""
    B, H, P, _ = cache.shape
    out = []
    scales = np.ascontiguousarray(cache[..., 32 * D:]).view(np.uint16).astype(np.uint32) << 16
    scales = scales.view(np.float32).astype(np.float64).reshape(B, H, P, 4, ROWS)
    for which, place in enumerate((_key_place, _value_place)):
        codes = np.zeros((B, H, P, ROWS, D))
        for r in range(ROWS):
            for d in range(D):
                byte, shift = place(D, r, d)
                codes[:, :, :, r, d] = (cache[..., byte].astype(np.int64) >> shift) & 15
        with np.errstate(invalid="ignore"):
            rows = scales[:, :, :, 2 * which, :, None] * (16.0 + codes) + scales[:, :, :, 2 * which + 1, :, None]
        out.append(rows.reshape(B, H, P * ROWS, D))
    return out[0], out[1]


def commit(cache, k_tree, v_tree, seq_lens, accept_len, out_nodes, best_root):
    """The winning root's and the accepted nodes' rows into the cache, in place; returns the new lengths."""
    B, H = cache.shape[:2]
    L_max = cache.shape[2] * ROWS
    new = np.array(seq_lens, copy=True)
    for b in range(B):
        nodes = [int(best_root[b])] + [int(x) for x in out_nodes[b][:int(accept_len[b])]]
        for i, n in enumerate(nodes):
            for h in range(H):
                write_row(cache, b, h, int(seq_lens[b]) + i, k_tree[b, h, n], v_tree[b, h, n])
        new[b] = min(L_max, int(seq_lens[b]) + len(nodes))
    return new


def norm_rope(x, weight, eps, freqs, positions, interleaved, rotate=True):
    """Rows x [B][N][H][D] normalised (where there is a weight), rotated by positions [B][N], as [B][H][N][D]; and the
    length of every rotated pair before rotation (the scale of its rounding errors), same shape."""
    x = np.asarray(x, dtype=np.float64).transpose(0, 2, 1, 3).copy()
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)
    size = np.abs(x)
    if not rotate:
        return x, size
    half = len(freqs)
    for i in range(half):
        a, c = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        ang = np.asarray(positions, dtype=np.float64)[:, None, :] * float(freqs[i])
        ya, yc = x[..., a].copy(), x[..., c].copy()
        x[..., a] = ya * np.cos(ang) - yc * np.sin(ang)
        x[..., c] = yc * np.cos(ang) + ya * np.sin(ang)
        size[..., a] = size[..., c] = np.abs(ya) + np.abs(yc)
    return x, size
