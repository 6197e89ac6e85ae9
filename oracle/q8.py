"""fp64 oracle of the 8-bit KV cache and the rotation -- TEST INFRASTRUCTURE ONLY.

The 8-bit types are taken from their definition (sign, exponent, mantissa of
every one of the 256 codes), and rounding is a search for the nearest value,
ties to the even code: no conversion of any library is used.

kv_write_q8 goes page by page in plain loops: a page of 16 tokens and one KV
head has one power-of-two scale; slots that a partial write leaves in a page
keep their values, requantised when the scale grows.  dequantise gives the
pools' values in fp64, which window_attention takes as they are.  rotary turns
pairs of dims by exact phases.
"""
from __future__ import annotations

import math
from fractions import Fraction

import numpy as np

PAGE = 16
FORMATS = {"e4m3": (4, 3, 7, 448.0), "e5m2": (5, 2, 15, 57344.0)}    # exponent and mantissa bits, bias, top
MIN_EXP, MAX_EXP = -100, 120


def decode_table(fmt):
    """The 256 codes' values: e4m3 has no infinities and NaN at 0x7F and 0xFF,
    e5m2 is IEEE-like (0x7C infinity, 0x7D to 0x7F NaN)."""
    eb, mb, bias, _ = FORMATS[fmt]
    out = np.empty(256)
    for code in range(256):
        sign = -1.0 if code & 0x80 else 1.0
        e, m = (code >> mb) & ((1 << eb) - 1), code & ((1 << mb) - 1)
        if fmt == "e4m3" and (code & 0x7F) == 0x7F:
            v = math.nan
        elif fmt == "e5m2" and e == 31:
            v = math.inf if m == 0 else math.nan
        elif e == 0:
            v = m * 2.0 ** (1 - bias - mb)
        else:
            v = (1 + m / (1 << mb)) * 2.0 ** (e - bias)
        out[code] = sign * v
    return out


def encode(x, fmt):
    """Codes of x (fp64): the nearest finite value, ties to the even code,
    infinities to the largest finite one, NaN to 0x7F."""
    x = np.asarray(x, dtype=np.float64)
    table = decode_table(fmt)[:128]
    n = int(np.sum(np.isfinite(table)))
    vals = table[:n]                                     # 0 .. top, ascending with the code
    a = np.minimum(np.abs(np.where(np.isnan(x), 0, x)), vals[-1])
    hi = np.clip(np.searchsorted(vals, a), 1, n - 1)
    lo = hi - 1
    below, above = a - vals[lo], vals[hi] - a
    pick = np.where(below < above, lo, np.where(above < below, hi, np.where(lo % 2 == 0, lo, hi)))
    code = pick.astype(np.int64) | np.where(np.signbit(x), 0x80, 0)
    return np.where(np.isnan(x), 0x7F, code).astype(np.uint8)


def page_scale(amax, fmt):
    """Smallest power of two s in [2^-100, 2^120] with amax / s <= top."""
    top = Fraction(FORMATS[fmt][3])
    e = MIN_EXP
    while e < MAX_EXP and Fraction(float(amax)) > top * Fraction(2) ** e:
        e += 1
    return 2.0 ** e


def _codes(t):
    if hasattr(t, "detach"):
        import torch
        return t.detach().cpu().contiguous().view(torch.uint8).numpy()
    return np.asarray(t)


def _np(t):
    if hasattr(t, "detach"):
        t = t.detach().cpu()
        return t.double().numpy() if t.is_floating_point() else t.numpy().astype(np.int64)
    return np.asarray(t)


def kv_write_q8(k_pages, v_pages, k_scales, v_scales, page_table, start_pos, lens, k_new, v_new, fmt, kv_lens=None,
                block_flags=None, block_size=None):
    """Updated copies: (K codes, V codes, K scales, V scales)."""
    pools = [_codes(k_pages).copy(), _codes(v_pages).copy()]
    scales = [_np(k_scales).astype(np.float32).copy(), _np(v_scales).astype(np.float32).copy()]
    new = [_np(k_new), _np(v_new)]
    pt, st, n = _np(page_table), _np(start_pos), _np(lens)
    held = st if kv_lens is None else np.maximum(st, _np(kv_lens))
    flags = None if block_flags is None else _np(block_flags)
    table = decode_table(fmt)
    heads = pools[0].shape[1]
    row0 = 0
    for b in range(len(st)):
        first, last = int(st[b]), int(st[b] + n[b])
        for j in range(first // PAGE, -(-last // PAGE) if last > first else 0):
            if j >= pt.shape[1] or not 0 <= pt[b, j] < pools[0].shape[0]:
                continue
            pid = int(pt[b, j])
            written, kept = [], []
            for s in range(PAGE):
                pos = j * PAGE + s
                inside = first <= pos < last
                if inside and (flags is None or flags[b, (pos - first) // block_size]):
                    written.append(s)
                elif pos < held[b]:
                    kept.append(s)
            if not written:
                continue
            for i in range(2):
                for g in range(heads):
                    x = np.stack([new[i][row0 + j * PAGE + s - first, g] for s in written])
                    fin = np.abs(x[np.isfinite(x)])
                    scale = page_scale(fin.max() if fin.size else 0.0, fmt)
                    page = pools[i][pid, g] if i == 0 else pools[i][pid, g].T       # [16, D], a view
                    if kept:
                        old = float(scales[i][pid, g])
                        scale = max(scale, old)
                        if scale > old:
                            page[kept] = encode(table[page[kept]] * (old / scale), fmt)
                    page[written] = encode(x / scale, fmt)
                    scales[i][pid, g] = scale
        row0 += int(n[b])
    return pools[0], pools[1], scales[0], scales[1]


def dequantise(pages, scales, fmt):
    """Values of a pool, fp64."""
    s = _np(scales).astype(np.float64)
    return decode_table(fmt)[_codes(pages)] * s[:, :, None, None]


def kv_read_q8(k_pages, v_pages, k_scales, v_scales, page_table, start_pos, lens, fmt):
    """K and V of the ranges, fp64 [rows, heads, D]; zeros off the table."""
    K, V = dequantise(k_pages, k_scales, fmt), dequantise(v_pages, v_scales, fmt)
    pt, st, n = _np(page_table), _np(start_pos), _np(lens)
    ks, vs = [], []
    for b in range(len(st)):
        for pos in range(int(st[b]), int(st[b] + n[b])):
            j, s = pos // PAGE, pos % PAGE
            if j >= pt.shape[1] or not 0 <= pt[b, j] < K.shape[0]:
                ks.append(np.zeros((K.shape[1], K.shape[3])))
                vs.append(np.zeros((K.shape[1], K.shape[3])))
            else:
                ks.append(K[pt[b, j], :, s])
                vs.append(V[pt[b, j], :, :, s])
    shape = (0, K.shape[1], K.shape[3])
    return (np.stack(ks), np.stack(vs)) if ks else (np.zeros(shape), np.zeros(shape))


def rotary(x, positions, turns, scale=1.0, interleaved=False, inverse=False):
    """x [rows, heads, D] fp64, position of each row; turns: integers, 2^-64 of
    a turn per position."""
    x = _np(x).astype(np.float64)
    half = len(turns)
    y = x.copy()
    for i, t in enumerate(int(v) for v in turns):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        # the phase in whole units of 2^-64 turns, exactly; then its angle in fp64
        angle = np.array([2 * math.pi * (((int(n) * t) % (1 << 64)) / 2.0 ** 64) for n in positions])
        c, s = scale * np.cos(angle)[:, None], scale * np.sin(angle)[:, None] * (-1 if inverse else 1)
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y
