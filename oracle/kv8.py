"""The cache held in 8 bits, and the append that fills it, in float64 numpy.  For
checking only.

TEST INFRASTRUCTURE ONLY: the product library never uses this module, and
nothing here is shared with it.

A value is code * 2^(byte - 127), a code one of e4m3's numbers (4 significant bits,
exponents -6 .. 8, multiples of 2^-9 below 2^-6, at most 448, no infinity).
"""
from __future__ import annotations

import numpy as np

from . import chunk

LOWEST, HIGHEST = 27, 227


def code_values() -> np.ndarray:
    """The number that each of the 256 codes stands for."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    x = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    x = np.where((c & 127) == 127, np.nan, x)
    return np.where(c < 128, x, -x)


def values(codes, scales, which):
    """codes uint8 [pages][heads][16][D] and their bytes as numbers (which: 0 keys, 1 values)."""
    return code_values()[codes] * np.exp2(scales[..., which].astype(np.float64) - 127)[..., None, None]


def half_step(x):
    """The largest error of rounding x to e4m3 (up to 448)."""
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.maximum(np.floor(np.log2(np.abs(x))), -6.0)
    return np.exp2(e - 4)


def power_byte(amax) -> int:
    """The byte of the smallest power with amax <= 448 * power, inside the range that is written."""
    if not amax > 0:
        return LOWEST
    m, e = np.frexp(amax)             # amax = m 2^e, 1/2 <= m < 1;  448 = 0.875 2^9
    return int(np.clip(e - (9 if m <= 0.875 else 8) + 127, LOWEST, HIGHEST))


def append(q, k, v, k_codes, v_codes, scales, table, ctx, starts, inv_freq, q_norm=None, k_norm=None, eps=1e-6,
           interleaved=False):
    """(q_out, want_k, want_v, scales): want[page][head][slot][:] is what the slot's
    codes stand for relative to the page's power, before the rounding to e4m3 (of
    held tokens too); NaN in slots that the call leaves alone, infinite where the
    code is NaN."""
    T, P = q.shape[0], k_codes.shape[2]
    shape = k_codes.shape
    q_out, kx, vx = chunk.rope_append(q, k, v, np.zeros(shape), np.zeros(shape), table, ctx, starts, inv_freq, q_norm,
                                      k_norm, eps, interleaved)
    scales = scales.copy()
    want = [np.full(shape, np.nan), np.full(shape, np.nan)]
    number = code_values()
    for b in range(len(ctx)):
        a, e = chunk._owned(starts, b, T)
        L = chunk._length(ctx, b, table, P)
        first = L - (e - a)
        for page in range(max(first, 0) // P, (L - 1) // P + 1 if L > 0 and e > a else 0):
            pid = int(table[b][page])
            if not 0 <= pid < shape[0]:
                continue
            lo, hi = max(first - page * P, 0), min(L - page * P, P)
            for which, (x, codes) in enumerate(((kx, k_codes), (vx, v_codes))):
                for g in range(shape[1]):
                    new = x[pid, g, lo:hi]
                    fine = np.abs(new[np.isfinite(new)])
                    byte = power_byte(fine.max() if fine.size else 0.0)
                    if lo > 0:
                        byte = min(max(byte, int(scales[pid, g, which])), HIGHEST)
                        held = number[codes[pid, g, :lo]] * 2.0 ** (int(scales[pid, g, which]) - byte)
                        want[which][pid, g, :lo] = np.where(np.isnan(held), np.inf, held)
                    scaled = np.clip(new / 2.0 ** (byte - 127), -448.0, 448.0)
                    want[which][pid, g, lo:hi] = np.where(np.isfinite(new), scaled, np.inf)
                    scales[pid, g, which] = byte
    return q_out, want[0], want[1], scales
