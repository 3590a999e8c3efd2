"""fp64 oracle of rotary positions, the norms on both sides of a block and their gradients, and an AdamW step with moments in 32 or 8 bits.
numpy, one formula a line; test infrastructure only."""
from __future__ import annotations

import numpy as np


def rotary(x, positions, frequencies, n_positions, interleaved=False, transpose=False, magnitude=1.0):
    """x [rows, heads, d]; a row whose position is none of [0, n_positions) stays as it is."""
    out, r = x.copy(), 2 * len(frequencies)
    for t, p in enumerate(positions):
        if not 0 <= p < n_positions:
            continue
        for i, f in enumerate(frequencies):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
            c, s = magnitude * np.cos(p * f), magnitude * np.sin(p * f) * (-1 if transpose else 1)
            out[t, :, a] = x[t, :, a] * c - x[t, :, b] * s
            out[t, :, b] = x[t, :, a] * s + x[t, :, b] * c
    return out


def statistics(x, kind, eps):
    """[mean, 1 / deviation] of each row; the RMS norm has no mean."""
    mean = x.mean(1) if kind == "layer" else np.zeros(len(x))
    return np.stack([mean, 1 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)])


def normed(x, stats, weight, bias=None):
    out = (x - stats[0][:, None]) * stats[1][:, None] * weight
    return out if bias is None else out + bias


def norm_back(g, x, stats, kind):
    """Gradient of (x - mean) * rstd under g."""
    hat = (x - stats[0][:, None]) * stats[1][:, None]
    out = g - hat * (g * hat).mean(1, keepdims=True)
    if kind == "layer":
        out = out - g.mean(1, keepdims=True)
    return out * stats[1][:, None]


def gates(gate, rows, rows_per_gate):
    return 1.0 if gate is None else gate[np.arange(rows) // rows_per_gate]


# ---- moments in 8 bits --------------------------------------------------------------------------

BLOCK = 256
A, B = 0xC13FA9A9, 0x91E10DA5
CODES = np.sort(np.unique([m * 2.0 ** (max(e, 1) - 10) for e in range(16) for m in ([*range(8, 16)] if e else range(8)) if not (e == 15 and m == 15)]))


def exponent(x):
    return np.frexp(x)[1] - 1


def block_scale(values):
    """2^(e-7) of a block's values, e the exponent of the largest finite one, at least -119."""
    fine = np.abs(values[np.isfinite(values)])
    top = fine.max() if fine.size else 0.0
    return 2.0 ** (max(int(exponent(top)) if top > 0 else -119, -119) - 7)


def spread(i, step, a, b):
    """u of entry i at a step: 24 binary digits of the fraction of i a + step b."""
    return (((np.asarray(i, dtype=np.uint64) * np.uint64(a) + np.uint64((step * b) & 0xFFFFFFFF)) & np.uint64(0xFFFFFFFF)) >> np.uint64(8)).astype(np.float64) / 2 ** 24


def neighbours(x):
    """The codes around x in [0, 256)."""
    at = np.searchsorted(CODES, x, side="right") - 1
    return CODES[at], CODES[at + 1]


def code_m(m, scale, u):
    lo, hi = neighbours(np.abs(m) / scale)
    return np.sign(m) * np.where((np.abs(m) / scale - lo) / (hi - lo) > u, hi, lo)


def code_v(v, scale, u):
    x = np.maximum(v, 0.0) / scale ** 2
    lo, hi = neighbours(np.sqrt(x))
    code = np.where((x - lo ** 2) / (hi ** 2 - lo ** 2) > u, hi, lo)
    return np.where((v > 0) & (code == 0), CODES[1], code)


def adamw(w, g, m, v, step, lr, beta1, beta2, eps, weight_decay):
    """(w, m, v) after a step; g is what is left of the gradient after scale and clipping."""
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g ** 2
    w = w - lr * (m / (1 - beta1 ** step) / (np.sqrt(v / (1 - beta2 ** step)) + eps) + weight_decay * w)
    return w, m, v
