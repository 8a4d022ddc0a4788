"""Plain fp64 definitions of 8-bit codes with a power of two as scale for each 128 columns, of products of their values, of the
root-mean-square norm with its gradients, and of the limit on the norm of all gradients. Independent of the library."""
from __future__ import annotations

import numpy as np

BLOCK = 128
NAN_CODE = 0x7F


def code_values() -> np.ndarray:
    """The number that each byte stands for: sign, 4 exponent bits (bias 7), 3 fraction bits; all ones is NaN."""
    out = np.empty(256)
    for b in range(256):
        sign = -1.0 if b & 0x80 else 1.0
        e, f = (b >> 3) & 15, b & 7
        out[b] = sign * (f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))
        if b & 0x7F == 0x7F:
            out[b] = np.nan
    return out


_VALUES = code_values()


def nearest_codes(v: np.ndarray) -> np.ndarray:
    """Bytes of the numbers nearest to v (|v| <= 448), the even fraction where two are as near; NaN for what is not finite."""
    mags = _VALUES[:0x7F]                                    # ascending, 0 .. 448
    a = np.abs(np.where(np.isfinite(v), v, 0.0))
    hi = np.clip(np.searchsorted(mags, a), 0, len(mags) - 1)     # first magnitude >= a
    lo = np.maximum(hi - 1, 0)
    up, down = mags[hi] - a, a - mags[lo]
    pick = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    pick = np.where(mags[hi] == a, hi, pick)
    out = np.where(np.signbit(v), pick | 0x80, pick)
    return np.where(np.isfinite(v), out, NAN_CODE).astype(np.uint8)


def exponent(a: float) -> int:
    """Smallest e >= -127 with a 2^-e <= 448; 0 for a = 0."""
    if a == 0:
        return 0
    e = -127
    while a > 448.0 * 2.0 ** e:
        e += 1
    return e


def _block_exponent(v):
    f = np.abs(v[np.isfinite(v)])
    return exponent(float(f.max())) if f.size else 0


def quantize_rows(v: np.ndarray):
    """(codes [n, w], exponents [n, blocks])."""
    n, w = v.shape
    nb = -(-w // BLOCK)
    codes, exps = np.empty((n, w), dtype=np.uint8), np.empty((n, nb), dtype=np.int64)
    for i in range(n):
        for b in range(nb):
            at = slice(BLOCK * b, BLOCK * (b + 1))
            exps[i, b] = _block_exponent(v[i, at])
            codes[i, at] = nearest_codes(v[i, at] * 2.0 ** -float(exps[i, b]))
    return codes, exps


def quantize_weights(h: np.ndarray):
    """(codes [r, c], exponents [blocks of r, blocks of c])."""
    r, c = h.shape
    exps = np.empty((-(-r // BLOCK), -(-c // BLOCK)), dtype=np.int64)
    codes = np.empty((r, c), dtype=np.uint8)
    for i in range(exps.shape[0]):
        for j in range(exps.shape[1]):
            at = (slice(BLOCK * i, BLOCK * (i + 1)), slice(BLOCK * j, BLOCK * (j + 1)))
            exps[i, j] = _block_exponent(h[at])
            codes[at] = nearest_codes(h[at] * 2.0 ** -float(exps[i, j]))
    return codes, exps


def values(codes: np.ndarray, exps: np.ndarray) -> np.ndarray:
    """What rows of codes stand for."""
    w = codes.shape[1]
    return _VALUES[codes] * np.repeat(2.0 ** exps.astype(np.float64), BLOCK, axis=1)[:, :w]


def weight_values(codes: np.ndarray, exps: np.ndarray) -> np.ndarray:
    r, c = codes.shape
    s = 2.0 ** exps.astype(np.float64)
    return _VALUES[codes] * np.repeat(np.repeat(s, BLOCK, axis=0)[:r], BLOCK, axis=1)[:, :c]


def rms_norm(u: np.ndarray, gain, eps: float):
    """(y, 1 / rms) of rows u."""
    inv = 1.0 / np.sqrt((u * u).mean(axis=1) + eps)
    return u * inv[:, None] * gain, inv


def rms_norm_backward(dy: np.ndarray, u: np.ndarray, gain, inv: np.ndarray):
    """(gradient of u, gradient of the gain) of rms_norm, 1 / rms given."""
    v = u * inv[:, None]
    h = dy * gain
    return inv[:, None] * (h - v * (h * v).mean(axis=1, keepdims=True)), (dy * v).sum(axis=0)


def limit(grads, max_norm: float):
    """(norm of all gradients together, factor that limits it)."""
    norm = float(np.sqrt(sum(float((g.astype(np.float64) ** 2).sum()) for g in grads)))
    return norm, 1.0 if norm <= max_norm else max_norm / norm
