"""Oracle for 4-bit frozen weights and for the drawn dropout mask: numpy, 64 bits, written from the definitions.

The 4-bit weight: W[j, k] = scale[j, k // group] * v(q[j, k]), v(q) = q - zero (zero 8 where there are no zero points) or the
E2M1 float q.  The mask: Philox 4x32-10 (Salmon, Moraes, Dror, Shaw 2011), sixteen bits an element.
"""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0])


def four_bits(v, up=False):
    """v rounded to four significant bits: to nearest (ties to even), or upwards."""
    man, ex = np.frexp(np.asarray(v, dtype=np.float64))
    man = np.ceil(man * 16) if up else np.round(man * 16)
    return np.ldexp(man / 16, ex)


def groups_of(d_in, group):
    return -(-d_in // group)


def quantize(W, code, with_zero, group, store=lambda v: v, largest=np.inf):
    """(q, scale, zero or None) of W in 64 bits; `store` rounds the scale to the storage type, whose `largest` number no weight
    that is read back exceeds."""
    d_out, d_in = W.shape
    n = groups_of(d_in, group)
    q = np.zeros((d_out, d_in), dtype=np.uint8)
    scale = np.zeros((d_out, n))
    zero = np.zeros((d_out, n)) if with_zero else None
    for g in range(n):
        w = W[:, g * group:(g + 1) * group]
        odd = ~np.isfinite(w).all(axis=1)
        v = np.where(odd[:, None], 0.0, w)
        if with_zero:
            lo, hi = np.minimum(v.min(axis=1), 0), np.maximum(v.max(axis=1), 0)
            s = store(four_bits((hi - lo) / 15, up=True))
        else:
            s = store(four_bits(np.abs(v).max(axis=1) / (7 if code == "int4" else 6)))
            if code == "fp4" and np.isfinite(largest):      # the largest number of four bits whose six-fold is one
                s = np.minimum(s, four_bits(largest / 6 * (1 - 1 / 16)))
        some = s > 0
        d = np.where(some, s, 1.0)[:, None]
        most = np.floor(largest / d)
        if with_zero:
            z = np.where(some, np.clip(np.round(-lo / d[:, 0]), 0, 15), 0)
            c = np.where(some[:, None], np.clip(z[:, None] + np.clip(np.round(v / d), -most, most), 0, 15), z[:, None])
            zero[:, g] = np.where(odd, 0, z)
            c = np.where(odd[:, None], 0, c)
        elif code == "int4":
            c = np.where(some[:, None], np.clip(8 + np.clip(np.round(v / d), -most, most), 0, 15), 8)
            c = np.where(odd[:, None], 8, c)
        else:
            t = np.abs(v / d)
            dist = np.abs(t[:, :, None] - E2M1[:8])
            near = dist.min(axis=2, keepdims=True)
            # of the codes that are nearest the even one, where two are
            c = np.argmin(np.where(dist == near, np.arange(8) % 2, 2), axis=2) + 8 * (v < 0)
            c = np.where(some[:, None] & ~odd[:, None], c, 0)
        q[:, g * group:(g + 1) * group] = c
        scale[:, g] = np.where(odd, np.nan, s)
    return q, scale, zero


def pack(q):
    return q[:, 0::2] | (q[:, 1::2] << 4)


def weight(q, scale, zero, code, group):
    """The weight that codes and scales stand for."""
    at = np.arange(q.shape[1]) // group
    v = E2M1[q] if code == "fp4" else q.astype(np.float64) - (8 if zero is None else zero[:, at])
    return v * scale[:, at]


def philox(counter, key):
    """Ten rounds over a counter of four and a key of two 32-bit words."""
    c, k = [int(v) for v in counter], [int(v) for v in key]
    for _ in range(10):
        p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(q >> 32) ^ c[1] ^ k[0], q & 0xFFFFFFFF, (p >> 32) ^ c[3] ^ k[1], p & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def keep(seed, offset, n, p):
    """The first n decisions of a mask."""
    t = min(65535, int(np.rint(p * 65536)))
    out = np.zeros(-(-n // 8) * 8, dtype=bool)
    for b in range(-(-n // 8)):
        at = (offset + b) % 2 ** 64
        words = philox([at & 0xFFFFFFFF, at >> 32, 0, 0], [seed & 0xFFFFFFFF, seed >> 32])
        for j in range(8):
            out[b * 8 + j] = ((words[j // 2] >> (16 * (j % 2))) & 0xFFFF) >= t
    return out[:n]


def dropout(x, seed, offset, p):
    """keep (.) x / (1 - p), p as it is used."""
    t = min(65535, int(np.rint(p * 65536)))
    mask = keep(seed, offset, x.size, p).reshape(x.shape)
    return np.where(mask, x, 0.0) / (1 - t / 65536)
