"""The paged cache and the read over it, in float64 numpy.

``stored``/``codes_of`` give what a row holds once stored in a quantised cache,
from a table of every code's value; ``fem_paged`` is the softmax-prior read of
the packed new tokens of a ragged batch over per-sequence keys and values.
"""

from __future__ import annotations

import math

import numpy as np

from .fem_oracle import free_energy_read

BLOCK = 32          # channels of a scale
LEAST_EXP = -100
LARGEST = {"e4m3": 448.0, "int8": 127.0}


def code_values(kind: str):
    """(code, value) of every non-negative finite code of the element type, in
    ascending order: OCP e4m3 (bias 7, three fraction bits, subnormals of 2^-9,
    0x7f is NaN) or the integers 0..127."""
    if kind == "int8":
        return [(c, float(c)) for c in range(128)]
    out = []
    for c in range(0x7f):
        e, f = c >> 3, c & 7
        out.append((c, f * 2.0 ** -9 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7)))
    return out


def codes_of(x: np.ndarray, kind: str):
    """Codes (uint8 bits) and scale bytes of rows x [.., w], w a multiple of 32:
    the smallest exponent >= -100 whose largest code reaches the block's largest
    magnitude, and the nearest code, ties to the even one."""
    x = np.asarray(x, dtype=np.float64)
    b = x.reshape(*x.shape[:-1], -1, BLOCK)
    table = code_values(kind)
    values = np.array([v for _, v in table])
    codes = np.zeros(b.shape, dtype=np.uint8)
    byte = np.zeros(b.shape[:-1], dtype=np.uint8)
    for at in np.ndindex(*b.shape[:-1]):
        row = b[at]
        if not np.isfinite(row).all():
            byte[at] = 255
            continue
        top, e = np.abs(row).max(), LEAST_EXP
        while top > LARGEST[kind] * 2.0 ** e:
            e += 1
        byte[at] = e + 127
        y = np.abs(row) * 2.0 ** -e
        hi = np.clip(np.searchsorted(values, y), 1, len(values) - 1)
        up, down = values[hi] - y, y - values[hi - 1]
        pick = np.where(up < down, hi, hi - 1)
        tie = up == down
        pick = np.where(tie, np.where(hi % 2 == 0, hi, hi - 1), pick)
        c = np.array([table[i][0] for i in pick])
        neg = np.signbit(row)
        codes[at] = np.where(neg, c | 0x80, c) if kind == "e4m3" else np.where(neg, -c, c) & 0xff
    return codes.reshape(x.shape), byte


def values_of(codes: np.ndarray, byte: np.ndarray, kind: str) -> np.ndarray:
    """float64 values of codes [.., w] with scale bytes [.., w / 32]."""
    if kind == "int8":
        x = codes.astype(np.uint8).view(np.int8).astype(np.float64)
    else:
        t = np.full(256, np.nan)
        for c, v in code_values("e4m3"):
            t[c], t[c | 0x80] = v, -v
        x = t[codes]
    s = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127))
    return x * np.repeat(s, BLOCK, axis=-1)


def stored(x: np.ndarray, kind: str) -> np.ndarray:
    """What rows x [.., w] (bf16 numbers) read as once stored."""
    if kind == "bf16":
        return np.asarray(x, dtype=np.float64)
    return values_of(*codes_of(x, kind), kind)


def fem_paged(q, ks, vs, beta, starts, causal: bool = True) -> np.ndarray:
    """Packed queries q [N, H, d] of a ragged batch; ks[b] [Hkv, n_b, d] and vs[b]
    [Hkv, n_b, dv] the sequences' keys and values; beta [Hkv, dv]; starts [B + 1].
    Token i of sequence b sees the keys up to n_b - (its new tokens) + i, or all
    n_b of them.  A token that sees none, or that belongs to no sequence, is NaN."""
    q = np.asarray(q, dtype=np.float64)
    beta = np.asarray(beta, dtype=np.float64)
    N, H, d = q.shape
    Hkv, dv = beta.shape
    G = H // Hkv
    out = np.full((N, H, dv), np.nan)
    for b in range(len(starts) - 1):
        t0, t1 = int(starts[b]), int(starts[b + 1])
        n = ks[b].shape[1]
        if t1 == t0 or n == 0:
            continue
        last = n - (t1 - t0) + np.arange(t1 - t0) if causal else np.full(t1 - t0, n - 1)
        hidden = np.arange(n)[None, :] > last[:, None]
        for h in range(H):
            s = q[t0:t1, h] @ ks[b][h // G].T / math.sqrt(d)
            s = np.where(hidden, -np.inf, s)
            m = s.max(axis=1, keepdims=True)
            logp = s - (m + np.log(np.exp(s - m).sum(axis=1, keepdims=True)))
            out[t0:t1, h] = free_energy_read(np.exp(logp), vs[b][h // G], beta[h // G], logp)
    return out
