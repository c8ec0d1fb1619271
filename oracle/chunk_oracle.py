"""fp64 definitions of the multi-token step (test infrastructure only, like pad_oracle.py): 8-bit groups,
attention of chunk tokens, verification of drafted tokens.

An 8-bit group is the head_dim values of one token and kv-head: codes are e4m3 (four exponent bits,
bias 7, three mantissa bits, largest value 448) of x / 2^k to nearest even, k the smallest integer with
max|x| <= 448 * 2^k, kept in [-120, 7]; the scale byte is k + 127, 0 for zeros, 255 where a value is not
finite.  Chunk token t of an event sees its video's prefix and its branch's tokens up to itself
(Sec. 3.4).  Verification keeps drafted token i while u_i q_i(x_i) < p_i(x_i) and draws the next token
from integer weights floor(2^38 min(r, 1)).
"""
from __future__ import annotations

import math

import numpy as np


def e4m3_values() -> np.ndarray:
    """The value of each of the 256 codes (NaN for 0x7f and 0xff)."""
    out = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[c] = math.nan if (c & 127) == 127 else (-v if c > 127 else v)
    return out


def kv8_encode(x: np.ndarray):
    """x [..., d] float64 -> (codes uint8 [..., d], scale bytes uint8 [...]); NaN groups get byte 255 and code 0."""
    x = np.asarray(x, dtype=np.float64)
    grid = e4m3_values()[:127]                     # ascending, non-negative
    flat = x.reshape(-1, x.shape[-1])
    codes = np.zeros(flat.shape, dtype=np.uint8)
    byte = np.zeros(flat.shape[0], dtype=np.uint8)
    for i, row in enumerate(flat):
        if not np.all(np.isfinite(row)):
            byte[i] = 255
            continue
        big = float(np.max(np.abs(row)))
        if big == 0.0:
            continue
        k = -120
        while k < 7 and big > 448.0 * 2.0 ** k:
            k += 1
        byte[i] = k + 127
        y = np.minimum(np.abs(row) / 2.0 ** k, 448.0)
        hi = np.clip(np.searchsorted(grid, y), 0, 126)
        lo = np.maximum(hi - 1, 0)
        dh, dl = grid[hi] - y, y - grid[lo]
        near = np.where(dh < dl, hi, np.where(dl < dh, lo, np.where(lo % 2 == 0, lo, hi)))
        codes[i] = near + np.where(np.signbit(row), 128, 0)
    return codes.reshape(x.shape), byte.reshape(x.shape[:-1])


def kv8_decode(codes: np.ndarray, byte: np.ndarray) -> np.ndarray:
    scale = np.where(byte == 255, np.nan, np.where(byte == 0, 0.0, 2.0 ** (np.clip(byte.astype(np.float64), 7, 134) - 127)))
    return e4m3_values()[codes] * scale[..., None]


def chunk_attention(q, k, v, first_limit: int, scale: float):
    """One event: q [n, h_q, d], keys and values [L, h_kv, d] (prefix first), token t seeing the first
    first_limit + t keys.  Returns out [n, h_q, d], lse [n, h_q] and the weighted magnitudes sum p |v|, which the
    bounds of the tests are made of."""
    n, hq, d = q.shape
    g = hq // k.shape[1]
    out, lse, mag = np.zeros((n, hq, d)), np.full((n, hq), -np.inf), np.zeros((n, hq, d))
    for t in range(n):
        see = first_limit + t
        for h in range(hq):
            s = scale * (k[:see, h // g] @ q[t, h])
            if s.size == 0:
                continue
            m = s.max()
            p = np.exp(s - m)
            lse[t, h] = m + math.log(p.sum())
            p /= p.sum()
            out[t, h] = p @ v[:see, h // g]
            mag[t, h] = p @ np.abs(v[:see, h // g])
    return out, lse, mag


def draft_verify(p, q, draft, u_accept, u_pick):
    """One event: p [n + 1, V], q [n, V] float32 arrays (bf16 widened), drafted tokens [n], uniforms.
    Returns (accepted, token); Python integers throughout the draw."""
    n, vocab = len(draft), p.shape[1]
    a = 0
    while a < n and 0 <= draft[a] < vocab and np.float32(u_accept[a]) * np.float32(q[a, draft[a]]) < p[a, draft[a]]:
        a += 1

    def weights(r):
        r = np.where(r > 0, np.minimum(r, np.float32(1)), np.float32(0)).astype(np.float64)
        return [int(x) for x in np.floor(r * 2.0 ** 38)]

    with np.errstate(invalid="ignore"):
        w = weights(p[a] - q[a]) if a < n else weights(p[a])
    if sum(w) == 0:
        w = weights(p[a])
    total = sum(w)
    if total == 0:
        return a, -1
    goal = (int(math.floor(float(u_pick) * 2 ** 24)) * total) >> 24
    run = 0
    for i, x in enumerate(w):
        run += x
        if run > goal:
            return a, i
    raise AssertionError("unreachable")
