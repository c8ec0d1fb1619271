"""fp64 definitions of the multi-token step (test infrastructure only, like pad_oracle.py): 8-bit and 4-bit groups,
attention of chunk tokens, verification of drafted tokens.

An 8-bit group is the head_dim values of one token and kv-head: codes are e4m3 (four exponent bits,
bias 7, three mantissa bits, largest value 448) of x / 2^k to nearest even, k the smallest integer with
max|x| <= 448 * 2^k, kept in [-120, 7]; the scale byte is k + 127, 0 for zeros, 255 where a value is not
finite.  A 4-bit group is 16 consecutive values: the scale is max|x| / 6 to nearest even as an unsigned number of five
exponent bits (bias 15) and three mantissa bits, 10240 at most, codes are e2m1 of x / scale to nearest even, saturated;
byte 255 and codes of 0 where a value is not finite.  Chunk token t of an event sees its video's prefix and its branch's tokens up to itself
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


def _nearest(y: np.ndarray, grid: np.ndarray) -> np.ndarray:
    """Index of the entry of the ascending grid nearest to each y, ties to the even index."""
    y = np.minimum(y, grid[-1])
    hi = np.clip(np.searchsorted(grid, y), 0, len(grid) - 1)
    lo = np.maximum(hi - 1, 0)
    dh, dl = grid[hi] - y, y - grid[lo]
    return np.where(dh < dl, hi, np.where(dl < dh, lo, np.where(lo % 2 == 0, lo, hi)))


def kv4_scales() -> np.ndarray:
    """The value of each scale byte up to 226."""
    b = np.arange(227)
    return np.where(b < 8, b * 2.0 ** -17, (8 + b % 8) * 2.0 ** (b // 8 - 18.0))


_E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def kv4_encode(x: np.ndarray):
    """x [..., d] float64 -> (codes uint8 [..., d / 2], the even value's in the lower half, scale bytes uint8 [..., d / 16])."""
    g = np.asarray(x, dtype=np.float64).reshape(x.shape[:-1] + (x.shape[-1] // 16, 16))
    fine = np.all(np.isfinite(g), axis=-1)
    g = np.where(fine[..., None], g, 0.0)
    byte = _nearest(np.abs(g).max(-1) / 6.0, kv4_scales())
    scale = kv4_scales()[byte][..., None]
    y = np.divide(g, scale, out=np.zeros_like(g), where=scale > 0)
    code = (_nearest(np.abs(y), _E2M1) + 8 * np.signbit(g)).astype(np.uint8) * fine[..., None]
    code = code.reshape(x.shape)
    return (code[..., 0::2] + 16 * code[..., 1::2]).astype(np.uint8), np.where(fine, byte, 255).astype(np.uint8)


def kv4_decode(codes: np.ndarray, byte: np.ndarray) -> np.ndarray:
    c = np.stack([codes & 15, codes >> 4], -1).reshape(byte.shape + (16,))
    v = np.where(c > 7, -1.0, 1.0) * _E2M1[c & 7]
    scale = np.where(byte == 255, np.nan, kv4_scales()[np.minimum(byte, 226)])
    return (v * scale[..., None]).reshape(codes.shape[:-1] + (2 * codes.shape[-1],))


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


def rope_frequencies(rotary, theta, scaling="none", factor=1.0, original_len=0.0, low=1.0, high=4.0):
    """f_i of each rotary pair, scaled for long contexts."""
    if scaling == "base":
        theta = theta * factor ** (rotary / (rotary - 2))
    f = np.array([theta ** (-2.0 * i / rotary) for i in range(rotary // 2)])
    if scaling == "linear":
        return f / factor
    if scaling == "turns":
        g = np.clip((original_len * f / (2 * math.pi) - low) / (high - low), 0, 1)
        return f * (g + (1 - g) / factor)
    if scaling == "index":
        def index(n):
            return rotary * math.log(original_len / (2 * math.pi * n)) / (2 * math.log(theta))
        a, b = (min(max(x, 0), rotary - 1) for x in (math.floor(index(high)), math.ceil(index(low))))
        g = 1 - np.clip((np.arange(rotary // 2) - a) / max(b - a, 0.001), 0, 1)
        return f * (g + (1 - g) / factor)
    return f


def rope_turn(x, position, frequencies, layout="half", magnitude=1.0):
    """x [n, heads, d] float64 turned at position [n]; also |a| + |b| of each value's pair, 0 for those that stay."""
    r = 2 * len(frequencies)
    angle = np.asarray(position, dtype=np.float64)[:, None] * frequencies
    cos, sin = (magnitude * f(angle)[:, None] for f in (np.cos, np.sin))
    one, two = (slice(0, r // 2), slice(r // 2, r)) if layout == "half" else (slice(0, r, 2), slice(1, r, 2))
    a, b = x[..., one], x[..., two]
    out, size = x.copy(), np.zeros_like(x)
    out[..., one], out[..., two] = a * cos - b * sin, b * cos + a * sin
    size[..., one] = size[..., two] = np.abs(a) + np.abs(b)
    return out, size


def logits_to_probs(logits, temperature=1.0, repetition=1.0, frequency=0.0, presence=0.0, context=(), biases=(), allowed=None):
    """One row [vocab] in 64 bits: penalties for the tokens of ``context``, (token, value) ``biases``, a boolean mask, softmax.
    Returns p and the largest magnitude that a logit passes through."""
    x = np.asarray(logits, dtype=np.float64).copy()
    vocab = len(x)
    count = np.bincount([t for t in context if 0 <= t < vocab], minlength=vocab).astype(np.float64)
    size = np.abs(x) * max(repetition, 1 / repetition)
    x = np.where(count > 0, np.where(x > 0, x / repetition, x * repetition) - (frequency * count + presence), x)
    size += count * abs(frequency) + abs(presence)
    for t, v in biases:
        if 0 <= t < vocab:
            x[t] += v
            size[t] += abs(v)
    if allowed is not None:
        x[~np.asarray(allowed, bool)] = -np.inf
    size = float(np.max(np.where(np.isfinite(x) & np.isfinite(size), size, 0)))
    if not np.isnan(x).any() and x.max() == -np.inf:
        return np.zeros(vocab), size
    if not temperature > 0:
        p = np.zeros(vocab)
        if not np.isnan(x).any():
            p[int(np.argmax(x))] = 1.0
        return p, size
    with np.errstate(invalid="ignore"):
        e = np.exp((x - np.max(x)) / temperature)
    return e / e.sum(), size


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
