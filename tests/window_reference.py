"""Plain 64-bit implementations for the tests of the masked attention and of the 4-bit rows, and the bounds that their
results are held to."""

from __future__ import annotations

import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float64)


# ---- rows in 4 bits
def pack(x: np.ndarray):
    """codes [rows, D / 2], scales [rows, D / 32] of fp32 rows, from the definition."""
    rows, D = x.shape
    blocks = x.reshape(rows, D // 32, 32).astype(np.float64)
    top = np.abs(blocks).max(-1)
    odd = ~np.isfinite(top)
    # the smallest exponent with which the largest value rounds to at most 6, i.e. is below 7
    e = np.full(top.shape, -125)
    for k in range(-125, 125):
        e = np.where(top >= 7 * 2.0 ** k, k + 1, e)
    a = np.abs(np.where(odd[..., None], 0, blocks)) / 2.0 ** e[..., None]
    # nearest of the grid; halfway to the even position (its mantissa bit is 0)
    low = np.clip(np.searchsorted(GRID, a, side="right") - 1, 0, 6)
    middle = (GRID[low] + GRID[low + 1]) / 2
    code = low + ((a > middle) | ((a == middle) & (low % 2 == 1)))
    code = (code + 8 * np.signbit(blocks)).astype(np.uint8)
    code[odd] = 0
    code = code.reshape(rows, D // 2, 2)
    scales = np.where(odd, 255, e + 127).astype(np.uint8)
    return (code[..., 0] | code[..., 1] << 4).astype(np.uint8), scales


def unpack(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    rows, half = codes.shape
    nibbles = np.stack([codes & 15, codes >> 4], -1).reshape(rows, 2 * half)
    x = np.where(nibbles >= 8, -1.0, 1.0) * GRID[nibbles & 7]
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return x * np.repeat(s, 32, axis=1)


# ---- attention
def visible(n: int, W: int, causal: bool, span: int, sinks: int) -> np.ndarray:
    """[W, n]: which rows the query at each window position sees."""
    t = np.arange(n)
    pos = (n - W + np.arange(W) if causal else np.full(W, n - 1))[:, None]
    return (t <= pos) & ((t > pos - span) | (t < sinks) | (span == 0))


def attention(Q, K, V, *, causal, span, sinks, counts=None, scale=0.0, weight_bits=16, out_bits=24):
    """Q [G, W, D], K and V [n, D]: the outputs [G, W, D] in 64 bits, and how far an implementation may be off in each.

    The bound: a logit is a sum of D products (fp32 partial sums: D roundings of 2^-24 of the sum of magnitudes, and two
    more for the scale), the exponential and its argument round four times, the weight is taken with `weight_bits` bits, and
    both sums add up at most n terms in any order.  Every weight's relative error counts once in the numerator and once in
    the denominator.  The output is rounded to `out_bits` bits.  Below 2^-126 the types have no numbers of full precision: a
    term of which the largest is more than 2^126 times (or 2^118, where the reference is up to 2^8 above it) may be lost
    whole, and so may a result of that size."""
    Q, K, V = (np.asarray(x, dtype=np.float64) for x in (Q, K, V))
    G, W, D = Q.shape
    n = K.shape[0]
    scale = scale or D ** -0.5
    c = np.ones(n) if counts is None else np.asarray(counts, dtype=np.float64)
    out, off = np.zeros((G, W, D)), np.zeros((G, W, D))
    seen = visible(n, W, causal, span, sinks)
    for w in range(W):
        at = np.flatnonzero(seen[w])
        if len(at) == 0:
            continue
        e = scale * (Q[:, w] @ K[at].T)
        size = scale * (np.abs(Q[:, w]) @ np.abs(K[at]).T)
        p = np.exp(e - e.max(1, keepdims=True))
        den = (p * c[at]).sum(1, keepdims=True)
        with np.errstate(invalid="ignore"):
            out[:, w] = p @ V[at] / den
            u = 2.0 ** -24
            rel = (D + 2) * u * size + 4 * u * (1 + np.abs(e - e.max(1, keepdims=True))) + 2.0 ** -weight_bits + len(at) * u
            off[:, w] = (p * rel) @ np.abs(V[at]) / den + (p * rel * c[at]).sum(1, keepdims=True) / den * np.abs(out[:, w])
            off[:, w] += 2.0 ** -out_bits * np.abs(out[:, w])
            off[:, w] += 2.0 ** -126 + len(at) * 2.0 ** -118 * np.abs(V[at]).max(0)
    return out, off


def bf16(x: np.ndarray) -> np.ndarray:
    """fp32 numbers rounded to bf16 (nearest even), as fp32."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)
