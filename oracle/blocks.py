"""Operators for language models in 64 bits, CPU reference (numpy).

TEST INFRASTRUCTURE ONLY.  Written from the definitions: blocks of 128 with one scale each, e4m3 codes, products of
blocked matrices, and the adjustment of logits by the tokens that a sequence holds.
"""
from __future__ import annotations

import numpy as np

BLOCK = 128
TOP = 448.0


def _e4m3():
    code = np.arange(256)
    e, m = (code >> 3) & 15, code & 7
    v = np.where(e > 0, np.ldexp(1 + m / 8, e - 7), np.ldexp(m / 8, -6))
    v[(code & 127) == 127] = np.nan
    return np.where(code & 128, -v, v)


E4M3 = _e4m3()


def _amax(x: np.ndarray, kind: str) -> np.ndarray:
    """Largest finite magnitude of every block, [row or tile][block]."""
    rows, dim = x.shape
    whole = np.zeros((-(-rows // BLOCK) * BLOCK, -(-dim // BLOCK) * BLOCK))
    whole[:rows, :dim] = np.where(np.isfinite(x), np.abs(x), 0.0)
    m = whole.reshape(whole.shape[0], -1, BLOCK).max(axis=2)
    return m[:rows] if kind == "row" else m.reshape(-1, BLOCK, m.shape[1]).max(axis=1)


def scales(amax: np.ndarray, scale: str) -> np.ndarray:
    """The scale of blocks with these largest magnitudes, in 64 bits."""
    if scale == "f32":
        return np.where(amax > 0, np.maximum((amax / TOP).astype(np.float32).astype(np.float64), 2.0 ** -126), 1.0)
    e = np.full(amax.shape, -126)
    for k in range(-126, 130):
        e = np.where(amax > TOP * 2.0 ** k, k + 1, e)
    return np.where(amax > 0, 2.0 ** e, 1.0)


def encode(q: np.ndarray) -> np.ndarray:
    """e4m3 code nearest to each value, ties to the even mantissa; NaN for infinities and NaN."""
    middle = (E4M3[1:127] + E4M3[:126]) / 2
    mag = np.abs(np.where(np.isfinite(q), q, 0.0))
    below, above = np.searchsorted(middle, mag, side="left"), np.searchsorted(middle, mag, side="right")
    code = np.where(below % 2 == 0, below, above)
    return np.where(np.isfinite(q), code + 128 * np.signbit(q), 127).astype(np.uint8)


def quantize(x: np.ndarray, kind: str, scale: str):
    """(codes [rows][whole blocks], scales [block][row or tile] in 64 bits) of x, taken in 64 bits."""
    x = x.astype(np.float64)
    rows, dim = x.shape
    s = scales(_amax(x, kind), scale)
    each = (s if kind == "row" else s.repeat(BLOCK, axis=0)[:rows]).repeat(BLOCK, axis=1)[:, :dim]
    codes = np.zeros((rows, -(-dim // BLOCK) * BLOCK), dtype=np.uint8)
    with np.errstate(invalid="ignore"):
        codes[:, :dim] = encode(x / each)
    return codes, s.T.copy()


def values(codes: np.ndarray, s: np.ndarray, kind: str) -> np.ndarray:
    """What codes and scales [block][row or tile] stand for."""
    each = s if kind == "row" else s.repeat(BLOCK, axis=1)
    return E4M3[codes] * each[:, : codes.shape[0]].T.repeat(BLOCK, axis=1)


def count(seen: np.ndarray, counts, vocab: int, tokens, offsets, slots, prompt: bool = False, restart: bool = False):
    """seen bool [slots][vocab], counts [slots][vocab] or None, in place."""
    n = len(offsets) - 1
    if restart:
        for i in range(n):
            if 0 <= slots[i] < seen.shape[0]:
                seen[slots[i]] = False
                if counts is not None:
                    counts[slots[i]] = 0
    for i in range(n):
        for t in tokens[offsets[i]:offsets[i + 1]]:
            if 0 <= slots[i] < seen.shape[0] and 0 <= t < vocab:
                seen[slots[i], t] = True
                if counts is not None and not prompt:
                    counts[slots[i], t] += 1


def adjust(logits: np.ndarray, seen=None, counts=None, repetition=None, frequency=None, presence=None, biases=None, allowed=None) -> np.ndarray:
    """All by row of logits: seen, counts and allowed [n][vocab], penalties [n], biases a list of (token, value) lists; None: not
    applied."""
    v = logits.astype(np.float64).copy()
    with np.errstate(all="ignore"):
        if seen is not None:
            rep = np.ones(len(v)) if repetition is None else repetition.astype(np.float64)
            again = np.where(v > 0, v / rep[:, None], v * rep[:, None])
            v = np.where(seen, again, v)
            if counts is not None:
                c = np.where(seen, counts, 0)
                f = np.zeros(len(v)) if frequency is None else frequency.astype(np.float64)
                p = np.zeros(len(v)) if presence is None else presence.astype(np.float64)
                v = np.where(c > 0, v - f[:, None] * c - p[:, None], v)
        for i, row in enumerate(biases or []):
            for t, b in row:
                if 0 <= t < v.shape[1]:
                    v[i, t] += b
    if allowed is not None:
        v = np.where(allowed, v, -np.inf)
    return v


def pack_bits(bits: np.ndarray) -> np.ndarray:
    """bool [n][vocab] as bitmaps, int32 [n][ceil(vocab / 32)]."""
    whole = np.zeros((bits.shape[0], -(-bits.shape[1] // 32) * 32), dtype=np.uint8)
    whole[:, : bits.shape[1]] = bits
    return np.packbits(whole, axis=1, bitorder="little").view(np.int32)
