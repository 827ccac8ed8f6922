"""CPU oracle for steps with several new tokens per sequence: rotary positions, the quantised key/value cache, attention of
drafted tokens over the cache and over each other.

TEST INFRASTRUCTURE ONLY (see moe_oracle.py): plain fp64 NumPy, shares no code with the HIP path; only tests may import it.

    rope    f_i = base^(-2 i / rot), scaled; pair i of position p turned by p f_i, times amplitude (as a complex product)
    cache   blocks of 32 elements, e = smallest integer >= -100 with max|x| <= top 2^e, the nearest value of the format's
            table to x / 2^e (ties to the even code); e is at most 119 (fp8) or 125 (fp4), with which no value leaves bf16,
            and larger magnitudes take the format's largest value; a block with an infinity or NaN reads as NaN
    tree    softmax(q K^T / sqrt(dh)) V over the cached positions and the drafted tokens whose mask bit is set

Pins (tests/test_oracle_draft.py): rotation keeps lengths and makes products depend on the difference of positions only,
hand-worked angles; the tables against torch's float8_e4m3fn and the values of e2m1; a chain of drafted tokens equals
block_oracle.decode_attention token by token, a tree equals each path run as a chain of its own.
"""
from __future__ import annotations

from typing import Optional, Tuple

import numpy as np

_F64 = np.float64
TOP = {"fp8": 448.0, "fp4": 6.0}
LAST = {"fp8": 119, "fp4": 125}


def rope_frequencies(rot_dim: int, base: float, scaling: str = "plain", factor: float = 1.0, original_len: float = 1.0, low: float = 1.0,
                     high: float = 4.0) -> np.ndarray:
    """Radians per position."""
    f = np.array([base ** (-2.0 * i / rot_dim) for i in range(rot_dim // 2)], _F64)
    if scaling == "linear":
        return f / factor
    if scaling == "by_parts":
        r = original_len * f / (2 * np.pi)
        kept = np.where(r < low, 0.0, np.where(r > high, 1.0, (r - low) / (high - low)))
        return kept * f + (1 - kept) * f / factor
    return f


def rope(x: np.ndarray, pos: np.ndarray, f: np.ndarray, layout: str, amplitude: float = 1.0) -> np.ndarray:
    """x [R, heads, dh]; every head of row r turned to position pos[r]."""
    x = np.asarray(x, _F64)
    half = len(f)
    turn = amplitude * np.exp(1j * np.asarray(pos, _F64)[:, None] * f)[:, None, :]
    out = x.copy()
    a, b = (slice(0, half), slice(half, 2 * half)) if layout == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    z = (x[..., a] + 1j * x[..., b]) * turn
    out[..., a], out[..., b] = z.real, z.imag
    return out


def values(kind: str) -> np.ndarray:
    """The format's non-negative finite values in the order of their codes."""
    if kind == "fp4":
        return np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], _F64)
    return np.array([m / 512 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127], _F64)


def quantise(x: np.ndarray, kind: str) -> Tuple[np.ndarray, np.ndarray]:
    """(codes with the sign in front, scale bytes) of x [..., dh]: one code per element."""
    x = np.asarray(x, _F64)
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    table, sign_bit = values(kind), 128 if kind == "fp8" else 8
    codes = np.zeros(blocks.shape, np.uint8)
    scale = np.zeros(blocks.shape[:-1], np.uint8)
    for at in np.ndindex(*scale.shape):
        block = blocks[at]
        if not np.all(np.isfinite(block)):
            scale[at] = 255
            continue
        e = -100
        while np.max(np.abs(block)) > TOP[kind] * 2.0 ** e and e < LAST[kind]:
            e += 1
        scale[at] = e + 127
        far = np.abs(np.abs(block)[:, None] / 2.0 ** e - table[None, :])
        best = far.min(axis=1, keepdims=True)
        tied = far == best                                     # two neighbours at most: the one with the even code
        code = np.array([next((c for c in np.flatnonzero(t) if c % 2 == 0), np.flatnonzero(t)[0]) for t in tied])
        codes[at] = code + sign_bit * np.signbit(block)
    return codes.reshape(x.shape), scale


def dequantise(codes: np.ndarray, scale: np.ndarray, kind: str) -> np.ndarray:
    sign_bit, table = (128, values(kind)) if kind == "fp8" else (8, values(kind))
    v = np.append(table, np.nan)[codes % sign_bit] * np.where(codes >= sign_bit, -1.0, 1.0)
    unit = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(_F64) - 127))
    return v * np.repeat(unit, 32, axis=-1)


def sees(tree: Optional[np.ndarray], n: int, count: int) -> np.ndarray:
    """[n, n] truth values of one sequence's masks [n, words] (int32 bit patterns)."""
    if tree is None:
        m = np.tril(np.ones((n, n), bool))
    else:
        m = np.array([[(int(tree[i, j // 32]) >> (j % 32)) & 1 for j in range(n)] for i in range(n)], bool).reshape(n, n)
    m[:, count:] = False
    return m


def tree_attention(q, k, v, k_cache, v_cache, lens, counts, tree, keep: np.ndarray):
    """q [B, N, H, dh], k, v [B, N, G, dh], caches [B, G, L, dh] as the values that they hold; keep [B, N, H, dh]: what rows
    behind counts[b] hold.  Returns (out, weight): weight is the same sum with |v|, for error bounds."""
    B, N, H, dh = q.shape
    G = k.shape[2]
    out, weight = np.array(keep, _F64), np.zeros(keep.shape, _F64)
    for b in range(B):
        count = N if counts is None else int(np.clip(counts[b], 0, N))
        n = int(np.clip(lens[b], 0, k_cache.shape[2]))
        mask = sees(None if tree is None else tree[b], N, count)
        for h in range(H):
            g = h // (H // G)
            for i in range(count):
                new = np.flatnonzero(mask[i])
                K = np.concatenate([np.asarray(k_cache[b, g, :n], _F64), np.asarray(k[b, new, g], _F64)])
                V = np.concatenate([np.asarray(v_cache[b, g, :n], _F64), np.asarray(v[b, new, g], _F64)])
                out[b, i, h] = 0.0
                if len(K):
                    s = K @ np.asarray(q[b, i, h], _F64) / np.sqrt(dh)
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    out[b, i, h], weight[b, i, h] = p @ V, p @ np.abs(V)
    return out, weight
