"""CPU oracle for products in 8-bit integers: rows and weights in codes with scales, products of them, FFNs and layers.

TEST INFRASTRUCTURE ONLY (see moe_oracle.py): plain NumPy, shares no code with the HIP path; only tests may import it.

    codes   M = max(m, 2^-100) of a row's largest magnitude m, r = 127 / M and s = M / 127 rounded to float32, code = v r in float64
            (exact for float32 values) rounded to the nearest whole number, ties to even; a row with an infinity or NaN: codes 0, s NaN
    product (sum of products of codes, int64) * s_row * s_col + bias, float64
    ffn     h = gelu_tanh(product of x's codes) rounded to bf16, then the product of h's codes
    layer   the gate of moe_oracle, then ffn on the dispatched rows, combined in float64

Pins (tests/test_oracle_i8.py): hand-worked rows, ties, extremes; products against Python integers; the packed order against its
formula, byte by byte; the ffn near the one of moe_oracle on values that codes hold exactly.
"""
from __future__ import annotations

from typing import Dict, Optional, Tuple

import numpy as np

from . import moe_oracle as orc

_F64 = np.float64
LEAST = 2.0 ** -100


def quantise(x: np.ndarray, axis: int) -> Tuple[np.ndarray, np.ndarray]:
    """(codes int8, scales float32) along `axis`."""
    x = np.asarray(x, np.float32)
    with np.errstate(invalid="ignore", over="ignore"):
        m = np.max(np.abs(x), axis=axis, keepdims=True)
        fine = np.isfinite(x).all(axis=axis, keepdims=True)
        M = np.maximum(np.where(fine, m, 1.0).astype(_F64), LEAST)
        r, s = (127.0 / M).astype(np.float32), (M / 127.0).astype(np.float32)
        codes = np.where(fine, np.rint(np.where(fine, x, 0).astype(_F64) * r.astype(_F64)), 0)
    return codes.astype(np.int8), np.squeeze(np.where(fine, s, np.float32(np.nan)), axis)


def product(a: np.ndarray, s_row: np.ndarray, w: np.ndarray, s_col: np.ndarray, bias: Optional[np.ndarray] = None) -> np.ndarray:
    """codes a [R, K] by codes w [K, N]; float64 holds every sum exactly."""
    y = (a.astype(_F64) @ w.astype(_F64)) * s_row.astype(_F64)[:, None] * s_col.astype(_F64)[None, :]
    return y if bias is None else y + np.asarray(bias, _F64)


def bf16(x: np.ndarray) -> np.ndarray:
    """The nearest bf16 of float64 values, ties to even, as float64 (normal range)."""
    m, e = np.frexp(np.asarray(x, _F64))
    return np.ldexp(np.rint(m * 256.0), e - 8)


def ffn(x: np.ndarray, W1, b1, W2, b2) -> np.ndarray:
    """W1, W2: (codes, scales)."""
    h = bf16(orc.gelu_tanh(product(*quantise(x, 1), *W1, b1)))
    return product(*quantise(h, 1), *W2, b2)


def layer(x: np.ndarray, logits: np.ndarray, W1, b1, W2, b2, top_k: int, capacity: int, dense=None) -> Dict[str, np.ndarray]:
    """W1[e], W2[e]: (codes, scales); b1, b2: rows or None; dense: (W1, b1, W2, b2) of the dense branch or None."""
    r = orc.gate(logits, top_k, capacity)
    out = np.zeros(x.shape, _F64)
    for e in range(logits.shape[1]):
        tokens = r["slot_token"][e, :r["expert_rows"][e]]
        if len(tokens) == 0:
            continue
        y = ffn(x[tokens], W1[e], None if b1 is None else b1[e], W2[e], None if b2 is None else b2[e])
        for i, t in enumerate(tokens):
            j = list(r["expert_idx"][t]).index(e)
            out[t] += r["gate_w"][t, j] * y[i]
    if dense is not None:
        out += ffn(x, *dense)
    return {**r, "out": out}


def packed_index(k, n, K: int, N: int):
    """Where byte (k, n) of a group [K, N] lies in the group's packed bytes."""
    groups = (N + 127) // 128
    return ((((k // 64) * groups + n // 128) * 8 + n % 8) * 64 + (k % 64 // 16) * 16 + n % 128 // 8) * 16 + k % 16


def pack(codes: np.ndarray) -> np.ndarray:
    """int8 [G, K, N] in the order of the products, zeros behind K and N."""
    G, K, N = codes.shape
    out = np.zeros((G, (K + 63) // 64 * ((N + 127) // 128) * 8192), np.int8)
    k, n = np.meshgrid(np.arange(K), np.arange(N), indexing="ij")
    out[:, packed_index(k, n, K, N)] = codes
    return out.reshape(-1)
