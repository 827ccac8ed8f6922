"""Pins of oracle/i8_oracle.py."""
import numpy as np
import pytest
import torch

from oracle import i8_oracle as o
from oracle import moe_oracle as orc


def test_codes_by_hand():
    # largest magnitude 127 / 8: r = 8 and s = 1 / 8 exactly; ties go to even codes
    x = np.array([[127 / 8, 1.0, 0.0625, 0.1875, -0.0625, -0.1875, 0.3125, -15.875]], np.float32)
    codes, s = o.quantise(x, 1)
    assert codes.tolist() == [[127, 8, 0, 2, 0, -2, 2, -127]] and s.tolist() == [0.125]
    assert o.quantise(x.T, 0)[0].T.tolist() == codes.tolist()


def test_rows_without_numbers():
    x = np.array([[0, 0], [2.0 ** -126, -2.0 ** -101], [np.inf, 1], [np.nan, 1], [3.3e38, -1e38], [2.0 ** -100, 0]], np.float32)
    codes, s = o.quantise(x, 1)
    assert codes[0].tolist() == [0, 0] and s[0] == np.float32(2.0 ** -100 / 127)
    assert codes[1].tolist() == [0, -64] and s[1] == s[0]                 # 127 / 2, a tie
    assert codes[2].tolist() == [0, 0] and np.isnan(s[2]) and codes[3].tolist() == [0, 0] and np.isnan(s[3])
    assert codes[4].tolist() == [127, -38] and np.isfinite(s[4]) and codes[5].tolist() == [127, 0]


@pytest.mark.parametrize("seed", range(4))
def test_codes_are_the_nearest(seed):
    g = np.random.default_rng(seed)
    x = (g.standard_normal((50, 333)) * np.exp(3 * g.standard_normal((50, 1)))).astype(np.float32)
    codes, s = o.quantise(x, 1)
    assert np.abs(codes).max(1).tolist() == [127] * 50
    # r and s are off by 2^-24 of themselves each, so a value is off by half a step and 127 times that much
    assert (np.abs(codes * s[:, None].astype(np.float64) - x) <= s[:, None].astype(np.float64) * (0.5 + 127 * 2.0 ** -22)).all()


def test_product_by_integers():
    g = np.random.default_rng(1)
    a, w = g.integers(-127, 128, (3, 40)).astype(np.int8), g.integers(-128, 128, (40, 5)).astype(np.int8)
    sr, sc = np.array([0.5, 2, 1], np.float32), np.array([1, 0.25, 8, 1, 2], np.float32)
    b = np.arange(5.0)
    want = [[sum(int(a[r, k]) * int(w[k, n]) for k in range(40)) * float(sr[r]) * float(sc[n]) + n for n in range(5)] for r in range(3)]
    assert o.product(a, sr, w, sc, b).tolist() == want


def test_bf16():
    x = np.random.default_rng(2).standard_normal(4000) * np.exp(np.random.default_rng(3).standard_normal(4000) * 8)
    x = np.concatenate((x.astype(np.float32), [0.0, 1 + 2 ** -8, 1 + 3 * 2 ** -8])).astype(np.float32)
    assert (o.bf16(x) == torch.from_numpy(x).to(torch.bfloat16).double().numpy()).all()


@pytest.mark.parametrize("G,K,N", [(1, 8, 8), (2, 72, 136), (1, 200, 264)])
def test_packed_order(G, K, N):
    codes = np.random.default_rng(4).integers(-128, 128, (G, K, N)).astype(np.int8)
    p = o.pack(codes).reshape(G, (K + 63) // 64, (N + 127) // 128, 8, 64, 16)
    seen = 0
    for kb, ng, j, lane, i in np.ndindex(p.shape[1:]):
        k, n = kb * 64 + lane // 16 * 16 + i, ng * 128 + lane % 16 * 8 + j
        want = codes[:, k, n] if k < K and n < N else 0
        assert (p[:, kb, ng, j, lane, i] == want).all()
        seen += k < K and n < N
    assert seen == K * N


def test_ffn_on_values_that_codes_hold():
    """Whole numbers up to 127 with a 127 in each row and column are their own codes (s = 1): the first product is exact, and only h's
    two roundings lie between this and the FFN of moe_oracle."""
    g = np.random.default_rng(5)
    x, W1 = g.integers(-127, 128, (7, 24)).astype(np.float64), g.integers(-127, 128, (24, 16)).astype(np.float64)
    x[:, 0], W1[0, :] = 127, 127
    W2 = g.integers(-127, 128, (16, 8)).astype(np.float64)
    W2[0, :] = 127
    q = lambda W: o.quantise(W, 0)  # noqa: E731
    h = orc.gelu_tanh(x @ W1)
    assert (o.product(*o.quantise(x, 1), *q(W1)) == x @ W1).all()
    got, want = o.ffn(x, q(W1), None, q(W2), None), orc.ffn(x, W1, None, W2, None)
    step = np.abs(h).max(1, keepdims=True) / 127                          # h is off by half a code and half a step of bf16
    assert (np.abs(got - want) <= (0.51 * step + 2.0 ** -8 * np.abs(h)) @ np.abs(W2)).all()


def test_layer_is_gate_and_ffn():
    g = np.random.default_rng(6)
    T, d, f, E, C = 9, 16, 24, 4, 3
    x, logits = g.standard_normal((T, d)), g.standard_normal((T, E)).astype(np.float32)
    W1, W2 = ([o.quantise(g.standard_normal(s), 0) for _ in range(E)] for s in ((d, f), (f, d)))
    for k in (1, 2):
        r = o.layer(x, logits, W1, None, W2, None, k, C, (W1[0], None, W2[0], None))
        ye = np.zeros((E, C, d))
        for e in range(E):
            for c in range(r["expert_rows"][e]):
                ye[e, c] = o.ffn(x[r["slot_token"][e, c]][None], W1[e], None, W2[e], None)[0]
        want = orc.combine(ye, r["expert_idx"], r["slot_idx"], r["gate_w"], o.ffn(x, W1[0], None, W2[0], None))
        assert np.abs(r["out"] - want).max() <= 1e-12 * np.abs(want).max()
