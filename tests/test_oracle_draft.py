"""Pins of oracle/draft_oracle.py (CPU)."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as blk
from oracle import draft_oracle as drf

RNG = np.random.default_rng(5)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_turns(layout):
    f = np.array([np.pi / 2, np.pi / 6])
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 5.0]]])
    got = drf.rope(x, np.array([1]), f, layout)
    c, s = np.sqrt(3) / 2, 0.5
    if layout == "half":           # (1, 3) by 90 degrees, (2, 4) by 30
        want = [-3, 2 * c - 4 * s, 1, 4 * c + 2 * s, 5]
    else:                          # (1, 2) by 90 degrees, (3, 4) by 30
        want = [-2, 1, 3 * c - 4 * s, 4 * c + 3 * s, 5]
    assert np.allclose(got[0, 0], want, atol=1e-15)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_products_depend_on_the_difference(layout):
    f = drf.rope_frequencies(16, 10000.0)
    q, k = RNG.standard_normal((2, 1, 1, 16))
    at = lambda p, r: float(np.sum(drf.rope(q, [p], f, layout) * drf.rope(k, [r], f, layout)))  # noqa: E731
    assert at(7, 3) == pytest.approx(at(1004, 1000), rel=1e-9)
    assert np.linalg.norm(drf.rope(q, [12345], f, layout)) == pytest.approx(np.linalg.norm(q), rel=1e-12)


def test_rope_scalings():
    plain = drf.rope_frequencies(8, 100.0)
    assert np.allclose(plain, [1, 100 ** -0.25, 0.1, 100 ** -0.75])
    assert np.allclose(drf.rope_frequencies(8, 100.0, "linear", 4.0), plain / 4)
    # over 20 pi positions the pairs turn 10, 3.162, 1 and 0.316 times: kept, partly, partly, slowed down
    by = drf.rope_frequencies(8, 100.0, "by_parts", 4.0, 20 * np.pi, 0.5, 5.0)
    part = lambda r: (r - 0.5) / 4.5 + (1 - (r - 0.5) / 4.5) / 4  # noqa: E731
    assert np.allclose(by / plain, [1, part(10 ** 0.5), part(1.0), 0.25])


def test_formats():
    assert np.array_equal(drf.values("fp8"), torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy())
    x = RNG.standard_normal((50, 64)) * np.exp(RNG.standard_normal((50, 1)) * 5)
    for kind, step in (("fp8", 2.0 ** -4), ("fp4", 2.0 ** -2)):
        codes, scale = drf.quantise(x, kind)
        y = drf.dequantise(codes, scale, kind)
        big = np.repeat(np.abs(x).reshape(50, 2, 32).max(-1), 32, -1)
        # half a step of a normal number, or half the smallest step next to the block's largest (at least TOP / 2 after scaling)
        least = {"fp8": 2.0 ** -10 / 224, "fp4": 0.25 / 3}[kind]
        assert np.all(np.abs(y - x) <= np.maximum(step * np.abs(x), least * big) * (1 + 1e-12))
        assert np.all(np.abs(y).reshape(50, 2, 32).max(-1) <= drf.TOP[kind] * 2.0 ** (scale - 127.0))
    assert np.array_equal(drf.quantise(np.zeros(32), "fp8")[1], [27])
    assert drf.quantise(np.full(32, 448.0), "fp8")[1][0] == 127 and drf.quantise(np.full(32, 449.0), "fp8")[1][0] == 128
    assert drf.quantise(np.full(32, 6.0), "fp4")[1][0] == 127 and drf.quantise(np.full(32, 6.5), "fp4")[1][0] == 128
    assert np.all(np.isnan(drf.dequantise(*drf.quantise(np.r_[np.inf, np.zeros(31)], "fp4"), "fp4")))
    for kind, top in (("fp8", 1.75 * 2.0 ** 127), ("fp4", 1.5 * 2.0 ** 127)):        # nothing leaves bf16
        assert np.array_equal(drf.dequantise(*drf.quantise(np.full(32, -3.3e38), kind), kind), np.full(32, -top))
    ties = np.r_[6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, np.zeros(24)]
    assert np.array_equal(drf.dequantise(*drf.quantise(ties, "fp4"), "fp4")[:8], [6, 0, 1, 1, 2, 2, 4, 4])


def test_chain_equals_token_by_token():
    B, N, H, dh, L = 2, 4, 3, 8, 9
    q, k, v = RNG.standard_normal((3, B, N, H, dh))
    kc, vc = RNG.standard_normal((2, B, H, L, dh))
    lens = np.array([0, 5])
    got, _ = drf.tree_attention(q, k, v, kc, vc, lens, None, None, np.zeros((B, N, H, dh)))
    kc, vc = kc.copy(), vc.copy()
    for i in range(N):
        want = blk.decode_attention(q[:, i], k[:, i], v[:, i], kc, vc, lens + i)
        assert np.allclose(got[:, i], want, atol=1e-13)
        for b in range(B):
            kc[b, :, lens[b] + i], vc[b, :, lens[b] + i] = k[b, i], v[b, i]


def test_tree_equals_its_paths():
    N, H, G, dh, L = 5, 2, 1, 8, 6
    q = RNG.standard_normal((1, N, H, dh))
    k, v = RNG.standard_normal((2, 1, N, G, dh))
    kc, vc = RNG.standard_normal((2, 1, G, L, dh))
    parent = [-1, 0, 0, 1, 2]
    masks = []
    for i in range(N):
        masks.append((0 if parent[i] < 0 else masks[parent[i]]) | 1 << i)
    tree = np.array(masks, np.int32).reshape(1, N, 1)
    got, _ = drf.tree_attention(q, k, v, kc, vc, [4], None, tree, np.zeros((1, N, H, dh)))
    for path in ([0, 1, 3], [0, 2, 4]):
        want, _ = drf.tree_attention(q[:, path], k[:, path], v[:, path], kc, vc, [4], None, None, np.zeros((1, 3, H, dh)))
        assert np.allclose(got[:, path], want, atol=1e-13)
    # nothing to see: 0; rows behind the count: as they were
    got, _ = drf.tree_attention(q, k, v, kc, vc, [0], [2], np.zeros_like(tree), np.full((1, N, H, dh), 7.0))
    assert np.all(got[:, :2] == 0) and np.all(got[:, 2:] == 7)
