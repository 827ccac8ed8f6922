"""How exact moe_tree_attention is before its result is rounded: probabilities of 16 bits up to 32 rows per key/value head, of 8 beyond.

Error bound, from the formats, with w = sum_j p_j |v_j| over the softmax: a probability of 16 bits is the sum of two bf16 numbers, the
second of which is at most half a step of the first (2^-8) and off by half a step of its own: 2^-16 w in all, with one number 2^-8 w; a
score is a sum of dh products in 32 bits, off by at most dh 2^-24 sum |q k| / sqrt(dh) =: d, which moves every probability and their sum
by d (2 d w); exponentials and the sums over n positions are within (n + 64) 2^-23 w.  The result is then rounded by half a step, counted
here at the value itself.

Over many elements, roundings are as good as independent and spread evenly over a step: the mean square of one is at most a third of
2^-16 of its value's (at the lower end of a power of two).  So with one number per probability the mean square of the error is at most
(2^-16 / 3) (ref^2 + sum_j p_j^2 v_j^2), and 5 % more for what the number of elements (10^4 and more) leaves to chance."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as drf
from tests.test_gpu_tree_attention import KINDS, Step
from workloads.generate import to_f32_numpy


def bound(q, k, kc, ref, got, w, lens, one=False):
    """What |got - ref| may be."""
    B, N, H, dh = q.shape
    G = k.shape[2]
    near = np.zeros((B, N, H, 1))
    for b in range(B):
        for h in range(H):
            keys = np.concatenate([np.abs(kc[b, h // (H // G), :lens[b]]), np.abs(k[b, :, h // (H // G)])])
            near[b, :, h, 0] = (np.abs(q[b, :, h]) @ keys.T).max(-1) * dh ** 0.5 * 2.0 ** -24
    top = np.maximum(np.abs(ref), np.abs(got))
    half_step = 2.0 ** (np.floor(np.log2(np.maximum(top, 2.0 ** -100))) - 8)
    return half_step + ((2.0 ** -8 if one else 2.0 ** -16) + 2 * near + (kc.shape[2] + N + 64) * 2.0 ** -23) * w


def parts(s):
    B, N, H, G, dh, L = s.dims
    x = to_f32_numpy(s.qkv)[:, :(H + 2 * G) * dh].reshape(B, N, H + 2 * G, dh).astype(np.float64)
    return x[:, :, :H], x[:, :, H:H + G], x[:, :, H + G:]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("N,H,G", [(3, 4, 2), (8, 2, 1), (8, 4, 1), (32, 1, 1)])
def test_probabilities_of_16_bits(kind, dh, N, H, G):
    print("case precision", kind, dh, N, H, G, flush=True)
    for L, lens in ((64, [40, 17]), (900, [900, 301])):
        s = Step(kind, 2, N, H, G, dh, L, lens, seed=N + L)
        s.run()
        torch.cuda.synchronize()
        q, k, v = parts(s)
        kc, vc = s.values()
        ref, w = drf.tree_attention(q, k, v, kc, vc, lens, None, s.tree.cpu().numpy(), np.zeros(q.shape))
        got = to_f32_numpy(s.out).reshape(q.shape)
        over = np.abs(got - ref) - bound(q, k, kc, ref, got, w, lens)
        assert np.all(over <= 0), (float(np.max(over)), float((over > 0).mean()))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("N,H,G", [(33, 2, 2), (16, 8, 2), (65, 1, 1), (40, 8, 1)])
def test_probabilities_of_8_bits(kind, dh, N, H, G):
    print("case precision, many rows", kind, dh, N, H, G, flush=True)
    for L, lens in ((64, [40, 17]), (900, [900, 301])):
        s = Step(kind, 2, N, H, G, dh, L, lens, seed=N + L)
        s.run()
        torch.cuda.synchronize()
        q, k, v = parts(s)
        kc, vc = s.values()
        tree = s.tree.cpu().numpy()
        ref, w = drf.tree_attention(q, k, v, kc, vc, lens, None, tree, np.zeros(q.shape))
        got = to_f32_numpy(s.out).reshape(q.shape)
        over = np.abs(got - ref) - bound(q, k, kc, ref, got, w, lens, one=True)
        assert np.all(over <= 0), (float(np.max(over)), float((over > 0).mean()))
        mean = np.mean(np.abs(got - ref) ** 2)
        most = 2.0 ** -16 / 3 * np.mean(ref ** 2 + squares(q, k, v, kc, vc, lens, tree))
        assert mean <= 1.05 ** 2 * most, (float(mean), float(most))


def squares(q, k, v, kc, vc, lens, tree):
    """sum_j p_j^2 v_j^2: the softmax at twice the scores has the probabilities p_j^2 / sum p^2."""
    B, N, H, dh = q.shape
    twice, _ = drf.tree_attention(2 * q, k, v ** 2, kc, vc ** 2, lens, None, tree, np.zeros(q.shape))
    out = np.zeros(q.shape)
    for b in range(B):
        mask = drf.sees(tree[b], N, N)
        for h in range(H):
            g = h // (H // k.shape[2])
            for i in range(N):
                s = np.concatenate([kc[b, g, :lens[b]], k[b, np.flatnonzero(mask[i]), g]]) @ q[b, i, h] / dh ** 0.5
                p = np.exp(s - s.max())
                out[b, i, h] = np.sum((p / p.sum()) ** 2) * twice[b, i, h]
    return out


def test_the_bound_tells_8_bits_from_16():
    """On the CPU, the oracle's sums with probabilities of one and of two bf16 numbers: the first is outside, the second inside."""
    rng = np.random.default_rng(1)
    bf = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()  # noqa: E731
    B, N, H, dh, L = 1, 16, 4, 128, 64
    q, k, v = bf(rng.standard_normal((B, N, H, dh))), bf(rng.standard_normal((B, N, 1, dh))), bf(rng.standard_normal((B, N, 1, dh)))
    kc, vc = bf(rng.standard_normal((B, 1, L, dh))), bf(rng.standard_normal((B, 1, L, dh)))
    ref, w = drf.tree_attention(q, k, v, kc, vc, [40], None, None, np.zeros(q.shape))

    def rounded(two):
        out = np.zeros(q.shape)
        for i in range(N):
            K, V = np.concatenate([kc[0, 0, :40], k[0, :i + 1, 0]]), np.concatenate([vc[0, 0, :40], v[0, :i + 1, 0]])
            for h in range(H):
                p = K @ q[0, i, h] / dh ** 0.5
                p = np.exp(p - p.max())
                first = bf(p)
                out[0, i, h] = (first + (bf(p - first) if two else 0)) @ V / p.sum()
        return bf(out)

    for two in (False, True):
        got = rounded(two)
        over = np.abs(got - ref) > bound(q, k, kc, ref, got, w, [40])
        assert (over.mean() == 0) if two else (over.mean() > 0.05), over.mean()
