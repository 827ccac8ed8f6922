"""moe_tree_attention where scores are far larger than what separates them.

All scores here are integers times a power of two, with at most 24 bits even in their partial sums: exact in the kernel's 32 bits, so
none of the error is theirs.  What is left, with w = sum_j p_j |v_j| over the softmax: c = log2(e) / sqrt(dh) and its product with the
difference of two scores are within 2^-22 of values that are below 2^5 wherever a probability counts, which moves a probability by less than 2^-17; exponentials
and the sums over n positions are within (n + 64) 2^-23 w; a probability is rounded to bf16 at worst (half a step, 2^-8 w); the result
by half a step, 2^-8 of its value."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as drf
from tests import gpu_util as U
from tests.test_gpu_tree_attention import DEV, KINDS, Step
from workloads.generate import to_f32_numpy

pytestmark = pytest.mark.gpu
# every choice of tile: 1, 32, 64 and 132 rows per key/value head
ROWS = [(1, 1, 1), (8, 4, 1), (16, 4, 1), (33, 4, 1)]


def set_keys(s, cached, drafted):
    """Cached keys [B, G, L, dh], quantised if the cache is (exactly, for the values of these tests), and drafted keys [B, N, G, dh]."""
    B, N, H, G, dh, L = s.dims
    rows = torch.from_numpy(cached).to(DEV).to(torch.bfloat16).permute(0, 2, 1, 3).reshape(B * L, G * dh).contiguous()
    seq = torch.arange(B, dtype=torch.int32, device=DEV).repeat_interleave(L)
    pos = torch.arange(L, dtype=torch.int32, device=DEV).repeat(B)
    vc, vx = s.caches[1].clone(), None if s.caches[3] is None else s.caches[3].clone()
    U.amd().moe_cache_write(s.shape, rows, rows, seq, pos, *s.caches)
    s.caches[1].copy_(vc)
    if vx is not None:
        s.caches[3].copy_(vx)
    s.qkv[:, H * dh:(H + G) * dh] = torch.from_numpy(drafted.reshape(B * N, G * dh)).to(DEV).to(torch.bfloat16)
    assert np.array_equal(s.values()[0], cached)


def check(s):
    B, N, H, G, dh, L = s.dims
    x = to_f32_numpy(s.qkv)[:, :(H + 2 * G) * dh].reshape(B, N, H + 2 * G, dh).astype(np.float64)
    counts = None if s.counts is None else s.counts.cpu().numpy()
    ref, w = drf.tree_attention(x[:, :, :H], x[:, :, H:H + G], x[:, :, H + G:], *s.values(), s.lens.cpu().numpy(), counts,
                                None if s.tree is None else s.tree.cpu().numpy(), np.full((B, N, H, dh), 9.0))
    torch.cuda.synchronize()
    got = to_f32_numpy(s.out).reshape(B, N, H, dh)
    assert np.isfinite(got).all(), np.argwhere(~np.isfinite(got))[:5].tolist()
    tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -17 + (L + N + 64) * 2.0 ** -23) * w
    assert np.all(np.abs(got - ref) <= tol), float(np.max(np.abs(got - ref) - tol))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("power", [0, 15, 17, 30])
@pytest.mark.parametrize("N,H,G", ROWS)
def test_finite_scores_give_finite_results(kind, power, N, H, G):
    """Elements of 1 to 3 times 2^power: scores of up to 2^(2 power + 10), equal ones among them, and the largest of either sign."""
    print("case large scores", kind, power, N, H, G, flush=True)
    rng = np.random.default_rng(power)
    for dh, L, lens in ((128, 700, [700, 333]), (64, 90, [1, 0])):
        s = Step(kind, 2, N, H, G, dh, L, lens, seed=power)
        keys = rng.integers(1, 4, (2, G, L, dh)) * 2.0 ** power * rng.choice([-1.0, 1.0], (2, G, L, 1))
        keys[:, :, 5::11] = keys[:, :, 3:4]                    # the same key many times, all over
        set_keys(s, keys, rng.integers(1, 4, (2, N, G, dh)) * 2.0 ** power * rng.choice([-1.0, 1.0], (2, N, G, 1)))
        q = rng.integers(1, 4, (2 * N, H * dh)) * 2.0 ** power * rng.choice([-1.0, 1.0], (2 * N, 1))
        s.qkv[:, :H * dh] = torch.from_numpy(q).to(DEV).to(torch.bfloat16)
        s.run()
        check(s)


def test_one_position_is_its_value():
    """Whatever its score is."""
    s = Step("bf16", 1, 1, 2, 1, 64, 40, [1], tree=np.zeros((1, 1, 1), np.int32))
    for size in (1.0, 1e4, 1e5, 1e8, 1e17, -1e5, -1e17):
        s.qkv[:, :128], s.caches[0][0, 0, 0] = abs(size), size
        s.run()
        assert torch.equal(s.out.view(2, 64), s.caches[1][0, 0, :1].expand(2, 64)), size


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("N,H,G", ROWS)
def test_small_differences_of_large_scores(kind, sign, N, H, G):
    """Scores of 2^22 and a little: the same softmax as without the 2^22, also where parts with other maxima are joined."""
    print("case small differences", kind, sign, N, H, G, flush=True)
    rng = np.random.default_rng(3)
    B, dh, L = 2, 128, 3000
    s = Step(kind, B, N, H, G, dh, L, [L, 1111], seed=4)
    # in blocks of 32 that share a scale: 2^11 alone, then zeros and ones of which more and more are ones along the positions
    often = np.linspace(0.05, 0.95, L)[:, None]
    keys = np.zeros((B, G, L, dh))
    keys[..., 0], keys[..., 32:] = sign * 2048.0, rng.random((B, G, L, dh - 32)) < often
    new = np.zeros((B, N, G, dh))
    new[..., 0], new[..., 32:] = sign * 2048.0, rng.random((B, N, G, dh - 32)) < 0.9
    set_keys(s, keys, new)
    s.qkv[:, :H * dh] = 0.0
    q = s.qkv[:, :H * dh].view(B * N, H, dh)
    q[..., 0], q[..., 32:] = 2048.0, 1.0
    s.run()
    check(s)


@pytest.mark.parametrize("N,H,G", ROWS)
def test_infinite_drafted_value_of_no_weight(N, H, G):
    """A drafted value that every token sees is infinite in one element, and cached scores are larger by thousands: that element is an
    infinity or NaN, the others are what they are without it."""
    s = Step("bf16", 2, N, H, G, 64, 300, [300, 7], tree=None, seed=9)
    nq, nk = H * 64, G * 64
    s.qkv[:, :nq], s.caches[0][:, :, 5] = s.qkv[:, :nq].abs() + 1, 100.0
    want = s.run().clone().view(2, N, H, 64)
    s.qkv.view(2, N, -1)[:, 0, nq + nk + 3] = float("inf")
    s.out.fill_(9.0)
    got = s.run().view(2, N, H, 64)
    rest = [i for i in range(64) if i != 3]
    assert not torch.isfinite(got[..., 3]).any() and torch.equal(got[..., rest], want[..., rest])
