"""moe_tree_attention and the caches at the ends of their ranges: NaN right behind every length on every choice of tile, the most heads,
rows of one head over many blocks, the longest distances between rows."""
import numpy as np
import pytest
import torch

from tests import gpu_util as U
from tests.test_gpu_cache import check as check_cache
from tests.test_gpu_tree_attention import DEV, KINDS, Step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("N,H,G", [(3, 4, 2), (8, 4, 1), (16, 4, 1), (33, 4, 1)])
def test_tree_nan_behind_every_length(kind, dh, N, H, G):
    lens = list(range(67))
    print("case tree behind", kind, dh, N, H, G, flush=True)
    s = Step(kind, len(lens), N, H, G, dh, 70, lens, [1 + b % N for b in lens], seed=N + dh)
    for b, n in enumerate(lens):
        for cache, scale in zip(s.caches[:2], s.caches[2:]):
            if kind == "bf16":
                cache[b, :, n:] = float("nan")
            else:
                scale[b, :, n:] = 255
    new = s.qkv.view(len(lens), N, -1)
    for b in lens:
        new[b, 1 + b % N:] = float("nan")
    s.run()
    s.check()


@pytest.mark.parametrize("N,H,G,L,lens", [(1, 1024, 1024, 33, [33, 5]), (8, 1024, 1, 40, [40, 0]), (2, 1024, 8, 130, [7, 129])])
def test_tree_1024_heads(N, H, G, L, lens):
    for kind in KINDS:
        print("case tree heads", kind, N, H, G, flush=True)
        s = Step(kind, 2, N, H, G, 64, L, lens, seed=H + G)
        s.run()
        s.check()


@pytest.mark.parametrize("kind", KINDS)
def test_cache_1024_heads(kind):
    print("case cache heads", kind, flush=True)
    check_cache(kind, 2, 1024, 64, 5, [0, 1, 1, 0, 2, 1, 0], [4, 0, 3, -1, 0, 5, 2], H=1024)


def test_tree_longest_distances():
    """Rows 2^24 elements apart: the last drafted token of a tile is a gigabyte behind the first."""
    m = U.amd()
    N, dh, far = 33, 64, 1 << 24
    s = Step("bf16", 1, N, 1, 1, dh, 40, [40], seed=5)
    want = s.run().clone()
    room = torch.zeros((N - 1) * far + 4 * dh, dtype=torch.bfloat16, device=DEV)
    q, k, v, out = (room.as_strided((N, dh), (far, 1), i * dh) for i in range(4))
    q.copy_(s.qkv[:, :dh]), k.copy_(s.qkv[:, dh:2 * dh]), v.copy_(s.qkv[:, 2 * dh:3 * dh])
    print("case tree far rows", flush=True)
    m.moe_tree_attention(s.shape, N, q, k, v, *s.caches, s.lens, None, s.tree, out, s.ws)
    assert torch.equal(out, want)
    rows = torch.arange(N, dtype=torch.int32, device=DEV)
    m.moe_cache_write(s.shape, k, v, torch.zeros_like(rows), rows, *s.caches)
    assert torch.equal(s.caches[0][0, 0, :N], k) and torch.equal(s.caches[1][0, 0, :N], v)
    rope = m.make_rope(dh, dh, "half", "bf16")
    turns = m.moe_rope_frequencies(rope, DEV)
    near = q.contiguous()
    m.moe_rope(rope, near, turns, rows, near)
    m.moe_rope(rope, q, turns, rows, out)
    assert torch.equal(out, near)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("N,H,G", [(5, 2, 1), (31, 1, 1), (40, 2, 2), (33, 4, 1), (70, 2, 1)])
def test_tree_all_bits_set(kind, N, H, G):
    """Every token sees every other, later ones too; bits from the count on are ignored, those behind n_draft in the last word too."""
    counts = [N, 1, 0, (N + 1) // 2, N - 1]
    print("case tree all bits", kind, N, H, G, flush=True)
    s = Step(kind, 5, N, H, G, 64, 50, [50, 0, 20, 33, 0], counts, tree=np.full((5, N, (N + 31) // 32), -1, np.int32), seed=N)
    for b, n in enumerate(counts):
        s.qkv.view(5, N, -1)[b, n:] = float("nan")
    s.run()
    s.check()
