"""moe_tree_attention against oracle/draft_oracle.py.

Error bound, from the formats, with w = sum_j p_j |v_j| over the softmax: probabilities are rounded to bf16 (half a step: 2^-8 of
each, 2^-8 w); a score is a sum of dh products in 32 bits, off by at most dh 2^-24 sum |q k| / sqrt(dh) =: d, which moves every
probability and their sum by d (2 d w); exponentials and the sums over n positions are within (n + 64) 2^-23 w; the result is
rounded by half a step, 2^-8 of its value."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as drf
from tests import gpu_util as U
from tests.test_gpu_cache import codes_of
from workloads.generate import to_f32_numpy

pytestmark = pytest.mark.gpu
DEV = "cuda"
KINDS = ["bf16", "fp8", "fp4"]


def random_tree(B, N, seed, branch=4):
    """Each token's parent is one of the `branch` tokens before it, or the last cached one."""
    rng = np.random.default_rng(seed)
    bits = np.zeros((B, N, N), bool)
    for b in range(B):
        for i in range(N):
            p = i - 1 - rng.integers(0, min(branch, i + 1))
            if p >= 0:
                bits[b, i] = bits[b, p]
            bits[b, i, i] = True
    return bits


def words(bits):
    B, N, _ = bits.shape
    out = np.zeros((B, N, (N + 31) // 32), np.uint32)
    for j in range(N):
        out[:, :, j // 32] |= bits[:, :, j].astype(np.uint32) << np.uint32(j % 32)
    return out.view(np.int32)


class Step:
    """Inputs of one call; a test changes them before run() and check()."""

    def __init__(self, kind, B, N, H, G, dh, L, lens, counts=None, tree="random", seed=0, spread=1.0):
        m = U.amd()
        self.kind, self.dims = kind, (B, N, H, G, dh, L)
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.shape = m.make_cache_shape(B, H, G, dh, L, kind)
        rnd = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
        self.qkv = (spread * rnd(B * N, (H + 2 * G) * dh + 8)).to(torch.bfloat16)
        if kind == "bf16":
            self.caches = [rnd(B, G, L, dh).to(torch.bfloat16) for _ in "kv"] + [None, None]
        else:
            cols = dh if kind == "fp8" else dh // 2
            # any code but e4m3's NaN, scales that bring the values near 1
            code = lambda: torch.randint(0, 256, (B, G, L, cols), generator=g, device=DEV).to(torch.uint8)  # noqa: E731
            fine = lambda c: torch.where((c & 127) == 127, c - 1, c) if kind == "fp8" else c  # noqa: E731
            exp = lambda: torch.randint(*((115, 120) if kind == "fp8" else (123, 127)), (B, G, L, dh // 32), generator=g, device=DEV).to(torch.uint8)  # noqa: E731
            self.caches = [fine(code()), fine(code()), exp(), exp()]
        self.lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
        self.counts = None if counts is None else torch.tensor(counts, dtype=torch.int32, device=DEV)
        tree = words(random_tree(B, N, seed)) if isinstance(tree, str) else tree
        self.tree = None if tree is None else torch.from_numpy(tree).to(DEV)
        self.room = torch.full((B * N + 2, H * dh + 16), 9.0, dtype=torch.bfloat16, device=DEV)
        self.out = self.room[1:B * N + 1, 8:8 + H * dh]
        self.ws = torch.full((m.moe_tree_attention_workspace_bytes(self.shape, N),), 255, dtype=torch.uint8, device=DEV)

    def run(self):
        B, N, H, G, dh, L = self.dims
        nq, nk = H * dh, G * dh
        U.amd().moe_tree_attention(self.shape, N, self.qkv[:, :nq], self.qkv[:, nq:nq + nk], self.qkv[:, nq + nk:nq + 2 * nk], *self.caches, self.lens,
                                   self.counts, self.tree, self.out, self.ws)
        return self.out

    def values(self):
        ks, vs, kx, vx = self.caches
        if self.kind == "bf16":
            return to_f32_numpy(ks), to_f32_numpy(vs)
        return tuple(drf.dequantise(codes_of(c, self.kind), x.cpu().numpy(), self.kind) for c, x in ((ks, kx), (vs, vx)))

    def check(self):
        B, N, H, G, dh, L = self.dims
        x = to_f32_numpy(self.qkv)[:, :(H + 2 * G) * dh].reshape(B, N, H + 2 * G, dh).astype(np.float64)
        q, k, v = x[:, :, :H], x[:, :, H:H + G], x[:, :, H + G:]
        kc, vc = self.values()
        lens, counts = self.lens.cpu().numpy(), None if self.counts is None else self.counts.cpu().numpy()
        ref, w = drf.tree_attention(q, k, v, kc, vc, lens, counts, None if self.tree is None else self.tree.cpu().numpy(), np.full((B, N, H, dh), 9.0))
        torch.cuda.synchronize()
        got = to_f32_numpy(self.out).reshape(B, N, H, dh)
        near = np.zeros((B, N, H, 1))
        for b in range(B):
            n = int(np.clip(lens[b], 0, L))
            for h in range(H):
                keys = np.concatenate([np.abs(kc[b, h // (H // G), :n]), np.abs(k[b, :, h // (H // G)])])
                keys = np.where(np.isfinite(keys), keys, 0.0)
                near[b, :, h, 0] = (np.abs(q[b, :, h]) @ keys.T).max(-1) * dh ** 0.5 * 2.0 ** -24
        tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2 * near + (L + N + 64) * 2.0 ** -23) * w
        fine = np.isfinite(ref)
        assert not (np.isfinite(got) != fine).any(), np.argwhere(np.isfinite(got) != fine)[:5].tolist()
        d = np.abs(np.where(fine, got - np.where(fine, ref, 0), 0))
        left = np.array([[i >= (N if counts is None else counts[b]) for i in range(N)] for b in range(B)])
        tol[left] = 0                                  # rows behind the count are as they were (a query there may be NaN)
        off = d > np.where(fine, tol, 1)
        assert not off.any() and not np.isnan(tol[fine]).any(), (float(d.max()), np.argwhere(off)[:5].tolist())
        room = self.room.clone()
        room[1:B * N + 1, 8:8 + H * dh] = 9.0
        assert bool((room == 9.0).all()), "write outside out"
        return got, ref


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("B,N,H,G,L,lens", [
    (1, 1, 1, 1, 1, [0]), (1, 1, 1, 1, 1, [1]), (2, 1, 4, 1, 40, [0, 40]), (3, 5, 2, 2, 70, [1, 33, 70]), (2, 16, 3, 1, 129, [128, 129]),
    (4, 7, 8, 2, 300, [0, 31, 32, 257]), (2, 33, 4, 2, 65, [64, 65]), (1, 64, 8, 1, 200, [199]), (2, 12, 10, 2, 520, [511, 513])])
def test_tree_sizes(kind, dh, B, N, H, G, L, lens):
    print("case tree", kind, dh, B, N, H, G, L, lens, flush=True)
    s = Step(kind, B, N, H, G, dh, L, lens)
    s.run()
    s.check()


@pytest.mark.parametrize("kind", KINDS)
def test_tree_counts_and_chain(kind):
    print("case tree counts", kind, flush=True)
    for N, counts in ((9, [0, 9, 3, 1]), (40, [40, 33, 0, 17])):
        s = Step(kind, 4, N, 4, 2, 128, 90, [0, 90, 45, 64], counts)
        s.run()
        s.check()
        s = Step(kind, 4, N, 4, 2, 64, 90, [0, 90, 45, 64], counts, tree=None, seed=1)
        s.run()
        s.check()
    # out of range: clamped
    s = Step(kind, 4, 3, 2, 2, 64, 30, [-5, 31, 2**31 - 1, -2**31], [-1, 4, 2**31 - 1, 2])
    s.run()
    s.check()


@pytest.mark.parametrize("dh", [64, 128])
def test_tree_rows_that_see_nothing(dh):
    N = 35
    bits = random_tree(3, N, 7)
    bits[:, ::3] = False                               # every third token sees no drafted token, not even itself
    s = Step("bf16", 3, N, 4, 2, dh, 64, [0, 0, 20], [N, 20, N], words(bits))
    s.run()
    got, _ = s.check()
    assert np.all(got[0, ::3] == 0) and np.all(got[1, 0:20:3] == 0) and np.any(got[2, 0] != 0)


@pytest.mark.parametrize("kind", KINDS)
def test_tree_not_seen_may_hold_anything(kind):
    """Infinities and NaN behind a sequence's length, behind its count, and in drafted tokens that others do not see."""
    B, N, H, G, dh, L = 2, 20, 4, 2, 128, 100
    bits = random_tree(B, N, 3)
    bits[:, :, 4], bits[:, :, 11] = False, False       # nobody but themselves sees tokens 4 and 11
    bits[:, 4, 4] = bits[:, 11, 11] = True
    s = Step(kind, B, N, H, G, dh, L, [37, 64], [N, 15], words(bits), seed=2)
    nq, nk = H * dh, G * dh
    x = s.qkv.view(B, N, -1)
    x[:, 4, nq + 3], x[:, 4, nq + nk + 5] = float("nan"), float("inf")
    x[:, 11, nq:nq + 2 * nk] = float("-inf")
    x[1, 15:, :nq + 2 * nk] = float("nan")
    ks, vs, kx, vx = s.caches
    for b, n in enumerate((37, 64)):
        if kind == "bf16":
            ks[b, :, n:], vs[b, :, n:] = float("nan"), float("inf")
        else:
            kx[b, :, n:], vx[b, :, n:] = 255, 255
    s.run()
    got, ref = s.check()
    fine = np.isfinite(ref).all(axis=(2, 3))
    assert fine.sum() == 2 * N - 4                     # all rows but 4 and 11 (those behind the count hold what they held)


def test_tree_peaked_and_large_scores():
    for spread in (20.0, 200.0):
        s = Step("bf16", 2, 6, 4, 2, 128, 700, [700, 333], spread=spread, seed=5)
        s.run()
        s.check()


def test_tree_long():
    """Lengths at which the positions are split over many work-groups, with one that holds little."""
    for kind, dh in (("bf16", 64), ("fp8", 128), ("fp4", 128)):
        print("case tree long", kind, flush=True)
        s = Step(kind, 3, 5, 4, 1, dh, 9001, [9001, 3, 4097], seed=8)
        s.run()
        s.check()


@pytest.mark.parametrize("N", [100, 256])
def test_tree_many_tokens(N):
    print("case tree many", N, flush=True)
    s = Step("bf16", 2, N, 2, 1, 64, 40, [40, 7], seed=9)
    s.run()
    s.check()


def test_tree_same_bits_again():
    s = Step("fp8", 3, 9, 8, 2, 128, 3001, [3001, 17, 1200], seed=10)
    first = s.run().clone()
    for _ in range(3):
        s.ws.fill_(255)
        s.out.fill_(9.0)
        assert torch.equal(s.run(), first)


def test_tree_captured():
    """Two captured calls with workspaces of their own, replayed with other lengths and rows, against the eager call."""
    steps = [Step("fp8", 3, 9, 8, 2, 128, 3001, [3001, 17, 1200], seed=11), Step("bf16", 2, 3, 4, 4, 64, 500, [500, 1], seed=12)]
    for s in steps:
        s.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for s in steps:
            s.run()
    for n in (1, 0, 2500):
        for s in steps:
            s.lens[0] = min(n, s.dims[5])
            s.qkv.add_(0.25)
            s.out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        for s in steps:
            got = s.out.clone()
            s.check()
            s.out.fill_(9.0)
            assert torch.equal(s.run(), got)


def test_tree_on_another_stream():
    s = Step("bf16", 2, 4, 4, 2, 64, 300, [300, 150], seed=13)
    want = s.run().clone()
    s.out.fill_(9.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = s.run()
    side.synchronize()
    assert torch.equal(got, want)


def test_tree_cache_behind_32_bits():
    """The last sequence's cache begins 4 GB behind the first one's."""
    m = U.amd()
    L, dh, N = 1 << 22, 128, 2
    print("case tree far", flush=True)
    shape = m.make_cache_shape(5, 1, 1, dh, L, "bf16")
    kc, vc = (torch.zeros((5, 1, L, dh), dtype=torch.bfloat16, device=DEV) for _ in "kv")
    small = Step("bf16", 5, N, 1, 1, dh, 100, [100, 50, 3, 77, 99], seed=14)
    for big, little in ((kc, small.caches[0]), (vc, small.caches[1])):
        big[:, :, :100] = little
    want = small.run().clone()
    small.shape, small.caches = shape, [kc, vc, None, None]
    small.ws = torch.empty(m.moe_tree_attention_workspace_bytes(shape, N), dtype=torch.uint8, device=DEV)
    small.out.fill_(9.0)
    assert (small.run().float() - want.float()).abs().max() <= 2.0 ** -7 * want.float().abs().max()
    # every position of the last sequence: equal keys, so the mean of the values
    kc[4, 0], vc[4, 0] = 0, 0
    vc[4, 0, L // 2:] = 2.0
    small.lens[4] = L
    small.qkv.zero_()
    got = small.run()[4 * N:].float()
    assert (got - 1.0).abs().max() <= 2.0 ** -7


@pytest.mark.parametrize("kind,dh", [("bf16", 128), ("fp8", 64)])
def test_tree_many_sequences(kind, dh):
    """More sequences than a wave has lanes, ragged, with empty ones and such without drafted tokens among them, at both ends too."""
    rng = np.random.default_rng(4)
    for B, N in ((65, 3), (203, 5)):
        lens, counts = rng.integers(0, 120, B), rng.integers(0, N + 1, B)
        lens[::7], counts[::5] = 0, 0
        lens[3] = 1200                                  # one that takes as long as many others
        print("case tree many sequences", kind, B, flush=True)
        s = Step(kind, B, N, 2, 1, dh, 1200, [int(v) for v in lens], [int(v) for v in counts], seed=B)
        s.run()
        s.check()


def test_tree_nothing_to_do():
    """No drafted token anywhere: out stays as it is."""
    s = Step("bf16", 3, 4, 2, 1, 64, 50, [50, 0, 7], [0, 0, 0])
    s.run()
    s.check()


@pytest.mark.parametrize("N,H,G", [(8, 2, 1), (16, 2, 1), (17, 2, 1), (32, 2, 1), (33, 2, 1), (64, 2, 1), (65, 2, 1), (100, 6, 2)])
def test_tree_rows_at_the_edges_of_the_blocks(N, H, G):
    """Rows per key/value head on both sides of every choice of tile, and blocks of rows beyond 128, over shares that end inside an item."""
    for kind, dh, L in (("fp8", 128, 700), ("bf16", 128, 333), ("fp4", 64, 500)):
        print("case tree rows", N, H, G, kind, flush=True)
        s = Step(kind, 2, N, H, G, dh, L, [L, L // 3], seed=N)
        s.run()
        s.check()


def test_tree_rows_with_distances_of_their_own():
    s = Step("bf16", 2, 5, 4, 2, 64, 90, [90, 44], seed=3)
    want = s.run().clone()
    q, k, v = (s.qkv[:, a:b] for a, b in ((0, 256), (256, 384), (384, 512)))
    far = torch.zeros((10, 4096), dtype=torch.bfloat16, device=DEV)
    far[:, 1024:1152] = k
    apart = torch.zeros((10, 136), dtype=torch.bfloat16, device=DEV)
    apart[:, 8:] = v
    s.out.fill_(9.0)
    U.amd().moe_tree_attention(s.shape, 5, q.contiguous(), far[:, 1024:1152], apart[:, 8:], *s.caches, s.lens, s.counts, s.tree, s.out, s.ws)
    assert torch.equal(s.out, want)


def test_tree_seen_nonfinite():
    """NaN in a cached key or value is for all that see it; keys of minus infinity alone leave no probability (NaN), one among others none of it."""
    s = Step("bf16", 3, 4, 2, 2, 64, 40, [40, 40, 1], tree=np.zeros((3, 4, 1), np.int32), seed=6)
    ks, vs = s.caches[0], s.caches[1]
    ks[0, 0, 5, 3] = float("nan")
    vs[1, 1, 39, 7] = float("nan")
    s.qkv[:, :64] = s.qkv[:, :64].abs()
    ks[2, 0, 0] = float("-inf")
    got, ref = (s.run(), s.check())[1]
    assert np.isnan(got[0, :, 0]).all() and np.isfinite(got[0, :, 1]).all()
    assert np.isnan(got[1, :, 1, 7]).all() and np.isfinite(got[1, :, 1, :7]).all() and np.isfinite(got[1, :, 0]).all()
    assert np.isnan(got[2, :, 0]).all() and np.isfinite(got[2, :, 1]).all()


def test_tree_two_calls_at_once():
    """Two streams, a workspace each."""
    a, b = Step("fp8", 4, 8, 8, 2, 128, 2000, [2000, 5, 999, 1500], seed=1), Step("bf16", 2, 40, 4, 1, 64, 900, [900, 33], seed=2)
    wants = [s.run().clone() for s in (a, b)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in (a, b):
        s.out.fill_(9.0)
    torch.cuda.synchronize()
    for _ in range(5):
        for s, st in zip((a, b), streams):
            with torch.cuda.stream(st):
                s.run()
    torch.cuda.synchronize()
    assert torch.equal(a.out, wants[0]) and torch.equal(b.out, wants[1])


@pytest.mark.parametrize("kind,dh,N", [("bf16", 64, 4), ("bf16", 128, 70), ("fp8", 128, 16), ("fp4", 64, 3), ("fp4", 128, 33), ("fp8", 64, 20)])
def test_tree_every_length(kind, dh, N):
    """Lengths that leave every number of positions in a tile, with NaN right behind each."""
    lens = list(range(70))
    print("case tree every length", kind, dh, N, flush=True)
    s = Step(kind, len(lens), N, 2, 1, dh, 70, lens, [1 + b % N for b in lens], seed=N)
    for b, n in enumerate(lens):
        for cache, scale in zip(s.caches[:2], s.caches[2:]):
            if kind == "bf16":
                cache[b, :, n:] = float("nan")
            else:
                scale[b, :, n:] = 255
    s.run()
    s.check()


def test_tree_graphs_that_share_a_workspace():
    """Two captured calls of different kinds on one workspace, replayed in turn: each finds what it needs written by itself."""
    steps = [Step("fp8", 3, 9, 8, 2, 128, 3001, [3001, 17, 1200], seed=21), Step("fp4", 2, 20, 8, 2, 64, 900, [900, 1], seed=22)]
    ws = max((s.ws for s in steps), key=torch.numel)
    graphs = []
    for s in steps:
        s.ws = ws
        s.run()
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            s.run()
    wants = [s.run().clone() for s in steps]
    for _ in range(3):
        for s, graph, want in zip(steps, graphs, wants):
            s.out.fill_(9.0)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(s.out, want)
            s.check()


def test_tree_thousands_of_sequences():
    B, rng = 4000, np.random.default_rng(7)
    print("case tree thousands", flush=True)
    s = Step("fp8", B, 2, 2, 1, 64, 24, [int(v) for v in rng.integers(0, 25, B)], [int(v) for v in rng.integers(0, 3, B)], seed=23)
    s.run()
    s.check()
