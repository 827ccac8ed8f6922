"""moe_cache_write and moe_cache_read against oracle/draft_oracle.py: codes, scales and what is read back are equal."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as drf
from tests import gpu_util as U
from workloads.generate import to_f32_numpy

pytestmark = pytest.mark.gpu
DEV = "cuda"
KINDS = ["bf16", "fp8", "fp4"]


def codes_of(cache, kind):
    """One code per element, on the host."""
    c = cache.cpu().numpy()
    if kind == "fp4":
        both = np.stack((c & 15, c >> 4), -1)
        return both.reshape(*c.shape[:-1], -1)
    return c


def garbage(cache, gen):
    """Caches filled with anything, so that what a call leaves alone can be told."""
    full = U.amd().alloc_cache(cache, DEV)
    for t in full:
        if t is not None:
            t.copy_(torch.randint(0, 255, t.shape, generator=gen, device=DEV).to(t.dtype))
    return full


def rows_for(R, G, dh, gen, special=True):
    """[R, G, dh] bf16 of many magnitudes; with odd blocks at the front."""
    x = torch.randn((R, G, dh), generator=gen, device=DEV) * torch.exp(4 * torch.randn((R, G, 1), generator=gen, device=DEV))
    if special:
        x[0, 0, :32] = 0
        x[0, -1, -32:] = torch.tensor([448.0, -449.0, 0.25, 5.0] * 8, device=DEV)
        if R > 2:
            x[1, 0, 5], x[1, -1, dh - 1], x[2, 0, 0] = float("inf"), float("nan"), float("-inf")
        if R > 5:
            x[3] = x[3].abs() * 0 + torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=DEV).repeat(dh // 8)
            x[4, 0, :32] = 1e-39                           # below bf16's normal numbers
            x[4, 0, 32:64] = 2.0 ** -110
            x[5, 0, :32] = 3e38
            x[5, 0, 1:32] = 1e-3
    return x.to(torch.bfloat16)


def check(kind, B, G, dh, L, seq, pos, seed=0, H=None):
    m = U.amd()
    gen = torch.Generator(device=DEV).manual_seed(seed)
    cache = m.make_cache_shape(B, H or G, G, dh, L, kind)
    kc, vc, kx, vx = garbage(cache, gen)
    before = [None if t is None else t.clone() for t in (kc, vc, kx, vx)]
    R = len(seq)
    k, v = rows_for(R, G, dh, gen), rows_for(R, G, dh, gen).flip(0).contiguous()
    wide = torch.zeros((R, 2 * G * dh + 24), dtype=torch.bfloat16, device=DEV)
    wide[:, 8:8 + G * dh], wide[:, 16 + G * dh:16 + 2 * G * dh] = k.flatten(1), v.flatten(1)
    s, p = (torch.tensor(t, dtype=torch.int32, device=DEV) for t in (seq, pos))
    m.moe_cache_write(cache, wide[:, 8:8 + G * dh], wide[:, 16 + G * dh:16 + 2 * G * dh], s, p, kc, vc, kx, vx)
    ok = [r for r in range(R) if 0 <= seq[r] < B and 0 <= pos[r] < L]
    out = torch.full((R + 2, 2 * G * dh + 8), 55.0, dtype=torch.bfloat16, device=DEV)
    ko, vo = out[1:R + 1, :G * dh], out[1:R + 1, G * dh + 8:]
    m.moe_cache_read(cache, kc, vc, kx, vx, s, p, ko, vo)
    torch.cuda.synchronize()
    for rows, got, now, was, scale_now, scale_was in ((k, ko, kc, before[0], kx, before[2]), (v, vo, vc, before[1], vx, before[3])):
        x, back = to_f32_numpy(rows), to_f32_numpy(got).reshape(R, G, dh)
        want = np.full((R, G, dh), 55.0)
        if kind == "bf16":
            expect = was.clone()
            for r in ok:
                expect[seq[r], :, pos[r]] = rows[r]
            assert torch.equal(now.view(torch.int16), expect.view(torch.int16))
            want[ok] = x[ok]
        else:
            codes, scales = codes_of(was, kind).copy(), scale_was.cpu().numpy().copy()
            if ok:
                c, e = drf.quantise(x[ok], kind)
                for n, r in enumerate(ok):
                    codes[seq[r], :, pos[r]], scales[seq[r], :, pos[r]] = c[n], e[n]
                want[ok] = drf.dequantise(c, e, kind)
            assert np.array_equal(scale_now.cpu().numpy(), scales)
            assert np.array_equal(codes_of(now, kind), codes)
        off = ~((back == want) | (np.isnan(back) & np.isnan(want)))
        assert not off.any(), [(a, back[a], want[a]) for a in map(tuple, np.argwhere(off)[:5].tolist())]
    out[1:R + 1, :G * dh] = out[1:R + 1, G * dh + 8:] = 55.0
    assert bool((out == 55.0).all()), "write outside the rows"


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dh", [64, 128])
def test_cache_rows(kind, dh):
    print("case cache", kind, dh, flush=True)
    check(kind, 1, 1, dh, 1, [0], [0])
    check(kind, 3, 2, dh, 50, [0] * 7 + [2] * 9, list(range(7)) + list(range(41, 50)), H=4)
    order = np.random.default_rng(1).permutation(2 * 40)
    check(kind, 2, 3, dh, 40, [int(o) // 40 for o in order], [int(o) % 40 for o in order], seed=2)
    check(kind, 2, 1, dh, 300, [1] * 263, list(range(300 - 263, 300)), seed=3)


@pytest.mark.parametrize("kind", KINDS)
def test_cache_leaves_out_rows(kind):
    print("case cache left out", kind, flush=True)
    check(kind, 2, 2, 64, 9, [0, 0, -1, 2, 1, 1, 0, -2**31, 2**31 - 1], [0, -1, 3, 3, 9, 8, 2**31 - 1, 1, 1])
    check(kind, 2, 2, 128, 9, [-1, -1], [-1, 0])


@pytest.mark.parametrize("kind", KINDS)
def test_cache_one_place_read_by_many(kind):
    m = U.amd()
    gen = torch.Generator(device=DEV).manual_seed(4)
    cache = m.make_cache_shape(2, 2, 2, 64, 5, kind)
    full = m.alloc_cache(cache, DEV)
    x = rows_for(1, 2, 64, gen, special=False).flatten(1)
    one = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    m.moe_cache_write(cache, x, x, one(1), one(3), *full)
    k, v = (torch.empty((70, 128), dtype=torch.bfloat16, device=DEV) for _ in "kv")
    m.moe_cache_read(cache, *full, one(*[1] * 70), one(*[3] * 70), k, v)
    assert torch.equal(k, k[:1].expand_as(k)) and torch.equal(k, v)
    # what was read is exact in the format: writing it once more changes nothing
    again = m.alloc_cache(cache, DEV)
    m.moe_cache_write(cache, k[:1], v[:1], one(1), one(3), *again)
    m.moe_cache_read(cache, *again, one(1), one(3), k[:1], v[:1])
    assert torch.equal(k, v) and torch.equal(k, k[1:2].expand_as(k))


@pytest.mark.parametrize("kind,L", [("bf16", 1 << 22), ("fp8", 1 << 23), ("fp4", 1 << 24)])
def test_cache_behind_32_bits(kind, L):
    """Offsets past 2^32 bytes: the last positions of a cache of 5 GB, two sequences of heads."""
    m = U.amd()
    cache = m.make_cache_shape(5, 1, 1, 128, L, kind)
    assert m.moe_cache_bytes(cache) > 1 << 32
    print("case cache far", kind, flush=True)
    dt, cols = (torch.bfloat16, 128) if kind == "bf16" else (torch.uint8, 128 if kind == "fp8" else 64)
    kc, vc = (torch.empty((5, 1, L, cols), dtype=dt, device=DEV) for _ in "kv")
    kx, vx = (None, None) if kind == "bf16" else (torch.empty((5, 1, L, 4), dtype=torch.uint8, device=DEV) for _ in "kv")
    kc[0, 0, :4], kc[0, 0, L - 4:] = 3, 3
    x = rows_for(3, 1, 128, torch.Generator(device=DEV).manual_seed(6), special=False).flatten(1)
    at = [torch.tensor(t, dtype=torch.int32, device=DEV) for t in ((4, 4, 3), (L - 1, 0, L - 2))]
    m.moe_cache_write(cache, x, x, *at, kc, vc, kx, vx)
    k, v = torch.zeros_like(x), torch.zeros_like(x)
    m.moe_cache_read(cache, kc, vc, kx, vx, *at, k, v)
    want = to_f32_numpy(x) if kind == "bf16" else drf.dequantise(*drf.quantise(to_f32_numpy(x), kind), kind)
    assert np.array_equal(to_f32_numpy(k), want) and torch.equal(k, v)
    assert bool((kc[0, 0, :4] == 3).all()) and bool((kc[0, 0, L - 4:] == 3).all())


@pytest.mark.parametrize("kind,dh", [("bf16", 64), ("fp8", 128), ("fp4", 64), ("fp4", 128), ("fp8", 64)])
def test_cache_many_rows(kind, dh):
    """Rows enough for two units per thread, an odd number of them, some left out; what is read equals what a few rows at a time give."""
    m = U.amd()
    gen = torch.Generator(device=DEV).manual_seed(8)
    B, G, L = 3, 4, 11003
    n = B * L - 2
    assert n * G * dh >= 1 << 23
    print("case cache many", kind, dh, flush=True)
    cache = m.make_cache_shape(B, G, G, dh, L, kind)
    x, y = (torch.randn((n, G * dh), generator=gen, device=DEV).to(torch.bfloat16) for _ in "kv")
    order = torch.randperm(B * L, generator=gen, device=DEV)[:n]
    seq, pos = (order // L).to(torch.int32), (order % L).to(torch.int32)
    pos[7::13] = -1
    one, few = m.alloc_cache(cache, DEV), m.alloc_cache(cache, DEV)
    m.moe_cache_write(cache, x, y, seq, pos, *one)
    for a in range(0, n, 4096 // 16 * 16):
        b = min(n, a + 4096 // 16 * 16)
        m.moe_cache_write(cache, x[a:b], y[a:b], seq[a:b].clone(), pos[a:b].clone(), *few)
    assert all(s is None or torch.equal(s, t) for s, t in zip(one, few))
    k, v = torch.full_like(x, 5.0), torch.full_like(y, 5.0)
    m.moe_cache_read(cache, *one, seq, pos, k, v)
    some = torch.arange(0, n, 997, device=DEV)
    for rows, back in ((x, k), (y, v)):
        want = to_f32_numpy(rows[some]).reshape(-1, G, dh)
        if kind != "bf16":
            want = drf.dequantise(*drf.quantise(want, kind), kind)
        want[(pos[some] < 0).cpu().numpy()] = 5.0
        assert np.array_equal(to_f32_numpy(back[some]).reshape(-1, G, dh), want)


def test_cache_more_rows_than_one_grid_dimension():
    m = U.amd()
    gen = torch.Generator(device=DEV).manual_seed(9)
    n = (1 << 20) + 4099
    print("case cache grid", flush=True)
    cache = m.make_cache_shape(1, 1, 1, 128, n, "fp8")
    x, y = (torch.randn((n, 128), generator=gen, device=DEV).to(torch.bfloat16) for _ in "kv")
    seq, pos = torch.zeros(n, dtype=torch.int32, device=DEV), torch.arange(n, dtype=torch.int32, device=DEV).flip(0).contiguous()
    held = m.alloc_cache(cache, DEV)
    m.moe_cache_write(cache, x, y, seq, pos, *held)
    k, v = torch.zeros_like(x), torch.zeros_like(y)
    m.moe_cache_read(cache, *held, seq, pos, k, v)
    some = torch.cat((torch.arange(0, n, 9973, device=DEV), torch.arange(n - 40, n, device=DEV)))
    for rows, back in ((x, k), (y, v)):
        want = drf.dequantise(*drf.quantise(to_f32_numpy(rows[some]), "fp8"), "fp8")
        assert np.array_equal(to_f32_numpy(back[some]), want)
    assert bool((k.float() - x.float()).abs().max() < 0.5) and bool((v.float() - y.float()).abs().max() < 0.5)
