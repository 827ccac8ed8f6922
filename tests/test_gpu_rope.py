"""moe_rope against oracle/draft_oracle.py.

Error bound, from the formats: the angle in half turns is at most 1 and rounded to 32 bits (2^-25, 2^-23 in radians), sine and
cosine are within 2 units (2^-23), amplitude, two products and a sum round four times (2^-24 each): less than 2^-21 amplitude
(|x| + |y|) in all, and the result is rounded by half a step, eps / 2 of its value."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as drf
from tests import gpu_util as U
from workloads.generate import to_f32_numpy

pytestmark = pytest.mark.gpu
DEV = "cuda"
SCALED = {"plain": dict(base=10000.0), "linear": dict(base=500000.0, factor=8.0),
          "by_parts": dict(base=500000.0, factor=32.0, original_len=8192.0, low=1.0, high=4.0)}


def _check(rows, heads, dh, rot, layout, scaling="plain", dtype="bf16", amplitude=1.0, pos=None, before=0, behind=0, in_place=False, seed=0):
    """`before`, `behind`: columns of the row around the heads."""
    m = U.amd()
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    n = heads * dh
    wide = torch.randn((rows, before + n + behind), generator=g, device=DEV).to(dt)
    start = wide.clone()
    x = wide[:, before:before + n]
    if pos is None:
        pos = torch.randint(0, 5000, (rows,), generator=g, device=DEV, dtype=torch.int32)
    rope = m.make_rope(dh, rot, layout, dtype, amplitude=amplitude, scaling=scaling, **SCALED[scaling])
    turns = m.moe_rope_frequencies(rope, DEV)
    room = torch.full((rows + 2, n + 16), 77.0, dtype=dt, device=DEV)
    out = x if in_place else room[1:1 + rows, 8:8 + n]
    m.moe_rope(rope, x, turns, pos, out)
    torch.cuda.synchronize()
    f = drf.rope_frequencies(rot, scaling=scaling, **SCALED[scaling])
    host = to_f32_numpy(start)[:, before:before + n].reshape(rows, heads, dh).astype(np.float64)
    p = pos.cpu().numpy()
    ref = drf.rope(host, p, f, layout, np.float32(amplitude))
    amp = abs(float(np.float32(amplitude)))
    size = np.zeros_like(ref)
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    size[..., a] = size[..., b] = np.abs(host[..., a]) + np.abs(host[..., b])
    got = to_f32_numpy(out).reshape(rows, heads, dh)
    live = p >= 0
    tol = torch.finfo(dt).eps / 2 * np.abs(ref) + 2.0 ** -21 * amp * size
    assert np.all(np.abs(got - ref)[live] <= tol[live]), float(np.max((np.abs(got - ref) - tol)[live]))
    assert np.array_equal(got[..., rot:][live], host[..., rot:][live])
    was = to_f32_numpy(start)[:, before:before + n] if in_place else np.full((rows, n), 77.0)
    assert np.array_equal(got[~live].reshape(-1, n), was[~live])
    if in_place:
        assert torch.equal(wide[:, :before], start[:, :before]) and torch.equal(wide[:, before + n:], start[:, before + n:])
    else:
        assert torch.equal(wide, start)
        room[1:1 + rows, 8:8 + n] = 77.0
        assert bool((room == 77.0).all()), "write outside out"


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,heads,dh,rot", [(1, 1, 8, 8), (1, 5, 64, 64), (3, 2, 64, 24), (33, 3, 128, 128), (257, 7, 80, 32), (64, 1, 128, 8),
                                               (5, 4, 512, 512), (2, 2, 96, 72)])
def test_rope_sizes(rows, heads, dh, rot, layout, dtype):
    print("case rope", rows, heads, dh, rot, layout, dtype, flush=True)
    _check(rows, heads, dh, rot, layout, dtype=dtype, before=16, behind=24)
    _check(rows, heads, dh, rot, layout, dtype=dtype, before=8, in_place=True, seed=1)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("scaling", sorted(SCALED))
def test_rope_scalings_and_far_positions(layout, scaling):
    pos = torch.tensor([0, 1, 2047, 100000, 999999, 16777217, 2**31 - 1, 5], dtype=torch.int32, device=DEV)
    print("case rope far", layout, scaling, flush=True)
    _check(8, 3, 128, 128, layout, scaling, "f32", amplitude=1.3465736, pos=pos)
    _check(8, 3, 64, 32, layout, scaling, "bf16", amplitude=0.75, pos=pos, in_place=True)


def test_rope_leaves_out_negative_positions():
    pos = torch.tensor([4, -1, 0, -2**31, 7], dtype=torch.int32, device=DEV)
    for in_place in (False, True):
        _check(5, 2, 64, 48, "half", pos=pos, in_place=in_place)
    _check(5, 2, 64, 48, "interleaved", pos=torch.full((5,), -1, dtype=torch.int32, device=DEV))


def test_rope_many_rows():
    print("case rope 20011 rows", flush=True)
    _check(20011, 2, 64, 64, "half")
    _check(4097, 5, 128, 64, "interleaved", dtype="f32")


def test_rope_nonfinite_stays_in_its_pair():
    m = U.amd()
    rope = m.make_rope(64, 32, "half", "bf16")
    x = torch.ones((2, 128), dtype=torch.bfloat16, device=DEV)
    x[0, 3], x[1, 64 + 20] = float("nan"), float("inf")
    out = torch.zeros_like(x)
    m.moe_rope(rope, x, m.moe_rope_frequencies(rope, DEV), torch.tensor([3, 9], dtype=torch.int32, device=DEV), out)
    bad = ~torch.isfinite(out)
    assert sorted(map(tuple, bad.nonzero().tolist())) == [(0, 3), (0, 19), (1, 64 + 4), (1, 64 + 20)]


@pytest.mark.parametrize("heads,dh", [(1, 64), (3, 128), (2, 8)])
def test_rope_several_rows_per_work_group(heads, dh):
    pos = torch.randint(-3, 9000, (16387,), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV, dtype=torch.int32)
    print("case rope rows", heads, dh, flush=True)
    _check(16387, heads, dh, dh, "half", pos=pos, before=8)
    _check(16387, heads, dh, 8, "interleaved", dtype="f32", pos=pos, in_place=True, behind=4)


def test_rope_captured():
    m = U.amd()
    rope = m.make_rope(64, 64, "half", "bf16", scaling="linear", factor=3.0)
    turns, pos = m.moe_rope_frequencies(rope, DEV), torch.arange(9, dtype=torch.int32, device=DEV)
    x = torch.randn((9, 256), device=DEV).to(torch.bfloat16)
    out = torch.zeros_like(x)
    m.moe_rope(rope, x, turns, pos, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.moe_rope(rope, x, turns, pos, out)
    for _ in range(3):
        pos.add_(1000)
        x.mul_(-1.5)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        m.moe_rope(rope, x, turns, pos, out)
        assert torch.equal(got, out)


@pytest.mark.parametrize("layout,dh,rot,dtype", [("half", 128, 128, "bf16"), ("half", 64, 24, "bf16"), ("interleaved", 64, 16, "bf16"), ("half", 64, 64, "f32")])
def test_rope_many_rows(layout, dh, rot, dtype):
    """Rows enough for the stores of large calls: the same bits as in small calls, in place and into another tensor."""
    m = U.amd()
    n, heads = (1 << 24) // (8 * dh) + 5, 8
    rope = m.make_rope(dh, rot, layout, dtype)
    turns = m.moe_rope_frequencies(rope, DEV)
    gen = torch.Generator(device=DEV).manual_seed(2)
    x = torch.randn((n, heads * dh), generator=gen, device=DEV).to(torch.float32 if dtype == "f32" else torch.bfloat16)
    pos = torch.randint(-2, 100000, (n,), generator=gen, device=DEV, dtype=torch.int32)
    print("case rope many", layout, dh, rot, dtype, flush=True)
    out, want = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    m.moe_rope(rope, x, turns, pos, out)
    for a in range(0, n, n // 2 + 1):
        m.moe_rope(rope, x[a:a + n // 2 + 1], turns, pos[a:a + n // 2 + 1].clone(), want[a:a + n // 2 + 1])
    assert torch.equal(out, want)
    want = torch.where((pos < 0)[:, None], x, want)
    m.moe_rope(rope, x, turns, pos, x)
    assert torch.equal(x, want)
