"""moe_rope on many rows against oracle/draft_oracle.py: several rows per work-group, and the stores of large calls."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as drf
from tests import gpu_util as U
from tests.test_gpu_rope import DEV, _check
from workloads.generate import to_f32_numpy

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,heads,dh,rot,layout,dtype", [(20011, 2, 64, 64, "half", "bf16"), (4097, 5, 128, 64, "interleaved", "f32")])
def test_rope_thousands_of_rows(rows, heads, dh, rot, layout, dtype):
    print("case rope rows", rows, heads, dh, layout, dtype, flush=True)
    _check(rows, heads, dh, rot, layout, dtype=dtype)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("layout,dh,rot,dtype", [("half", 128, 128, "bf16"), ("half", 64, 24, "bf16"), ("interleaved", 64, 16, "bf16"), ("half", 64, 64, "f32"),
                                                 ("interleaved", 128, 128, "f32")])
def test_rope_large_calls_against_the_oracle(layout, dh, rot, dtype, in_place):
    """Elements enough for the stores that go past the caches; some rows of the beginning, the end and between.  The bound is that of
    test_gpu_rope."""
    m = U.amd()
    n, heads = (1 << 24) // (8 * dh) + 5, 8
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    rope = m.make_rope(dh, rot, layout, dtype)
    gen = torch.Generator(device=DEV).manual_seed(6)
    x = torch.randn((n, heads * dh), generator=gen, device=DEV).to(dt)
    pos = torch.randint(-2, 100000, (n,), generator=gen, device=DEV, dtype=torch.int32)
    at = torch.cat((torch.arange(40), torch.randint(40, n - 40, (120,), generator=torch.Generator().manual_seed(7)), torch.arange(n - 40, n))).to(DEV)
    host, p = to_f32_numpy(x[at]).reshape(len(at), heads, dh).astype(np.float64), pos[at].cpu().numpy()
    print("case rope large", layout, dh, rot, dtype, in_place, flush=True)
    out = x if in_place else torch.full_like(x, 7.0)
    m.moe_rope(rope, x, m.moe_rope_frequencies(rope, DEV), pos, out)
    got = to_f32_numpy(out[at]).reshape(host.shape)
    ref = drf.rope(host, p, drf.rope_frequencies(rot, 10000.0), layout)
    size = np.zeros_like(ref)
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    size[..., a] = size[..., b] = np.abs(host[..., a]) + np.abs(host[..., b])
    live = p >= 0
    assert np.all(np.abs(got - ref)[live] <= (torch.finfo(dt).eps / 2 * np.abs(ref) + 2.0 ** -21 * size)[live])
    assert np.array_equal(got[..., rot:][live], host[..., rot:][live])
    assert np.array_equal(got[~live], host[~live] if in_place else np.full_like(got[~live], 7.0))
