"""moe_rope with as many rows as it takes."""
import ctypes

import pytest
import torch

from tests import gpu_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_rope_2_24_wide_rows():
    """Rows so wide that each has a work-group of its own.  All but the first 16 are left out, so that only those need memory."""
    m = U.amd()
    heads, dh, rows, live = 32, 128, 1 << 24, 16
    rope = m.make_rope(dh, dh, "half", "bf16")
    turns = m.moe_rope_frequencies(rope, DEV)
    x = torch.randn((live, heads * dh), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).to(torch.bfloat16)
    out, want = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    pos = torch.full((rows,), -1, dtype=torch.int32, device=DEV)
    pos[:live:2] = torch.arange(live // 2, dtype=torch.int32, device=DEV) * 1000
    m.moe_rope(rope, x, turns, pos[:live].clone(), want)
    print("case rope", rows, "rows of", heads, "heads", flush=True)
    rc = m.load_library().moe_rope(ctypes.byref(rope), rows, heads, x.data_ptr(), heads * dh, turns.data_ptr(), pos.data_ptr(), out.data_ptr(), heads * dh,
                                   torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert rc == 0
    assert torch.equal(out, want) and bool((out[1::2] == 7.0).all())
