"""Limits of the entry points for several new tokens per sequence, on the CPU: nothing is launched, so pointers are made up."""
import pytest
import torch

from paper_2201_05596_amd import binding as B
from tests.test_draft_refusals import FakeDevice, block_call, cache_shape


def test_draft_block_rows():
    """Fewer than 2^24 rows: the LayerNorms take a work-group of 256 threads for each, and a grid has fewer than 2^32."""
    sizes = dict(n_seq=1 << 16, n_heads=1, n_kv_heads=1, head_dim=64)
    shape = dict(T=1 << 24, d_model=64, d_ffn=64, E=4, top_k=1, capacity=1 << 22)
    assert block_call(shape=shape, c=sizes, n=256) == -2
    most = B.make_shape(1 << 24, 64, 64, 4, 1, 1 << 22, "bf16")
    assert B.moe_draft_block_workspace_bytes(most, cache_shape(**sizes), 256) == 0
    fewer = dict(sizes, n_seq=(1 << 16) - 1)
    assert B.moe_draft_block_workspace_bytes(B.make_shape((1 << 24) - 256, 64, 64, 4, 1, 1 << 22, "bf16"), cache_shape(**fewer), 256) > 0


def test_binding_rope_without_a_head(monkeypatch):
    """A head of no dimensions is the library's to refuse, as every other shape."""
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 0, raising=False)
    rows = FakeDevice((5, 128), torch.bfloat16)
    for head_dim in (0, -8):
        with pytest.raises(B.MoeError):
            B.moe_rope(B.make_rope(head_dim, 64, "half", "bf16"), rows, FakeDevice((32,), torch.float64), FakeDevice((5,), torch.int32), rows)
