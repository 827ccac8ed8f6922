"""What the binding makes of tensors before the library sees them: distances of single rows, sizes beyond 32 bits."""
import pytest
import torch

from paper_2201_05596_amd import binding as B


@pytest.mark.parametrize("width", [1024, 1032, 2000])
def test_one_row_of_wider_codes(width):
    """Where there is one row there is no distance to the next: any width is as good as the row itself, as it is with more rows of a wider buffer."""
    codes = torch.zeros((1, width), dtype=torch.int8)
    at, stride = B._i8_rows(codes, -1, torch.int8, 1, 1024, "codes")
    assert at == codes.data_ptr() and stride == 1024
    wide = torch.zeros((4, 2048), dtype=torch.int8)[:, :width]
    assert B._i8_rows(wide, -1, torch.int8, 4, 1024, "codes") == (wide.data_ptr(), 2048)


def test_sizes_beyond_32_bits():
    """They are refused, not taken for what is left of them in 32 bits."""
    for size in ((1, (1 << 32) + 64, 128), (1, 64, (1 << 32) + 128), ((1 << 32) + 1, 64, 128), (1 << 31, 64, 128), (1, 64, 128 - (1 << 32))):
        assert B.moe_i8_weights_bytes(*size) == 0, size
    for pack in (B.moe_i8_pack_weights, B.moe_i8_quantize_weights):
        dtype = torch.int8 if pack is B.moe_i8_pack_weights else torch.bfloat16
        with pytest.raises(B.MoeError) as e:
            pack(torch.empty(((1 << 32) + 64, 128), dtype=dtype, device="meta"))
        assert e.value.status == -2
    for shape in ((1, (1 << 32) + 64), ((1 << 32) + 1, 64), (1, 1 << 31)):
        with pytest.raises(B.MoeError) as e:
            B.moe_i8_quantize_rows(torch.empty(shape, device="meta"), None, None)
        assert e.value.status == -2
