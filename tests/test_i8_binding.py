"""What the binding makes of tensors before the library sees them: distances of single rows."""
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
