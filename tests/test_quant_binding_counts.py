"""Rows and columns that the library's 32-bit counts cannot hold are refused, not cut off to their low 32 bits."""
import pytest

from paper_2601_20655_amd import binding as B

FAR = (1 << 32) + 4  # (whose low 32 bits are 4)


def test_more_rows_or_columns_than_32_bits():
    import torch

    def rows(M, N, dtype):
        return torch.zeros((1, 1), dtype=dtype).expand(M, N)

    f, i8 = torch.float32, torch.int8
    for call in (lambda: B.dit_quant_rows_forward(rows(FAR, 16, f)),
                 lambda: B.dit_quant_rows_forward(rows(4, FAR, f)),
                 lambda: B.dit_rms_norm_quant_forward(rows(FAR, 16, f)),
                 lambda: B.dit_dequant_rows_forward(rows(4, FAR, i8), torch.ones(4)),
                 lambda: B.dit_dequant_rows_forward(rows(1 << 31, 16, i8), torch.ones(1)),
                 lambda: B.dit_linear_quant_forward(rows(FAR, 16, i8), torch.ones(4), rows(8, 16, i8), torch.ones(8)),
                 lambda: B.dit_linear_quant_forward(rows(4, 16, i8), torch.ones(4), rows(FAR, 16, i8), torch.ones(4)),
                 lambda: B.dit_linear_quant_forward(rows(4, FAR, i8), torch.ones(4), rows(8, FAR, i8), torch.ones(8))):
        with pytest.raises(ValueError, match="2147483647"):
            call()


@pytest.mark.gpu
def test_one_row_of_more_than_32_bits():
    """The same on the device, where the call went on with the low 32 bits."""
    import torch

    q = torch.zeros((1, FAR + 12), dtype=torch.int8, device="cuda")
    out = torch.empty((1, FAR + 12), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="2147483647"):
        B.dit_dequant_rows_forward(q, torch.ones(1, device="cuda"), out=out)
