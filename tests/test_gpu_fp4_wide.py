"""The 4-bit quantiser on a row too long for registers and for 32-bit offsets of its scales' bytes."""
import pytest

pytestmark = pytest.mark.gpu


def test_a_very_long_row():
    """2^28 + 77 columns: their codes are 134 MB, their scale tiles 2.1 GB; the far end is compared with the same numbers quantised alone."""
    import torch
    from paper_2510_01565_b200 import binding as B
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 8 GB")
    cols, tail = 2 ** 28 + 77, 64 * 1000 + 77
    x = torch.zeros(1, cols, dtype=torch.float16, device="cuda")
    x[0, -tail:] = torch.randn(tail, generator=torch.Generator().manual_seed(1)).half().cuda()
    codes, scales, rows = B.dit_quantize_fp4(x)
    end = B.dit_quantize_fp4(x[:, -tail:].contiguous())
    assert torch.equal(rows, end[2]) and torch.equal(codes[:, -end[0].shape[1]:], end[0]) and not codes[:, :-end[0].shape[1]].any()
    assert torch.equal(scales[:, -end[1].shape[1]:], end[1])
    back = B.dit_dequantize_fp4(codes, scales, cols, 16, rows)
    assert torch.equal(back[:, -tail:], B.dit_dequantize_fp4(end[0], end[1], tail, 16, end[2])) and not back[:, :-tail].any()
