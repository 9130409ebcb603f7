"""What vfl_softmax_loss_workspace_size asks for, against what the calls lay out there."""
import pytest

from paper_2510_12494_amd import vfl as V


@pytest.mark.parametrize("dtype,e", [(V.VFL_F32, 4), (V.VFL_BF16, 2)])
@pytest.mark.parametrize("rows,dim,classes", [(1, 64, 100_000), (16, 1024, 2**21), (16, 1024, 2**18), (40, 4096, 2**19), (48, 250, 2**20),
                                              (3, 32768, 2**16)])
def test_gradients_of_weights_that_are_written_at_once_take_no_sums(dtype, e, rows, dim, classes):
    """Few rows are one part of dw's sum: the operands' copies (of x twice, in rows of whole
    tiles), a piece of G, dx's sums of at most 4 full rounds of the largest tiles (256 CUs of
    256 x 256 results), sums of dbias and the forward's pairs, and no float32 dw."""
    wide = -(-dim * e // 128) * 128
    copies = (classes + 2 * 256) * wide
    sums = 4 * 256 * 256 * 256 * 4
    others = (classes + 512) * 4 * 2 + (classes // 64 + 1) * rows * 8
    assert copies <= V.vfl_softmax_loss_workspace_size(dtype, rows, dim, classes) + 512 * wide
    assert V.vfl_softmax_loss_workspace_size(dtype, rows, dim, classes) <= copies + (1 << 30) + sums + others + (1 << 20)
