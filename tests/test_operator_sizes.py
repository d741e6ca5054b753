"""Sizes that 32 bits do not hold are refused, not cut down to what they leave of them; needs no GPU and no memory."""
import pytest
import torch

from paper_2207_01260_amd import binding as B


class OnDevice(torch.Tensor):
    """(the checks of sizes stand behind the one that asks where a tensor is)"""
    is_cuda = True


@pytest.mark.parametrize("shape", [(1, 2 ** 32 + 9, 1), (2 ** 32 + 1, 4, 8), (2, 3, 2 ** 32 + 16), (2 ** 16, 2 ** 15, 1), (1, 2 ** 31)])
def test_dense_sizes(shape):
    x = torch.empty(shape, dtype=torch.float16, device="meta")
    for image_dims in (0, 1):
        with pytest.raises(ValueError, match="2.31"):
            B._rows_of(x, image_dims)
    assert B._rows_of(torch.empty(1, 2 ** 31 - 1, device="meta"), 0) == (1, 1, 2 ** 31 - 1, 2 ** 31 - 1)


def test_sizes_with_gaps():
    x = torch.empty(4, 2 ** 32 + 8, device="meta")
    for part in (x[:, :8], x[:3, :5], torch.empty(2 ** 20, 2 ** 11, device="meta")[:, :3]):
        with pytest.raises(ValueError, match="2.31"):
            B._rows_of(part, 0)
    assert B._rows_of(torch.empty(2 ** 20, 2 ** 11 - 1, device="meta")[:, :3], 0) == (1, 2 ** 20, 3, 2 ** 11 - 1)


def test_codes_and_groups():
    for rows, blocks in ((2 ** 32 + 4, 1), (1, 2 ** 27 + 1), (2 ** 16, 2 ** 10)):
        codes = torch.empty(rows, 16 * blocks, dtype=torch.uint8, device="meta")
        scales = torch.empty(rows, blocks, dtype=torch.uint8, device="meta")
        with pytest.raises(ValueError, match="2.31"):
            B._mx4_pair(codes, scales, None)
    with pytest.raises(ValueError, match="groups"):
        B._norm_desc(torch.empty(2, 3, 8).as_subclass(OnDevice), 2 ** 32 + 2, 0, 1e-5)
    assert B._norm_desc(torch.empty(2, 3, 8).as_subclass(OnDevice), 2, 0, 1e-5).groups == 2
