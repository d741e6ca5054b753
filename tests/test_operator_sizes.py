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


FAKE = 0x1000   # never dereferenced: refused first


def _norm(n, pixels, c, groups, dtype=B.F16, stride=None):
    return B.NormDesc(n, pixels, c, groups, dtype, 0, stride or c, stride or c, 1e-5)


def _calls(d):
    L = B.lib()
    return (L.cprune_group_norm_act(d, FAKE, None, None, FAKE, None, None, FAKE, 1 << 60, None),
            L.cprune_group_norm_act_backward(d, FAKE, FAKE, FAKE, FAKE, None, None, FAKE, FAKE, FAKE, FAKE, 1 << 60, None))


@pytest.mark.parametrize("dtype", [B.F32, B.F16, B.BF16])
def test_the_most_pixels_are_counted(dtype):
    """A superrow of one channel is four or eight pixels: the last ones begin a superrow more."""
    L = B.lib()
    for back in (0, 1):
        whole = L.cprune_group_norm_workspace_bytes(_norm(1, 2 ** 31 - 8, 1, 1, dtype), back)
        assert whole > 0
        for pixels in (2 ** 31 - 7, 2 ** 31 - 3, 2 ** 31 - 1):
            assert L.cprune_group_norm_workspace_bytes(_norm(1, pixels, 1, 1, dtype), back) >= whole


@pytest.mark.parametrize("d", [(1, 1, 2 ** 31 - 1, 1), (1, 1, 2 ** 31 - 255, 1), (1, 1, 2 ** 29 + 1, 1), (1, 1, 2 ** 28 + 1, 1), (1, 2, 2 ** 27 + 4, 2)])
def test_channels_past_what_a_launch_holds(d):
    """(scratch asked for a call that is refused: 1.8e19 bytes at the first)"""
    for dtype in (B.F16, B.BF16) + ((B.F32,) if d[2] % 4 else ()):
        desc = _norm(*d, dtype)
        assert _calls(desc) == (B.ERR_UNSUPPORTED, B.ERR_UNSUPPORTED)
        assert B.lib().cprune_group_norm_workspace_bytes(desc, 0) == B.lib().cprune_group_norm_workspace_bytes(desc, 1) == 0


def test_gradients_of_too_many_channels_of_several_images():
    """One launch holds the maps; the one that sums 2^29 channels' vectors over the images would take 2^34 threads."""
    d = _norm(2, 1, 2 ** 29, 2 ** 26)
    assert _calls(d)[1] == B.ERR_UNSUPPORTED and B.lib().cprune_group_norm_workspace_bytes(d, 1) == 0


@pytest.mark.parametrize("d", [(2 ** 22, 1, 3, 1, B.F16, 4), (2 ** 21, 2, 3, 3, B.F32, 4), (2 ** 17, 1, 63, 63, B.BF16, 64)])
def test_many_images_of_few_channels_are_taken(d):
    """(image, group) pairs count where a launch has a work-group for each, and these have none"""
    for back in (0, 1):
        assert B.lib().cprune_group_norm_workspace_bytes(_norm(*d), back) > 0
