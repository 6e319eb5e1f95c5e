"""The ends of the sizes and numbers that the attention entry points take: refused on the host, before anything is launched."""
import pytest

from paper_2602_19362_amd import oapl
from tests.test_attention_abi import AT, BETA, SHAPE, H, fwd


@pytest.mark.parametrize("scale", [2.4e38, -3e38])
def test_a_scale_that_is_infinite_in_base_2_is_refused(scale):
    """Scores are scaled by scale * log2(e) on the device."""
    assert fwd(scale=scale) == BETA
    assert oapl.lib().oapl_attention_bwd(H(), H(), H(), H(), AT, H(), AT, AT, 4, 4, 1, 2, 1, 64, 1, 1, scale, H(), H(), H(), AT, 1 << 24,
                                         None) == BETA


# HIP takes fewer than 2^32 threads in a dimension of a grid, a tile is a workgroup of 256, and a sequence has a tile at least.
@pytest.mark.parametrize("n, hk", [(1 << 24, 1), (1 << 21, 8), (1 << 8, 1 << 16), ((1 << 23) + 1, 2)])
def test_more_tiles_than_a_launch_takes_are_refused(n, hk):
    assert fwd(n=n, hq=hk, hk=hk, D=8) == SHAPE
    assert oapl.lib().oapl_attention_bwd(H(), H(), H(), H(), AT, H(), AT, AT, 4, 4, n, hk, hk, 8, 1, 1, 0.1, H(), H(), H(), AT, 1 << 30,
                                         None) == SHAPE
    for with_backward in (0, 1):
        assert oapl.attention_workspace_bytes(4, 4, n, hk, hk, 8, 1, with_backward) == 0


def test_long_caches_and_many_sequences_are_served():
    """A cache's capacity is no part of a forward launch; 2^20 sequences of 8 heads are half of what one takes."""
    assert oapl.attention_workspace_bytes(8, 1 << 27, 8, 64, 64, 128, 1, False) > 0
    assert oapl.attention_workspace_bytes(1 << 20, 1 << 20, 1 << 20, 8, 8, 64, 1, True) > 0


@pytest.mark.parametrize("hq, head", [(65536, 1 << 48), (1 << 15, 1 << 48), (3, 1 << 48), (65536, 1 << 47), (2, (1 << 29) + 8)])
def test_a_group_further_apart_than_32_bit_offsets_reach_is_refused(hq, head):
    """The span of a group's heads is compared without being multiplied out of 64 bits."""
    for q, dout in ((H(AT, 128, head), H()), (H(), H(AT, 128, head))):
        assert oapl.lib().oapl_attention_bwd(q, H(), H(), H(), AT, dout, AT, AT, 4, 4, 1, hq, 1, 64, 1, 1, 0.1, H(), H(), H(), AT, 1 << 40,
                                             None) == SHAPE
