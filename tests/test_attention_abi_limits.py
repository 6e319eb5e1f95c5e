"""The ends of the sizes and numbers that the attention entry points take: refused on the host, before anything is launched."""
import pytest

from paper_2602_19362_amd import oapl
from tests.test_attention_abi import AT, BETA, H, fwd


@pytest.mark.parametrize("scale", [2.4e38, -3e38])
def test_a_scale_that_is_infinite_in_base_2_is_refused(scale):
    """Scores are scaled by scale * log2(e) on the device."""
    assert fwd(scale=scale) == BETA
    assert oapl.lib().oapl_attention_bwd(H(), H(), H(), H(), AT, H(), AT, AT, 4, 4, 1, 2, 1, 64, 1, 1, scale, H(), H(), H(), AT, 1 << 24,
                                         None) == BETA
