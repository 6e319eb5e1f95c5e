"""NaN and infinities in keys, values, queries and gradients: where they reach, and where not."""
import math

import pytest

from tests.test_gpu_attention import test_what_is_not_finite_among_many_tiles as check_reach

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("n, hq, hk, D", [(150, 32, 1, 64), (40, 64, 2, 128), (150, 130, 1, 32), (700, 130, 1, 64), (1000, 130, 1, 64),
                                          (600, 128, 1, 128)])
def test_tiles_whose_rows_are_all_of_one_token(dtype, bad, n, hq, hk, D):
    """Groups of as many heads as a tile has rows, and more: the step that ends a token's reach holds keys behind it."""
    check_reach(dtype, bad, n, hq, hk, D)
