"""NaN and infinities in keys, values, queries and gradients: where they reach, and where not."""
import math

import pytest
import torch

from paper_2602_19362_amd import oapl
from tests.test_gpu_attention import DEV, _offsets, _qkv
from tests.test_gpu_attention import test_what_is_not_finite_among_many_tiles as check_reach

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("n, hq, hk, D", [(150, 32, 1, 64), (40, 64, 2, 128), (150, 130, 1, 32), (700, 130, 1, 64), (1000, 130, 1, 64),
                                          (600, 128, 1, 128)])
def test_tiles_whose_rows_are_all_of_one_token(dtype, bad, n, hq, hk, D):
    """Groups of as many heads as a tile has rows, and more: the step that ends a token's reach holds keys behind it."""
    check_reach(dtype, bad, n, hq, hk, D)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("nq, nk, hq, hk, D", [([150], [150], 4, 2, 64), ([9, 40], [30, 77], 8, 1, 128), ([1300, 900], [1300, 900], 16, 8, 64),
                                               ([1000, 500], [700, 900], 48, 8, 64), ([2500], [2500], 8, 1, 128)])
def test_a_value_that_is_not_finite_is_no_part_of_the_log_sum_exp(dtype, bad, nq, nk, hq, hk, D):
    q, k, v = _qkv(dtype, nq, nk, hq, hk, D, seed=340)
    qo, ko = _offsets(nq), _offsets(nk)
    want = oapl.attention_fwd(q, k, v, qo, ko)
    for at in (0, nk[0] // 2, nk[0] - 1):
        x = v.clone()
        x[at, 0, 3] = bad
        got = oapl.attention_fwd(q, k, x, qo, ko)
        assert torch.equal(got.lse, want.lse)
        # the rows that see it are not finite in its channel, all others are what they were
        sees = torch.arange(nq[0], device=DEV) >= at - (nk[0] - nq[0])
        group = slice(0, hq // hk)
        assert not bool(got.out[:nq[0]][sees][:, group, 3].isfinite().any())
        assert torch.equal(got.out[:nq[0]][~sees], want.out[:nq[0]][~sees]) and torch.equal(got.out[nq[0]:], want.out[nq[0]:])
        assert torch.equal(got.out[:, hq // hk:], want.out[:, hq // hk:])
