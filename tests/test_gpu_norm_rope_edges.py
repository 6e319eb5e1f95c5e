"""Norm and rotation at the ends of what the header allows."""
import math

import pytest
import torch

from oracle import attention_oracle as orc
from paper_2602_19362_amd import oapl
from tests.test_gpu_norm_rope import DEV, _gen, _inputs, _near, _table

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 7, 1500, 5000])
@pytest.mark.parametrize("hq, hk", [(4, 2), (1, 1), (6, 2), (32, 8), (5, 4)])
def test_gradients_without_eps(dtype, T, hq, hk):
    """Few tokens and many, head counts that do and do not fill the wavefronts that share them."""
    q, k, _, pos, table, (gq, gk) = _inputs(dtype, T, hq, hk, 64, 64, True, seed=20)
    dq_out, dk_out = (torch.randn(x.shape, generator=_gen(21), device=DEV).to(x.dtype) for x in (q, k))
    r = oapl.qk_norm_rope_bwd(q, k, dq_out, dk_out, pos, table, gq, gk, eps=0.0)
    for dx, dgain, x, dy, gain in ((r.dq, r.dq_gain, q, dq_out, gq), (r.dk, r.dk_gain, k, dk_out, gk)):
        want, gain_want, bound, gain_bound = orc.norm_rope_grads(x, dy, gain, pos, table, 0.0)
        _near(dx, want, bound)
        _near(dgain, gain_want, gain_bound)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D, rot", [(24, 8), (80, 40), (16, 0), (128, 64)])
def test_what_is_not_finite_stays_in_channels_that_are_not_rotated(dtype, bad, D, rot):
    """Without a norm a channel behind the rotated ones is copied, forward and backward, whatever its neighbours hold."""
    q, k, _, pos, table, _ = _inputs(dtype, 5, 3, 2, D, rot, False, seed=22)
    q, k = q.contiguous(), k.contiguous()
    want = oapl.qk_norm_rope_fwd(q, k, pos, table)
    for c in (rot, rot + 5, D - 1):
        x, y = q.clone(), k.clone()
        x[2, 1, c] = y[3, 0, c] = bad
        others = torch.arange(D, device=DEV) != c
        r = oapl.qk_norm_rope_fwd(x, y, pos, table)
        g = oapl.qk_norm_rope_bwd(q, k, x, y, pos, table)
        back = oapl.qk_norm_rope_bwd(q, k, q, k, pos, table)
        for got, plain, given in ((r.q, want.q, x), (r.k, want.k, y), (g.dq, back.dq, x), (g.dk, back.dk, y)):
            assert torch.equal(got[..., others], plain[..., others])
            assert torch.equal(got[..., rot:].nan_to_num(7.0, 8.0, 9.0), given[..., rot:].nan_to_num(7.0, 8.0, 9.0))


def test_a_position_without_angles_reaches_the_channels_that_are_not_rotated():
    q, k, _, pos, table, (gq, gk) = _inputs("bf16", 6, 4, 2, 64, 32, True, seed=23)
    pos[2] = -1
    got = oapl.qk_norm_rope_fwd(q, k, pos, table, gq, gk)
    back = oapl.qk_norm_rope_bwd(q, k, q, k, pos, table, gq, gk)
    for x in (got.q, got.k, back.dq, back.dk):
        assert bool(x[2].isnan().all()) and bool(x[[0, 1, 3, 4, 5]].isfinite().all())


def test_more_tokens_than_workgroups_in_one_dimension_of_a_grid():
    """2^26 tokens and a few: four of them a workgroup, and HIP takes fewer than 2^32 threads in a dimension."""
    T, D = (1 << 26) + 5, 8
    q, k = (torch.empty(T, 1, D, dtype=torch.bfloat16, device=DEV).normal_(generator=_gen(s)) for s in (24, 25))
    pos = torch.randint(0, 100, (T,), generator=_gen(26), device=DEV, dtype=torch.int32)
    table = _table(100, D)
    r = oapl.qk_norm_rope_fwd(q, k, pos, table)
    for at in (slice(0, 1000), slice(T // 2, T // 2 + 1000), slice(T - 1000, T)):
        part = oapl.qk_norm_rope_fwd(q[at], k[at], pos[at].contiguous(), table)
        assert torch.equal(r.q[at], part.q) and torch.equal(r.k[at], part.k)
    # every token was written: the rotation keeps a head's length (to a rounding of each channel)
    for x, y in ((q, r.q), (k, r.k)):
        for i in range(0, T, 1 << 24):
            a, b = (z[i:i + (1 << 24)].float().square().sum((1, 2)) for z in (x, y))
            assert bool(((a - b).abs() <= 2.0 ** -6 * a).all())
