"""Norm and rotation at the ends of what the header allows."""
import pytest
import torch

from oracle import attention_oracle as orc
from paper_2602_19362_amd import oapl
from tests.test_gpu_norm_rope import DEV, _gen, _inputs, _near

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
