"""Attention at scales other than 1 / sqrt(D): queries that were scaled beforehand (scale 1), sharp and negative ones, rows that see nothing
of a step, and both ends of the range.  Against the 64-bit oracle, within its error bounds."""
import math

import pytest
import torch

from oracle import attention_oracle as orc
from paper_2602_19362_amd import oapl
from tests.test_gpu_attention import DEV, DTYPES, _check, _near, _normal, _offsets, _qkv

pytestmark = pytest.mark.gpu

# Heads (query, key, channels) and lengths whose rows see nothing of a step that their tile walks over.
SIZES = [
    ("bf16", [600], [600], 32, 8, 128),             # tiles of 64 rows: the first 32 tokens see none of the second half of the first keys
    ("bf16", [1500], [1500], 32, 8, 128),
    ("bf16", [50], [90], 1, 1, 64),                 # tiles of 32 rows: n_k - n_q is no multiple of a step
    ("bf16", [50, 3], [90, 17], 7, 1, 64),
    ("f32", [50, 3], [90, 17], 7, 1, 64),
    ("bf16", [90, 9, 33], [50, 5, 0], 4, 2, 64),    # fewer keys than queries: rows that see nothing beside rows that do
    ("f32", [90, 9, 33], [50, 5, 0], 4, 2, 64),
    ("bf16", [2500], [2500], 8, 1, 128),            # keys split over workgroups
    ("bf16", [64] * 16, [2000] * 16, 8, 8, 128),
    ("f32", [4, 2], [700, 1500], 8, 2, 64),
    ("f32", [2500], [2400], 8, 1, 64),
    ("bf16", [1000, 500], [700, 900], 48, 8, 64),   # tiles of 128 rows
    ("f32", [1000, 800], [700, 900], 16, 8, 80),
]


@pytest.mark.parametrize("scale", [1.0, -1.0, 4.0, -2.0])
@pytest.mark.parametrize("dtype, nq, nk, hq, hk, D", SIZES)
def test_scales(dtype, nq, nk, hq, hk, D, scale):
    _check(dtype, nq, nk, hq, hk, D, True, scale=scale, seed=300)


@pytest.mark.parametrize("scale", [1.0, -3.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales_without_a_mask(dtype, scale):
    _check(dtype, [70, 500], [33, 500], 8, 2, 64, False, scale=scale, seed=310)


@pytest.mark.parametrize("scale, spread", [(1e30, 1e-30), (-1e20, 1e-20), (1e-30, 1e20)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales_far_from_one(dtype, scale, spread):
    """Scores of ordinary size (or far below one) from queries that are not."""
    _check(dtype, [90, 40], [50, 97], 4, 2, 64, True, scale=scale, seed=320, spread=spread)
    _check(dtype, [600], [600], 16, 8, 64, True, scale=scale, seed=323, spread=spread, grads=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_cache_with_queries_scaled_beforehand(dtype):
    """Several new tokens over a cache: their reach ends within a step of the keys."""
    hq, hk, D, room, used = 8, 2, 128, 300, [5, 300, 0, 67, 128, 250]
    nq = [5, 3, 2, 7, 33, 1]
    q, k, v = _qkv(dtype, nq, [room] * 6, hq, hk, D, seed=330)
    q = (q.float() * D ** -0.5).to(DTYPES[dtype])
    ko, n = _offsets([room] * 6), torch.tensor(used, device=DEV)
    for scale in (1.0, 8.0):
        r = oapl.attention_fwd(q, k, v, _offsets(nq), ko, k_used=n, scale=scale)
        out, lse, bound, lse_bound = orc.attention(q, k, v, _offsets(nq), ko, causal=True, scale=scale, k_used=n)
        _near(r.out, out, bound)
        _near(r.lse, lse, lse_bound)
        assert not r.out[8:10].any() and bool((r.lse[8:10] == -math.inf).all())
