"""Every form of the three attention kernels (tiles of 32, 64 and 128 rows or keys, walks whole and in parts) in either type and at every
compiled width.  Which form a case's sizes lead to is asserted on the host, in tests/test_attention_plan.py."""
import math

import pytest
import torch

from tests.test_gpu_attention import _check
from tests.test_gpu_attention import test_what_is_not_finite_among_many_tiles as check_reach

pytestmark = pytest.mark.gpu

RAGGED = [(7 * i * i + i) % 97 for i in range(66)]      # 66 sequences: more than one wavefront orders by length

# dtype, queries, keys, query heads, key heads, channels, mask, and what the sizes lead to: rows (keys) of a tile, parts (0: one, 1: several)
CASES = [
    ("bf16", [50], [50], 8, 1, (24, 64, 80, 128), True, {"fwd": 32, "dq": 32, "dkdv": 32, "dkdv_parts": 1}),
    ("bf16", [3, 2], [1500, 2000], 8, 2, (24, 64, 80, 128), True, {"fwd": 32, "fwd_parts": 1, "dq": 32, "dq_parts": 1}),
    ("bf16", [1500], [1500], 32, 8, (24, 64, 80, 128), True, {"fwd": 64, "fwd_parts": 0, "dkdv": 64, "dkdv_parts": 1}),
    ("bf16", [700, 500], [650, 550], 24, 8, (24, 64, 80, 128), True, {"dq": 64, "dq_parts": 0}),
    ("bf16", [2500], [2500], 8, 8, (24, 64), True, {"fwd": 128, "fwd_parts": 1}),
    ("bf16", [2500], [2500], 8, 8, (80, 128), False, {"fwd": 128, "fwd_parts": 1}),
    ("bf16", [4000], [4000], 8, 8, (64, 128), True, {"dq": 128, "dq_parts": 1}),
    ("bf16", [4000], [4000], 8, 8, (24, 80), False, {"dq": 128, "dq_parts": 1}),
    ("bf16", [50], [45], 8, 8, (24, 64, 80, 128), True, {"dkdv": 32, "dkdv_parts": 0}),
    ("bf16", RAGGED, RAGGED[::-1], 8, 8, (24, 64), True, {"dkdv": 64, "dkdv_parts": 0}),
    ("bf16", [60, 40, 50, 51], [50, 57, 43, 51], 64, 64, (80, 128), True, {"dkdv": 64, "dkdv_parts": 0}),
    ("bf16", [1200], [1200], 48, 8, (24, 64), False, {"dkdv": 64, "dkdv_parts": 1}),
    ("bf16", RAGGED, RAGGED[::-1], 32, 32, (24, 64), True, {"fwd": 128, "fwd_parts": 0, "dq": 128, "dq_parts": 0, "dkdv": 128}),
    ("bf16", RAGGED, RAGGED[::-1], 16, 8, (80, 128), True, {"fwd": 128, "fwd_parts": 0, "dq": 128, "dq_parts": 0, "dkdv": 128}),
    ("bf16", [1300, 1000], [1200, 1150], 64, 64, (24, 64), True, {"dkdv": 128, "dkdv_parts": 0}),
    ("bf16", [1100, 1050], [1150, 1000], 32, 32, (80, 128), True, {"dkdv": 128, "dkdv_parts": 0}),
    ("f32", [50], [45], 8, 8, (24, 64, 80, 128), True, {"dkdv": 32, "dkdv_parts": 0}),
    ("f32", [50], [50], 8, 1, (24, 64, 80, 128), True, {"fwd": 32, "dq": 32, "dkdv": 32, "dkdv_parts": 1}),
    ("f32", [3, 2], [1500, 2000], 8, 2, (24, 64, 80, 128), True, {"fwd": 32, "fwd_parts": 1, "dq": 32, "dq_parts": 1}),
    ("f32", RAGGED, RAGGED[::-1], 32, 8, (24, 64, 80, 128), True, {"fwd": 128, "fwd_parts": 0, "dq": 128, "dq_parts": 0}),
    ("f32", [1200], [1200], 48, 8, (24, 64, 80, 128), True, {"dkdv": 128, "dkdv_parts": 1}),
    ("f32", [1000, 900], [950, 1000], 64, 64, (24, 64, 80, 128), True, {"dkdv": 128, "dkdv_parts": 0}),
    ("f32", [4000], [4000], 12, 2, (24, 80), True, {"dq": 128, "dq_parts": 1}),
    ("f32", [4000], [4000], 12, 2, (64, 128), False, {"dq": 128, "dq_parts": 1}),
]

# dtype, tokens, query heads, key heads, channels, what they lead to
REACH = [
    ("bf16", 2200, 32, 32, 128, {"dkdv": 128, "dkdv_parts": 0, "dq": 128, "fwd": 128}),
    ("bf16", 2400, 64, 64, 64, {"dkdv": 128, "dkdv_parts": 0, "dq": 128, "fwd": 128}),
    ("bf16", 1500, 32, 8, 128, {"dkdv": 64, "dkdv_parts": 1, "dq": 64, "fwd": 64}),
    ("bf16", 2500, 8, 8, 64, {"fwd": 128, "fwd_parts": 1}),
    ("f32", 1200, 64, 64, 80, {"dkdv": 128, "dkdv_parts": 0, "dq": 128, "fwd": 128}),
]


@pytest.mark.parametrize("dtype, nq, nk, hq, hk, D, causal", [(*c[:5], D, c[6]) for c in CASES for D in c[5]])
def test_forms(dtype, nq, nk, hq, hk, D, causal):
    _check(dtype, nq, nk, hq, hk, D, causal, seed=500)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("dtype, n, hq, hk, D", [c[:5] for c in REACH])
def test_what_is_not_finite_by_form(dtype, bad, n, hq, hk, D):
    check_reach(dtype, bad, n, hq, hk, D)
    torch.cuda.empty_cache()
