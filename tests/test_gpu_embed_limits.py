"""The embedding's gradient in numbers that are sums of whole ones below 2^24, so that every bit is known."""
import pytest
import torch

from paper_2602_19362_amd import oapl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_gradient_in_more_than_one_row_of_workgroups():
    """2^20 tokens of 65540 channels, all of which have the same row: 1064960 workgroups add rows up, 2^20 of them in a row of the launch.  A
    workspace of 8.6 GB."""
    T, d, V = 1 << 20, 65540, 3
    row = torch.randint(1, 8, (1, d), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    tokens = torch.randint(0, V, (T,), generator=torch.Generator(device=DEV).manual_seed(2), device=DEV, dtype=torch.int32)
    got = oapl.embed_bwd(row.bfloat16().expand(T, d), tokens, V).dE
    want = torch.bincount(tokens, minlength=V)[:, None] * row
    assert int(want.max()) < 1 << 24
    assert torch.equal(got, want.float())
