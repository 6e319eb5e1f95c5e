"""Sums over many tokens in the residual norm's gradients."""
import pytest
import torch

from paper_2602_19362_amd import oapl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F = torch.float64
U32 = 2.0 ** -24


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


# A wavefront and fewer a row, a workgroup a row, several rows a workgroup slot.
@pytest.mark.parametrize("types", ["bf16", "f32", "mixed"])
@pytest.mark.parametrize("T, d", [(1, 24), (9001, 24), (70001, 40), (2500, 300), (20003, 513), (1501, 768), (5003, 4096), (777, 5120), (1031, 8192), (600, 10000)])
def test_sums_of_whole_numbers(types, T, d):
    """Channels of +-1 have a norm of one without eps, and a gain of zero leaves the norm no part in dX: the sums are of whole numbers below
    2^24, none of them zero, and a row that is missing or there twice shows in every channel."""
    tx, t = {"bf16": (torch.bfloat16,) * 2, "f32": (torch.float32,) * 2, "mixed": (torch.float32, torch.bfloat16)}[types]

    def whole(seed, most, dtype):
        sign = torch.randint(0, 2, (T, d), generator=_gen(seed), device=DEV) * 2 - 1
        return (sign * torch.randint(1, most + 1, (T, d), generator=_gen(seed + 1), device=DEV)).to(dtype)

    x, y, dx_out, dout = whole(1, 1, tx), whole(3, 1, t), whole(5, 7, tx), whole(7, 7, t)
    # mostly of the sign that makes a sum grow
    grows = torch.rand(T, 1, generator=_gen(9), device=DEV) < 0.8
    dout = torch.where(grows, dout.abs() * x.to(t), dout)
    dx_out = torch.where(grows, dx_out.abs() * y.to(tx), dx_out)
    zero, one = torch.zeros(d, device=DEV, dtype=t), torch.ones(d, device=DEV, dtype=t)
    r = oapl.residual_norm_bwd(x, y, dx_out, dout, zero, y_gain=one, gate=one, eps=0.0)
    want = (dout.long() * x.long()).sum(0), (dx_out.long() * y.long()).sum(0)
    assert 7 * T < 1 << 24
    assert torch.equal(r.dgain, want[0].float())
    assert torch.equal(r.dy_gain, want[1].float()) and torch.equal(r.dgate, want[1].float())
    assert torch.equal(r.dx, dx_out)


@pytest.mark.parametrize("T, d", [(65535 * 256, 129), (65535 * 256, 40), (3000000, 520)])
def test_long_sums(T, d):
    """One row for all tokens, whose part of the sum is rounded in the same direction again and again.  A part is off by 70 roundings (64
    of one over the root, as sums of up to 64 lanes and 16 of each are, the products, the mean); adding up takes as many as rows follow each other in 32 bits, 1024,
    and a workgroup's up to 16; the rest is in 64 bits and rounded once.  All parts have one sign, so each rounding is one of no more than the sum."""
    x, dout = (torch.randn(1, d, generator=_gen(i), device=DEV) for i in (1, 2))
    gain = torch.randn(d, generator=_gen(3), device=DEV)
    r = oapl.residual_norm_bwd(x.expand(T, d), None, None, dout.expand(T, d), gain)
    want = T * (dout.to(F) * x.to(F) / torch.sqrt(x.to(F).pow(2).mean() + 1e-6))[0]
    off = (r.dgain.to(F) - want).abs() / (U32 * want.abs())
    assert float(off.max()) <= 70 + 1024 + 16 + 1, float(off.max())
    # and no row behind the first launch's is another one
    assert torch.equal(r.dx, r.dx[:1].expand(T, d))
