"""Where the lookup and clipping round, bit by bit: products in 32 or 64 bits, then 32, then the type that is stored."""
import pytest
import torch

from paper_2602_19362_amd import oapl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = [torch.float32, torch.bfloat16]


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("out", DTYPES)
def test_lookup(dtype, out):
    E = torch.randn(999, 264, generator=_gen(1), device=DEV).to(dtype)
    tokens = torch.randint(0, 999, (5000,), generator=_gen(2), device=DEV, dtype=torch.int32)
    scale = torch.tensor(0.7, device=DEV)
    assert torch.equal(oapl.embed_fwd(E, tokens, scale=float(scale), out_dtype=out), (E.float() * scale)[tokens.long()].to(out))


@pytest.mark.parametrize("dtype", DTYPES)
def test_clipping(dtype):
    grads = [torch.randn(n, generator=_gen(n), device=DEV).to(dtype) for n in (70001, 4096, 3)]
    most = torch.tensor(0.37)
    kept = [g.clone() for g in grads]
    norm = oapl.clip_grads(kept, float(most)).norm
    factor = most.double().to(DEV) / norm.double()
    for got, g in zip(kept, grads):
        assert torch.equal(got, (g.double() * factor).float().to(dtype))
