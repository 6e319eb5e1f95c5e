"""The norm of many tensors and clipping by it against the 64-bit oracle within its error bounds."""
import math

import pytest
import torch

from oracle import blocks_oracle as orc
from paper_2602_19362_amd import oapl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def near(got, want, bound):
    assert got.shape == want.shape
    off = (got.to(torch.float64) - want).abs()
    assert bool((off <= bound + 1e-300).all()), float((off / (bound + 1e-300)).max())


def tensors(sizes, types="mixed", seed=0):
    g = _gen(seed)
    kinds = {"f32": [torch.float32], "bf16": [torch.bfloat16], "mixed": [torch.float32, torch.bfloat16, torch.float32]}[types]
    return [(torch.randn(n, generator=g, device=DEV) * 10.0 ** (i % 5 - 3)).to(kinds[i % len(kinds)]) for i, n in enumerate(sizes)]


SIZES = [[1], [7], [0], [0, 5, 0], [16384], [16383, 16385, 1, 32768], [100003, 12, 3], [256] * 97, [33, 8, 1] * 131, [3000001, 5, 70000],
         # the norm in a launch of its own, from one list and from two; what does not fit the caches
         [17000000, 3], [150001] * 113, [70000001, 2049], [40000000] * 3]


@pytest.mark.parametrize("types", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("sizes", SIZES, ids=[str(len(s)) + "x" + str(max(s)) for s in SIZES])
def test_norm_and_clipping(types, sizes):
    grads = tensors(sizes, types)
    want, bound = orc.grad_norm(grads)
    r = oapl.grad_norm(grads)
    near(r.norm, want.to(DEV), bound.to(DEV))
    for share in (0.3, 2.0):
        most = float(want) * share
        out = [torch.full_like(g, 5.0) for g in grads]
        kept = [g.clone() for g in grads]
        c = oapl.clip_grads(grads, most, out=out, workspace=r.workspace)
        assert torch.equal(c.norm, r.norm)
        for o, g, k, (v, b) in zip(out, grads, kept, orc.clipped(grads, most, want)):
            assert torch.equal(g, k)
            near(o, v, b)
            assert share < 1 or torch.equal(o, g)
        # in place, and by a norm that is given: the same bits
        oapl.clip_grads(kept, most)
        assert all(torch.equal(k, o) for k, o in zip(kept, out))
        kept = [g.clone() for g in grads]
        assert oapl.clip_grads(kept, most, norm=c.norm).workspace is None
        assert all(torch.equal(k, o) for k, o in zip(kept, out))


@pytest.mark.parametrize("n", [2047, 2048, 2049, 2055, 2056, 2057, 4091, 4095, 4096, 4097, 4103, 4104, 6145])
def test_chunks_that_end_inside_two_pieces(n):
    """A lane's two pieces of a chunk, and what is left of it, with the norm in one launch and in its own; the same bits in place."""
    for more in ([], [17000000]):
        for types in ("f32", "bf16"):
            grads = tensors([n] + more, types)
            norm = orc.grad_norm(grads)[0]
            out = [torch.full_like(g, 5.0) for g in grads]
            oapl.clip_grads(grads, float(norm) / 3, out=out)
            for o, (v, b) in zip(out, orc.clipped(grads, float(norm) / 3, norm)):
                near(o, v, b)
            oapl.clip_grads(grads, float(norm) / 3)
            assert all(torch.equal(g, o) for g, o in zip(grads, out))


def test_any_element_of_a_buffer():
    """Tensors that start anywhere, results that start anywhere else; nothing beside them is touched."""
    for dtype in (torch.float32, torch.bfloat16):
        src = torch.randn(60000, generator=_gen(1), device=DEV).to(dtype)
        grads = [src[1:20000], src[20001:20004], src[20007:59999].view(2, -1)]
        dst = torch.full((60010,), 3.0, device=DEV, dtype=dtype)
        out = [dst[3:20002], dst[20005:20008], dst[20009:60001].view(2, -1)]
        norm = orc.grad_norm(grads)[0]
        oapl.clip_grads(grads, float(norm) / 7, out=out)
        for o, (v, b) in zip(out, orc.clipped(grads, float(norm) / 7, norm)):
            near(o, v, b)
        rest = torch.ones(60010, dtype=torch.bool, device=DEV)
        rest[3:20002], rest[20005:20008], rest[20009:60001] = False, False, False
        assert bool((dst[rest] == 3).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", [1e30, 1e-30, 1e-37])
def test_numbers_whose_squares_32_bits_do_not_hold(dtype, size):
    grads = [(torch.randn(5000, generator=_gen(i), device=DEV) * size).to(dtype) for i in range(3)]
    want, bound = orc.grad_norm(grads)
    near(oapl.grad_norm(grads).norm, want, bound + 2.0 ** -150)
    for most in (float(want) / 3, 1e-38):
        out = [torch.empty_like(g) for g in grads]
        oapl.clip_grads(grads, most, out=out)
        most = torch.tensor(most, dtype=torch.float32).item()
        for o, (v, b) in zip(out, orc.clipped(grads, most, want)):
            near(o, v, b)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_what_is_not_finite_shows_in_the_norm_and_is_not_spread(bad):
    grads = tensors([3000, 20, 17000])
    grads[2][16500] = bad
    kept = [g.clone() for g in grads]
    r = oapl.clip_grads(grads, 1e-3)
    assert not bool(r.norm.isfinite().any()) and bool(r.norm.isnan().all()) == math.isnan(bad)
    for g, k in zip(grads, kept):
        assert torch.equal(torch.nan_to_num(g, nan=7.0), torch.nan_to_num(k, nan=7.0))


def test_a_norm_of_zero():
    grads = [torch.randn(100, generator=_gen(3), device=DEV)]
    oapl.clip_grads(grads, 0.0)
    assert bool((grads[0] == 0).all())
    assert oapl.clip_grads(grads, 0.0).norm.item() == 0 and bool((grads[0] == 0).all())


def test_the_list_may_go_when_the_call_returns():
    """More tensors than one launch takes, the list's memory used for something else right away."""
    grads = tensors([5000 + i for i in range(300)])
    wants = []
    for k in range(4):
        mine = grads[k * 50:k * 50 + 120]
        wants.append((oapl.grad_norm(mine).norm, orc.grad_norm(mine)))
    for got, (want, bound) in wants:
        near(got, want, bound)


@pytest.mark.parametrize("count", [1, 112, 113, 300])
def test_nothing_beside_the_workspace_is_touched(count):
    n = oapl.clip_workspace_bytes(count)
    room = torch.full((n + 512,), 0x5a, dtype=torch.uint8, device=DEV)
    grads = tensors([3000] * count)
    near(oapl.clip_grads(grads, 1e-3, workspace=room[256:256 + n]).norm, *orc.grad_norm(tensors([3000] * count)))
    assert bool((room[:256] == 0x5a).all()) and bool((room[256 + n:] == 0x5a).all())


def test_refusals():
    a, b = torch.zeros(8, device=DEV), torch.zeros(9, device=DEV)
    for call in (lambda: oapl.grad_norm([]), lambda: oapl.clip_grads([a, b], 1.0, out=[a]), lambda: oapl.clip_grads([a], 1.0, out=[b]),
                 lambda: oapl.grad_norm([a[::2]]), lambda: oapl.grad_norm([a, a.cpu()]), lambda: oapl.clip_grads([a], 1.0, norm=b)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: oapl.grad_norm([a.half()]), lambda: oapl.grad_norm([a.long()]), lambda: oapl.clip_grads([a], 1.0, out=[a.bfloat16()]),
                 lambda: oapl.clip_grads([a], 1.0, norm=a[:1].double())):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: oapl.clip_grads([a], -1.0), lambda: oapl.clip_grads([a], math.nan), lambda: oapl.clip_grads([a, a], 1.0),
                 lambda: oapl.clip_grads([a, b], 1.0, out=[b[:8], a.new_zeros(9)]), lambda: oapl.clip_grads([b[:8]], 1.0, out=[b[1:]]),
                 lambda: oapl.grad_norm([a], workspace=torch.zeros(256, device=DEV, dtype=torch.uint8))):
        with pytest.raises(oapl.OaplError):
            call()
