"""The attention oracle against closed forms, library soft-max and finite differences (CPU, 64 bits)."""
import math

import pytest
import torch

from oracle import attention_oracle as orc

F = torch.float64


def _normal(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=F)


def _offsets(lengths):
    return torch.tensor([0] + lengths).cumsum(0)


def _angles(n, rot):
    a = torch.arange(n, dtype=F)[:, None] * 100.0 ** (-torch.arange(0, rot, 2, dtype=F) / max(rot, 1))
    return torch.cat((a.cos(), a.sin()), 1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_unit_is_what_one_rounding_takes(dtype):
    """Numbers half way between two neighbours are off by the unit (nearly, relative to the number itself), others by less."""
    u = orc.store_unit(dtype)
    x = 1 + u * (1 - 2.0 ** -20) * torch.tensor([1.0, -0.25, 3.0], dtype=F)
    off = (x.to(dtype).to(F) - x).abs() / x
    assert bool((off <= u).all()) and off.max() > 0.98 * u


def test_rotation_keeps_lengths_and_depends_on_distance_only():
    table = _angles(50, 8)
    a, b = _normal(1, 1, 8, seed=1), _normal(1, 1, 8, seed=2)
    at = lambda x, p: orc.norm_rope(x, None, torch.tensor([p]), table, 0.0)[0]     # noqa: E731
    assert torch.allclose(at(a, 17).norm(), a.norm())
    assert torch.allclose((at(a, 17) * at(b, 11)).sum(), (at(a, 36) * at(b, 30)).sum())
    assert torch.equal(at(a, 0), a)


def test_norm_gives_unit_mean_square():
    x = _normal(5, 3, 16, seed=3)
    y = orc.norm_rope(x, torch.ones(16, dtype=F), torch.arange(5), _angles(5, 16), 0.0)[0]
    assert torch.allclose(y.pow(2).mean(-1), torch.ones(5, 3, dtype=F))


def test_channels_behind_the_rotated_ones_stay():
    x = _normal(4, 2, 16, seed=4)
    y = orc.norm_rope(x, None, torch.arange(4), _angles(4, 8), 0.0)[0]
    assert torch.equal(y[..., 8:], x[..., 8:]) and not torch.equal(y[1:, :, :8], x[1:, :, :8])


def test_attention_of_one_key_is_its_value_and_of_none_is_zero():
    q, k, v = _normal(3, 2, 8, seed=5), _normal(2, 1, 8, seed=6), _normal(2, 1, 8, seed=7)
    out, lse, _, _ = orc.attention(q, k, v, _offsets([1, 2]), _offsets([1, 1]), causal=True, scale=0.3)
    assert torch.allclose(out[0], v[0].expand(2, 8)) and torch.allclose(out[2], v[1].expand(2, 8))
    assert torch.equal(out[1], torch.zeros(2, 8, dtype=F)) and (lse[1] == -math.inf).all()   # two queries, one key: the first sees none
    assert torch.allclose(lse[0], 0.3 * (q[0] * k[0]).sum(-1))


def test_attention_of_equal_keys_is_the_mean():
    q, v = _normal(4, 1, 8, seed=8), _normal(4, 1, 8, seed=9)
    out, lse, _, _ = orc.attention(q, torch.zeros(4, 1, 8, dtype=F), v, _offsets([4]), _offsets([4]), causal=True, scale=1.0)
    for i in range(4):
        assert torch.allclose(out[i, 0], v[:i + 1, 0].mean(0))
        assert math.isclose(lse[i, 0].item(), math.log(i + 1), abs_tol=1e-15)


@pytest.mark.parametrize("causal", [True, False])
def test_attention_matches_the_library_soft_max(causal):
    q, k, v = _normal(6, 4, 8, seed=10), _normal(9, 2, 8, seed=11), _normal(9, 2, 8, seed=12)
    out, lse, _, _ = orc.attention(q, k, v, _offsets([6]), _offsets([9]), causal=causal, scale=0.5)
    for h in range(4):
        z = q[:, h] @ k[:, h // 2].t() * 0.5
        if causal:
            z = z + torch.full((6, 9), -math.inf, dtype=F).triu(4)
        assert torch.allclose(out[:, h], torch.softmax(z, 1) @ v[:, h // 2])
        assert torch.allclose(lse[:, h], torch.logsumexp(z, 1))


def test_keys_behind_a_cache_s_length_do_not_count():
    q, k, v = _normal(2, 1, 8, seed=13), _normal(10, 1, 8, seed=14), _normal(10, 1, 8, seed=15)
    k[3:5] = math.nan
    v[9:] = math.inf
    out, _, _, _ = orc.attention(q, k, v, _offsets([1, 1]), _offsets([5, 5]), causal=True, scale=1.0, k_used=torch.tensor([3, 4]))
    ref, _, _, _ = orc.attention(q, torch.cat((k[:3], k[5:9])), torch.cat((v[:3], v[5:9])), _offsets([1, 1]), _offsets([3, 4]),
                                 causal=True, scale=1.0)
    assert torch.equal(out, ref)


@pytest.mark.parametrize("causal, nq, nk", [(True, [3, 2], [3, 5]), (True, [4, 1], [2, 1]), (False, [2, 3], [4, 1])])
def test_attention_gradients_are_differences(causal, nq, nk):
    hq, hk, D, scale, e = 4, 2, 8, 0.4, 1e-5
    x = [_normal(sum(nq), hq, D, seed=20), _normal(sum(nk), hk, D, seed=21), _normal(sum(nk), hk, D, seed=22)]
    dout = _normal(sum(nq), hq, D, seed=23)
    run = lambda *a: orc.attention(*a, _offsets(nq), _offsets(nk), causal=causal, scale=scale)   # noqa: E731
    out, lse, _, _ = run(*x)
    grads, _ = orc.attention_grads(*x, out, lse, dout, _offsets(nq), _offsets(nk), causal=causal, scale=scale)
    for which in range(3):
        for at in torch.randperm(x[which].numel(), generator=torch.Generator().manual_seed(which))[:40].tolist():
            side = []
            for step in (e, -e):
                y = [t.clone() for t in x]
                y[which].view(-1)[at] += step
                side.append((run(*y)[0] * dout).sum())
            assert math.isclose(((side[0] - side[1]) / (2 * e)).item(), grads[which].reshape(-1)[at].item(), rel_tol=1e-6, abs_tol=1e-8)


@pytest.mark.parametrize("norm, rot", [(True, 8), (True, 16), (False, 16), (True, 0)])
def test_norm_and_rotation_gradients_are_differences(norm, rot):
    x, dy = _normal(3, 2, 16, seed=30), _normal(3, 2, 16, seed=31)
    gain = 1 + 0.3 * _normal(16, seed=32) if norm else None
    pos, table, e = torch.tensor([4, 0, 9]), _angles(10, rot), 1e-6
    f = lambda a, g: (orc.norm_rope(a, g, pos, table, 1e-3)[0] * dy).sum()     # noqa: E731
    dx, dgain, _, _ = orc.norm_rope_grads(x, dy, gain, pos, table, 1e-3)
    for at in range(0, x.numel(), 5):
        a, b = x.clone(), x.clone()
        a.view(-1)[at] += e
        b.view(-1)[at] -= e
        assert math.isclose(((f(a, gain) - f(b, gain)) / (2 * e)).item(), dx.reshape(-1)[at].item(), rel_tol=1e-6, abs_tol=1e-8)
    for at in range(16 if norm else 0):
        a, b = gain.clone(), gain.clone()
        a[at] += e
        b[at] -= e
        assert math.isclose(((f(x, a) - f(x, b)) / (2 * e)).item(), dgain[at].item(), rel_tol=1e-6, abs_tol=1e-8)
