"""The oracle of embedding, residual stream and clipping, pinned by differences, by invariances and by hand."""
import math

import pytest
import torch

from oracle import blocks_oracle as orc

F = torch.float64


def _rand(*shape, seed):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=F)


def _forward(x0, y, gain, y_gain, gate, scale, eps=1e-6):
    first, second = orc.residual_norm(x0, y, gain, y_gain, gate, scale, eps)
    return (x0 if first is None else first[0]), (None if second is None else second[0])


@pytest.mark.parametrize("block, post, gated, pre, stream", [
    (True, True, "channel", True, True), (True, True, "token", True, True), (True, False, "channel", True, False),
    (True, False, "", True, True), (True, True, "", False, True), (False, False, "", True, True), (False, False, "", True, False)])
def test_gradients_are_differences(block, post, gated, pre, stream):
    T, d, scale, h = 3, 5, 0.7, 1e-6
    x, y = _rand(T, d, seed=1), _rand(T, d, seed=2) if block else None
    gain, y_gain = _rand(d, seed=3) if pre else None, _rand(d, seed=4) if post else None
    gate = {"channel": _rand(d, seed=5), "token": _rand(T, d, seed=6), "": None}[gated]
    a, b = (_rand(T, d, seed=7) if stream else torch.zeros(T, d, dtype=F)), _rand(T, d, seed=8)

    def loss(**kw):
        v = dict(x=x, y=y, gain=gain, y_gain=y_gain, gate=gate)
        v.update(kw)
        s, n = _forward(v["x"], v["y"], v["gain"], v["y_gain"], v["gate"], scale)
        return (a * s).sum() + ((b * n).sum() if n is not None else 0)

    behind = _forward(x, y, gain, y_gain, gate, scale)[0]
    got = orc.residual_norm_grads(behind, y, a if stream else None, b if pre else None, gain, y_gain, gate, scale, 1e-6)
    names = {"dx": ("x", x), "dy": ("y", y), "dgain": ("gain", gain), "dy_gain": ("y_gain", y_gain), "dgate": ("gate", gate)}
    assert set(got) == {k for k, (_, v) in names.items() if v is not None}
    for k, (value, _) in got.items():
        name, at = names[k]
        for i in range(at.numel()):
            step = torch.zeros_like(at)
            step.view(-1)[i] = h
            want = (loss(**{name: at + step}) - loss(**{name: at - step})) / (2 * h)
            # differences of order h^2 and of the loss's own rounding, 2^-53 of some tens over 2 h
            assert abs(value.reshape(-1)[i] - want) < 1e-7, (k, i)


def test_a_norm_by_hand():
    x = torch.tensor([[3.0, 4.0]], dtype=F)
    (s, _), (n, _) = orc.residual_norm(x, x * 0, torch.tensor([1.0, 2.0], dtype=F), None, None, 1.0, 0.0)
    r = math.sqrt(2 / 25)
    assert torch.equal(s, x) and torch.allclose(n, torch.tensor([[3 * r, 8 * r]], dtype=F), rtol=1e-15)


def test_embedding_by_hand():
    E = torch.arange(6, dtype=torch.float32).view(3, 2)
    out, bound = orc.embed(E, torch.tensor([2, 0, 2, 7]), 3.0, torch.float32)
    # the bound: two roundings of 2^-24 of the magnitude
    assert out[:3].tolist() == [[12, 15], [0, 3], [12, 15]] and out[3].isnan().all() and torch.equal(bound[:3], out[:3] * 2.0 ** -23)
    dE, bound = orc.embed_grads(torch.ones(4, 2), torch.tensor([2, 0, 2, -1]), 3, 0.5, old=torch.full((3, 2), 7.0))
    assert dE.tolist() == [[7.5, 7.5], [7, 7], [8, 8]] and (bound[1] == 0).all()


def test_the_gradient_of_the_lookup_is_its_transpose():
    E, tokens, dout = _rand(7, 3, seed=1), torch.tensor([1, 6, 1, 0, 1]), _rand(5, 3, seed=2)
    out = orc.embed(E, tokens, 1.5, torch.float32)[0]
    dE = orc.embed_grads(dout, tokens, 7, 1.5)[0]
    assert abs((out * dout).sum() - (E * dE).sum()) < 1e-13


def test_clipping_by_hand():
    grads = [torch.tensor([3.0, 0.0]), torch.tensor([[4.0]])]
    norm, _ = orc.grad_norm(grads)
    assert norm.item() == 5
    assert [g.tolist() for g, _ in orc.clipped(grads, 1.0, norm)] == [[0.6000000000000001, 0.0], [[0.8]]]
    assert [g.tolist() for g, _ in orc.clipped(grads, 5.0, norm)] == [[3.0, 0.0], [[4.0]]]
    assert [g.tolist() for g, _ in orc.clipped(grads, 1.0, norm * math.inf)] == [[3.0, 0.0], [[4.0]]]
    assert orc.grad_norm([])[0].item() == 0
