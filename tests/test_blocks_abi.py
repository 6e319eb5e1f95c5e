"""Host-side checks of the embedding, residual-norm and clipping entry points: they answer without a GPU, before anything is launched."""
import ctypes

import pytest
import torch

from paper_2602_19362_amd import oapl

NULL, SHAPE, DTYPE, BETA, WORKSPACE, ALIGN = 1, 2, 3, 6, 7, 11
AT = 4096      # an address that no check follows
NAN, INF = float("nan"), float("inf")


def R(at=AT, stride=64):
    return oapl.Rows(at, stride)


def embed(E=AT, tokens=AT, T=4, d=64, V=10, dtype=1, out_dtype=1, scale=1.0, out=R()):
    return oapl.lib().oapl_embed_fwd(E, tokens, T, d, V, dtype, out_dtype, scale, out, None)


def embed_bwd(dout=R(), tokens=AT, T=4, d=64, V=10, dtype=1, scale=1.0, dE=AT, ws=AT, have=1 << 24):
    return oapl.lib().oapl_embed_bwd(dout, tokens, T, d, V, dtype, scale, 0, dE, ws, have, None)


def norm(x=R(), y=R(), y_gain=AT, gate=R(), per_token=1, gain=AT, T=4, d=64, x_dtype=1, dtype=1, scale=1.0, eps=1e-6, x_out=R(), out=R()):
    return oapl.lib().oapl_residual_norm_fwd(x, y, y_gain, gate, per_token, gain, T, d, x_dtype, dtype, scale, eps, x_out, out, None)


def norm_bwd(x=R(), y=R(), y_gain=AT, gate=R(), per_token=1, gain=AT, dx_out=R(), dout=R(), T=4, d=64, x_dtype=1, dtype=1, scale=1.0,
             eps=1e-6, dx=R(), dy=R(), dgain=AT, dy_gain=AT, dgate_rows=R(), dgate=AT, ws=AT, have=1 << 24):
    return oapl.lib().oapl_residual_norm_bwd(x, y, y_gain, gate, per_token, gain, dx_out, dout, T, d, x_dtype, dtype, scale, eps, dx, dy,
                                             dgain, dy_gain, dgate_rows, dgate, ws, have, None)


def tensors(*items):
    return (oapl.Tensor * max(1, len(items)))(*(oapl.Tensor(*x) for x in items))


def clip(items=((AT, AT, 4, 0),), n=None, max_norm=1.0, given=None, norm_out=AT, ws=AT, have=1 << 24):
    return oapl.lib().oapl_clip_grads(tensors(*items), len(items) if n is None else n, max_norm, given, norm_out, ws, have, None)


def grad_norm(items=((AT, None, 4, 0),), n=None, norm=AT, ws=AT, have=1 << 24):
    return oapl.lib().oapl_grad_norm(tensors(*items), len(items) if n is None else n, norm, ws, have, None)


@pytest.mark.parametrize("kw, want", [
    ({"dtype": 2}, DTYPE), ({"out_dtype": -1}, DTYPE), ({"T": -1}, SHAPE), ({"T": 65535 * 256 + 1}, SHAPE), ({"d": 0}, SHAPE), ({"V": 0}, SHAPE),
    ({"d": (1 << 21) + 1}, SHAPE), ({"V": (1 << 21) + 1}, SHAPE), ({"T": 1 << 23, "d": 1 << 18}, SHAPE), ({"scale": INF}, BETA),
    ({"scale": NAN}, BETA), ({"E": None}, NULL),
    ({"tokens": None}, NULL), ({"out": None}, NULL), ({"out": R(None)}, NULL), ({"out": R(AT, 63)}, SHAPE), ({"out": R(AT, -64)}, SHAPE),
    ({"out": R(AT, 1 << 46)}, SHAPE), ({"tokens": AT + 2}, ALIGN), ({"E": AT + 1}, ALIGN), ({"out": R(AT + 1)}, ALIGN), ({"dtype": 0, "E": AT + 2}, ALIGN),
])
def test_the_lookup_refuses(kw, want):
    assert embed(**kw) == want


@pytest.mark.parametrize("kw, want", [
    ({"dtype": 5}, DTYPE), ({"T": -1}, SHAPE), ({"T": 65535 * 256 + 1}, SHAPE), ({"V": 0}, SHAPE), ({"d": 0}, SHAPE), ({"scale": INF}, BETA),
    ({"dE": None}, NULL), ({"tokens": None}, NULL), ({"dout": None}, NULL), ({"dout": R(None)}, NULL), ({"dout": R(AT, -1)}, SHAPE),
    ({"dout": R(AT + 1)}, ALIGN), ({"dE": AT + 2}, ALIGN), ({"tokens": AT + 1}, ALIGN), ({"ws": None}, WORKSPACE), ({"ws": AT + 8}, WORKSPACE), ({"have": 255}, WORKSPACE),
])
def test_the_lookups_gradient_refuses(kw, want):
    assert embed_bwd(**kw) == want


@pytest.mark.parametrize("kw, want", [
    ({"dtype": 2}, DTYPE), ({"x_dtype": 2}, DTYPE), ({"x_dtype": 1, "dtype": 0}, DTYPE), ({"T": -1}, SHAPE), ({"T": 65535 * 256 + 1}, SHAPE),
    ({"d": 0}, SHAPE), ({"d": 16385}, SHAPE), ({"eps": -1.0}, BETA), ({"eps": NAN}, BETA), ({"scale": INF}, BETA), ({"x": None}, NULL),
    ({"x": R(None)}, NULL), ({"y": None}, NULL), ({"y": R(None)}, NULL), ({"gate": R(None)}, NULL), ({"x_out": None}, NULL), ({"out": None}, NULL),
    ({"gain": None}, NULL), ({"y": None, "y_gain": None, "gate": None, "x_out": None, "gain": None, "out": None}, NULL),
    ({"x": R(AT, -1)}, SHAPE), ({"x_out": R(AT, 63)}, SHAPE), ({"out": R(AT, 0)}, SHAPE), ({"y": R(AT + 1)}, ALIGN), ({"gain": AT + 1}, ALIGN),
    ({"y_gain": AT + 1}, ALIGN), ({"gate": R(AT + 1)}, ALIGN), ({"x_dtype": 0, "x": R(AT + 2)}, ALIGN), ({"x_dtype": 0, "x_out": R(AT + 2)}, ALIGN),
])
def test_the_residual_norm_refuses(kw, want):
    assert norm(**kw) == want


@pytest.mark.parametrize("kw, want", [
    ({"dtype": 2}, DTYPE), ({"d": 16385}, SHAPE), ({"dx": None}, NULL), ({"dy": None}, NULL), ({"dgain": None}, NULL), ({"dy_gain": None}, NULL),
    ({"dgate_rows": None}, NULL), ({"per_token": 0, "dgate": None}, NULL), ({"dout": None}, NULL), ({"dx": R(AT, 1)}, SHAPE),
    ({"dy": R(AT + 1)}, ALIGN), ({"dgain": AT + 2}, ALIGN), ({"dy_gain": AT + 1}, ALIGN), ({"dgate": AT + 1}, ALIGN), ({"ws": None}, WORKSPACE),
    ({"ws": AT + 16}, WORKSPACE), ({"have": 16}, WORKSPACE), ({"y": None}, NULL), ({"dx_out": R(None)}, NULL),
])
def test_the_residual_norms_gradients_refuse(kw, want):
    assert norm_bwd(**kw) == want


@pytest.mark.parametrize("kw, want", [
    ({"items": ((AT, AT, 4, 2),)}, DTYPE), ({"n": -1}, SHAPE), ({"n": (1 << 20) + 1}, SHAPE), ({"items": ((AT, AT, -1, 0),)}, SHAPE),
    ({"items": ((AT, AT, 1 << 45, 0),)}, SHAPE), ({"items": ((None, AT, 4, 0),)}, NULL), ({"items": ((AT, None, 4, 0),)}, NULL),
    ({"items": ((AT + 2, AT + 2, 4, 0),)}, ALIGN), ({"items": ((AT, AT + 1, 4, 1),)}, ALIGN), ({"max_norm": -1.0}, BETA), ({"max_norm": NAN}, BETA),
    ({"max_norm": INF}, BETA), ({"given": AT}, NULL), ({"norm_out": None}, NULL), ({"norm_out": AT + 2}, ALIGN), ({"ws": None}, WORKSPACE),
    ({"ws": AT + 8}, WORKSPACE), ({"have": 8}, WORKSPACE),
    # written twice; written where another is read; shifted over its own input; more than 2^42 elements, of one and of two
    ({"items": ((AT, AT, 4, 0), (AT, AT, 4, 0))}, SHAPE), ({"items": ((AT, 2 * AT, 64, 0), (3 * AT, 2 * AT + 252, 64, 0))}, SHAPE),
    ({"items": ((AT, 2 * AT, 64, 0), (2 * AT + 4, 3 * AT, 64, 0))}, SHAPE), ({"items": ((AT, AT + 4, 64, 0),)}, SHAPE),
    ({"items": ((AT, AT, (1 << 42) + 1, 0),)}, SHAPE), ({"items": ((AT, AT, 1 << 42, 0), (1 << 60, 1 << 60, 1, 1))}, SHAPE),
])
def test_clipping_refuses(kw, want):
    assert clip(**kw) == want


@pytest.mark.parametrize("kw, want", [
    ({"items": ((AT, None, 4, 2),)}, DTYPE), ({"n": -1}, SHAPE), ({"items": ((None, None, 4, 0),)}, NULL), ({"norm": None}, NULL),
    ({"norm": AT + 1}, ALIGN), ({"ws": None}, WORKSPACE), ({"have": 1}, WORKSPACE), ({"items": ((AT + 1, None, 4, 1),)}, ALIGN),
])
def test_the_norm_refuses(kw, want):
    assert grad_norm(**kw) == want


def test_calls_without_tokens_launch_nothing():
    assert embed(T=0, E=None, tokens=None, out=R(None)) == 0
    assert norm(T=0, x=R(None), y=R(None), gate=R(None), x_out=R(None), out=R(None)) == 0


def test_workspaces():
    ws = oapl.embed_workspace_bytes
    assert 0 < ws(0, 1, 1) <= ws(1000, 64, 1000) and ws(1000, 64, 1000) % 256 == 0
    for bad in ((-1, 1, 1), (1, 0, 1), (1, 1, 0), (65535 * 256 + 1, 1, 1), (1, 1, (1 << 21) + 1)):
        assert ws(*bad) == 0
    assert ws(65535 * 256, 1 << 16, 1 << 21) > 0 and ws(1 << 20, 1 << 20, 9) > 0 and ws(1 << 20, (1 << 20) + 1, 9) == 0
    ws = oapl.residual_norm_workspace_bytes
    assert 0 < ws(0, 1) and ws(1000, 4096) % 256 == 0 and ws(1000, 4096) >= 2 * 4096 * 4
    assert ws(-1, 4) == 0 and ws(1, 0) == 0 and ws(1, 16385) == 0 and ws(65535 * 256, 16384) > 0
    ws = oapl.clip_workspace_bytes
    assert 0 < ws(0) <= ws(1) <= ws(1 << 20) and ws(-1) == 0 and ws((1 << 20) + 1) == 0


def test_structures():
    assert ctypes.sizeof(oapl.Rows) == 16 and ctypes.sizeof(oapl.Tensor) == 32


@pytest.mark.parametrize("call", [
    lambda x, t: oapl.embed_fwd(x, t), lambda x, t: oapl.embed_bwd(x, t, 5), lambda x, t: oapl.residual_norm_fwd(x, x, x[0]),
    lambda x, t: oapl.residual_norm_bwd(x, x, x, x, x[0]), lambda x, t: oapl.grad_norm([x]), lambda x, t: oapl.clip_grads([x], 1.0),
    lambda x, t: oapl.clip_grads([], 1.0)])
def test_host_tensors_are_refused(call):
    with pytest.raises(ValueError):
        call(torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32))
