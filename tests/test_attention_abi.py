"""The attention entry points' host-side checks: they answer without a GPU, before anything is launched."""
import ctypes

import pytest

from paper_2602_19362_amd import oapl

NULL, SHAPE, DTYPE, BETA, WORKSPACE, ALIGN = 1, 2, 3, 6, 7, 11
AT = 4096      # an address that no check follows


def H(at=AT, token=128, head=64):
    return oapl.Heads(at, token, head)


def rope(T=4, hq=2, hk=1, D=64, rot=64, n_pos=10, n_rows=4, dtype=1, eps=1e-6, q=H(), k=H(), v=None, pos=AT, cs=AT, gq=AT, gk=AT,
         rows=None, q_out=H(), k_out=H(), v_out=None):
    return oapl.lib().oapl_qk_norm_rope_fwd(q, k, v, pos, cs, gq, gk, rows, T, hq, hk, D, rot, n_pos, n_rows, dtype, eps, q_out, k_out,
                                            v_out, None)


def rope_bwd(T=4, D=64, gq=AT, gk=AT, dgq=AT, dgk=AT, dq=H(), dk=H(), ws=AT, have=1 << 20):
    return oapl.lib().oapl_qk_norm_rope_bwd(H(), H(), H(), H(), AT, AT, gq, gk, T, 2, 1, D, D, 10, 1, 1e-6, dq, dk, dgq, dgk, ws, have, None)


def fwd(Tq=4, Tk=4, n=1, hq=2, hk=1, D=64, dtype=1, scale=0.1, q=H(), k=H(), v=H(), qo=AT, ko=AT, out=H(), ws=AT, have=1 << 24):
    return oapl.lib().oapl_attention_fwd(q, k, v, qo, ko, None, Tq, Tk, n, hq, hk, D, dtype, 1, scale, out, None, ws, have, None)


def bwd(lse=AT, dq=H(), dk=H(), dv=H(), dout=H(), D=64, have=1 << 24, q=H()):
    return oapl.lib().oapl_attention_bwd(q, H(), H(), H(), lse, dout, AT, AT, 4, 4, 1, 2, 1, D, 1, 1, 0.1, dq, dk, dv, AT, have, None)


@pytest.mark.parametrize("kw, want", [
    ({"dtype": 2}, DTYPE), ({"T": -1}, SHAPE), ({"hq": 0}, SHAPE), ({"hk": 0}, SHAPE), ({"D": 60}, SHAPE), ({"D": 136, "rot": 0}, SHAPE),
    ({"D": 0, "rot": 0}, SHAPE), ({"rot": 72}, SHAPE), ({"rot": 12}, SHAPE), ({"n_pos": -1}, SHAPE), ({"eps": -1.0}, BETA),
    ({"eps": float("nan")}, BETA), ({"gq": None}, NULL), ({"gk": None}, NULL), ({"pos": None}, NULL), ({"cs": None}, NULL),
    ({"q": None}, NULL), ({"k_out": None}, NULL), ({"q": H(None)}, NULL), ({"q": H(AT + 8)}, ALIGN), ({"k": H(AT, 129)}, ALIGN),
    ({"q": H(AT, 128, 63)}, ALIGN), ({"cs": AT + 4}, ALIGN), ({"gq": AT + 2}, ALIGN), ({"v": H()}, NULL), ({"v_out": H()}, NULL),
    ({"rows": AT, "n_rows": -1}, SHAPE), ({"q_out": H(AT, 0)}, SHAPE), ({"q_out": H(AT, 128, 0)}, SHAPE), ({"q": H(AT, -128)}, SHAPE),
    ({"q": H(AT, 1 << 24)}, SHAPE),
])
def test_norm_rope_refuses(kw, want):
    assert rope(**kw) == want


def test_norm_rope_of_no_tokens_launches_nothing():
    assert rope(T=0, q=H(None), k=H(None), q_out=H(None), k_out=H(None), pos=None, cs=None, n_rows=0) == 0


@pytest.mark.parametrize("kw, want", [
    ({"dgq": None}, NULL), ({"dgk": None}, NULL), ({"dq": None}, NULL), ({"dk": H(AT + 1)}, ALIGN), ({"ws": None}, WORKSPACE),
    ({"ws": AT + 16}, WORKSPACE), ({"have": 16}, WORKSPACE), ({"D": 4}, SHAPE),
])
def test_norm_rope_gradients_refuse(kw, want):
    assert rope_bwd(**kw) == want


@pytest.mark.parametrize("kw, want", [
    ({"dtype": 7}, DTYPE), ({"Tq": -1}, SHAPE), ({"Tk": -1}, SHAPE), ({"n": -1}, SHAPE), ({"n": 0}, SHAPE), ({"hq": 3, "hk": 2}, SHAPE),
    ({"hq": 1, "hk": 2}, SHAPE), ({"hk": 0}, SHAPE), ({"D": 12}, SHAPE), ({"D": 256}, SHAPE), ({"Tk": 1 << 31}, SHAPE), ({"Tq": 1 << 40}, SHAPE),
    ({"scale": float("inf")}, BETA), ({"scale": float("nan")}, BETA), ({"qo": None}, NULL), ({"ko": None}, NULL), ({"q": None}, NULL),
    ({"k": H(None)}, NULL), ({"out": None}, NULL), ({"q": H(AT + 2)}, ALIGN), ({"v": H(AT, 100)}, ALIGN), ({"out": H(AT, 32)}, SHAPE),
    ({"out": H(AT, 128, 0)}, SHAPE), ({"ws": None}, WORKSPACE), ({"ws": AT + 128}, WORKSPACE), ({"have": 255}, WORKSPACE),
])
def test_attention_refuses(kw, want):
    assert fwd(**kw) == want


@pytest.mark.parametrize("kw, want", [
    ({"lse": None}, NULL), ({"dq": None}, NULL), ({"dk": None}, NULL), ({"dv": H(None)}, NULL), ({"dout": H(AT + 4)}, ALIGN),
    ({"dv": H(AT, 0)}, SHAPE), ({"D": 4}, SHAPE), ({"have": 256}, WORKSPACE), ({"q": H(AT, 128, 1 << 30)}, SHAPE),
])
def test_attention_gradients_refuse(kw, want):
    assert bwd(**kw) == want


def test_workspaces():
    ws = oapl.attention_workspace_bytes
    assert 0 < ws(100, 100, 2, 8, 2, 64, 1, False) <= ws(100, 100, 2, 8, 2, 64, 1, True)
    assert ws(100, 100, 2, 8, 2, 64, 1, True) >= 256 + 100 * 8 * 4
    assert ws(0, 0, 0, 1, 1, 8, 0, True) > 0
    for bad in ((-1, 1, 1, 1, 1, 8, 0), (1, 1, 1, 3, 2, 8, 0), (1, 1, 1, 1, 1, 12, 0), (1, 1, 1, 1, 1, 8, 2), (1, 0, 0, 1, 1, 8, 0)):
        assert ws(*bad, True) == 0
    rope_ws = oapl.lib().oapl_qk_norm_rope_workspace_bytes
    assert rope_ws(1000, 8, 2, 128) % 256 == 0 and rope_ws(1000, 8, 2, 128) > 0 and rope_ws(0, 1, 1, 8) > 0
    assert rope_ws(-1, 8, 2, 128) == 0 and rope_ws(5, 8, 2, 100) == 0 and rope_ws(5, 0, 2, 128) == 0


def test_a_status_of_its_own():
    assert b"16 bytes" in oapl.lib().oapl_status_string(ALIGN)
    assert ctypes.sizeof(oapl.Heads) == 24
