"""The residual stream with its norms, and the gradients, against the 64-bit oracle within its error bounds."""
import pytest
import torch

from oracle import blocks_oracle as orc
from paper_2602_19362_amd import oapl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": (torch.bfloat16, torch.bfloat16), "f32": (torch.float32, torch.float32), "mixed": (torch.float32, torch.bfloat16)}


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def near(got, want, bound, name=""):
    assert got.shape == want.shape
    off = (got.to(torch.float64) - want).abs()
    assert bool((off <= bound + 1e-300).all()), (name, float((off / (bound + 1e-300)).max()))


def inputs(types, T, d, parts, seed=0):
    """parts: of "pre", "block", "post", "channel", "token"."""
    tx, t = TYPES[types]
    g = _gen(seed)

    def rand(*shape, dtype=t, scale=1.0):
        return (torch.randn(*shape, generator=g, device=DEV) * scale).to(dtype)

    v = {"x": rand(T, d, dtype=tx, scale=3), "y": rand(T, d) if "block" in parts else None, "gain": rand(d) if "pre" in parts else None,
         "y_gain": rand(d) if "post" in parts else None, "gate": rand(d) if "channel" in parts else rand(T, d) if "token" in parts else None}
    return v, rand(T, d, dtype=tx), rand(T, d) if "pre" in parts else None


def check_forward(v, scale, eps=1e-6, **kw):
    want = orc.residual_norm(v["x"], v["y"], v["gain"], v["y_gain"], v["gate"], scale, eps)
    r = oapl.residual_norm_fwd(v["x"], v["y"], v["gain"], y_gain=v["y_gain"], gate=v["gate"], scale=scale, eps=eps, **kw)
    if want[0] is None:
        assert r.x is v["x"]
    else:
        near(r.x, *want[0], "x")
    if want[1] is None:
        assert r.out is None
    else:
        near(r.out, *want[1], "out")
    return r


def check_backward(v, dx_out, dout, scale, eps=1e-6, **kw):
    want = orc.residual_norm_grads(v["x"], v["y"], dx_out, dout, v["gain"], v["y_gain"], v["gate"], scale, eps)
    r = oapl.residual_norm_bwd(v["x"], v["y"], dx_out, dout, v["gain"], y_gain=v["y_gain"], gate=v["gate"], scale=scale, eps=eps, **kw)
    for name in ("dx", "dy", "dgain", "dy_gain", "dgate"):
        got = getattr(r, name)
        if name in want:
            near(got, *want[name], name)
        else:
            assert got is None
    return r


PARTS = ["pre", "block", "pre block", "pre block post", "block post", "pre block channel", "pre block post channel", "pre block token",
         "pre block post token", "block post channel"]
# widths: a wavefront and four rows a workgroup, a workgroup a row, ends inside a piece of eight channels, more lanes than channels
SHAPES = [(1, 8), (5, 64), (3, 100), (9, 512), (4, 513), (6, 1000), (2, 1024), (3, 1025), (5, 2048), (2, 2056), (3, 4096), (2, 5120), (1, 8192),
          (2, 8201), (3, 16384), (700, 72), (2100, 40), (5, 1), (1, 7), (3, 3000),
          # more rows than workgroups have room for at once
          (9001, 24), (2500, 300), (1300, 700), (600, 2000), (300, 3000), (300, 8000), (270, 10000)]


@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("parts", PARTS)
def test_parts(types, parts):
    for T, d in ((6, 200), (601, 1032)):
        v, dx_out, dout = inputs(types, T, d, parts.split())
        check_forward(v, 0.7)
        check_backward(v, dx_out, dout, 0.7)
        check_backward(v, None, dout, -1.3)


@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("T, d", SHAPES)
def test_shapes(types, T, d):
    for parts in ("pre block post channel", "pre block post token", "pre"):
        v, dx_out, dout = inputs(types, T, d, parts.split(), seed=d)
        check_forward(v, 1.0)
        r = check_backward(v, dx_out, dout, 1.0)
        r.workspace.fill_(255)
        again = oapl.residual_norm_bwd(v["x"], v["y"], dx_out, dout, v["gain"], y_gain=v["y_gain"], gate=v["gate"], workspace=r.workspace)
        for a, b in zip(r[:5], again[:5]):
            assert (a is None and b is None) or torch.equal(a, b)


@pytest.mark.parametrize("types", list(TYPES))
def test_rows_inside_larger_buffers(types):
    """Rows further apart than their channels, that start at any element, and one row for all tokens."""
    T, d = 23, 136
    v, dx_out, dout = inputs(types, T, d, ["pre", "block", "post", "token"])

    def inside(x, shift):
        wide = torch.full((T, d + 13), 9.0, device=DEV, dtype=x.dtype)
        wide[:, shift:shift + d] = x
        return wide, wide[:, shift:shift + d]

    for n, shift in (("x", 1), ("y", 3), ("gate", 5)):
        _, v[n] = inside(v[n], shift)
    for n in ("gain", "y_gain"):
        v[n] = torch.cat((v[n][:1], v[n]))[1:]
    (_, a), (_, b) = inside(dx_out, 7), inside(dout, 9)
    (bx, x_out), (bo, out), (bdx, dx), (bdy, dy) = (inside(t, s) for t, s in ((dx_out, 2), (dout, 4), (dx_out, 6), (dout, 8)))
    check_forward(v, 0.5, x_out=x_out, out=out)
    check_backward(v, a, b, 0.5, dx=dx, dy=dy)
    for buffer, shift in ((bx, 2), (bo, 4), (bdx, 6), (bdy, 8)):
        assert bool((buffer[:, :shift] == 9).all()) and bool((buffer[:, shift + d:] == 9).all())
    for n in ("x", "y", "gate"):
        v[n] = v[n][3].expand(T, d)
    check_forward(v, 0.5)
    check_backward(v, a[:1].expand(T, d), b[:1].expand(T, d), 0.5)


@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("d", [2, 3, 4, 5, 9, 10, 11, 12, 13, 14, 15, 125, 131, 509, 515, 777, 1021, 2047, 4099, 6002, 8191, 8193, 16381])
def test_widths_that_end_inside_a_piece(types, d):
    """With NaN on both sides of every row, and in place."""
    T = 37 if d < 2000 else 5
    v, dx_out, dout = inputs(types, T, d, ["pre", "block", "post", "token"], seed=d)

    def inside(x):
        wide = torch.full((T, d + 20), torch.nan, device=DEV, dtype=x.dtype)
        wide[:, 9:9 + d] = x
        return wide, wide[:, 9:9 + d]

    for n in ("x", "y", "gate"):
        _, v[n] = inside(v[n])
    for n in ("gain", "y_gain"):
        v[n] = torch.cat((v[n] * torch.nan, v[n], v[n] * torch.nan))[d:2 * d]
    (_, dx_out), (_, dout) = inside(dx_out), inside(dout)
    plain = check_forward(v, 0.7)
    want = check_backward(v, dx_out, dout, 0.7)
    (wx, x), (wy, y), (wdx, dx), (wdy, dy) = (inside(t) for t in (v["x"], v["y"], dx_out, dout))
    r = oapl.residual_norm_fwd(x, y, v["gain"], y_gain=v["y_gain"], gate=v["gate"], scale=0.7, x_out=x, out=y)
    assert torch.equal(r.x, plain.x) and torch.equal(r.out, plain.out)
    got = oapl.residual_norm_bwd(v["x"], v["y"], dx, dy, v["gain"], y_gain=v["y_gain"], gate=v["gate"], scale=0.7, dx=dx, dy=dy)
    for a, b in zip(got[:5], want[:5]):
        assert torch.equal(a, b)
    for wide in (wx, wy, wdx, wdy):
        assert bool(wide[:, :9].isnan().all()) and bool(wide[:, 9 + d:].isnan().all())


@pytest.mark.parametrize("types", list(TYPES))
def test_in_place(types):
    v, dx_out, dout = inputs(types, 300, 1500, ["pre", "block", "post", "token"])
    plain = check_forward(v, 1.0)
    x, y = v["x"].clone(), v["y"].clone()
    r = oapl.residual_norm_fwd(x, y, v["gain"], y_gain=v["y_gain"], gate=v["gate"], x_out=x, out=y)
    assert r.x is x and r.out is y and torch.equal(x, plain.x) and torch.equal(y, plain.out)
    want = check_backward(v, dx_out, dout, 1.0)
    for dx, dy in ((dx_out.clone(), dout.clone()), (v["x"].clone(), v["y"].clone())):
        first = dx if torch.equal(dx, dx_out) else dx_out
        second = dy if torch.equal(dy, dout) else dout
        got = oapl.residual_norm_bwd(v["x"] if first is dx else dx, v["y"] if second is dy else dy, first, second, v["gain"],
                                     y_gain=v["y_gain"], gate=v["gate"], dx=dx, dy=dy)
        for a, b in zip(got[:5], want[:5]):
            assert torch.equal(a, b)


def test_what_is_not_finite_stays_in_its_row():
    v, dx_out, dout = inputs("bf16", 40, 600, ["pre", "block", "post"])
    v["y"][3, 17], v["x"][11, 2] = torch.nan, torch.inf
    r = oapl.residual_norm_fwd(v["x"], v["y"], v["gain"], y_gain=v["y_gain"])
    rows = torch.tensor([i not in (3, 11) for i in range(40)], device=DEV)
    assert torch.equal(r.out.isfinite().all(1), rows)
    b = oapl.residual_norm_bwd(v["x"], v["y"], dx_out, dout, v["gain"], y_gain=v["y_gain"])
    assert bool(b.dx[rows].isfinite().all()) and bool(b.dy[rows].isfinite().all())


@pytest.mark.parametrize("types", list(TYPES))
def test_rows_of_zeros_and_of_large_and_small_numbers(types):
    v, dx_out, dout = inputs(types, 6, 328, ["pre", "block", "post"])
    for n in ("x", "y"):
        v[n][0] = 0
        v[n][1] *= 1e15
        v[n][2] *= 1e-12
    check_forward(v, 1.0)
    check_backward(v, dx_out, dout, 1.0)
    check_forward(v, 1.0, eps=0.01)


@pytest.mark.parametrize("T, d", [(1, 40), (9000, 100), (300, 4096), (260, 9000)])
def test_nothing_beside_the_workspace_is_touched(T, d):
    n = oapl.residual_norm_workspace_bytes(T, d)
    room = torch.full((n + 512,), 0x5a, dtype=torch.uint8, device=DEV)
    v, dx_out, dout = inputs("mixed", T, d, ["pre", "block", "post", "channel"])
    check_backward(v, dx_out, dout, 1.0, workspace=room[256:256 + n])
    assert bool((room[:256] == 0x5a).all()) and bool((room[256 + n:] == 0x5a).all())


def test_no_tokens():
    v, dx_out, dout = inputs("bf16", 0, 64, ["pre", "block", "post", "channel"])
    r = oapl.residual_norm_fwd(v["x"], v["y"], v["gain"], y_gain=v["y_gain"], gate=v["gate"])
    assert r.x.shape == r.out.shape == (0, 64)
    b = oapl.residual_norm_bwd(v["x"], v["y"], dx_out, dout, v["gain"], y_gain=v["y_gain"], gate=v["gate"])
    assert all(bool((x == 0).all()) and x.shape == (64,) for x in (b.dgain, b.dy_gain, b.dgate))


@pytest.mark.parametrize("parts", ["pre", "pre block post channel", "pre block token"])
def test_gradients_are_differences(parts):
    """Along a direction: the quotient of the kernel's outputs is off by what the oracle bounds at either end; how far a quotient of
    this step is from the derivative is taken from the oracle's."""
    T, d, scale, h = 7, 96, 0.8, 2.0 ** -6
    v, a, b = inputs("f32", T, d, parts.split(), seed=3)
    names = [n for n in ("x", "y", "gain", "y_gain", "gate") if v[n] is not None]
    way = {n: torch.randn(v[n].shape, generator=_gen(20 + i), device=DEV) for i, n in enumerate(names)}
    F = torch.float64

    def moved(sign):
        return {n: None if v[n] is None else (v[n] + sign * h * way[n]) for n in v}

    def value(w):
        """The loss of the kernel's outputs, of the oracle's, and a bound of their difference."""
        r = oapl.residual_norm_fwd(w["x"], w["y"], w["gain"], y_gain=w["y_gain"], gate=w["gate"], scale=scale)
        first, second = orc.residual_norm(w["x"], w["y"], w["gain"], w["y_gain"], w["gate"], scale, 1e-6)
        mine = (b.to(F) * r.out).sum()
        theirs, off = (b.to(F) * second[0]).sum(), (b.to(F).abs() * second[1]).sum()
        if first is not None:
            mine, theirs, off = mine + (a.to(F) * r.x).sum(), theirs + (a.to(F) * first[0]).sum(), off + (a.to(F).abs() * first[1]).sum()
        return mine, theirs, off

    hi, lo = value(moved(1)), value(moved(-1))
    # (the ends lie where the sums rounded to: the step is what lies between them)
    ends = {n: (moved(1)[n].to(F) - moved(-1)[n].to(F)) / (2 * h) for n in names}
    behind = orc.residual_norm(v["x"], v["y"], v["gain"], v["y_gain"], v["gate"], scale, 1e-6)[0]
    x = v["x"] if behind is None else behind[0].float()
    stream = a if behind is not None else None
    got = oapl.residual_norm_bwd(x, v["y"], stream, b, v["gain"], y_gain=v["y_gain"], gate=v["gate"], scale=scale)
    want = orc.residual_norm_grads(x, v["y"], stream, b, v["gain"], v["y_gain"], v["gate"], scale, 1e-6)
    key = {"x": "dx", "y": "dy", "gain": "dgain", "y_gain": "dy_gain", "gate": "dgate"}
    slope = sum((getattr(got, key[n]).to(F) * ends[n]).sum() for n in names)
    true = sum((want[key[n]][0] * ends[n]).sum() for n in names)
    bound = sum((want[key[n]][1] * ends[n].abs()).sum() for n in names)
    quotient, exact = (hi[0] - lo[0]) / (2 * h), (hi[1] - lo[1]) / (2 * h)
    assert abs(quotient - slope) <= abs(exact - true) + (hi[2] + lo[2]) / (2 * h) + bound
    assert abs(exact - true) <= 0.01 * abs(true) + 1       # the step is a small one


def test_refusals():
    x, g = torch.zeros(4, 16, device=DEV), torch.zeros(16, device=DEV)
    with pytest.raises(ValueError):
        oapl.residual_norm_fwd(x)
    with pytest.raises(ValueError):
        oapl.residual_norm_fwd(x, None, g, gate=g)
    with pytest.raises(ValueError):
        oapl.residual_norm_fwd(x, x, g[:8])
    with pytest.raises(ValueError):
        oapl.residual_norm_fwd(x, x, g, gate=g[:4])
    with pytest.raises(ValueError):
        oapl.residual_norm_fwd(x, x[:3], g)
    with pytest.raises(ValueError):
        oapl.residual_norm_fwd(x, x, x_out=x, out=x)
    with pytest.raises(TypeError):
        oapl.residual_norm_fwd(x, x.bfloat16(), g)
    with pytest.raises(oapl.OaplError):
        oapl.residual_norm_fwd(x.bfloat16(), x, g)
    with pytest.raises(ValueError):
        oapl.residual_norm_fwd(x.t(), None, torch.zeros(4, device=DEV))
    with pytest.raises(oapl.OaplError):
        oapl.residual_norm_fwd(torch.zeros(1, 16385, device=DEV), None, torch.zeros(16385, device=DEV))
    with pytest.raises(oapl.OaplError):
        oapl.residual_norm_fwd(x, None, g, eps=-1.0)
    with pytest.raises(oapl.OaplError):
        oapl.residual_norm_fwd(x, x, g, out=x[:1].expand(4, 16))
    with pytest.raises(ValueError):
        oapl.residual_norm_bwd(x, x, None, x)
    with pytest.raises(ValueError):
        oapl.residual_norm_bwd(x, x, x, None, g)
    with pytest.raises(oapl.OaplError):
        oapl.residual_norm_bwd(x, None, x, x, g, workspace=torch.zeros(64, device=DEV, dtype=torch.uint8))
