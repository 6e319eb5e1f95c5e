"""Attention over packed sequences and caches, and its gradients, against the 64-bit oracle within its error bounds."""
import math

import pytest
import torch

from oracle import attention_oracle as orc
from paper_2602_19362_amd import oapl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _offsets(lengths):
    return torch.tensor([0] + list(lengths), device=DEV).cumsum(0)


def _normal(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g, device=DEV)).to(dtype)


def _qkv(dtype, nq, nk, hq, hk, D, seed=0, scale=1.0):
    dt = DTYPES[dtype]
    return (_normal((sum(nq), hq, D), dt, seed, scale), _normal((sum(nk), hk, D), dt, seed + 1), _normal((sum(nk), hk, D), dt, seed + 2))


def _near(got, want, bound):
    assert got.shape == want.shape
    got = got.to(torch.float64)
    same = (got == want) | ((got - want).abs() <= bound + 1e-30)        # equal infinities are equal
    assert bool(same.all()), (int((~same).sum()), float(((got - want).abs() / (bound + 1e-30))[~same].max()))


def _check(dtype, nq, nk, hq, hk, D, causal, scale=None, seed=0, spread=1.0, grads=True):
    q, k, v = _qkv(dtype, nq, nk, hq, hk, D, seed, spread)
    qo, ko = _offsets(nq), _offsets(nk)
    s = D ** -0.5 if scale is None else scale
    r = oapl.attention_fwd(q, k, v, qo, ko, causal=causal, scale=scale)
    assert oapl.read_device_status(r.workspace) == 0
    out, lse, bound, lse_bound = orc.attention(q, k, v, qo, ko, causal=causal, scale=s)
    _near(r.out, out, bound)
    _near(r.lse, lse, lse_bound)
    if not grads:
        return
    dout = _normal(q.shape, q.dtype, seed + 3)
    b = oapl.attention_bwd(q, k, v, r.out, r.lse, dout, qo, ko, causal=causal, scale=scale)
    assert oapl.read_device_status(b.workspace) == 0
    want, bounds = orc.attention_grads(q, k, v, r.out, r.lse, dout, qo, ko, causal=causal, scale=s)
    for x, y, z in zip(b[:3], want, bounds):
        _near(x, y, z)


LENGTHS = [
    ([1], [1]),
    ([0, 1, 0, 2, 0], [0, 1, 0, 2, 0]),                                    # empty sequences among others
    ([31, 32, 33, 63, 64, 65], [31, 32, 33, 63, 64, 65]),
    ([127, 128, 129, 255, 257], [127, 128, 129, 255, 257]),
    ([5, 3, 70, 1], [9, 200, 70, 130]),                                    # more keys than queries
    ([9, 200, 70, 4], [5, 3, 0, 1]),                                       # fewer: rows that see nothing
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("nq, nk", LENGTHS)
def test_lengths(dtype, causal, nq, nk):
    _check(dtype, nq, nk, 4, 2, 64, causal)


# Many more queries than keys beside sequences with several tiles of keys: every tile of keys has its gradients written, once.
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq, nk", [([9, 400, 300], [200, 3, 90]), ([300, 500, 30], [20, 300, 30]), ([150, 9, 600], [140, 5, 3])])
def test_sequences_that_outgrow_their_keys(dtype, nq, nk):
    _check(dtype, nq, nk, 4, 2, 64, True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq, hk, D", [(1, 1, 8), (3, 3, 16), (5, 1, 24), (8, 2, 40), (6, 3, 72), (14, 2, 80), (2, 1, 96), (16, 2, 104),
                                       (7, 1, 120), (12, 3, 128), (48, 1, 64), (130, 1, 32)])
def test_head_layouts(dtype, hq, hk, D):
    _check(dtype, [70, 1, 45], [70, 1, 45], hq, hk, D, True, seed=10)


@pytest.mark.parametrize("causal", [True, False])
def test_many_sequences(causal):
    nq = [(7 * i * i + i) % 23 for i in range(300)]
    nk = [(5 * i * i + 3 * i) % 31 for i in range(300)]
    _check("bf16", nq, nk, 2, 1, 64, causal, seed=20)


@pytest.mark.parametrize("dtype, n", [("bf16", 1100), ("bf16", 2500), ("f32", 700)])
def test_longer_sequences(dtype, n):
    _check(dtype, [n, 300], [n, 813], 4, 2, 128, True, seed=30)


def test_few_rows_over_many_keys():
    _check("bf16", [1, 1, 3], [5000, 64, 2049], 8, 2, 128, True, seed=40)
    _check("bf16", [2, 0, 1], [1, 700, 9000], 5, 5, 80, True, seed=41)
    _check("f32", [1, 2], [1500, 333], 8, 2, 64, True, seed=42)


@pytest.mark.parametrize("spread, scale", [(30.0, None), (1.0, 0.0), (1.0, -0.4), (1e-3, None)])
def test_score_ranges(spread, scale):
    """One key taking nearly everything, equal scores, a negative scale, scores near zero."""
    _check("bf16", [150, 40], [150, 90], 4, 2, 64, True, scale=scale, seed=50, spread=spread)
    _check("f32", [50], [50], 4, 2, 64, True, scale=scale, seed=51, spread=spread)


def test_scores_that_rise_along_the_keys():
    """The running maximum moves at every tile."""
    n, D = 900, 64
    q = torch.ones(n, 2, D, device=DEV).to(torch.bfloat16)
    k = (torch.arange(n, device=DEV, dtype=torch.float32)[:, None, None] * 0.02).expand(n, 1, D).to(torch.bfloat16)
    v = _normal((n, 1, D), torch.bfloat16, 60)
    o = _offsets([n])
    for kk in (k, k.flip(0).contiguous()):
        r = oapl.attention_fwd(q, kk, v, o)
        out, lse, bound, lse_bound = orc.attention(q, kk, v, o, o, causal=True, scale=D ** -0.5)
        _near(r.out, out, bound)
        _near(r.lse, lse, lse_bound)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cache_with_room(dtype):
    """Rows behind a sequence's keys hold whatever was there; they are not read into any result."""
    hq, hk, D, room, used = 8, 2, 128, 300, [1, 300, 0, 65, 128, 250]
    nq = [1] * 6
    q, k, v = _qkv(dtype, nq, [room] * 6, hq, hk, D, seed=70)
    ko, n = _offsets([room] * 6), torch.tensor(used, device=DEV)
    for s, u in enumerate(used):
        k[s * room + u:(s + 1) * room] = math.nan
        v[s * room + u:(s + 1) * room] = math.inf
    r = oapl.attention_fwd(q, k, v, _offsets(nq), ko, k_used=n)
    out, lse, bound, lse_bound = orc.attention(q, k, v, _offsets(nq), ko, causal=True, scale=D ** -0.5, k_used=n)
    _near(r.out, out, bound)
    _near(r.lse, lse, lse_bound)
    assert not r.out[2].any() and bool((r.lse[2] == -math.inf).all())


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_is_not_finite_stays_in_its_sequence(bad):
    nq = [40, 33, 50]
    q, k, v = _qkv("bf16", nq, nq, 4, 2, 64, seed=80)
    o, dout = _offsets(nq), _normal(q.shape, q.dtype, 83)
    want = oapl.attention_fwd(q, k, v, o)
    grads = oapl.attention_bwd(q, k, v, want.out, want.lse, dout, o)
    for x in (q, k, v):
        x[40:73] = bad
    got = oapl.attention_fwd(q, k, v, o)
    keep = torch.cat((torch.arange(40), torch.arange(73, 123))).to(DEV)
    assert torch.equal(got.out[keep], want.out[keep]) and torch.equal(got.lse[keep], want.lse[keep])
    bwd = oapl.attention_bwd(q, k, v, got.out, got.lse, dout, o)
    for a, b in zip(bwd[:3], grads[:3]):
        assert torch.equal(a[keep], b[keep])


def test_strides_and_orders():
    """Views of one projection, heads before tokens, broadcast keys, gradients into one buffer: the same values."""
    n, hq, hk, D = [130, 77], 6, 2, 64
    T = sum(n)
    q, k, v = _qkv("bf16", n, n, hq, hk, D, seed=90)
    o, dout = _offsets(n), _normal(q.shape, q.dtype, 93)
    want = oapl.attention_fwd(q, k, v, o)
    grads = oapl.attention_bwd(q, k, v, want.out, want.lse, dout, o)
    qkv = torch.cat((q, k, v), 1)
    a, b, c = qkv.split((hq, hk, hk), 1)
    out = torch.full((hq, T, D), 7.0, device=DEV, dtype=q.dtype).transpose(0, 1)
    got = oapl.attention_fwd(a, b, c, o, out=out)
    assert got.out is out and torch.equal(out, want.out) and torch.equal(got.lse, want.lse)
    d = torch.full_like(qkv, 7.0)
    da, db, dc = d.split((hq, hk, hk), 1)
    oapl.attention_bwd(a, b, c, out, got.lse, dout.transpose(0, 1).contiguous().transpose(0, 1), o, dq=da, dk=db, dv=dc)
    assert torch.equal(d, torch.cat(grads[:3], 1))
    one = k[:, :1].expand(T, hk, D)
    x = oapl.attention_fwd(q, one, v, o)
    assert torch.equal(x.out, oapl.attention_fwd(q, one.contiguous(), v, o).out)


def test_a_second_run_gives_the_same_bits():
    n = [500, 1, 260]
    q, k, v = _qkv("bf16", n, n, 8, 2, 128, seed=100)
    o, dout = _offsets(n), _normal(q.shape, q.dtype, 103)
    a = oapl.attention_fwd(q, k, v, o)
    b = oapl.attention_fwd(q, k, v, o, workspace=a.workspace)
    assert torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse)
    x = oapl.attention_bwd(q, k, v, a.out, a.lse, dout, o)
    y = oapl.attention_bwd(q, k, v, a.out, a.lse, dout, o, workspace=x.workspace.fill_(0xA5))
    assert all(torch.equal(s, t) for s, t in zip(x[:3], y[:3]))


@pytest.mark.parametrize("q_offsets, k_offsets", [([1, 5, 9], [0, 5, 9]), ([0, 6, 4], [0, 5, 9]), ([0, 5, 8], [0, 5, 9]),
                                                  ([0, 5, 9], [0, 5, 10]), ([0, 5, 9], [0, -1, 9]), ([0, 2 ** 40, 9], [0, 5, 9])])
def test_malformed_offsets_are_reported_and_nothing_else_is_touched(q_offsets, k_offsets):
    q, k, v = _qkv("bf16", [9], [9], 4, 2, 64, seed=110)
    qo, ko = torch.tensor(q_offsets, device=DEV), torch.tensor(k_offsets, device=DEV)
    r = oapl.attention_fwd(q, k, v, qo, ko)
    assert oapl.read_device_status(r.workspace) == 4
    assert bool(r.out.isnan().all()) and bool(r.lse.isnan().all())
    b = oapl.attention_bwd(q, k, v, q, torch.zeros(9, 4, device=DEV), q, qo, ko)
    assert oapl.read_device_status(b.workspace) == 4
    assert all(bool(x.isnan().all()) for x in b[:3])
    good = torch.tensor([0, 5, 9], device=DEV)
    r = oapl.attention_fwd(q, k, v, good, k_used=torch.tensor([5, 5], device=DEV), workspace=r.workspace)
    assert oapl.read_device_status(r.workspace) == 4 and bool(r.out.isnan().all())
    r = oapl.attention_fwd(q, k, v, good, workspace=r.workspace)
    assert oapl.read_device_status(r.workspace) == 0 and bool(r.out.isfinite().all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nothing_is_written_outside_the_outputs(dtype):
    n, hq, hk, D = [37, 130], 6, 2, 80
    T, dt = sum(n), DTYPES[dtype]
    q, k, v = _qkv(dtype, n, n, hq, hk, D, seed=120)
    o, dout = _offsets(n), _normal(q.shape, dt, 123)

    def banded(shape, kind):
        size, band = math.prod(shape) * torch.empty(0, dtype=kind).element_size(), 1 << 16
        raw = torch.full((size + 2 * band,), 0xA5, dtype=torch.uint8, device=DEV)
        return raw, raw[band:band + size].view(kind).view(shape), band

    bwd_bytes = oapl.attention_workspace_bytes(T, T, 2, hq, hk, D, oapl._dtype_code(q), True)
    fwd_bytes = oapl.attention_workspace_bytes(T, T, 2, hq, hk, D, oapl._dtype_code(q), False)
    held = [banded(q.shape, dt), banded((fwd_bytes,), torch.uint8), banded(q.shape, dt), banded(k.shape, dt), banded(k.shape, dt),
            banded((bwd_bytes,), torch.uint8)]
    out, ws, dq, dk, dv, ws2 = (x[1] for x in held)
    r = oapl.attention_fwd(q, k, v, o, out=out, workspace=ws)
    oapl.attention_bwd(q, k, v, out, r.lse, dout, o, dq=dq, dk=dk, dv=dv, workspace=ws2)
    for raw, _, band in held:
        assert bool((raw[:band] == 0xA5).all()) and bool((raw[-band:] == 0xA5).all())
    assert all(bool(x.isfinite().all()) for x in (out, dq, dk, dv))


def test_rows_further_apart_than_32_bits_reach():
    """A cache whose rows lie 8 MiB apart: the last ones start behind 4 GiB."""
    n, D = 600, 64
    room = torch.empty(n, 4 << 20, dtype=torch.bfloat16, device=DEV)
    k, v = room[:, :D].unsqueeze(1), room[:, D:2 * D].unsqueeze(1)
    k.copy_(_normal((n, 1, D), torch.bfloat16, 130))
    v.copy_(_normal((n, 1, D), torch.bfloat16, 131))
    q = _normal((n, 2, D), torch.bfloat16, 132)
    o = _offsets([n])
    a, b = oapl.attention_fwd(q, k, v, o), oapl.attention_fwd(q, k.contiguous(), v.contiguous(), o)
    assert torch.equal(a.out, b.out)
    x = oapl.attention_bwd(q, k, v, a.out, a.lse, q, o)
    y = oapl.attention_bwd(q, k.contiguous(), v.contiguous(), a.out, a.lse, q, o)
    assert all(torch.equal(s, t) for s, t in zip(x[:3], y[:3]))
    few, last = q[:2].contiguous(), _offsets([2])
    a, b = oapl.attention_fwd(few, k, v, last, o), oapl.attention_fwd(few, k.contiguous(), v.contiguous(), last, o)
    assert torch.equal(a.out, b.out)


def test_no_sequences_no_queries_no_keys():
    q, k, v = _qkv("bf16", [0], [0], 4, 2, 64)
    r = oapl.attention_fwd(q, k, v, _offsets([]))
    assert r.out.shape == (0, 4, 64) and oapl.read_device_status(r.workspace) == 0
    q, k, v = _qkv("bf16", [0], [5], 4, 2, 64)
    r = oapl.attention_fwd(q, k, v, _offsets([0]), _offsets([5]))
    b = oapl.attention_bwd(q, k, v, r.out, r.lse, q, _offsets([0]), _offsets([5]))
    assert not b.dk.any() and not b.dv.any()
    q, k, v = _qkv("bf16", [5], [0], 4, 2, 64)
    r = oapl.attention_fwd(q, k, v, _offsets([5]), _offsets([0]))
    assert not r.out.any() and bool((r.lse == -math.inf).all())
    b = oapl.attention_bwd(q, k, v, r.out, r.lse, q, _offsets([5]), _offsets([0]))
    assert not b.dq.any()


def test_on_another_stream():
    n = [700, 300]
    q, k, v = _qkv("bf16", n, n, 8, 2, 128, seed=140)
    o = _offsets(n)
    want = oapl.attention_fwd(q, k, v, o)
    grads = oapl.attention_bwd(q, k, v, want.out, want.lse, q, o)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        x = q * 1.0
        got = oapl.attention_fwd(x, k, v, o)
        b = oapl.attention_bwd(x, k, v, got.out, got.lse, x, o)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got.out, want.out) and all(torch.equal(s, t) for s, t in zip(b[:3], grads[:3]))


def test_without_the_log_sum_exp():
    q, k, v = _qkv("bf16", [50], [50], 4, 2, 64, seed=150)
    r = oapl.attention_fwd(q, k, v, _offsets([50]), want_lse=False)
    assert r.lse is None and torch.equal(r.out, oapl.attention_fwd(q, k, v, _offsets([50])).out)


def test_refusals_of_the_binding():
    q, k, v = _qkv("bf16", [9], [9], 4, 2, 64)
    o = _offsets([9])
    with pytest.raises(oapl.OaplError):          # three key heads do not divide four query heads
        oapl.attention_fwd(q, k[:, :1].expand(9, 3, 64), v[:, :1].expand(9, 3, 64), o)
    with pytest.raises(oapl.OaplError):          # 2-byte steps between rows of 16-byte loads
        oapl.attention_fwd(torch.empty(9, 4 * 64 + 1, device=DEV, dtype=q.dtype)[:, 1:].unflatten(1, (4, 64)), k, v, o)
    with pytest.raises(TypeError):
        oapl.attention_fwd(q, k.float(), v, o)
    with pytest.raises(TypeError):
        oapl.attention_fwd(q.half(), k.half(), v.half(), o)
    with pytest.raises(TypeError):
        oapl.attention_fwd(q, k, v, o.int())
    with pytest.raises(ValueError):
        oapl.attention_fwd(q, k, v[:5], o)
    with pytest.raises(ValueError):
        oapl.attention_fwd(q, k.cpu(), v, o)
    with pytest.raises(oapl.OaplError):          # rows that are written must not overlap
        oapl.attention_fwd(q, k, v, o, out=torch.empty(9, 1, 64, device=DEV, dtype=q.dtype).expand(9, 4, 64))
    with pytest.raises(oapl.OaplError):
        oapl.attention_fwd(q, k, v, o, workspace=torch.empty(0, dtype=torch.uint8, device=DEV))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("n, hq, D", [(150, 4, 64), (9, 8, 128), (700, 2, 80)])
def test_what_is_not_finite_reaches_only_who_sees_it(dtype, bad, n, hq, D):
    """Causal: a key's or value's NaN stays out of the rows before it, a query's or gradient's out of the keys behind it."""
    at, hk = 2 * n // 3, 2
    o = _offsets([n])
    before, behind = torch.arange(at, device=DEV), torch.arange(at + 1, n, device=DEV)
    for which in range(4):
        q, k, v = _qkv(dtype, [n], [n], hq, hk, D, seed=160)
        dout = _normal(q.shape, q.dtype, 163)
        want = oapl.attention_fwd(q, k, v, o)
        grads = oapl.attention_bwd(q, k, v, want.out, want.lse, dout, o)
        (q, k, v, dout)[which][at] = bad
        got = oapl.attention_fwd(q, k, v, o)
        assert torch.equal(got.out[before], want.out[before]) and torch.equal(got.lse[before], want.lse[before])
        assert which == 3 or not bool(got.out[at].isfinite().all())
        b = oapl.attention_bwd(q, k, v, got.out, got.lse, dout, o)
        assert torch.equal(b.dq[before], grads.dq[before])
        if which in (0, 3):      # row `at` alone is touched: keys behind it do not see it
            assert torch.equal(b.dk[behind], grads.dk[behind]) and torch.equal(b.dv[behind], grads.dv[behind])
            assert not bool(b.dv[at].isfinite().all())


@pytest.mark.parametrize("nq, nk, hq, hk", [([300], [300], 32, 8), ([2500], [2500], 8, 1), ([64] * 16, [2000] * 16, 8, 8), ([1] * 3, [3000, 5, 900], 16, 8),
                                            ([1000], [1000], 6, 6)])
def test_cuts_give_the_same_in_fixed_order(nq, nk, hq, hk):
    """Sizes whose keys or rows are split over workgroups: within the bounds, and the same bits again."""
    _check("bf16", nq, nk, hq, hk, 128, True, seed=170)
    q, k, v = _qkv("bf16", nq, nk, hq, hk, 128, seed=174)
    qo, ko, dout = _offsets(nq), _offsets(nk), _normal(q.shape, q.dtype, 177)
    a, b = (oapl.attention_fwd(q, k, v, qo, ko) for _ in range(2))
    assert torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse)
    x, y = (oapl.attention_bwd(q, k, v, a.out, a.lse, dout, qo, ko) for _ in range(2))
    assert all(torch.equal(s, t) for s, t in zip(x[:3], y[:3]))


def test_in_a_graph_with_other_values():
    """A decode step and a training step replayed: new values and cached lengths, eager work between the replays."""
    nq, room, hq, hk, D = [1, 1, 1], 400, 8, 2, 128
    q, k, v = _qkv("bf16", nq, [room] * 3, hq, hk, D, seed=180)
    qo, ko, used = _offsets(nq), _offsets([room] * 3), torch.tensor([5, 400, 131], device=DEV)
    n = [70, 200]
    tq, tk, tv = _qkv("bf16", n, n, hq, hk, D, seed=184)
    to, dout = _offsets(n), _normal(tq.shape, tq.dtype, 187)

    def step():
        a = oapl.attention_fwd(q, k, v, qo, ko, k_used=used)
        b = oapl.attention_fwd(tq, tk, tv, to)
        return [a.out, a.lse, b.out, b.lse, *oapl.attention_bwd(tq, tk, tv, b.out, b.lse, dout, to)[:3]]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(4):
        for j, x in enumerate((q, k, v, tq, tk, tv, dout)):
            x.copy_(_normal(x.shape, x.dtype, 200 + 10 * i + j))
        used.copy_(torch.tensor([i, 400 - i, 64 * (i + 1)], device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, step()))


# Enough tiles for larger ones in some of the three kernels (which ones is asserted for the cases of test_gpu_attention_forms.py).
MANY = [("bf16", [1100, 70], [1100, 333], 48, 8), ("bf16", [1500], [1500], 32, 8), ("bf16", [5000], [5000], 8, 2),
        ("f32", [1000, 37, 600, 901, 300, 700, 650, 612], [1000, 37, 600, 901, 400, 600, 650, 612], 16, 16)]


@pytest.mark.parametrize("D", [16, 64, 80, 128])
@pytest.mark.parametrize("dtype, nq, nk, hq, hk", MANY)
def test_many_tiles(dtype, nq, nk, hq, hk, D):
    _check(dtype, nq, nk, hq, hk, D, True, seed=210)


def test_many_tiles_of_many_sequences():
    nq = [(7 * i * i + i) % 61 for i in range(300)]
    nk = [(5 * i * i + 3 * i) % 67 for i in range(300)]
    _check("f32", nq, nk, 16, 8, 64, True, seed=220)
    _check("bf16", nq, nk, 16, 8, 64, False, seed=223)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("dtype, n, hq, hk, D", [("bf16", 1500, 32, 8, 128), ("f32", 2100, 32, 32, 64)])
def test_what_is_not_finite_among_many_tiles(dtype, bad, n, hq, hk, D):
    at, o = 2 * n // 3 + 5, _offsets([n])
    for which in range(4):
        q, k, v = _qkv(dtype, [n], [n], hq, hk, D, seed=230)
        dout = _normal(q.shape, q.dtype, 233)
        want = oapl.attention_fwd(q, k, v, o)
        grads = oapl.attention_bwd(q, k, v, want.out, want.lse, dout, o)
        (q, k, v, dout)[which][at] = bad
        got = oapl.attention_fwd(q, k, v, o)
        assert torch.equal(got.out[:at], want.out[:at]) and torch.equal(got.lse[:at], want.lse[:at])
        assert which == 3 or not bool(got.out[at].isfinite().all())
        b = oapl.attention_bwd(q, k, v, got.out, got.lse, dout, o)
        assert torch.equal(b.dq[:at], grads.dq[:at])
        if which in (0, 3):
            assert torch.equal(b.dk[at + 1:], grads.dk[at + 1:]) and torch.equal(b.dv[at + 1:], grads.dv[at + 1:])
            assert not bool(b.dv[at].isfinite().all())


def test_large_tiles_of_many_sequences_and_in_fp32():
    """Long enough walks that tiles of 128 keys are taken, found by either search."""
    nq = [(7 * i * i + i) % 201 for i in range(66)]
    nk = [(5 * i * i + 3 * i) % 211 for i in range(66)]
    assert min(sum(nq), sum(nk)) >= 66 * 80
    _check("bf16", nq, nk, 64, 4, 64, True, seed=240)
    _check("f32", [2500], [2500], 32, 8, 64, True, seed=243)
    _check("f32", [1700, 800], [1700, 800], 32, 16, 128, True, seed=246)


@pytest.mark.parametrize("lengths, hq, hk, D", [([3500], 32, 8, 128), ([1600] * 11 + [1400], 8, 8, 64), ([1600] * 11 + [1400], 8, 8, 16),
                                                ([2100, 1900], 16, 8, 80), ([140] * 66, 64, 8, 128)])
def test_tiles_of_128_keys(lengths, hq, hk, D):
    _check("bf16", lengths, lengths, hq, hk, D, True, seed=250)


@pytest.mark.parametrize("bad", [math.nan, -math.inf])
def test_what_is_not_finite_among_tiles_of_128_keys(bad):
    test_what_is_not_finite_among_many_tiles("bf16", bad, 3500, 32, 8, 128)


@pytest.mark.parametrize("D", [80, 128])
def test_tiles_of_128_keys_of_wide_heads(D):
    _check("bf16", [2100, 2000, 1900, 2400], [2100, 2000, 1900, 2400], 16, 8, D, True, seed=260)


def test_what_is_not_finite_among_tiles_of_128_keys_of_wide_heads():
    test_what_is_not_finite_among_many_tiles("bf16", math.nan, 2100, 32, 32, 128)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D", [24, 64, 96, 128])
def test_tiles_of_64_rows(D, causal):
    _check("bf16", [1300, 900, 50], [1300, 1000, 700], 16, 8, D, causal, seed=270)
    _check("bf16", [1100, 0, 1200], [900, 700, 1200], 16, 8, D, causal, seed=273)


@pytest.mark.parametrize("causal", [True, False])
def test_one_long_sequence_of_few_tiles(causal):
    """Cut otherwise with a mask than without one."""
    _check("bf16", [1200], [1200], 8, 8, 128, causal, seed=280)
    _check("bf16", [2300], [2300], 6, 3, 128, causal, seed=283)
