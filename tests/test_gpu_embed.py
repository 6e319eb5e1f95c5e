"""Embedding lookup and its gradient against the 64-bit oracle within its error bounds."""
import pytest
import torch

from oracle import blocks_oracle as orc
from paper_2602_19362_amd import oapl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _tokens(kind, T, V, seed=0):
    """even: any; zipf: few very frequent ones; one: the same; each: all different as far as there are (shuffled); ends: the two last rows."""
    g = _gen(seed)
    if kind == "even":
        return torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    if kind == "zipf":
        return (V * torch.rand(T, generator=g, device=DEV, dtype=torch.float64) ** 12).to(torch.int32).clamp_(max=V - 1)
    if kind == "one":
        return torch.full((T,), V // 2, device=DEV, dtype=torch.int32)
    if kind == "ends":
        return (V - 1 - torch.randint(0, min(2, V), (T,), generator=g, device=DEV)).to(torch.int32)
    return (torch.randperm(T, generator=g, device=DEV) % V).to(torch.int32)


def near(got, want, bound):
    assert got.shape == want.shape
    off = (got.to(torch.float64) - want).abs()
    assert bool((off <= bound + 1e-300).all()), float((off / (bound + 1e-300)).max())


@pytest.mark.parametrize("dtype, out, T, d, V, scale", [
    ("bf16", "bf16", 1, 8, 1, 1.0), ("bf16", "bf16", 64, 4096, 1000, 1.0), ("bf16", "f32", 37, 520, 300, 22.6), ("f32", "f32", 5, 7, 3, -0.3),
    ("f32", "bf16", 333, 65, 50, 3.0), ("bf16", "bf16", 3001, 1, 9, 0.1), ("f32", "f32", 70001, 12, 2000, 1.7), ("bf16", "bf16", 3, 8200, 5, 0.0),
    # results past the caches
    ("bf16", "bf16", 140000, 1000, 3000, 1.1), ("f32", "f32", 70000, 1001, 3000, 0.9), ("bf16", "f32", 300000, 250, 300, 1.0)])
def test_lookup(dtype, out, T, d, V, scale):
    E = torch.randn(V, d, generator=_gen(1), device=DEV).to(DTYPES[dtype])
    tokens = _tokens("even", T, V)
    got = oapl.embed_fwd(E, tokens, scale=scale, out_dtype=DTYPES[out])
    assert got.dtype == DTYPES[out]
    near(got, *orc.embed(E, tokens, scale, DTYPES[out]))


def test_lookup_from_and_into_parts_of_buffers():
    """An embedding that starts at any element, rows of the output further apart than their channels and not aligned either."""
    for dtype in DTYPES.values():
        E = torch.randn(1 + 40 * 72, generator=_gen(2), device=DEV).to(dtype)[1:].view(40, 72)
        tokens = _tokens("even", 29, 40)
        wide = torch.full((29, 101), 7.0, device=DEV, dtype=dtype)
        got = oapl.embed_fwd(E, tokens, scale=1.5, out=wide[:, 3:75])
        assert got.data_ptr() == wide.data_ptr() + 3 * wide.element_size()
        near(got, *orc.embed(E, tokens, 1.5, dtype))
        assert bool((wide[:, :3] == 7).all()) and bool((wide[:, 75:] == 7).all())


def test_lookup_outside_the_embedding_is_nan():
    E = torch.randn(10, 24, generator=_gen(3), device=DEV)
    tokens = torch.tensor([3, 10, -1, 9, 2 ** 31 - 1, -2 ** 31, 0], device=DEV, dtype=torch.int32)
    got = oapl.embed_fwd(E, tokens)
    assert got.isnan().all(1).tolist() == [False, True, True, False, True, True, False]
    assert torch.equal(got[[0, 3, 6]], E[[3, 9, 0]])


def test_lookup_without_tokens():
    assert oapl.embed_fwd(torch.zeros(3, 4, device=DEV), torch.zeros(0, device=DEV, dtype=torch.int32)).shape == (0, 4)


CASES = [("bf16", 1, 8, 1, "one"), ("bf16", 5, 64, 100, "even"), ("f32", 63, 20, 17, "zipf"), ("f32", 64, 20, 17, "one"), ("bf16", 65, 7, 64, "one"),
         ("bf16", 1000, 264, 1544, "zipf"), ("f32", 1501, 768, 8192, "even"), ("bf16", 2048, 40, 2047, "each"), ("bf16", 2049, 9, 2048, "ends"),
         ("f32", 5000, 33, 3000, "zipf"), ("bf16", 4097, 1024, 151936, "each"), ("bf16", 20000, 520, 700, "zipf"), ("f32", 20011, 8, 5, "even"),
         ("bf16", 30000, 2056, 32000, "one"), ("f32", 300001, 4, 70000, "zipf"), ("bf16", 262145, 3, 1 << 21, "even"), ("f32", 9000, 1, 1 << 21, "ends")]


# On both sides of the rules: sorting by counting or in passes, tiles of sorted rows, rows past the caches.
RULES = [("bf16", 8192, 512, 700, "zipf"), ("bf16", 8193, 512, 700, "zipf"), ("bf16", 4096, 516, 900, "one"), ("f32", 4097, 516, 900, "zipf"),
         ("bf16", 8192, 2050, 300, "zipf"), ("f32", 262144, 12, 5000, "zipf"), ("f32", 262145, 12, 5000, "zipf"), ("bf16", 8192, 4096, 500, "even"),
         ("bf16", 8193, 4096, 500, "even"), ("f32", 4097, 4099, 300, "zipf"), ("bf16", 100000, 64, 8192, "one"), ("f32", 20000, 66, 1000, "one")]


@pytest.mark.parametrize("dtype, T, d, V, kind", CASES)
def test_gradient(dtype, T, d, V, kind):
    tokens = _tokens(kind, T, V)
    dout = torch.randn(T, d, generator=_gen(4), device=DEV).to(DTYPES[dtype])
    r = oapl.embed_bwd(dout, tokens, V, scale=0.7)
    assert r.dE.dtype == torch.float32
    want, bound = orc.embed_grads(dout, tokens, V, 0.7)
    near(r.dE, want, bound)
    assert oapl.read_device_status(r.workspace) == 0
    # added to what is there
    old = torch.randn(V, d, generator=_gen(5), device=DEV)
    into = old.clone()
    again = oapl.embed_bwd(dout, tokens, scale=0.7, dE=into, accumulate=True, workspace=r.workspace)
    assert again.dE is into
    want, bound = orc.embed_grads(dout, tokens, V, 0.7, old=old)
    near(into, want, bound)
    absent = torch.ones(V, dtype=torch.bool, device=DEV)
    absent[tokens.long()] = False
    assert torch.equal(into[absent], old[absent])
    # the same bits again, on a workspace and a result that held something else
    r.workspace.fill_(255)
    third = oapl.embed_bwd(dout, tokens, scale=0.7, dE=torch.full_like(r.dE, torch.nan), workspace=r.workspace)
    assert torch.equal(third.dE, r.dE)


def _want(dout, tokens, V):
    """The oracle on the CPU, which adds up many rows of one token sooner."""
    return [x.to(DEV) for x in orc.embed_grads(dout.cpu(), tokens.cpu(), V, 1.0)]


@pytest.mark.parametrize("dtype, T, d, V, kind", RULES)
def test_gradient_beside_the_rules(dtype, T, d, V, kind):
    tokens = _tokens(kind, T, V)
    dout = torch.randn(T, d, generator=_gen(4), device=DEV).to(DTYPES[dtype])
    r = oapl.embed_bwd(dout, tokens, V)
    near(r.dE, *_want(dout, tokens, V))
    r.workspace.fill_(255)
    again = oapl.embed_bwd(dout, tokens, dE=torch.full_like(r.dE, torch.nan), workspace=r.workspace)
    assert torch.equal(again.dE, r.dE)


@pytest.mark.parametrize("T, d", [(500, 40), (7000, 64), (9001, 64), (9001, 70), (50000, 256)])
def test_gradient_of_a_padded_batch(T, d):
    """Half of the tokens are the same one, and tokens outside the embedding lie among them."""
    V = 1544
    tokens = _tokens("even", T, V)
    tokens[1::2] = 7
    tokens[::97] = V
    dout = torch.randn(T, d, generator=_gen(6), device=DEV).bfloat16()
    r = oapl.embed_bwd(dout, tokens, V)
    assert oapl.read_device_status(r.workspace) != 0
    inside = tokens < V
    near(r.dE, *_want(dout[inside], tokens[inside], V))



@pytest.mark.parametrize("T", [6, 3000])
def test_gradient_of_tokens_outside_the_embedding(T):
    tokens = _tokens("even", T, 50)
    tokens[::3] = torch.tensor([50, -1, 2 ** 31 - 1, -2 ** 31], device=DEV, dtype=torch.int32).repeat(T)[:len(tokens[::3])]
    dout = torch.randn(T, 24, generator=_gen(6), device=DEV)
    dout[::3] = torch.nan
    r = oapl.embed_bwd(dout, tokens, 50)
    near(r.dE, *orc.embed_grads(dout, tokens, 50, 1.0))
    assert oapl.read_device_status(r.workspace) == 9
    r = oapl.embed_bwd(dout, tokens.clamp(0, 49), 50, workspace=r.workspace)
    assert oapl.read_device_status(r.workspace) == 0


@pytest.mark.parametrize("T", [7, 2500])
def test_gradient_from_and_into_parts_of_buffers(T):
    for dtype in DTYPES.values():
        wide = torch.randn(T, 91, generator=_gen(7), device=DEV).to(dtype)
        tokens = _tokens("zipf", T, 60)
        flat = torch.full((2 + 60 * 73,), 5.0, device=DEV)
        r = oapl.embed_bwd(wide[:, 5:78], tokens, dE=flat[1:-1].view(60, 73))
        near(r.dE, *orc.embed_grads(wide[:, 5:78], tokens, 60, 1.0))
        assert flat[0] == 5 and flat[-1] == 5
        # one row for all tokens
        row = wide[:1, 5:78].expand(T, 73)
        near(oapl.embed_bwd(row, tokens, 60).dE, *orc.embed_grads(row, tokens, 60, 1.0))


@pytest.mark.parametrize("T, d, V", [(0, 8, 3), (5, 24, 60), (8000, 40, 300), (9000, 72, 3000), (9000, 1024, 3000)])
def test_nothing_beside_the_buffers_is_touched(T, d, V):
    """A workspace of the bytes that the call asks for, and dE, inside larger buffers."""
    n = oapl.embed_workspace_bytes(T, d, V)
    room = torch.full((n + 512,), 0x5a, dtype=torch.uint8, device=DEV)
    flat = torch.full((V * d + 64,), 7.0, device=DEV)
    tokens = _tokens("zipf", T, V)
    dout = torch.randn(T, d, generator=_gen(11), device=DEV)
    oapl.embed_bwd(dout, tokens, dE=flat[32:-32].view(V, d), workspace=room[256:256 + n])
    near(flat[32:-32].view(V, d), *orc.embed_grads(dout, tokens, V, 1.0))
    assert bool((room[:256] == 0x5a).all()) and bool((room[256 + n:] == 0x5a).all())
    assert bool((flat[:32] == 7).all()) and bool((flat[-32:] == 7).all())


def test_what_is_not_finite_stays_in_its_row():
    tokens = _tokens("zipf", 4000, 500)
    dout = torch.randn(4000, 16, generator=_gen(8), device=DEV)
    dout[17, 3], dout[1234, 9] = torch.inf, torch.nan
    got = oapl.embed_bwd(dout, tokens, 500).dE
    want = torch.ones_like(got, dtype=torch.bool)
    want[tokens[17], 3], want[tokens[1234], 9] = False, False
    assert torch.equal(got.isfinite(), want)


@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_without_tokens(accumulate):
    dE = torch.full((30, 12), 3.0, device=DEV)
    oapl.embed_bwd(torch.zeros(0, 12, device=DEV), torch.zeros(0, device=DEV, dtype=torch.int32), dE=dE, accumulate=accumulate)
    assert bool((dE == (3 if accumulate else 0)).all())


def test_the_same_weights_at_both_ends():
    """A tied embedding's gradient: the head's dW with the lookup's rows added to it."""
    W = (torch.randn(600, 64, generator=_gen(9), device=DEV) / 8).bfloat16()
    tokens = _tokens("zipf", 200, 600)
    H = torch.randn(200, 64, generator=_gen(10), device=DEV).bfloat16()
    offsets = torch.tensor([0, 120, 200], device=DEV)
    r = oapl.loss_fwd_bwd(H, W, tokens, torch.full((200,), -6.0, device=DEV), offsets, torch.tensor([1.0, 0.0], device=DEV),
                          torch.zeros(2, dtype=torch.int32, device=DEV), 1, 0.5)
    before = r.dW.clone()
    oapl.embed_bwd(r.dH, tokens, dE=r.dW, accumulate=True)
    near(r.dW, *orc.embed_grads(r.dH, tokens, 600, 1.0, old=before))


@pytest.mark.parametrize("T, d, V", [(300, 40, 77), (9000, 24, 500)])
def test_the_gradient_is_the_lookups_difference(T, d, V):
    """The lookup is linear, so a difference along a direction is off by roundings alone: of the two products (2^-24 each), of the moved
    embedding (2^-24, of what it holds), and of the gradient by the oracle's bound."""
    F, h = torch.float64, 0.5
    E, way = (torch.randn(V, d, generator=_gen(i), device=DEV) for i in (12, 13))
    tokens, dout = _tokens("zipf", T, V), torch.randn(T, d, generator=_gen(14), device=DEV)
    hi, lo = (oapl.embed_fwd(E + s * h * way, tokens, scale=1.5) for s in (1, -1))
    quotient = (dout.to(F) * (hi.to(F) - lo.to(F))).sum() / (2 * h)
    slope = (oapl.embed_bwd(dout, tokens, V, scale=1.5).dE.to(F) * way).sum()
    bound = (dout.to(F).abs() * (hi.to(F).abs() + lo.to(F).abs())).sum() * 2 * 2.0 ** -24 / (2 * h)
    bound += (orc.embed_grads(dout, tokens, V, 1.5)[1] * way.abs()).sum()
    assert abs(quotient - slope) <= bound


def test_refusals():
    E, t = torch.zeros(5, 8, device=DEV), torch.zeros(3, device=DEV, dtype=torch.int32)
    with pytest.raises(TypeError):
        oapl.embed_fwd(E, t.long())
    with pytest.raises(TypeError):
        oapl.embed_fwd(E.half(), t)
    with pytest.raises(ValueError):
        oapl.embed_fwd(E[:, ::2], t)
    with pytest.raises(ValueError):
        oapl.embed_fwd(E, t, out=torch.zeros(3, 9, device=DEV))
    with pytest.raises(TypeError):
        oapl.embed_fwd(E, t, out=torch.zeros(3, 8, device=DEV), out_dtype=torch.bfloat16)
    with pytest.raises(oapl.OaplError):
        oapl.embed_fwd(E, t, scale=float("inf"))
    with pytest.raises(oapl.OaplError):
        oapl.embed_fwd(E, t, out=torch.zeros(1, 8, device=DEV).expand(3, 8))
    with pytest.raises(ValueError):
        oapl.embed_bwd(E, t, 5)
    with pytest.raises(ValueError):
        oapl.embed_bwd(E[:3], t)
    with pytest.raises(ValueError):
        oapl.embed_bwd(E[:3], t, 5, accumulate=True)
    with pytest.raises(ValueError):
        oapl.embed_bwd(E[:3], t, 5, dE=torch.zeros(6, 8, device=DEV))
    with pytest.raises(TypeError):
        oapl.embed_bwd(E[:3], t, dE=torch.zeros(5, 8, device=DEV).bfloat16())
    with pytest.raises(oapl.OaplError):
        oapl.embed_bwd(E[:3], t, 5, workspace=torch.zeros(255, device=DEV, dtype=torch.uint8))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("d", [1, 2, 3, 5, 6, 7, 9, 11, 253, 254, 255, 257, 509, 515, 1023, 1029])
def test_widths_that_end_inside_a_piece(dtype, d):
    """With NaN on both sides of every row of the gradient, and of the embedding."""
    for T, V in ((41, 6), (8300, 60)):
        tokens = _tokens("zipf", T, V)
        E = torch.full((V * d + 40,), torch.nan, device=DEV, dtype=DTYPES[dtype])
        E[11:11 + V * d] = torch.randn(V * d, generator=_gen(d), device=DEV)
        rows = E[11:11 + V * d].view(V, d)
        assert torch.equal(oapl.embed_fwd(rows, tokens), rows[tokens.long()])
        wide = torch.full((T, d + 20), torch.nan, device=DEV, dtype=DTYPES[dtype])
        wide[:, 9:9 + d] = torch.randn(T, d, generator=_gen(d + 1), device=DEV)
        dout = wide[:, 9:9 + d]
        into = torch.full((V * d + 40,), 3.0, device=DEV)
        dE = into[13:13 + V * d].view(V, d)
        oapl.embed_bwd(dout, tokens, dE=dE)
        near(dE, *orc.embed_grads(dout, tokens, V, 1.0))
        assert bool((into[:13] == 3).all()) and bool((into[13 + V * d:] == 3).all())


@pytest.mark.parametrize("T, run", [(8192, 8192), (8192, 4096), (8192, 4161), (5000, 95), (5000, 96), (5000, 97), (5000, 160), (5000, 4160), (9000, 2048),
                                    (9000, 2049), (140000, 131072), (140000, 139999), (262144, 200001)])
def test_one_token_among_others(T, run):
    """Its sorted rows end, and begin, at steps of the search for where they do, and beside them."""
    V = 50
    tokens = _tokens("even", T, V)
    tokens[torch.randperm(T, generator=_gen(7), device=DEV)[:run]] = 23
    dout = torch.randn(T, 8, generator=_gen(8), device=DEV)
    near(oapl.embed_bwd(dout, tokens, V).dE, *_want(dout, tokens, V))
    tokens = torch.arange(T, device=DEV, dtype=torch.int32).clamp_(max=T - run)         # all others before it, and behind it
    near(oapl.embed_bwd(dout, tokens, T).dE, *_want(dout, tokens, T))
    tokens = (tokens - (T - run)).neg_()
    near(oapl.embed_bwd(dout, tokens, T).dE, *_want(dout, tokens, T))
