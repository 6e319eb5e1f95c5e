"""The embedding's gradient in numbers that are sums of whole ones below 2^24, so that every bit is known."""
import pytest
import torch

from paper_2602_19362_amd import oapl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_gradient_in_more_than_one_row_of_workgroups():
    """2^20 tokens of 65540 channels, all of which have the same row: 1064960 workgroups add rows up, 2^20 of them in a row of the launch.  A
    workspace of 8.6 GB."""
    T, d, V = 1 << 20, 65540, 3
    row = torch.randint(1, 8, (1, d), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    tokens = torch.randint(0, V, (T,), generator=torch.Generator(device=DEV).manual_seed(2), device=DEV, dtype=torch.int32)
    got = oapl.embed_bwd(row.bfloat16().expand(T, d), tokens, V).dE
    want = torch.bincount(tokens, minlength=V)[:, None] * row
    assert int(want.max()) < 1 << 24
    assert torch.equal(got, want.float())


def _exact(dout, tokens, V):
    """The sums as whole numbers.  No element of dout is zero, so a row that is missing or there twice shows in every channel."""
    assert bool((dout != 0).all())
    want = torch.zeros(V, dout.shape[1], dtype=torch.int64, device=DEV).index_add_(0, tokens.long(), dout.long())
    size = torch.zeros(V, dout.shape[1], dtype=torch.int64, device=DEV).index_add_(0, tokens.long(), dout.long().abs())
    assert int(size.max()) < 1 << 23      # in any order, so are the sums on the way, and what they are added to below
    return want


def _whole(T, d, dtype, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    sign = torch.randint(0, 2, (T, d), generator=gen, device=DEV) * 2 - 1
    # mostly positive, so that sums grow as those of magnitudes do
    sign = torch.where(torch.rand(T, 1, generator=gen, device=DEV) < 0.8, 1, sign)
    return (sign * torch.randint(1, 8, (T, d), generator=gen, device=DEV)).to(dtype)


def _check(dout, tokens, V, accumulate=False):
    want = _exact(dout, tokens, V)
    r = oapl.embed_bwd(dout, tokens, V)
    assert torch.equal(r.dE, want.float())
    if accumulate:
        old = torch.randint(-99, 100, want.shape, generator=torch.Generator(device=DEV).manual_seed(9), device=DEV)
        assert torch.equal(oapl.embed_bwd(dout, tokens, dE=old.float(), accumulate=True).dE, (want + old).float())


# Runs of one token that begin and end at steps of the search for where they do (64, 64^2, 64^3 sorted rows, and of tiles of 32 and 64 rows), and
# beside them; as many as 30000 tiles of one token.
RUNS = [(8192, 8192), (8192, 4096), (8192, 4095), (8192, 4097), (8192, 64), (8191, 6000), (9000, 2048), (9000, 2049), (100000, 65536), (262144, 131072),
        (262144, 131073), (262144, 131104), (262144, 200001), (262145, 262144), (300000, 262143), (300000, 262208), (600000, 524288), (600000, 524351),
        (600000, 570001), (2000000, 1900003)]


@pytest.mark.parametrize("T, run", RUNS)
def test_one_frequent_token(T, run):
    """Behind all others, before all others, and between them; its rows anywhere among theirs."""
    dout = _whole(T, 4, torch.float32, T + run)
    order = torch.randperm(T, generator=torch.Generator(device=DEV).manual_seed(run), device=DEV)
    behind = torch.arange(T, device=DEV).clamp_(max=T - run)
    between = torch.arange(T, device=DEV)
    at = (T - run) // 3
    between = torch.where(between < at, between, torch.where(between < at + run, at, between - run + 1))
    for tokens in (behind, T - run - behind, between):
        _check(dout, tokens[order].int(), T - run + 1)


# Both sides of the rules: sorting by counting or in passes, tiles of sorted rows, rows past the caches, few and many ids.
@pytest.mark.parametrize("dtype, T, d, V, kind", [
    ("bf16", 1, 8, 1, "one"), ("bf16", 4096, 520, 900, "one"), ("bf16", 4097, 520, 900, "one"), ("f32", 8192, 64, 1000, "zipf"), ("f32", 8193, 64, 1000, "zipf"),
    ("bf16", 8192, 66, 151936, "half"), ("bf16", 20011, 1024, 700, "zipf"), ("f32", 20011, 1025, 700, "half"), ("bf16", 40000, 2048, 8192, "zipf"),
    ("bf16", 100000, 64, 8192, "one"), ("f32", 100000, 65, 3, "even"), ("bf16", 140897, 260, 151936, "zipf"), ("bf16", 9000, 4100, 50, "half"),
    ("f32", 300001, 12, 70000, "zipf"), ("bf16", 262145, 3, 1 << 21, "even")])
def test_sums_of_whole_numbers(dtype, T, d, V, kind):
    gen = torch.Generator(device=DEV).manual_seed(T + d)
    if kind == "one":
        tokens = torch.full((T,), V - 1, device=DEV)
    elif kind == "zipf":
        tokens = (V * torch.rand(T, generator=gen, device=DEV, dtype=torch.float64) ** 8).long().clamp_(max=V - 1)
    else:
        tokens = torch.randint(0, V, (T,), generator=gen, device=DEV)
        if kind == "half":
            tokens[::2] = V // 2
    _check(_whole(T, d, {"bf16": torch.bfloat16, "f32": torch.float32}[dtype], 3), tokens.int(), V, accumulate=True)
