"""Very many sequences, whose offsets are looked at once for all workgroups."""
import pytest
import torch

from paper_2602_19362_amd import oapl
from tests.test_gpu_attention import DEV, _check, _normal, _offsets, _qkv

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n", [128, 129, 700, 1500])
def test_results(dtype, causal, n):
    """On both sides of the number from which one workgroup looks, and over several turns of its threads."""
    nq = [(7 * i * i + i) % 9 for i in range(n)]
    nk = [(5 * i * i + 3 * i) % 11 for i in range(n)]
    _check(dtype, nq, nk, 2, 1, 32, causal, seed=400)


@pytest.mark.parametrize("n", [129, 1500])
@pytest.mark.parametrize("where", ["first", "middle", "last", "falls", "used"])
def test_malformed_ones_are_reported(n, where):
    lengths = [1 + i % 3 for i in range(n)]
    T = sum(lengths)
    q, k, v = _qkv("bf16", lengths, lengths, 2, 1, 32, seed=410)
    good = _offsets(lengths)
    bad, used = good.clone(), torch.tensor(lengths, device=DEV)
    if where == "first":
        bad[0] = 1
    elif where == "middle":
        bad[n // 2] = 2 ** 40
    elif where == "last":
        bad[n] = T - 1
    elif where == "falls":
        bad[n - 3] = bad[n - 4] - 1
    else:
        used[n - 2] = 4
    if where == "used":
        r = oapl.attention_fwd(q, k, v, good, k_used=used)
    else:
        r = oapl.attention_fwd(q, k, v, good, bad)
        b = oapl.attention_bwd(q, k, v, q, torch.zeros(T, 2, device=DEV), q, good, bad)
        assert oapl.read_device_status(b.workspace) == 4 and all(bool(x.isnan().all()) for x in b[:3])
    assert oapl.read_device_status(r.workspace) == 4
    assert bool(r.out.isnan().all()) and bool(r.lse.isnan().all())
    r = oapl.attention_fwd(q, k, v, good, workspace=r.workspace)
    assert oapl.read_device_status(r.workspace) == 0 and bool(r.out.isfinite().all())


def test_time_does_not_grow_with_their_square():
    """16384 tokens as 1024 and as 16384 sequences: the tiles are 10.7 times as many, not 170 times the work (18.4 ms where every workgroup looked at all
    offsets); bounds between the two."""
    def least(n):
        lengths = [16384 // n] * n
        q, k, v = _qkv("bf16", lengths, lengths, 8, 8, 64, seed=420)
        o = _offsets(lengths)
        ws = oapl.attention_fwd(q, k, v, o).workspace
        times = []
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            oapl.attention_fwd(q, k, v, o, workspace=ws)
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    assert least(16384) < 40 * least(1024) and least(16384) < 5.0


def test_in_a_graph_with_other_lengths():
    """Replayed with other offsets, malformed ones among them: every replay looks for itself."""
    n, total = 300, 900
    q, k, v = _qkv("bf16", [total], [total], 2, 1, 32, seed=430)
    o = torch.arange(n + 1, device=DEV) * 3
    ws = oapl.attention_fwd(q, k, v, o).workspace
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = oapl.attention_fwd(q, k, v, o, workspace=ws)
    for i in range(4):
        x = torch.arange(n + 1, device=DEV) * 3
        x[1:n:2] += i % 3 - 1
        o.copy_(x)
        if i == 2:
            o[n] = total + 1
        q.copy_(_normal(q.shape, q.dtype, 440 + i))
        graph.replay()
        torch.cuda.synchronize()
        want = oapl.attention_fwd(q, k, v, o)
        assert oapl.read_device_status(ws) == oapl.read_device_status(want.workspace) == (4 if i == 2 else 0)
        assert torch.equal(held.out.nan_to_num(7.0), want.out.nan_to_num(7.0))
