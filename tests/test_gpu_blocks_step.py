"""Embedding, residual stream, attention, head and clipping together: the example's policy with norms against a plain model in 64
bits, and the calls of a step captured into graphs and on other streams."""
import math

import pytest
import torch

from examples import policy_step as ex
from paper_2602_19362_amd import oapl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F = torch.float64


def _policy(dtype):
    policy = ex.Policy(ex.Sizes(norms=True), dtype=dtype)
    gen = torch.Generator(device=DEV).manual_seed(3)
    for n in ("in_gain", "post_gain", "final_gain"):
        getattr(policy, n).copy_(1 + 0.2 * torch.randn(policy.sizes.hidden, generator=gen, device=DEV))
    return policy


def _batch(policy):
    prompts = [torch.arange(n, device=DEV, dtype=torch.int32) * 7 % 50 for n in (3, 3, 11, 11, 1, 1)]
    answers = [17, 30, 1, 9, 40, 22]
    texts, logq = ex.rollouts(policy, prompts, answers, seed=5)
    ids = torch.tensor([0, 0, 1, 1, 2, 2], dtype=torch.int32, device=DEV)
    return texts, answers, logq, torch.tensor([1.0, 0, 0, 1, 1, 1], device=DEV), ids


def _plain(policy, texts, answers, logq, rewards, ids, beta, w):
    """The same model's OAPL loss in 64 bits, one sequence at a time, from torch's elementary operations."""
    s = policy.sizes
    g, half, table = s.q_heads // s.k_heads, s.head_dim // 2, policy.cos_sin.to(F)

    def normed(x, gain):
        return x / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + 1e-6) * gain

    def turned(x, gain):
        x = normed(x, gain)
        c, n = table[:len(x), None, :half], table[:len(x), None, half:]
        return torch.cat((x[..., :half] * c - x[..., half:] * n, x[..., half:] * c + x[..., :half] * n), -1)

    deltas = []
    for i, (t, a) in enumerate(zip(texts, answers)):
        x = w["embedding"][t[:-1].long()]
        q, k, v = (normed(x, w["in_gain"]) @ w["qkv"].t()).unflatten(1, (-1, s.head_dim)).split((s.q_heads, s.k_heads, s.k_heads), 1)
        q, k = turned(q, w["q_gain"]), turned(k, w["k_gain"])
        out = []
        for h in range(s.q_heads):
            z = q[:, h] @ k[:, h // g].t() * s.head_dim ** -0.5
            z = z.masked_fill(torch.ones_like(z, dtype=torch.bool).triu(1), -math.inf)
            out.append(torch.softmax(z, 1) @ v[:, h // g])
        H = normed(x + normed(torch.cat(out, 1) @ w["out"].t(), w["post_gain"]), w["final_gain"])
        lp = torch.log_softmax(H[-a:] @ w["head"].t(), 1).gather(1, t[-a:].long()[:, None])[:, 0]
        deltas.append((lp - logq[i].to(F)).sum())
    loss = 0
    for i, d in enumerate(deltas):
        value = beta * torch.log(torch.exp(rewards[ids == ids[i]].to(F) / beta).mean())
        loss = loss + (beta * d - (rewards[i].to(F) - value)) ** 2
    return loss


def test_rollouts_and_the_packed_pass_give_the_same_log_probs():
    policy = _policy(torch.float32)
    texts, answers, logq, rewards, ids = _batch(policy)
    r = ex.train_step(policy, texts, answers, logq, rewards, ids, 3, beta=0.5)
    # fp32 throughout: the products over 256 and 1544 terms are summed in different orders in the two passes
    assert (r.logprob - torch.cat(logq)).abs().max() < 1e-4


@pytest.mark.parametrize("dtype, near", [(torch.float32, 1e-4), (torch.bfloat16, 0.07)])
def test_gradients_of_the_whole_step(dtype, near):
    """fp32: sums of a few thousand terms in other orders, 1e-4 of a gradient's norm.  bf16: eight roundings of up to 2^-8 on the way of a
    gradient from the head to the embedding (the head's, the norm's two, the product's, attention's two, the projection's, the norm's), half
    a per cent of it in root mean square, as many on the way up, through a loss whose residual multiplies log-prob errors (by up to ten
    here, 40 tokens' errors over a residual of 2): 7 %."""
    policy = _policy(dtype)
    texts, answers, logq, rewards, ids = _batch(policy)
    logq = [x - 0.05 for x in logq]           # a residual of some size
    r = ex.train_step(policy, texts, answers, logq, rewards, ids, 3, beta=0.5)
    assert {"in_gain", "post_gain", "final_gain", "embedding"} <= set(r.grads)
    weights = {n: getattr(policy, n).to(F).requires_grad_() for n in r.grads}
    loss = _plain(policy, texts, answers, logq, rewards, ids, 0.5, weights)
    loss.backward()
    assert abs(r.loss.item() - loss.item()) <= near * loss.item()
    for name, w in weights.items():
        assert (r.grads[name].to(F) - w.grad).norm() <= near * w.grad.norm(), name


@pytest.mark.parametrize("norms", [False, True])
def test_the_example_runs(norms, capsys):
    ex.main(3, norms=norms)
    lines = [x for x in capsys.readouterr().out.splitlines() if x.startswith("step")]
    assert len(lines) == 3 and all(math.isfinite(float(x.split()[-1])) for x in lines)


class Step:
    """The calls of a step below and above a product that stands for a block, every buffer held."""

    def __init__(self, T, d, V, seed, workspaces=None):
        g = torch.Generator(device=DEV).manual_seed(seed)

        def rand(*shape):
            return torch.randn(*shape, generator=g, device=DEV).bfloat16()

        self.E, self.W, self.gain, self.post, self.gate = rand(V, d), rand(d, d) / d ** 0.5, rand(d), rand(d), rand(d)
        self.tokens = (V * torch.rand(T, generator=g, device=DEV) ** 4).int().clamp_(max=V - 1)
        self.dn = rand(T, d)
        self.ws = workspaces or [torch.empty(n, dtype=torch.uint8, device=DEV) for n in (
            oapl.embed_workspace_bytes(T, d, V), oapl.residual_norm_workspace_bytes(T, d), oapl.clip_workspace_bytes(4))]

    def run(self):
        x = oapl.embed_fwd(self.E, self.tokens, scale=2.0)
        n = oapl.residual_norm_fwd(x, None, self.gain).out
        y = n @ self.W
        r = oapl.residual_norm_fwd(x, y, self.gain, y_gain=self.post, gate=self.gate, scale=0.5)
        b = oapl.residual_norm_bwd(r.x, y, None, self.dn, self.gain, y_gain=self.post, gate=self.gate, scale=0.5, workspace=self.ws[1])
        dy, sums = b.dy @ self.W.t(), [b.dgain.clone(), b.dy_gain, b.dgate]
        b = oapl.residual_norm_bwd(x, None, b.dx, dy, self.gain, workspace=self.ws[1])
        dE = oapl.embed_bwd(b.dx, self.tokens, len(self.E), scale=2.0, workspace=self.ws[0]).dE
        grads = [dE] + sums
        norm = oapl.clip_grads(grads, 1.0, workspace=self.ws[2]).norm
        return grads + [norm, r.out, b.dgain]


def _same(a, b):
    assert len(a) == len(b) and all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("T, d, V", [(5, 64, 30), (1500, 256, 1544), (9000, 264, 3000), (9000, 64, 300000)])
def test_replayed_graphs_give_the_eager_results(T, d, V):
    """Two graphs that share their workspaces, replayed in turn with eager work between, on other inputs in the same buffers."""
    a = Step(T, d, V, 1)
    b = Step(T, d, V, 2, a.ws)
    eager = [[x.clone() for x in s.run()] for s in (a, b)]
    graphs, outs = [], []
    for s in (a, b):
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(s.run())
        graphs.append(graph)
    for _ in range(3):
        for graph, out, want in zip(graphs, outs, eager):
            for x in out:
                x.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            _same(out, want)
            a.ws[0].fill_(255)      # eager work between replays
            _same(a.run(), eager[0])
    a.tokens.copy_(b.tokens), a.E.copy_(b.E), a.W.copy_(b.W), a.dn.copy_(b.dn)
    for n in ("gain", "post", "gate"):
        getattr(a, n).copy_(getattr(b, n))
    graphs[0].replay()
    torch.cuda.synchronize()
    _same(outs[0], eager[1])


def test_two_streams_at_once():
    steps = [Step(3000, 512, 900, 1), Step(2500, 512, 900, 2)]
    want = [[x.clone() for x in s.run()] for s in steps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(4):
        got = []
        for s, stream in zip(steps, streams):
            with torch.cuda.stream(stream):
                got.append(s.run())
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            _same(g, w)
