"""The example's policy: rollouts over a cache against the packed pass, and its gradients against a plain model's in 64 bits."""
import math

import pytest
import torch

from examples import policy_step as ex

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F = torch.float64


def _batch(policy):
    prompts = [torch.arange(n, device=DEV, dtype=torch.int32) * 7 % 50 for n in (3, 3, 11, 11, 1, 1)]
    answers = [17, 30, 1, 9, 40, 22]
    texts, logq = ex.rollouts(policy, prompts, answers, seed=5)
    ids = torch.tensor([0, 0, 1, 1, 2, 2], dtype=torch.int32, device=DEV)
    rewards = torch.tensor([1.0, 0, 0, 1, 1, 1], device=DEV)
    return texts, answers, logq, rewards, ids


def _plain(policy, texts, answers, logq, rewards, ids, beta, weights):
    """The same model's OAPL loss in 64 bits, one sequence at a time, from torch's elementary operations."""
    s = policy.sizes
    g = s.q_heads // s.k_heads
    table = policy.cos_sin.to(F)
    half = s.head_dim // 2

    def turned(x, gain):
        x = x / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + 1e-6) * gain
        c, n = table[:len(x), None, :half], table[:len(x), None, half:]
        return torch.cat((x[..., :half] * c - x[..., half:] * n, x[..., half:] * c + x[..., :half] * n), -1)

    deltas = []
    for i, (t, a) in enumerate(zip(texts, answers)):
        x = weights["embedding"][t[:-1].long()]
        q, k, v = (x @ weights["qkv"].t()).unflatten(1, (-1, s.head_dim)).split((s.q_heads, s.k_heads, s.k_heads), 1)
        q, k = turned(q, weights["q_gain"]), turned(k, weights["k_gain"])
        out = []
        for h in range(s.q_heads):
            z = q[:, h] @ k[:, h // g].t() * s.head_dim ** -0.5
            z = z.masked_fill(torch.ones_like(z, dtype=torch.bool).triu(1), -math.inf)
            out.append(torch.softmax(z, 1) @ v[:, h // g])
        H = x + torch.cat(out, 1) @ weights["out"].t()
        lp = torch.log_softmax(H[-a:] @ weights["head"].t(), 1).gather(1, t[-a:].long()[:, None])[:, 0]
        deltas.append((lp - logq[i].to(F)).sum())
    loss = 0
    for i, d in enumerate(deltas):
        mine = rewards[ids == ids[i]].to(F)
        value = beta * torch.log(torch.exp(mine / beta).mean())
        loss = loss + (beta * d - (rewards[i].to(F) - value)) ** 2
    return loss


def test_rollouts_and_the_packed_pass_give_the_same_log_probs():
    policy = ex.Policy(dtype=torch.float32)
    texts, answers, logq, rewards, ids = _batch(policy)
    r = ex.train_step(policy, texts, answers, logq, rewards, ids, 3, beta=0.5)
    # fp32 throughout: the products over 256 and 1544 terms are summed in different orders in the two passes
    assert (r.logprob - torch.cat(logq)).abs().max() < 1e-4


@pytest.mark.parametrize("dtype, near", [(torch.float32, 1e-4), (torch.bfloat16, 0.05)])
def test_gradients_of_the_whole_step(dtype, near):
    """fp32: sums of a few thousand terms in other orders, 1e-4 of a gradient's norm.  bf16: five roundings of 2^-8 on the way of a
    gradient from the head to the embedding, each taking its root mean square of up to 2^-8 / sqrt(3) of it, through a loss
    whose residual multiplies log-prob errors: 5 %."""
    policy = ex.Policy(dtype=dtype)
    texts, answers, logq, rewards, ids = _batch(policy)
    logq = [x - 0.05 for x in logq]           # a residual of some size
    r = ex.train_step(policy, texts, answers, logq, rewards, ids, 3, beta=0.5)
    weights = {n: getattr(policy, n).to(F).requires_grad_() for n in r.grads}
    loss = _plain(policy, texts, answers, logq, rewards, ids, 0.5, weights)
    loss.backward()
    assert abs(r.loss.item() - loss.item()) <= near * loss.item()
    for name, w in weights.items():
        assert (r.grads[name].to(F) - w.grad).norm() <= near * w.grad.norm(), name


def test_the_example_runs_and_its_loss_falls(capsys):
    ex.main(8)
    lines = [x for x in capsys.readouterr().out.splitlines() if x.startswith("step")]
    losses = [float(x.split()[-1]) for x in lines]
    assert len(losses) == 8 and losses[-1] < 0.5 * losses[0] and all(math.isfinite(x) for x in losses)
