"""A policy of one attention layer, from rollouts to an OAPL step, on this library's operators.

    python examples/policy_step.py [steps [norms]]

Rollouts: prompts go through the layer in one packed call that fills a key / value cache, then one token per rollout and call
(embed_fwd, qk_norm_rope_fwd into the cache, attention_fwd over it, residual_norm_fwd, sample_tokens and logprob_fwd on the head).
Training: the rollouts packed back to back through the same calls, the objective and its gradient at the head (loss_fwd_bwd), and
down again (residual_norm_bwd, attention_bwd, qk_norm_rope_bwd, embed_bwd); the projections are plain matrix products of torch
here, as is the update, whose step goes by the gradients' norm (grad_norm).  The layer has no feed-forward part, and norms before
it, behind it and under the head only where `norms` asks for them: what is shown is how the operators meet.
"""
import os
import sys
from typing import NamedTuple

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2602_19362_amd import oapl  # noqa: E402


class Sizes(NamedTuple):
    hidden: int = 256
    vocabulary: int = 1544
    q_heads: int = 8
    k_heads: int = 2
    head_dim: int = 64
    longest: int = 96          # tokens of a prompt and its answer
    norms: bool = False        # of the residual stream, with gains, and of the layer's output


class Policy:
    """Weights in bf16 (gradients and updates in fp32), all on one GPU."""

    def __init__(self, sizes=Sizes(), seed=0, device="cuda:0", dtype=torch.bfloat16):
        s = self.sizes = sizes
        gen = torch.Generator(device=device).manual_seed(seed)

        def weights(*shape, scale):
            return (torch.randn(*shape, generator=gen, device=device) * scale).to(dtype)

        rows = (s.q_heads + 2 * s.k_heads) * s.head_dim
        self.embedding = weights(s.vocabulary, s.hidden, scale=1.0)
        self.qkv = weights(rows, s.hidden, scale=s.hidden ** -0.5)
        self.out = weights(s.hidden, s.q_heads * s.head_dim, scale=(s.q_heads * s.head_dim) ** -0.5)
        self.head = weights(s.vocabulary, s.hidden, scale=s.hidden ** -0.5)
        self.q_gain, self.k_gain = (torch.ones(s.head_dim, device=device, dtype=dtype) for _ in range(2))
        self.in_gain, self.post_gain, self.final_gain = (
            torch.ones(s.hidden, device=device, dtype=dtype) if s.norms else None for _ in range(3))
        angle = torch.arange(s.longest, dtype=torch.float64)[:, None] * 1e4 ** (
            -torch.arange(0, s.head_dim, 2, dtype=torch.float64) / s.head_dim)
        self.cos_sin = torch.cat((angle.cos(), angle.sin()), 1).float().to(device)

    def embedded(self, tokens):
        """The residual stream of tokens, and what the projections take."""
        x = oapl.embed_fwd(self.embedding, tokens)
        return x, x if self.in_gain is None else oapl.residual_norm_fwd(x, None, self.in_gain).out

    def projected(self, n):
        """Queries, keys and values of the rows n, as views of one product."""
        s = self.sizes
        return (n @ self.qkv.t()).unflatten(1, (-1, s.head_dim)).split((s.q_heads, s.k_heads, s.k_heads), 1)

    def hidden(self, x, attended):
        """The layer's output, the residual stream behind it, and what the head takes."""
        y = attended.flatten(1) @ self.out.t()
        r = oapl.residual_norm_fwd(x, y, self.final_gain, y_gain=self.post_gain)
        return y, r.x, r.x if r.out is None else r.out


class Cache:
    """Keys and values of n sequences with room for `longest` tokens each."""

    def __init__(self, policy, n):
        s, like = policy.sizes, policy.embedding
        self.k, self.v = (like.new_zeros((n * s.longest, s.k_heads, s.head_dim)) for _ in range(2))
        self.offsets = torch.arange(n + 1, device=like.device) * s.longest
        self.used = torch.zeros(n, dtype=torch.int64, device=like.device)

    def extend(self, policy, tokens, q_offsets, positions, seq):
        """The final hidden states of new tokens (packed; token i belongs to sequence seq[i], at positions[i] of it)."""
        x, n = policy.embedded(tokens)
        q, k, v = policy.projected(n)
        rows = self.offsets[seq] + positions
        q = oapl.qk_norm_rope_fwd(q, k, positions.int(), policy.cos_sin, policy.q_gain, policy.k_gain, v=v, rows=rows, k_out=self.k,
                                  v_out=self.v).q
        self.used += q_offsets.diff()
        a = oapl.attention_fwd(q, self.k, self.v, q_offsets, self.offsets, k_used=self.used, want_lse=False).out
        return policy.hidden(x, a)[2]


def rollouts(policy, prompts, answers, seed, temperature=1.0):
    """`answers[i]` sampled tokens behind each prompt; (tokens of prompt and answer, log-probs of the answer) by sequence."""
    n, device = len(prompts), policy.embedding.device
    lengths = torch.tensor([len(p) for p in prompts], device=device)
    offsets = torch.zeros(n + 1, dtype=torch.int64, device=device)
    offsets[1:] = lengths.cumsum(0)
    seq = torch.repeat_interleave(torch.arange(n, device=device), lengths)
    cache = Cache(policy, n)
    H = cache.extend(policy, torch.cat(prompts), offsets, torch.arange(int(offsets[-1]), device=device) - offsets[seq], seq)
    h = H[offsets[1:] - 1].contiguous()
    one, all_seq = torch.arange(n + 1, device=device), torch.arange(n, device=device)
    tokens, logq = [], []
    for step in range(max(answers)):
        t, _ = oapl.sample_tokens(h, policy.head, temperature, seed + step)
        tokens.append(t)
        logq.append(oapl.logprob_fwd(h, policy.head, t)[0])
        if step + 1 < max(answers):
            h = cache.extend(policy, t, one, cache.used.clone(), all_seq)
    tokens, logq = torch.stack(tokens, 1), torch.stack(logq, 1)
    return [torch.cat((p, tokens[i, :answers[i]])) for i, p in enumerate(prompts)], [logq[i, :answers[i]] for i in range(n)]


class Step(NamedTuple):
    loss: torch.Tensor
    logprob: torch.Tensor
    grads: dict


def train_step(policy, texts, answers, logq, rewards, group_ids, n_groups, beta):
    """The OAPL loss of rollouts and its gradients with respect to every weight."""
    s, device = policy.sizes, policy.embedding.device
    fed = [len(t) - 1 for t in texts]                   # the last token is predicted, not fed
    offsets = torch.tensor([0] + fed, device=device).cumsum(0)
    tokens = torch.cat([t[:-1] for t in texts])
    positions = torch.cat([torch.arange(n, device=device, dtype=torch.int32) for n in fed])
    # rows that predict an answer's tokens, and these
    scored = torch.cat([offsets[i] + torch.arange(fed[i] - a, fed[i], device=device) for i, a in enumerate(answers)])
    targets = torch.cat([t[-a:] for t, a in zip(texts, answers)])

    x, n = policy.embedded(tokens)
    q0, k0, v = policy.projected(n)
    turned = oapl.qk_norm_rope_fwd(q0, k0, positions, policy.cos_sin, policy.q_gain, policy.k_gain)
    a = oapl.attention_fwd(turned.q, turned.k, v, offsets)
    y, behind, H = policy.hidden(x, a.out)

    answer_offsets = torch.tensor([0] + list(answers), device=device).cumsum(0)
    r = oapl.loss_fwd_bwd(H[scored].contiguous(), policy.head, targets, torch.cat(logq), answer_offsets, rewards, group_ids, n_groups, beta)

    dH = torch.zeros_like(H)
    dH[scored] = r.dH
    grads = {}
    dx, dy = dH, dH
    if s.norms:
        g = oapl.residual_norm_bwd(behind, y, None, dH, policy.final_gain, y_gain=policy.post_gain)
        dx, dy, grads["final_gain"], grads["post_gain"] = g.dx, g.dy, g.dgain, g.dy_gain
    da = (dy @ policy.out).unflatten(1, (s.q_heads, s.head_dim))
    dqkv = x.new_empty((len(x), policy.qkv.shape[0]))
    dq, dk, dv = dqkv.unflatten(1, (-1, s.head_dim)).split((s.q_heads, s.k_heads, s.k_heads), 1)
    g = oapl.attention_bwd(turned.q, turned.k, v, a.out, a.lse, da, offsets, dv=dv)
    g = oapl.qk_norm_rope_bwd(q0, k0, g.dq, g.dk, positions, policy.cos_sin, policy.q_gain, policy.k_gain, dq=dq, dk=dk)
    grads.update(head=r.dW, out=(dy.t() @ a.out.flatten(1)).float(), qkv=(dqkv.t() @ n).float(), q_gain=g.dq_gain, k_gain=g.dk_gain)
    dn = dqkv @ policy.qkv
    if s.norms:
        g = oapl.residual_norm_bwd(x, None, dx, dn, policy.in_gain)
        dx, grads["in_gain"] = g.dx, g.dgain
    else:
        dx = dx + dn
    grads["embedding"] = oapl.embed_bwd(dx, tokens, s.vocabulary).dE
    return Step(r.loss, r.logprob, grads)


def main(steps=20, norms=False):
    policy = Policy(Sizes(norms=norms))
    prompt = [torch.arange(5 + 3 * i, device="cuda:0", dtype=torch.int32) % 97 for i in range(2)]
    group = 4
    prompts = [p for p in prompt for _ in range(group)]
    answers = [24 + 5 * (i % 3) for i in range(len(prompts))]
    texts, logq = rollouts(policy, prompts, answers, seed=1)
    ids = torch.tensor([i // group for i in range(len(prompts))], dtype=torch.int32, device="cuda:0")
    # reward: an even first token
    rewards = torch.tensor([float(t[-a] % 2 == 0) for t, a in zip(texts, answers)], device="cuda:0")
    masters = {}
    for step in range(steps):
        r = train_step(policy, texts, answers, logq, rewards, ids, len(prompt), beta=0.5)
        if step == 0:
            drift = (r.logprob - torch.cat(logq)).abs().max().item()
            print(f"log-probs of the packed pass differ from the rollouts' by at most {drift:.4f}")
        print(f"step {step}: loss {r.loss.item():.4f}", flush=True)
        # the loss's least value is 0: half the step that would get there if it were linear
        rate = 0.5 * r.loss / oapl.grad_norm(list(r.grads.values())).norm.square()
        for name, grad in r.grads.items():
            weights = getattr(policy, name)
            weights.copy_(masters.setdefault(name, weights.float()).sub_(rate * grad))


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 20, norms="norms" in sys.argv[2:])
