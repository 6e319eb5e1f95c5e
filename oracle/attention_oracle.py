"""Oracle of the policy's attention in 64 bits: norm and rotation of heads, soft-max attention of packed sequences, their
gradients, and how far an implementation that rounds where the library says it rounds may be from them.

Written from the formulas with torch's elementary operations in float64, one sequence and one head at a time; runs on the CPU
or, for larger checks, on the device its inputs are on.  It shares nothing with the library.

Error bounds.  A correctly rounded product or sum of n terms in 32 bits is off by at most (n + 1) 2^-24 of the sum of the terms'
magnitudes; `u` below is what one rounding to the storage type may take (2^-8 for bf16, whose numbers have 8 bits, nothing beyond the
32-bit terms for fp32).  Results are off by their own rounding, by the rounding of the operands that the library rounds (probabilities, dS), and
by the 32-bit terms; every bound is the sum of these magnitudes, element by element.
"""
import math

import torch

F = torch.float64
U32 = 2.0 ** -24


def store_unit(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24


# ------------------------------------------------------------------------------------------------- norm and rotation
def _turn(x, pos, cos_sin, back=False):
    half = cos_sin.shape[1] // 2
    at = cos_sin[pos.long()].to(F)[:, None]
    cos, sin = at[..., :half], at[..., half:] * (-1 if back else 1)
    a, b, rest = x[..., :half], x[..., half:2 * half], x[..., 2 * half:]
    return torch.cat((a * cos - b * sin, a * sin + b * cos, rest), -1)


def norm_rope(x, gain, pos, cos_sin, eps):
    """y, and the bound of its error, for one tensor of heads [T, H, D]."""
    u = store_unit(x.dtype)
    x = x.to(F)
    if gain is not None:
        x = x / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + eps) * gain.to(F)
    y = _turn(x, pos, cos_sin)
    half = cos_sin.shape[1] // 2
    a, b, rest = x[..., :half].abs(), x[..., half:2 * half].abs(), x[..., 2 * half:].abs()
    size = torch.cat((a + b, a + b, rest), -1)
    return y, u * y.abs() + 32 * U32 * size


def norm_rope_grads(x, dy, gain, pos, cos_sin, eps):
    """dx, dgain (or None) and the bounds of their errors."""
    u, D = store_unit(x.dtype), x.shape[-1]
    x, w = x.to(F), _turn(dy.to(F), pos, cos_sin, back=True)
    half = cos_sin.shape[1] // 2
    m = dy.to(F).abs()
    m = torch.cat((m[..., :half] + m[..., half:2 * half],) * 2 + (m[..., 2 * half:],), -1)      # magnitude of w's terms
    if gain is None:
        return w, None, u * w.abs() + 8 * U32 * m, None
    r = 1 / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + eps)
    g = gain.to(F)
    dgain = (w * x * r).sum((0, 1))
    t = w * g
    dx = r * (t - x * r.pow(2) * (t * x).mean(-1, keepdim=True))
    size = r * (m * g.abs() + x.abs() * r.pow(2) * (m * g.abs() * x.abs()).mean(-1, keepdim=True))
    n = x.shape[0] * x.shape[1]
    dgain_size = (m * x.abs() * r).sum((0, 1))
    return dx, dgain, u * dx.abs() + (D + 64) * U32 * size, (math.sqrt(n) + 64) * U32 * dgain_size


# ------------------------------------------------------------------------------------------------- attention
def visible(nq, nk, causal, device):
    """[nq, nk] truth: query i sees key j."""
    if not causal:
        return torch.ones(nq, nk, dtype=torch.bool, device=device)
    return torch.arange(nk, device=device) <= torch.arange(nq, device=device)[:, None] + (nk - nq)


def _sequences(q_offsets, k_offsets, k_used):
    qo, ko = q_offsets.tolist(), k_offsets.tolist()
    used = k_used.tolist() if k_used is not None else [b - a for a, b in zip(ko, ko[1:])]
    return [(slice(qo[s], qo[s + 1]), slice(ko[s], ko[s] + used[s])) for s in range(len(qo) - 1)]


def attention(q, k, v, q_offsets, k_offsets, *, causal, scale, k_used=None):
    """out, lse and the bounds of their errors."""
    u, (Tq, hq, D), g = store_unit(q.dtype), q.shape, q.shape[1] // k.shape[1]
    out, bound = (torch.zeros(q.shape, dtype=F, device=q.device) for _ in range(2))
    lse = torch.full((Tq, hq), -math.inf, dtype=F, device=q.device)
    lse_bound = torch.zeros_like(lse)
    rounded = u if q.dtype == torch.bfloat16 else 0.0
    for Q, K in _sequences(q_offsets, k_offsets, k_used):
        nq, nk = Q.stop - Q.start, K.stop - K.start
        if nq == 0 or nk == 0:
            continue
        seen = visible(nq, nk, causal, q.device)
        some = seen.any(1)
        for h in range(hq):
            a, b, c = q[Q, h].to(F), k[K, h // g].to(F), v[K, h // g].to(F)
            z = (a @ b.t()) * scale
            off = (a.abs() @ b.abs().t()) * abs(scale) * (D + 3) * U32            # of a score
            z = z.masked_fill(~seen, -math.inf)
            top = z.amax(1, keepdim=True).masked_fill(~some[:, None], 0.0)
            e = torch.exp(z - top).masked_fill(~seen, 0.0)
            total = e.sum(1, keepdim=True)
            p = e / total.masked_fill(~some[:, None], 1.0)
            lse[Q, h] = torch.where(some, (top + total.log())[:, 0], -math.inf)
            out[Q, h] = p @ c
            # relative error of a probability: twice the scores' (its own and the normaliser's), exponentials, sums
            off = 2 * off.masked_fill(~seen, 0.0).amax(1, keepdim=True) + (8 + 4 * top.abs()) * U32 + (math.sqrt(nk) + 16) * U32
            bound[Q, h] = u * out[Q, h].abs() + (rounded + off + math.sqrt(nk) * U32) * (p @ c.abs())
            lse_bound[Q, h] = torch.where(some, off[:, 0] + 4 * U32 * lse[Q, h].abs(), 0.0)
    return out, lse, bound, lse_bound


def attention_grads(q, k, v, out, lse, dout, q_offsets, k_offsets, *, causal, scale):
    """(dq, dk, dv) and the bounds of their errors; out and lse are inputs, as they are of the library."""
    u, D, g = store_unit(q.dtype), q.shape[2], q.shape[1] // k.shape[1]
    rounded = u if q.dtype == torch.bfloat16 else 0.0
    dq, bq = (torch.zeros(q.shape, dtype=F, device=q.device) for _ in range(2))
    dk, bk, dv, bv = (torch.zeros(k.shape, dtype=F, device=q.device) for _ in range(4))
    for Q, K in _sequences(q_offsets, k_offsets, None):
        nq, nk = Q.stop - Q.start, K.stop - K.start
        if nq == 0 or nk == 0:
            continue
        seen = visible(nq, nk, causal, q.device)
        for h in range(q.shape[1]):
            a, b, c = q[Q, h].to(F), k[K, h // g].to(F), v[K, h // g].to(F)
            do, o, le = dout[Q, h].to(F), out[Q, h].to(F), lse[Q, h].to(F)[:, None]
            z = (a @ b.t()) * scale
            p = torch.exp(z - le).masked_fill(~seen, 0.0)
            off = (a.abs() @ b.abs().t()) * abs(scale) * (D + 3) * U32 + (8 + 4 * z.abs() + 4 * le.abs().nan_to_num(posinf=0)) * U32
            inner = do @ c.t() - (do * o).sum(1, keepdim=True)
            inner_off = (do.abs() @ c.abs().t() + (do * o).abs().sum(1, keepdim=True)) * (D + 3) * U32
            ds = p * inner
            ds_off = off * ds.abs() + p * inner_off
            n32 = lambda n: (math.sqrt(n) + 16) * U32                                 # noqa: E731
            dq[Q, h] = ds @ b * scale
            bq[Q, h] = ((rounded + n32(nk)) * ds.abs() + ds_off) @ b.abs() * abs(scale) + u * dq[Q, h].abs()
            dk[K, h // g] += ds.t() @ a * scale
            bk[K, h // g] += ((rounded + n32(nq * g)) * ds.abs() + ds_off).t() @ a.abs() * abs(scale)
            dv[K, h // g] += p.t() @ do
            bv[K, h // g] += ((rounded + n32(nq * g) + off) * p).t() @ do.abs()
    return (dq, dk, dv), (bq, bk + u * dk.abs(), bv + u * dv.abs())
