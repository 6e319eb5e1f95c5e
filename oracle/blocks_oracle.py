"""Oracle of what lies around the policy's blocks in 64 bits: embedding lookup, residual stream with its norms, the gradients of both,
and clipping by a common norm; and how far an implementation that rounds where the library says it rounds may be from them.

Written from the formulas with torch's elementary operations in float64, on the device that its inputs are on.  It shares nothing with
the library.

Error bounds, element by element, to first order.  U32 is what one rounding in 32 bits may take, u one to the storage type (2^-8 for bf16).
A row's sum of squares is one of positive terms: with lanes that add up to 16 terms each, six exchanges in a wavefront and up to 16
wavefronts it is off by 40 roundings of itself, and one over its root by half of that and the root's own; R = 64 U32 is more than both.  A sum of n terms in
any order is off by n roundings of the sum of their magnitudes.
"""
import torch

F = torch.float64
U32 = 2.0 ** -24
R = 64 * U32


def store_unit(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24


# ------------------------------------------------------------------------------------------------- embedding
def embed(E, tokens, scale, out_dtype):
    """out, and the bound of its error: the product's rounding and the one to the output's type.  Rows outside the embedding: NaN."""
    V = E.shape[0]
    inside = (tokens >= 0) & (tokens < V)
    y = E.to(F)[torch.where(inside, tokens, 0).long()] * scale if V else None
    y[~inside] = torch.nan
    return y, (store_unit(out_dtype) + U32) * y.abs()


def embed_grads(dout, tokens, V, scale, old=None):
    """dE, and the bound of its error: as many roundings as the token has rows, of their magnitudes, the scale's and the addition's."""
    inside = (tokens >= 0) & (tokens < V)
    g, at = dout.to(F)[inside] * scale, tokens[inside].long()
    dE, size = (torch.zeros(V, dout.shape[1], dtype=F, device=dout.device).index_add_(0, at, x) for x in (g, g.abs()))
    n = torch.bincount(at, minlength=V)[:, None]
    if old is not None:
        dE, size = dE + old.to(F), size + old.to(F).abs()
    return dE, (n + 3) * U32 * size * (n > 0)


# ------------------------------------------------------------------------------------------------- residual stream
def _normed(x, eps):
    r = 1 / torch.sqrt(x.pow(2).mean(1, keepdim=True) + eps)
    return x * r, r


def residual_norm(x, y, gain, y_gain, gate, scale, eps):
    """(x', bound), (n, bound); None in the place of what there is not."""
    ux, kind = store_unit(x.dtype), (gain if y is None else y).dtype
    x, e = x.to(F), torch.zeros(x.shape, dtype=F, device=x.device)
    first = None
    if y is not None:
        z = y.to(F)
        if y_gain is not None:
            z = _normed(z, eps)[0] * y_gain.to(F)
        z = z * scale if gate is None else z * gate.to(F) * scale
        x = x + z
        e = (R + 6 * U32) * z.abs() + U32 * x.abs()
        first = x, e + ux * x.abs()
    if gain is None:
        return first, None
    v, r = _normed(x, eps)
    n = v * gain.to(F)
    off = gain.to(F).abs() * r * e + n.abs() * (R + 3 * U32 + r.pow(2) * (x.abs() * e).mean(1, keepdim=True))
    return first, (n, off + store_unit(kind) * n.abs())


def residual_norm_grads(x, y, dx_out, dout, gain, y_gain, gate, scale, eps):
    """{name: (value, bound)} of dx, dy, dgain, dy_gain, dgate, as far as there are any."""
    kind = (gain if y is None else y).dtype
    ux, u, T = store_unit(x.dtype), store_unit(kind), x.shape[0]
    n_sum = (T + 4) * U32
    x = x.to(F)
    dX = torch.zeros_like(x) if dx_out is None else dx_out.to(F)
    e = 2 * U32 * dX.abs()
    got = {}
    if gain is not None:
        v, r = _normed(x, eps)
        dn = dout.to(F)
        a = dn * gain.to(F)
        M = (a * v).abs().mean(1, keepdim=True)
        dX = dX + r * (a - v * (a * v).mean(1, keepdim=True))
        e = e + 3 * R * r * (a.abs() + v.abs() * M) + U32 * dX.abs()
        got["dgain"] = (dn * v).sum(0), (R + 2 * U32 + n_sum) * (dn * v).abs().sum(0)
    got["dx"] = dX, e + ux * dX.abs()
    if y is None:
        return got
    y = y.to(F)
    w, ry = _normed(y, eps) if y_gain is not None else (y, None)
    rel_w = R + 2 * U32 if y_gain is not None else 0.0
    yg = 1.0 if y_gain is None else y_gain.to(F)
    gg = 1.0 if gate is None else gate.to(F)
    z, dz = w * yg, scale * gg * dX
    e_dz = abs(scale) * (e * (gg if gate is None else gg.abs())) + 2 * U32 * dz.abs()
    if gate is not None:
        dg = scale * z * dX
        e_dg = abs(scale) * z.abs() * e + (rel_w + 3 * U32) * dg.abs()
        got["dgate"] = (dg.sum(0), e_dg.sum(0) + n_sum * dg.abs().sum(0)) if gate.dim() == 1 else (dg, e_dg + u * dg.abs())
    if y_gain is None:
        got["dy"] = dz, e_dz + u * dz.abs()
        return got
    got["dy_gain"] = (dz * w).sum(0), (w.abs() * e_dz + rel_w * (dz * w).abs()).sum(0) + n_sum * (dz * w).abs().sum(0)
    t = yg * dz
    e_t = yg.abs() * e_dz + U32 * t.abs()
    M = (t * w).abs().mean(1, keepdim=True)
    e_m = (w.abs() * e_t).mean(1, keepdim=True) + 2 * R * M
    dy = ry * (t - w * (t * w).mean(1, keepdim=True))
    got["dy"] = dy, ry * (e_t + w.abs() * e_m + 3 * R * (t.abs() + w.abs() * M)) + u * dy.abs()
    return got


# ------------------------------------------------------------------------------------------------- clipping
def grad_norm(grads):
    """The norm, whose bound is one rounding of it to 32 bits (and 2^-48 of it for the sums of 64 bits)."""
    norm = torch.sqrt(sum((g.to(F) ** 2).sum() for g in grads)).reshape(1) if grads else torch.zeros(1, dtype=F)
    return norm, (U32 + 2.0 ** -48) * norm


def clipped(grads, max_norm, norm):
    """[(value, bound)]: the product's rounding, for bf16 to 32 bits first, and what was rounded in the norm; half a step among the smallest numbers."""
    factor = max_norm / norm if bool(torch.isfinite(norm)) and float(norm) > max_norm else 1.0
    least = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134}
    return [(g.to(F) * factor, (store_unit(g.dtype) + 2 * U32) * (g.to(F) * factor).abs() + least[g.dtype]) for g in grads]
