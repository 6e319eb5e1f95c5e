"""What the performance of a trainer step's remaining operators is measured on.

Around the policy's attention and the loss head a trainer step looks tokens up, adds blocks to the residual stream between
norms, and brings all gradients to a common length.  A case is one call of a public entry point of `paper_2602_19362_amd.oapl`:

    embed      embed_fwd: rows of the embedding, scaled
    embed_bwd  embed_bwd: the embedding's gradient, fp32 as the head's dW is, rows without tokens zero
    norm       residual_norm_fwd: a block's output, normed (`post`), gated (`gate`: one gate for all tokens, or one a token) and
               scaled, added to the residual stream, and the norm of the sum for the next block
    norm_bwd   residual_norm_bwd: gradients of the residual stream, the block's output, both gains and the gate
    clip       clip_grads: the norm of all gradients together, and the gradients scaled to `max_norm` where it is larger, into the
               flat buffers that an optimizer reads (in place they could be measured only once)

Hidden sizes and the vocabulary are those of this repository's workloads, tokens follow Zipf's law over a shuffled vocabulary,
channels of the residual stream differ in scale as a trained model's do, and gradients differ in scale from tensor to tensor.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
VOCAB = 151936
EPS = 1e-6


# ------------------------------------------------------------------------------------------------------------- cases
def _embed(kind, dtype, T, d, V, scale=1.0, out=None, name=None):
    """`dtype` of the embedding, `out` that of the residual stream."""
    c = {"kind": kind, "dtype": dtype, "out": out or dtype, "T": T, "d": d, "V": V, "scale": scale}
    return dict(c, name=name) if name else c


def _norm(kind, dtype, T, d, res=None, block=True, post=True, pre=True, gate="", scale=1.0, name=None):
    """`res`: type of the residual stream; `block`: there is one to add; `gate`: "" for none, "channel" or "token"."""
    c = {"kind": kind, "dtype": dtype, "res": res or dtype, "T": T, "d": d, "block": block, "post": block and post, "pre": pre,
         "gate": gate if block else "", "scale": scale if block else 1.0}
    return dict(c, name=name) if name else c


def _clip(dtype, hidden, V, layers, heads, k_heads, D, clips=True, name=None):
    """The gradients of a policy: `layers` times projections and gains in `dtype`, embedding and head in fp32."""
    c = {"kind": "clip", "dtype": dtype, "hidden": hidden, "V": V, "layers": layers, "heads": heads, "k_heads": k_heads, "D": D,
         "clips": clips}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one decode step of eight prompts' eight rollouts
        _embed("embed", "bf16", 64, 4096, VOCAB, name="embed_decode_step"),
        # the benchmark batch, its residual stream scaled by the root of the hidden size
        _embed("embed", "bf16", 140897, 4096, VOCAB, scale=64.0, name="embed_full_batch"),
        # a small policy in full precision
        _embed("embed_bwd", "f32", 1501, 768, 8192, name="embed_bwd_f32_small"),
        # a micro-batch of one prompt whose answers are short
        _embed("embed_bwd", "bf16", 1003, 4096, VOCAB, name="embed_bwd_short_answers"),
        # the benchmark batch
        _embed("embed_bwd", "bf16", 140897, 4096, VOCAB, scale=64.0, name="embed_bwd_full_batch"),
        # the same decode step between two blocks
        _norm("norm", "bf16", 64, 4096, name="norm_decode_step"),
        # one prompt's eight answers, gains on both sides of the block and a gate for every channel
        _norm("norm", "bf16", 16411, 4096, gate="channel", scale=0.5, name="norm_batch"),
        # a wider policy whose residual stream is fp32, gates that the layer computes for every token
        _norm("norm", "bf16", 6007, 5120, res="f32", post=False, gate="token", name="norm_f32_stream"),
        # a small policy in full precision
        _norm("norm_bwd", "f32", 1501, 768, gate="channel", name="norm_bwd_f32_small"),
        _norm("norm_bwd", "bf16", 16411, 4096, gate="channel", scale=0.5, name="norm_bwd_batch"),
        # a debugging-size policy
        _clip("f32", 256, 1544, 1, 8, 2, 64, name="clip_small_policy"),
        # sixteen layers of the 4096-wide policy with embedding and head
        _clip("bf16", 4096, VOCAB, 16, 32, 8, 128, name="clip_layers"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("embed", "embed_bwd", "embed_bwd", "norm", "norm", "norm_bwd", "norm_bwd", "clip"))
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if kind == "clip":
        heads, k_heads, D = rng.choice(((32, 8, 128), (16, 8, 128), (14, 2, 64), (6, 2, 80), (8, 2, 64)))
        return _clip(dtype, rng.choice((64, 256, 768, 2048, 4096, 8 * rng.randint(8, 512))), _log_int(rng, 500, VOCAB),
                     _log_int(rng, 1, 16) if dtype == "bf16" else _log_int(rng, 1, 8), heads, k_heads, D, clips=rng.random() < 0.7)
    d = rng.choice((64, 256, 768, 2048, 4096, 5120, 8 * rng.randint(4, 640), 8 * rng.randint(4, 640)))
    if rng.random() < 0.15:
        d = rng.randint(17, 1024)
    if kind in ("embed", "embed_bwd"):
        V = min(rng.choice((VOCAB, VOCAB, _log_int(rng, 300, VOCAB))), VOCAB * 4096 // d)
        T = _log_int(rng, 1, min(140897, 140897 * 4096 // (d * (2 if dtype == "f32" else 1))))
        out = rng.choice((dtype, dtype, "f32")) if T * d <= 70000 * 4096 else dtype
        return _embed(kind, dtype, T, d, V, scale=rng.choice((1.0, round(math.sqrt(d), 3))), out=out)
    T = _log_int(rng, 1, min(16411, 8000 * 4096 // d))
    return _norm(kind, dtype, T, d, res=rng.choice((dtype, dtype, "f32")), block=rng.random() < 0.85, post=rng.random() < 0.6,
                 pre=True, gate=rng.choice(("", "", "channel", "token")), scale=rng.choice((1.0, 1.0, 0.5, 0.179)))


def _shapes(case):
    """(shape, type) of every gradient, in the order of a policy's weights."""
    h, D = case["hidden"], case["D"]
    rows = (case["heads"] + 2 * case["k_heads"]) * D
    layer = [((rows, h), case["dtype"]), ((h, case["heads"] * D), case["dtype"]), ((D,), "f32"), ((D,), "f32"), ((h,), "f32"), ((h,), "f32")]
    return [((case["V"], h), "f32")] + layer * case["layers"] + [((case["V"], h), "f32")]


# ------------------------------------------------------------------------------------------------------------- inputs
def _shares(V):
    """Zipf's law: the k-th most frequent token's share of the text."""
    share = 1.0 / (torch.arange(1, V + 1, dtype=torch.float64) + 2.7)
    return share / share.sum()


def _tokens(T, V, gen):
    """Drawn by _shares; which token is the k-th most frequent is shuffled."""
    share = _shares(V).cumsum(0).to(DEVICE)
    at = torch.rand(T, generator=gen, device=DEVICE, dtype=torch.float64) * share[-1]
    names = torch.randperm(V, generator=gen, device=DEVICE)
    return names[torch.searchsorted(share, at).clamp_(max=V - 1)].to(torch.int32)


def _randn(rows, cols, dtype, gen, scale=1.0):
    """Normal values times `scale`, drawn in fp32 and rounded once."""
    return (torch.randn(rows, cols, generator=gen, device=DEVICE) * scale).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    s = {"case": case}
    if case["kind"] == "clip":
        shapes = _shapes(case)
        flat = {k: torch.zeros(sum(math.prod(a) for a, t in shapes if t == k), dtype=DTYPES[k], device=DEVICE) for k in ("f32", "bf16")}
        s["grads"], s["out"], at, total = [], [], {"f32": 0, "bf16": 0}, 0.0
        for i, (shape, kind) in enumerate(shapes):
            n, scale = math.prod(shape), 1e-3 * math.exp(math.sin(seed + i))
            s["grads"].append(_randn(-(-n // shape[-1]), shape[-1], DTYPES[kind], gen, scale).view(shape))
            s["out"].append(flat[kind][at[kind]:at[kind] + n].view(shape))
            at[kind] += n
            total += n * scale ** 2
        s["flat"] = {k: x for k, x in flat.items() if x.numel()}
        s["max_norm"] = math.sqrt(total) * (0.4 if case["clips"] else 1.6)
        return s
    T, d, dt = case["T"], case["d"], DTYPES[case["dtype"]]
    if case["kind"] in ("embed", "embed_bwd"):
        s["tokens"] = _tokens(T, case["V"], gen)
        if case["kind"] == "embed":
            s["E"] = _randn(case["V"], d, dt, gen, 0.02)
        else:
            s["dout"] = _randn(T, d, DTYPES[case["out"]], gen, 1e-3)
        return s
    res = DTYPES[case["res"]]
    # channels of a trained model's stream and of a block's output differ in scale
    wide, narrow = (torch.exp(0.7 * torch.randn(d, generator=gen, device=DEVICE)) for _ in range(2))
    gains = [(1 + 0.3 * torch.randn(d, generator=gen, device=DEVICE)).to(dt) for _ in range(2)]
    s["x"] = _randn(T, d, res, gen, 3 * wide)            # of a gradient: the stream behind the block
    s["gain"] = gains[0] if case["pre"] else None
    s["y"] = _randn(T, d, dt, gen, 0.5 * narrow) if case["block"] else None
    s["y_gain"] = gains[1] if case["post"] else None
    s["gate"] = None
    if case["gate"] == "channel":
        s["gate"] = torch.rand(d, generator=gen, device=DEVICE).to(dt)
    elif case["gate"] == "token":
        s["gate"] = torch.sigmoid(torch.randn(T, d, generator=gen, device=DEVICE)).to(dt)
    if case["kind"] == "norm_bwd":
        s["dx_out"], s["dout"] = _randn(T, d, res, gen, 1e-2), _randn(T, d, dt, gen, 1e-2)
    return s


# ------------------------------------------------------------------------------------------------------------- plain forms
def _embed_plain(s):
    case = s["case"]
    return (s["E"][s["tokens"].long()].float() * case["scale"]).to(DTYPES[case["out"]])


def _embed_bwd_plain(s):
    case = s["case"]
    dE = torch.zeros((case["V"], case["d"]), device=DEVICE)
    return dE.index_add_(0, s["tokens"].long(), s["dout"].float() * case["scale"])


def _normed(x):
    """x over its root mean square, and one over that."""
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    return x * r, r


def _norm_plain(s):
    case, got, x = s["case"], {}, s["x"].float()
    if case["block"]:
        z = s["y"].float()
        z = _normed(z)[0] * s["y_gain"].float() if case["post"] else z
        z = z * s["gate"].float() if case["gate"] else z
        x = x + z * case["scale"]
        got["x"] = x.to(s["x"].dtype)
    got["out"] = (_normed(x)[0] * s["gain"].float()).to(DTYPES[case["dtype"]])
    return got


def _norm_bwd_plain(s):
    case, dt = s["case"], DTYPES[s["case"]["dtype"]]
    v, r = _normed(s["x"].float())
    dn = s["dout"].float()
    u = dn * s["gain"].float()
    dx = s["dx_out"].float() + r * (u - v * (u * v).mean(-1, keepdim=True))
    got = {"dx": dx.to(s["x"].dtype), "dgain": (dn * v).sum(0)}
    if not case["block"]:
        return got
    y = s["y"].float()
    w, r = _normed(y) if case["post"] else (y, None)
    z = w * s["y_gain"].float() if case["post"] else y
    dz = dx * case["scale"]
    if case["gate"]:
        g = dz * z
        got["dgate"] = g.sum(0) if case["gate"] == "channel" else g.to(dt)
        dz = dz * s["gate"].float()
    if case["post"]:
        got["dy_gain"] = (dz * w).sum(0)
        t = dz * s["y_gain"].float()
        dz = r * (t - w * (t * w).mean(-1, keepdim=True))
    return dict(got, dy=dz.to(dt))


def _clip_plain(s):
    norm = torch.stack([g.float().square().sum(dtype=torch.float64) for g in s["grads"]]).sum().sqrt().float()
    factor = torch.where(torch.isfinite(norm) & (norm > s["max_norm"]), s["max_norm"] / norm, 1.0)
    _ = [o.copy_(g.float() * factor) for g, o in zip(s["grads"], s["out"])]
    return dict(s["flat"], norm=norm.reshape(1))


# ------------------------------------------------------------------------------------------------------------- one pass
def run(state):
    case = state["case"]
    if own:
        return _run_own(case, state)
    plain = {"embed": _embed_plain, "embed_bwd": _embed_bwd_plain, "norm": _norm_plain, "norm_bwd": _norm_bwd_plain, "clip": _clip_plain}
    return plain[case["kind"]](state)


def _run_own(case, s):
    from paper_2602_19362_amd import oapl

    if case["kind"] == "embed":
        return oapl.embed_fwd(s["E"], s["tokens"], scale=case["scale"], out_dtype=DTYPES[case["out"]])
    if case["kind"] == "embed_bwd":
        r = oapl.embed_bwd(s["dout"], s["tokens"], case["V"], scale=case["scale"], workspace=s.get("workspace"))
        s["workspace"] = r.workspace
        return r.dE
    if case["kind"] == "norm":
        r = oapl.residual_norm_fwd(s["x"], s["y"], s["gain"], y_gain=s["y_gain"], gate=s["gate"], scale=case["scale"], eps=EPS)
        return {"x": r.x, "out": r.out} if case["block"] else {"out": r.out}
    if case["kind"] == "norm_bwd":
        r = oapl.residual_norm_bwd(s["x"], s["y"], s["dx_out"], s["dout"], s["gain"], y_gain=s["y_gain"], gate=s["gate"],
                                   scale=case["scale"], eps=EPS, workspace=s.get("workspace"))
        s["workspace"] = r.workspace
        got = {"dx": r.dx, "dgain": r.dgain, "dy": r.dy, "dy_gain": r.dy_gain, "dgate": r.dgate}
        return {k: x for k, x in got.items() if x is not None}
    r = oapl.clip_grads(s["grads"], s["max_norm"], out=s["out"], workspace=s.get("workspace"))
    s["workspace"] = r.workspace
    return dict(s["flat"], norm=r.norm)


# ------------------------------------------------------------------------------------------------------------- work
def _size(dtype):
    return 2 if dtype == "bf16" else 4


def work(case):
    if case["kind"] == "clip":
        sizes = [(math.prod(a), _size(t)) for a, t in _shapes(case)]
        return {"bytes": sum(2 * n * b for n, b in sizes), "flops": sum(3 * n for n, _ in sizes)}
    T, d, a = case["T"], case["d"], _size(case["dtype"])
    if case["kind"] == "embed":
        rows = round((1 - (1 - _shares(case["V"])) ** T).sum().item())       # that occur, on average
        return {"bytes": rows * d * a + T * (d * _size(case["out"]) + 4), "flops": T * d}
    if case["kind"] == "embed_bwd":
        return {"bytes": T * (d * _size(case["out"]) + 4) + case["V"] * d * 4, "flops": 2 * T * d}
    res, gate = _size(case["res"]), a if case["gate"] == "token" else 0
    if case["kind"] == "norm":
        return {"bytes": T * d * ((2 * res + a if case["block"] else res) + a + gate), "flops": T * d * (11 if case["block"] else 4)}
    return {"bytes": T * d * (3 * res + a + (2 * a if case["block"] else 0) + 2 * gate), "flops": T * d * (24 if case["block"] else 11)}


# ------------------------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    f, s = torch.float64, prepare(case, seed)
    if case["kind"] == "embed":
        return torch.index_select(s["E"], 0, s["tokens"]).to(f).mul_(case["scale"])
    if case["kind"] == "embed_bwd":
        dE = torch.zeros((case["V"], case["d"]), dtype=f, device=DEVICE)
        return dE.index_put_((s["tokens"].long(),), s["dout"].to(f), accumulate=True).mul_(case["scale"])
    if case["kind"] == "clip":
        norm = math.sqrt(sum(torch.linalg.vector_norm(g, dtype=f).item() ** 2 for g in s["grads"]))
        factor = min(1.0, s["max_norm"] / norm)
        got = {"norm": torch.tensor([norm], dtype=f, device=DEVICE)}
        for k in s["flat"]:
            got[k] = torch.cat([g.reshape(-1) for g in s["grads"] if g.dtype == DTYPES[k]]).to(f).mul_(factor)
        return got

    def leaf(x):
        return None if x is None else x.to(f).requires_grad_()

    def scaled(x, gain):
        return gain * x / torch.sqrt(torch.mean(x ** 2, 1, keepdim=True) + EPS)

    x, y, gain, y_gain, gate = (leaf(s[k]) for k in ("x", "y", "gain", "y_gain", "gate"))
    add = None
    if case["block"]:
        add = scaled(y, y_gain) if case["post"] else y * 1.0
        add = (add if gate is None else add * gate) * case["scale"]
    if case["kind"] == "norm":
        with torch.no_grad():
            total = x if add is None else x + add
            out = scaled(total, gain)
        return {"x": total.detach(), "out": out} if case["block"] else {"out": out}
    # the derivatives by differentiating the definition
    dx, dgain = torch.autograd.grad(scaled(x, gain), (x, gain), s["dout"].to(f))
    dx = dx + s["dx_out"].to(f)
    got = {"dx": dx, "dgain": dgain}
    if case["block"]:
        names = [n for n, v in (("dy", y), ("dy_gain", y_gain), ("dgate", gate)) if v is not None]
        got.update(zip(names, torch.autograd.grad(add, [v for v in (y, y_gain, gate) if v is not None], dx)))
    return got
