"""What the performance of the policy's attention is measured on.

The loss head turns final hidden states into a gradient with respect to them; these are the operators of the transformer
below it that a trainer step (and the rollouts that feed it) spends its time in, on the same packed rollouts.  A case is one
call of a public entry point of `paper_2602_19362_amd.oapl`:

    rope      qk_norm_rope_fwd: root-mean-square norm of every query and key head, then the position rotation, from the
              projection's packed rows; with `cache` the keys and values go to the rows of a cache (a decode step)
    rope_bwd  qk_norm_rope_bwd: gradients of the projection's rows and of the two gains
    attn      attention_fwd: soft-max attention over packed sequences, causal unless the case says otherwise, output and
              log-sum-exp; with `cap` the keys are a cache with room for `cap` tokens a sequence (a decode step)
    attn_bwd  attention_bwd: gradients of queries, keys and values, from the forward pass's output and log-sum-exp

Head counts are those of 128-wide heads at the hidden sizes that this repository's workloads have (4096: 32, 2048: 16, 5120:
40) with 8 key heads, shares of them, and small odd ones.  Rollout lengths are lognormal (sigma 0.6) around half the
generation limit, cut at the limit, and belong to the case; values come from the seed.  Queries and keys are unit Gaussians
(what a norm leaves), so scores spread over several units; the projection's rows have another scale in every channel.
"""
import math
import random

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
ROPE_BASE = 1000000.0


# ------------------------------------------------------------------------------------------------------------- cases
def _rope(kind, dtype, T, hq, hk, D, rot=None, norm=True, cache=0, name=None):
    c = {"kind": kind, "dtype": dtype, "T": T, "hq": hq, "hk": hk, "D": D, "rot": rot or D, "norm": norm, "cache": cache}
    return dict(c, name=name) if name else c


def _attn(kind, dtype, n, limit, hq, hk, D, lengths="lognormal", extra=0, causal=True, cap=0, q=0, name=None):
    """`limit`: longest sequence; `extra`: keys that a sequence has beyond its queries (fewer where negative); `q` queries a
    sequence on a cache of `cap` rows each."""
    c = {"kind": kind, "dtype": dtype, "n": n, "limit": limit, "lengths": lengths, "extra": extra, "hq": hq, "hk": hk, "D": D,
         "causal": causal, "cap": cap, "q": q}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one decode step of one prompt's eight rollouts: queries normed and rotated, keys and values into the cache
        _rope("rope", "bf16", 8, 32, 8, 128, cache=512, name="rope_decode_step"),
        # a trainer step's packed micro-batch
        _rope("rope", "bf16", 16411, 32, 8, 128, name="rope_batch"),
        # a small policy in full precision, an odd token count, half of each head rotated
        _rope("rope_bwd", "f32", 1501, 6, 2, 80, rot=40, name="rope_bwd_f32_small"),
        _rope("rope_bwd", "bf16", 16411, 32, 8, 128, name="rope_bwd_batch"),
        # the exactness configuration: eight rollouts of 32 tokens in fp32, hidden size 64
        _attn("attn", "f32", 8, 32, 4, 2, 16, lengths="fixed", name="attn_f32_tiny"),
        # one decode step of eight prompts x eight rollouts
        _attn("attn", "bf16", 64, 4096, 32, 8, 128, cap=4096, q=1, name="attn_decode_step"),
        # one prompt's rollouts near the end of a 32768-token generation
        _attn("attn", "bf16", 8, 32768, 40, 8, 128, lengths="fixed", cap=32768, q=1, name="attn_decode_long"),
        # one prompt's eight rollouts scored or trained on, 4096-token limit
        _attn("attn", "bf16", 8, 4096, 32, 8, 128, name="attn_rollouts"),
        # a 16384-token rollout, half of the heads of a 5120-wide policy
        _attn("attn", "bf16", 1, 16384, 20, 4, 128, lengths="fixed", name="attn_long"),
        # a debugging-size policy: narrow heads in groups of seven, short ragged answers on a shared prefix
        _attn("attn_bwd", "bf16", 13, 400, 14, 2, 64, extra=77, name="attn_bwd_small"),
        _attn("attn_bwd", "f32", 4, 512, 6, 2, 80, name="attn_bwd_f32_small"),
        _attn("attn_bwd", "bf16", 8, 4096, 32, 8, 128, name="attn_bwd_rollouts"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("rope", "rope_bwd", "attn", "decode", "attn", "attn_bwd", "attn_bwd"))
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    hq, hk = rng.choice(((32, 8), (16, 8), (40, 8), (20, 4), (14, 2), (8, 1), (6, 6), (4, 2)))
    D = rng.choice((128, 128, 128, 64, 80, 96, 16))
    if kind in ("rope", "rope_bwd"):
        T = _log_int(rng, 1, 16411)
        cache = rng.choice((0, 2 * T + 5)) if kind == "rope" and T <= 512 else 0
        return _rope(kind, dtype, T, hq, hk, D, rot=rng.choice((D, D, D // 2)), norm=rng.random() < 0.8, cache=cache)
    if kind == "decode":
        cap = _log_int(rng, 16, 32768)
        n = _log_int(rng, 1, max(1, min(64, 262144 // cap)))
        return _attn("attn", dtype, n, cap, hq, hk, D, cap=cap, q=rng.choice((1, 1, 1, 2, 5)))
    most = 8 * 32 * 4096 ** 2 if dtype == "bf16" else 8 * 32 * 1024 ** 2     # scores that the plain form holds at once
    limit = _log_int(rng, 2, 8192 if dtype == "bf16" else 2048)
    limit = min(limit, int(math.sqrt(most / hq)))
    n = _log_int(rng, 1, max(1, min(32, most // (hq * limit * limit))))
    extra = rng.choice((0, 0, 0, 33, -5))
    while extra > 0 and n > 1 and n * hq * limit * (limit + extra) > most:
        n -= 1
    return _attn(kind, dtype, n, limit, hq, hk, D, extra=extra if n * hq * limit * (limit + max(extra, 0)) <= most else 0,
                 causal=rng.random() < 0.85)


def _lengths(case):
    """(queries, keys) of every sequence."""
    rng = random.Random("%(n)s %(limit)s %(hq)s" % case)
    if case["lengths"] == "fixed":
        k = [case["limit"]] * case["n"]
    else:
        k = [max(1, min(case["limit"], round(case["limit"] / 2 * math.exp(0.6 * rng.gauss(0, 1))))) for _ in range(case["n"])]
        k[rng.randrange(case["n"])] = case["limit"]
    if case["cap"]:
        return [case["q"]] * case["n"], k
    return k, [max(0, x + case["extra"]) for x in k]


# ------------------------------------------------------------------------------------------------------------- inputs
def _offsets(lengths):
    t = torch.zeros(len(lengths) + 1, dtype=torch.int64)
    t[1:] = torch.tensor(lengths, dtype=torch.int64).cumsum(0)
    return t.to(DEVICE)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    hq, hk, D = case["hq"], case["hk"], case["D"]

    def normal(*shape, dtype=dt):
        return torch.randn(*shape, generator=gen, device=DEVICE).to(dtype)

    if case["kind"] in ("rope", "rope_bwd"):
        T, rot = case["T"], case["rot"]
        # one projection's output: queries, keys and values of a token side by side
        scale = torch.exp(0.5 * torch.randn((hq + 2 * hk) * D, generator=gen, device=DEVICE))
        qkv = (torch.randn(T, (hq + 2 * hk) * D, generator=gen, device=DEVICE) * scale).to(dt)
        q, k, v = (x.unflatten(1, (-1, D)) for x in qkv.split((hq * D, hk * D, hk * D), 1))
        span = 32768
        angle = torch.arange(span, dtype=torch.float64)[:, None] * ROPE_BASE ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
        s = {"case": case, "q": q, "k": k, "positions": torch.randint(0, span, (T,), generator=gen, device=DEVICE, dtype=torch.int32),
             "cos_sin": torch.cat((angle.cos(), angle.sin()), 1).float().to(DEVICE), "q_gain": None, "k_gain": None}
        if case["norm"]:
            s["q_gain"], s["k_gain"] = ((1 + 0.3 * torch.randn(D, generator=gen, device=DEVICE)).to(dt) for _ in range(2))
        if case["kind"] == "rope_bwd":
            s["dq_out"], s["dk_out"] = normal(T, hq, D), normal(T, hk, D)
        elif case["cache"]:
            s["v"], s["k_cache"], s["v_cache"] = v, normal(case["cache"], hk, D), normal(case["cache"], hk, D)
            s["rows"] = torch.randperm(case["cache"], generator=gen, device=DEVICE)[:T]
        return s
    ql, kl = _lengths(case)
    room = [case["cap"]] * case["n"] if case["cap"] else kl
    s = {"case": case, "q_offsets": _offsets(ql), "k_offsets": _offsets(room), "longest": (max(ql), max(kl)),
         "k_used": torch.tensor(kl, device=DEVICE) if case["cap"] else None,
         "q": normal(sum(ql), hq, D), "k": normal(sum(room), hk, D), "v": normal(sum(room), hk, D)}
    if case["kind"] == "attn_bwd":
        s["out"], s["lse"] = _attention(s)
        s["dout"] = normal(sum(ql), hq, D)
    return s


# ------------------------------------------------------------------------------------------------------------- plain forms
def _turned(x, s, back=False):
    """x [T, H, D] in 32 bits with the first `rot` channels turned by the token's angles, pairs (i, i + rot / 2)."""
    half = s["case"]["rot"] // 2
    at = s["cos_sin"][s["positions"].long()][:, None]
    cos, sin = at[..., :half], at[..., half:]
    sin = -sin if back else sin
    a, b = x[..., :half], x[..., half:2 * half]
    return torch.cat((a * cos - b * sin, b * cos + a * sin, x[..., 2 * half:]), -1)


def _rope_plain(s):
    def normed(x, gain):
        x = x.float()
        return x if gain is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain.float()

    q = _turned(normed(s["q"], s["q_gain"]), s).to(s["q"].dtype)
    k = _turned(normed(s["k"], s["k_gain"]), s).to(s["k"].dtype)
    if not s["case"]["cache"]:
        return {"q": q, "k": k}
    s["k_cache"].index_copy_(0, s["rows"], k)
    s["v_cache"].index_copy_(0, s["rows"], s["v"])
    return {"q": q, "k": s["k_cache"], "v": s["v_cache"]}


def _rope_bwd_plain(s):
    def grad(x, dy, gain):
        x, u = x.float(), _turned(dy.float(), s, back=True)
        if gain is None:
            return u.to(dy.dtype), None
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        t = u * gain.float()
        dx = r * (t - x * r.square() * (t * x).mean(-1, keepdim=True))
        return dx.to(dy.dtype), (u * x * r).sum((0, 1))

    (dq, gq), (dk, gk) = grad(s["q"], s["dq_out"], s["q_gain"]), grad(s["k"], s["dk_out"], s["k_gain"])
    return {"dq": dq, "dk": dk} if gq is None else {"dq": dq, "dk": dk, "dq_gain": gq, "dk_gain": gk}


def _padded(x, offsets, lengths, longest, groups):
    """The packed rows x [T, H, C] as [n, H / groups, groups * longest, C] in 32 bits, zeros behind a sequence's end."""
    at = torch.arange(longest, device=x.device)
    inside = at < lengths[:, None]
    y = x[torch.where(inside, offsets[:-1, None] + at, 0)].float().masked_fill_(~inside[..., None, None], 0.0)
    return y.unflatten(2, (-1, groups)).permute(0, 2, 3, 1, 4).flatten(2, 3)


def _packed(y, offsets, T, groups):
    """_padded's way back."""
    t = torch.arange(T, device=y.device)
    seq = torch.searchsorted(offsets[1:], t, right=True)
    return y.unflatten(2, (groups, -1)).permute(0, 3, 1, 2, 4)[seq, t - offsets[seq]].flatten(1, 2)


def _scores(s):
    """Scaled scores [n, Hk, groups * queries, keys], and which of them count."""
    case = s["case"]
    g = case["hq"] // case["hk"]
    lq, lk = s["longest"]
    ql = s["q_offsets"].diff()
    kl = s["k_used"] if s["k_used"] is not None else s["k_offsets"].diff()
    q, k, v = (_padded(s["q"], s["q_offsets"], ql, lq, g), _padded(s["k"], s["k_offsets"], kl, lk, 1),
               _padded(s["v"], s["k_offsets"], kl, lk, 1))
    i, j = torch.arange(lq, device=DEVICE)[:, None], torch.arange(lk, device=DEVICE)
    seen = (j < kl[:, None, None]) & (i < ql[:, None, None])
    if case["causal"]:
        seen = seen & (j <= i + (kl - ql)[:, None, None])
    return torch.matmul(q, k.transpose(-1, -2)).mul_(case["D"] ** -0.5), seen[:, None].repeat(1, 1, g, 1), q, k, v, ql, kl


def _attention(s):
    case = s["case"]
    g, T = case["hq"] // case["hk"], s["q"].shape[0]
    p, seen, _, _, v, _, _ = _scores(s)
    p.masked_fill_(~seen, -math.inf)
    m = p.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = p.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    lse = torch.where(total > 0, m + total.log(), -math.inf)
    return _packed(o, s["q_offsets"], T, g).to(s["q"].dtype), _packed(lse, s["q_offsets"], T, g)[..., 0]


def _attention_bwd(s):
    case = s["case"]
    g, (lq, _), scale = case["hq"] // case["hk"], s["longest"], case["D"] ** -0.5
    p, seen, q, k, v, ql, kl = _scores(s)
    do, o = (_padded(s[x], s["q_offsets"], ql, lq, g) for x in ("dout", "out"))
    p = p.sub_(_padded(s["lse"][..., None], s["q_offsets"], ql, lq, g)).exp_().masked_fill_(~seen, 0.0)
    dv = torch.matmul(p.transpose(-1, -2), do)
    ds = torch.matmul(do, v.transpose(-1, -2)).sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(-1, -2), q)
    dt, T, R = s["q"].dtype, s["q"].shape[0], s["k"].shape[0]
    return {"dq": _packed(dq, s["q_offsets"], T, g).to(dt), "dk": _packed(dk, s["k_offsets"], R, 1).to(dt),
            "dv": _packed(dv, s["k_offsets"], R, 1).to(dt)}


# ------------------------------------------------------------------------------------------------------------- one pass
def run(state):
    case = state["case"]
    if own:
        return _run_own(case, state)
    if case["kind"] == "rope":
        return _rope_plain(state)
    if case["kind"] == "rope_bwd":
        return _rope_bwd_plain(state)
    if case["kind"] == "attn":
        out, lse = _attention(state)
        return {"out": out, "lse": lse}
    return _attention_bwd(state)


def _run_own(case, s):
    from paper_2602_19362_amd import oapl

    if case["kind"] == "rope":
        cached = {"v": s["v"], "rows": s["rows"], "k_out": s["k_cache"], "v_out": s["v_cache"]} if case["cache"] else {}
        r = oapl.qk_norm_rope_fwd(s["q"], s["k"], s["positions"], s["cos_sin"], s["q_gain"], s["k_gain"], eps=EPS, **cached)
        return {"q": r.q, "k": r.k, "v": r.v} if case["cache"] else {"q": r.q, "k": r.k}
    if case["kind"] == "rope_bwd":
        r = oapl.qk_norm_rope_bwd(s["q"], s["k"], s["dq_out"], s["dk_out"], s["positions"], s["cos_sin"], s["q_gain"], s["k_gain"],
                                  eps=EPS, workspace=s.get("workspace"))
        s["workspace"] = r.workspace
        got = {"dq": r.dq, "dk": r.dk}
        return dict(got, dq_gain=r.dq_gain, dk_gain=r.dk_gain) if case["norm"] else got
    if case["kind"] == "attn":
        r = oapl.attention_fwd(s["q"], s["k"], s["v"], s["q_offsets"], s["k_offsets"], causal=case["causal"], k_used=s["k_used"],
                               workspace=s.get("workspace"))
        s["workspace"] = r.workspace
        return {"out": r.out, "lse": r.lse}
    r = oapl.attention_bwd(s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], s["q_offsets"], s["k_offsets"],
                           causal=case["causal"], workspace=s.get("workspace"))
    s["workspace"] = r.workspace
    return {"dq": r.dq, "dk": r.dk, "dv": r.dv}


# ------------------------------------------------------------------------------------------------------------- work
def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    hq, hk, D = case["hq"], case["hk"], case["D"]
    if case["kind"] in ("rope", "rope_bwd"):
        T = case["T"]
        rows, tables = T * (hq + hk) * D * size, T * (case["rot"] * 4 + 4)
        if case["kind"] == "rope":
            return {"bytes": 2 * rows + tables + (T * (2 * hk * D * size + 8) if case["cache"] else 0), "flops": 10 * T * (hq + hk) * D}
        return {"bytes": 3 * rows + tables, "flops": 20 * T * (hq + hk) * D}
    ql, kl = _lengths(case)
    pairs = 0
    for a, b in zip(ql, kl):
        if case["causal"]:
            first = max(0, b - a + 1)            # keys that the first query sees, or 0
            rows = a if b - a + 1 > 0 else b      # queries that see any
            last = b
            first = last - rows + 1 if rows else 0
            pairs += rows * (first + last) // 2
        else:
            pairs += a * b
    q_rows, k_rows = sum(ql) * hq * D * size, sum(kl) * hk * D * size
    lse = sum(ql) * hq * 4
    if case["kind"] == "attn":
        return {"bytes": 2 * q_rows + 2 * k_rows + lse, "flops": 4 * pairs * hq * D}
    return {"bytes": 4 * q_rows + 4 * k_rows + lse, "flops": 10 * pairs * hq * D}


# ------------------------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("rope", "rope_bwd"):
        return _rope_exact(case, s)
    g, scale, n = case["hq"] // case["hk"], case["D"] ** -0.5, case["n"]
    ql, kl = _lengths(case)
    qo, ko = s["q_offsets"].tolist(), s["k_offsets"].tolist()
    f = torch.float64
    fwd = case["kind"] == "attn"
    a, b = (torch.zeros(s["q"].shape, dtype=f, device=DEVICE) for _ in range(2))
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=f, device=DEVICE)
    dk, dv = (torch.zeros(s["k"].shape, dtype=f, device=DEVICE) for _ in range(2)) if not fwd else (None, None)
    for x in range(n):
        Q, K = slice(qo[x], qo[x] + ql[x]), slice(ko[x], ko[x] + kl[x])
        if ql[x] == 0 or kl[x] == 0:
            continue
        hidden = torch.arange(kl[x], device=DEVICE) > torch.arange(ql[x], device=DEVICE)[:, None] + (kl[x] - ql[x])
        for h in range(case["hq"]):
            q, k, v = s["q"][Q, h].to(f), s["k"][K, h // g].to(f), s["v"][K, h // g].to(f)
            z = torch.mm(q, k.t().contiguous()) * scale
            if case["causal"]:
                z[hidden] = -math.inf
            if fwd:
                lse[Q, h] = torch.logsumexp(z, 1)
                w = torch.nan_to_num(torch.softmax(z, 1), nan=0.0)
                a[Q, h] = torch.mm(w, v)
                continue
            w = torch.exp(z - s["lse"][Q, h].to(f)[:, None])
            w[z == -math.inf] = 0
            do = s["dout"][Q, h].to(f)
            dz = w * (torch.mm(do, v.t().contiguous()) - (do * s["out"][Q, h].to(f)).sum(1, keepdim=True)) * scale
            a[Q, h] = torch.mm(dz, k)
            dk[K, h // g] += torch.mm(dz.t().contiguous(), q)
            dv[K, h // g] += torch.mm(w.t().contiguous(), do)
    return {"out": a, "lse": lse} if fwd else {"dq": a, "dk": dk, "dv": dv}


def _rope_exact(case, s):
    f = torch.float64
    half, D = case["rot"] // 2, case["D"]
    table = s["cos_sin"].to(f)[s["positions"].long()]
    # a token's rotation as a matrix [D, D]
    turn = torch.eye(D, dtype=f, device=DEVICE).repeat(case["T"], 1, 1)
    i = torch.arange(half, device=DEVICE)
    turn[:, i, i] = table[:, :half]
    turn[:, i + half, i + half] = table[:, :half]
    turn[:, i, i + half] = -table[:, half:]
    turn[:, i + half, i] = table[:, half:]
    got = {}
    for name in ("q", "k"):
        x, gain = s[name].to(f), s[name + "_gain"]
        r = (x.pow(2).mean(-1, keepdim=True) + EPS).pow(-0.5)
        if case["kind"] == "rope":
            y = x if gain is None else x * r * gain.to(f)
            got[name] = torch.matmul(y, turn.transpose(1, 2).contiguous())
            continue
        u = torch.matmul(s["d%s_out" % name].to(f), turn)
        if gain is None:
            got["d" + name] = u
            continue
        got["d%s_gain" % name] = (u * x * r).sum((0, 1))
        w = u * gain.to(f)
        got["d" + name] = w * r - x * (w * x).sum(-1, keepdim=True) * r.pow(3) / D
    if case["kind"] == "rope" and case["cache"]:
        for name, new in (("k", got["k"]), ("v", s["v"].to(f))):
            got[name] = s[name + "_cache"].to(f)
            got[name][s["rows"]] = new
    return got
