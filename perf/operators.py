"""The operators that stand around a sparse attention layer in a transformer block, as cases that can be timed and compared.

* ``dense``: attention over all keys (low resolutions, conditioning tokens, a cache that one new token reads), forward alone or a
  training step of forward and backward: ``llsa.dense_forward``, ``llsa.dense_backward``;
* ``norm``: what lies between two blocks, ``x' = x + alpha gate norm(branch)`` and ``y = norm(x') (1 + scale) + shift`` in one pass, forward or
  backward: ``llsa.norm_forward``, ``llsa.norm_backward``;
* ``glue``: the gradient of QK-Norm and RoPE in front of the layer: ``llsa.qknorm_rope_backward``.

A program keeps plans, workspaces and output buffers from step to step, so ``prepare`` makes them.
"""
import math

import torch

own = False


def _dense(name, mode, batch, heads, Nq, Nkv, d, kv_heads=0, dtype="bf16", causal=False, lens="", tokens_first=False):
    return dict(name=name, op="dense", mode=mode, dtype=dtype, batch=batch, heads=heads, kv_heads=kv_heads or heads, Nq=Nq, Nkv=Nkv, d=d,
                causal=causal, lens=lens, tokens_first=tokens_first)


def _norm(name, mode, batch, N, C, dtype="bf16", kind="rms", branch=True, post=True, mod=True, shared=False, shift=True):
    return dict(name=name, op="norm", mode=mode, dtype=dtype, kind=kind, batch=batch, N=N, C=C, branch=branch, post=post, mod=mod, shared=shared,
                shift=shift)


def _glue(name, batch, heads, N, d, B=16, L=2, dtype="bf16"):
    return dict(name=name, op="glue", mode="backward", dtype=dtype, batch=batch, heads=heads, N=N, d=d, B=B, L=L)


def listed():
    return [
        # the smallest layer, one fp32 head of a 16 x 16 grid, as in a unit test or a toy training run
        _dense("dense_tiny_fp32_step", "step", 1, 1, 256, 256, 32, dtype="f32"),
        # eight requests, each with one new token that reads the keys and values it has so far: bytes
        _dense("dense_one_token_forward", "forward", 8, 32, 1, 16384, 128, kv_heads=8, lens="kv"),
        # 64 x 64 pixel tokens that attend to up to 120 conditioning tokens, both as a projection leaves them ([batch, N, heads, d])
        _dense("dense_condition_forward", "forward", 2, 16, 4096, 120, 64, lens="kv", tokens_first=True),
        # a padded batch of sequences of odd lengths with shared key and value heads, causal
        _dense("dense_causal_padded_step", "step", 3, 16, 1999, 1999, 128, kv_heads=4, causal=True, lens="both", tokens_first=True),
        # 128 x 128 pixel tokens with every key, what a model is trained with before its layers are made sparse
        _dense("dense_n16384_step", "step", 1, 16, 16384, 16384, 64),
        # 128 x 256 pixel tokens of wide heads, the dense answer that a sparse layer is held against: matrix instructions
        _dense("dense_n32768_forward", "forward", 1, 4, 32768, 32768, 128),
        # one small grid of 16 heads of 64 channels: latency
        _norm("norm_n256_forward", "forward", 1, 256, 1024),
        # 128 x 128 tokens, batch 2: bytes
        _norm("norm_n16384_forward", "forward", 2, 16384, 1024),
        _norm("norm_n16384_backward", "backward", 2, 16384, 1024),
        # fp32, a width that is no multiple of a vector, LayerNorm before the block and none behind it
        _norm("norm_fp32_odd_backward", "backward", 3, 2704, 1001, dtype="f32", kind="layer", post=False),
        # the layer glue at the lowest and at the highest resolution
        _glue("glue_n4096_backward", 1, 16, 4096, 64),
        _glue("glue_n65536_backward", 1, 16, 65536, 64, L=3),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    """Attention of 1 to 65536 queries and 1 to 65536 keys, with a fp32 score matrix of at most 8 GB and, in fp32, 2048 tokens; norms of
    1 to 60000 rows of 8 to 8192 channels; glue of 256 to 65536 tokens."""
    op = rng.choice(["dense", "dense", "dense", "norm", "norm", "glue"])
    if op == "dense":
        while True:
            f32 = rng.random() < 0.2
            mode = rng.choice(["forward", "step"])
            kv_heads = rng.choice([1, 2, 3, 4, 8, 16])
            shared = rng.choice([1, 1, 2, 4, 8])
            d = rng.choice([64, 64, 128, 128, 32, 16])
            batch = rng.choice([1, 1, 2, 3, 5])
            form = rng.choice(["self", "self", "self", "cross", "few"])
            top = 2048 if f32 else 65536
            Nkv = _log(rng, 1, top)
            Nq = Nkv if form == "self" else _log(rng, 1, top) if form == "cross" else rng.choice([1, 2, 5, 16])
            heads = kv_heads * shared
            if heads <= 32 and batch * heads * Nq * Nkv <= 2 ** 31:
                return {k: v for k, v in _dense("", mode, batch, heads, Nq, Nkv, d, kv_heads, "f32" if f32 else "bf16", rng.random() < 0.4,
                                                rng.choice(["", "kv", "both"]), rng.random() < 0.5).items() if k != "name"}
    if op == "norm":
        while True:
            batch, N, C = rng.choice([1, 2, 3, 8]), _log(rng, 1, 30000), rng.choice([8 * _log(rng, 1, 1024), 8 * _log(rng, 1, 1024), _log(rng, 8, 8192)])
            if batch * N * C <= 2 ** 25:
                branch = rng.random() < 0.8
                return {k: v for k, v in _norm("", rng.choice(["forward", "backward"]), batch, N, C, rng.choice(["bf16", "bf16", "f32"]), rng.choice(["rms", "layer"]), branch,
                                               branch and rng.random() < 0.5, rng.random() < 0.8, rng.random() < 0.3, rng.random() < 0.7).items() if k != "name"}
    d, B = rng.choice([64, 64, 128, 32]), 16
    L = rng.choice([1, 2])
    while True:
        N = B ** L * _log(rng, 1, 4096)
        batch, heads = rng.choice([1, 2]), rng.choice([1, 2, 3, 8, 16])
        if 256 <= N <= 65536 and N // B ** L <= 4096 and batch * heads * N * d <= 2 ** 26:
            return {k: v for k, v in _glue("", batch, heads, N, d, B, L, rng.choice(["bf16", "bf16", "f32"])).items() if k != "name"}


# ------------------------------------------------------------------------------------------------ inputs

def _type(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _lens(c, gen):
    """(q_lens, kv_lens) of a padded batch: the longest has the whole length, the others any; in self attention both are the same."""
    if not c["lens"]:
        return None, None
    share = torch.rand(c["batch"], generator=gen, device="cuda")
    share[0] = 1.0
    kv = (share * c["Nkv"]).ceil().clamp(1, c["Nkv"]).to(torch.int32)
    q = (share * c["Nq"]).ceil().clamp(1, c["Nq"]).to(torch.int32) if c["lens"] == "both" else None
    return q, kv


def _heads(c, gen, heads, N):
    x = torch.randn(c["batch"], *((N, heads) if c["tokens_first"] else (heads, N)), c["d"], generator=gen, device="cuda").to(_type(c))
    return x.transpose(1, 2) if c["tokens_first"] else x


def _dense_inputs(c, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"Q": _heads(c, gen, c["heads"], c["Nq"]), "K": _heads(c, gen, c["kv_heads"], c["Nkv"]), "V": _heads(c, gen, c["kv_heads"], c["Nkv"])}
    s["q_lens"], s["kv_lens"] = _lens(c, gen)
    if c["mode"] == "step":
        s["dO"] = _heads(c, gen, c["heads"], c["Nq"])
    return s


def _norm_inputs(c, seed):
    """The residual stream grows with depth and has a few wide channels; gains, gates and modulations are what some training leaves."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rows = lambda k: (k * torch.randn(c["batch"], c["N"], c["C"], generator=gen, device="cuda"))
    vec = lambda a, k, *n: a + k * torch.randn(*n, c["C"], generator=gen, device="cuda")
    width = 1.0 + 3.0 * (torch.rand(c["C"], generator=gen, device="cuda") < 0.02)
    mods = 1 if c["shared"] else c["batch"]
    s = {"x": (rows(2.0) * width + 0.1).to(_type(c))}
    s["gain"] = vec(1.0, 0.1, 1)[0]
    s["branch"] = rows(0.7).add_(0.05).to(_type(c)) if c["branch"] else None
    s["gain_branch"] = vec(0.5, 0.1, 1)[0] if c["post"] else None
    s["gate"] = vec(0.3, 0.2, mods).to(_type(c)) if c["branch"] and c["mod"] else None
    s["scale"] = vec(0.0, 0.2, mods).to(_type(c)) if c["mod"] else None
    s["shift"] = vec(0.0, 0.2, mods).to(_type(c)) if c["mod"] and c["shift"] else None
    if c["mode"] == "backward":           # x is the stream behind the sum, as the forward pass stored it, with its rows' statistics
        s["dy"], s["dx_out"] = rows(0.02).to(_type(c)), rows(0.02).to(_type(c))
        mean = [t.double().mean(2) if c["kind"] == "layer" else torch.zeros(c["batch"], c["N"], dtype=torch.float64, device="cuda") for t in (s["x"], s["branch"]) if t is not None]
        rstd = [((t.double() - m[..., None]).square().mean(2) + 1e-6).rsqrt() for t, m in zip((t for t in (s["x"], s["branch"]) if t is not None), mean)]
        if not c["post"]:
            mean, rstd = mean[:1], rstd[:1]
        pad = [torch.zeros_like(mean[0])] * (2 - 2 * (len(mean) - 1))
        s["stats"] = torch.stack([v for p in zip(mean, rstd) for v in p] + pad, 2).float().contiguous()
    return s


def _glue_inputs(c, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    shape = (c["batch"], c["heads"], c["N"], c["d"])
    s = {n: (k * torch.randn(*shape, generator=gen, device="cuda")).to(_type(c)) for n, k in (("Q", 3.0), ("K", 3.0), ("dQ", 0.02), ("dK", 0.02))}
    s["gq"], s["gk"] = (1.0 + 0.1 * torch.randn(c["d"], generator=gen, device="cuda") for _ in range(2))
    pos = torch.arange(c["N"], dtype=torch.float64, device="cuda")
    freq = 10000.0 ** (-torch.arange(c["d"] // 2, dtype=torch.float64, device="cuda") / (c["d"] // 2))
    angle = pos[:, None] * freq
    s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    return s


def prepare(case, seed):
    c = case
    s = {"case": c}
    if c["op"] == "dense":
        s |= _dense_inputs(c, seed)
        if own:
            from paper_2512_16615_amd import llsa
            strides = {n + "_stride": s[t].stride()[:3] for n, t in (("q", "Q"), ("k", "K"), ("v", "V"), ("o", "Q"))}
            s["plan"] = llsa.DensePlan(c["batch"], c["heads"], c["Nq"], c["Nkv"], c["d"], kv_heads=c["kv_heads"], causal=c["causal"],
                                       dtype=llsa.F32 if c["dtype"] == "f32" else llsa.BF16, **strides)
            s["ws"] = s["plan"].alloc_workspace(c["mode"] == "step")
            s["O"] = torch.empty_like(s["Q"])
            s["LSE"] = torch.empty(c["batch"], c["heads"], c["Nq"], dtype=torch.float32, device="cuda")
            if c["mode"] == "step":
                s["grads"] = [torch.empty_like(s[n]) for n in ("Q", "K", "V")]
    elif c["op"] == "norm":
        s |= _norm_inputs(c, seed)
        if own:
            from paper_2512_16615_amd import llsa
            s["plan"] = llsa.NormPlan(c["batch"], c["N"], c["C"], kind=llsa.NORM_LAYER if c["kind"] == "layer" else llsa.NORM_RMS, eps=1e-6, residual_scale=0.8,
                                      dtype=llsa.F32 if c["dtype"] == "f32" else llsa.BF16, mod_dtype=llsa.F32 if c["dtype"] == "f32" else llsa.BF16,
                                      mod_stride=0 if c["shared"] else c["C"])
            s["ws"] = s["plan"].alloc_workspace()
            s["a"], s["b"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
            if c["mode"] == "forward":
                s["stats"] = torch.empty(c["batch"], c["N"], 4, dtype=torch.float32, device="cuda")
    else:
        s |= _glue_inputs(c, seed)
        if own:
            from paper_2512_16615_amd import llsa
            s["plan"] = llsa.Plan(c["batch"], c["heads"], c["N"], c["d"], c["B"], 8, c["L"], dtype=llsa.F32 if c["dtype"] == "f32" else llsa.BF16)
            s["ws"] = s["plan"].alloc_glue_workspace()
            s["dQpre"], s["dKpre"] = torch.empty_like(s["Q"]), torch.empty_like(s["K"])
    return s


# ------------------------------------------------------------------------------------------------ the plain forms, and the calls

def _own_dense(s):
    from paper_2512_16615_amd import llsa
    O, LSE = llsa.dense_forward(s["plan"], s["Q"], s["K"], s["V"], s["q_lens"], s["kv_lens"], s["O"], s["LSE"], s["ws"])
    out = {"O": O, "LSE": LSE}
    if "dO" in s:
        out["dQ"], out["dK"], out["dV"] = llsa.dense_backward(s["plan"], s["Q"], s["K"], s["V"], O, LSE, s["dO"], s["q_lens"], s["kv_lens"], *s["grads"], s["ws"])
    return out


def _own_norm(s):
    from paper_2512_16615_amd import llsa
    names = ("gain_branch", "gate", "gain", "scale", "shift")
    if "dy" not in s:
        x_out, y, stats = llsa.norm_forward(s["plan"], s["x"], s["branch"], **{n: s[n] for n in names}, x_out=s["a"] if s["branch"] is not None else None, y=s["b"], stats=s["stats"])
        return {"x_out": x_out if s["branch"] is not None else None, "y": y}
    return llsa.norm_backward(s["plan"], s["x"], s["dy"], s["stats"], s["branch"], **{n: s[n] for n in names}, dx_out=s["dx_out"], dx=s["a"],
                              dbranch=s["b"] if s["branch"] is not None else None, workspace=s["ws"])


def _own_glue(s):
    from paper_2512_16615_amd import llsa
    dQ, dK, dgq, dgk = llsa.qknorm_rope_backward(s["plan"], s["Q"], s["K"], s["gq"], s["gk"], s["cos"], s["sin"], s["dQ"], s["dK"], 1e-6,
                                                 dQpre=s["dQpre"], dKpre=s["dKpre"], workspace=s["ws"])
    return {"dQ": dQ, "dK": dK, "dgq": dgq, "dgk": dgk}


def _plain_dense(s):
    c = s["case"]
    b, H, G, d = c["batch"], c["kv_heads"], c["heads"] // c["kv_heads"], c["d"]
    Q, K, V = (s[n].float() for n in ("Q", "K", "V"))
    i, j = torch.arange(c["Nq"], device="cuda"), torch.arange(c["Nkv"], device="cuda")
    nq = torch.full((b,), c["Nq"], device="cuda") if s["q_lens"] is None else s["q_lens"]
    nk = torch.full((b,), c["Nkv"], device="cuda") if s["kv_lens"] is None else s["kv_lens"]
    masked = c["causal"] or s["kv_lens"] is not None
    Kt = K.transpose(2, 3).contiguous()
    rows = Q.reshape(b, H, G * c["Nq"], d)                                                         # the heads that share one key head, one after the other
    P = torch.matmul(rows, Kt).view(b, H, G, c["Nq"], c["Nkv"]).mul_(1.0 / math.sqrt(d))
    if masked:
        seen = (i[None, :, None] < nq[:, None, None]) & (j[None, None, :] < nk[:, None, None])
        if c["causal"]:
            seen &= j[None, None, :] <= i[None, :, None] + (nk - nq)[:, None, None]
        P.masked_fill_(~seen[:, None, None], -math.inf)
    m = P.amax(4, keepdim=True).clamp_min(-3e38)
    P.sub_(m).exp_()
    l = P.sum(4, keepdim=True)
    LSE = (m + l.log())[..., 0].reshape(b, c["heads"], c["Nq"])
    P.div_(l.clamp_min(1e-38))
    O = torch.matmul(P.view(b, H, G * c["Nq"], c["Nkv"]), V)
    out = {"O": O.view(b, c["heads"], c["Nq"], d).to(s["Q"].dtype), "LSE": LSE}
    if "dO" in s:
        dO = s["dO"].float().reshape(b, H, G * c["Nq"], d)
        if s["q_lens"] is not None:
            dO = dO.view(b, c["heads"], c["Nq"], d).masked_fill(i[None, None, :, None] >= nq[:, None, None, None], 0.0).view(b, H, G * c["Nq"], d)
        P = P.view(b, H, G * c["Nq"], c["Nkv"])
        dS = torch.matmul(dO, V.transpose(2, 3).contiguous()).sub_((dO * O).sum(3, keepdim=True)).mul_(P).mul_(1.0 / math.sqrt(d))
        out["dV"] = torch.matmul(P.transpose(2, 3), dO).to(s["V"].dtype)
        out["dQ"] = torch.matmul(dS, K).view(b, c["heads"], c["Nq"], d).to(s["Q"].dtype)
        out["dK"] = torch.matmul(dS.transpose(2, 3), rows).to(s["K"].dtype)
    return out


def _normed(c, x):
    x = x - x.mean(2, keepdim=True) if c["kind"] == "layer" else x
    return x * torch.rsqrt(x.square().mean(2, keepdim=True) + 1e-6)


def _plain_norm(s):
    c, kind = s["case"], s["x"].dtype
    up = lambda t: None if t is None else t.float()
    x, b, gb, gate, gain, scale, shift = (up(s[n]) for n in ("x", "branch", "gain_branch", "gate", "gain", "scale", "shift"))
    mod = lambda t, a: a if t is None else t[:, None, :]
    if "dy" not in s:
        if b is not None:
            z = _normed(c, b) * gb if c["post"] else b
            x = x + 0.8 * mod(gate, 1.0) * z
            x_out = x.to(kind)
            x = x_out.float()                # the block's own input is the stream as it is stored
        y = _normed(c, x) * gain * (1.0 + mod(scale, 0.0)) + mod(shift, 0.0)
        return {"x_out": x_out if b is not None else None, "y": y.to(kind)}
    over = (0, 1) if c["shared"] else (1,)
    st = s["stats"][..., None]
    fold = lambda t, n: t.sum(over).view(n, c["C"])
    n = 1 if c["shared"] else c["batch"]
    dy, out = s["dy"].float(), {}
    xhat = (x - st[:, :, 0]) * st[:, :, 1]
    g = dy * gain * (1.0 + mod(scale, 0.0))
    dx = g - xhat * (g * xhat).mean(2, keepdim=True)
    dx = (dx - g.mean(2, keepdim=True) if c["kind"] == "layer" else dx) * st[:, :, 1] + s["dx_out"].float()
    out["dx"] = dx.to(kind)
    out["dgain"] = (dy * xhat * (1.0 + mod(scale, 0.0))).sum((0, 1))
    if scale is not None:
        out["dscale"] = fold(dy * xhat * gain, n)
    if shift is not None:
        out["dshift"] = fold(dy, n)
    if b is not None:
        u = (b - st[:, :, 2]) * st[:, :, 3] if c["post"] else b
        w = 0.8 * mod(gate, 1.0) * dx
        if gate is not None:
            out["dgate"] = fold(0.8 * dx * (u * gb if c["post"] else u), n)
        if c["post"]:
            out["dgain_branch"] = (w * u).sum((0, 1))
            w = w * gb
            db = w - u * (w * u).mean(2, keepdim=True)
            w = (db - w.mean(2, keepdim=True) if c["kind"] == "layer" else db) * st[:, :, 3]
        out["dbranch"] = w.to(kind)
    return out


def _plain_glue_of(x, dy, gamma, cos, sin):
    x, dy = x.float(), dy.float()
    a, b = dy[..., 0::2], dy[..., 1::2]
    dy = torch.stack([a * cos + b * sin, b * cos - a * sin], 4).flatten(3)
    r = torch.rsqrt(x.square().mean(3, keepdim=True) + 1e-6)
    xhat, g = x * r, dy * gamma
    return r * (g - xhat * (g * xhat).mean(3, keepdim=True)), (dy * xhat).sum((0, 1, 2))


def _plain_glue(s):
    dQ, dgq = _plain_glue_of(s["Q"], s["dQ"], s["gq"], s["cos"], s["sin"])
    dK, dgk = _plain_glue_of(s["K"], s["dK"], s["gk"], s["cos"], s["sin"])
    return {"dQ": dQ.to(s["Q"].dtype), "dK": dK.to(s["K"].dtype), "dgq": dgq, "dgk": dgk}


def run(s):
    op = s["case"]["op"]
    if own:
        return _own_dense(s) if op == "dense" else _own_norm(s) if op == "norm" else _own_glue(s)
    return _plain_dense(s) if op == "dense" else _plain_norm(s) if op == "norm" else _plain_glue(s)


# ------------------------------------------------------------------------------------------------ 64 bits

def _exact_dense(c, s):
    out = {"O": torch.zeros(c["batch"], c["heads"], c["Nq"], c["d"], dtype=torch.float64, device="cuda"),
           "LSE": torch.full((c["batch"], c["heads"], c["Nq"]), -math.inf, dtype=torch.float64, device="cuda")}
    step = c["mode"] == "step"
    if step:
        out |= {n: torch.zeros(c["batch"], h, N, c["d"], dtype=torch.float64, device="cuda") for n, h, N in (("dQ", c["heads"], c["Nq"]), ("dK", c["kv_heads"], c["Nkv"]), ("dV", c["kv_heads"], c["Nkv"]))}
    for b in range(c["batch"]):
        nq, nk = (N if t is None else int(t[b]) for t, N in ((s["q_lens"], c["Nq"]), (s["kv_lens"], c["Nkv"])))
        first = max(0, nq - nk) if c["causal"] else 0                 # the queries before see nothing
        for h in range(c["heads"]):
            k = h // (c["heads"] // c["kv_heads"])
            K, V = s["K"][b, k, :nk].double(), s["V"][b, k, :nk].double()
            for r0 in range(first, nq, 16384):
                r1 = min(nq, r0 + 16384)
                Q = s["Q"][b, h, r0:r1].double()
                S = Q @ K.T / math.sqrt(c["d"])
                if c["causal"]:
                    S += torch.triu(torch.full_like(S, -math.inf), nk - nq + r0 + 1)
                lse = torch.logsumexp(S, 1)
                out["LSE"][b, h, r0:r1] = lse
                P = torch.exp(S - lse[:, None])
                O = P @ V
                out["O"][b, h, r0:r1] = O
                if step:
                    dO = s["dO"][b, h, r0:r1].double()
                    dS = P * (dO @ V.T - (dO * O).sum(1, keepdim=True)) / math.sqrt(c["d"])
                    out["dQ"][b, h, r0:r1] = dS @ K
                    out["dK"][b, k, :nk] += dS.T @ Q
                    out["dV"][b, k, :nk] += P.T @ dO
    return out


def _exact_norm(c, s):
    """The definition, differentiated by automatic differentiation; the backward pass starts from the stream as it is given."""
    D = lambda n: None if s[n] is None else s[n].double().requires_grad_(c["mode"] == "backward")
    t = {n: D(n) for n in ("x", "branch", "gain_branch", "gate", "gain", "scale", "shift")}
    rows = lambda v: v[:, None, :] if v.shape[0] == c["batch"] else v[None]

    def unit(v):
        if c["kind"] == "layer":
            return (v - v.mean(-1, keepdim=True)) / (v.var(-1, unbiased=False, keepdim=True) + 1e-6).sqrt()
        return v / ((v * v).mean(-1, keepdim=True) + 1e-6).sqrt()

    add = None
    if t["branch"] is not None:
        add = unit(t["branch"]) * t["gain_branch"] if c["post"] else t["branch"]
        add = 0.8 * (add if t["gate"] is None else rows(t["gate"]) * add)
    x = t["x"]
    if c["mode"] == "forward" and add is not None:
        x = (x + add).to(s["x"].dtype)
        x_out, x = x, x.double()
    y = unit(x) * t["gain"]
    y = y if t["scale"] is None else y * (1.0 + rows(t["scale"]))
    y = y if t["shift"] is None else y + rows(t["shift"])
    if c["mode"] == "forward":
        return {"x_out": None if add is None else t["x"] + add, "y": y}
    y.backward(s["dy"].double())
    dx = t["x"].grad + s["dx_out"].double()
    if add is not None:
        add.backward(dx)
    out = {"dx": dx}
    for n in ("branch", "gain_branch", "gate", "gain", "scale", "shift"):
        if t[n] is not None:
            out["d" + n] = t[n].grad
    return out


def _exact_glue(c, s):
    turn = torch.complex(s["cos"].double(), s["sin"].double())
    out = {}
    for x, dy, g, n, dg in (("Q", "dQ", "gq", "dQ", "dgq"), ("K", "dK", "gk", "dK", "dgk")):
        X, gamma = s[x].double().requires_grad_(), s[g].double().requires_grad_()
        Y = X / ((X * X).mean(-1, keepdim=True) + 1e-6).sqrt() * gamma
        Z = torch.view_as_complex(Y.unflatten(-1, (-1, 2))) * turn
        torch.view_as_real(Z).flatten(-2).backward(s[dy].double())
        out[n], out[dg] = X.grad, gamma.grad
    return out


def exact(case, seed):
    c = case
    if c["op"] == "dense":
        return _exact_dense(c, _dense_inputs(c, seed))
    return _exact_norm(c, _norm_inputs(c, seed)) if c["op"] == "norm" else _exact_glue(c, _glue_inputs(c, seed))


# ------------------------------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    """Dense attention: two products of every pair of a query and a key that the mask leaves, a step five more; lengths of a padded batch are taken
    as half, on the average.  Norms and glue: bytes; some operations a value."""
    c = case
    elt = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "dense":
        share = 1.0 if not c["lens"] else (1.0 + 0.5 * (c["batch"] - 1)) / c["batch"]
        q, kv = c["batch"] * c["heads"] * c["Nq"] * c["d"], c["batch"] * c["kv_heads"] * c["Nkv"] * c["d"]
        nq, nk = q * (share if c["lens"] == "both" else 1.0), kv * share
        first = max(0.0, c["Nkv"] - c["Nq"] + 0.5) / c["Nkv"]                                    # share of the keys that the first query sees
        seen = 1.0 if not c["causal"] else 0.5 * (1.0 + first) if c["Nq"] <= c["Nkv"] else 0.5 * c["Nkv"] / c["Nq"]
        pairs = c["heads"] * c["Nq"] * c["Nkv"] * c["batch"] * seen * (share if c["lens"] == "" or c["lens"] == "kv" else (1.0 + 0.33 * (c["batch"] - 1)) / c["batch"])
        data, flops = elt * (nq + q + 2 * nk) + 4 * q // c["d"], 4.0 * c["d"] * pairs
        if c["mode"] == "step":
            data, flops = data + elt * (nq + q + 2 * kv), flops + 10.0 * c["d"] * pairs
        return {"bytes": data, "flops": flops}
    if c["op"] == "norm":
        rows = c["batch"] * c["N"] * c["C"]
        moved = (2 + 2 * c["branch"]) if c["mode"] == "forward" else (4 + 2 * c["branch"])
        return {"bytes": moved * rows * elt, "flops": (10.0 if c["mode"] == "forward" else 30.0) * rows}
    rows = c["batch"] * c["heads"] * c["N"] * c["d"]
    return {"bytes": 6 * rows * elt + 4 * c["N"] * c["d"], "flops": 2 * 20.0 * rows}
