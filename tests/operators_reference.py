"""Plain 64-bit forms of dense attention, the norms between two blocks and the glue's gradient, with bounds on how far a kernel may be from
them.  Elementary torch operations on whichever device the tensors are on; nothing of the package.

Bounds.  u = half a step of the I/O type (finfo.eps / 2), w = 2^-24.  Every bound is formed element by element from the 64-bit values:

* a sum of n products in fp32 is off by at most n w times the sum of their magnitudes;
* a probability is off by a relative e_p = 2 max_j |error of the exponent| + 2^-20 (the hardware's exponential and logarithm are good to 2 steps
  each), the exponent by scale (d + 2) w |q| |k| + 4 w |s|;
* the products with P and dS take them rounded to the I/O type (bf16 path): u more for each;
* O, which D = rowsum(dO O) is formed from, is off by its own bound.
"""
import math

import torch

W = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def expand(t, G):
    return t.repeat_interleave(G, 1)


def dense(Q, K, V, dO=None, causal=False, q_lens=None, kv_lens=None, sm_scale=None, dtype=torch.float32, bounds=True):
    """O, LSE (and dQ, dK, dV) in 64 bits, and a dict of bounds of the same names.  Rows behind the lengths and unseen keys are taken out before
    anything is computed, so that nothing that they hold can reach a result."""
    b, H, Nq, d = Q.shape
    kvh, Nkv = K.shape[1:3]
    G = H // kvh
    scale = sm_scale or 1.0 / math.sqrt(d)
    dev = Q.device
    out = {"O": torch.zeros(b, H, Nq, d, dtype=torch.float64, device=dev), "LSE": torch.full((b, H, Nq), -math.inf, dtype=torch.float64, device=dev)}
    if dO is not None:
        out |= {"dQ": torch.zeros(b, H, Nq, d, dtype=torch.float64, device=dev), "dK": torch.zeros(b, kvh, Nkv, d, dtype=torch.float64, device=dev),
                "dV": torch.zeros(b, kvh, Nkv, d, dtype=torch.float64, device=dev)}
    tol = {n: torch.zeros_like(t) for n, t in out.items()}
    u = half_step(dtype)
    for i in range(b):
        nq = Nq if q_lens is None else max(0, min(Nq, int(q_lens[i])))
        nk = Nkv if kv_lens is None else max(0, min(Nkv, int(kv_lens[i])))
        if nq == 0 or nk == 0:
            continue
        first = max(0, nq - nk) if causal else 0
        if first >= nq:
            continue
        q = Q[i, :, first:nq].double()
        k, v = expand(K[i:i + 1, :, :nk], G)[0].double(), expand(V[i:i + 1, :, :nk], G)[0].double()
        seen = torch.ones(nq - first, nk, dtype=torch.bool, device=dev)
        if causal:
            seen = torch.arange(nk, device=dev)[None] <= torch.arange(first, nq, device=dev)[:, None] + nk - nq
        # what no query sees must not reach a product: with a NaN there, 0 times it would
        zero = lambda t, at: torch.where(at, t, torch.zeros((), dtype=torch.float64, device=dev))
        s = q @ k.transpose(1, 2) * scale
        s = torch.where(seen, s, torch.full((), -math.inf, dtype=torch.float64, device=dev))
        lse = torch.logsumexp(s, 2)
        p = torch.exp(s - lse[..., None])
        clean = lambda t: torch.where(torch.isfinite(t), t, torch.zeros((), dtype=torch.float64, device=dev))
        product = lambda m, t: m @ t if bool(torch.isfinite(t).all()) else _masked_product(m, t)
        o = product(p, v)
        out["O"][i, :, first:nq], out["LSE"][i, :, first:nq] = o, lse
        if bounds:
            es = scale * (d + 2) * W * (q.abs() @ clean(k).abs().transpose(1, 2)) + 4 * W * clean(s).abs()
            es = zero(es, seen).amax(2)
            ep = (2 * es + 2.0 ** -20)[..., None] + (nk + 4) * W
            av = p @ clean(v).abs()
            to = u * o.abs() + (ep + (u if u > W else 0.0)) * av
            tol["O"][i, :, first:nq] = to
            tol["LSE"][i, :, first:nq] = es + 2.0 ** -20 + 4 * W * lse.abs() + nk * W
        if dO is None:
            continue
        g = dO[i, :, first:nq].double()
        dp = product_t(g, v, seen)
        delta = (g * clean(o)).sum(2, keepdim=True) if not bool(torch.isfinite(o).all()) else (g * o).sum(2, keepdim=True)
        ds = torch.where(seen, p * (dp - delta) * scale, torch.zeros((), dtype=torch.float64, device=dev))
        dq = product(ds, k)
        dv, dk = product(p.transpose(1, 2), g), product(ds.transpose(1, 2), q)
        fold = lambda t: t.view(kvh, G, nk, d).sum(1)
        out["dQ"][i, :, first:nq], out["dK"][i, :, :nk], out["dV"][i, :, :nk] = dq, fold(dk), fold(dv)
        if bounds:
            ga, va, ka, qa = g.abs(), clean(v).abs(), clean(k).abs(), clean(q).abs()
            ed = (ga * (to + (d + 1) * W * clean(o).abs())).sum(2, keepdim=True)
            edp = (d + 2) * W * (ga @ va.transpose(1, 2))
            eds = clean(ds).abs() * (ep + 4 * W + (u if u > W else 0.0)) + scale * p * (ed + edp)
            tol["dQ"][i, :, first:nq] = u * dq.abs() + eds @ ka + nk * W * (clean(ds).abs() @ ka)
            n = G * nq
            tk = eds.transpose(1, 2) @ qa + n * W * (clean(ds).abs().transpose(1, 2) @ qa)
            pv = (p * (ep + n * W + (u if u > W else 0.0))).transpose(1, 2) @ ga
            tol["dK"][i, :, :nk] = u * out["dK"][i, :, :nk].abs() + fold(tk)
            tol["dV"][i, :, :nk] = u * out["dV"][i, :, :nk].abs() + fold(pv)
    return out, {n: t * 1.01 + 1e-30 for n, t in tol.items()}


def _masked_product(m, t):
    """m @ t where the rows of t that m's zeros meet may hold anything: what is not finite is added where m is not 0."""
    fine = torch.isfinite(t)
    zero = torch.zeros((), dtype=t.dtype, device=t.device)
    out = m @ torch.where(fine, t, zero)
    for h, r, c in (~fine).nonzero():
        out[h, :, c] += torch.where(m[h, :, r] != 0, m[h, :, r] * t[h, r, c], zero)
    return out


def product_t(g, v, seen):
    """g v^T at the places that are seen."""
    out = g @ v.transpose(1, 2)
    return torch.where(seen, out, torch.zeros((), dtype=out.dtype, device=out.device))


def unit(x, layer, eps):
    m = x.mean(-1, keepdim=True) if layer else torch.zeros_like(x[..., :1])
    r = ((x - m).square().mean(-1, keepdim=True) + eps).rsqrt()
    return (x - m) * r, m, r


def _rows(t):
    return t[:, None, :]


def norm_forward(x, branch=None, gain_branch=None, gate=None, gain=None, scale=None, shift=None, layer=False, eps=1e-6, alpha=1.0, store=None):
    """x', y in 64 bits; `store`: the type x' is rounded to before y is formed (as the operator does)."""
    D = lambda t: None if t is None else t.double()
    x, branch, gain_branch, gate, gain, scale, shift = (D(t) for t in (x, branch, gain_branch, gate, gain, scale, shift))
    if branch is not None:
        z = branch if gain_branch is None else unit(branch, layer, eps)[0] * gain_branch
        x = x + alpha * (z if gate is None else _rows(gate) * z)
    h = x if store is None else x.to(store).double()
    y = unit(h, layer, eps)[0]
    y = y if gain is None else y * gain
    y = y if scale is None else y * (1 + _rows(scale))
    y = y if shift is None else y + _rows(shift)
    return x, y


def norm_backward(x_out, dy, branch=None, gain_branch=None, gate=None, gain=None, scale=None, dx_out=None, layer=False, eps=1e-6, alpha=1.0, shared=False):
    """The formulas of the header in 64 bits; each sum over rows comes with the sum of its magnitudes (for the bound of its rounding)."""
    D = lambda t: None if t is None else t.double()
    h, dy, branch, gain_branch, gate, gain, scale, dx_out = (D(t) for t in (x_out, dy, branch, gain_branch, gate, gain, scale, dx_out))
    one = torch.ones((), dtype=torch.float64, device=h.device)
    opt = lambda t: one if t is None else t
    s1, ga = (1 + (_rows(scale) if scale is not None else 0.0)), opt(gain)
    res, mag = {}, {}

    def sums(name, t, over_rows_only, w=1.0):
        t = t * w * torch.ones_like(h)
        if over_rows_only:
            res[name], mag[name] = t.sum((0, 1)), t.abs().sum((0, 1))
        else:
            res[name], mag[name] = t.sum(1), t.abs().sum(1)
            if shared:
                res[name], mag[name] = res[name].sum(0, keepdim=True), mag[name].sum(0, keepdim=True)

    d = torch.zeros_like(h) if dx_out is None else dx_out
    if dy is not None:
        hh, _, r = unit(h, layer, eps)
        p = dy * ga * s1
        d = d + r * (p - hh * (p * hh).mean(-1, keepdim=True) - (p.mean(-1, keepdim=True) if layer else 0.0))
        sums("dgain", dy * hh, True, s1)
        sums("dscale", dy * hh, False, ga)
        sums("dshift", dy, False)
    res["dx"] = d
    if branch is not None:
        gt = alpha * (_rows(gate) if gate is not None else one)
        u, _, r = unit(branch, layer, eps) if gain_branch is not None else (branch, None, None)
        sums("dgate", alpha * d * u, False, opt(gain_branch))
        w = gt * d * opt(gain_branch)
        if gain_branch is not None:
            sums("dgain_branch", gt * d * u, True)
            w = r * (w - u * (w * u).mean(-1, keepdim=True) - (w.mean(-1, keepdim=True) if layer else 0.0))
        res["dbranch"] = w
    return res, mag


def glue(x, gamma, cos, sin, eps=1e-6):
    y = unit(x, False, eps)[0] * gamma
    a, b = y[..., 0::2], y[..., 1::2]
    return torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)


def glue_backward(x, gamma, cos, sin, g, eps=1e-6):
    """dx, dgamma and the sum of dgamma's magnitudes, in 64 bits."""
    x, gamma, cos, sin, g = (t.double() for t in (x, gamma, cos, sin, g))
    a, b = g[..., 0::2], g[..., 1::2]
    dy = torch.stack([a * cos + b * sin, b * cos - a * sin], -1).flatten(-2)
    xh, _, r = unit(x, False, eps)
    p = dy * gamma
    return r * (p - xh * (p * xh).mean(-1, keepdim=True)), (dy * xh).sum((0, 1, 2)), (dy * xh).abs().sum((0, 1, 2))
