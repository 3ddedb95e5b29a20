"""The norms between two blocks and the glue's gradient against 64 bits.

Bounds, u half a step of the I/O type and w = 2^-24: a row's statistics are sums of C values in fp32, off by a relative (C / 16 + 16) w at most
(a thread adds 16 in turn, the rest is a tree; the bound takes C w, which is more), so every value of a normed row is off by a few C w of the row's
largest magnitude, and x' by one more rounding.  y is compared with the 64-bit norm of the x' that the kernel stored.  A sum over R rows: at most
R w of the sum of its magnitudes, plus what its terms are off by."""
import math

import pytest
import torch

from paper_2512_16615_amd import inputs, llsa
from tests import operators_reference as R

pytestmark = pytest.mark.gpu

W = 2.0 ** -24
SHAPES = [(1, 1, 1), (2, 3, 5), (1, 7, 8), (3, 5, 64), (2, 33, 127), (1, 300, 128), (2, 19, 129), (3, 40, 255), (2, 17, 512), (1, 9, 513), (2, 130, 1000), (2, 33, 1024),
          (1, 5, 1025), (2, 6, 2048), (1, 21, 2049), (3, 2, 4097), (1, 3, 8191), (2, 4, 8192), (5, 700, 24), (1, 3000, 72)]
#: branch, norm behind it, gate, gain, scale, shift
PARTS = [(1, 1, 1, 1, 1, 1), (1, 0, 1, 0, 1, 1), (1, 1, 0, 1, 0, 0), (0, 0, 0, 1, 1, 1), (0, 0, 0, 0, 0, 0), (1, 0, 0, 0, 0, 0)]


def _inputs(batch, N, C, dtype, mod_dtype, parts, shared, packed, seed=0):
    gen = torch.Generator().manual_seed(seed)
    rows = lambda k, a=0.0: (a + k * torch.randn(batch, N, C, generator=gen)).to(dtype).cuda()
    m = 1 if shared else batch
    pack = (0.3 * torch.randn(m, 3 * C if packed else C, generator=gen)).to(mod_dtype).cuda()
    mod = lambda i: pack[:, i * C:(i + 1) * C] if packed else (0.3 * torch.randn(m, C, generator=gen)).to(mod_dtype).cuda()
    gain = lambda: (1 + 0.1 * torch.randn(C, generator=gen)).cuda()
    x, branch, dy, dx_out = rows(2.0, 0.5), rows(0.7, -0.2), rows(0.5), rows(0.5)
    b, post, gate, g, s, t = parts
    return dict(x=x, branch=branch if b else None, gain_branch=gain() if post else None, gate=mod(0) if gate else None, gain=gain() if g else None,
                scale=mod(1) if s else None, shift=mod(2) if t else None), dy, dx_out


def _plan(batch, N, C, dtype, mod_dtype, layer, shared, packed):
    f = lambda t: llsa.F32 if t == torch.float32 else llsa.BF16
    return llsa.NormPlan(batch, N, C, kind=llsa.NORM_LAYER if layer else llsa.NORM_RMS, eps=1e-5, residual_scale=0.75, dtype=f(dtype), mod_dtype=f(mod_dtype),
                         mod_stride=0 if shared else 3 * C if packed else C)


def _close(name, got, want, bound):
    err = (got.double() - want).abs()
    over = float((err / (bound + 1e-30)).max())
    assert over <= 1.0, f"{name}: {over:.2f} of the bound, largest error {float(err.max()):.3e}"


def _run(shape, dtype, mod_dtype, layer, parts, shared, packed, want_dx_out=True):
    B, N, C = shape
    t, dy, dx_out = _inputs(B, N, C, dtype, mod_dtype, parts, shared, packed)
    dx_out = dx_out if want_dx_out else None
    p = _plan(B, N, C, dtype, mod_dtype, layer, shared, packed)
    u = R.half_step(dtype)
    x_out, y, stats = llsa.norm_forward(p, **t)
    want_x, _ = R.norm_forward(**t, layer=layer, eps=1e-5, alpha=0.75)
    _, want_y = R.norm_forward(x_out, None, None, None, t["gain"], t["scale"], t["shift"], layer, 1e-5)
    top = lambda v: v.abs().amax(-1, keepdim=True)
    cw = 8 * (C + 8) * W
    if t["branch"] is not None:
        _close("x_out", x_out, want_x, u * want_x.abs() + cw * (top(want_x) + top(t["x"].double()) + 4.0))
    # 1 / deviation of a row: at C = 1 or a constant row LayerNorm's deviation is eps alone, and an error of the mean is that much larger
    hr = R.unit(x_out.double(), layer, 1e-5)
    _close("y", y, want_y, u * want_y.abs() + cw * (top(want_y) + (hr[2] * top(x_out.double())) * 2.0 + 1.0))
    _close("stats", stats[..., 1], hr[2][..., 0], cw * (1 + hr[2][..., 0] * top(x_out.double())[..., 0]) * hr[2][..., 0])
    grads = llsa.norm_backward(p, x_out, dy, stats, t["branch"], t["gain_branch"], t["gate"], t["gain"], t["scale"], t["shift"], dx_out)
    torch.cuda.synchronize()
    want, mag = R.norm_backward(x_out, dy, t["branch"], t["gain_branch"], t["gate"], t["gain"], t["scale"], dx_out, layer, 1e-5, 0.75, shared)
    names = {"dx"} | {"d" + n for n in ("branch", "gain_branch", "gate", "gain", "scale", "shift") if t[n] is not None}
    assert set(grads) == names
    # a row's factor of its own error: what its statistics multiply
    f = 1 + hr[2] * top(x_out.double())
    rb = R.unit(t["branch"].double(), layer, 1e-5)[2] if t["gain_branch"] is not None else None
    fb = f if rb is None else f * (1 + rb * top(t["branch"].double()))
    _close("dx", grads["dx"], want["dx"], u * want["dx"].abs() + cw * f * (top(want["dx"]) + 4 * hr[2] * top(dy.double()) * 2))
    if t["branch"] is not None:
        _close("dbranch", grads["dbranch"], want["dbranch"], u * want["dbranch"].abs() + cw * fb * (top(want["dbranch"]) + 8 * (1.0 if rb is None else rb) * (top(want["dx"]) + hr[2] * top(dy.double()))))
    worst = float(f.max()) if rb is None else float(fb.max())
    for n in sorted(names - {"dx", "dbranch"}):
        bound = (B * N + 8) * W * mag[n] + cw * worst * (mag[n] + mag[n].amax() * (1 + float(hr[2].max()) if C < 16 else 1.0))
        _close(n, grads[n], want[n].view_as(grads[n]), bound)
    return p, t, dy, dx_out, x_out, stats, grads


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_norm_sizes(shape, dtype):
    _run(shape, dtype, dtype, shape[2] > 1 and shape[1] % 2 == 0, PARTS[0], False, False)


@pytest.mark.parametrize("layer", [False, True], ids=["rms", "layer"])
@pytest.mark.parametrize("parts", PARTS, ids=lambda p: "".join(map(str, p)))
@pytest.mark.parametrize("shared,packed", [(False, False), (True, False), (False, True)], ids=["own", "shared", "packed"])
def test_norm_parts(layer, parts, shared, packed):
    _run((3, 21, 200), torch.bfloat16, torch.float32, layer, parts, shared, packed)
    _run((2, 10, 333), torch.float32, torch.bfloat16, layer, parts, shared, packed, want_dx_out=not shared)


def test_norm_in_place_and_without_a_next_block():
    """x' over x, the gradients over what they are formed from; a residual step without a norm in front of the next block."""
    p, t, dy, dx_out, x_out, stats, grads = _run((2, 50, 320), torch.bfloat16, torch.bfloat16, False, PARTS[0], False, False)
    x, br = t["x"].clone(), t["branch"].clone()
    a, y, _ = llsa.norm_forward(p, x, **{k: v for k, v in t.items() if k != "x"}, x_out=x)
    assert a.data_ptr() == x.data_ptr() and torch.equal(x, x_out)
    args = [t[n] for n in ("gain_branch", "gate", "gain", "scale", "shift")]
    for into in ("dy", "dx_out"):
        g, r = dy.clone(), dx_out.clone()
        br = t["branch"].clone()
        got = llsa.norm_backward(p, x_out, g, stats, br, *args, dx_out=r, dx=g if into == "dy" else r, dbranch=br)
        assert all(torch.equal(got[n], grads[n]) for n in grads)
    b, none, st = llsa.norm_forward(p, t["x"], t["branch"], t["gain_branch"], t["gate"], want_y=False)
    assert none is None and torch.equal(b, x_out) and torch.equal(st[..., 2:], stats[..., 2:]) and not st[..., :2].any()
    got = llsa.norm_backward(p, x_out, None, stats, t["branch"], t["gain_branch"], t["gate"], dx_out=dx_out)
    want, mag = R.norm_backward(x_out, None, t["branch"], t["gain_branch"], t["gate"], None, None, dx_out, False, 1e-5, 0.75)
    assert set(got) == {"dx", "dbranch", "dgain_branch", "dgate"} and torch.equal(got["dx"], dx_out)
    _close("dgate", got["dgate"], want["dgate"], 1e-4 * mag["dgate"])
    # without statistics kept: the same x' and y
    c, y2, _ = llsa.norm_forward(p, **t)
    assert torch.equal(c, x_out) and torch.equal(y2, y)


@pytest.mark.parametrize("layer", [False, True], ids=["rms", "layer"])
@pytest.mark.parametrize("shape,dtype", [((2, 9, 5), torch.bfloat16), ((2, 9, 511), torch.float32), ((1, 700, 1023), torch.bfloat16), ((2, 1100, 2050), torch.bfloat16), ((1, 2, 8189), torch.float32)], ids=str)
def test_norm_in_place_over_every_row_length(shape, dtype, layer):
    """Rows that several waves share, whose last vectors overlap, and that one thread has alone; a workspace that holds NaN."""
    p, t, dy, dx_out, x_out, stats, grads = _run(shape, dtype, torch.float32, layer, PARTS[0], False, False)
    rest = {k: v for k, v in t.items() if k not in ("x", "branch")}
    x, br = t["x"].clone(), t["branch"].clone()
    assert torch.equal(llsa.norm_forward(p, x, br, **rest, x_out=x)[0], x_out)
    x = t["x"].clone()
    assert torch.equal(llsa.norm_forward(p, x, br, **rest, x_out=br)[0], x_out)
    args = [t[n] for n in ("gain_branch", "gate", "gain", "scale", "shift")]
    ws = p.alloc_workspace()
    for into in ("dy", "dx_out"):
        g, r, br = dy.clone(), dx_out.clone(), t["branch"].clone()
        ws.fill_(0xff)
        got = llsa.norm_backward(p, x_out, g, stats, br, *args, dx_out=r, dx=g if into == "dy" else r, dbranch=br, workspace=ws)
        assert all(torch.equal(got[n], grads[n]) for n in grads), into


def test_a_row_that_is_not_finite_stays_alone():
    p, t, dy, dx_out, x_out, stats, grads = _run((2, 40, 136), torch.bfloat16, torch.bfloat16, True, PARTS[0], False, False)
    t["x"][0, 7, 3], t["branch"][1, 0, 135] = math.nan, math.inf
    a, y, _ = llsa.norm_forward(p, **t)
    bad = torch.zeros(2, 40, dtype=torch.bool, device="cuda")
    bad[0, 7] = bad[1, 0] = True
    assert torch.equal(a[~bad], x_out[~bad]) and torch.isfinite(y[~bad].float()).all() and not torch.isfinite(y[bad].float()).any()


def test_norm_replays_from_a_graph():
    B, N, C = 2, 100, 264
    t, dy, dx_out = _inputs(B, N, C, torch.bfloat16, torch.bfloat16, PARTS[0], False, False)
    p = _plan(B, N, C, torch.bfloat16, torch.bfloat16, False, False, False)
    ws = p.alloc_workspace()
    out = {}

    def step():
        x_out, y, stats = llsa.norm_forward(p, **t)
        out.update(llsa.norm_backward(p, x_out, dy, stats, t["branch"], t["gain_branch"], t["gate"], t["gain"], t["scale"], t["shift"], dx_out, workspace=ws), y=y)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    captured = dict(out)
    for rep in range(3):
        new, _, _ = _inputs(B, N, C, torch.bfloat16, torch.bfloat16, PARTS[0], False, False, seed=rep + 1)
        for n in t:
            t[n].copy_(new[n])
        step()
        torch.cuda.synchronize()
        want = {n: v.clone() for n, v in out.items()}
        ws.fill_(0xff)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(captured[n], want[n]) for n in want), rep


def test_norm_binding_refuses_what_does_not_fit():
    t, dy, _ = _inputs(2, 8, 32, torch.bfloat16, torch.float32, PARTS[0], False, False)
    p = _plan(2, 8, 32, torch.bfloat16, torch.float32, False, False, False)
    for n, bad in (("x", t["x"].float()), ("x", t["x"].cpu()), ("branch", t["branch"][:, :4]), ("gate", t["gate"].bfloat16()), ("gain", t["gain"][:31]), ("scale", t["scale"][:1]),
                   ("scale", t["scale"].repeat(1, 2)[:, :32]), ("x", t["x"].transpose(0, 1).contiguous().transpose(0, 1))):
        with pytest.raises(llsa.LlsaError):
            llsa.norm_forward(p, **(t | {n: bad}))
    x_out, y, stats = llsa.norm_forward(p, **t)
    with pytest.raises(llsa.LlsaError):
        llsa.norm_backward(p, x_out, dy, stats[..., :2], gain=t["gain"])
    with pytest.raises(llsa.LlsaError):
        llsa.norm_backward(p, x_out, dy, stats, gain=t["gain"], workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))


# ---- the gradient of the layer glue

GLUE = [dict(batch=1, heads=1, N=4, d=16, B=2, dtype="f32"), dict(batch=2, heads=3, N=36, d=32, B=6, dtype="bf16"), dict(batch=1, heads=5, N=320, d=64, B=16, dtype="bf16"),
        dict(batch=2, heads=2, N=272, d=128, B=16, dtype="bf16"), dict(batch=1, heads=3, N=1024, d=64, B=16, dtype="f32"), dict(batch=1, heads=2, N=130, d=128, B=2, dtype="f32"),
        dict(batch=3, heads=16, N=16, d=16, B=16, dtype="bf16")]


@pytest.mark.parametrize("c", GLUE, ids=lambda c: f"{c['dtype']}-{c['batch']}x{c['heads']}x{c['N']}-d{c['d']}")
def test_glue_backward(c):
    dtype = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    gen = torch.Generator().manual_seed(0)
    shape = (c["batch"], c["heads"], c["N"], c["d"])
    Q, K, dQ, dK = ((k * torch.randn(*shape, generator=gen)).to(dtype).cuda() for k in (3.0, 0.5, 1.0, 0.1))
    K[0, 0, 1] = 0                                   # a row of zeros: eps alone is under its root
    gq, gk = ((1 + 0.1 * torch.randn(c["d"], generator=gen)).cuda() for _ in range(2))
    cos, sin = (torch.from_numpy(t).cuda() for t in inputs.rope_tables(c["N"], c["d"]))
    p = llsa.Plan(c["batch"], c["heads"], c["N"], c["d"], c["B"], 2, 1, dtype=llsa.F32 if dtype == torch.float32 else llsa.BF16)
    ws = p.alloc_glue_workspace()
    ws.fill_(0xff)
    eps = 1e-4
    out = llsa.qknorm_rope_backward(p, Q, K, gq, gk, cos, sin, dQ, dK, eps, workspace=ws)
    u, cw = R.half_step(dtype), 8 * (c["d"] + 8) * W
    for x, g, gamma, dx, dgamma in ((Q, dQ, gq, out[0], out[2]), (K, dK, gk, out[1], out[3])):
        want, wantg, mag = R.glue_backward(x, gamma, cos, sin, g, eps)
        r = R.unit(x.double(), False, eps)[2]
        top = g.double().abs().amax(-1, keepdim=True) * r * 4
        _close("dx", dx, want, u * want.abs() + cw * top)
        _close("dgamma", dgamma, wantg, (c["batch"] * c["heads"] * c["N"] + 8) * W * mag + cw * mag)
    # over the incoming gradients, and the same bits again
    dQ2, dK2 = dQ.clone(), dK.clone()
    again = llsa.qknorm_rope_backward(p, Q, K, gq, gk, cos, sin, dQ2, dK2, eps, dQpre=dQ2, dKpre=dK2)
    assert again[0].data_ptr() == dQ2.data_ptr() and all(torch.equal(a, b) for a, b in zip(again, out))
    with pytest.raises(llsa.LlsaError):
        llsa.qknorm_rope_backward(p, Q, K, gq.double(), gk, cos, sin, dQ, dK)
    with pytest.raises(llsa.LlsaError):
        llsa.qknorm_rope_backward(p, Q, K, gq, gk, cos, sin, dQ[:, :, 1:], dK)


def test_glue_backward_replays_from_a_graph():
    gen = torch.Generator().manual_seed(1)
    p = llsa.Plan(1, 4, 256, 64, 16, 2, 1)
    Q, K, dQ, dK = (torch.randn(1, 4, 256, 64, generator=gen).bfloat16().cuda() for _ in range(4))
    gq, gk = (torch.ones(64, device="cuda") for _ in range(2))
    cos, sin = (torch.from_numpy(t).cuda() for t in inputs.rope_tables(256, 64))
    ws = p.alloc_glue_workspace()
    call = lambda: llsa.qknorm_rope_backward(p, Q, K, gq, gk, cos, sin, dQ, dK, workspace=ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for rep in range(3):
        dQ.copy_(torch.randn(1, 4, 256, 64, generator=gen).bfloat16())
        want = [t.clone() for t in call()]
        ws.fill_(0xff)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), rep


# ---- a block, forward and backward

def test_a_block_of_all_of_them_against_automatic_differentiation():
    """norm -> projections -> QK-Norm, RoPE, pooling -> sparse attention -> norm with gate and residual -> dense attention over conditioning tokens of two
    lengths -> residual, forward and backward, fp32.  With every block picked and no coarse tokens (K = N / B, Le = 0) the sparse layer is dense
    attention, so automatic differentiation in 64 bits says what every gradient is.  Twelve operators one after the other, each good to about 1e-6
    of the largest value: 1e-4 of it, the library's bound in fp32."""
    gen = torch.Generator().manual_seed(9)
    B, H, N, d, M, blk = 2, 2, 64, 32, 21, 4
    C = H * d
    r = lambda *s, k=1.0, a=0.0: (a + k * torch.randn(*s, generator=gen)).cuda()
    par = dict(x=r(B, N, C), scale=r(B, C, k=0.2), shift=r(B, C, k=0.2), gain=r(C, k=0.1, a=1.0), wq=r(C, C, k=C ** -0.5), wk=r(C, C, k=C ** -0.5), wv=r(C, C, k=C ** -0.5),
               gq=r(d, k=0.1, a=1.0), gk=r(d, k=0.1, a=1.0), gain_b=r(C, k=0.1, a=1.0), gate=r(B, C, k=0.3), gain2=r(C, k=0.1, a=1.0), wc=r(C, C, k=C ** -0.5),
               kc=r(B, M, H, d), vc=r(B, M, H, d))
    lens = torch.tensor([M, 8], dtype=torch.int32, device="cuda")
    cos, sin = (torch.from_numpy(t).cuda() for t in inputs.rope_tables(N, d))
    go = r(B, N, C)
    # 64 bits
    D = {n: t.double().requires_grad_() for n, t in par.items()}
    heads = lambda t: t.view(B, N, H, d).transpose(1, 2)
    flat = lambda t: t.transpose(1, 2).reshape(B, N, C)
    _, y = R.norm_forward(D["x"], gain=D["gain"], scale=D["scale"], shift=D["shift"])
    q, k, v = (heads(y @ D[n]) for n in ("wq", "wk", "wv"))
    q, k = R.glue(q, D["gq"], cos.double(), sin.double()), R.glue(k, D["gk"], cos.double(), sin.double())
    att = flat(torch.softmax(q @ k.transpose(2, 3) / math.sqrt(d), 3) @ v)
    x2, y2 = R.norm_forward(D["x"], att, D["gain_b"], D["gate"], D["gain2"])
    qc = heads(y2 @ D["wc"])
    s = (qc @ D["kc"].transpose(1, 2).transpose(2, 3) / math.sqrt(d)).masked_fill(torch.arange(M, device="cuda")[None, None, None] >= lens[:, None, None, None], -math.inf)
    out = x2 + flat(torch.softmax(s, 3) @ D["vc"].transpose(1, 2))
    (out * go.double()).sum().backward()
    # the operators
    n1 = llsa.NormPlan(B, N, C, dtype=llsa.F32)
    layer = llsa.Plan(B, H, N, d, blk, N // blk, 1, Le=0, dtype=llsa.F32)
    tok = (N * C, d, C)
    cross = llsa.DensePlan(B, H, N, M, d, dtype=llsa.F32, q_stride=tok, k_stride=(M * C, d, C), v_stride=(M * C, d, C), o_stride=tok)
    _, y1, st1 = llsa.norm_forward(n1, par["x"], gain=par["gain"], scale=par["scale"], shift=par["shift"])
    qp, kp, vv = (heads(y1 @ par[n]).contiguous() for n in ("wq", "wk", "wv"))
    Q, K, ws = llsa.qknorm_rope_pool(layer, qp, kp, vv, par["gq"], par["gk"], cos, sin, 1e-6, layer.alloc_workspace(True))
    O, LSE, idx = llsa.forward_pooled(layer, Q, K, vv, ws)
    branch = flat(O).contiguous()
    xo, yo, st2 = llsa.norm_forward(n1, par["x"], branch, par["gain_b"], par["gate"], par["gain2"])
    qx = heads(yo @ par["wc"])
    kc, vc = par["kc"].transpose(1, 2), par["vc"].transpose(1, 2)
    Oc, LSEc = llsa.dense_forward(cross, qx, kc, vc, None, lens)
    got_out = xo + flat(Oc)
    # and back
    got = {}
    dOc = heads(go)
    dqx, dkc, dvc = llsa.dense_backward(cross, qx, kc, vc, Oc, LSEc, dOc, None, lens)
    got["kc"], got["vc"] = dkc.transpose(1, 2), dvc.transpose(1, 2)
    got["wc"] = yo.reshape(-1, C).T @ flat(dqx).reshape(-1, C)
    dyo = (flat(dqx) @ par["wc"].T).contiguous()
    b2 = llsa.norm_backward(n1, xo, dyo, st2, branch, par["gain_b"], par["gate"], par["gain2"], dx_out=go)
    got["gain_b"], got["gate"], got["gain2"] = b2["dgain_branch"], b2["dgate"], b2["dgain"]
    dO = heads(b2["dbranch"]).contiguous()
    dQ, dK, dV = llsa.backward(layer, Q, K, vv, O, LSE, idx, dO, ws)
    dq, dk, got["gq"], got["gk"] = llsa.qknorm_rope_backward(layer, qp, kp, par["gq"], par["gk"], cos, sin, dQ, dK)
    dy1 = torch.zeros(B, N, C, device="cuda")
    for n, g in (("wq", dq), ("wk", dk), ("wv", dV)):
        got[n] = y1.reshape(-1, C).T @ flat(g).reshape(-1, C)
        dy1 += flat(g) @ par[n].T
    b1 = llsa.norm_backward(n1, par["x"], dy1, st1, gain=par["gain"], scale=par["scale"], shift=par["shift"], dx_out=b2["dx"])
    got["x"], got["gain"], got["scale"], got["shift"] = b1["dx"], b1["dgain"], b1["dscale"], b1["dshift"]
    out = out.detach()
    assert float((got_out.double() - out).abs().max()) <= 1e-4 * float(out.abs().max())
    assert set(got) == set(par)
    for n in par:
        want = D[n].grad
        assert float((got[n].double() - want).abs().max()) <= 1e-4 * float(want.abs().max()), n
