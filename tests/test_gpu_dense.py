"""Dense attention, forward and backward, against 64 bits (tests/operators_reference.py holds the forms and derives the bounds)."""
import math

import pytest
import torch

from paper_2512_16615_amd import llsa
from tests import operators_reference as R

pytestmark = pytest.mark.gpu


def _case(dtype, batch, heads, kv_heads, Nq, Nkv, d, causal=False, lens=None, layout="heads", sm_scale=0.0, path=0):
    return dict(dtype=dtype, batch=batch, heads=heads, kv_heads=kv_heads, Nq=Nq, Nkv=Nkv, d=d, causal=causal, lens=lens, layout=layout, sm_scale=sm_scale, path=path)


def _id(c):
    lens = "" if c["lens"] is None else "-" + ("q" if c["lens"][0] else "") + "kv" + "_".join(map(str, c["lens"][1] or c["lens"][0]))
    return (f"{c['dtype']}-{c['batch']}x{c['heads']}_{c['kv_heads']}-{c['Nq']}x{c['Nkv']}-d{c['d']}{'-causal' if c['causal'] else ''}{lens}-{c['layout']}"
            f"{'-rows' if c['path'] else ''}{'-scale' if c['sm_scale'] else ''}")


def _tensor(c, heads, N, gen, k=1.0):
    """[batch, heads, N, d] as a view: heads first, tokens first, or a piece of a wider projection (with what lies between poisoned)."""
    b, d = c["batch"], c["d"]
    x = k * torch.randn(b, heads, N, d, generator=gen)
    x = x.to(torch.bfloat16 if c["dtype"] == "bf16" else torch.float32).cuda()
    if c["layout"] == "tokens":
        return x.transpose(1, 2).contiguous().transpose(1, 2)
    if c["layout"] == "piece":
        wide = torch.full((b, N, heads + 1, d), math.nan, dtype=x.dtype, device="cuda")
        wide[:, :, :heads] = x.transpose(1, 2)
        return wide[:, :, :heads].transpose(1, 2)
    return x


def _inputs(c, seed=0, k=1.0):
    gen = torch.Generator().manual_seed(seed)
    Q, dO = (_tensor(c, c["heads"], c["Nq"], gen, s) for s in (k, 1.0))
    K, V = (_tensor(c, c["kv_heads"], c["Nkv"], gen, s) for s in (k, 1.0))
    lens = [None if c["lens"] is None or v is None else torch.tensor(v, dtype=torch.int32, device="cuda") for v in (c["lens"] or (None, None))]
    return Q, K, V, dO, *lens


def _plan(c, Q, K, V, O=None):
    st = lambda t: t.stride()[:3]
    return llsa.DensePlan(c["batch"], c["heads"], c["Nq"], c["Nkv"], c["d"], kv_heads=c["kv_heads"], causal=c["causal"], sm_scale=c["sm_scale"],
                          dtype=llsa.BF16 if c["dtype"] == "bf16" else llsa.F32, kernel_path=c["path"], q_stride=st(Q), k_stride=st(K), v_stride=st(V),
                          o_stride=st(Q if O is None else O))


def _poisoned(p, which):
    """A tensor of the plan's layout whose every element, also between the rows, is a NaN."""
    st, size = p._strides[which], p._q if which in "qo" else p._kv
    n = 1 + sum((a - 1) * s for a, s in zip(size, st))
    store = torch.full((n,), math.nan, dtype=p.torch_dtype, device="cuda")
    return store.as_strided(size, st), store


def _run(c, Q, K, V, dO, ql, kl, workspace=None):
    p = _plan(c, Q, K, V)
    O = _poisoned(p, "o")[0]
    LSE = torch.full((c["batch"], c["heads"], c["Nq"]), math.nan, device="cuda")
    ws = p.alloc_workspace(True) if workspace is None else workspace
    ws.fill_(0xff)
    llsa.dense_forward(p, Q, K, V, ql, kl, O, LSE, ws)
    ws.fill_(0xff)
    grads = {n: _poisoned(p, w) for n, w in (("dQ", "q"), ("dK", "k"), ("dV", "v"))}
    llsa.dense_backward(p, Q, K, V, O, LSE, dO, ql, kl, *(t for t, _ in grads.values()), ws)
    torch.cuda.synchronize()
    out = {"O": O, "LSE": LSE} | {n: t for n, (t, _) in grads.items()}
    for n, (t, store) in grads.items():              # what lies between the rows is left alone
        assert int((~torch.isnan(store)).sum()) == t.numel() - int(torch.isnan(t).sum()), n
    return out


def _check(c, got, Q, K, V, dO, ql, kl, names=("O", "LSE", "dQ", "dK", "dV")):
    want, tol = R.dense(Q, K, V, dO, c["causal"], ql, kl, c["sm_scale"] or None, torch.bfloat16 if c["dtype"] == "bf16" else torch.float32)
    worst = {}
    for n in names:
        g, w = got[n].double(), want[n]
        fine = torch.isfinite(w)
        assert torch.equal(fine, torch.isfinite(g)), f"{n}: other places are finite"
        assert torch.equal(g[~fine].isnan(), w[~fine].isnan()) and torch.equal(g[~fine].nan_to_num(0.0), w[~fine].nan_to_num(0.0)), f"{n}: values that are not finite"
        err = (g - w).abs()[fine]
        over = err / tol[n][fine]
        worst[n] = float(over.max()) if over.numel() else 0.0
        assert worst[n] <= 1.0, f"{n}: {worst[n]:.2f} of the bound; largest error {float(err.max()):.3e} of {float(w[fine].abs().max()):.3e}"
    print({n: round(v, 3) for n, v in worst.items()}, flush=True)


CASES = [
    # one token, one key; a few of each
    _case("bf16", 1, 1, 1, 1, 1, 64), _case("f32", 2, 2, 1, 1, 1, 16), _case("bf16", 1, 2, 2, 2, 3, 128), _case("f32", 1, 3, 1, 5, 2, 32),
    # around the tiles' sizes
    *[_case("bf16", 1, 2, 2, n, n, 64) for n in (31, 32, 33, 63, 64, 65, 127, 128, 129, 257)],
    *[_case("bf16", 1, 1, 1, n, m, 128) for n, m in ((33, 95), (64, 96), (129, 63), (255, 191), (300, 64))],
    *[_case("f32", 1, 2, 2, n, m, d) for n, m, d in ((31, 33, 128), (64, 64, 64), (65, 130, 64), (129, 31, 32), (40, 70, 16), (130, 97, 128))],
    *[_case("bf16", 2, 3, 3, 100, 77, d) for d in (16, 32)],
    # shared key heads: 2, 3, 8 and all
    _case("bf16", 2, 6, 3, 70, 90, 64), _case("bf16", 1, 6, 2, 50, 128, 128, causal=True), _case("bf16", 2, 8, 1, 33, 65, 64, causal=True), _case("f32", 1, 6, 2, 45, 67, 64, causal=True),
    _case("bf16", 1, 40, 1, 1, 100, 128),
    # causal: square, more keys than queries, more queries than keys (rows that see nothing)
    *[_case("bf16", 1, 2, 2, n, m, d, causal=True) for n, m, d in ((1, 1, 64), (64, 64, 64), (65, 65, 128), (200, 200, 64), (33, 200, 64), (200, 33, 64), (5, 300, 128), (300, 5, 32), (513, 513, 64))],
    *[_case("f32", 1, 2, 1, n, m, 64, causal=True) for n, m in ((70, 70), (20, 90), (90, 20))],
    # lengths: zeros, ones, whole, beyond the tensor, below 0
    _case("bf16", 4, 2, 2, 80, 100, 64, lens=(None, [100, 0, 1, 65])),
    _case("bf16", 4, 2, 1, 130, 130, 128, causal=True, lens=([130, 1, 0, 77], [130, 1, 0, 77])),
    _case("bf16", 5, 2, 1, 70, 90, 64, causal=True, lens=([70, 64, 3, 70, 500], [90, 10, 90, 0, -4])),
    _case("f32", 3, 2, 1, 40, 60, 32, causal=True, lens=([40, 40, 7], [60, 20, 33])),
    _case("bf16", 3, 4, 4, 100, 100, 64, lens=([100, 40, 0], None)),
    # layouts
    *[_case("bf16", 2, 4, 2, 75, 75, 64, causal=True, layout=s) for s in ("tokens", "piece")],
    *[_case("f32", 2, 4, 2, 45, 45, 32, lens=(None, [45, 20]), layout=s) for s in ("tokens", "piece")],
    # long axes with few of the other: split and joined
    _case("bf16", 1, 2, 1, 1, 5001, 128), _case("bf16", 2, 4, 1, 3, 4100, 64, lens=(None, [4100, 129])), _case("bf16", 1, 2, 2, 4100, 3, 64), _case("bf16", 1, 1, 1, 3000, 70, 128, causal=True),
    _case("f32", 1, 2, 1, 2, 3001, 64), _case("f32", 1, 1, 1, 3001, 2, 64), _case("bf16", 1, 8, 2, 16, 2000, 64, causal=True),
    # middling
    _case("bf16", 1, 4, 4, 1024, 1024, 64), _case("bf16", 1, 4, 2, 1000, 1100, 128, causal=True), _case("f32", 1, 2, 2, 512, 512, 64), _case("bf16", 1, 2, 2, 700, 700, 32), _case("bf16", 1, 2, 2, 600, 600, 16, causal=True),
    # a sharp softmax: scores of tens
    _case("bf16", 1, 2, 2, 150, 150, 64, sm_scale=1.0), _case("f32", 1, 2, 2, 100, 100, 64, sm_scale=1.0),
    # many tiles: eight waves a tile (128 to 256 tiles of 128 rows and eight steps, causal to 512 from 32 steps), four waves a tile otherwise
    *[_case("bf16", 4, 16, 16, 390, 500, d, causal=c) for d in (16, 32, 64, 128) for c in (False, True)], *[_case("f32", 4, 16, 16, 390, 500, d, causal=True) for d in (16, 32, 64)],
    *[_case("bf16", 4, 28, 14, 257, 500, d, causal=True, lens=([257, 100, 3, 0], [500, 100, 500, 20]), layout="tokens") for d in (64, 128)], _case("bf16", 2, 10, 10, 2050, 2080, 64, causal=True),
    *[_case("bf16", 4, 16, 16, 200, 200, d, causal=c) for d in (16, 32, 64, 128) for c in (False, True)], *[_case("f32", 4, 16, 16, 200, 200, d, causal=True) for d in (16, 32, 64, 128)],
    *[_case("bf16", 10, 13, 13, 270, 300, d) for d in (16, 32, 64, 128)], *[_case("bf16", 12, 16, 16, 290, 270, d, causal=True) for d in (32, 64, 128)],
    *[_case("f32", 10, 13, 13, 140, 300, d) for d in (16, 32, 64, 128)], _case("bf16", 6, 48, 12, 150, 129, 128, causal=True, layout="tokens"), _case("bf16", 6, 48, 12, 150, 129, 64, layout="piece"),
    _case("bf16", 12, 32, 16, 140, 260, 64, causal=True, lens=([140, 3, 0, 77, 128, 129, 140, 1, 64, 65, 100, 139], [260, 3, 5, 0, 256, 257, 70, 260, 64, 33, 100, 1])),
    # and their other axis cut
    _case("bf16", 2, 15, 15, 200, 4200, 128), _case("bf16", 2, 15, 15, 4200, 200, 64), _case("bf16", 2, 30, 15, 100, 6400, 64, causal=True), _case("f32", 2, 15, 15, 200, 4100, 128), _case("f32", 2, 15, 15, 4100, 200, 128),
    # causal sequences of different lengths, their tiles sorted by work (768 workgroups and more, up to 8 sequences)
    _case("bf16", 8, 12, 12, 1000, 1000, 64, causal=True, lens=([1000, 0, 130, 700, 1, 999, 128, 300], [1000, 50, 0, 800, 1, 999, 130, 256])),
    _case("bf16", 5, 40, 20, 600, 513, 128, causal=True, lens=([513, 600, 3, 256, 0], [513, 513, 3, 200, 9])), _case("f32", 3, 44, 44, 700, 700, 32, causal=True, lens=([700, 65, 300], None)),
    _case("bf16", 2, 60, 60, 150, 900, 32, causal=True, lens=(None, [900, 140])), _case("bf16", 9, 40, 40, 270, 270, 16, causal=True, lens=([270, 1, 0, 5, 128, 129, 200, 270, 64],) * 2),
    # few rows and many keys: the row tiles narrow, the key tiles not
    *[_case("bf16", 1, 4, 4, 1, 5000, d) for d in (32, 64, 128)], _case("bf16", 1, 16, 16, 20, 1100, 64, causal=True), _case("bf16", 10, 16, 16, 33, 130, 128), _case("f32", 1, 16, 16, 20, 1100, 16, causal=True),
    _case("bf16", 8, 32, 32, 30, 300, 64, lens=([30, 1, 0, 15, 30, 30, 29, 2], [300, 300, 300, 0, 129, 128, 1, 64])),
    # the kernels of one wave a row
    _case("bf16", 2, 4, 2, 40, 50, 64, causal=True, lens=([40, 17], [50, 9]), path=1), _case("f32", 1, 2, 1, 33, 20, 128, path=1), _case("bf16", 1, 2, 1, 20, 33, 16, causal=True, path=1),
]


@pytest.mark.parametrize("c", CASES, ids=_id)
def test_dense_against_64_bits(c):
    x = _inputs(c)
    _check(c, _run(c, *x), *x)


MASKED = [("bf16", 64, math.nan, 2, 2, 100, 0), ("bf16", 128, math.inf, 2, 2, 100, 0), ("f32", 32, -math.inf, 2, 2, 100, 0), ("bf16", 16, math.nan, 2, 2, 100, 0),
          ("bf16", 64, math.nan, 2, 2, 100, 1), ("f32", 128, math.inf, 2, 2, 100, 1), ("bf16", 128, math.nan, 2, 16, 520, 0), ("bf16", 64, math.inf, 2, 64, 520, 0), ("bf16", 64, math.nan, 2, 14, 500, 0), ("bf16", 128, math.inf, 2, 14, 500, 0), ("f32", 128, math.nan, 2, 16, 520, 0),
          ("bf16", 64, math.nan, 2, 1, 1800, 0), ("bf16", 128, math.inf, 2, 1, 1800, 0)]


@pytest.mark.parametrize("dtype,d,bad,batch,kv_heads,N,path", MASKED, ids=str)
def test_nothing_behind_a_mask_is_seen(dtype, d, bad, batch, kv_heads, N, path):
    """Infinities and NaN behind the lengths and in keys and queries that a causal mask hides: what is not masked is as if they were zeros.  One tile a
    group, many, and few with the other axis cut."""
    short = N * 2 // 5
    c = _case(dtype, batch, 2 * kv_heads, kv_heads, N, N, d, causal=True, lens=([N, short], [N, short]), path=path)
    Q, K, V, dO, ql, kl = _inputs(c)
    clean = [t.clone() for t in (Q, K, V, dO)]
    for t in (Q, K, V, dO):
        t[1, :, short:] = bad                       # behind the lengths
    K[0, 0, 71], V[0, 0, 71, 3] = bad, bad         # seen by queries 71 and on
    got = _run(c, Q, K, V, dO, ql, kl)
    want = _run(c, *clean, ql, kl)
    near = lambda g, w: torch.isfinite(g).all() and float((g - w).abs().max()) <= 2.0 ** -6 * float(w.abs().max())      # another kernel's rounding: a few of P's and the result's half steps
    for n in ("O", "LSE", "dQ"):
        assert torch.equal(got[n][1], want[n][1]) and torch.equal(got[n][0, 2:], want[n][0, 2:]), n
        assert near(got[n][0, :2, :71].double(), want[n][0, :2, :71].double()), n
    for n in ("dK", "dV"):
        assert torch.equal(got[n][1], want[n][1]) and torch.equal(got[n][0, 1:], want[n][0, 1:]), n
    # a query and its gradient that hold a NaN: keys behind it do not see it
    Q, K, V, dO = clean
    Q[0, 1, 20, 1], dO[0, 1, 30, 2] = bad, bad
    got2 = _run(c, Q, K, V, dO, ql, kl)
    keep = [i for i in range(N) if i != 20]
    others = [h for h in range(2 * kv_heads) if h != 1]
    assert torch.isfinite(got2["O"][0, 1, keep].float()).all() and torch.equal(got2["O"][0, others], want["O"][0, others])
    for n in ("dK", "dV"):
        assert near(got2[n][0, 0, 31:].double(), want[n][0, 0, 31:].double()), n


@pytest.mark.parametrize("dtype,d,heads,N", [("bf16", 64, 2, 130), ("f32", 64, 2, 130), ("bf16", 128, 64, 200), ("bf16", 64, 64, 600), ("bf16", 32, 1, 3000)], ids=str)
def test_nothing_behind_the_lengths_is_seen_without_a_causal_mask(dtype, d, heads, N):
    c = _case(dtype, 2, heads, heads, N, N, d, lens=([N, N // 3], [N - 1, N // 3 + 1]))
    Q, K, V, dO, ql, kl = _inputs(c)
    want = _run(c, Q.clone(), K.clone(), V.clone(), dO.clone(), ql, kl)
    for b in range(2):
        for t, n in ((Q, ql), (K, kl), (V, kl), (dO, ql)):
            t[b, :, int(n[b]):] = math.nan
    got = _run(c, Q, K, V, dO, ql, kl)
    for n in want:
        assert torch.equal(got[n], want[n]), n


def test_two_problems_at_once_on_two_streams():
    """A plan, a workspace and a stream each, enqueued in turn and waited for once."""
    jobs = []
    for c in (_case("bf16", 2, 8, 4, 500, 900, 64, causal=True), _case("bf16", 1, 4, 4, 1, 5000, 128)):
        x = _inputs(c)
        p = _plan(c, *x[:3])
        want = _run(c, *x)
        jobs.append((p, x, p.alloc_workspace(True), torch.cuda.Stream(), want, []))
    torch.cuda.synchronize()
    for _ in range(5):
        for p, (Q, K, V, dO, _, _), ws, stream, _, out in jobs:
            with torch.cuda.stream(stream):
                O, LSE = llsa.dense_forward(p, Q, K, V, workspace=ws)
                out.append((O, LSE, *llsa.dense_backward(p, Q, K, V, O, LSE, dO, workspace=ws)))
    torch.cuda.synchronize()
    for *_, want, out in jobs:
        for o in out:
            assert all(torch.equal(a, want[n]) for a, n in zip(o, ("O", "LSE", "dQ", "dK", "dV")))


def test_dense_is_the_same_bits_from_call_to_call_and_stream_to_stream():
    c = _case("bf16", 2, 4, 2, 300, 700, 64, causal=True)
    x = _inputs(c)
    first = _run(c, *x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = _run(c, *x)
    for n in first:
        assert torch.equal(first[n], second[n]), n


@pytest.mark.parametrize("c", [_case("bf16", 2, 4, 2, 200, 200, 64, causal=True), _case("bf16", 1, 2, 1, 1, 3000, 128), _case("f32", 1, 2, 2, 60, 60, 32)], ids=_id)
def test_dense_replays_from_a_graph(c):
    """A step captured into a graph, replayed with the program's own work on the same workspace between the replays; then with other inputs and
    other lengths in the same buffers."""
    Q, K, V, dO, _, _ = _inputs(c)
    kl = torch.full((c["batch"],), c["Nkv"], dtype=torch.int32, device="cuda")
    p = _plan(c, Q, K, V)
    ws, O, LSE = p.alloc_workspace(True), p.empty("o"), torch.empty(c["batch"], c["heads"], c["Nq"], device="cuda")
    grads = [p.empty(w) for w in "qkv"]

    def step():
        llsa.dense_forward(p, Q, K, V, None, kl, O, LSE, ws)
        llsa.dense_backward(p, Q, K, V, O, LSE, dO, None, kl, *grads, ws)

    step()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for rep in range(4):
        new = _inputs(c, seed=rep)
        for t, n in zip((Q, K, V, dO), new):
            t.copy_(n)
        kl.fill_(max(1, c["Nkv"] - 37 * rep))
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (O, LSE, *grads)]
        ws.fill_(0xff)
        for t in (O, LSE, *grads):
            t.fill_(math.nan)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for t, w in zip((O, LSE, *grads), want):
            assert torch.equal(t, w), rep


def test_dense_reads_broadcast_keys_and_offsets_beyond_32_bits():
    """Keys and values 2 MB apart, the last of them more than 4 GB behind the first, and one set of keys for all batch entries (a stride of 0)."""
    gen = torch.Generator().manual_seed(5)
    n, step = 2200, 1 << 20
    store = torch.zeros(n * step, dtype=torch.bfloat16, device="cuda")
    at = lambda off: store.as_strided((2, 1, n, 64), (0, 0, step, 1), off)
    K, V = at(0), at(64)
    kv = [torch.randn(1, 1, n, 64, generator=gen).to(torch.bfloat16).cuda() for _ in range(2)]
    for t, s in ((K, kv[0]), (V, kv[1])):
        t[0, 0].copy_(s[0, 0])
    for Nq, causal in ((3, False), (150, True)):
        Q = torch.randn(2, 2, Nq, 64, generator=gen).to(torch.bfloat16).cuda()
        p = llsa.DensePlan(2, 2, Nq, n, 64, kv_heads=1, causal=causal, k_stride=(0, 0, step), v_stride=(0, 0, step))
        O, LSE = llsa.dense_forward(p, Q, K, V)
        want, tol = R.dense(Q, kv[0].expand(2, 1, n, 64), kv[1].expand(2, 1, n, 64), None, causal, dtype=torch.bfloat16)
        assert bool(((O.double() - want["O"]).abs() <= tol["O"]).all()) and bool(((LSE.double() - want["LSE"]).abs() <= tol["LSE"]).all())
    del store, K, V


@pytest.mark.parametrize("heads,kv_heads,causal,d", [(16, 16, False, 64), (8, 4, True, 128), (1, 1, False, 32)], ids=str)
def test_dense_step_on_tensors_beyond_32_bits(heads, kv_heads, causal, d):
    """Everything 2 MB from token to token, read and written more than 4 GB behind its first element: the same bits as contiguous."""
    n, step = 2200, 1 << 20
    c = _case("bf16", 1, heads, kv_heads, n, n, d, causal=causal)
    Q, K, V, dO, _, _ = _inputs(c)
    want = _run(c, Q, K, V, dO, None, None)
    stores = [torch.empty(n * step, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    far = lambda store, i, h: store.as_strided((1, h, n, d), (n * step, d, step, 1), i * heads * d)
    x = [far(stores[0], i, t.shape[1]) for i, t in enumerate((Q, K, V, dO))]
    for t, s in zip(x, (Q, K, V, dO)):
        t.copy_(s)
    p = _plan(c, *x[:3])
    O, dQ, dK, dV = (far(stores[1], i, h) for i, h in enumerate((heads, heads, kv_heads, kv_heads)))
    _, LSE = llsa.dense_forward(p, *x[:3], O=O)
    llsa.dense_backward(p, *x[:3], O, LSE, x[3], dQ=dQ, dK=dK, dV=dV)
    for t, w in ((O, "O"), (LSE, "LSE"), (dQ, "dQ"), (dK, "dK"), (dV, "dV")):
        assert torch.equal(t, want[w]), w
    del stores, x


def test_dense_binding_refuses_what_does_not_fit():
    c = _case("bf16", 2, 2, 2, 40, 40, 64)
    Q, K, V, dO, _, _ = _inputs(c)
    p = _plan(c, Q, K, V)
    lens = torch.tensor([40, 40], dtype=torch.int32, device="cuda")
    for args in ((Q.float(), K, V), (Q, K[:, :, :39], V), (Q, K.transpose(1, 2).contiguous().transpose(1, 2), V), (Q, K, V.cpu())):
        with pytest.raises(llsa.LlsaError):
            llsa.dense_forward(p, *args)
    for bad in (lens.long(), lens[:1], lens.cpu()):
        with pytest.raises(llsa.LlsaError):
            llsa.dense_forward(p, Q, K, V, bad)
    O, LSE = llsa.dense_forward(p, Q, K, V)
    with pytest.raises(llsa.LlsaError):
        llsa.dense_backward(p, Q, K, V, O, LSE, dO, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(llsa.LlsaError):
        llsa.dense_backward(p, Q, K, V, O, LSE.half(), dO)
