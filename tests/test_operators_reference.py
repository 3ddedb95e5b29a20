"""The 64-bit forms that the operators' GPU tests compare with, held against differences and automatic differentiation (CPU)."""
import math

import pytest
import torch

from tests import operators_reference as R

F64 = torch.float64


def _difference(f, x, grad, n=6, h=1e-6):
    """Central differences of the scalar f along n coordinates of x against grad."""
    g = torch.Generator().manual_seed(1)
    for at in torch.randint(0, x.numel(), (n,), generator=g).tolist():
        flat = x.reshape(-1)
        keep = flat[at].item()
        flat[at] = keep + h
        up = f().item()
        flat[at] = keep - h
        down = f().item()
        flat[at] = keep
        want = (up - down) / (2 * h)
        assert abs(want - grad.reshape(-1)[at].item()) <= 1e-6 * max(1.0, abs(want)), at


@pytest.mark.parametrize("causal,lens", [(False, False), (True, False), (True, True)])
def test_dense_gradients_are_differences(causal, lens):
    g = torch.Generator().manual_seed(0)
    r = lambda *s: torch.randn(*s, generator=g, dtype=F64)
    Q, K, V, dO = r(2, 4, 7, 16), r(2, 2, 9, 16), r(2, 2, 9, 16), r(2, 4, 7, 16)
    ql, kl = (torch.tensor([7, 4]), torch.tensor([5, 3])) if lens else (None, None)
    call = lambda grad=None: R.dense(Q, K, V, grad, causal, ql, kl, bounds=False)[0]
    out = call(dO)
    f = lambda: (call()["O"] * dO).sum()
    for t, n in ((Q, "dQ"), (K, "dK"), (V, "dV")):
        _difference(f, t, out[n])
    if lens:                                          # the second sequence: query 0 of 4 sees none of 3 keys, query 1 the first
        assert (out["LSE"][1, :, 0] == -math.inf).all() and not out["O"][1, :, 0].any() and not out["dQ"][1, :, 0].any()
        assert not out["dK"][1, :, 3:].any() and not out["O"][1, :, 4:].any()


def test_dense_reference_lets_nothing_masked_through():
    g = torch.Generator().manual_seed(2)
    r = lambda *s: torch.randn(*s, generator=g, dtype=F64)
    Q, K, V, dO = r(1, 2, 6, 16), r(1, 1, 6, 16), r(1, 1, 6, 16), r(1, 2, 6, 16)
    fine = R.dense(Q, K, V, dO, True, bounds=False)[0]
    V[0, 0, 5, 3], K[0, 0, 5, 1] = math.nan, math.inf
    Q2 = Q.clone()
    Q2[0, :, 5] = math.nan
    bad = R.dense(Q2, K, V, dO, True, bounds=False)[0]
    assert torch.equal(fine["O"][:, :, :5], bad["O"][:, :, :5]) and torch.equal(fine["dQ"][:, :, :5], bad["dQ"][:, :, :5])


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("post,shared", [(True, False), (False, True)])
def test_norm_gradients_are_the_graph_s(layer, post, shared):
    g = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g, dtype=F64, requires_grad=True)
    B, N, C, m = 3, 5, 13, 1 if shared else 3
    t = dict(x=r(B, N, C), branch=r(B, N, C), gain_branch=r(C) if post else None, gate=r(m, C), gain=r(C), scale=r(m, C), shift=r(m, C))
    x_out, y = R.norm_forward(**t, layer=layer, alpha=0.7)
    dy, dx_out = torch.randn(B, N, C, dtype=F64, generator=g), torch.randn(B, N, C, dtype=F64, generator=g)
    ((y * dy).sum() + (x_out * dx_out).sum()).backward()
    with torch.no_grad():
        got, _ = R.norm_backward(x_out, dy, *(t[n] for n in ("branch", "gain_branch", "gate", "gain", "scale")), dx_out, layer, 1e-6, 0.7, shared)
    assert torch.allclose(got["dx"], t["x"].grad, rtol=1e-10, atol=1e-12)
    for n in ("branch", "gain_branch", "gate", "gain", "scale", "shift"):
        if t[n] is not None:
            assert torch.allclose(got["d" + n], t[n].grad, rtol=1e-10, atol=1e-12), n


def test_glue_gradient_is_the_graph_s():
    from paper_2512_16615_amd import inputs
    g = torch.Generator().manual_seed(4)
    x = torch.randn(2, 3, 16, 8, generator=g, dtype=F64, requires_grad=True)
    gamma = torch.randn(8, generator=g, dtype=F64, requires_grad=True)
    cos, sin = (torch.from_numpy(t).double() for t in inputs.rope_tables(16, 8))
    go = torch.randn(2, 3, 16, 8, generator=g, dtype=F64)
    (R.glue(x, gamma, cos, sin) * go).sum().backward()
    dx, dgamma, _ = R.glue_backward(x.detach(), gamma.detach(), cos, sin, go)
    assert torch.allclose(dx, x.grad, rtol=1e-10, atol=1e-12) and torch.allclose(dgamma, gamma.grad, rtol=1e-10, atol=1e-12)
