"""What dense attention, the norms between two blocks and the glue's gradient refuse, on the host, before anything is enqueued."""
import ctypes
import re

import pytest
import torch

from tests.test_abi_host import ROOT, llsa  # noqa: F401

import os

A = ctypes.c_void_p(4096)                       # never dereferenced: every call below is refused
ODD = ctypes.c_void_p(4100)


def _fields(name):
    text = open(os.path.join(ROOT, "include", "llsa.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    body = re.search(r"typedef struct \{([^{}]*)\} " + name + ";", text).group(1)
    return [re.sub(r"\[.*", "", n.strip()) for decl in body.split(";") if decl.strip() for n in decl.strip().split(None, 1)[1].split(",")]


def test_layouts_match_the_header(llsa):  # noqa: F811
    assert _fields("llsa_dense_desc") == [f[0] for f in llsa._DenseDesc._fields_]
    assert _fields("llsa_norm_desc") == [f[0] for f in llsa._NormDesc._fields_]


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), 2), (dict(heads=0), 2), (dict(Nq=0), 2), (dict(Nkv=0), 2), (dict(kv_heads=3), 2), (dict(kv_heads=0), 2),
    (dict(d=48), 3), (dict(d=256), 3), (dict(dtype=5), 3), (dict(causal=2), 3), (dict(kernel_path=2), 3), (dict(sm_scale=float("inf")), 3),
    (dict(Nq=(1 << 30) + 1), 3), (dict(batch=70000, heads=1), 3),
    (dict(q_stride=(0, 0, 65)), 2),             # rows that are no multiple of 16 bytes apart
    (dict(k_stride=(-64, 64, 64)), 2),
    (dict(o_stride=(0, 64, 512)), 2),           # batch entries of O on top of each other
    (dict(o_stride=(1 << 20, 64, 256)), 2),     # heads 4 .. 7 of a token are heads 0 .. 3 of the next
    (dict(batch=1, heads=60000, Nq=1 << 20), 3),                             # more tiles than a launch takes
    (dict(batch=2, heads=8, Nq=1 << 27), 3), (dict(batch=1, heads=1, Nkv=1 << 26, kernel_path=1), 3),
    (dict(batch=1, heads=64, kv_heads=1, Nq=1 << 25), 3),
    (dict(k_stride=(1 << 33, 1 << 32, 1 << 23)), 3),                         # 256 tokens 4 GiB apart
    (dict(q_stride=(1 << 34, 1 << 31, 64), kv_heads=4), 3),                  # two heads of a key head 4 GiB apart
])
def test_dense_plan_refuses(llsa, kw, status):  # noqa: F811
    args = dict(batch=2, heads=8, Nq=128, Nkv=128, d=64)
    args.update(kw)
    with pytest.raises(llsa.LlsaError) as e:
        llsa.DensePlan(**args)
    assert f"status {status}" in str(e.value)


def test_dense_plan_takes_layouts_of_projections(llsa):  # noqa: F811
    s = (128 * 3 * 8 * 64, 64, 3 * 8 * 64)      # a piece of a projection to queries, keys and values
    llsa.DensePlan(2, 8, 128, 128, 64, q_stride=s, k_stride=s, v_stride=s, o_stride=(128 * 8 * 64, 64, 8 * 64))
    llsa.DensePlan(2, 8, 128, 128, 64, k_stride=(0, 0, 64), v_stride=(0, 0, 64))
    llsa.DensePlan(2, 8, 128, 128, 64, k_stride=(1 << 33, 1 << 32, 1 << 23), kernel_path=1)
    llsa.DensePlan(2, 8, 128, 128, 64, q_stride=(1 << 34, 1 << 31, 64))     # heads with keys of their own are any distance apart
    llsa.DensePlan(1, 1, 1, 1, 16, q_stride=(3, 5, 7))                      # strides that nobody takes a step with


def test_dense_calls_refuse(llsa):  # noqa: F811
    lib = llsa.load()
    p = llsa.DensePlan(2, 8, 128, 128, 64)
    w = ctypes.c_void_p(1 << 20)
    f, b = lib.llsa_dense_forward, lib.llsa_dense_backward
    assert f(None, A, A, A, None, None, A, A, w, None) == 1
    for i in (0, 1, 2, 5, 6):
        args = [A, A, A, None, None, A, A, w, None]
        args[i] = None
        assert f(p._h, *args) == 1
        args[i] = ODD
        assert f(p._h, *args) == 2
    assert f(p._h, A, A, A, ctypes.c_void_p(4098), None, A, A, w, None) == 2
    assert f(p._h, A, A, A, None, None, A, A, ctypes.c_void_p(4096 + 16), None) == 2
    for i in (0, 1, 2, 5, 6, 7, 8, 9, 10, 11):
        args = [A, A, A, None, None, A, A, A, A, A, A, w, None]
        args[i] = None
        assert b(p._h, *args) == 1
    assert b(p._h, A, A, A, None, None, A, A, A, A, ODD, A, w, None) == 2
    shared = llsa.DensePlan(2, 8, 128, 128, 64, k_stride=(0, 0, 64), v_stride=(0, 0, 64))
    assert b(shared._h, A, A, A, None, None, A, A, A, A, A, A, w, None) == 2     # the gradients of broadcast keys would overlap
    with pytest.raises(llsa.LlsaError):
        shared.empty("k", "cpu")
    assert lib.llsa_dense_plan(None, None) == 1
    lib.llsa_dense_plan_destroy(None)
    assert lib.llsa_dense_workspace_bytes(None, 0) == 0


def test_dense_binding_refuses_tensors(llsa):  # noqa: F811
    p = llsa.DensePlan(1, 2, 8, 8, 16)
    t = torch.zeros(1, 2, 8, 16, dtype=torch.bfloat16)
    for bad in (t, t.float(), t[:, :, :4], t.transpose(1, 2)):               # on the host; another type, shape, layout
        with pytest.raises(llsa.LlsaError):
            llsa.dense_forward(p, bad, t, t)


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), 2), (dict(N=0), 2), (dict(C=0), 2), (dict(eps=-1.0), 2), (dict(eps=float("nan")), 2), (dict(mod_stride=63), 2), (dict(mod_stride=-1), 2),
    (dict(C=8193), 3), (dict(dtype=2), 3), (dict(mod_dtype=7), 3), (dict(kind=2), 3), (dict(batch=70000), 3),
])
def test_norm_plan_refuses(llsa, kw, status):  # noqa: F811
    args = dict(batch=2, N=8, C=64)
    args.update(kw)
    with pytest.raises(llsa.LlsaError) as e:
        llsa.NormPlan(**args)
    assert f"status {status}" in str(e.value)


def test_norm_calls_refuse(llsa):  # noqa: F811
    lib, n = llsa.load(), None
    p = llsa.NormPlan(2, 8, 64)
    f, b = lib.llsa_norm_forward, lib.llsa_norm_backward
    #          x  branch gb gate gain scale shift x_out y stats
    assert f(p._h, n, n, n, n, n, n, n, n, A, n, n) == 1
    assert f(p._h, A, A, n, n, n, n, n, n, A, n, n) == 1                     # a branch and nowhere to put x'
    assert f(p._h, A, n, A, n, n, n, n, n, A, n, n) == 1                     # the gain of a branch that is not there
    assert f(p._h, A, n, n, A, n, n, n, n, A, n, n) == 1
    assert f(p._h, A, A, n, n, A, n, n, A, n, n, n) == 1                     # the gain of a norm that is not taken
    assert f(p._h, A, n, n, n, n, n, n, n, n, n, n) == 1                     # nothing to do
    assert f(p._h, ODD, n, n, n, n, n, n, n, A, n, n) == 2
    assert f(p._h, A, n, n, n, ctypes.c_void_p(4098), n, n, n, A, n, n) == 2
    #          x' branch gb gate gain scale stats dy dx_out dx db dgb dgate dgain dscale dshift ws
    ok = [A, A, A, A, A, A, A, A, A, A, A, A, A, A, A, A, A, n]
    for i in (0, 6, 9, 10, 16):
        args = list(ok)
        args[i] = n
        assert b(p._h, *args) == 1, i
    args = list(ok)
    args[1] = n
    assert b(p._h, *args) == 1
    assert b(p._h, A, n, n, n, n, n, A, n, n, A, n, n, n, n, n, n, A, n) == 1       # neither dy nor dx_out
    assert b(p._h, A, n, n, n, n, n, A, n, A, A, n, n, n, A, n, n, A, n) == 1       # dgain without dy
    assert b(p._h, A, A, n, n, n, n, A, A, n, A, A, A, n, n, n, n, A, n) == 1       # dgain_branch without the norm behind the block
    args = list(ok)
    args[9] = ODD
    assert b(p._h, *args) == 2
    args = list(ok)
    args[16] = ctypes.c_void_p(4096 + 64)
    assert b(p._h, *args) == 2
    assert lib.llsa_norm_plan(None, None) == 1
    lib.llsa_norm_plan_destroy(None)
    assert lib.llsa_norm_workspace_bytes(None) == 0


def test_glue_backward_refuses(llsa):  # noqa: F811
    lib = llsa.load()
    p = llsa.Plan(1, 2, 64, 16, 4, 2, 1)
    f = lib.llsa_qknorm_rope_backward
    ok = [A, A, A, A, A, A, ctypes.c_float(1e-6), A, A, A, A, A, A, A, None]
    for i in (0, 1, 2, 3, 4, 5, 7, 8, 9, 10, 11, 12, 13):
        args = list(ok)
        args[i] = None
        assert f(p._h, *args) == 1, i
    for i in (0, 1, 4, 5, 7, 8, 9, 10):
        args = list(ok)
        args[i] = ODD
        assert f(p._h, *args) == 2, i
    args = list(ok)
    args[6] = ctypes.c_float(-1.0)
    assert f(p._h, *args) == 2
    args = list(ok)
    args[13] = ctypes.c_void_p(4096 + 16)
    assert f(p._h, *args) == 2
    assert lib.llsa_qknorm_rope_backward_bytes(None) == 0 and lib.llsa_qknorm_rope_backward_bytes(p._h) % 256 == 0
