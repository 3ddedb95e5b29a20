"""Thin ctypes binding of ``libllsa.so`` (see ``include/llsa.h``).

Argument marshalling only: PyTorch owns the device memory and the stream, every
step of the path runs in the library's HIP kernels.  There is no fallback: if
the library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libllsa.so")
_lib = None

F32, BF16 = 0, 1
NORM_RMS, NORM_LAYER = 0, 1


class LlsaError(RuntimeError):
    pass


class _Desc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("heads", ctypes.c_int32), ("N", ctypes.c_int64), ("d", ctypes.c_int32),
                ("B", ctypes.c_int32), ("K", ctypes.c_int32), ("L", ctypes.c_int32), ("Le", ctypes.c_int32),
                ("sm_scale", ctypes.c_float), ("dtype", ctypes.c_int32), ("reweight", ctypes.c_int32),
                ("bwd_repool", ctypes.c_int32), ("kernel_path", ctypes.c_int32), ("single_stream", ctypes.c_int32)]


class _DenseDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("d", ctypes.c_int32),
                ("Nq", ctypes.c_int64), ("Nkv", ctypes.c_int64), ("sm_scale", ctypes.c_float), ("dtype", ctypes.c_int32),
                ("causal", ctypes.c_int32), ("kernel_path", ctypes.c_int32), ("q_stride", ctypes.c_int64 * 3),
                ("k_stride", ctypes.c_int64 * 3), ("v_stride", ctypes.c_int64 * 3), ("o_stride", ctypes.c_int64 * 3)]


class _NormDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("C", ctypes.c_int32), ("N", ctypes.c_int64), ("kind", ctypes.c_int32),
                ("eps", ctypes.c_float), ("residual_scale", ctypes.c_float), ("dtype", ctypes.c_int32),
                ("mod_dtype", ctypes.c_int32), ("mod_stride", ctypes.c_int64)]


EXPORTS = ["llsa_plan", "llsa_plan_destroy", "llsa_plan_workspace_bytes", "llsa_plan_indices_bytes",
           "llsa_plan_level_info", "llsa_plan_pyramid_info", "llsa_plan_csc_info", "llsa_forward", "llsa_backward",
           "llsa_pool", "llsa_select_level", "llsa_attention", "llsa_index_transpose", "llsa_reorder", "llsa_status_string",
           "llsa_stage_count", "llsa_stage_name", "llsa_stage_timing_begin", "llsa_stage_timing_end",
           "llsa_static_workspace_bytes", "llsa_forward_static", "llsa_qknorm_rope_pool", "llsa_forward_pooled",
           "llsa_kv_backward_mask_bytes", "llsa_kv_backward_level0", "llsa_calibrate_mfma", "llsa_calibrate_copy",
           "llsa_dense_plan", "llsa_dense_plan_destroy", "llsa_dense_workspace_bytes", "llsa_dense_forward", "llsa_dense_backward",
           "llsa_norm_plan", "llsa_norm_plan_destroy", "llsa_norm_workspace_bytes", "llsa_norm_forward", "llsa_norm_backward",
           "llsa_qknorm_rope_backward_bytes", "llsa_qknorm_rope_backward"]


def load():
    """Load the library built by ``paper_2512_16615_amd.build``; raises if it is not there."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise LlsaError(f"{LIB_PATH} not found: run `python -m paper_2512_16615_amd.build` (needs hipcc)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    lib.llsa_plan.argtypes = [ctypes.POINTER(_Desc), ctypes.POINTER(vp)]
    lib.llsa_plan.restype = ctypes.c_int
    lib.llsa_plan_destroy.argtypes = [vp]
    lib.llsa_plan_destroy.restype = None
    lib.llsa_plan_workspace_bytes.argtypes = [vp, ctypes.c_int]
    lib.llsa_plan_workspace_bytes.restype = sz
    lib.llsa_plan_indices_bytes.argtypes = [vp]
    lib.llsa_plan_indices_bytes.restype = sz
    lib.llsa_plan_level_info.argtypes = [vp, i32, ctypes.POINTER(i64), ctypes.POINTER(i32), ctypes.POINTER(sz)]
    lib.llsa_plan_level_info.restype = i32
    lib.llsa_plan_pyramid_info.argtypes = [vp, i32, i32, ctypes.POINTER(i64), ctypes.POINTER(sz)]
    lib.llsa_plan_pyramid_info.restype = i32
    lib.llsa_plan_csc_info.argtypes = [vp, i32, ctypes.POINTER(sz), ctypes.POINTER(sz)]
    lib.llsa_plan_csc_info.restype = i32
    lib.llsa_forward.argtypes = [vp] * 9
    lib.llsa_forward.restype = ctypes.c_int
    lib.llsa_forward_static.argtypes = [vp] * 8
    lib.llsa_forward_static.restype = ctypes.c_int
    lib.llsa_static_workspace_bytes.argtypes = []
    lib.llsa_static_workspace_bytes.restype = sz
    lib.llsa_forward_pooled.argtypes = [vp] * 9
    lib.llsa_forward_pooled.restype = ctypes.c_int
    lib.llsa_qknorm_rope_pool.argtypes = [vp] * 8 + [ctypes.c_float] + [vp] * 4
    lib.llsa_qknorm_rope_pool.restype = ctypes.c_int
    lib.llsa_kv_backward_mask_bytes.argtypes = [vp]
    lib.llsa_kv_backward_mask_bytes.restype = sz
    lib.llsa_kv_backward_level0.argtypes = [vp, i32] + [vp] * 11
    lib.llsa_kv_backward_level0.restype = ctypes.c_int
    lib.llsa_calibrate_mfma.argtypes = [vp, i32, i32, vp]
    lib.llsa_calibrate_mfma.restype = ctypes.c_int
    lib.llsa_calibrate_copy.argtypes = [vp, vp, i64, vp]
    lib.llsa_calibrate_copy.restype = ctypes.c_int
    lib.llsa_backward.argtypes = [vp] * 13
    lib.llsa_backward.restype = ctypes.c_int
    lib.llsa_pool.argtypes = [vp] * 6
    lib.llsa_pool.restype = ctypes.c_int
    lib.llsa_select_level.argtypes = [vp, i32, vp, vp, vp, vp]
    lib.llsa_select_level.restype = ctypes.c_int
    lib.llsa_attention.argtypes = [vp] * 9
    lib.llsa_attention.restype = ctypes.c_int
    lib.llsa_index_transpose.argtypes = [vp] * 4
    lib.llsa_index_transpose.restype = ctypes.c_int
    lib.llsa_reorder.argtypes = [i64, i64, i32, i32, i32, vp, vp, vp]
    lib.llsa_reorder.restype = ctypes.c_int
    lib.llsa_stage_count.argtypes = []
    lib.llsa_stage_count.restype = i32
    lib.llsa_stage_name.argtypes = [i32]
    lib.llsa_stage_name.restype = ctypes.c_char_p
    lib.llsa_stage_timing_begin.argtypes = [i32, i32]
    lib.llsa_stage_timing_begin.restype = ctypes.c_int
    lib.llsa_stage_timing_end.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(i32)]
    lib.llsa_stage_timing_end.restype = ctypes.c_int
    lib.llsa_dense_plan.argtypes = [ctypes.POINTER(_DenseDesc), ctypes.POINTER(vp)]
    lib.llsa_dense_plan.restype = ctypes.c_int
    lib.llsa_dense_plan_destroy.argtypes = [vp]
    lib.llsa_dense_plan_destroy.restype = None
    lib.llsa_dense_workspace_bytes.argtypes = [vp, ctypes.c_int]
    lib.llsa_dense_workspace_bytes.restype = sz
    lib.llsa_dense_forward.argtypes = [vp] * 10
    lib.llsa_dense_forward.restype = ctypes.c_int
    lib.llsa_dense_backward.argtypes = [vp] * 14
    lib.llsa_dense_backward.restype = ctypes.c_int
    lib.llsa_norm_plan.argtypes = [ctypes.POINTER(_NormDesc), ctypes.POINTER(vp)]
    lib.llsa_norm_plan.restype = ctypes.c_int
    lib.llsa_norm_plan_destroy.argtypes = [vp]
    lib.llsa_norm_plan_destroy.restype = None
    lib.llsa_norm_workspace_bytes.argtypes = [vp]
    lib.llsa_norm_workspace_bytes.restype = sz
    lib.llsa_norm_forward.argtypes = [vp] * 12
    lib.llsa_norm_forward.restype = ctypes.c_int
    lib.llsa_norm_backward.argtypes = [vp] * 19
    lib.llsa_norm_backward.restype = ctypes.c_int
    lib.llsa_qknorm_rope_backward_bytes.argtypes = [vp]
    lib.llsa_qknorm_rope_backward_bytes.restype = sz
    lib.llsa_qknorm_rope_backward.argtypes = [vp] * 7 + [ctypes.c_float] + [vp] * 8
    lib.llsa_qknorm_rope_backward.restype = ctypes.c_int
    lib.llsa_status_string.argtypes = [ctypes.c_int]
    lib.llsa_status_string.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _check(st: int, what: str):
    if st != 0:
        raise LlsaError(f"{what}: {load().llsa_status_string(st).decode()} (status {st})")


def _ptr(t: torch.Tensor | None):
    return None if t is None else t.data_ptr()


# The current device's current stream as a number.  torch.cuda.current_stream() builds an object around it, which takes 2.9 of the 5.8 us
# that a call of this binding spent outside the library (a training step of one head of 256 tokens, 7 launches: 38.0 -> 34.4 us).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    return torch.cuda.current_stream().cuda_stream if _raw_stream is None else _raw_stream(torch.cuda.current_device())


@dataclass
class LevelInfo:
    rows: int
    K_l: int
    byte_offset: int


class Plan:
    """``llsa_plan``: validated problem description, level table and buffer sizes (host only)."""

    def __init__(self, batch, heads, N, d, B, K, L, Le=None, sm_scale=0.0, dtype=BF16, reweight=1, bwd_repool=0,
                 kernel_path=0, single_stream=0):
        lib = load()
        self.desc = _Desc(batch, heads, N, d, B, K, L, L if Le is None else Le, sm_scale, dtype, reweight,
                          bwd_repool, kernel_path, single_stream)
        h = ctypes.c_void_p()
        st = lib.llsa_plan(ctypes.byref(self.desc), ctypes.byref(h))
        self._h = h if st == 0 else None
        _check(st, "llsa_plan")
        self.batch, self.heads, self.N, self.d, self.B, self.K, self.L = batch, heads, N, d, B, K, L
        self.Le = self.desc.Le
        self.torch_dtype = torch.float32 if dtype == F32 else torch.bfloat16
        self._shape = torch.Size((batch, heads, N, d))
        self._workspace_bytes = tuple(lib.llsa_plan_workspace_bytes(self._h, i) for i in (0, 1))
        self._indices_bytes = lib.llsa_plan_indices_bytes(self._h)
        self._glue_bytes = lib.llsa_qknorm_rope_backward_bytes(self._h)
        self.levels = [self.level_info(l) for l in range(L)]

    def __del__(self):
        if getattr(self, "_h", None) is not None and _lib is not None:
            _lib.llsa_plan_destroy(self._h)
            self._h = None

    def workspace_bytes(self, for_backward: bool) -> int:
        return self._workspace_bytes[bool(for_backward)]

    def indices_bytes(self) -> int:
        return self._indices_bytes

    def level_info(self, l: int) -> LevelInfo:
        rows, kl, off = ctypes.c_int64(), ctypes.c_int32(), ctypes.c_size_t()
        if load().llsa_plan_level_info(self._h, l, ctypes.byref(rows), ctypes.byref(kl), ctypes.byref(off)) < 0:
            raise LlsaError("llsa_plan_level_info: bad level")
        return LevelInfo(rows.value, kl.value, off.value)

    def pyramid_info(self, tensor: int, l: int):
        tok, off = ctypes.c_int64(), ctypes.c_size_t()
        if load().llsa_plan_pyramid_info(self._h, tensor, l, ctypes.byref(tok), ctypes.byref(off)) < 0:
            raise LlsaError("llsa_plan_pyramid_info: bad arguments")
        return tok.value, off.value

    def csc_info(self, l: int):
        c, iq = ctypes.c_size_t(), ctypes.c_size_t()
        if load().llsa_plan_csc_info(self._h, l, ctypes.byref(c), ctypes.byref(iq)) < 0:
            raise LlsaError("llsa_plan_csc_info: bad level")
        return c.value, iq.value

    # ---- buffers (torch allocates, the library only reads the pointers) ----
    def alloc_workspace(self, for_backward: bool, device="cuda") -> torch.Tensor:
        return torch.empty(max(self.workspace_bytes(for_backward), 256), dtype=torch.uint8, device=device)

    def alloc_indices(self, device="cuda") -> torch.Tensor:
        return torch.empty(self.indices_bytes() // 4, dtype=torch.int32, device=device)

    def alloc_glue_workspace(self, device="cuda") -> torch.Tensor:
        """Workspace of ``qknorm_rope_backward``."""
        return torch.empty(self._glue_bytes, dtype=torch.uint8, device=device)

    def level_indices(self, indices: torch.Tensor, l: int) -> torch.Tensor:
        """View of I^(l) inside ``indices``: ``[batch, heads, rows, K_l]``."""
        li = self.levels[l]
        n = self.batch * self.heads * li.rows * li.K_l
        return indices[li.byte_offset // 4: li.byte_offset // 4 + n].view(self.batch, self.heads, li.rows, li.K_l)

    def pyramid_level(self, workspace: torch.Tensor, tensor: int, l: int) -> torch.Tensor:
        """View of pooled level l (>= 1) of Q/K/V (tensor 0/1/2) inside ``workspace``."""
        tok, off = self.pyramid_info(tensor, l)
        nbytes = self.batch * self.heads * tok * self.d * self.torch_dtype.itemsize
        return workspace[off: off + nbytes].view(self.torch_dtype).view(self.batch, self.heads, tok, self.d)

    def csc_level(self, workspace: torch.Tensor, l: int):
        """(C [bh, rows+1], Iq [bh, rows*K_l]) views inside a backward workspace."""
        c_off, iq_off = self.csc_info(l)
        li, bh = self.levels[l], self.batch * self.heads
        C = workspace[c_off: c_off + bh * (li.rows + 1) * 4].view(torch.int32).view(bh, li.rows + 1)
        Iq = workspace[iq_off: iq_off + bh * li.rows * li.K_l * 4].view(torch.int32).view(bh, li.rows * li.K_l)
        return C, Iq


def _chk_tensor(p: Plan, t: torch.Tensor, name: str):
    if not t.is_cuda or not t.is_contiguous() or t.dtype != p.torch_dtype or t.shape != p._shape:
        raise LlsaError(f"{name}: expected a contiguous cuda {p.torch_dtype} tensor of shape "
                        f"{(p.batch, p.heads, p.N, p.d)}, got {t.dtype} {tuple(t.shape)} on {t.device}")


def forward(p: Plan, Q, K, V, O=None, LSE=None, indices=None, workspace=None):
    """``llsa_forward``: returns ``(O, LSE, indices, workspace)``."""
    for t, n in ((Q, "Q"), (K, "K"), (V, "V")):
        _chk_tensor(p, t, n)
    O = torch.empty_like(Q) if O is None else O
    LSE = torch.empty(p.batch, p.heads, p.N, dtype=torch.float32, device=Q.device) if LSE is None else LSE
    indices = p.alloc_indices(Q.device) if indices is None else indices
    workspace = p.alloc_workspace(False, Q.device) if workspace is None else workspace
    if workspace.numel() < p.workspace_bytes(False) or indices.numel() * 4 < p.indices_bytes():
        raise LlsaError("workspace or indices buffer too small")
    _check(load().llsa_forward(p._h, _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(LSE), _ptr(indices), _ptr(workspace),
                               _stream()), "llsa_forward")
    return O, LSE, indices, workspace


def qknorm_rope_pool(p: Plan, Qpre, Kpre, V, gamma_q, gamma_k, cos_table, sin_table, eps=1e-6, workspace=None):
    """``llsa_qknorm_rope_pool``: returns ``(Qout, Kout, workspace)`` (workspace holds every pooled level)."""
    for t, n in ((Qpre, "Qpre"), (Kpre, "Kpre"), (V, "V")):
        _chk_tensor(p, t, n)
    for t, shape, n in ((gamma_q, (p.d,), "gamma_q"), (gamma_k, (p.d,), "gamma_k"),
                        (cos_table, (p.N, p.d // 2), "cos_table"), (sin_table, (p.N, p.d // 2), "sin_table")):
        if not t.is_cuda or not t.is_contiguous() or t.dtype != torch.float32 or tuple(t.shape) != shape:
            raise LlsaError(f"{n}: expected a contiguous cuda float32 tensor of shape {shape}")
    Qout, Kout = torch.empty_like(Qpre), torch.empty_like(Kpre)
    workspace = p.alloc_workspace(False, Qpre.device) if workspace is None else workspace
    if workspace.numel() < p.workspace_bytes(False):
        raise LlsaError("workspace too small")
    _check(load().llsa_qknorm_rope_pool(p._h, _ptr(Qpre), _ptr(Kpre), _ptr(V), _ptr(gamma_q), _ptr(gamma_k),
                                        _ptr(cos_table), _ptr(sin_table), ctypes.c_float(eps), _ptr(Qout), _ptr(Kout),
                                        _ptr(workspace), _stream()), "llsa_qknorm_rope_pool")
    return Qout, Kout, workspace


_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _device() -> int:
    """The current device, on whose current stream the kernels run (torch.cuda.current_device() takes three times as long)."""
    try:
        return torch.cuda.current_device() if _raw_device is None else _raw_device()
    except RuntimeError as e:
        raise LlsaError(f"no current device: {e}") from None


def _chk_vec(t: torch.Tensor, name: str, dtype, shape, dev: int, rows_only=False):
    """A tensor of exactly this type and shape on device ``dev``; contiguous, or with contiguous rows."""
    if t.dtype is dtype and t.shape == shape and t.get_device() == dev and (t.is_contiguous() or rows_only and t.stride(-1) == 1):
        return
    raise LlsaError(f"{name}: expected a contiguous {dtype} tensor of shape {tuple(shape)} on device {dev}, got {t.dtype} {tuple(t.shape)} "
                    f"with strides {t.stride()} on {t.device}")


def _chk_ws(t: torch.Tensor | None, name: str, nbytes: int, dev: int):
    if t is not None and (t.get_device() != dev or not t.is_contiguous() or t.numel() * t.element_size() < nbytes):
        raise LlsaError(f"{name}: {nbytes} contiguous bytes on device {dev} are needed")


def qknorm_rope_backward(p: Plan, Qpre, Kpre, gamma_q, gamma_k, cos_table, sin_table, dQ, dK, eps=1e-6, dQpre=None, dKpre=None,
                         dgamma_q=None, dgamma_k=None, workspace=None):
    """``llsa_qknorm_rope_backward``: returns ``(dQpre, dKpre, dgamma_q, dgamma_k)`` from the gradients ``dQ``, ``dK`` of the tensors that
    ``qknorm_rope_pool`` made (as ``backward`` returns them).  ``dQpre`` may be ``dQ``, ``dKpre`` ``dK``."""
    dQpre = torch.empty_like(Qpre) if dQpre is None else dQpre
    dKpre = torch.empty_like(Kpre) if dKpre is None else dKpre
    dev, dt, shape, f32 = _device(), p.torch_dtype, p._shape, torch.float32
    for t, n in ((Qpre, "Qpre"), (Kpre, "Kpre"), (dQ, "dQ"), (dK, "dK"), (dQpre, "dQpre"), (dKpre, "dKpre")):
        _chk_vec(t, n, dt, shape, dev)
    dgamma_q = torch.empty(p.d, dtype=torch.float32, device=Qpre.device) if dgamma_q is None else dgamma_q
    dgamma_k = torch.empty(p.d, dtype=torch.float32, device=Qpre.device) if dgamma_k is None else dgamma_k
    vec, table = (p.d,), (p.N, p.d // 2)
    for t, n in ((gamma_q, "gamma_q"), (gamma_k, "gamma_k"), (dgamma_q, "dgamma_q"), (dgamma_k, "dgamma_k")):
        _chk_vec(t, n, f32, vec, dev)
    _chk_vec(cos_table, "cos_table", f32, table, dev)
    _chk_vec(sin_table, "sin_table", f32, table, dev)
    workspace = p.alloc_glue_workspace(Qpre.device) if workspace is None else workspace
    _chk_ws(workspace, "workspace", p._glue_bytes, dev)
    _check(load().llsa_qknorm_rope_backward(p._h, _ptr(Qpre), _ptr(Kpre), _ptr(gamma_q), _ptr(gamma_k), _ptr(cos_table), _ptr(sin_table),
                                            eps, _ptr(dQ), _ptr(dK), _ptr(dQpre), _ptr(dKpre), _ptr(dgamma_q),
                                            _ptr(dgamma_k), _ptr(workspace), _stream()), "llsa_qknorm_rope_backward")
    return dQpre, dKpre, dgamma_q, dgamma_k


def forward_pooled(p: Plan, Q, K, V, workspace, O=None, LSE=None, indices=None):
    """``llsa_forward_pooled``: forward pass on pooled levels already in ``workspace``."""
    for t, n in ((Q, "Q"), (K, "K"), (V, "V")):
        _chk_tensor(p, t, n)
    O = torch.empty_like(Q) if O is None else O
    LSE = torch.empty(p.batch, p.heads, p.N, dtype=torch.float32, device=Q.device) if LSE is None else LSE
    indices = p.alloc_indices(Q.device) if indices is None else indices
    if workspace.numel() < p.workspace_bytes(False) or indices.numel() * 4 < p.indices_bytes():
        raise LlsaError("workspace or indices buffer too small")
    _check(load().llsa_forward_pooled(p._h, _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(LSE), _ptr(indices),
                                      _ptr(workspace), _stream()), "llsa_forward_pooled")
    return O, LSE, indices


def forward_static(p: Plan, Q, K, V, O, LSE, indices):
    """``llsa_forward_static``: forward pass on the library's static workspace; the caller passes every
    output buffer, and neither the binding nor the library allocates."""
    for t, n in ((Q, "Q"), (K, "K"), (V, "V"), (O, "O")):
        _chk_tensor(p, t, n)
    if indices.numel() * 4 < p.indices_bytes() or LSE.numel() < p.batch * p.heads * p.N:
        raise LlsaError("indices or LSE buffer too small")
    _check(load().llsa_forward_static(p._h, _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(LSE), _ptr(indices), _stream()),
           "llsa_forward_static")


def static_workspace_bytes() -> int:
    return load().llsa_static_workspace_bytes()


def backward(p: Plan, Q, K, V, O, LSE, indices, dO, workspace, dQ=None, dK=None, dV=None):
    """``llsa_backward``: returns ``(dQ, dK, dV)``.  ``workspace`` must hold the backward size.  ``dQ`` may be ``O``; no other
    output may overlap an input or another output."""
    for t, n in ((Q, "Q"), (K, "K"), (V, "V"), (O, "O"), (dO, "dO")):
        _chk_tensor(p, t, n)
    if workspace.numel() < p.workspace_bytes(True):
        raise LlsaError("backward workspace too small")
    dQ = torch.empty_like(Q) if dQ is None else dQ
    dK = torch.empty_like(Q) if dK is None else dK
    dV = torch.empty_like(Q) if dV is None else dV
    _check(load().llsa_backward(p._h, _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(LSE), _ptr(indices), _ptr(dO),
                                _ptr(dQ), _ptr(dK), _ptr(dV), _ptr(workspace), _stream()), "llsa_backward")
    return dQ, dK, dV


def kv_backward_level0(p: Plan, via_mask: bool, Q, K, V, dO, LSE, indices, workspace, mask=None, dK0=None, dV0=None):
    """``llsa_kv_backward_level0``: level 0's dK, dV with the key-major lists from Alg. 2 or from a dense block mask.
    ``workspace`` must be the one a preceding ``backward`` call used (it holds D).  Returns ``(dK0, dV0, mask)``."""
    for t, n in ((Q, "Q"), (K, "K"), (V, "V"), (dO, "dO")):
        _chk_tensor(p, t, n)
    if via_mask and mask is None:
        mask = torch.empty(load().llsa_kv_backward_mask_bytes(p._h), dtype=torch.uint8, device=Q.device)
    dK0 = torch.empty_like(Q) if dK0 is None else dK0
    dV0 = torch.empty_like(Q) if dV0 is None else dV0
    _check(load().llsa_kv_backward_level0(p._h, int(via_mask), _ptr(Q), _ptr(K), _ptr(V), _ptr(dO), _ptr(LSE),
                                          _ptr(indices), _ptr(mask), _ptr(workspace), _ptr(dK0), _ptr(dV0), _stream()),
           "llsa_kv_backward_level0")
    return dK0, dV0, mask


def pool(p: Plan, Q, K, V, workspace):
    """``llsa_pool``: fills the pooled levels in ``workspace``."""
    for t, n in ((Q, "Q"), (K, "K"), (V, "V")):
        _chk_tensor(p, t, n)
    _check(load().llsa_pool(p._h, _ptr(Q), _ptr(K), _ptr(V), _ptr(workspace), _stream()), "llsa_pool")


def select_level(p: Plan, l: int, workspace, parent, out):
    """``llsa_select_level``: one selection level from given parent lists."""
    _check(load().llsa_select_level(p._h, l, _ptr(workspace), _ptr(parent), _ptr(out), _stream()),
           "llsa_select_level")


def attention(p: Plan, Q, K, V, indices, workspace, O=None, LSE=None):
    """``llsa_attention``: attention over given lists and pooled levels."""
    O = torch.empty_like(Q) if O is None else O
    LSE = torch.empty(p.batch, p.heads, p.N, dtype=torch.float32, device=Q.device) if LSE is None else LSE
    _check(load().llsa_attention(p._h, _ptr(Q), _ptr(K), _ptr(V), _ptr(indices), _ptr(workspace), _ptr(O), _ptr(LSE),
                                 _stream()), "llsa_attention")
    return O, LSE


def index_transpose(p: Plan, indices, workspace):
    """``llsa_index_transpose``: key-major lists of every level into a backward workspace."""
    _check(load().llsa_index_transpose(p._h, _ptr(indices), _ptr(workspace), _stream()), "llsa_index_transpose")


def reorder(x: torch.Tensor, inverse: bool = False, out: torch.Tensor | None = None) -> torch.Tensor:
    """``llsa_reorder``: tokens of ``x [..., N, d]`` (N = W*W, raster order) into nested-patch order, or back."""
    if not x.is_contiguous():
        raise LlsaError("llsa_reorder needs a contiguous tensor")
    dtype = {torch.float32: F32, torch.bfloat16: BF16}.get(x.dtype)
    if dtype is None:
        raise LlsaError("llsa_reorder: fp32 or bf16 only")
    N, d = x.shape[-2], x.shape[-1]
    out = torch.empty_like(x) if out is None else out
    _check(load().llsa_reorder(x.numel() // (N * d), N, d, dtype, int(inverse), _ptr(x), _ptr(out), _stream()), "llsa_reorder")
    return out


# ---- dense attention

class DensePlan:
    """``llsa_dense_plan``: attention over all keys (host only).  Strides are in elements, ``(batch, head, token)``, as the first three of
    ``tensor.stride()`` of a ``[batch, heads, N, d]`` view; None: contiguous."""

    def __init__(self, batch, heads, Nq, Nkv, d, kv_heads=None, sm_scale=0.0, dtype=BF16, causal=False, kernel_path=0, q_stride=None,
                 k_stride=None, v_stride=None, o_stride=None):
        lib = load()
        kv_heads = heads if kv_heads is None else kv_heads
        strides = [tuple(s) if s is not None else (0, 0, 0) for s in (q_stride, k_stride, v_stride, o_stride)]
        if any(len(s) != 3 for s in strides):
            raise LlsaError("llsa_dense_plan: strides are (batch, head, token)")
        self.desc = _DenseDesc(batch, heads, kv_heads, d, Nq, Nkv, sm_scale, dtype, int(causal), kernel_path,
                               *((ctypes.c_int64 * 3)(*s) for s in strides))
        h = ctypes.c_void_p()
        st = lib.llsa_dense_plan(ctypes.byref(self.desc), ctypes.byref(h))
        self._h = h if st == 0 else None
        _check(st, "llsa_dense_plan")
        self.batch, self.heads, self.kv_heads, self.Nq, self.Nkv, self.d = batch, heads, kv_heads, Nq, Nkv, d
        self.torch_dtype = torch.float32 if dtype == F32 else torch.bfloat16
        self._q, self._kv, self._rows = torch.Size((batch, heads, Nq, d)), torch.Size((batch, kv_heads, Nkv, d)), torch.Size((batch, heads, Nq))
        self._strides = {}
        for name, st, size in zip("qkvo", strides, (self._q, self._kv, self._kv, self._q)):
            if not any(st):
                st = (size[1] * size[2] * d, size[2] * d, d)
            self._strides[name] = (*st, 1)
        self._workspace_bytes = tuple(lib.llsa_dense_workspace_bytes(self._h, i) for i in (0, 1))

    def __del__(self):
        if getattr(self, "_h", None) is not None and _lib is not None:
            _lib.llsa_dense_plan_destroy(self._h)
            self._h = None

    def workspace_bytes(self, for_backward: bool) -> int:
        return self._workspace_bytes[bool(for_backward)]

    def alloc_workspace(self, for_backward: bool, device="cuda") -> torch.Tensor:
        """A workspace for the forward or for the backward; the backward's serves both."""
        n = self.workspace_bytes(False)
        return torch.empty(max(n, self.workspace_bytes(True) if for_backward else n, 256), dtype=torch.uint8, device=device)

    def empty(self, which: str, device="cuda") -> torch.Tensor:
        """An uninitialised tensor with the plan's strides: ``"q"`` (Q, dQ), ``"k"``, ``"v"`` or ``"o"`` (O, dO)."""
        size, st = (self._q if which in "qo" else self._kv), self._strides[which]
        if any(s == 0 and n > 1 for n, s in zip(size, st)):
            raise LlsaError(f"{which}: rows of a tensor to be written would overlap")
        return torch.empty_strided(size, st, dtype=self.torch_dtype, device=device)

    def _check(self, tensors, vectors, dev: int):
        """Tensors of the plan's layout ("q", "k", "v" or "o") and contiguous ones of a type and shape, all on device ``dev``; None: not given."""
        dt = self.torch_dtype
        for t, name, which in tensors:
            size, st = self._kv if which in "kv" else self._q, self._strides[which]
            if t.dtype is dt and t.shape == size and t.get_device() == dev and \
                    (t.stride() == st or all(n == 1 or a == b for n, a, b in zip(size, t.stride(), st))):
                continue
            raise LlsaError(f"{name}: expected {dt} {tuple(size)} with strides {st} on device {dev}, got {t.dtype} {tuple(t.shape)} "
                            f"with strides {t.stride()} on {t.device}")
        for t, name, dtype, shape in vectors:
            if t is not None:
                _chk_vec(t, name, dtype, shape, dev)


def dense_forward(p: DensePlan, Q, K, V, q_lens=None, kv_lens=None, O=None, LSE=None, workspace=None):
    """``llsa_dense_forward``: returns ``(O, LSE)``.  ``q_lens``, ``kv_lens``: ``[batch]`` int32 on the device."""
    dev, lens = _device(), (p.batch,)
    O = p.empty("o", Q.device) if O is None else O
    LSE = torch.empty(p._rows, dtype=torch.float32, device=Q.device) if LSE is None else LSE
    p._check(((Q, "Q", "q"), (K, "K", "k"), (V, "V", "v"), (O, "O", "o")),
             ((LSE, "LSE", torch.float32, p._rows), (q_lens, "q_lens", torch.int32, lens), (kv_lens, "kv_lens", torch.int32, lens)), dev)
    need = p._workspace_bytes[0]
    if need:
        workspace = p.alloc_workspace(False, Q.device) if workspace is None else workspace
        _chk_ws(workspace, "workspace", need, dev)
    _check(load().llsa_dense_forward(p._h, Q.data_ptr(), K.data_ptr(), V.data_ptr(), _ptr(q_lens), _ptr(kv_lens), O.data_ptr(), LSE.data_ptr(),
                                     workspace.data_ptr() if need else None, _stream()), "llsa_dense_forward")
    return O, LSE


def dense_backward(p: DensePlan, Q, K, V, O, LSE, dO, q_lens=None, kv_lens=None, dQ=None, dK=None, dV=None, workspace=None):
    """``llsa_dense_backward``: returns ``(dQ, dK, dV)``, with the strides of Q, K and V."""
    dev, lens = _device(), (p.batch,)
    dQ = p.empty("q", Q.device) if dQ is None else dQ
    dK = p.empty("k", Q.device) if dK is None else dK
    dV = p.empty("v", Q.device) if dV is None else dV
    p._check(((Q, "Q", "q"), (K, "K", "k"), (V, "V", "v"), (O, "O", "o"), (dO, "dO", "o"), (dQ, "dQ", "q"), (dK, "dK", "k"), (dV, "dV", "v")),
             ((LSE, "LSE", torch.float32, p._rows), (q_lens, "q_lens", torch.int32, lens), (kv_lens, "kv_lens", torch.int32, lens)), dev)
    workspace = p.alloc_workspace(True, Q.device) if workspace is None else workspace
    _chk_ws(workspace, "workspace", p._workspace_bytes[1], dev)
    _check(load().llsa_dense_backward(p._h, Q.data_ptr(), K.data_ptr(), V.data_ptr(), _ptr(q_lens), _ptr(kv_lens), O.data_ptr(), LSE.data_ptr(),
                                      dO.data_ptr(), dQ.data_ptr(), dK.data_ptr(), dV.data_ptr(), workspace.data_ptr(), _stream()),
           "llsa_dense_backward")
    return dQ, dK, dV


# ---- the norms between two blocks

class NormPlan:
    """``llsa_norm_plan`` (host only).  ``mod_stride``: elements between the rows of ``gate``, ``scale`` and ``shift`` for two batch entries; None:
    ``C``; 0: they have one row, ``[1, C]``, for all batch entries."""

    def __init__(self, batch, N, C, kind=NORM_RMS, eps=1e-6, residual_scale=1.0, dtype=BF16, mod_dtype=F32, mod_stride=None):
        lib = load()
        mod_stride = C if mod_stride is None else mod_stride
        self.desc = _NormDesc(batch, C, N, kind, eps, residual_scale, dtype, mod_dtype, mod_stride)
        h = ctypes.c_void_p()
        st = lib.llsa_norm_plan(ctypes.byref(self.desc), ctypes.byref(h))
        self._h = h if st == 0 else None
        _check(st, "llsa_norm_plan")
        self.batch, self.N, self.C, self.mod_stride = batch, N, C, mod_stride
        self.torch_dtype = torch.float32 if dtype == F32 else torch.bfloat16
        self.mod_torch_dtype = torch.float32 if mod_dtype == F32 else torch.bfloat16
        self._shape, self._vec, self._mods = torch.Size((batch, N, C)), torch.Size((C,)), torch.Size((batch if mod_stride else 1, C))
        self._stats = torch.Size((batch, N, 4))
        self._workspace_bytes = lib.llsa_norm_workspace_bytes(self._h)

    def __del__(self):
        if getattr(self, "_h", None) is not None and _lib is not None:
            _lib.llsa_norm_plan_destroy(self._h)
            self._h = None

    def workspace_bytes(self) -> int:
        return self._workspace_bytes

    def alloc_workspace(self, device="cuda") -> torch.Tensor:
        return torch.empty(self._workspace_bytes, dtype=torch.uint8, device=device)

    def _check(self, rows, vecs, mods, dev: int):
        for t, n in rows:
            if t is not None:
                _chk_vec(t, n, self.torch_dtype, self._shape, dev)
        for t, n in vecs:
            if t is not None:
                _chk_vec(t, n, torch.float32, self._vec, dev)
        for t, n in mods:
            if t is not None:
                _chk_vec(t, n, self.mod_torch_dtype, self._mods, dev, rows_only=True)
                if self._mods[0] > 1 and t.stride(0) != self.mod_stride:
                    raise LlsaError(f"{n}: expected rows {self.mod_stride} elements apart, got strides {t.stride()}")


def norm_forward(p: NormPlan, x, branch=None, gain_branch=None, gate=None, gain=None, scale=None, shift=None, x_out=None, y=None, stats=None,
                 want_y=True):
    """``llsa_norm_forward``: returns ``(x_out, y, stats)``; ``x_out`` is ``x`` where there is no branch, ``y`` None if not wanted."""
    dev = _device()
    x_out = None if branch is None else torch.empty_like(x) if x_out is None else x_out
    y = None if not want_y else torch.empty_like(x) if y is None else y
    stats = torch.empty(p._stats, dtype=torch.float32, device=x.device) if stats is None else stats
    p._check(((x, "x"), (branch, "branch"), (x_out, "x_out"), (y, "y")), ((gain_branch, "gain_branch"), (gain, "gain")),
             ((gate, "gate"), (scale, "scale"), (shift, "shift")), dev)
    _chk_vec(stats, "stats", torch.float32, p._stats, dev)
    _check(load().llsa_norm_forward(p._h, x.data_ptr(), _ptr(branch), _ptr(gain_branch), _ptr(gate), _ptr(gain), _ptr(scale), _ptr(shift),
                                    _ptr(x_out), _ptr(y), stats.data_ptr(), _stream()), "llsa_norm_forward")
    return x if branch is None else x_out, y, stats


def norm_backward(p: NormPlan, x_out, dy, stats, branch=None, gain_branch=None, gate=None, gain=None, scale=None, shift=None, dx_out=None, dx=None,
                  dbranch=None, workspace=None):
    """``llsa_norm_backward``: a dict with ``dx``, ``dbranch`` and the fp32 gradients of those of ``gain_branch``, ``gate``, ``gain``, ``scale``, ``shift``
    (whose values are not needed) that are given.  ``dx`` may be ``dy`` or ``dx_out``, ``dbranch`` may be ``branch``."""
    dev = _device()
    out = {"dx": torch.empty_like(x_out) if dx is None else dx}
    if branch is not None:
        out["dbranch"] = torch.empty_like(branch) if dbranch is None else dbranch
    p._check(((x_out, "x_out"), (dy, "dy"), (branch, "branch"), (dx_out, "dx_out"), (out["dx"], "dx"), (out.get("dbranch"), "dbranch")),
             ((gain_branch, "gain_branch"), (gain, "gain")), ((gate, "gate"), (scale, "scale"), (shift, "shift")), dev)
    _chk_vec(stats, "stats", torch.float32, p._stats, dev)
    sums = [None] * 5
    for i, (t, n) in enumerate(((gain_branch, "dgain_branch"), (gate, "dgate"), (gain, "dgain"), (scale, "dscale"), (shift, "dshift"))):
        if t is not None:                                    # (contiguous; torch.empty takes twice as long, 5 of the 26 us of a call)
            out[n] = torch.empty_like(t, dtype=torch.float32, memory_format=torch.contiguous_format)
            sums[i] = out[n].data_ptr()
    if workspace is None and any(sums):
        workspace = p.alloc_workspace(x_out.device)
    _chk_ws(workspace, "workspace", p._workspace_bytes, dev)
    _check(load().llsa_norm_backward(p._h, x_out.data_ptr(), _ptr(branch), _ptr(gain_branch), _ptr(gate), _ptr(gain), _ptr(scale), stats.data_ptr(),
                                     _ptr(dy), _ptr(dx_out), out["dx"].data_ptr(), _ptr(out.get("dbranch")), *sums, _ptr(workspace), _stream()),
           "llsa_norm_backward")
    return out


def measured_peaks(mfma_iters: int = 20000, copy_bytes: int = 1 << 30, reps: int = 5) -> dict:
    """Times ``llsa_calibrate_mfma`` (2048 workgroups: 8 per CU) and ``llsa_calibrate_copy`` with HIP events: the
    bf16 MFMA rate and the copy bandwidth this GPU delivers, best of ``reps``."""
    lib = load()
    out = torch.zeros(4, dtype=torch.float32, device="cuda")
    src = torch.zeros(copy_bytes, dtype=torch.uint8, device="cuda")
    dst = torch.empty_like(src)
    wgs = 2048
    best = {"mfma": float("inf"), "copy": float("inf")}
    for rep in range(reps + 1):
        for name, call in (("mfma", lambda: lib.llsa_calibrate_mfma(_ptr(out), mfma_iters, wgs, _stream())),
                           ("copy", lambda: lib.llsa_calibrate_copy(_ptr(src), _ptr(dst), copy_bytes, _stream()))):
            e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            e0.record()
            _check(call(), f"llsa_calibrate_{name}")
            e1.record()
            e1.synchronize()
            if rep > 0:                                      # the first round warms up
                best[name] = min(best[name], e0.elapsed_time(e1))
    flop = wgs * 4 * 8 * mfma_iters * 16384.0
    return {"mfma_bf16_tflops": flop / (best["mfma"] * 1e-3) / 1e12, "copy_gbps": 2.0 * copy_bytes / (best["copy"] * 1e-3) / 1e9,
            "mfma_ms": best["mfma"], "copy_ms": best["copy"]}


def stage_names() -> list[str]:
    lib = load()
    return [lib.llsa_stage_name(i).decode() for i in range(lib.llsa_stage_count())]


def stage_timing_begin(stage: int | str = -1, max_calls: int = 64):
    """``llsa_stage_timing_begin``: bracket one stage (index or name; -1 = all) with HIP events."""
    if isinstance(stage, str):
        stage = stage_names().index(stage)
    _check(load().llsa_stage_timing_begin(stage, max_calls), "llsa_stage_timing_begin")


def stage_timing_end() -> dict[str, tuple[float, int]]:
    """``llsa_stage_timing_end``: ``{stage name: (summed ms, number of brackets)}``."""
    lib = load()
    n = lib.llsa_stage_count()
    ms = (ctypes.c_double * n)()
    cnt = (ctypes.c_int32 * n)()
    _check(lib.llsa_stage_timing_end(ms, cnt), "llsa_stage_timing_end")
    return {name: (ms[i], cnt[i]) for i, name in enumerate(stage_names())}
