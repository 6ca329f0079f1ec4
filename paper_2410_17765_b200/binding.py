"""ctypes binding of libcpmtp.so: argument marshalling only.

Every step of the computation runs in the library's CUDA kernels; torch is used
for device memory and the current stream.  There is no fallback: if the shared
library is missing or fails to load, importing this module's functions raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import operator
import os
import struct
from array import array
from dataclasses import dataclass
from typing import Optional

import torch

from .build import DEBUG_LIB_PATH, LIB_PATH

OP_FORWARD, OP_BACKWARD, OP_SCORE, OP_SAMPLE, OP_FORWARD_FULL, OP_BACKWARD_FULL = 0, 1, 2, 3, 4, 5
OP_DISTILL_FORWARD, OP_DISTILL_BACKWARD = 6, 7
FLAG_AUX = 1
FLAG_PER_TOKEN = 2
FLAG_RECOMPUTE_Z = 4
FLAG_ACCUM_GRADS = 8

EXPORTS = [
    "cpmtp_version", "cpmtp_status_string", "cpmtp_workspace_bytes", "cpmtp_forward", "cpmtp_backward",
    "cpmtp_score_draft", "cpmtp_host_staging_bytes", "cpmtp_forward_host", "cpmtp_profile_begin",
    "cpmtp_profile_end", "cpmtp_score_draft_static", "cpmtp_sample_draft",
    "cpmtp_forward_full", "cpmtp_backward_full", "cpmtp_verify_draft",
    "cpmtp_distill_forward", "cpmtp_distill_backward", "cpmtp_reload_knobs", "cpmtp_debug_status",
    "cpmtp_embed_forward", "cpmtp_embed_workspace_bytes", "cpmtp_embed_backward",
    "cpmtp_norm_forward", "cpmtp_norm_workspace_bytes", "cpmtp_norm_backward",
    "cpmtp_adamw_step", "cpmtp_adamw_step_clocked", "cpmtp_adamw_state_values", "cpmtp_grad_norm_workspace_bytes", "cpmtp_grad_norm",
    "cpmtp_cache_append", "cpmtp_cache_attend_workspace_bytes", "cpmtp_cache_attend", "cpmtp_cache_evict_workspace_bytes",
    "cpmtp_cache_evict", "cpmtp_sample_logits",
]

STATIC_SCRATCH_BYTES = 4 << 20
BF16, F32 = 0, 1
EMBED_PAD = -1
GATE_NONE, GATE_ROW, GATE_CHANNEL = 0, 1, 2
ADAMW_BLOCK = 256
CACHE_MAX_D = 128
SAMPLE_MAX_V = 1 << 24

STAGES = ["gate", "proj", "lse", "mixture", "finalize", "coeff", "logit_grad", "dz", "de", "de_convert",
          "dw_head", "dh", "dw_g", "draft_step", "teacher_lse", "kl", "embed", "embed_grad", "norm", "norm_grad", "grad_norm",
          "adamw", "cache_append", "cache_attend", "cache_evict", "sample"]


class CShape(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int32), ("d", ctypes.c_int32), ("V", ctypes.c_int32), ("n", ctypes.c_int32),
                ("r", ctypes.c_int32), ("flags", ctypes.c_uint32), ("aux_coef", ctypes.c_float)]


class CSaved(ctypes.Structure):
    _fields_ = [("lse", ctypes.c_void_p), ("tgt", ctypes.c_void_p), ("logw", ctypes.c_void_p),
                ("q", ctypes.c_void_p), ("wbar", ctypes.c_void_p), ("z", ctypes.c_void_p)]


class CDistillSaved(ctypes.Structure):
    _fields_ = [("lse_t", ctypes.c_void_p), ("logpi", ctypes.c_void_p), ("pm", ctypes.c_void_p),
                ("kl", ctypes.c_void_p)]


class CEmbedShape(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("V", ctypes.c_int32), ("d", ctypes.c_int32), ("type", ctypes.c_int32),
                ("ld_table", ctypes.c_int64), ("ld_rows", ctypes.c_int64), ("scale", ctypes.c_float),
                ("flags", ctypes.c_uint32)]


def _rows_fields(*names):
    return [f for n in names for f in ((n, ctypes.c_void_p), ("ld_" + n, ctypes.c_int64))]


class CNormArgs(ctypes.Structure):
    _fields_ = ([("N", ctypes.c_int32), ("d", ctypes.c_int32), ("stream_type", ctypes.c_int32), ("gate_kind", ctypes.c_int32),
                 ("flags", ctypes.c_uint32), ("eps", ctypes.c_float), ("res_scale", ctypes.c_float)]
                + _rows_fields("x", "block", "gate") + [("w_post", ctypes.c_void_p), ("w_pre", ctypes.c_void_p)]
                + _rows_fields("x_out", "y") + [("rstd_post", ctypes.c_void_p), ("rstd_pre", ctypes.c_void_p)]
                + _rows_fields("dy", "dx_out", "dx", "dblock", "dgate")
                + [("dw_post", ctypes.c_void_p), ("dw_pre", ctypes.c_void_p)])


class CAdamWTensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("master", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("m_exp", ctypes.c_void_p), ("v_exp", ctypes.c_void_p), ("numel", ctypes.c_int64),
                ("param_type", ctypes.c_int32), ("grad_type", ctypes.c_int32), ("lr_scale", ctypes.c_float),
                ("decay_scale", ctypes.c_float)]


class CAdamWHyper(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("weight_decay", ctypes.c_double), ("step", ctypes.c_int64), ("seed", ctypes.c_uint32),
                ("state_bits", ctypes.c_int32), ("coef", ctypes.c_void_p)]


class CAdamWClock(ctypes.Structure):
    _fields_ = [("step", ctypes.c_int64), ("lr", ctypes.c_double), ("seed", ctypes.c_uint32), ("key", ctypes.c_uint32), ("bc1", ctypes.c_double),
                ("rsqrt_bc2", ctypes.c_float), ("unused", ctypes.c_float)]


class CCache(ctypes.Structure):
    _fields_ = ([("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("acc", ctypes.c_void_p), ("pages", ctypes.c_int32),
                 ("page_slots", ctypes.c_int32), ("H", ctypes.c_int32), ("D", ctypes.c_int32)]
                + [(n, ctypes.c_int64) for n in ("k_page", "k_slot", "k_head", "v_page", "v_slot", "v_head", "acc_page", "acc_head")])


class CCacheSeqs(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("lens", ctypes.c_void_p), ("q_lens", ctypes.c_void_p), ("ld_table", ctypes.c_int64),
                ("B", ctypes.c_int32), ("width", ctypes.c_int32), ("Q", ctypes.c_int32), ("unused", ctypes.c_int32)]


class CTokens(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("seq", ctypes.c_int64), ("token", ctypes.c_int64), ("head", ctypes.c_int64)]


class CAttendArgs(ctypes.Structure):
    _fields_ = [("q", CTokens), ("out", CTokens), ("lse", ctypes.c_void_p), ("Hq", ctypes.c_int32), ("scale", ctypes.c_float)]


class CEvictArgs(ctypes.Structure):
    _fields_ = [("table_out", ctypes.c_void_p), ("ld_table_out", ctypes.c_int64), ("budget", ctypes.c_int32), ("recent", ctypes.c_int32),
                ("lens_out", ctypes.c_void_p), ("kept", ctypes.c_void_p)]


class CSampleArgs(ctypes.Structure):
    _fields_ = [("logits", ctypes.c_void_p), ("ld", ctypes.c_int64), ("N", ctypes.c_int32), ("V", ctypes.c_int32), ("type", ctypes.c_int32),
                ("top_k", ctypes.c_int32), ("temperature", ctypes.c_float), ("top_p", ctypes.c_float), ("min_p", ctypes.c_float),
                ("unused", ctypes.c_int32)] + [(n, ctypes.c_void_p) for n in (
                    "temperatures", "top_ks", "top_ps", "min_ps", "uniform", "given", "tokens", "logp", "logp_given", "kept")]


_lib = None


def load_library() -> ctypes.CDLL:
    """Load libcpmtp.so (built in-tree by build.py); raise if it is absent."""
    global _lib
    if _lib is not None:
        return _lib
    # CPMTP_LIBRARY=debug selects the checked build (index checks in every epilogue), made by
    # `python -m paper_2410_17765_b200.build --debug`; any other value is taken as a path
    choice = os.environ.get("CPMTP_LIBRARY", "")
    path = LIB_PATH if not choice else DEBUG_LIB_PATH if choice == "debug" else choice
    if not os.path.exists(path):
        raise RuntimeError(f"{path} not found: build it with `python -m paper_2410_17765_b200.build`")
    lib = ctypes.CDLL(path)
    vp, sz, i32p, fp = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p
    shp = ctypes.POINTER(CShape)
    svp = ctypes.POINTER(CSaved)
    lib.cpmtp_version.restype = ctypes.c_int
    lib.cpmtp_status_string.restype = ctypes.c_char_p
    lib.cpmtp_status_string.argtypes = [ctypes.c_int]
    lib.cpmtp_workspace_bytes.restype = sz
    lib.cpmtp_workspace_bytes.argtypes = [shp, ctypes.c_int]
    lib.cpmtp_host_staging_bytes.restype = sz
    lib.cpmtp_host_staging_bytes.argtypes = [shp]
    lib.cpmtp_forward.restype = ctypes.c_int
    lib.cpmtp_forward.argtypes = [shp, vp, vp, vp, vp, i32p, fp, fp, svp, i32p, vp, sz, i32p, vp]
    lib.cpmtp_backward.restype = ctypes.c_int
    lib.cpmtp_backward.argtypes = [shp, vp, vp, vp, vp, i32p, svp, fp, vp, vp, vp, vp, vp, sz, i32p, vp]
    lib.cpmtp_score_draft.restype = ctypes.c_int
    lib.cpmtp_score_draft.argtypes = [shp, vp, vp, vp, vp, i32p, fp, fp, vp, sz, i32p, vp]
    lib.cpmtp_forward_host.restype = ctypes.c_int
    lib.cpmtp_forward_host.argtypes = [shp, vp, vp, vp, vp, i32p, fp, fp, svp, vp, sz, i32p, vp]
    lib.cpmtp_sample_draft.restype = ctypes.c_int
    lib.cpmtp_sample_draft.argtypes = [shp, vp, vp, vp, vp, fp, ctypes.c_float, ctypes.c_int32, i32p, i32p, fp, i32p,
                                       fp, vp, sz, i32p, vp]
    lib.cpmtp_forward_full.restype = ctypes.c_int
    lib.cpmtp_forward_full.argtypes = [shp, vp, vp, vp, i32p, fp, fp, fp, svp, i32p, vp, sz, i32p, vp]
    lib.cpmtp_backward_full.restype = ctypes.c_int
    lib.cpmtp_backward_full.argtypes = [shp, vp, vp, vp, i32p, svp, fp, vp, vp, vp, vp, sz, i32p, vp]
    lib.cpmtp_verify_draft.restype = ctypes.c_int
    lib.cpmtp_verify_draft.argtypes = [ctypes.c_int32, ctypes.c_int32, i32p, i32p, fp, fp, fp, i32p, vp]
    lib.cpmtp_score_draft_static.restype = ctypes.c_int
    lib.cpmtp_score_draft_static.argtypes = [shp, vp, vp, vp, vp, i32p, fp, fp, i32p, vp]
    dsp = ctypes.POINTER(CDistillSaved)
    lib.cpmtp_distill_forward.restype = ctypes.c_int
    lib.cpmtp_distill_forward.argtypes = [shp, vp, vp, vp, vp, i32p, vp, ctypes.c_float, ctypes.c_float, fp, fp, fp,
                                          svp, dsp, vp, sz, i32p, vp]
    lib.cpmtp_distill_backward.restype = ctypes.c_int
    lib.cpmtp_distill_backward.argtypes = [shp, vp, vp, vp, vp, i32p, vp, svp, dsp, ctypes.c_float, ctypes.c_float,
                                           fp, fp, vp, vp, vp, vp, vp, sz, i32p, vp]
    esp, nap, atp = ctypes.POINTER(CEmbedShape), ctypes.POINTER(CNormArgs), vp   # atp: an array's address
    lib.cpmtp_embed_forward.restype = ctypes.c_int
    lib.cpmtp_embed_forward.argtypes = [esp, vp, i32p, vp, i32p, vp]
    lib.cpmtp_embed_workspace_bytes.restype = sz
    lib.cpmtp_embed_workspace_bytes.argtypes = [esp]
    lib.cpmtp_embed_backward.restype = ctypes.c_int
    lib.cpmtp_embed_backward.argtypes = [esp, vp, i32p, vp, vp, sz, i32p, vp]
    lib.cpmtp_norm_forward.restype = ctypes.c_int
    lib.cpmtp_norm_forward.argtypes = [nap, vp]
    lib.cpmtp_norm_workspace_bytes.restype = sz
    lib.cpmtp_norm_workspace_bytes.argtypes = [nap]
    lib.cpmtp_norm_backward.restype = ctypes.c_int
    lib.cpmtp_norm_backward.argtypes = [nap, vp, sz, vp]
    lib.cpmtp_adamw_step.restype = ctypes.c_int
    lib.cpmtp_adamw_step.argtypes = [atp, ctypes.c_int32, ctypes.POINTER(CAdamWHyper), vp]
    lib.cpmtp_adamw_step_clocked.restype = ctypes.c_int
    lib.cpmtp_adamw_step_clocked.argtypes = [atp, ctypes.c_int32, ctypes.POINTER(CAdamWHyper), vp, vp]
    lib.cpmtp_adamw_state_values.restype = ctypes.c_int
    lib.cpmtp_adamw_state_values.argtypes = [vp, vp, ctypes.c_int64, ctypes.c_int32, vp, vp]
    lib.cpmtp_grad_norm_workspace_bytes.restype = sz
    lib.cpmtp_grad_norm_workspace_bytes.argtypes = [atp, ctypes.c_int32]
    lib.cpmtp_grad_norm.restype = ctypes.c_int
    lib.cpmtp_grad_norm.argtypes = [atp, ctypes.c_int32, ctypes.c_float, fp, fp, vp, sz, vp]
    csp, cqp, tkp = ctypes.POINTER(CCache), ctypes.POINTER(CCacheSeqs), ctypes.POINTER(CTokens)
    lib.cpmtp_cache_append.restype = ctypes.c_int
    lib.cpmtp_cache_append.argtypes = [csp, cqp, tkp, tkp, i32p, vp]
    lib.cpmtp_cache_attend_workspace_bytes.restype = sz
    lib.cpmtp_cache_attend_workspace_bytes.argtypes = [csp, cqp, ctypes.c_int32]
    lib.cpmtp_cache_attend.restype = ctypes.c_int
    lib.cpmtp_cache_attend.argtypes = [csp, cqp, ctypes.POINTER(CAttendArgs), vp, sz, i32p, vp]
    lib.cpmtp_cache_evict_workspace_bytes.restype = sz
    lib.cpmtp_cache_evict_workspace_bytes.argtypes = [csp, cqp, ctypes.c_int32]
    lib.cpmtp_cache_evict.restype = ctypes.c_int
    lib.cpmtp_cache_evict.argtypes = [csp, cqp, ctypes.POINTER(CEvictArgs), vp, sz, i32p, vp]
    lib.cpmtp_sample_logits.restype = ctypes.c_int
    lib.cpmtp_sample_logits.argtypes = [ctypes.POINTER(CSampleArgs), i32p, vp]
    lib.cpmtp_reload_knobs.restype = ctypes.c_int
    lib.cpmtp_debug_status.restype = ctypes.c_int
    lib.cpmtp_profile_begin.restype = ctypes.c_int
    lib.cpmtp_profile_end.restype = ctypes.c_int
    lib.cpmtp_profile_end.argtypes = [ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_int32), ctypes.c_int]
    _lib = lib
    return lib


def debug_status() -> int:
    """cpmtp_debug_status: -1 for the release library; for the checked build 0 while every index check has
    passed and 3 once one has failed (synchronizes the device)."""
    return int(load_library().cpmtp_debug_status())


def reload_knobs() -> None:
    """cpmtp_reload_knobs: have the library read its CPMTP_* environment knobs again."""
    _check(load_library().cpmtp_reload_knobs())


@contextlib.contextmanager
def knobs(**values):
    """Set CPMTP_* environment knobs (name=value; None leaves a knob alone) for the calls made inside the
    block, then restore the environment; the library re-reads its knobs on entry and on exit."""
    values = {k: v for k, v in values.items() if v is not None}
    old = {k: os.environ.get(k) for k in values}
    try:
        for k, v in values.items():
            os.environ[k] = str(v)
        reload_knobs()
        yield
    finally:
        for k, v in old.items():
            if v is None:
                os.environ.pop(k, None)
            else:
                os.environ[k] = v
        reload_knobs()


def profile_begin() -> None:
    _check(load_library().cpmtp_profile_begin())


def profile_end() -> dict:
    """Stop per-stage timing; returns {stage: (total_ms, launches)} for stages that ran."""
    n = len(STAGES)
    ms = (ctypes.c_float * n)()
    cnt = (ctypes.c_int32 * n)()
    total = load_library().cpmtp_profile_end(ms, cnt, n)
    if total < 0:
        _check(total)
    return {STAGES[i]: (float(ms[i]), int(cnt[i])) for i in range(n) if cnt[i] > 0}


class CpmtpError(RuntimeError):
    pass


def _check(rc: int) -> None:
    if rc != 0:
        raise CpmtpError(f"cpmtp error {rc}: {load_library().cpmtp_status_string(rc).decode()}")


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def make_shape(N, d, V, n, r, aux_coef: Optional[float] = None) -> CShape:
    flags = FLAG_AUX if aux_coef is not None else 0
    return CShape(N, d, V, n, r, flags, float(aux_coef or 0.0))


def workspace_bytes(shape: CShape, op: int) -> int:
    return int(load_library().cpmtp_workspace_bytes(ctypes.byref(shape), op))


def host_staging_bytes(shape: CShape) -> int:
    return int(load_library().cpmtp_host_staging_bytes(ctypes.byref(shape)))


def alloc_workspace(nbytes: int, device="cuda") -> torch.Tensor:
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


@dataclass
class Saved:
    """Forward results kept for cpmtp_backward (device tensors)."""
    lse: torch.Tensor
    tgt: torch.Tensor
    logw: torch.Tensor
    q: torch.Tensor
    wbar: torch.Tensor
    z: torch.Tensor

    @staticmethod
    def alloc_full(shape: CShape, device="cuda") -> "Saved":
        """Saved state for the full-head entry points (no projected hidden states)."""
        K = shape.n * shape.r
        f = dict(dtype=torch.float32, device=device)
        return Saved(lse=torch.empty((shape.N, K), **f), tgt=torch.empty((shape.N, K), **f),
                     logw=torch.empty((shape.N, shape.r), **f), q=torch.empty((shape.N, shape.r), **f),
                     wbar=torch.empty((32,), **f), z=torch.empty(8, dtype=torch.bfloat16, device=device))

    @staticmethod
    def alloc(shape: CShape, device="cuda") -> "Saved":
        K = shape.n * shape.r
        f = dict(dtype=torch.float32, device=device)
        return Saved(lse=torch.empty((shape.N, K), **f), tgt=torch.empty((shape.N, K), **f),
                     logw=torch.empty((shape.N, shape.r), **f), q=torch.empty((shape.N, shape.r), **f),
                     wbar=torch.empty((32,), **f),
                     z=torch.empty((shape.N, K, shape.d), dtype=torch.bfloat16, device=device))

    def c_struct(self) -> CSaved:
        return CSaved(self.lse.data_ptr(), self.tgt.data_ptr(), self.logw.data_ptr(), self.q.data_ptr(),
                      self.wbar.data_ptr(), self.z.data_ptr() if self.z is not None else None)


def _shape_of(h, W_head, E, W_g, x, aux_coef) -> CShape:
    N, d = h.shape
    V = E.shape[0]
    n = x.shape[1]
    r = W_g.shape[0]
    assert W_head.shape == (n * r, d, d) and E.shape[1] == d and W_g.shape[1] == d and x.shape[0] == N
    for t in (h, W_head, E, W_g):
        assert t.dtype == torch.bfloat16 and t.is_contiguous()
    assert x.dtype == torch.int32 and x.is_contiguous()
    return make_shape(N, d, V, n, r, aux_coef)


def forward(h, W_head, E, W_g, x, *, aux_coef: Optional[float] = None, saved: Optional[Saved] = None,
            want_loss: bool = True, want_counts: bool = False, workspace: Optional[torch.Tensor] = None,
            dev_status: Optional[torch.Tensor] = None, out: Optional[dict] = None,
            recompute_z: bool = False) -> dict:
    """cpmtp_forward on device tensors; returns {"logp", "loss", "counts"} (device tensors).
    recompute_z: do not keep z in `saved` (CPMTP_FLAG_RECOMPUTE_Z; pass the same to backward)."""
    lib = load_library()
    shape = _shape_of(h, W_head, E, W_g, x, aux_coef)
    if recompute_z:
        shape.flags |= FLAG_RECOMPUTE_Z
    dev = h.device
    if workspace is None:
        workspace = alloc_workspace(workspace_bytes(shape, OP_FORWARD), dev)
    res = out if out is not None else {}
    if "logp" not in res:
        res["logp"] = torch.empty(shape.N, dtype=torch.float32, device=dev)
    if want_loss and "loss" not in res:
        res["loss"] = torch.empty(1, dtype=torch.float32, device=dev)
    if want_counts and "counts" not in res:
        res["counts"] = torch.empty(shape.r, dtype=torch.int32, device=dev)
    cs = saved.c_struct() if saved is not None else None
    rc = lib.cpmtp_forward(ctypes.byref(shape), _ptr(h), _ptr(W_head), _ptr(E), _ptr(W_g), _ptr(x),
                           _ptr(res["logp"]), _ptr(res.get("loss")) if want_loss else None,
                           ctypes.byref(cs) if cs is not None else None,
                           _ptr(res.get("counts")) if want_counts else None, _ptr(workspace),
                           workspace.numel(), _ptr(dev_status), _stream())
    _check(rc)
    return res


def backward(h, W_head, E, W_g, x, saved: Saved, *, aux_coef: Optional[float] = None,
             dloss_dlogp: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
             dev_status: Optional[torch.Tensor] = None, out: Optional[dict] = None,
             skip: tuple = (), dloss_dprefix: Optional[torch.Tensor] = None,
             recompute_z: bool = False, accumulate: bool = False) -> dict:
    """cpmtp_backward on device tensors; returns {"dh", "dW_head", "dE", "dW_g"} (bf16 device tensors).
    Names listed in `skip` are not computed (passed as NULL).  dloss_dprefix [N, n] fp32 selects the
    per-token objective sum_i sum_s dloss_dprefix[i, s] * log P(x[i, 0..s]) (CPMTP_FLAG_PER_TOKEN).
    accumulate: add to the tensors given in `out` instead of overwriting them (CPMTP_FLAG_ACCUM_GRADS)."""
    lib = load_library()
    shape = _shape_of(h, W_head, E, W_g, x, aux_coef)
    if recompute_z:
        shape.flags |= FLAG_RECOMPUTE_Z
    if accumulate:
        assert out is not None, "accumulation needs the tensors to add to"
        shape.flags |= FLAG_ACCUM_GRADS
    if dloss_dprefix is not None:
        assert dloss_dlogp is None and dloss_dprefix.shape == (shape.N, shape.n) and dloss_dprefix.dtype == torch.float32
        shape.flags |= FLAG_PER_TOKEN
        dloss_dlogp = dloss_dprefix.contiguous()
    if workspace is None:
        workspace = alloc_workspace(workspace_bytes(shape, OP_BACKWARD), h.device)
    res = out if out is not None else {}
    for name, ref in (("dh", h), ("dW_head", W_head), ("dE", E), ("dW_g", W_g)):
        if name not in res and name not in skip:
            res[name] = torch.empty_like(ref)
    cs = saved.c_struct()
    rc = lib.cpmtp_backward(ctypes.byref(shape), _ptr(h), _ptr(W_head), _ptr(E), _ptr(W_g), _ptr(x),
                            ctypes.byref(cs), _ptr(dloss_dlogp), _ptr(res.get("dh")), _ptr(res.get("dW_head")),
                            _ptr(res.get("dE")), _ptr(res.get("dW_g")), _ptr(workspace), workspace.numel(),
                            _ptr(dev_status), _stream())
    _check(rc)
    return res


def score_draft(h, W_head, E, W_g, draft, *, want_prefix: bool = True,
                workspace: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None,
                out: Optional[dict] = None) -> dict:
    """cpmtp_score_draft; returns {"logp_joint", "logp_prefix"} (device tensors)."""
    lib = load_library()
    shape = _shape_of(h, W_head, E, W_g, draft, None)
    if workspace is None:
        workspace = alloc_workspace(workspace_bytes(shape, OP_SCORE), h.device)
    res = out if out is not None else {}
    if "logp_joint" not in res:
        res["logp_joint"] = torch.empty(shape.N, dtype=torch.float32, device=h.device)
    if want_prefix and "logp_prefix" not in res:
        res["logp_prefix"] = torch.empty((shape.N, shape.n), dtype=torch.float32, device=h.device)
    rc = lib.cpmtp_score_draft(ctypes.byref(shape), _ptr(h), _ptr(W_head), _ptr(E), _ptr(W_g), _ptr(draft),
                               _ptr(res["logp_joint"]), _ptr(res.get("logp_prefix")) if want_prefix else None,
                               _ptr(workspace), workspace.numel(), _ptr(dev_status), _stream())
    _check(rc)
    return res


def sample_draft(h, W_head, E, W_g, n: int, *, uniform: Optional[torch.Tensor] = None, temperature: float = 1.0,
                 topk: int = 1, forced: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                 dev_status: Optional[torch.Tensor] = None, out: Optional[dict] = None) -> dict:
    """cpmtp_sample_draft; returns {"draft", "logp_joint", "topk_tokens", "topk_logp"} (device tensors).
    uniform: [N, n, V] fp32 strictly inside (0, 1) for Gumbel-max sampling, or None for the greedy draft.
    forced: [N, n] int32, entries >= 0 fix the token of that step (-1: left to the sampler), or None."""
    lib = load_library()
    N, d = h.shape
    V, r = E.shape[0], W_g.shape[0]
    assert W_head.shape == (n * r, d, d)
    for t in (h, W_head, E, W_g):
        assert t.dtype == torch.bfloat16 and t.is_contiguous()
    if uniform is not None:
        assert uniform.shape == (N, n, V) and uniform.dtype == torch.float32 and uniform.is_contiguous()
    if forced is not None:
        assert forced.shape == (N, n) and forced.dtype == torch.int32 and forced.is_contiguous()
    shape = make_shape(N, d, V, n, r)
    if workspace is None:
        workspace = alloc_workspace(workspace_bytes(shape, OP_SAMPLE), h.device)
    res = out if out is not None else {}
    dev = h.device
    res.setdefault("draft", torch.empty((N, n), dtype=torch.int32, device=dev))
    res.setdefault("logp_joint", torch.empty(N, dtype=torch.float32, device=dev))
    res.setdefault("topk_tokens", torch.empty((N, n, topk), dtype=torch.int32, device=dev))
    res.setdefault("topk_logp", torch.empty((N, n, topk), dtype=torch.float32, device=dev))
    rc = lib.cpmtp_sample_draft(ctypes.byref(shape), _ptr(h), _ptr(W_head), _ptr(E), _ptr(W_g), _ptr(uniform),
                                ctypes.c_float(temperature), topk, _ptr(forced), _ptr(res["draft"]),
                                _ptr(res["logp_joint"]),
                                _ptr(res["topk_tokens"]), _ptr(res["topk_logp"]), _ptr(workspace), workspace.numel(),
                                _ptr(dev_status), _stream())
    _check(rc)
    return res


def _shape_full(h, W_full, W_g, x, aux_coef) -> CShape:
    N, d = h.shape
    K, V, d2 = W_full.shape
    n, r = x.shape[1], W_g.shape[0]
    assert K == n * r and d2 == d and W_g.shape[1] == d and x.shape[0] == N
    for t in (h, W_full, W_g):
        assert t.dtype == torch.bfloat16 and t.is_contiguous()
    assert x.dtype == torch.int32 and x.is_contiguous()
    return make_shape(N, d, V, n, r, aux_coef)


def forward_full(h, W_full, W_g, x, *, aux_coef: Optional[float] = None, saved: Optional[Saved] = None,
                 want_prefix: bool = False, workspace: Optional[torch.Tensor] = None,
                 dev_status: Optional[torch.Tensor] = None, out: Optional[dict] = None) -> dict:
    """cpmtp_forward_full (W_full [n*r, V, d]); returns {"logp", "loss", "counts"[, "logp_prefix"]}."""
    lib = load_library()
    shape = _shape_full(h, W_full, W_g, x, aux_coef)
    dev = h.device
    if workspace is None:
        workspace = alloc_workspace(workspace_bytes(shape, OP_FORWARD_FULL), dev)
    res = out if out is not None else {}
    res.setdefault("logp", torch.empty(shape.N, dtype=torch.float32, device=dev))
    res.setdefault("loss", torch.empty(1, dtype=torch.float32, device=dev))
    res.setdefault("counts", torch.empty(shape.r, dtype=torch.int32, device=dev))
    if want_prefix:
        res.setdefault("logp_prefix", torch.empty((shape.N, shape.n), dtype=torch.float32, device=dev))
    cs = saved.c_struct() if saved is not None else None
    rc = lib.cpmtp_forward_full(ctypes.byref(shape), _ptr(h), _ptr(W_full), _ptr(W_g), _ptr(x), _ptr(res["logp"]),
                                _ptr(res["loss"]), _ptr(res.get("logp_prefix")) if want_prefix else None,
                                ctypes.byref(cs) if cs is not None else None, _ptr(res["counts"]), _ptr(workspace),
                                workspace.numel(), _ptr(dev_status), _stream())
    _check(rc)
    return res


def backward_full(h, W_full, W_g, x, saved: Saved, *, aux_coef: Optional[float] = None,
                  dloss_dlogp: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                  dev_status: Optional[torch.Tensor] = None, out: Optional[dict] = None,
                  dloss_dprefix: Optional[torch.Tensor] = None, accumulate: bool = False) -> dict:
    """cpmtp_backward_full; returns {"dh", "dW_full", "dW_g"} (bf16 device tensors).
    dloss_dprefix and accumulate as for backward()."""
    lib = load_library()
    shape = _shape_full(h, W_full, W_g, x, aux_coef)
    if accumulate:
        assert out is not None, "accumulation needs the tensors to add to"
        shape.flags |= FLAG_ACCUM_GRADS
    if dloss_dprefix is not None:
        assert dloss_dlogp is None and dloss_dprefix.shape == (shape.N, shape.n) and dloss_dprefix.dtype == torch.float32
        shape.flags |= FLAG_PER_TOKEN
        dloss_dlogp = dloss_dprefix.contiguous()
    if workspace is None:
        workspace = alloc_workspace(workspace_bytes(shape, OP_BACKWARD_FULL), h.device)
    res = out if out is not None else {}
    for name, ref in (("dh", h), ("dW_full", W_full), ("dW_g", W_g)):
        if name not in res:
            res[name] = torch.empty_like(ref)
    cs = saved.c_struct()
    rc = lib.cpmtp_backward_full(ctypes.byref(shape), _ptr(h), _ptr(W_full), _ptr(W_g), _ptr(x), ctypes.byref(cs),
                                 _ptr(dloss_dlogp), _ptr(res["dh"]), _ptr(res["dW_full"]), _ptr(res["dW_g"]),
                                 _ptr(workspace), workspace.numel(), _ptr(dev_status), _stream())
    _check(rc)
    return res


def verify_draft(draft: Optional[torch.Tensor] = None, base_tokens: Optional[torch.Tensor] = None, *,
                 logp_prefix: Optional[torch.Tensor] = None, logp_base: Optional[torch.Tensor] = None,
                 uniform: Optional[torch.Tensor] = None) -> torch.Tensor:
    """cpmtp_verify_draft: accepted draft length per position (int32 device tensor).
    Greedy: pass draft and base_tokens [N, n]; probabilistic: pass logp_prefix, logp_base, uniform [N, n]."""
    ref = base_tokens if base_tokens is not None else logp_prefix
    N, n = ref.shape
    accepted = torch.empty(N, dtype=torch.int32, device=ref.device)
    rc = load_library().cpmtp_verify_draft(N, n, _ptr(draft), _ptr(base_tokens), _ptr(logp_prefix), _ptr(logp_base),
                                           _ptr(uniform), _ptr(accepted), _stream())
    _check(rc)
    return accepted


def score_draft_static(h, W_head, E, W_g, draft, *, want_prefix: bool = True,
                       dev_status: Optional[torch.Tensor] = None, out: Optional[dict] = None) -> dict:
    """cpmtp_score_draft_static: draft scoring for callers that cannot provide scratch memory.

    Same results as score_draft, but the library's built-in fixed scratch array is used instead
    of a workspace, so no device memory is requested from anyone; the output tensors are the
    only thing this wrapper creates, and only when `out` does not already hold them.  Shapes
    needing more than STATIC_SCRATCH_BYTES raise CpmtpError (code -7).  Calls share the array:
    do not let two of them overlap on the GPU.
    """
    lib = load_library()
    shape = _shape_of(h, W_head, E, W_g, draft, None)
    res = out if out is not None else {}
    if "logp_joint" not in res:
        res["logp_joint"] = torch.empty(shape.N, dtype=torch.float32, device=h.device)
    if want_prefix and "logp_prefix" not in res:
        res["logp_prefix"] = torch.empty((shape.N, shape.n), dtype=torch.float32, device=h.device)
    rc = lib.cpmtp_score_draft_static(ctypes.byref(shape), _ptr(h), _ptr(W_head), _ptr(E), _ptr(W_g), _ptr(draft),
                                      _ptr(res["logp_joint"]), _ptr(res.get("logp_prefix")) if want_prefix else None,
                                      _ptr(dev_status), _stream())
    _check(rc)
    return res


def forward_host(h_host, W_head, E, W_g, x_host, logp_host, loss_host, *, aux_coef: Optional[float] = None,
                 saved: Optional[Saved] = None, workspace: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None) -> None:
    """cpmtp_forward_host: h_host / x_host / logp_host / loss_host are (pinned) CPU tensors; weights on device.
    Asynchronous: synchronise the current stream before reading the host outputs."""
    lib = load_library()
    N, d = h_host.shape
    shape = make_shape(N, d, E.shape[0], x_host.shape[1], W_g.shape[0], aux_coef)
    need = workspace_bytes(shape, OP_FORWARD) + host_staging_bytes(shape) + 256
    if workspace is None:
        workspace = alloc_workspace(need, E.device)
    cs = saved.c_struct() if saved is not None else None
    rc = lib.cpmtp_forward_host(ctypes.byref(shape), _ptr(h_host), _ptr(W_head), _ptr(E), _ptr(W_g), _ptr(x_host),
                                _ptr(logp_host), _ptr(loss_host), ctypes.byref(cs) if cs is not None else None,
                                _ptr(workspace), workspace.numel(),
                                _ptr(dev_status), _stream())
    _check(rc)


@dataclass
class DistillSaved:
    """Results of cpmtp_distill_forward kept for cpmtp_distill_backward (device tensors); `kl` is also
    the entry point's output, KL(p^d_k, p^c_k) per (position, token)."""
    lse_t: torch.Tensor
    logpi: torch.Tensor
    pm: torch.Tensor
    kl: torch.Tensor

    @staticmethod
    def alloc(shape: CShape, device="cuda") -> "DistillSaved":
        f = dict(dtype=torch.float32, device=device)
        K = shape.n * shape.r
        return DistillSaved(lse_t=torch.empty((shape.N, shape.n), **f), logpi=torch.empty((shape.N, K), **f),
                            pm=torch.empty((shape.N, K), **f), kl=torch.empty((shape.N, shape.n), **f))

    def c_struct(self) -> CDistillSaved:
        return CDistillSaved(self.lse_t.data_ptr(), self.logpi.data_ptr(), self.pm.data_ptr(), self.kl.data_ptr())


def _check_teacher(teacher, shape: CShape) -> None:
    assert teacher.shape == (shape.N, shape.n, shape.V) and teacher.dtype == torch.bfloat16 and teacher.is_contiguous()


def distill_forward(h, W_head, E, W_g, x, teacher, saved: Saved, dsaved: DistillSaved, *, beta: float = 0.9,
                    gamma: float = 1.0, aux_coef: Optional[float] = None, want_loss: bool = True,
                    workspace: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None,
                    out: Optional[dict] = None, recompute_z: bool = False) -> dict:
    """cpmtp_distill_forward; returns {"logp", "logp_prefix", "kl", "loss"} (device tensors; kl is dsaved.kl)."""
    lib = load_library()
    shape = _shape_of(h, W_head, E, W_g, x, aux_coef)
    _check_teacher(teacher, shape)
    if recompute_z:
        shape.flags |= FLAG_RECOMPUTE_Z
    dev = h.device
    if workspace is None:
        workspace = alloc_workspace(workspace_bytes(shape, OP_DISTILL_FORWARD), dev)
    res = out if out is not None else {}
    res.setdefault("logp", torch.empty(shape.N, dtype=torch.float32, device=dev))
    res.setdefault("logp_prefix", torch.empty((shape.N, shape.n), dtype=torch.float32, device=dev))
    if want_loss:
        res.setdefault("loss", torch.empty(1, dtype=torch.float32, device=dev))
    res["kl"] = dsaved.kl
    cs, ds = saved.c_struct(), dsaved.c_struct()
    rc = lib.cpmtp_distill_forward(ctypes.byref(shape), _ptr(h), _ptr(W_head), _ptr(E), _ptr(W_g), _ptr(x),
                                   _ptr(teacher), ctypes.c_float(beta), ctypes.c_float(gamma), _ptr(res["logp"]),
                                   _ptr(res["logp_prefix"]), _ptr(res.get("loss")) if want_loss else None,
                                   ctypes.byref(cs), ctypes.byref(ds), _ptr(workspace), workspace.numel(),
                                   _ptr(dev_status), _stream())
    _check(rc)
    return res


def distill_backward(h, W_head, E, W_g, x, teacher, saved: Saved, dsaved: DistillSaved, *, beta: float = 0.9,
                     gamma: float = 1.0, aux_coef: Optional[float] = None,
                     dloss_dprefix: Optional[torch.Tensor] = None, dloss_dkl: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None,
                     out: Optional[dict] = None, skip: tuple = (), recompute_z: bool = False,
                     accumulate: bool = False) -> dict:
    """cpmtp_distill_backward; returns {"dh", "dW_head", "dE", "dW_g"} (bf16 device tensors)."""
    lib = load_library()
    shape = _shape_of(h, W_head, E, W_g, x, aux_coef)
    _check_teacher(teacher, shape)
    if recompute_z:
        shape.flags |= FLAG_RECOMPUTE_Z
    if accumulate:
        assert out is not None, "accumulation needs the tensors to add to"
        shape.flags |= FLAG_ACCUM_GRADS
    for w in (dloss_dprefix, dloss_dkl):
        assert w is None or (w.shape == (shape.N, shape.n) and w.dtype == torch.float32 and w.is_contiguous())
    if workspace is None:
        workspace = alloc_workspace(workspace_bytes(shape, OP_DISTILL_BACKWARD), h.device)
    res = out if out is not None else {}
    for name, ref in (("dh", h), ("dW_head", W_head), ("dE", E), ("dW_g", W_g)):
        if name not in res and name not in skip:
            res[name] = torch.empty_like(ref)
    cs, ds = saved.c_struct(), dsaved.c_struct()
    rc = lib.cpmtp_distill_backward(ctypes.byref(shape), _ptr(h), _ptr(W_head), _ptr(E), _ptr(W_g), _ptr(x),
                                    _ptr(teacher), ctypes.byref(cs), ctypes.byref(ds), ctypes.c_float(beta),
                                    ctypes.c_float(gamma), _ptr(dloss_dprefix), _ptr(dloss_dkl), _ptr(res.get("dh")),
                                    _ptr(res.get("dW_head")), _ptr(res.get("dE")), _ptr(res.get("dW_g")),
                                    _ptr(workspace), workspace.numel(), _ptr(dev_status), _stream())
    _check(rc)
    return res


# ---------------------------------------------------------------------------------------------------------------
# Around the head in a training step: embedding lookup, norms with gate and residual addition, AdamW.

_TYPES = {torch.bfloat16: BF16, torch.float32: F32}
_dtype_of = operator.attrgetter("dtype")
_address_of, _size_of, _device_of, _contiguous = torch.Tensor.data_ptr, torch.Tensor.numel, torch.Tensor.get_device, torch.Tensor.is_contiguous
_ADAMW_WORDS = ctypes.sizeof(CAdamWTensor) // 8      # a descriptor in 8-byte words: param, grad, master, m, v, m_exp, v_exp, numel, types, factors


# The checks below run before every launch and cost a few hundred nanoseconds each, so they test first and put the
# message together only when there is something to say.

def _need(ok: bool, what: str) -> None:
    if not ok:
        raise CpmtpError(f"cpmtp: {what}")


def _device(ref: torch.Tensor) -> int:
    """Index of `ref`'s device, which has to be the current one: its current stream is used."""
    dev = ref.get_device()
    if dev < 0 or dev != torch.cuda.current_device():
        raise CpmtpError("cpmtp: tensors must be on the current CUDA device")
    return dev


def _raw_stream(dev: int) -> int:
    return torch._C._cuda_getCurrentRawStream(dev)


def _rows(t: torch.Tensor, size: tuple, dtype, dev: int, name: str) -> tuple:
    """(pointer, row stride) of a matrix [n, d] = size whose rows are contiguous and do not overlap."""
    if t.shape != size or t.dtype is not dtype:
        raise CpmtpError(f"cpmtp: {name} must be {list(size)} {dtype}, not {list(t.shape)} {t.dtype}")
    if t.get_device() != dev:
        raise CpmtpError(f"cpmtp: {name} is on another device")
    ld, one = t.stride()
    n, d = size
    if n <= 1:
        ld = d
    if (one != 1 and d > 1) or ld < d:
        raise CpmtpError(f"cpmtp: {name}: the elements of a row must be contiguous and rows must not overlap")
    return t.data_ptr(), ld


def _vector(t: torch.Tensor, n: int, dtype, dev: int, name: str) -> int:
    if t.shape != (n,) or t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous():
        raise CpmtpError(f"cpmtp: {name} must be a contiguous [{n}] {dtype} on the same device")
    return t.data_ptr()


def _int32(t: torch.Tensor, dev: int, name: str) -> int:
    if t.dtype is not torch.int32 or t.get_device() != dev or not t.is_contiguous():
        raise CpmtpError(f"cpmtp: {name} must be contiguous int32 on the same device")
    return t.data_ptr()


def _workspace(t: torch.Tensor, dev: int) -> tuple:
    if t.dtype is not torch.uint8 or t.get_device() != dev or not t.is_contiguous():
        raise CpmtpError("cpmtp: workspace must be contiguous uint8 on the same device")
    return t.data_ptr(), t.numel()


def embed_forward(E: torch.Tensor, x: torch.Tensor, *, scale: float = 1.0, out_dtype: torch.dtype = torch.bfloat16,
                  out: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """cpmtp_embed_forward: scale * E[x] for tokens x (any shape, int32, EMBED_PAD = a row of zeros); E [V, d] bf16.
    Returns x.shape + (d,) of `out_dtype` (bf16 or fp32), or `out` ([x.numel(), d], rows may be strided)."""
    dev = _device(E)
    size = E.shape
    _need(len(size) == 2, "E must be [V, d]")
    V, d = size
    T = x.numel()
    px = _int32(x, dev, "x")
    if out is None:
        _need(out_dtype in _TYPES, "out_dtype must be bfloat16 or float32")
        out = torch.empty((*x.shape, d), dtype=out_dtype, device=E.device)
        po, ldo = out.data_ptr(), d
    else:
        out_dtype = out.dtype
        _need(out_dtype in _TYPES, "out must be bfloat16 or float32")
        po, ldo = _rows(out, (T, d), out_dtype, dev, "out")
    pe, lde = _rows(E, size, torch.bfloat16, dev, "E")
    shape = CEmbedShape(T, V, d, _TYPES[out_dtype], lde, ldo, scale, 0)
    rc = load_library().cpmtp_embed_forward(ctypes.byref(shape), pe, px, po, None if dev_status is None else _int32(dev_status, dev, "dev_status"),
                                            _raw_stream(dev))
    if rc:
        _check(rc)
    return out


def embed_backward(dy: torch.Tensor, x: torch.Tensor, V: int, *, scale: float = 1.0, out: Optional[torch.Tensor] = None,
                   accumulate: bool = False, workspace: Optional[torch.Tensor] = None,
                   dev_status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """cpmtp_embed_backward: dE [V, d] bf16, the scaled sums of the rows of dy (x.shape + (d,), bf16 or fp32; a 2-D dy may
    have strided rows) over equal tokens.  accumulate: add to `out`, touching only the rows that occur."""
    dev = _device(dy)
    _need(dy.dim() > 0, "dy must be x.shape + (d,)")
    T, d = x.numel(), dy.shape[-1]
    px = _int32(x, dev, "x")
    dtype = dy.dtype
    _need(dtype in _TYPES, "dy must be bfloat16 or float32")
    if dy.dim() != 2:
        _need(dy.shape[:-1] == x.shape and dy.is_contiguous(), "dy must be x.shape + (d,)")
        dy = dy.view(T, d)
    pd, ldd = _rows(dy, (T, d), dtype, dev, "dy")
    if out is None:
        _need(not accumulate, "accumulation needs the tensor to add to")
        _need(V >= 1, "V must be at least 1")
        out = torch.empty((V, d), dtype=torch.bfloat16, device=dy.device)
    pe, lde = _rows(out, (V, d), torch.bfloat16, dev, "out")
    shape = CEmbedShape(T, V, d, _TYPES[dtype], lde, ldd, scale, FLAG_ACCUM_GRADS if accumulate else 0)
    lib, ref = load_library(), ctypes.byref(shape)
    if workspace is None:
        workspace = alloc_workspace(lib.cpmtp_embed_workspace_bytes(ref), dy.device)
    pw, nw = _workspace(workspace, dev)
    rc = lib.cpmtp_embed_backward(ref, pd, px, pe, pw, nw, None if dev_status is None else _int32(dev_status, dev, "dev_status"), _raw_stream(dev))
    if rc:
        _check(rc)
    return out


def embed_workspace_bytes(T: int, V: int, d: int) -> int:
    """Scratch bytes of embed_backward for T tokens and a [V, d] table."""
    shape = CEmbedShape(T, V, d, BF16, d, d, 1.0, 0)
    return int(load_library().cpmtp_embed_workspace_bytes(ctypes.byref(shape)))


def _empty(size, dtype, like: torch.Tensor) -> torch.Tensor:
    """A new contiguous tensor on like's device; a contiguous one of that size and type is the cheapest thing to copy from."""
    if like.dtype is dtype and like.shape == size and like.is_contiguous():
        return torch.empty_like(like)
    return torch.empty(size, dtype=dtype, device=like.device)


def _row_gate(t: torch.Tensor, n: int, dev: int, name: str) -> tuple:
    if t.shape != (n,) or t.dtype is not torch.bfloat16 or t.get_device() != dev or (n > 1 and t.stride(0) < 1):
        raise CpmtpError(f"cpmtp: {name} must be [{n}] bfloat16, or have the rows' shape")
    return t.data_ptr(), t.stride(0) if n > 1 else 1


def _norm_args(ref, dev, w_pre, block, gate, w_post, res_scale, eps) -> tuple:
    """The arguments that both directions share, and the rows' shape; `ref` is x or x_out."""
    size, dtype = ref.shape, ref.dtype
    _need(len(size) == 2 and dtype in _TYPES, "the residual stream must be [N, d] bfloat16 or float32")
    N, d = size
    a = CNormArgs(N, d, _TYPES[dtype], GATE_NONE, 0, eps, res_scale)
    bf16 = torch.bfloat16
    if w_pre is not None:
        a.w_pre = _vector(w_pre, d, bf16, dev, "w_pre")
    if w_post is not None:
        a.w_post = _vector(w_post, d, bf16, dev, "w_post")
    if block is not None:
        a.block, a.ld_block = _rows(block, size, bf16, dev, "block")
    if gate is not None:
        if gate.dim() == 1:
            a.gate_kind = GATE_ROW
            a.gate, a.ld_gate = _row_gate(gate, N, dev, "gate")
        else:
            a.gate_kind = GATE_CHANNEL
            a.gate, a.ld_gate = _rows(gate, size, bf16, dev, "gate")
    return a, size, dtype


def norm_forward(x: torch.Tensor, w_pre: Optional[torch.Tensor] = None, *, block: Optional[torch.Tensor] = None,
                 gate: Optional[torch.Tensor] = None, w_post: Optional[torch.Tensor] = None, res_scale: float = 1.0,
                 eps: float = 1e-6, out: Optional[dict] = None) -> dict:
    """cpmtp_norm_forward: x_out = res_scale * x + sigmoid(gate) * rmsnorm(block, w_post), y = rmsnorm(x_out, w_pre).
    x [N, d] bf16 or fp32; block and gate ([N, d], or one logit per row [N]) bf16, rows may be strided (the halves of one
    projection's output).  Without w_post the block is added as it is, without w_pre there is no y, without a block
    x_out is x itself and y its norm.  Returns {"x_out", "y", "rstd_post", "rstd_pre"} (None where there is none);
    tensors given in `out` are written instead of new ones (x_out may be x), the dictionary itself is left as it is."""
    dev = _device(x)
    a, size, dtype = _norm_args(x, dev, w_pre, block, gate, w_post, res_scale, eps)
    a.x, a.ld_x = _rows(x, size, dtype, dev, "x")
    N = size[0]
    given, res = {} if out is None else out, {}
    device, d = x.device, size[1]
    if block is None:
        res["x_out"] = x
    elif (t := given.get("x_out")) is None:
        t = res["x_out"] = _empty(size, dtype, x)
        a.x_out, a.ld_x_out = t.data_ptr(), d
    else:
        res["x_out"] = t
        a.x_out, a.ld_x_out = _rows(t, size, dtype, dev, "x_out")
    if w_pre is None:
        res["y"] = res["rstd_pre"] = None
    else:
        if (t := given.get("y")) is None:
            t = res["y"] = _empty(size, torch.bfloat16, x)
            a.y, a.ld_y = t.data_ptr(), d
        else:
            res["y"] = t
            a.y, a.ld_y = _rows(t, size, torch.bfloat16, dev, "y")
        if (t := given.get("rstd_pre")) is None:
            t = res["rstd_pre"] = torch.empty(N, dtype=torch.float32, device=device)
            a.rstd_pre = t.data_ptr()
        else:
            res["rstd_pre"] = t
            a.rstd_pre = _vector(t, N, torch.float32, dev, "rstd_pre")
    if w_post is None:
        res["rstd_post"] = None
    elif (t := given.get("rstd_post")) is None:
        t = res["rstd_post"] = torch.empty(N, dtype=torch.float32, device=device)
        a.rstd_post = t.data_ptr()
    else:
        res["rstd_post"] = t
        a.rstd_post = _vector(t, N, torch.float32, dev, "rstd_post")
    rc = load_library().cpmtp_norm_forward(ctypes.byref(a), _raw_stream(dev))
    if rc:
        _check(rc)
    return res


def norm_backward(dy: Optional[torch.Tensor], x_out: torch.Tensor, w_pre: Optional[torch.Tensor] = None,
                  rstd_pre: Optional[torch.Tensor] = None, *, dx_out: Optional[torch.Tensor] = None,
                  block: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                  w_post: Optional[torch.Tensor] = None, rstd_post: Optional[torch.Tensor] = None, res_scale: float = 1.0,
                  eps: float = 1e-6, out: Optional[dict] = None, skip: tuple = (), accumulate: bool = False,
                  workspace: Optional[torch.Tensor] = None) -> dict:
    """cpmtp_norm_backward; x_out, rstd_pre and rstd_post as norm_forward returned them, the other inputs as it was given.
    dy [N, d] bf16 (None: no gradient of y), dx_out [N, d] of the stream's type (None: zero).
    Returns {"dx", "dblock", "dgate", "dw_post", "dw_pre"}: None where there is nothing to differentiate or the name is
    in `skip`.  accumulate: dw_post and dw_pre are added to those given in `out`, which itself is left as it is."""
    dev = _device(x_out)
    a, size, dtype = _norm_args(x_out, dev, w_pre, block, gate, w_post, res_scale, eps)
    N, d = size
    bf16, device = torch.bfloat16, x_out.device
    _need(dy is not None or dx_out is not None, "no gradient comes in: dy and dx_out are both None")
    _need(not accumulate or out is not None, "accumulation needs the tensors to add to")
    a.x_out, a.ld_x_out = _rows(x_out, size, dtype, dev, "x_out")
    if dy is not None:
        _need(w_pre is not None and rstd_pre is not None, "dy needs w_pre and rstd_pre")
        a.dy, a.ld_dy = _rows(dy, size, bf16, dev, "dy")
        a.rstd_pre = _vector(rstd_pre, N, torch.float32, dev, "rstd_pre")
    if dx_out is not None:
        a.dx_out, a.ld_dx_out = _rows(dx_out, size, dtype, dev, "dx_out")
    if w_post is not None:
        _need(rstd_post is not None, "w_post needs rstd_post")
        a.rstd_post = _vector(rstd_post, N, torch.float32, dev, "rstd_post")
    given, res = {} if out is None else out, {}

    # outputs: not there or not wanted, given, or new ones, which need no check
    if "dx" in skip:
        res["dx"] = None
    elif (t := given.get("dx")) is None:
        t = res["dx"] = _empty(size, dtype, x_out)
        a.dx, a.ld_dx = t.data_ptr(), d
    else:
        res["dx"] = t
        a.dx, a.ld_dx = _rows(t, size, dtype, dev, "dx")
    if block is None or "dblock" in skip:
        res["dblock"] = None
    elif (t := given.get("dblock")) is None:
        t = res["dblock"] = _empty(size, bf16, x_out if dy is None else dy)
        a.dblock, a.ld_dblock = t.data_ptr(), d
    else:
        res["dblock"] = t
        a.dblock, a.ld_dblock = _rows(t, size, bf16, dev, "dblock")
    if gate is None or "dgate" in skip:
        res["dgate"] = None
    elif (t := given.get("dgate")) is None:
        t = res["dgate"] = _empty(gate.shape, bf16, x_out if dy is None else dy)
        a.dgate, a.ld_dgate = t.data_ptr(), d if a.gate_kind == GATE_CHANNEL else 1
    else:
        res["dgate"] = t
        a.dgate, a.ld_dgate = _rows(t, size, bf16, dev, "dgate") if a.gate_kind == GATE_CHANNEL else _row_gate(t, N, dev, "dgate")
    for name, there in (("dw_post", w_post is not None), ("dw_pre", dy is not None)):
        if not there or name in skip:
            res[name] = None
        elif (t := given.get(name)) is None:
            _need(not accumulate, "accumulation needs dw_post and dw_pre in out")
            t = res[name] = torch.empty(d, dtype=bf16, device=device)
            setattr(a, name, t.data_ptr())
        else:
            res[name] = t
            setattr(a, name, _vector(t, d, bf16, dev, name))
    if accumulate:
        a.flags = FLAG_ACCUM_GRADS
    lib, ref = load_library(), ctypes.byref(a)
    if workspace is None:
        workspace = alloc_workspace(lib.cpmtp_norm_workspace_bytes(ref), device)
    pw, nw = _workspace(workspace, dev)
    rc = lib.cpmtp_norm_backward(ref, pw, nw, _raw_stream(dev))
    if rc:
        _check(rc)
    return res


def norm_workspace_bytes(N: int, d: int) -> int:
    """Scratch bytes of norm_backward for [N, d]."""
    a = CNormArgs(N, d, BF16, GATE_NONE, 0, 1e-6, 1.0)
    a.w_pre = 256
    return int(load_library().cpmtp_norm_workspace_bytes(ctypes.byref(a)))


def _spread(values, where: list, n: int) -> list:
    """n zeros, and the values at their places."""
    full = [0] * n
    for i, v in zip(where, values):
        full[i] = v
    return full


class _Descriptors:
    """An array of cpmtp_adamw_tensor, written a column at a time (a step updates hundreds of them before its one launch)."""

    def __init__(self, n: int):
        self.n = n
        self.words = array("q", bytes(8 * _ADAMW_WORDS * n))
        self.address = self.words.buffer_info()[0]
        self.grad_kind = None              # the gradients' common type as it stands in the words, if they have one

    def put(self, word: int, values) -> None:
        if self.n:
            self.words[word::_ADAMW_WORDS] = array("q", values)

    def put_grads(self, grads, dev: int, param_types: Optional[list] = None, numels: Optional[list] = None) -> None:
        """Addresses, sizes and types of the gradients, one per parameter of `numels` elements; None: no address."""
        # one property of all of them at a time: half the cost of a loop over the tensors
        there, where = grads, None
        try:
            kinds = list(map(_dtype_of, there))
        except AttributeError:                             # (None has no type)
            where = [i for i, g in enumerate(grads) if g is not None]
            there = [grads[i] for i in where]
            kinds = list(map(_dtype_of, there))
        if there:
            same = kinds.count(kinds[0]) == len(kinds)
            ok = kinds[0] in _TYPES if same else all(k in _TYPES for k in kinds)
            devices = list(map(_device_of, there))
            if not ok or devices.count(dev) != len(devices) or not all(map(_contiguous, there)):
                raise CpmtpError("cpmtp: gradients must be contiguous bfloat16 or float32 tensors on the current CUDA device")
            kind = _TYPES[kinds[0]] << 32
        else:
            kind, same = 0, True
        at, sizes, n = list(map(_address_of, there)), list(map(_size_of, there)), len(grads)
        if numels is not None and sizes != (numels if where is None else [numels[i] for i in where]):
            raise CpmtpError("cpmtp: a gradient must have its parameter's size")
        if numels is None:
            self.put(7, sizes if where is None else _spread(sizes, where, n))
        self.put(1, at if where is None else _spread(at, where, n))
        if not same or kind != self.grad_kind:             # (the types seldom change from step to step)
            types = [_TYPES[k] << 32 for k in kinds] if not same else [kind] * n     # (a missing gradient's type does not matter)
            if not same and where is not None:
                types = _spread(types, where, n)
            self.put(8, types if param_types is None else map(operator.or_, types, param_types))
            self.grad_kind = kind if same else None


def _grad_descriptors(grads) -> tuple:
    ref = next((g for g in grads if g is not None), None)
    _need(ref is not None, "there is no gradient")
    dev = _device(ref)
    table = _Descriptors(len(grads))
    table.put_grads(grads, dev)
    return table, dev, ref.device


def grad_norm_workspace_bytes(grads) -> int:
    """Scratch bytes of grad_norm for these gradients."""
    table, _, _ = _grad_descriptors(grads)
    return int(load_library().cpmtp_grad_norm_workspace_bytes(table.address, table.n))


def grad_norm(grads, *, max_norm: float = float("inf"), workspace: Optional[torch.Tensor] = None, out: Optional[dict] = None) -> dict:
    """cpmtp_grad_norm over a list of gradients (None entries are left out): {"norm", "coef"}, fp32 [1] on the device; coef
    is what AdamW.step takes to clip to max_norm (NaN where the norm is not finite, which skips the step)."""
    table, dev, device = _grad_descriptors(grads)
    lib = load_library()
    if workspace is None:
        workspace = alloc_workspace(lib.cpmtp_grad_norm_workspace_bytes(table.address, table.n), device)
    pw, nw = _workspace(workspace, dev)
    res = {} if out is None else out
    for name in ("norm", "coef"):
        if res.get(name) is None:
            res[name] = torch.empty(1, dtype=torch.float32, device=device)
    rc = lib.cpmtp_grad_norm(table.address, table.n, max_norm, _vector(res["norm"], 1, torch.float32, dev, "norm"),
                             _vector(res["coef"], 1, torch.float32, dev, "coef"), pw, nw, _raw_stream(dev))
    if rc:
        _check(rc)
    return res


def _state_column(name: str):
    """An attribute of AdamW: aliases of the state tensors, in a tuple; assigning to it replaces them all."""

    def read(self) -> tuple:
        return tuple(None if t is None else t.detach() for t in self._states[name])

    def write(self, tensors) -> None:
        # Aliases, too: other memory given to the caller's tensors changes nothing here, and this memory stays
        try:
            self._states[name] = [None if t is None else t.detach() for t in tensors]
        except AttributeError:
            raise CpmtpError(f"cpmtp: {name} takes a list of tensors") from None
        self._at = None                    # the descriptors are out of date

    return property(read, write)


def _same_kind(tensors, dtype, sizes: list, dev: int) -> bool:
    """Whether these are contiguous tensors of one type, of the given sizes, on the device."""
    try:
        return (list(map(_size_of, tensors)) == sizes and {dtype} >= set(map(_dtype_of, tensors)) and {dev} >= set(map(_device_of, tensors))
                and all(map(_contiguous, tensors)))
    except TypeError:                      # (None among them)
        return False


class StepClock:
    """Step number, learning rate and seed on the device (cpmtp_adamw_clock), for optimiser steps that are captured in a CUDA graph: every
    replay is the next step.  `step` (int64 [1], of the last step taken) and `lr` (float64 [1]) are views to read, and to write between steps
    in the stream's order, as a schedule does (`clock.lr.fill_(...)`)."""

    def __init__(self, lr: float, *, step: int = 0, seed: int = 0, device="cuda"):
        _need(step >= 0 and 0.0 <= lr < float("inf"), "a clock's step and learning rate are finite and not negative")
        block = CAdamWClock(step=step, lr=lr, seed=seed & 0xFFFFFFFF)
        self.block = torch.frombuffer(bytearray(block), dtype=torch.uint8).to(device)
        self.step, self.lr = self.block[:8].view(torch.int64), self.block[8:16].view(torch.float64)


class AdamW:
    """Parameters and their optimiser states, stepped by cpmtp_adamw_step in one launch per 300 tensors.

    params: contiguous bf16 or fp32 tensors, each once, updated in place.  bits: 32 (fp32 moments) or 8 (one byte per element and
    one exponent byte per ADAMW_BLOCK elements).  master: True for fp32 copies of the bf16 parameters, or a list of
    them (None entries: none); without one a bf16 parameter is rounded stochastically.  lr_scale, decay_scale: factors per
    tensor.  state: {"m", "v"[, "m_exp", "v_exp"]}, lists of tensors of an earlier run, all of them; new states are zero.

    The list `params` and its tensors' memory may change between steps (`p.data = other`): every step compares their addresses
    and sizes with those it knows, and on a difference checks all tensors again as at first.  Memory that was replaced is held until
    then.  The states `m`, `v`, `m_exp`, `v_exp` and `master` are the memory that was given or made at first: read as tuples of
    aliases, written in place, or replaced by assigning a whole list (`opt.m = tensors`); their storages are not to be resized."""

    m, v, m_exp, v_exp, master = map(_state_column, ("m", "v", "m_exp", "v_exp", "master"))

    def __init__(self, params, *, bits: int = 32, master=False, lr_scale=None, decay_scale=None, state: Optional[dict] = None):
        self.params = list(params)
        n = len(self.params)
        _need(bits in (32, 8), "bits must be 32 or 8")
        self.bits = bits
        for name, given in (("lr_scale", lr_scale), ("decay_scale", decay_scale)):
            _need(given is None or len(given) == n, f"{name} needs one entry per parameter")
        ones = [1.0] * n
        self._factors = [struct.unpack("q", struct.pack("ff", a, b))[0] for a, b in zip(lr_scale or ones, decay_scale or ones)]
        self._check_params()
        if master is True:
            master = [p.float() if p.dtype == torch.bfloat16 else None for p in self.params]
        self._states = {}
        self.master = list(master) if master else [None] * n
        expected = self._expected()
        known = [k for k in expected if state is not None and state.get(k) is not None]
        _need(len(known) in (0, len(expected)), f"a state has {', '.join(expected)}: all of them are needed")
        for name, (dtype, sizes) in expected.items():
            given = state[name] if known else None
            setattr(self, name, [torch.zeros(k, dtype=dtype, device=p.device) for k, p in zip(sizes, self.params)] if given is None else given)
        if bits == 32:
            self.m_exp = self.v_exp = [None] * n
        self._bind()

    def _check_params(self) -> int:
        """Index of the parameters' device."""
        dev = _device(self.params[0]) if self.params else -1
        if not (_TYPES.keys() >= set(map(_dtype_of, self.params)) and all(map(_contiguous, self.params)) and {dev} >= set(map(_device_of, self.params))):
            raise CpmtpError("cpmtp: parameters must be contiguous bfloat16 or float32 tensors on one CUDA device")
        return dev

    def _expected(self) -> dict:
        """Type and lengths of the moments, by name."""
        sizes = [p.numel() for p in self.params]
        if self.bits == 32:
            return dict(m=(torch.float32, sizes), v=(torch.float32, sizes))
        blocks = [-(-k // ADAMW_BLOCK) for k in sizes]
        return dict(m=(torch.uint8, sizes), v=(torch.uint8, sizes), m_exp=(torch.uint8, blocks), v_exp=(torch.uint8, blocks))

    def _bind(self) -> None:
        """Checks all tensors and writes them into the descriptors.  The parameters' memory, too, is held by aliases from here on: as
        no other tensor can then come to lie at their addresses, comparing those is enough to notice a change."""
        dev, n, states = self._check_params(), len(self.params), self._states
        _need(len(self._factors) == n, "the number of parameters has changed")
        _need(len(states["master"]) == n, "master needs one entry per parameter")
        held = [p.detach() for p in self.params]
        masters = [(w, p) for w, p in zip(states["master"], held) if w is not None]
        if not (_same_kind([w for w, _ in masters], torch.float32, [p.numel() for _, p in masters], dev)
                and all(p.dtype is torch.bfloat16 for _, p in masters)):
            raise CpmtpError("cpmtp: a master copy is a contiguous float32 tensor of a bfloat16 parameter's size")
        written = held + [w for w, _ in masters]
        for name, (dtype, sizes) in self._expected().items():
            if len(states[name]) != n or not _same_kind(states[name], dtype, sizes, dev):
                raise CpmtpError(f"cpmtp: {name} must be a contiguous {dtype} tensor per parameter, of its size"
                                 + (f" in blocks of {ADAMW_BLOCK}" if name.endswith("exp") else ""))
            written += states[name]
        at = list(map(_address_of, written))
        spans = sorted((a, a + t.nbytes) for a, t in zip(at, written) if t.nbytes > 0)
        _need(all(a[1] <= b[0] for a, b in zip(spans, spans[1:])), "a tensor that a step writes is there twice, or overlaps another")
        table = _Descriptors(n)
        for word, tensors in ((0, held), (2, states["master"]), (3, states["m"]), (4, states["v"]), (5, states["m_exp"]), (6, states["v_exp"])):
            table.put(word, [0 if t is None else t.data_ptr() for t in tensors])
        self._numels, self._types = list(map(_size_of, held)), [_TYPES[k] for k in map(_dtype_of, held)]
        table.put(7, self._numels)
        table.put(9, self._factors)
        self._table, self._held, self._at = table, held, at[:n]

    def step(self, grads, t, *, lr: Optional[float] = None, betas: tuple = (0.9, 0.95), eps: float = 1e-8, weight_decay: float = 0.1,
             coef: Optional[torch.Tensor] = None, seed: int = 0) -> None:
        """Step t (1 for the first) with one gradient per parameter (bf16 or fp32, contiguous; None leaves a parameter alone).
        coef: fp32 [1] on the device that multiplies the gradients (grad_norm's), or None.
        t may be a StepClock, which has the learning rate and the seed as well.  A step that is captured for replaying needs one: with a
        number, each replay would be that step again, with the same bias corrections and rounding noise.  (What a graph has captured goes
        on writing to the memory that the parameters had then.)"""
        n = len(self.params)
        _need(len(grads) == n, "one gradient per parameter")
        if n == 0:
            return
        dev = _device(self.params[0])
        if list(map(_address_of, self.params)) != self._at or list(map(_size_of, self.params)) != self._numels:
            self._bind()
        self._table.put_grads(grads, dev, self._types, self._numels)
        clock = t if isinstance(t, StepClock) else None
        _need((lr is None) == (clock is not None), "a learning rate is needed, here or in the clock")
        _need(clock is None or seed == 0, "the seed is the clock's")
        hyper = CAdamWHyper(0.0 if clock else lr, betas[0], betas[1], eps, weight_decay, 1 if clock else t, seed & 0xFFFFFFFF, self.bits,
                            None if coef is None else _vector(coef, 1, torch.float32, dev, "coef"))
        if clock is None:
            rc = load_library().cpmtp_adamw_step(self._table.address, n, ctypes.byref(hyper), _raw_stream(dev))
        else:
            at = _vector(clock.block, ctypes.sizeof(CAdamWClock), torch.uint8, dev, "the clock")
            rc = load_library().cpmtp_adamw_step_clocked(self._table.address, n, ctypes.byref(hyper), at, _raw_stream(dev))
        if rc:
            _check(rc)


def adamw_state_values(codes: torch.Tensor, exps: torch.Tensor, *, second: bool, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """cpmtp_adamw_state_values: the values of an 8-bit moment (second: v, else m) as bf16, exactly."""
    dev = _device(codes)
    n = codes.numel()
    if codes.dtype is not torch.uint8 or not codes.is_contiguous():
        raise CpmtpError("cpmtp: codes must be contiguous uint8")
    if exps.dtype is not torch.uint8 or exps.numel() != -(-n // ADAMW_BLOCK) or exps.get_device() != dev or not exps.is_contiguous():
        raise CpmtpError(f"cpmtp: exps must be {-(-n // ADAMW_BLOCK)} contiguous bytes on the same device")
    if out is None:
        out = torch.empty_like(codes, dtype=torch.bfloat16)
    elif out.dtype is not torch.bfloat16 or out.numel() != n or out.get_device() != dev or not out.is_contiguous():
        raise CpmtpError(f"cpmtp: out must be {n} contiguous bfloat16 on the same device")
    rc = load_library().cpmtp_adamw_state_values(codes.data_ptr(), exps.data_ptr(), n, 1 if second else 0, out.data_ptr(), _raw_stream(dev))
    if rc:
        _check(rc)
    return out


# ---------------------------------------------------------------------------------------------------------------
# The base model's pass over a draft: paged cache of keys and values, attention over it, sampling from logits.

class PagedCache:
    """Keys and values of many sequences in pages, as the cache_* functions take them.

    k, v: [pages, page_slots, H, D] bf16 with any strides that keep rows of D contiguous (a cache kept as [pages, H, page_slots, D] is
    passed as its transpose(1, 2)); acc: [pages, H, page_slots] fp32, the attention weight that each slot has received, or None.
    The object holds the tensors, so that their memory stays theirs."""

    __slots__ = ("k", "v", "acc", "device", "_dev", "_c", "_plain")

    def __init__(self, k: torch.Tensor, v: torch.Tensor, acc: Optional[torch.Tensor] = None):
        _need(k.dim() == 4 and k.dtype is torch.bfloat16, "k must be [pages, page_slots, H, D] bfloat16")
        _need(v.shape == k.shape and v.dtype is torch.bfloat16, "v must have k's shape and type")
        dev = k.get_device()
        _need(v.get_device() == dev, "v is on another device")
        P, S, H, D = k.shape
        _need(min(P, S, H, D) > 0, "a cache has one page, slot, head and column at least")
        _need(S % 8 == 0 and S <= 65536, "page_slots must be a multiple of 8, at most 65536")
        _need(D % 8 == 0 and D <= CACHE_MAX_D, f"D must be a multiple of 8, at most {CACHE_MAX_D}")
        a = CCache(k.data_ptr(), v.data_ptr(), None, P, S, H, D)
        for name, t in (("k", k), ("v", v)):
            _need(t.stride(3) == 1, f"{name}: the elements of a head must be contiguous")
            for d, part in ((0, "page"), (1, "slot"), (2, "head")):
                stride = t.stride(d) if t.shape[d] > 1 else D
                _need(stride % 8 == 0, f"{name}: distances must be multiples of 8 elements")
                setattr(a, f"{name}_{part}", stride)
            _need(t.data_ptr() % 16 == 0, f"{name} must start on a 16-byte boundary")
        self._plain = a
        self._c = a
        if acc is not None:
            _need(acc.shape == (P, H, S) and acc.dtype is torch.float32 and acc.get_device() == dev, f"acc must be {[P, H, S]} float32 on the same device")
            _need(acc.stride(2) == 1, "acc: the slots of a head must be contiguous")
            self._c = CCache.from_buffer_copy(a)
            self._c.acc = acc.data_ptr()
            self._c.acc_page = acc.stride(0) if P > 1 else H * S
            self._c.acc_head = acc.stride(1) if H > 1 else S
        self.k, self.v, self.acc, self.device, self._dev = k, v, acc, k.device, dev

    page_slots = property(lambda self: self._plain.page_slots)
    heads = property(lambda self: self._plain.H)


def _seqs(cache: PagedCache, dev: int, table: torch.Tensor, lens: torch.Tensor, q_lens: Optional[torch.Tensor], B: int, Q: int) -> CCacheSeqs:
    if cache._dev != dev:
        raise CpmtpError("cpmtp: the cache is on another device")
    shape = table.shape
    if len(shape) != 2 or shape[0] != B or table.dtype is not torch.int32 or table.get_device() != dev or (shape[1] > 1 and table.stride(1) != 1):
        raise CpmtpError(f"cpmtp: table must be [{B}, pages] int32 with contiguous rows on the same device")
    ld = table.stride(0) if B > 1 else shape[1]
    if ld < shape[1]:
        raise CpmtpError("cpmtp: table: rows must not overlap")
    return CCacheSeqs(table.data_ptr(), _ints(lens, B, dev, "lens"), None if q_lens is None else _ints(q_lens, B, dev, "q_lens"), ld, B, shape[1], Q, 0)


def _ints(t: torch.Tensor, n: int, dev: int, name: str) -> int:
    if t.shape != (n,) or t.dtype is not torch.int32 or t.get_device() != dev or not t.is_contiguous():
        raise CpmtpError(f"cpmtp: {name} must be a contiguous [{n}] int32 on the same device")
    return t.data_ptr()


def _tokens(t: torch.Tensor, size: tuple, dev: int, name: str, written: bool = False) -> CTokens:
    """[B, Q, heads, D] bf16 tokens whose heads are contiguous."""
    if t.shape != size or t.dtype is not torch.bfloat16 or t.get_device() != dev:
        raise CpmtpError(f"cpmtp: {name} must be {list(size)} bfloat16 on the same device, not {list(t.shape)} {t.dtype}")
    seq, token, head, one = t.stride()
    B, Q, H, D = size
    if (one != 1 and D > 1) or (H > 1 and head < D) or (Q > 1 and token < D) or (written and B > 1 and seq < D):
        raise CpmtpError(f"cpmtp: {name}: the elements of a head must be contiguous and heads must not overlap")
    return CTokens(t.data_ptr(), seq if B > 1 else 0, token if Q > 1 else 0, head if H > 1 else 0)


def _status(dev_status: Optional[torch.Tensor], dev: int):
    return None if dev_status is None else _int32(dev_status, dev, "dev_status")


def cache_append(cache: PagedCache, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, *,
                 q_lens: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None) -> None:
    """cpmtp_cache_append: the keys and values [B, Q, H, D] bf16 of new tokens into their slots, the last ones of lens [B] int32 (the new
    tokens included); q_lens [B] int32: how many of the Q rows a sequence has (None: all).  table [B, pages] int32.  acc of the slots becomes 0."""
    dev = _device(k)
    _need(k.dim() == 4, "k must be [B, Q, H, D]")
    B, Q = k.shape[0], k.shape[1]
    size = (B, Q, cache._plain.H, cache._plain.D)
    s = _seqs(cache, dev, table, lens, q_lens, B, Q)
    rc = load_library().cpmtp_cache_append(cache._c, s, _tokens(k, size, dev, "k"), _tokens(v, size, dev, "v"), _status(dev_status, dev), _raw_stream(dev))
    if rc:
        _check(rc)


def cache_attend_workspace_bytes(cache: PagedCache, B: int, width: int, Q: int, Hq: int) -> int:
    """Scratch bytes of cache_attend for B sequences whose tables have `width` pages, Q new tokens and Hq query heads."""
    return int(load_library().cpmtp_cache_attend_workspace_bytes(cache._c, CCacheSeqs(None, None, None, width, B, width, Q, 0), Hq))


def cache_attend(cache: PagedCache, q: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, *, q_lens: Optional[torch.Tensor] = None,
                 scale: Optional[float] = None, accumulate: bool = True, want_lse: bool = False, out: Optional[dict] = None,
                 workspace: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None) -> dict:
    """cpmtp_cache_attend: attention of the new tokens q [B, Q, Hq, D] bf16 over the cache, which holds their own keys and values already
    (cache_append); token j of q_lens[b] sees lens[b] - (q_lens[b] - 1 - j) slots.  scale: D ** -0.5 if None.  Returns {"out" [B, Q, Hq, D] bf16
    [, "lse" [B, Q, Hq] fp32]}; rows behind q_lens are zeros, or left as they were in tensors given by `out`.  accumulate: add the
    weights to cache.acc, if the cache has it.  The dictionary `out` is the one that is returned: tensors that it lacks are made and put there, so a call with the same one
    writes over them."""
    dev = _device(q)
    size = q.shape
    _need(len(size) == 4, "q must be [B, Q, Hq, D]")
    B, Q, Hq, D = size
    c = cache._c if accumulate else cache._plain
    _need(D == c.D and Hq > 0 and Hq % c.H == 0, f"q must be [B, Q, a multiple of {c.H}, {c.D}]")
    s = _seqs(cache, dev, table, lens, q_lens, B, Q)
    res = out if out is not None else {}
    fresh = torch.empty if q_lens is None else torch.zeros
    if "out" not in res:
        res["out"] = fresh(size, dtype=torch.bfloat16, device=q.device)
    if want_lse and "lse" not in res:
        res["lse"] = fresh((B, Q, Hq), dtype=torch.float32, device=q.device)
    lse = res.get("lse")
    if lse is not None and (lse.shape != (B, Q, Hq) or lse.dtype is not torch.float32 or lse.get_device() != dev or not lse.is_contiguous()):
        raise CpmtpError(f"cpmtp: lse must be a contiguous {[B, Q, Hq]} float32 on the same device")
    a = CAttendArgs(_tokens(q, size, dev, "q"), _tokens(res["out"], size, dev, "out", True), None if lse is None else lse.data_ptr(), Hq,
                    D ** -0.5 if scale is None else scale)
    lib = load_library()
    if workspace is None:
        workspace = alloc_workspace(lib.cpmtp_cache_attend_workspace_bytes(c, s, Hq), q.device)
    pw, nw = _workspace(workspace, dev)
    rc = lib.cpmtp_cache_attend(c, s, a, pw, nw, _status(dev_status, dev), _raw_stream(dev))
    if rc:
        _check(rc)
    return res


def cache_evict(cache: PagedCache, table: torch.Tensor, lens: torch.Tensor, table_out: torch.Tensor, budget: int, *, recent: int = 0,
                out: Optional[dict] = None, dev_status: Optional[torch.Tensor] = None) -> dict:
    """cpmtp_cache_evict: cut every sequence down to `budget` slots for each head, the `recent` last ones and those of the others with the
    largest cache.acc, and move them into the pages of table_out [B, ceil(budget / page_slots) or more] int32, which must not be among those of
    `table`.  Returns {"lens" [B], "kept" [B, H, budget] slots (-1 behind the last)} int32: the dictionary `out`, if given, which tensors that it lacks are put into."""
    dev = _device(lens)
    _need(cache.acc is not None, "eviction needs a cache with acc")
    _need(budget >= 1 and 0 <= recent <= budget, "budget must be at least 1, recent between 0 and budget")
    B, c = lens.numel(), cache._c
    s = _seqs(cache, dev, table, lens, None, B, 0)
    pages = -(-budget // c.page_slots)
    if table_out.dim() != 2 or table_out.shape[0] != B or table_out.shape[1] < pages or table_out.dtype is not torch.int32 or \
            table_out.get_device() != dev or (table_out.shape[1] > 1 and table_out.stride(1) != 1):
        raise CpmtpError(f"cpmtp: table_out must be [{B}, {pages} or more] int32 with contiguous rows on the same device")
    ld = table_out.stride(0) if B > 1 else table_out.shape[1]
    _need(ld >= pages, "table_out: rows must not overlap")
    res = out if out is not None else {}
    if "lens" not in res:
        res["lens"] = torch.empty_like(lens)
    if "kept" not in res:
        res["kept"] = torch.empty((B, c.H, budget), dtype=torch.int32, device=lens.device)
    kept = res["kept"]
    if kept.shape != (B, c.H, budget) or kept.dtype is not torch.int32 or kept.get_device() != dev or not kept.is_contiguous():
        raise CpmtpError(f"cpmtp: kept must be a contiguous {[B, c.H, budget]} int32 on the same device")
    a = CEvictArgs(table_out.data_ptr(), ld, budget, recent, _ints(res["lens"], B, dev, "out lens"), kept.data_ptr())
    rc = load_library().cpmtp_cache_evict(c, s, a, None, 0, _status(dev_status, dev), _raw_stream(dev))
    if rc:
        _check(rc)
    return res


_INT_MAX = (1 << 31) - 1


def _setting(v, N: int, dtype, dev: int, name: str) -> tuple:
    """(number for all rows, address of the rows' own numbers)"""
    if isinstance(v, torch.Tensor):
        if v.shape != (N,) or v.dtype is not dtype or v.get_device() != dev or not v.is_contiguous():
            raise CpmtpError(f"cpmtp: {name} must be a number or a contiguous [{N}] {dtype} on the same device")
        return 0, v.data_ptr()
    if not v >= 0:
        raise CpmtpError(f"cpmtp: {name} must not be negative")
    return min(v, _INT_MAX) if dtype is torch.int32 else v, None


def sample_logits(logits: torch.Tensor, uniform: torch.Tensor, *, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0,
                  given: Optional[torch.Tensor] = None, want_kept: bool = False, out: Optional[dict] = None,
                  dev_status: Optional[torch.Tensor] = None) -> dict:
    """cpmtp_sample_logits: a token from each row of logits [N, V] (bf16 or fp32, rows may be strided) by uniform [N] fp32 in [0, 1).
    temperature, top_k, top_p, min_p: numbers, or tensors [N] (fp32, int32, fp32, fp32) with a setting for each row; 0, 0, 1 and 0 mean
    greedy and no filter.  given [N] int32: tokens to be scored, EMBED_PAD for none.  Returns {"tokens" [N] int32, "logp" [N] fp32
    [, "logp_given" [N] fp32][, "kept" [N] int32]}: log-probabilities under the filtered distribution.  The dictionary `out`, if given, is the one
    that is returned, and tensors that it lacks are put there."""
    dev = _device(logits)
    size, dtype = logits.shape, logits.dtype
    _need(len(size) == 2 and dtype in _TYPES, "logits must be [N, V] bfloat16 or float32")
    N, V = size
    pl, ld = _rows(logits, size, dtype, dev, "logits")
    (t, pt), (k, pk) = _setting(temperature, N, torch.float32, dev, "temperature"), _setting(top_k, N, torch.int32, dev, "top_k")
    (p, pp), (m, pm) = _setting(top_p, N, torch.float32, dev, "top_p"), _setting(min_p, N, torch.float32, dev, "min_p")
    res = out if out is not None else {}
    f32, i32 = torch.float32, torch.int32
    pu = _vector(uniform, N, f32, dev, "uniform")
    if "tokens" not in res:
        res["tokens"] = torch.empty_like(uniform, dtype=i32)
    if "logp" not in res:
        res["logp"] = torch.empty_like(uniform)
    if given is not None and "logp_given" not in res:
        res["logp_given"] = torch.empty_like(uniform)
    if want_kept and "kept" not in res:
        res["kept"] = torch.empty_like(uniform, dtype=i32)
    a = CSampleArgs(pl, ld, N, V, _TYPES[dtype], k, t, p, m, 0, pt, pk, pp, pm, pu,
                    None if given is None else _ints(given, N, dev, "given"), _ints(res["tokens"], N, dev, "tokens"), _vector(res["logp"], N, f32, dev, "logp"),
                    None if given is None else _vector(res["logp_given"], N, f32, dev, "logp_given"),
                    _ints(res["kept"], N, dev, "kept") if "kept" in res else None)
    rc = load_library().cpmtp_sample_logits(a, _status(dev_status, dev), _raw_stream(dev))
    if rc:
        _check(rc)
    return res
