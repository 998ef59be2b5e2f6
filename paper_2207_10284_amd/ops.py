"""Thin Python binding of libmra (C ABI in include/mra.h).

Argument marshalling only: every function checks tensor placement, dtype and
shape, allocates outputs with torch (device memory is plumbing here), and
calls the library on the current torch stream. All arithmetic runs in the HIP
kernels. The forward calls and ``mra_attention`` do this in native code
(csrc/binding.cpp, loaded by the first of them). There is no fallback: if the
library is not built, ``load`` raises, and these calls do if the binding is not.

Shapes: q, k, v are [B, H, n, d] tensors on a ROCm device, float32 or
bfloat16, contiguous; n is a multiple of 32 and d is 32, 64 or 128.

``exact_attention`` and its parts are the softmax attention that MRA-2
approximates (C ABI in include/mra_exact.h, a library of its own): any lengths,
strided tensors, padded and causal batches, shared key heads, a learned
position bias, single tokens.
"""
from __future__ import annotations

import ctypes
import functools
import math
import os
import warnings

import torch

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libmra.so")
BLOCK = 32

MRA_F32, MRA_BF16 = 0, 1
STATUS = {0: "MRA_OK", 1: "MRA_ERR_INVALID_ARG", 2: "MRA_ERR_UNSUPPORTED",
          3: "MRA_ERR_MISALIGNED", 4: "MRA_ERR_WORKSPACE", 5: "MRA_ERR_HIP", 6: "MRA_ERR_SCRATCH"}

# name -> (restype, argtypes); mirrors include/mra.h
_P, _I, _Z = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
SIGNATURES = {
    "mra_pool": (_I, [_P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _P]),
    "mra_coarse_scores": (_I, [_P, _P, _P, _I, _I, _I, _I, _I, _P]),
    "mra_select": (_I, [_P, _P, _I, _I, _I, _I, _I, _P]),
    "mra_coarse_term": (_I, [_P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _P]),
    "mra_block_sddmm_spmm": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _I, _P]),
    "mra_forward_workspace_bytes": (_Z, [_I, _I, _I, _I, _I, _I, _I]),
    "mra_attention_forward": (_I, [_P, _P, _P, _P, _P, _P, _P, _Z, _I, _I, _I, _I, _I, _I, _I, _P]),
    "mra_sparse_attention_forward": (_I, [_P, _P, _P, _P, _P, _P, _P, _Z, _I, _I, _I, _I, _I, _I, _I, _P]),
    "mra_attention_forward_noalloc": (_I, [_P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _I, _P]),
    "mra_select_global": (_I, [_P, _P, _I, _I, _I, _I, _I, _I, _P]),
    "mra_forward_global_workspace_bytes": (_Z, [_I, _I, _I, _I, _I, _I]),
    "mra_attention_forward_global": (_I, [_P, _P, _P, _P, _P, _P, _P, _Z, _I, _I, _I, _I, _I, _I, _I, _I, _P]),
    "mra_forward_multilevel_workspace_bytes": (_Z, [_I, _I, _I, _I, _I, _I, _I, _I, _I]),
    "mra_attention_forward_multilevel": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _Z, _I, _I, _I, _I, _I, _I,
                                              _I, _I, _I, _P]),
    "mra_forward_levels_workspace_bytes": (_Z, [_I, _I, _I, _I, _I, _I, _P, _P, _I]),
    "mra_attention_forward_levels": (_I, [_P, _P, _P, _P, _P, _P, _P, _Z, _I, _I, _I, _I, _I, _I,
                                          _P, _P, _I, _P]),
    "mra_backward_workspace_bytes": (_Z, [_I, _I, _I, _I, _I, _I]),
    "mra_attention_backward": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _Z,
                                    _I, _I, _I, _I, _I, _I, _I, _I, _P]),
    "mra_attention_backward_pooled": (_I, [_P] * 14 + [_Z] + [_I] * 8 + [_P]),
    "mra_forward_pooled_rows": (_I, [_P, _I, _I, _I, _I, _I, _P, _P, _P]),
    "mra_status_str": (ctypes.c_char_p, [_I]),
    "mra_last_hip_error": (_I, []),
}

_lib = None
_native = None          # csrc/binding.cpp, bound to _lib by the first call that needs it


class MraError(RuntimeError):
    def __init__(self, fn: str, status: int, lib):
        msg = lib.mra_status_str(status).decode()
        if status == 5:
            msg += f" (hipError_t {lib.mra_last_hip_error()})"
        super().__init__(f"{fn}: {msg}")
        self.status = status


def load(path: str = LIB_PATH):
    """Open libmra.so once and declare its signatures. Raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is not built; run `python -m paper_2207_10284_amd.build` "
                               "(hipcc, gfx950) first")
        lib = ctypes.CDLL(path)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


def bind():
    """The native binding, holding the library's entry points. Raises if it
    cannot be imported (it is built for one Python and one torch); the other
    calls need only the library."""
    global _native
    if _native is None:
        lib = load()
        try:
            from paper_2207_10284_amd import _binding
        except ImportError as e:
            raise RuntimeError(f"the torch binding is not built ({e}); run `python -m paper_2207_10284_amd.build` "
                               "first") from e
        _binding.bind({name: ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in SIGNATURES},
                      lambda fn, status: MraError(fn, status, lib))
        _native = _binding
    return _native


def _call(name: str, *args):
    lib = load()
    st = getattr(lib, name)(*args)
    if st != 0:
        raise MraError(name, st, lib)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(device):
    return torch.cuda.current_stream(device).cuda_stream


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return MRA_F32
    if t.dtype == torch.bfloat16:
        return MRA_BF16
    raise TypeError(f"unsupported dtype {t.dtype}; expected float32 or bfloat16")


def _check_qkv(*ts):
    ref = next(t for t in ts if t is not None)
    for t in ts:
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError("tensors must be on a ROCm device")
        if t.dim() != 4 or t.shape != ref.shape or t.dtype != ref.dtype or t.device != ref.device:
            raise ValueError("q, k, v must share shape [B, H, n, d], dtype and device")
        if not t.is_contiguous():
            raise ValueError("q, k, v must be contiguous")
    return ref


def _check_f32(t, shape, name):
    if t.dtype != torch.float32 or tuple(t.shape) != tuple(shape) or not t.is_contiguous() or not t.is_cuda:
        raise ValueError(f"{name} must be a contiguous float32 device tensor of shape {tuple(shape)}")


def pool(q, k=None, v=None):
    """Block means (Sec. 4.1/4.3): returns (qp, kp, vp), float32 [B, H, n/32, d]
    (None for a tensor not given)."""
    ref = _check_qkv(q, k, v)
    B, H, n, d = ref.shape
    outs = [None if t is None else torch.empty(B, H, n // BLOCK, d, device=ref.device, dtype=torch.float32)
            for t in (q, k, v)]
    _call("mra_pool", _ptr(q), _ptr(k), _ptr(v), *(_ptr(o) for o in outs),
          B, H, n, d, BLOCK, _dtype_code(ref), _stream(ref.device))
    return tuple(outs)


def coarse_scores(qp, kp):
    """Coarse logits S~ = Q~ K~^T / sqrt(d): float32 [B, H, nb, nb]."""
    B, H, nb, d = qp.shape
    _check_f32(qp, (B, H, nb, d), "qp")
    _check_f32(kp, (B, H, nb, d), "kp")
    S = torch.empty(B, H, nb, nb, device=qp.device, dtype=torch.float32)
    _call("mra_coarse_scores", _ptr(qp), _ptr(kp), _ptr(S), B, H, nb * BLOCK, d, BLOCK, _stream(qp.device))
    return S


def select(scores, budget: int):
    """Per block-row top-`budget` column blocks, ascending: int32 [B, H, nb, budget]."""
    B, H, nb, _ = scores.shape
    _check_f32(scores, (B, H, nb, nb), "scores")
    idx = torch.empty(B, H, nb, budget, device=scores.device, dtype=torch.int32)
    _call("mra_select", _ptr(scores), _ptr(idx), B, H, nb * BLOCK, BLOCK, budget, _stream(scores.device))
    return idx


def select_global(scores, budget: int, prior_diagonal: bool = False):
    """Head-wide selection of Alg. 1: the `budget` best blocks of each head
    (plus the diagonal blocks with ``prior_diagonal``); int32 [B, H, nb, nb],
    each row ascending, padded with -1."""
    B, H, nb, _ = scores.shape
    _check_f32(scores, (B, H, nb, nb), "scores")
    idx = torch.empty(B, H, nb, nb, device=scores.device, dtype=torch.int32)
    _call("mra_select_global", _ptr(scores), _ptr(idx), B, H, nb * BLOCK, BLOCK, budget,
          int(bool(prior_diagonal)), _stream(scores.device))
    return idx


def _check_idx(idx, B, H, nb, budget, device):
    if idx.dtype != torch.int32 or tuple(idx.shape) != (B, H, nb, budget) or not idx.is_contiguous() \
            or idx.device != device:
        raise ValueError(f"idx must be a contiguous int32 tensor of shape {(B, H, nb, budget)}")


def coarse_term(scores, idx, vp):
    """Low-resolution term of the unselected blocks: (cmax, csum, cvec)."""
    B, H, nb, d = vp.shape
    budget = idx.shape[-1]
    _check_f32(scores, (B, H, nb, nb), "scores")
    _check_f32(vp, (B, H, nb, d), "vp")
    _check_idx(idx, B, H, nb, budget, vp.device)
    cmax = torch.empty(B, H, nb, device=vp.device, dtype=torch.float32)
    csum = torch.empty_like(cmax)
    cvec = torch.empty(B, H, nb, d, device=vp.device, dtype=torch.float32)
    _call("mra_coarse_term", _ptr(scores), _ptr(idx), _ptr(vp), _ptr(cmax), _ptr(csum), _ptr(cvec),
          B, H, nb * BLOCK, d, BLOCK, budget, _stream(vp.device))
    return cmax, csum, cvec


def block_sddmm_spmm(q, k, v, idx, cmax=None, csum=None, cvec=None, out=None, lse_out=None):
    """Selected tiles exp(c Q_x K_y^T) V_y, merged with the coarse term (if
    given) and normalised: the output Z, [B, H, n, d] in the input dtype.
    ``lse_out`` (float32 [B, H, n]) receives each query's log normaliser."""
    ref = _check_qkv(q, k, v)
    B, H, n, d = ref.shape
    nb = n // BLOCK
    budget = idx.shape[-1]
    _check_idx(idx, B, H, nb, budget, ref.device)
    if cmax is not None:
        _check_f32(cmax, (B, H, nb), "cmax")
        _check_f32(csum, (B, H, nb), "csum")
        _check_f32(cvec, (B, H, nb, d), "cvec")
    if out is None:
        out = torch.empty_like(ref)
    if lse_out is not None:
        _check_f32(lse_out, (B, H, n), "lse_out")
    _call("mra_block_sddmm_spmm", _ptr(q), _ptr(k), _ptr(v), _ptr(idx), _ptr(cmax), _ptr(csum),
          _ptr(cvec), _ptr(out), _ptr(lse_out), B, H, n, d, BLOCK, budget, _dtype_code(ref), _stream(ref.device))
    return out


def forward_workspace_bytes(B: int, H: int, n: int, d: int, budget: int, dtype=torch.bfloat16) -> int:
    code = MRA_BF16 if dtype == torch.bfloat16 else MRA_F32
    return int(load().mra_forward_workspace_bytes(B, H, n, d, BLOCK, budget, code))


_PLAIN = (torch.Tensor, torch.nn.Parameter)


def _result(q, out):
    """``out``, allocated here for a tensor subclass (its own ``empty_like``
    decides the result's type), else where it is needed."""
    if out is None and type(q) not in _PLAIN and isinstance(q, torch.Tensor):
        return torch.empty_like(q)
    return out


def attention_forward(q, k, v, budget: int, out=None, idx_out=None, workspace=None, lse_out=None):
    """The whole MRA-2 forward pass. Returns the output Z ([B, H, n, d], input
    dtype); the selection is written to ``idx_out`` and each query's log
    normaliser (float32 [B, H, n]) to ``lse_out`` when given."""
    return bind().forward(0, q, k, v, budget, False, _result(q, out), idx_out, workspace, lse_out)


def attention_forward_noalloc(q, k, v, budget: int, out=None, idx_out=None, lse_out=None):
    """``attention_forward`` through the entry point that allocates nothing:
    its workspace is the library's static per-GPU scratch (calls on one GPU
    must not overlap). ``out`` is allocated here only when not given."""
    ref = _check_qkv(q, k, v)
    B, H, n, d = ref.shape
    nb = n // BLOCK
    if out is None:
        out = torch.empty_like(ref)
    if idx_out is not None:
        _check_idx(idx_out, B, H, nb, budget, ref.device)
    if lse_out is not None:
        _check_f32(lse_out, (B, H, n), "lse_out")
    _call("mra_attention_forward_noalloc", _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(idx_out), _ptr(lse_out),
          B, H, n, d, BLOCK, budget, _dtype_code(ref), _stream(ref.device))
    return out


def sparse_attention_forward(q, k, v, budget: int, out=None, idx_out=None, workspace=None, lse_out=None):
    """The sparse-only variant MRA-2-s (Sec. 5): softmax over the selected
    blocks only, no low-resolution term; budget >= 1. Same arguments and
    result as ``attention_forward``."""
    return bind().forward(1, q, k, v, budget, False, _result(q, out), idx_out, workspace, lse_out)


def forward_global_workspace_bytes(B: int, H: int, n: int, d: int, dtype=torch.bfloat16) -> int:
    code = MRA_BF16 if dtype == torch.bfloat16 else MRA_F32
    return int(load().mra_forward_global_workspace_bytes(B, H, n, d, BLOCK, code))


def attention_forward_global(q, k, v, budget: int, prior_diagonal: bool = False, out=None, idx_out=None,
                             workspace=None, lse_out=None):
    """MRA-2 with the head-wide budget of Alg. 1 (``budget`` blocks per head,
    plus the diagonal with ``prior_diagonal``). Returns Z; the selection
    (int32 [B, H, nb, nb], rows padded with -1) goes to ``idx_out`` and the
    log normalisers to ``lse_out`` when given."""
    return bind().forward(2, q, k, v, budget, bool(prior_diagonal), _result(q, out), idx_out, workspace, lse_out)


def forward_multilevel_workspace_bytes(B: int, H: int, n: int, d: int, coarse_block: int, budget1: int,
                                       budget2: int, dtype=torch.bfloat16) -> int:
    code = MRA_BF16 if dtype == torch.bfloat16 else MRA_F32
    return int(load().mra_forward_multilevel_workspace_bytes(B, H, n, d, BLOCK, coarse_block, budget1, budget2,
                                                             code))


def attention_forward_multilevel(q, k, v, coarse_block: int, budget1: int, budget2: int, out=None,
                                 idx1_out=None, idx2_out=None, lse_out=None, workspace=None):
    """Three resolutions R = {coarse_block, 32, 1} (Alg. 1 with two refinement
    levels, per-row budgets). Returns Z; the selections go to ``idx1_out``
    (int32 [B, H, n/coarse_block, budget1]) and ``idx2_out`` (int32
    [B, H, n/32, budget2]) when given."""
    ref = _check_qkv(q, k, v)
    B, H, n, d = ref.shape
    if out is None:
        out = torch.empty_like(ref)
    if idx1_out is not None:
        _check_idx(idx1_out, B, H, n // coarse_block if coarse_block else 0, budget1, ref.device)
    if idx2_out is not None:
        _check_idx(idx2_out, B, H, n // BLOCK, budget2, ref.device)
    if lse_out is not None:
        _check_f32(lse_out, (B, H, n), "lse_out")
    need = forward_multilevel_workspace_bytes(B, H, n, d, coarse_block, budget1, budget2, ref.dtype)
    if workspace is None:
        workspace = torch.empty(max(need, 1), device=ref.device, dtype=torch.uint8)
    _call("mra_attention_forward_multilevel", _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(idx1_out),
          _ptr(idx2_out), _ptr(lse_out), _ptr(workspace), workspace.numel() * workspace.element_size(),
          B, H, n, d, BLOCK, coarse_block, budget1, budget2, _dtype_code(ref), _stream(ref.device))
    return out


def _int_array(vals):
    vals = [int(x) for x in vals]
    return (ctypes.c_int * max(len(vals), 1))(*vals)


def forward_levels_workspace_bytes(B: int, H: int, n: int, d: int, scales, budgets, dtype=torch.bfloat16) -> int:
    code = MRA_BF16 if dtype == torch.bfloat16 else MRA_F32
    sc, bu = _int_array(scales), _int_array(budgets)
    return int(load().mra_forward_levels_workspace_bytes(B, H, n, d, BLOCK, len(scales),
                                                         ctypes.cast(sc, _P), ctypes.cast(bu, _P), code))


def attention_forward_levels(q, k, v, scales, budgets, out=None, idx_outs=None, lse_out=None,
                             workspace=None):
    """Any number of resolutions R = {scales[0] > ... > scales[-1] = 32, 1}
    (Alg. 1 refined level by level, a per-row budget at every level). Returns
    Z; level l's selection goes to ``idx_outs[l]`` (int32
    [B, H, n/scales[l], budgets[l]]) when that entry is given."""
    ref = _check_qkv(q, k, v)
    B, H, n, d = ref.shape
    L = len(scales)
    if len(budgets) != L or L < 1:
        raise ValueError("one budget per scale")
    if out is None:
        out = torch.empty_like(ref)
    outs = list(idx_outs) if idx_outs is not None else [None] * L
    if len(outs) != L:
        raise ValueError("one selection output (or None) per scale")
    for l, t in enumerate(outs):
        if t is not None:
            _check_idx(t, B, H, n // int(scales[l]) if int(scales[l]) > 0 else 0, int(budgets[l]), ref.device)
    if lse_out is not None:
        _check_f32(lse_out, (B, H, n), "lse_out")
    need = forward_levels_workspace_bytes(B, H, n, d, scales, budgets, ref.dtype)
    if workspace is None:
        workspace = torch.empty(max(need, 1), device=ref.device, dtype=torch.uint8)
    sc, bu = _int_array(scales), _int_array(budgets)
    ptrs = (ctypes.c_void_p * L)(*[_ptr(t) for t in outs])
    _call("mra_attention_forward_levels", _ptr(q), _ptr(k), _ptr(v), _ptr(out), ctypes.cast(ptrs, _P),
          _ptr(lse_out), _ptr(workspace), workspace.numel() * workspace.element_size(), B, H, n, d, BLOCK,
          L, ctypes.cast(sc, _P), ctypes.cast(bu, _P), _dtype_code(ref), _stream(ref.device))
    return out


def backward_workspace_bytes(B: int, H: int, n: int, d: int, dtype=torch.bfloat16) -> int:
    code = MRA_BF16 if dtype == torch.bfloat16 else MRA_F32
    return int(load().mra_backward_workspace_bytes(B, H, n, d, BLOCK, code))


def forward_pooled_rows(workspace, B: int, H: int, n: int, d: int):
    """The block means (Q~, K~, V~: float32 [B, H, nb, d] each) that
    ``attention_forward`` or ``attention_forward_global`` left in
    ``workspace`` (a uint8 device tensor) for these sizes, as views of it (no
    copy); they change when the workspace is used again."""
    if workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor")
    nb = n // BLOCK
    if B * H * nb * d == 0:
        return tuple(torch.empty(B, H, nb, d, dtype=torch.float32, device=workspace.device) for _ in range(3))
    ptrs = [ctypes.c_void_p() for _ in range(3)]
    _call("mra_forward_pooled_rows", _ptr(workspace), B, H, n, d, BLOCK, *(ctypes.byref(p) for p in ptrs))
    size = B * H * nb * d * 4
    views = []
    for p in ptrs:
        off = (p.value or 0) - workspace.data_ptr()
        if p.value is None or off < 0 or off + size > workspace.numel():
            raise ValueError("workspace too small for the pooled rows of these sizes")
        views.append(workspace[off:off + size].view(torch.float32).view(B, H, nb, d))
    return tuple(views)


def attention_backward(q, k, v, out, dout, lse, idx, coarse: bool = True, dq=None, dk=None, dv=None,
                       workspace=None, pooled=None):
    """Gradients (dq, dk, dv) through one forward (``coarse=True``: MRA-2,
    per-row or head-wide budget; ``False``: MRA-2-s) with its selection
    ``idx`` (int32 [B, H, nb, width]) held fixed; ``out`` and ``lse`` are the
    forward's output and log normalisers, ``dout`` the gradient of the output.
    ``pooled``: the block means of q, k, v (float32 [B, H, nb, d] each, e.g.
    from ``forward_pooled_rows``), so that the backward does not compute them
    again; the gradients are the same bits either way."""
    ref = _check_qkv(q, k, v, out, dout)
    B, H, n, d = ref.shape
    nb = n // BLOCK
    width = idx.shape[-1]
    _check_idx(idx, B, H, nb, width, ref.device)
    _check_f32(lse, (B, H, n), "lse")
    dq = torch.empty_like(ref) if dq is None else dq
    dk = torch.empty_like(ref) if dk is None else dk
    dv = torch.empty_like(ref) if dv is None else dv
    _check_qkv(ref, dq, dk, dv)
    need = backward_workspace_bytes(B, H, n, d, ref.dtype)
    if workspace is None:
        workspace = torch.empty(max(need, 1), device=ref.device, dtype=torch.uint8)
    head = (_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(dout), _ptr(lse), _ptr(idx))
    tail = (_ptr(dq), _ptr(dk), _ptr(dv), _ptr(workspace), workspace.numel() * workspace.element_size(),
            B, H, n, d, BLOCK, width, int(bool(coarse)), _dtype_code(ref), _stream(ref.device))
    if pooled is None:
        _call("mra_attention_backward", *head, *tail)
    else:
        for name, t in zip(("qp", "kp", "vp"), pooled):
            _check_f32(t, (B, H, nb, d), name)
            if t.device != ref.device:
                raise ValueError(f"{name} must be on {ref.device}")
        _call("mra_attention_backward_pooled", *head, *(_ptr(t) for t in pooled), *tail)
    return dq, dk, dv


class MraAttention(torch.autograd.Function):
    """Z = MRA-2 attention of (q, k, v) as a differentiable op: the forward
    keeps its selection and log normalisers, the backward hands them to
    ``attention_backward`` (selection held fixed). ``variant`` is "mra2"
    (per-row budget), "mra2s" (sparse only) or "global" (head-wide budget,
    with ``prior_diagonal``)."""

    @staticmethod
    def forward(ctx, q, k, v, budget: int, variant: str = "mra2", prior_diagonal: bool = False):
        ref = _check_qkv(q, k, v)
        B, H, n, d = ref.shape
        nb = n // BLOCK
        lse = torch.empty(B, H, n, device=ref.device, dtype=torch.float32)
        pooled = ()
        if variant == "global":
            idx = torch.empty(B, H, nb, nb, device=ref.device, dtype=torch.int32)
            ws = torch.empty(max(forward_global_workspace_bytes(B, H, n, d, ref.dtype), 1), device=ref.device,
                             dtype=torch.uint8)
            out = attention_forward_global(q, k, v, budget, prior_diagonal, idx_out=idx, workspace=ws, lse_out=lse)
            pooled = forward_pooled_rows(ws, B, H, n, d)
        elif variant == "mra2":
            idx = torch.empty(B, H, nb, budget, device=ref.device, dtype=torch.int32)
            ws = torch.empty(max(forward_workspace_bytes(B, H, n, d, budget, ref.dtype), 1), device=ref.device,
                             dtype=torch.uint8)
            out = attention_forward(q, k, v, budget, idx_out=idx, workspace=ws, lse_out=lse)
            pooled = forward_pooled_rows(ws, B, H, n, d)
        elif variant == "mra2s":
            idx = torch.empty(B, H, nb, budget, device=ref.device, dtype=torch.int32)
            out = sparse_attention_forward(q, k, v, budget, idx_out=idx, lse_out=lse)
        else:
            raise ValueError(f"unknown variant {variant!r}")
        # the forward's block means (views of its workspace) go to the backward
        ctx.save_for_backward(q, k, v, out, lse, idx, *pooled)
        ctx.coarse = variant != "mra2s"
        return out

    @staticmethod
    def backward(ctx, dout):
        q, k, v, out, lse, idx, *pooled = ctx.saved_tensors
        dq, dk, dv = attention_backward(q, k, v, out, dout.contiguous(), lse, idx, coarse=ctx.coarse,
                                        pooled=tuple(pooled) if pooled else None)
        return dq, dk, dv, None, None, None


_VARIANTS = ("mra2", "mra2s", "global")       # the native variants, in their order


def mra_attention(q, k, v, budget: int, variant: str = "mra2", prior_diagonal: bool = False):
    """Differentiable MRA-2 attention (see ``MraAttention``, whose native
    counterpart runs here; under functorch transforms, tracing or compilation,
    and for tensor subclasses, the Python function itself)."""
    if (type(q) in _PLAIN and type(k) in _PLAIN and type(v) in _PLAIN and variant in _VARIANTS
            and not torch._C._are_functorch_transforms_active() and torch._C._get_tracing_state() is None
            and not torch.compiler.is_compiling()):
        return bind().mra_attention(q, k, v, budget, _VARIANTS.index(variant), bool(prior_diagonal))
    return MraAttention.apply(q, k, v, budget, variant, prior_diagonal)


# ---------------------------------------------------------------------------
# Exact softmax attention (include/mra_exact.h)
EXACT_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libmra_exact.so")
MAX_FAR = 512                 # distances with a bucket of their own on either side
MAX_BUCKETS = 1024


class _Strided(ctypes.Structure):
    _fields_ = [("data", _P), ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64),
                ("stride_n", ctypes.c_int64)]


class _Problem(ctypes.Structure):
    _fields_ = [("B", _I), ("H", _I), ("H_kv", _I), ("n_q", _I), ("n_k", _I), ("d", _I), ("dtype", _I),
                ("scale", ctypes.c_float), ("causal", _I), ("lengths", _P), ("q_start", _P), ("key_mask", _P),
                ("key_mask_stride", ctypes.c_int64), ("bias", _P), ("bias_dtype", _I), ("buckets", _I),
                ("bucket_map", _P), ("far", _I)]


# name -> (restype, argtypes); mirrors include/mra_exact.h
EXACT_SIGNATURES = {
    "mra_exact_forward_workspace_bytes": (_Z, [_P]),
    "mra_exact_forward": (_I, [_P] * 7 + [_Z, _P]),
    "mra_exact_backward_workspace_bytes": (_Z, [_P]),
    "mra_exact_backward": (_I, [_P] * 12 + [_Z, _P]),
    "mra_exact_last_hip_error": (_I, []),
}

_exact_lib = None
_exact_native = None    # csrc/exact_binding.cpp, bound to _exact_lib by the first call that needs it


class _ExactStatus:
    """What MraError asks of a library: the shared status texts, this library's HIP error."""

    def mra_status_str(self, status):
        return load().mra_status_str(status)

    def mra_last_hip_error(self):
        return load_exact().mra_exact_last_hip_error()


def load_exact(path: str = EXACT_LIB_PATH):
    """Open libmra_exact.so once and declare its signatures. Raises if it is missing."""
    global _exact_lib
    if _exact_lib is None:
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is not built; run `python -m paper_2207_10284_amd.build` "
                               "(hipcc, gfx950) first")
        lib = ctypes.CDLL(path)
        for name, (res, args) in EXACT_SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _exact_lib = lib
    return _exact_lib


def bind_exact():
    """The native binding of the exact-attention calls (as ``bind``)."""
    global _exact_native
    if _exact_native is None:
        lib = load_exact()
        try:
            from paper_2207_10284_amd import _binding_exact
        except ImportError as e:
            raise RuntimeError(f"the torch binding is not built ({e}); run `python -m paper_2207_10284_amd.build` "
                               "first") from e
        _binding_exact.bind({name: ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in EXACT_SIGNATURES},
                            lambda fn, status: MraError(fn, status, _ExactStatus()))
        _exact_native = _binding_exact
    return _exact_native


def _call_exact(name: str, *args):
    st = getattr(load_exact(), name)(*args)
    if st != 0:
        raise MraError(name, st, _ExactStatus())


@functools.lru_cache(maxsize=64)
def _bucket_row(num_buckets: int, max_distance: int, bidirectional: bool):
    if num_buckets < (4 if bidirectional else 2) or (bidirectional and num_buckets % 2) or num_buckets > MAX_BUCKETS:
        raise ValueError(f"num_buckets must be 2 to {MAX_BUCKETS} (4 or more, and even, for both directions)")
    n = num_buckets // 2 if bidirectional else num_buckets
    e = n // 2
    if max_distance <= e:
        raise ValueError(f"max_distance must be above {e}, the distances with a bucket of their own")
    # floor((n - e) log(r / e) / log(max_distance / e)) >= t as a comparison of whole
    # numbers, so that distances on a border fall where the formula says
    lefts = [max_distance ** t * e ** (n - e) for t in range(n - e)]

    def bucket(r):
        if r < e:
            return r
        t = 0
        while t < n - e - 1 and r ** (n - e) * e ** (t + 1) >= lefts[t + 1]:
            t += 1
        return e + t

    side = []
    while not side or side[-1] != n - 1:
        side.append(bucket(len(side)))
        if len(side) > MAX_FAR + 1:
            raise ValueError(f"the last bucket may begin at distance {MAX_FAR} at most")
    back = side[:0:-1]                                       # keys before the query, the farthest first
    return tuple(back + [0] + ([n + x for x in side[1:]] if bidirectional else [0] * len(back)))


def distance_buckets(num_buckets: int, max_distance: int, bidirectional: bool = True, device="cuda"):
    """The map of a learned position bias: int32 [2 far + 1], the bucket of each
    distance key - query from -far to far; beyond, the outer buckets hold. Each
    direction has num_buckets / 2 of them (one direction: all; later keys then
    share bucket 0 with distance 0). Half of a direction's buckets hold one
    distance each; from there on the width grows by a constant factor: distance
    r >= e has bucket e + floor((n - e) log(r / e) / log(max_distance / e)), at
    most n - 1. Any other map of whole numbers in this form serves as well."""
    return torch.tensor(_bucket_row(int(num_buckets), int(max_distance), bool(bidirectional)), dtype=torch.int32,
                        device=device)


def _strides(t):
    """Element strides of the outer three axes (0 where an axis has at most one entry)."""
    return tuple(st if n > 1 else 0 for st, n in zip(t.stride()[:3], t.shape[:3]))


def _dense_rows(t) -> bool:
    per = 16 // t.element_size()
    return (t.stride(3) == 1 and t.data_ptr() % 16 == 0 and all(st % per == 0 for st in _strides(t))) or t.numel() == 0


def _check_rows(t, ref, shape, name):
    if not t.is_cuda:
        raise ValueError("tensors must be on a ROCm device")
    if tuple(t.shape) != tuple(shape) or t.dtype != ref.dtype or t.device != ref.device:
        raise ValueError(f"{name} must be a {ref.dtype} tensor of shape {tuple(shape)} on {ref.device}")
    if not _dense_rows(t):
        raise ValueError(f"{name} must have dense rows, 16-byte aligned")


def _check_out(t, ref, name):
    _check_rows(t, ref, ref.shape, name)
    if t.numel() and any(n > 1 and not st for n, st in zip(t.shape, _strides(t))):
        raise ValueError(f"{name} must not be broadcast")


def _view(t):
    return _Strided(t.data_ptr(), *_strides(t))


def _rows_like(t):
    """An output for t: its layout where that has dense rows."""
    o = torch.empty_like(t)
    return o if _dense_rows(o) else torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _check_int(t, shape, name, device):
    if t.dtype != torch.int32 or tuple(t.shape) != shape or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{name} must be a contiguous int32 tensor of shape {shape} on {device}")


_EXACT_KEYS = ("scale", "causal", "lengths", "key_mask", "q_start", "bias", "buckets")


def _exact_problem(q, k, v, scale, causal, lengths, key_mask, q_start, bias, buckets):
    if not (q.is_cuda and k.is_cuda and v.is_cuda):
        raise ValueError("tensors must be on a ROCm device")
    if q.dim() != 4 or k.dim() != 4 or v.dim() != 4:
        raise ValueError("q, k, v must have shape [B, heads, n, d]")
    code = _dtype_code(q)
    B, H, nq, d = q.shape
    Hkv, nk = k.shape[1], k.shape[2]
    if k.shape != (B, Hkv, nk, d) or v.shape != k.shape or (H % Hkv if Hkv else H):
        raise ValueError("k, v must share shape [B, H_kv, n_k, d] with q's B and d, H a multiple of H_kv")
    if max(*q.shape, Hkv, nk) >= 1 << 31:
        raise ValueError("sizes must be below 2^31")
    for t, name in ((q, "q"), (k, "k"), (v, "v")):
        _check_rows(t, q, t.shape, name)
    dev = q.device
    if lengths is not None:
        _check_int(lengths, (B,), "lengths", dev)
    if q_start is not None:
        _check_int(q_start, (B,), "q_start", dev)
    if key_mask is not None and (key_mask.dtype not in (torch.bool, torch.uint8) or key_mask.shape != (B, nk)
                                 or (nk > 1 and key_mask.stride(1) != 1) or key_mask.device != dev):
        raise ValueError(f"key_mask must be a bool or uint8 tensor of shape {(B, nk)} with dense rows on {dev}")
    if (bias is None) != (buckets is None):
        raise ValueError("bias and buckets go together")
    far = num = 0
    if bias is not None:
        if bias.dim() != 2 or bias.shape[1] != H or bias.dtype not in (q.dtype, torch.float32) \
                or not bias.is_contiguous() or bias.device != dev:
            raise ValueError(f"bias must be a contiguous tensor of shape [buckets, {H}], float32 or q's dtype, on {dev}")
        if buckets.dim() != 1 or buckets.numel() % 2 != 1:
            raise ValueError("buckets must be int32 of odd length (see distance_buckets)")
        _check_int(buckets, tuple(buckets.shape), "buckets", dev)
        num, far = bias.shape[0], buckets.numel() // 2
    return _Problem(B, H, Hkv, nq, nk, d, code, d ** -0.5 if scale is None else float(scale), int(bool(causal)),
                    _ptr(lengths), _ptr(q_start), _ptr(key_mask),
                    key_mask.stride(0) if key_mask is not None and B > 1 else 0, _ptr(bias),
                    _dtype_code(bias) if bias is not None else 0, num, _ptr(buckets), far)


def exact_forward_workspace_bytes(q, k, v, **kw) -> int:
    """Workspace of ``exact_attention_forward`` for these arguments (0: none)."""
    p = _exact_problem(q, k, v, *(kw.get(n) for n in _EXACT_KEYS))
    return int(load_exact().mra_exact_forward_workspace_bytes(ctypes.byref(p)))


def exact_backward_workspace_bytes(q, k, v, **kw) -> int:
    """Workspace of ``exact_attention_backward`` for these arguments."""
    p = _exact_problem(q, k, v, *(kw.get(n) for n in _EXACT_KEYS))
    return int(load_exact().mra_exact_backward_workspace_bytes(ctypes.byref(p)))


def exact_attention_forward(q, k, v, *, scale=None, causal: bool = False, lengths=None, key_mask=None, q_start=None,
                            bias=None, buckets=None, out=None, lse_out=None, workspace=None):
    """Softmax attention softmax(scale q k^T + bias) v, [B, H, n_q, d]; query head
    h reads key head h // (H / H_kv).

    q: [B, H, n_q, d]; k, v: [B, H_kv, n_k, d], any strides with dense 16-byte
    aligned rows. ``scale``: 1 / sqrt(d) if not given; 2^-64 to 2^64. Query i stands
    at position ``q_start[b] + i`` (int32 [B]; n_k - n_q + i if not given). A key j
    counts if j < ``lengths[b]`` (int32 [B]), ``key_mask[b, j]`` (bool or uint8
    [B, n_k]) and, with ``causal``, j is at most the position; each only where
    given. What lies at other keys may be anything; a query for which no key
    counts gives zeros. ``bias`` ([buckets, H], float32 or q's dtype) adds
    bias[buckets[distance], h] for the distance j - position (``buckets``: see
    ``distance_buckets``); an entry below -2^14, -inf and the usual mask values
    among them, takes its distances out, one above 2^14 is taken as that.
    ``lse_out`` (float32 [B, H, n_q]) receives the log normalisers; it and ``out`` overlap no other
    argument. A call whose ``workspace`` (uint8) a graph captured must not run
    beside another with the same one."""
    return bind_exact().forward(q, k, v, scale, causal, lengths, key_mask, q_start, bias, buckets, _result(q, out),
                                lse_out, workspace)


def exact_attention_backward(q, k, v, out, dout, lse, *, scale=None, causal: bool = False, lengths=None,
                             key_mask=None, q_start=None, bias=None, buckets=None, dq=None, dk=None, dv=None,
                             dbias=None, workspace=None):
    """Gradients (dq, dk, dv, dbias; the last None without a bias) of one
    ``exact_attention_forward`` with the same arguments: ``out`` and ``lse`` are
    its results, ``dout`` the gradient of the output. The probabilities are formed
    again from the log normalisers. The same bits every time."""
    p = _exact_problem(q, k, v, scale, causal, lengths, key_mask, q_start, bias, buckets)
    _check_rows(out, q, q.shape, "out")
    _check_rows(dout, q, q.shape, "dout")
    _check_f32(lse, q.shape[:3], "lse")
    if lse.device != q.device:
        raise ValueError(f"lse must be on {q.device}")
    grads = []
    for t, g, name in ((q, dq, "dq"), (k, dk, "dk"), (v, dv, "dv")):
        if g is None:
            g = _rows_like(t)
        else:
            _check_out(g, t, name)
        grads.append(g)
    if bias is None and dbias is not None:
        raise ValueError("dbias without a bias")
    if bias is not None:
        if dbias is None:
            dbias = torch.empty_like(bias)
        elif dbias.shape != bias.shape or dbias.dtype != bias.dtype or dbias.device != bias.device \
                or not dbias.is_contiguous():
            raise ValueError("dbias must be like bias")
    if workspace is not None and (workspace.device != q.device or not workspace.is_contiguous()):
        raise ValueError(f"workspace must be a contiguous tensor on {q.device}")
    with torch.cuda.device(q.device):
        if workspace is None:
            workspace = torch.empty(max(int(load_exact().mra_exact_backward_workspace_bytes(ctypes.byref(p))), 1),
                                    device=q.device, dtype=torch.uint8)
        _call_exact("mra_exact_backward", ctypes.byref(p), *(ctypes.byref(_view(t)) for t in (q, k, v, out, dout)),
                    _ptr(lse), *(ctypes.byref(_view(t)) for t in grads), _ptr(dbias), _ptr(workspace),
                    workspace.numel() * workspace.element_size(), _stream(q.device))
    return (*grads, dbias)


_ONCE = "the gradients of exact_attention are not differentiable"


class _DifferentiatedOnce(torch.autograd.Function):
    """Gradients (the first four) as functions of what follows, whose derivatives raise."""

    @staticmethod
    def forward(ctx, *tensors):
        return tuple(None if t is None else t.detach() for t in tensors[:4])

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError(f"{_ONCE}: trying to differentiate twice")


class ExactAttention(torch.autograd.Function):
    """``exact_attention_forward`` as a differentiable op of q, k, v and bias."""

    @staticmethod
    def forward(ctx, q, k, v, bias, buckets, lengths, key_mask, q_start, scale, causal):
        lse = torch.empty(q.shape[:3], device=q.device, dtype=torch.float32)
        out = exact_attention_forward(q, k, v, scale=scale, causal=causal, lengths=lengths, key_mask=key_mask,
                                      q_start=q_start, bias=bias, buckets=buckets, lse_out=lse)
        ctx.save_for_backward(q, k, v, out, lse, bias, buckets, lengths, key_mask, q_start)
        ctx.scale, ctx.causal = scale, causal
        return out

    @staticmethod
    def backward(ctx, dout):
        if not torch.compiler.is_compiling() and torch.cuda.is_current_stream_capturing():
            bind_exact().check_capture()
        q, k, v, out, lse, bias, buckets, lengths, key_mask, q_start = ctx.saved_tensors
        with torch.no_grad():
            g = dout if _dense_rows(dout) else dout.contiguous()
            grads = exact_attention_backward(q, k, v, out, g, lse, scale=ctx.scale, causal=ctx.causal, lengths=lengths,
                                             key_mask=key_mask, q_start=q_start, bias=bias, buckets=buckets)
        if torch.is_grad_enabled():
            if dout.requires_grad:
                grads = _DifferentiatedOnce.apply(*grads, q, k, v, bias, dout)
            else:
                warnings.warn(f"{_ONCE}: these are constants of the graph")
        return (*grads, None, None, None, None, None, None)


def exact_attention(q, k, v, *, scale=None, causal: bool = False, lengths=None, key_mask=None, q_start=None,
                    bias=None, buckets=None):
    """Differentiable exact softmax attention (arguments and result as
    ``exact_attention_forward``), with gradients of q, k, v and bias, which are not
    differentiable themselves: taken with create_graph, they raise where they are
    differentiated, or warn if the output's gradient is a constant; native where ``mra_attention`` is. A backward pass
    that a graph captures needs leaves of which no eager graph is alive (with one
    on the default stream, torch's engine can end the process): a RuntimeError where
    such a leaf is an input, unseen where the inputs were computed from it."""
    tensors = (q, k, v, lengths, key_mask, q_start, bias, buckets)
    if (all(t is None or type(t) in _PLAIN for t in tensors)
            and not torch._C._are_functorch_transforms_active() and torch._C._get_tracing_state() is None
            and not torch.compiler.is_compiling()):
        return bind_exact().exact_attention(q, k, v, scale, causal, lengths, key_mask, q_start, bias, buckets)
    return ExactAttention.apply(q, k, v, bias, buckets, lengths, key_mask, q_start, scale, causal)


# ---------------------------------------------------------------------------
# Rotary positions, head norms and the 4-bit cache (include/mra_layer.h)
LAYER_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libmra_layer.so")

# name -> (restype, argtypes); mirrors include/mra_layer.h
LAYER_SIGNATURES = {
    "mra_rotary_forward": (_I, [_P] * 6),
    "mra_rotary_backward_workspace_bytes": (_Z, [_P]),
    "mra_rotary_backward": (_I, [_P] * 10 + [_Z, _P]),
    "mra_fp4_page_bytes": (_Z, [_I, _I]),
    "mra_fp4_cache_write": (_I, [_P, _P, _P, _I, _I, _P, _P, _P]),
    "mra_fp4_cache_read": (_I, [_P, _P, _P, _I, _I, _P, _P, _P]),
    "mra_fp4_attention_workspace_bytes": (_Z, [_P, _P]),
    "mra_fp4_attention": (_I, [_P] * 6 + [_Z, _P]),
    "mra_layer_last_hip_error": (_I, []),
}

_layer_lib = None
_layer_native = None    # csrc/layer_binding.cpp, bound to _layer_lib by the first call that needs it


class _LayerStatus:
    """What MraError asks of a library: the shared status texts, this library's HIP error."""

    def mra_status_str(self, status):
        return load().mra_status_str(status)

    def mra_last_hip_error(self):
        return load_layer().mra_layer_last_hip_error()


def load_layer(path: str = LAYER_LIB_PATH):
    """Open libmra_layer.so once and declare its signatures. Raises if it is missing."""
    global _layer_lib
    if _layer_lib is None:
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is not built; run `python -m paper_2207_10284_amd.build` "
                               "(hipcc, gfx950) first")
        lib = ctypes.CDLL(path)
        for name, (res, args) in LAYER_SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _layer_lib = lib
    return _layer_lib


def bind_layer():
    """The native binding of these calls (as ``bind``)."""
    global _layer_native
    if _layer_native is None:
        lib = load_layer()
        try:
            from paper_2207_10284_amd import _binding_layer
        except ImportError as e:
            raise RuntimeError(f"the torch binding is not built ({e}); run `python -m paper_2207_10284_amd.build` "
                               "first") from e
        _binding_layer.bind({name: ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in LAYER_SIGNATURES},
                            lambda fn, status: MraError(fn, status, _LayerStatus()))
        _layer_native = _binding_layer
    return _layer_native


def rotary_frequencies(rotary_dim: int, base: float = 10000.0, *, scaling: str | None = None, factor: float = 1.0,
                       original: int | None = None, device="cuda"):
    """The frequencies of rotary positions, radians a position: float64
    [rotary_dim / 2], base^(-2i / rotary_dim). ``scaling`` stretches them to contexts
    ``factor`` times as long (arXiv 2306.15595, 2309.00071): "linear" divides all by the factor; "ntk" raises
    the base so that the first stays and the last is divided; "by_parts" divides those that
    turn at most once within the ``original`` context, keeps those that turn 32 times or more, and mixes
    the two in between, linearly in the turns (with it belongs ``rotary_magnitude``). Any other
    float64 tensor serves as well."""
    rotary_dim, base, factor = int(rotary_dim), float(base), float(factor)
    if rotary_dim < 0 or rotary_dim % 16:
        raise ValueError("rotary_dim must be a multiple of 16")
    if not (1.0 < base < math.inf and 0.0 < factor < math.inf):
        raise ValueError("base must be above 1 and factor above 0")
    if scaling not in (None, "linear", "ntk", "by_parts"):
        raise ValueError(f"unknown scaling {scaling!r}")
    if scaling == "by_parts" and (original is None or original <= 0):
        raise ValueError("by_parts needs the original context")
    if scaling == "ntk":
        base *= factor ** (rotary_dim / (rotary_dim - 2))
    f = base ** (-torch.arange(0, rotary_dim, 2, dtype=torch.float64) / max(rotary_dim, 1))
    if scaling == "linear":
        f = f / factor
    elif scaling == "by_parts":
        keep = ((original / (2 * math.pi) * f - 1) / 31).clamp(0, 1)
        f = keep * f + (1 - keep) * f / factor
    return f.to(device)


def rotary_magnitude(factor: float) -> float:
    """The magnitude that belongs to "by_parts" frequencies: 0.1 ln(factor) + 1 (1 up to factor 1)."""
    return 0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0


def rotary_forward(q, k=None, freqs=None, *, positions=None, interleaved: bool = False, magnitude: float = 1.0,
                   q_weight=None, k_weight=None, eps: float = 1e-6, q_out=None, k_out=None):
    """Rotary positions of queries and keys, and before them their norms: (q', k'),
    k' None without k.

    q: [B, H, n, d], k: [B, H_kv, n, d] as in ``exact_attention``. ``freqs`` (float64
    [r / 2], r at most d: ``rotary_frequencies``) turns the first r elements of a row, in pairs i and i + r/2
    (``interleaved``: 2i and 2i + 1), by position times frequency and times ``magnitude``;
    none: no rotation. ``positions``: int32 [n] or [B, n], 0 to n - 1 if not given. With
    ``q_weight`` or ``k_weight`` ([d], float32 or q's dtype) a row x is x / sqrt(mean(x^2) + eps) times the weight
    before it is turned. ``q_out`` may be q and ``k_out`` k: changed in place; they
    overlap no other argument. A tensor given for a result, here and in the calls below, must not require a gradient (it may
    under ``torch.no_grad``), and autograd sees that it was written."""
    return bind_layer().rotary_forward(q, k, freqs, positions, interleaved, magnitude, q_weight, k_weight, eps,
                                       _result(q, q_out), k_out if k is None else _result(k, k_out))


def rotary_backward(dq_out, dk_out, q=None, k=None, freqs=None, *, positions=None, interleaved: bool = False,
                    magnitude: float = 1.0, q_weight=None, k_weight=None, eps: float = 1e-6, dq=None, dk=None):
    """Gradients (dq, dk, dq_weight, dk_weight) of one ``rotary_forward`` with the
    same arguments, for those of its results; one of ``dq_out`` and ``dk_out`` may be None, and so are
    then its gradients. q and k are needed with their weights only. ``dq`` may be ``dq_out`` and
    ``dk`` ``dk_out``. The same bits every time."""
    return bind_layer().rotary_backward(dq_out, dk_out, q, k, freqs, positions, interleaved, magnitude, q_weight,
                                        k_weight, eps, dq, dk)


_TURNED_ONCE = "the gradients of rotary are not differentiable"


class _TurnedOnce(torch.autograd.Function):
    """Gradients (the first four) as functions of what follows, whose derivatives raise."""

    @staticmethod
    def forward(ctx, *tensors):
        return tuple(None if t is None else t.detach() for t in tensors[:4])

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError(f"{_TURNED_ONCE}: trying to differentiate twice")


class Rotary(torch.autograd.Function):
    """``rotary_forward`` as a differentiable op of q, k and the weights."""

    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, freqs, positions, interleaved, magnitude, eps):
        yq, yk = rotary_forward(q, k, freqs, positions=positions, interleaved=interleaved, magnitude=magnitude,
                                q_weight=q_weight, k_weight=k_weight, eps=eps)
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(q if q_weight is not None else None, k if k_weight is not None else None, q_weight,
                              k_weight, freqs, positions)
        ctx.args = dict(interleaved=interleaved, magnitude=magnitude, eps=eps)
        return yq, yk

    @staticmethod
    def backward(ctx, gq, gk):
        if not torch.compiler.is_compiling() and torch.cuda.is_current_stream_capturing():
            bind_layer().check_capture()
        if gq is None and gk is None:
            return (None,) * 9
        q, k, q_weight, k_weight, freqs, positions = ctx.saved_tensors
        with torch.no_grad():
            rows = [None if g is None else g if _dense_rows(g) else g.contiguous() for g in (gq, gk)]
            grads = rotary_backward(*rows, q, k, freqs, positions=positions, q_weight=q_weight, k_weight=k_weight,
                                    **ctx.args)
        if torch.is_grad_enabled():
            if any(g is not None and g.requires_grad for g in (gq, gk)):
                grads = _TurnedOnce.apply(*grads, q, k, q_weight, k_weight, gq, gk)
            else:
                warnings.warn(f"{_TURNED_ONCE}: these are constants of the graph")
        return (*grads, None, None, None, None, None)


def rotary(q, k=None, freqs=None, *, positions=None, interleaved: bool = False, magnitude: float = 1.0, q_weight=None,
           k_weight=None, eps: float = 1e-6):
    """Differentiable rotary positions and head norms (arguments and result as
    ``rotary_forward``), with gradients of q, k and the weights, which are not differentiable
    themselves, and captured into graphs, as those of ``exact_attention``. Without a weight nothing of
    q and k is kept for the backward."""
    tensors = (q, k, freqs, positions, q_weight, k_weight)
    if (all(t is None or type(t) in _PLAIN for t in tensors)
            and not torch._C._are_functorch_transforms_active() and torch._C._get_tracing_state() is None
            and not torch.compiler.is_compiling()):
        return bind_layer().rotary(q, k, freqs, positions, interleaved, magnitude, q_weight, k_weight, eps)
    return Rotary.apply(q, k, q_weight, k_weight, freqs, positions, interleaved, magnitude, eps)


class Fp4Cache:
    """A paged cache of keys and values in 4 bits: ``data`` (uint8 [pages, H_kv,
    page bytes] on the device, include/mra_layer.h has its layout), ``page_size`` tokens a page, head width ``d``.
    Pages may be copied, moved and shared whole."""
    __slots__ = ("data", "page_size", "d")

    def __init__(self, data, page_size: int, d: int):
        page_size, d = int(page_size), int(d)
        if not (need := fp4_page_bytes(page_size, d)):
            raise ValueError("page_size must be 32, 64, .. 1024 and d 32, 64 or 128")
        if data.dtype != torch.uint8 or data.dim() != 3 or data.shape[2] != need or not data.is_contiguous():
            raise ValueError(f"data must be a contiguous uint8 tensor [pages, H_kv, {need}]")
        self.data, self.page_size, self.d = data, page_size, d

    def _args(self):
        return self.data, self.page_size, self.d


def fp4_page_bytes(page_size: int, d: int) -> int:
    """Bytes of one page of one head: 17/32 byte a value (0: sizes that are not supported)."""
    if not (0 <= page_size < 1 << 31 and 0 <= d < 1 << 31):      # what the library's integers hold
        return 0
    return int(load_layer().mra_fp4_page_bytes(page_size, d))


def fp4_cache(pages: int, kv_heads: int, page_size: int, d: int, device="cuda") -> Fp4Cache:
    """An empty cache of ``pages`` pages (all values 0). page_size: a power of two from 32 to 1024."""
    if not (need := fp4_page_bytes(page_size, d)):
        raise ValueError("page_size must be 32, 64, .. 1024 and d 32, 64 or 128")
    return Fp4Cache(torch.zeros(pages, kv_heads, need, dtype=torch.uint8, device=device), page_size, d)


def fp4_cache_write(cache: Fp4Cache, k, v, table, *, starts=None, counts=None) -> None:
    """Writes the first ``counts[b]`` (all if not given) tokens of sequence b to its
    places from ``starts[b]`` (0) on.

    k, v: [B, H_kv, n, d], float32 or bfloat16, any strides with dense 16-byte aligned
    rows. ``table`` (int32 [B, m]): the pages of each sequence; place t is in its page
    t // page_size. ``starts``, ``counts``: int32 [B]. Places beyond the table or in an entry that is no page (-1) are not
    written. 32 consecutive channels share a power-of-two step, the smallest with
    their largest magnitude at most 7 steps; a value is held as the nearest of 0, 1/2, 1, 3/2, 2, 3, 4
    and 6 steps, ties to the even one in this order. Only the written tokens' bytes change. Two sequences that write to one place leave
    either's values, or a mix."""
    bind_layer().cache_write(*cache._args(), k, v, table, starts, counts)


def fp4_cache_read(cache: Fp4Cache, table, n: int, *, starts=None, counts=None, dtype=torch.bfloat16, k_out=None,
                   v_out=None):
    """The values held for the first ``counts[b]`` (n) tokens from place ``starts[b]``
    (0) on: (k, v), [B, H_kv, n, d] of ``dtype`` (float32 or bfloat16: exact in either); 0
    behind them and where there is no page. Arguments as in ``fp4_cache_write``."""
    return bind_layer().cache_read(*cache._args(), table, n, starts, counts, dtype, k_out, v_out)


def fp4_attention_workspace_bytes(q, cache: Fp4Cache, table, lengths) -> int:
    """Workspace of ``fp4_cache_attention`` for these arguments (0: none)."""
    return int(bind_layer().attention_workspace(*cache._args(), q, table, lengths))


def fp4_cache_attention(q, cache: Fp4Cache, table, lengths, *, scale=None, causal: bool = False, q_start=None,
                        out=None, lse_out=None, workspace=None):
    """Softmax attention softmax(scale q k^T) v of q [B, H, n_q, d] over the first
    ``lengths[b]`` (int32 [B]) tokens that the cache holds for each sequence; query
    head h reads key head h // (H / H_kv). Query i stands at ``q_start[b] + i`` (int32 [B];
    lengths[b] - n_q + i if not given) and with ``causal`` sees the tokens up to there. Tokens in an
    entry of the table that is no page do not count; a query for which none counts gives zeros, another that holds a NaN or an infinity NaN. ``scale``, ``out``, ``lse_out`` and
    ``workspace`` as in ``exact_attention_forward``. Not differentiable."""
    return bind_layer().attention(*cache._args(), q, table, lengths, scale, causal, q_start, _result(q, out), lse_out,
                                  workspace)
