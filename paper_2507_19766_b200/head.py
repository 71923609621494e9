"""Token scores and distillation on the LM head: argument checks and marshalling for libulorl.so.

token_scores       log-prob of given tokens, entropy and the most likely alternatives from hidden states and W
                   (what a rollout records as old_logp, a reference policy as ref_logp, a teacher for its student)
token_scores_bwd   gradients of a caller's loss on those log-probs and entropies
logits_scores      the same scores from logits that are already there (a decoding step)
distill_fwd/_bwd   distillation from a teacher's top logits

Calls run on the current stream of the tensors' device and never synchronise; findings of the kernels are read with
binding.check_status(workspace).  There is no CPU path.
"""
from __future__ import annotations

import contextlib
import ctypes
from dataclasses import dataclass
from typing import Optional

import torch

from .binding import BF16, F32, OK, CHeadParams, UlorlError, _PATH, load_library, status_string

MAX_TOP, MAX_LIST = 32, 128
_MAX_SIZE = 1 << 30
_DISTILL = {"raw": 0, "renorm": 1, "tail": 2}
_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_LOGITS = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: 2}


@dataclass
class HeadParams:
    """Mirror of ulorl_head_params_t.  top_k: alternatives that token_scores returns, or entries of a teacher's list."""
    T: int
    H: int
    V: int
    dtype: str = "bf16"
    top_k: int = 0
    kernel_path: str = "auto"
    inv_temperature: float = 1.0
    bwd_panel_tokens: int = 0
    dw_accumulate: bool = False
    dw_dtype: str = "f32"
    distill_mode: str = "raw"
    teacher_inv_temperature: float = 1.0
    norm_tokens: int = 0

    def to_c(self) -> CHeadParams:
        for name, value, known in (("dtype", self.dtype, _DTYPES), ("dw_dtype", self.dw_dtype, _DTYPES),
                                   ("kernel_path", self.kernel_path, _PATH), ("distill_mode", self.distill_mode, _DISTILL)):
            if value not in known:
                raise UlorlError(f"{name}: {value!r} is not one of {sorted(known)}")
        if self.T > _MAX_SIZE or self.H > _MAX_SIZE or self.V > _MAX_SIZE or self.top_k > MAX_LIST or self.bwd_panel_tokens > _MAX_SIZE:
            raise UlorlError(f"sizes beyond {_MAX_SIZE} (top_k {MAX_LIST}) are not supported")      # the C side takes 32 bits
        return CHeadParams(self.T, self.H, self.V, BF16 if self.dtype == "bf16" else F32, self.top_k,
                           _PATH[self.kernel_path], self.inv_temperature, self.bwd_panel_tokens, int(self.dw_accumulate),
                           BF16 if self.dw_dtype == "bf16" else F32, _DISTILL[self.distill_mode],
                           self.teacher_inv_temperature, self.norm_tokens)


@dataclass
class ScoresOut:
    logp: Optional[torch.Tensor]         # [T], None without targets
    entropy: torch.Tensor                # [T]
    lse: torch.Tensor                    # [T]
    norm: Optional[torch.Tensor]         # [T, 2], read by token_scores_bwd; None from logits_scores
    top_ids: Optional[torch.Tensor]      # [T, top_k] int32, None with top_k = 0
    top_logp: Optional[torch.Tensor]     # [T, top_k]


@dataclass
class DistillOut:
    loss: torch.Tensor                   # [1]
    kl: torch.Tensor                     # [T]
    lse: torch.Tensor                    # [T]
    norm: torch.Tensor                   # [T, 2], and with it for distill_bwd:
    coef: torch.Tensor                   # [T]
    entry_grad: torch.Tensor             # [T, top_k]


def _raise(code: int, what: str):
    raise UlorlError(f"{what} failed: {status_string(code)} ({code})")


def _take(t: Optional[torch.Tensor], name: str, dtype, n: int, device: int, optional: bool = False):
    """The tensor's device pointer, after the checks that keep the kernels inside it."""
    if t is None:
        if optional:
            return None
        raise UlorlError(f"{name} is missing")
    if t.dtype != dtype or t.numel() != n:
        raise UlorlError(f"{name}: expected {n} elements of {dtype}, got {t.numel()} of {t.dtype}")
    if not t.is_cuda or t.get_device() != device or not t.is_contiguous():
        raise UlorlError(f"{name}: expected a contiguous tensor on cuda:{device}")
    return t.data_ptr()


def _device_of(t: torch.Tensor, name: str) -> int:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise UlorlError(f"{name}: expected a CUDA tensor (there is no CPU path)")
    return t.get_device()


def _elsewhere(device: int) -> bool:
    """Whether the tensors' device is not the current one: the call then repeats itself with it made current."""
    return device != torch.cuda.current_device()


def _stream(device: int) -> int:
    return torch._C._cuda_getCurrentRawStream(device)


def head_workspace_bytes(p: HeadParams, backward: bool = True) -> int:
    n = load_library().ulorl_head_workspace_bytes(ctypes.byref(p.to_c()), int(backward))
    if n == 0:
        raise UlorlError("ulorl_head_workspace_bytes: invalid parameters")
    return int(n)


def alloc_head_workspace(p: HeadParams, device, backward: bool = True) -> torch.Tensor:
    """Scratch of the calls with these params; backward=False is enough (and far smaller) for the forward ones."""
    device = torch.device(device)
    with contextlib.nullcontext() if device.index is None else torch.cuda.device(device):
        # sizes go by the device's multiprocessor count
        workspace = torch.empty(head_workspace_bytes(p, backward), dtype=torch.uint8, device=device)
        workspace[:256].zero_()                              # the status word: backward calls only add to it
        return workspace


def _workspace(lib, cp: CHeadParams, workspace, hidden, device: int, backward: bool):
    """(tensor to keep, pointer, bytes); allocates for this call where the caller keeps none."""
    if workspace is None:
        n = lib.ulorl_head_workspace_bytes(ctypes.byref(cp), int(backward))
        if n == 0:
            raise UlorlError("ulorl_head_workspace_bytes: invalid parameters")
        workspace = torch.empty(n, dtype=torch.uint8, device=hidden.device)
        return workspace, workspace.data_ptr(), n
    if not workspace.is_cuda or workspace.get_device() != device or not workspace.is_contiguous():
        raise UlorlError(f"workspace: expected a contiguous tensor on cuda:{device}")
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _operands(p: HeadParams, hidden, W):
    device = _device_of(hidden, "hidden")
    dtype = _DTYPES.get(p.dtype)
    return device, _take(hidden, "hidden", dtype, p.T * p.H, device), _take(W, "W", dtype, p.V * p.H, device)


def _alternatives(T: int, k: int, like: torch.Tensor):
    if k <= 0:
        return None, None
    return (torch.empty((T, k), dtype=torch.int32, device=like.device), torch.empty((T, k), dtype=torch.float32, device=like.device))


def token_scores(p: HeadParams, hidden, W, targets=None, out: Optional[ScoresOut] = None,
                 workspace: Optional[torch.Tensor] = None) -> ScoresOut:
    """ulorl_token_scores on the current stream of the tensors' device."""
    lib = load_library()
    cp = p.to_c()
    device, ph, pw = _operands(p, hidden, W)
    if _elsewhere(device):
        with torch.cuda.device(device):
            return token_scores(p, hidden, W, targets, out, workspace)
    f32, T, k = torch.float32, p.T, p.top_k
    pt = _take(targets, "targets", torch.int32, T, device, optional=True)
    if out is None:
        logp, entropy, lse = torch.empty((3, T), dtype=f32, device=hidden.device).unbind(0)
        out = ScoresOut(None if targets is None else logp, entropy, lse,
                        torch.empty((T, 2), dtype=f32, device=hidden.device), *_alternatives(T, k, hidden))
        ptrs = [None if x is None else x.data_ptr() for x in (out.logp, entropy, lse, out.norm, out.top_ids, out.top_logp)]
    else:
        ptrs = [_take(out.logp, "logp", f32, T, device, targets is None), _take(out.entropy, "entropy", f32, T, device, True),
                _take(out.lse, "lse", f32, T, device, True), _take(out.norm, "norm", f32, 2 * T, device, True),
                _take(out.top_ids, "top_ids", torch.int32, T * k, device, k == 0),
                _take(out.top_logp, "top_logp", f32, T * k, device, k == 0)]
    workspace, pws, nws = _workspace(lib, cp, workspace, hidden, device, False)
    code = lib.ulorl_token_scores(ctypes.byref(cp), ph, pw, pt, *ptrs, pws, nws, _stream(device))
    if code != OK:
        _raise(code, "ulorl_token_scores")
    return out


def _grad_outputs(p: HeadParams, d_hidden, d_W, hidden, device: int):
    if d_hidden is None:
        d_hidden = torch.empty_like(hidden)
    if d_W is None:
        d_W = (torch.zeros if p.dw_accumulate else torch.empty)((p.V, p.H), dtype=_DTYPES[p.dw_dtype], device=hidden.device)
    return (d_hidden, d_W, _take(d_hidden, "d_hidden", _DTYPES[p.dtype], p.T * p.H, device),
            _take(d_W, "d_W", _DTYPES[p.dw_dtype], p.V * p.H, device))


def token_scores_bwd(p: HeadParams, hidden, W, targets, scores: ScoresOut, d_logp=None, d_entropy=None, d_hidden=None,
                     d_W=None, workspace: Optional[torch.Tensor] = None):
    """ulorl_token_scores_bwd: (d_hidden, d_W) for d loss / d logp and d loss / d entropy (None = zero), given what
    token_scores returned for the same operands."""
    lib = load_library()
    cp = p.to_c()
    device, ph, pw = _operands(p, hidden, W)
    if _elsewhere(device):
        with torch.cuda.device(device):
            return token_scores_bwd(p, hidden, W, targets, scores, d_logp, d_entropy, d_hidden, d_W, workspace)
    f32, T = torch.float32, p.T
    d_hidden, d_W, pdh, pdw = _grad_outputs(p, d_hidden, d_W, hidden, device)
    workspace, pws, nws = _workspace(lib, cp, workspace, hidden, device, True)
    code = lib.ulorl_token_scores_bwd(
        ctypes.byref(cp), ph, pw, _take(targets, "targets", torch.int32, T, device, d_logp is None),
        _take(scores.norm, "norm", f32, 2 * T, device), _take(scores.logp, "logp", f32, T, device, d_logp is None),
        _take(scores.entropy, "entropy", f32, T, device, d_entropy is None),
        _take(d_logp, "d_logp", f32, T, device, True), _take(d_entropy, "d_entropy", f32, T, device, True),
        pdh, pdw, pws, nws, _stream(device))
    if code != OK:
        _raise(code, "ulorl_token_scores_bwd")
    return d_hidden, d_W


def logits_scores(logits: torch.Tensor, targets=None, top_k: int = 0, inv_temperature: float = 1.0,
                  out: Optional[ScoresOut] = None) -> ScoresOut:
    """ulorl_logits_scores: scores from logits [T, V] (float32, bfloat16 or float16; rows may be strided)."""
    # a decoding step's call is mostly what the host does: few allocations, no more checks than the kernel needs
    lib = load_library()
    device = _device_of(logits, "logits")
    code = _LOGITS.get(logits.dtype)
    if code is None or logits.dim() != 2 or logits.shape[1] == 0:
        raise UlorlError("logits: expected float32, bfloat16 or float16 [T, V]")
    T, V = logits.shape
    ld, step = logits.stride()
    if T <= 1:
        ld = V
    if T > _MAX_SIZE or V > _MAX_SIZE:
        raise UlorlError(f"logits: sizes beyond {_MAX_SIZE} are not supported")
    if (V > 1 and step != 1) or ld < V:
        raise UlorlError("logits: a row must be contiguous and rows must not overlap")
    if _elsewhere(device):
        with torch.cuda.device(device):
            return logits_scores(logits, targets, top_k, inv_temperature, out)
    f32, k = torch.float32, top_k
    pt = _take(targets, "targets", torch.int32, T, device, optional=True)
    if out is None:
        logp, entropy, lse = torch.empty((3, T), dtype=f32, device=logits.device).unbind(0)
        ids, top_logp = _alternatives(T, k, logits)
        if targets is None:
            logp = None
        code = lib.ulorl_logits_scores(logits.data_ptr(), code, T, V, ld, k, inv_temperature, pt,
                                       None if logp is None else logp.data_ptr(), entropy.data_ptr(), lse.data_ptr(),
                                       ids.data_ptr() if k > 0 else None, top_logp.data_ptr() if k > 0 else None, _stream(device))
        out = ScoresOut(logp, entropy, lse, None, ids, top_logp)
    else:
        code = lib.ulorl_logits_scores(
            logits.data_ptr(), code, T, V, ld, k, inv_temperature, pt,
            _take(out.logp, "logp", f32, T, device, targets is None), _take(out.entropy, "entropy", f32, T, device, True),
            _take(out.lse, "lse", f32, T, device, True), _take(out.top_ids, "top_ids", torch.int32, T * k, device, k <= 0),
            _take(out.top_logp, "top_logp", f32, T * k, device, k <= 0), _stream(device))
    if code != OK:
        _raise(code, "ulorl_logits_scores")
    return out


def selftest_logits_wait(logits: torch.Tensor, top_k: int, workspace: torch.Tensor, limit_cycles: int = 1_000_000) -> ScoresOut:
    """ulorl_selftest_logits_wait on float32 logits [T, V]: lse and alternatives of a kernel whose waits ran out; the timeout
    shows up in binding.check_status(workspace)."""
    device = _device_of(logits, "logits")
    T, V = logits.shape
    pl, pws = _take(logits, "logits", torch.float32, T * V, device), _take(workspace, "workspace", torch.uint8, workspace.numel(), device)
    lse, (ids, top_logp) = torch.empty(T, device=logits.device), _alternatives(T, top_k, logits)
    with torch.cuda.device(device):
        code = load_library().ulorl_selftest_logits_wait(pl, T, V, top_k, lse.data_ptr(), None if ids is None else ids.data_ptr(),
                                                         None if ids is None else top_logp.data_ptr(), pws, limit_cycles, _stream(device))
    if code != OK:
        _raise(code, "ulorl_selftest_logits_wait")
    return ScoresOut(None, None, lse, None, ids, top_logp)


def distill_fwd(p: HeadParams, hidden, W, teacher_ids, teacher_logp, weights=None, out: Optional[DistillOut] = None,
                workspace: Optional[torch.Tensor] = None) -> DistillOut:
    """ulorl_distill_fwd: loss of the student's softmax against the teacher's top_k entries per token."""
    lib = load_library()
    cp = p.to_c()
    device, ph, pw = _operands(p, hidden, W)
    if _elsewhere(device):
        with torch.cuda.device(device):
            return distill_fwd(p, hidden, W, teacher_ids, teacher_logp, weights, out, workspace)
    f32, T, k = torch.float32, p.T, p.top_k
    pi = _take(teacher_ids, "teacher_ids", torch.int32, T * k, device)
    pl = _take(teacher_logp, "teacher_logp", f32, T * k, device)
    pwt = _take(weights, "weights", f32, T, device, optional=True)
    if out is None:
        kl, lse, coef = torch.empty((3, T), dtype=f32, device=hidden.device).unbind(0)
        out = DistillOut(torch.empty(1, dtype=f32, device=hidden.device), kl, lse,
                         torch.empty((T, 2), dtype=f32, device=hidden.device), coef,
                         torch.empty((T, max(k, 0)), dtype=f32, device=hidden.device))
        ptrs = [x.data_ptr() for x in (out.loss, kl, lse, out.norm, coef, out.entry_grad)]
    else:
        ptrs = [_take(out.loss, "loss", f32, 1, device), _take(out.kl, "kl", f32, T, device), _take(out.lse, "lse", f32, T, device, True),
                _take(out.norm, "norm", f32, 2 * T, device), _take(out.coef, "coef", f32, T, device),
                _take(out.entry_grad, "entry_grad", f32, T * k, device)]
    workspace, pws, nws = _workspace(lib, cp, workspace, hidden, device, False)
    code = lib.ulorl_distill_fwd(ctypes.byref(cp), ph, pw, pi, pl, pwt, *ptrs, pws, nws, _stream(device))
    if code != OK:
        _raise(code, "ulorl_distill_fwd")
    return out


def distill_bwd(p: HeadParams, hidden, W, teacher_ids, fwd: DistillOut, grad_loss=None, d_hidden=None, d_W=None,
                workspace: Optional[torch.Tensor] = None):
    """ulorl_distill_bwd: (d_hidden, d_W) given what distill_fwd returned for the same operands."""
    lib = load_library()
    cp = p.to_c()
    device, ph, pw = _operands(p, hidden, W)
    if _elsewhere(device):
        with torch.cuda.device(device):
            return distill_bwd(p, hidden, W, teacher_ids, fwd, grad_loss, d_hidden, d_W, workspace)
    f32, T, k = torch.float32, p.T, p.top_k
    d_hidden, d_W, pdh, pdw = _grad_outputs(p, d_hidden, d_W, hidden, device)
    workspace, pws, nws = _workspace(lib, cp, workspace, hidden, device, True)
    code = lib.ulorl_distill_bwd(
        ctypes.byref(cp), ph, pw, _take(teacher_ids, "teacher_ids", torch.int32, T * k, device),
        _take(fwd.norm, "norm", f32, 2 * T, device), _take(fwd.coef, "coef", f32, T, device),
        _take(fwd.entry_grad, "entry_grad", f32, T * k, device), _take(grad_loss, "grad_loss", f32, 1, device, True),
        pdh, pdw, pws, nws, _stream(device))
    if code != OK:
        _raise(code, "ulorl_distill_bwd")
    return d_hidden, d_W
