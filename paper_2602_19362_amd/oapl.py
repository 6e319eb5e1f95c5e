"""ctypes binding of liboapl_hip.so (the C ABI declared in include/oapl.h).

Argument marshalling only: every step of the path runs in the library's HIP
kernels.  PyTorch supplies device memory and the current HIP stream.  There is
no fallback: if the shared library has not been built, or no GPU is present,
the calls raise.
"""
from __future__ import annotations

import array
import ctypes
import os
from typing import NamedTuple, Optional

import torch

_LIB_NAME = "liboapl_hip.so"
_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), _LIB_NAME)

OAPL_F32 = 0
OAPL_BF16 = 1
OAPL_FLAG_TWO_PASS = 1

STATUS_NAMES = {
    0: "OAPL_OK", 1: "OAPL_ERR_NULL", 2: "OAPL_ERR_SHAPE", 3: "OAPL_ERR_DTYPE", 4: "OAPL_ERR_OFFSETS",
    5: "OAPL_ERR_GROUP", 6: "OAPL_ERR_BETA", 7: "OAPL_ERR_WORKSPACE", 8: "OAPL_ERR_HIP", 9: "OAPL_ERR_TOKEN_RANGE",
    10: "OAPL_ERR_SCRATCH_LIMIT", 11: "OAPL_ERR_ALIGN",
}

# Every symbol include/oapl.h declares, with its ctypes signature.
_c = ctypes


class Heads(ctypes.Structure):
    """oapl_heads: an operand [tokens][heads][channels], strides in elements."""

    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class Rows(ctypes.Structure):
    """oapl_rows: an operand [rows][channels], the stride in elements."""

    _fields_ = [("data", ctypes.c_void_p), ("row_stride", ctypes.c_int64)]


class Tensor(ctypes.Structure):
    """oapl_tensor: a dense tensor and where its result goes."""

    _fields_ = [("data", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_int64), ("dtype", ctypes.c_int32)]


_H = ctypes.POINTER(Heads)
_R = ctypes.POINTER(Rows)
_SIGNATURES = {
    "oapl_status_string": (_c.c_char_p, [_c.c_int32]),
    "oapl_workspace_bytes": (_c.c_size_t, [_c.c_int64, _c.c_int32, _c.c_int32, _c.c_int32, _c.c_int32, _c.c_int32,
                                           _c.c_int32]),
    "oapl_workspace_bytes_for": (_c.c_size_t, [_c.c_int64, _c.c_int32, _c.c_int32, _c.c_int32, _c.c_int32,
                                               _c.c_int32, _c.c_int32, _c.c_int64, _c.c_int64,
                                               _c.POINTER(_c.c_int64), _c.POINTER(_c.c_int32)]),
    "oapl_logprob_fwd": (_c.c_int32, [_c.c_void_p, _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int32, _c.c_int32,
                                      _c.c_int32, _c.c_void_p, _c.c_void_p, _c.c_void_p, _c.c_void_p, _c.c_size_t,
                                      _c.c_void_p]),
    "oapl_sample_tokens": (_c.c_int32, [_c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int32, _c.c_int32, _c.c_int32,
                                        _c.c_float, _c.c_uint64, _c.c_void_p, _c.c_void_p, _c.c_void_p, _c.c_size_t,
                                        _c.c_void_p]),
    "oapl_loss_fwd_bwd": (_c.c_int32, [_c.c_void_p] * 7 + [_c.c_int64] + [_c.c_int32] * 5 + [_c.c_float] * 2 +
                          [_c.c_void_p] * 7 + [_c.c_size_t, _c.c_void_p]),
    "oapl_loss_fwd_bwd_two_beta": (_c.c_int32, [_c.c_void_p] * 7 + [_c.c_int64] + [_c.c_int32] * 5 + [_c.c_float] * 3 +
                                   [_c.c_uint32] + [_c.c_void_p] * 7 + [_c.c_size_t, _c.c_void_p]),
    "oapl_loss_fwd_bwd_noalloc": (_c.c_int32, [_c.c_void_p] * 7 + [_c.c_int64] + [_c.c_int32] * 5 + [_c.c_float] * 2 +
                                  [_c.c_void_p] * 7),
    "oapl_grpo_loss_fwd_bwd": (_c.c_int32, [_c.c_void_p] * 8 + [_c.c_int64] + [_c.c_int32] * 5 + [_c.c_float] * 3 +
                               [_c.c_uint32] + [_c.c_void_p] * 6 + [_c.c_size_t, _c.c_void_p]),
    "oapl_segmented_sum_f32": (_c.c_int32, [_c.c_void_p, _c.c_void_p, _c.c_int32, _c.c_void_p, _c.c_void_p]),
    "oapl_qk_norm_rope_fwd": (_c.c_int32, [_H] * 3 + [_c.c_void_p] * 5 + [_c.c_int64] + [_c.c_int32] * 4 + [_c.c_int64] * 2 +
                              [_c.c_int32, _c.c_float] + [_H] * 3 + [_c.c_void_p]),
    "oapl_qk_norm_rope_workspace_bytes": (_c.c_size_t, [_c.c_int64] + [_c.c_int32] * 3),
    "oapl_qk_norm_rope_bwd": (_c.c_int32, [_H] * 4 + [_c.c_void_p] * 4 + [_c.c_int64] + [_c.c_int32] * 4 + [_c.c_int64] +
                              [_c.c_int32, _c.c_float] + [_H] * 2 + [_c.c_void_p] * 3 + [_c.c_size_t, _c.c_void_p]),
    "oapl_attention_workspace_bytes": (_c.c_size_t, [_c.c_int64] * 2 + [_c.c_int32] * 6),
    "oapl_attention_fwd": (_c.c_int32, [_H] * 3 + [_c.c_void_p] * 3 + [_c.c_int64] * 2 + [_c.c_int32] * 6 +
                           [_c.c_float, _H] + [_c.c_void_p] * 2 + [_c.c_size_t, _c.c_void_p]),
    "oapl_attention_bwd": (_c.c_int32, [_H] * 4 + [_c.c_void_p, _H] + [_c.c_void_p] * 2 + [_c.c_int64] * 2 + [_c.c_int32] * 6 +
                           [_c.c_float] + [_H] * 3 + [_c.c_void_p, _c.c_size_t, _c.c_void_p]),
    "oapl_embed_fwd": (_c.c_int32, [_c.c_void_p] * 2 + [_c.c_int64] + [_c.c_int32] * 4 + [_c.c_float, _R, _c.c_void_p]),
    "oapl_embed_workspace_bytes": (_c.c_size_t, [_c.c_int64] + [_c.c_int32] * 2),
    "oapl_embed_bwd": (_c.c_int32, [_R, _c.c_void_p, _c.c_int64] + [_c.c_int32] * 3 + [_c.c_float, _c.c_int32] + [_c.c_void_p] * 2 +
                       [_c.c_size_t, _c.c_void_p]),
    "oapl_residual_norm_fwd": (_c.c_int32, [_R, _R, _c.c_void_p, _R, _c.c_int32, _c.c_void_p, _c.c_int64] + [_c.c_int32] * 3 +
                               [_c.c_float] * 2 + [_R, _R, _c.c_void_p]),
    "oapl_residual_norm_workspace_bytes": (_c.c_size_t, [_c.c_int64, _c.c_int32]),
    "oapl_residual_norm_bwd": (_c.c_int32, [_R, _R, _c.c_void_p, _R, _c.c_int32, _c.c_void_p, _R, _R, _c.c_int64] + [_c.c_int32] * 3 +
                               [_c.c_float] * 2 + [_R, _R] + [_c.c_void_p] * 2 + [_R] + [_c.c_void_p] * 2 + [_c.c_size_t, _c.c_void_p]),
    "oapl_clip_workspace_bytes": (_c.c_size_t, [_c.c_int32]),
    "oapl_grad_norm": (_c.c_int32, [_c.c_void_p, _c.c_int32] + [_c.c_void_p] * 2 + [_c.c_size_t, _c.c_void_p]),
    "oapl_clip_grads": (_c.c_int32, [_c.c_void_p, _c.c_int32, _c.c_float] + [_c.c_void_p] * 3 + [_c.c_size_t, _c.c_void_p]),
    "oapl_read_device_status": (_c.c_int32, [_c.c_void_p, _c.c_void_p, _c.POINTER(_c.c_int32)]),
    "oapl_read_path_taken": (_c.c_int32, [_c.c_void_p, _c.c_void_p, _c.POINTER(_c.c_int32)]),
    "oapl_timing_enable": (_c.c_int32, [_c.c_int32]),
    "oapl_timing_read": (_c.c_int32, [_c.c_int32, _c.POINTER(_c.c_double), _c.POINTER(_c.c_int64)]),
}

DENSE_KERNELS = ("k_fwd_lse", "k_bwd_dz", "k_bwd_dh", "k_bwd_dw", "k_fwd_sample", "k_sweep")

_lib = None


class OaplError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = STATUS_NAMES.get(status, str(status))
        try:
            msg += ": " + lib().oapl_status_string(status).decode()
        except Exception:
            pass
        super().__init__(f"{where} failed with {msg}")


def lib_path() -> str:
    return _LIB_PATH


def lib():
    """Loads the shared library once; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(
                f"{_LIB_PATH} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()'). "
                "There is no CPU fallback.")
        handle = ctypes.CDLL(_LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _lib = handle
    return _lib


_CODES = {torch.float32: OAPL_F32, torch.bfloat16: OAPL_BF16}


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return OAPL_F32
    if t.dtype == torch.bfloat16:
        return OAPL_BF16
    raise TypeError(f"H and W must be float32 or bfloat16, got {t.dtype}")


def _dev(t: Optional[torch.Tensor], dtype: torch.dtype, name: str, device) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda or t.device != device:
        raise ValueError(f"{name} must live on {device}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _stream(device) -> int:
    return torch.cuda.current_stream(device).cuda_stream


# The same number without a stream object around it, where this torch has it (2 us less on calls that take 10).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: _stream(torch.device("cuda", index)))
_current_gpu = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device      # of a process that has a GPU tensor


def workspace_bytes(T: int, d: int, V: int, n_seq: int, n_groups: int, dtype: int, with_backward: bool,
                    max_panel_rows: Optional[int] = None, max_rollout_len: Optional[int] = None) -> int:
    """oapl_workspace_bytes, or oapl_workspace_bytes_for when a panel cap or a rollout length is given."""
    if max_panel_rows is None and max_rollout_len is None:
        return int(lib().oapl_workspace_bytes(T, d, V, n_seq, n_groups, dtype, 1 if with_backward else 0))
    return workspace_bytes_for(T, d, V, n_seq, n_groups, dtype, with_backward, max_panel_rows or 0,
                               max_rollout_len or 0)[0]


def workspace_bytes_for(T: int, d: int, V: int, n_seq: int, n_groups: int, dtype: int, with_backward: bool,
                        max_panel_rows: int = 0, max_rollout_len: int = 0):
    """oapl_workspace_bytes_for: (bytes, panel rows, panel buffers) of the plan."""
    rows = ctypes.c_int64(0)
    bufs = ctypes.c_int32(0)
    n = lib().oapl_workspace_bytes_for(T, d, V, n_seq, n_groups, dtype, 1 if with_backward else 0,
                                       int(max_panel_rows), int(max_rollout_len), ctypes.byref(rows),
                                       ctypes.byref(bufs))
    return int(n), int(rows.value), int(bufs.value)


def _workspace(nbytes: int, device, workspace: Optional[torch.Tensor]) -> torch.Tensor:
    if workspace is None:
        workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
    if workspace.dtype != torch.uint8 or not workspace.is_contiguous() or workspace.device != device:
        raise ValueError("workspace must be a contiguous uint8 tensor on the inputs' device")
    return workspace


def _panel_rows(H: torch.Tensor, W: torch.Tensor, max_panel_rows: Optional[int]) -> Optional[int]:
    """The panel cap to size a loss call's workspace for: less than a bf16 tile asks for the least workspace, which has no
    room for the copies that operands off 16-byte alignment need, so for those it is a whole tile."""
    if max_panel_rows is not None and 0 < max_panel_rows < 384 and H.dtype == torch.bfloat16 \
            and (H.data_ptr() | W.data_ptr()) % 16:
        return 384
    return max_panel_rows


def read_device_status(workspace: torch.Tensor) -> int:
    out = ctypes.c_int32(0)
    rc = lib().oapl_read_device_status(workspace.data_ptr(), _stream(workspace.device), ctypes.byref(out))
    if rc != 0:
        raise OaplError(rc, "oapl_read_device_status")
    return int(out.value)


def took_two_passes(workspace: torch.Tensor) -> bool:
    """oapl_read_path_taken: True if the last loss call on this workspace fell back to the two-pass schedule."""
    out = ctypes.c_int32(0)
    rc = lib().oapl_read_path_taken(workspace.data_ptr(), _stream(workspace.device), ctypes.byref(out))
    if rc != 0:
        raise OaplError(rc, "oapl_read_path_taken")
    return bool(out.value)


def _check_device(t: torch.Tensor) -> None:
    """The C ABI works on the current HIP device: the inputs must live there."""
    if not t.is_cuda:
        raise ValueError("inputs must be device tensors (there is no CPU path)")
    if t.device.index != torch.cuda.current_device():
        raise ValueError(f"inputs live on {t.device} but the current device is cuda:{torch.cuda.current_device()}; "
                         "wrap the call in torch.cuda.device(...)")


def logprob_fwd(H: torch.Tensor, W: torch.Tensor, tokens: torch.Tensor, *, want_lse: bool = False,
                want_entropy: bool = False, workspace: Optional[torch.Tensor] = None):
    """oapl_logprob_fwd: per-token log-probs of the sampled tokens (and lse, and the policy entropy).

    Returns (logprob, [lse], [entropy], workspace) with the optional items present when asked for.
    """
    L = lib()
    _check_device(H)
    dt = _dtype_code(H)
    T, d = H.shape
    V = W.shape[0]
    if W.shape[1] != d or tokens.shape != (T,):
        raise ValueError("shape mismatch between H, W and tokens")
    dev = H.device
    nbytes = workspace_bytes(T, d, V, 0, 1, dt, False)
    if nbytes == 0:
        raise OaplError(2, "oapl_workspace_bytes")
    ws = _workspace(nbytes, dev, workspace)
    logprob = torch.empty(T, dtype=torch.float32, device=dev)
    lse = torch.empty(T, dtype=torch.float32, device=dev) if want_lse else None
    ent = torch.empty(T, dtype=torch.float32, device=dev) if want_entropy else None
    rc = L.oapl_logprob_fwd(_dev(H, H.dtype, "H", dev), _dev(W, H.dtype, "W", dev),
                            _dev(tokens, torch.int32, "tokens", dev), T, d, V, dt, logprob.data_ptr(),
                            lse.data_ptr() if want_lse else None, ent.data_ptr() if want_entropy else None,
                            ws.data_ptr(), ws.numel(), _stream(dev))
    if rc != 0:
        raise OaplError(rc, "oapl_logprob_fwd")
    return tuple(x for x in (logprob, lse, ent) if x is not None) + (ws,)


def sample_tokens(H: torch.Tensor, W: torch.Tensor, temperature: float, seed: int, *, want_scores: bool = False,
                  workspace: Optional[torch.Tensor] = None):
    """oapl_sample_tokens: one Gumbel-max draw per row from softmax(H W^T / temperature)."""
    _check_device(H)
    dt = _dtype_code(H)
    T, d = H.shape
    V = W.shape[0]
    if W.shape[1] != d:
        raise ValueError("shape mismatch between H and W")
    dev = H.device
    nbytes = workspace_bytes(T, d, V, 0, 1, dt, False)
    if nbytes == 0:
        raise OaplError(2, "oapl_workspace_bytes")
    ws = _workspace(nbytes, dev, workspace)
    tokens = torch.empty(T, dtype=torch.int32, device=dev)
    scores = torch.empty(T, dtype=torch.float32, device=dev) if want_scores else None
    rc = lib().oapl_sample_tokens(_dev(H, H.dtype, "H", dev), _dev(W, H.dtype, "W", dev), T, d, V, dt,
                                  float(temperature), int(seed) & 0xFFFFFFFFFFFFFFFF, tokens.data_ptr(),
                                  scores.data_ptr() if want_scores else None, ws.data_ptr(), ws.numel(), _stream(dev))
    if rc != 0:
        raise OaplError(rc, "oapl_sample_tokens")
    return (tokens, scores, ws) if want_scores else (tokens, ws)


class LossResult(NamedTuple):
    loss: torch.Tensor            # [1] float32
    logprob: torch.Tensor         # [T] float32
    seq_logratio: torch.Tensor    # [N] float32
    vstar: torch.Tensor           # [P] float32
    dH: Optional[torch.Tensor]    # [T, d] in H's dtype
    dW: Optional[torch.Tensor]    # [V, d] float32
    workspace: torch.Tensor


def loss_fwd_bwd(H, W, tokens, logq, seq_offsets, rewards, group_ids, n_groups: int, beta: float, *,
                 beta_value: Optional[float] = None, loss_scale: float = 1.0, backward: bool = True,
                 two_pass: bool = False, max_panel_rows: Optional[int] = None,
                 max_rollout_len: Optional[int] = None, workspace: Optional[torch.Tensor] = None,
                 dH: Optional[torch.Tensor] = None, dW: Optional[torch.Tensor] = None) -> LossResult:
    """oapl_loss_fwd_bwd (or the two-beta entry point when beta_value or two_pass is given).

    max_panel_rows / max_rollout_len only size the workspace this wrapper allocates when none is
    passed; the library derives its plan from the bytes it is handed.
    """
    L = lib()
    _check_device(H)
    dt = _dtype_code(H)
    T, d = H.shape
    V = W.shape[0]
    n_seq = rewards.shape[0]
    if W.shape[1] != d or tokens.shape != (T,) or logq.shape != (T,) or seq_offsets.shape != (n_seq + 1,) \
            or group_ids.shape != (n_seq,):
        raise ValueError("shape mismatch between the inputs")
    dev = H.device
    nbytes = workspace_bytes(T, d, V, n_seq, n_groups, dt, backward, _panel_rows(H, W, max_panel_rows), max_rollout_len)
    if nbytes == 0:
        raise OaplError(2, "oapl_workspace_bytes")
    ws = _workspace(nbytes, dev, workspace)
    loss = torch.empty(1, dtype=torch.float32, device=dev)
    logprob = torch.empty(T, dtype=torch.float32, device=dev)
    seq_lr = torch.empty(n_seq, dtype=torch.float32, device=dev)
    vstar = torch.empty(n_groups, dtype=torch.float32, device=dev)
    if backward:
        dH = torch.empty_like(H) if dH is None else dH
        dW = torch.empty((V, d), dtype=torch.float32, device=dev) if dW is None else dW
        if dH.shape != H.shape or dW.shape != (V, d):
            raise ValueError("dH / dW have the wrong shape")
    else:
        dH = dW = None
    head = [_dev(H, H.dtype, "H", dev), _dev(W, H.dtype, "W", dev), _dev(tokens, torch.int32, "tokens", dev),
            _dev(logq, torch.float32, "logq", dev), _dev(seq_offsets, torch.int64, "seq_offsets", dev),
            _dev(rewards, torch.float32, "rewards", dev), _dev(group_ids, torch.int32, "group_ids", dev),
            T, d, V, n_seq, n_groups, dt]
    tail = [loss.data_ptr(), logprob.data_ptr(), seq_lr.data_ptr(), vstar.data_ptr(),
            _dev(dH, H.dtype, "dH", dev), _dev(dW, torch.float32, "dW", dev), ws.data_ptr(), ws.numel(),
            _stream(dev)]
    if beta_value is None and not two_pass:
        rc = L.oapl_loss_fwd_bwd(*head, float(beta), float(loss_scale), *tail)
        where = "oapl_loss_fwd_bwd"
    else:
        rc = L.oapl_loss_fwd_bwd_two_beta(*head, float(beta if beta_value is None else beta_value), float(beta),
                                          float(loss_scale), OAPL_FLAG_TWO_PASS if two_pass else 0, *tail)
        where = "oapl_loss_fwd_bwd_two_beta"
    if rc != 0:
        raise OaplError(rc, where)
    return LossResult(loss, logprob, seq_lr, vstar, dH, dW, ws)


def loss_fwd_bwd_noalloc(H, W, tokens, logq, seq_offsets, rewards, group_ids, n_groups: int, beta: float,
                         loss: torch.Tensor, logprob: torch.Tensor, seq_logratio: torch.Tensor, vstar: torch.Tensor,
                         dH: Optional[torch.Tensor], dW: Optional[torch.Tensor], *, loss_scale: float = 1.0) -> None:
    """oapl_loss_fwd_bwd_noalloc: every output is passed in; neither this wrapper nor the library allocates."""
    _check_device(H)
    dt = _dtype_code(H)
    T, d = H.shape
    V = W.shape[0]
    n_seq = rewards.shape[0]
    if W.shape[1] != d or tokens.shape != (T,) or logq.shape != (T,) or seq_offsets.shape != (n_seq + 1,) \
            or group_ids.shape != (n_seq,) or loss.shape != (1,) or logprob.shape != (T,) \
            or seq_logratio.shape != (n_seq,) or vstar.shape != (n_groups,):
        raise ValueError("shape mismatch between the arguments")
    if (dH is None) != (dW is None) or (dH is not None and (dH.shape != H.shape or dW.shape != (V, d))):
        raise ValueError("dH / dW must come as a pair of the right shapes")
    dev = H.device
    rc = lib().oapl_loss_fwd_bwd_noalloc(
        _dev(H, H.dtype, "H", dev), _dev(W, H.dtype, "W", dev), _dev(tokens, torch.int32, "tokens", dev),
        _dev(logq, torch.float32, "logq", dev), _dev(seq_offsets, torch.int64, "seq_offsets", dev),
        _dev(rewards, torch.float32, "rewards", dev), _dev(group_ids, torch.int32, "group_ids", dev),
        T, d, V, n_seq, n_groups, dt, float(beta), float(loss_scale),
        _dev(loss, torch.float32, "loss", dev), _dev(logprob, torch.float32, "logprob", dev),
        _dev(seq_logratio, torch.float32, "seq_logratio", dev), _dev(vstar, torch.float32, "vstar", dev),
        _dev(dH, H.dtype, "dH", dev), _dev(dW, torch.float32, "dW", dev), _stream(dev))
    if rc != 0:
        raise OaplError(rc, "oapl_loss_fwd_bwd_noalloc")


class GrpoResult(NamedTuple):
    loss: torch.Tensor            # [1] float32
    logprob: torch.Tensor         # [T] float32
    advantages: torch.Tensor      # [N] float32
    dH: Optional[torch.Tensor]
    dW: Optional[torch.Tensor]
    workspace: torch.Tensor


def grpo_loss_fwd_bwd(H, W, tokens, logq, logp_old, seq_offsets, rewards, group_ids, n_groups: int, *,
                      clip_eps: float = 0.2, adv_eps: float = 1e-6, loss_scale: float = 1.0, backward: bool = True,
                      two_pass: bool = False, max_panel_rows: Optional[int] = None,
                      max_rollout_len: Optional[int] = None, workspace: Optional[torch.Tensor] = None,
                      dH: Optional[torch.Tensor] = None, dW: Optional[torch.Tensor] = None) -> GrpoResult:
    """oapl_grpo_loss_fwd_bwd: the paper's GRPO + token-level importance sampling baseline."""
    _check_device(H)
    dt = _dtype_code(H)
    T, d = H.shape
    V = W.shape[0]
    n_seq = rewards.shape[0]
    if W.shape[1] != d or tokens.shape != (T,) or logq.shape != (T,) or logp_old.shape != (T,) \
            or seq_offsets.shape != (n_seq + 1,) or group_ids.shape != (n_seq,):
        raise ValueError("shape mismatch between the inputs")
    dev = H.device
    nbytes = workspace_bytes(T, d, V, n_seq, n_groups, dt, backward, _panel_rows(H, W, max_panel_rows), max_rollout_len)
    if nbytes == 0:
        raise OaplError(2, "oapl_workspace_bytes")
    ws = _workspace(nbytes, dev, workspace)
    loss = torch.empty(1, dtype=torch.float32, device=dev)
    logprob = torch.empty(T, dtype=torch.float32, device=dev)
    adv = torch.empty(n_seq, dtype=torch.float32, device=dev)
    if backward:
        dH = torch.empty_like(H) if dH is None else dH
        dW = torch.empty((V, d), dtype=torch.float32, device=dev) if dW is None else dW
        if dH.shape != H.shape or dW.shape != (V, d):
            raise ValueError("dH / dW have the wrong shape")
    else:
        dH = dW = None
    rc = lib().oapl_grpo_loss_fwd_bwd(
        _dev(H, H.dtype, "H", dev), _dev(W, H.dtype, "W", dev), _dev(tokens, torch.int32, "tokens", dev),
        _dev(logq, torch.float32, "logq", dev), _dev(logp_old, torch.float32, "logp_old", dev),
        _dev(seq_offsets, torch.int64, "seq_offsets", dev), _dev(rewards, torch.float32, "rewards", dev),
        _dev(group_ids, torch.int32, "group_ids", dev), T, d, V, n_seq, n_groups, dt, float(clip_eps), float(adv_eps),
        float(loss_scale), OAPL_FLAG_TWO_PASS if two_pass else 0, loss.data_ptr(), logprob.data_ptr(), adv.data_ptr(),
        _dev(dH, H.dtype, "dH", dev),
        _dev(dW, torch.float32, "dW", dev), ws.data_ptr(), ws.numel(), _stream(dev))
    if rc != 0:
        raise OaplError(rc, "oapl_grpo_loss_fwd_bwd")
    return GrpoResult(loss, logprob, adv, dH, dW, ws)


def _heads(t: torch.Tensor, name: str, shape, dtype: torch.dtype, index: int) -> Heads:
    """The oapl_heads of a tensor [tokens, heads, channels] on GPU `index` whose channels lie side by side."""
    if t.get_device() != index:
        raise ValueError(f"{name} must live on cuda:{index}")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have the shape {tuple(shape)}, got {tuple(t.shape)}")
    token, head, channel = t.stride()
    if channel != 1 and t.numel() > 0:
        raise ValueError(f"the channels of {name} must lie side by side")
    return Heads(t.data_ptr(), token, head)


def _flat(t: Optional[torch.Tensor], dtype: torch.dtype, name: str, index: int) -> Optional[int]:
    """As _dev, for calls where its microseconds count."""
    if t is None:
        return None
    if t.get_device() != index:
        raise ValueError(f"{name} must live on cuda:{index}")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _scratch(nbytes: int, like: torch.Tensor, workspace: Optional[torch.Tensor], where: str) -> torch.Tensor:
    if nbytes == 0:
        raise OaplError(2, where)
    if workspace is None:
        return like.new_empty(nbytes, dtype=torch.uint8)
    return _workspace(nbytes, like.device, workspace)


def _qk_setup(q: torch.Tensor, k: torch.Tensor):
    """(tokens, heads, channels of q, heads of k, dtype code, GPU)."""
    index = q.get_device()
    if index < 0 or index != _current_gpu():
        _check_device(q)
    dt = _dtype_code(q)
    if q.dim() != 3 or k.dim() != 3 or q.shape[2] != k.shape[2]:
        raise ValueError("q and k must be [tokens, heads, channels] with the same channels")
    T, hq, D = q.shape
    return T, hq, D, k.shape[1], dt, index


def _check_rope(T, D, positions, cos_sin, q_gain, k_gain):
    if positions.shape != (T,) or cos_sin.dim() != 2:
        raise ValueError("shape mismatch between q, positions and cos_sin")
    if (q_gain is None) != (k_gain is None) or (q_gain is not None and (q_gain.shape != (D,) or k_gain.shape != (D,))):
        raise ValueError("q_gain and k_gain come as a pair, one value a channel")


class NormRopeResult(NamedTuple):
    q: torch.Tensor               # [T, n_q_heads, D]
    k: torch.Tensor               # [T, n_k_heads, D], or the cache it was written to
    v: Optional[torch.Tensor]     # the value cache


def qk_norm_rope_fwd(q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor, cos_sin: torch.Tensor,
                     q_gain: Optional[torch.Tensor] = None, k_gain: Optional[torch.Tensor] = None, *, eps: float = 1e-6,
                     v: Optional[torch.Tensor] = None, rows: Optional[torch.Tensor] = None,
                     q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None,
                     v_out: Optional[torch.Tensor] = None) -> NormRopeResult:
    """oapl_qk_norm_rope_fwd: norm of every query and key head and the position rotation, in one pass.

    q, k (and v) may be views into one projection's output.  With `rows`, keys (and values) go to those rows of the caches
    k_out (and v_out); without, k_out defaults to a new tensor.
    """
    T, hq, D, hk, dt, gpu = _qk_setup(q, k)
    _check_rope(T, D, positions, cos_sin, q_gain, k_gain)
    if rows is not None and rows.shape != (T,):
        raise ValueError("rows must have one entry a token")
    if (v is None) != (v_out is None) or (rows is not None and k_out is None):
        raise ValueError("rows need a cache k_out, values a cache v_out")
    kind, q_shape, k_shape = q.dtype, q.shape, (T, hk, D)
    q_out = q.new_empty(q_shape) if q_out is None else q_out
    k_out = q.new_empty(k_shape) if k_out is None else k_out
    n_rows = T if rows is None else k_out.shape[0]
    out_shape = (n_rows, hk, D)
    rc = lib().oapl_qk_norm_rope_fwd(
        _heads(q, "q", q_shape, kind, gpu), _heads(k, "k", k_shape, kind, gpu),
        None if v is None else _heads(v, "v", k_shape, kind, gpu), _flat(positions, torch.int32, "positions", gpu),
        _flat(cos_sin, torch.float32, "cos_sin", gpu), _flat(q_gain, kind, "q_gain", gpu), _flat(k_gain, kind, "k_gain", gpu),
        _flat(rows, torch.int64, "rows", gpu), T, hq, hk, D, cos_sin.shape[1], cos_sin.shape[0], n_rows, dt, eps,
        _heads(q_out, "q_out", q_shape, kind, gpu), _heads(k_out, "k_out", out_shape, kind, gpu),
        None if v is None else _heads(v_out, "v_out", out_shape, kind, gpu), _raw_stream(gpu))
    if rc != 0:
        raise OaplError(rc, "oapl_qk_norm_rope_fwd")
    return NormRopeResult(q_out, k_out, v_out)


class NormRopeGrads(NamedTuple):
    dq: torch.Tensor
    dk: torch.Tensor
    dq_gain: Optional[torch.Tensor]   # [D] float32
    dk_gain: Optional[torch.Tensor]
    workspace: Optional[torch.Tensor]


def qk_norm_rope_bwd(q: torch.Tensor, k: torch.Tensor, dq_out: torch.Tensor, dk_out: torch.Tensor, positions: torch.Tensor,
                     cos_sin: torch.Tensor, q_gain: Optional[torch.Tensor] = None, k_gain: Optional[torch.Tensor] = None, *,
                     eps: float = 1e-6, dq: Optional[torch.Tensor] = None, dk: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None) -> NormRopeGrads:
    """oapl_qk_norm_rope_bwd: gradients of the inputs (q, k) and of the gains, from those of the outputs."""
    T, hq, D, hk, dt, gpu = _qk_setup(q, k)
    _check_rope(T, D, positions, cos_sin, q_gain, k_gain)
    kind, q_shape, k_shape = q.dtype, q.shape, (T, hk, D)
    dq = q.new_empty(q_shape) if dq is None else dq
    dk = q.new_empty(k_shape) if dk is None else dk
    gains, ws, at = (None, None), None, 0
    if q_gain is not None:
        ws = _scratch(lib().oapl_qk_norm_rope_workspace_bytes(T, hq, hk, D), q, workspace, "oapl_qk_norm_rope_workspace_bytes")
        both = q.new_empty((2, D), dtype=torch.float32)
        gains, at = both.unbind(), both.data_ptr()
    rc = lib().oapl_qk_norm_rope_bwd(
        _heads(q, "q", q_shape, kind, gpu), _heads(k, "k", k_shape, kind, gpu), _heads(dq_out, "dq_out", q_shape, kind, gpu),
        _heads(dk_out, "dk_out", k_shape, kind, gpu), _flat(positions, torch.int32, "positions", gpu),
        _flat(cos_sin, torch.float32, "cos_sin", gpu), _flat(q_gain, kind, "q_gain", gpu), _flat(k_gain, kind, "k_gain", gpu),
        T, hq, hk, D, cos_sin.shape[1], cos_sin.shape[0], dt, eps, _heads(dq, "dq", q_shape, kind, gpu),
        _heads(dk, "dk", k_shape, kind, gpu), at or None, at + 4 * D if at else None, None if ws is None else ws.data_ptr(),
        0 if ws is None else ws.numel(), _raw_stream(gpu))
    if rc != 0:
        raise OaplError(rc, "oapl_qk_norm_rope_bwd")
    return NormRopeGrads(dq, dk, gains[0], gains[1], ws)


def attention_workspace_bytes(Tq: int, Tk: int, n_seq: int, n_q_heads: int, n_k_heads: int, head_dim: int, dtype: int,
                              with_backward: bool) -> int:
    """oapl_attention_workspace_bytes."""
    return int(lib().oapl_attention_workspace_bytes(Tq, Tk, n_seq, n_q_heads, n_k_heads, head_dim, dtype,
                                                    1 if with_backward else 0))


def _attention_setup(q, k, v, q_offsets, k_offsets, scale, with_backward, workspace):
    """What both attention calls check and pass on: heads, offsets, sizes, the scale, the workspace, the GPU."""
    Tq, hq, D, hk, dt, gpu = _qk_setup(q, k)
    k_offsets = q_offsets if k_offsets is None else k_offsets
    if q_offsets.dim() != 1 or q_offsets.shape[0] < 1 or k_offsets.shape != q_offsets.shape:
        raise ValueError("q_offsets and k_offsets must have one entry more than there are sequences")
    sizes = (Tq, k.shape[0], q_offsets.shape[0] - 1, hq, hk, D, dt)
    ws = _scratch(lib().oapl_attention_workspace_bytes(*sizes, with_backward), q, workspace, "oapl_attention_workspace_bytes")
    heads = (_heads(q, "q", q.shape, q.dtype, gpu), _heads(k, "k", k.shape, q.dtype, gpu), _heads(v, "v", k.shape, q.dtype, gpu))
    offsets = (_flat(q_offsets, torch.int64, "q_offsets", gpu), _flat(k_offsets, torch.int64, "k_offsets", gpu))
    return heads, offsets, sizes, D ** -0.5 if scale is None else scale, ws, gpu


class AttentionResult(NamedTuple):
    out: torch.Tensor             # [Tq, n_q_heads, D]
    lse: Optional[torch.Tensor]   # [Tq, n_q_heads] float32
    workspace: torch.Tensor


def attention_fwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_offsets: torch.Tensor,
                  k_offsets: Optional[torch.Tensor] = None, *, causal: bool = True, scale: Optional[float] = None,
                  k_used: Optional[torch.Tensor] = None, want_lse: bool = True, out: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None) -> AttentionResult:
    """oapl_attention_fwd: soft-max attention of packed sequences, or of a few new tokens over a cache (k_used).

    k_offsets defaults to q_offsets, scale to 1 / sqrt(D).
    """
    heads, offsets, sizes, scale, ws, gpu = _attention_setup(q, k, v, q_offsets, k_offsets, scale, 0, workspace)
    if k_used is not None and k_used.shape != (sizes[2],):
        raise ValueError("k_used must have one entry a sequence")
    out = q.new_empty(q.shape) if out is None else out
    lse = q.new_empty(q.shape[:2], dtype=torch.float32) if want_lse else None
    rc = lib().oapl_attention_fwd(*heads, *offsets, _flat(k_used, torch.int64, "k_used", gpu), *sizes, 1 if causal else 0, scale,
                                  _heads(out, "out", q.shape, q.dtype, gpu), None if lse is None else lse.data_ptr(),
                                  ws.data_ptr(), ws.numel(), _raw_stream(gpu))
    if rc != 0:
        raise OaplError(rc, "oapl_attention_fwd")
    return AttentionResult(out, lse, ws)


class AttentionGrads(NamedTuple):
    dq: torch.Tensor
    dk: torch.Tensor
    dv: torch.Tensor
    workspace: torch.Tensor


def attention_bwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, lse: torch.Tensor, dout: torch.Tensor,
                  q_offsets: torch.Tensor, k_offsets: Optional[torch.Tensor] = None, *, causal: bool = True,
                  scale: Optional[float] = None, dq: Optional[torch.Tensor] = None, dk: Optional[torch.Tensor] = None,
                  dv: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> AttentionGrads:
    """oapl_attention_bwd: gradients of q, k and v from attention_fwd's output and log-sum-exp and the output's gradient."""
    heads, offsets, sizes, scale, ws, gpu = _attention_setup(q, k, v, q_offsets, k_offsets, scale, 1, workspace)
    kind, q_shape, k_shape = q.dtype, q.shape, k.shape
    dq = q.new_empty(q_shape) if dq is None else dq
    dk = q.new_empty(k_shape) if dk is None else dk
    dv = q.new_empty(k_shape) if dv is None else dv
    if lse.shape != q_shape[:2]:
        raise ValueError("lse must be [tokens, heads] of q")
    rc = lib().oapl_attention_bwd(*heads, _heads(out, "out", q_shape, kind, gpu), _flat(lse, torch.float32, "lse", gpu),
                                  _heads(dout, "dout", q_shape, kind, gpu), *offsets, *sizes, 1 if causal else 0, scale,
                                  _heads(dq, "dq", q_shape, kind, gpu), _heads(dk, "dk", k_shape, kind, gpu),
                                  _heads(dv, "dv", k_shape, kind, gpu), ws.data_ptr(), ws.numel(), _raw_stream(gpu))
    if rc != 0:
        raise OaplError(rc, "oapl_attention_bwd")
    return AttentionGrads(dq, dk, dv, ws)


def _rows(t: torch.Tensor, name: str, shape, dtype: torch.dtype, index: int) -> Rows:
    """The oapl_rows of a tensor [rows, channels] on GPU `index` whose channels lie side by side."""
    if t.dtype is dtype and t.shape == shape and t.get_device() == index:
        row, channel = t.stride()
        if channel == 1 or shape[1] <= 1 or shape[0] == 0:
            return Rows(t.data_ptr(), row)
        raise ValueError(f"the channels of {name} must lie side by side")
    if t.get_device() != index:
        raise ValueError(f"{name} must live on cuda:{index}")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    raise ValueError(f"{name} must have the shape {tuple(shape)}, got {tuple(t.shape)}")


def _result(t: Optional[torch.Tensor], name: str, like: torch.Tensor, shape, dtype: torch.dtype, index: int):
    """The tensor that a result goes to, t or a new one beside `like`, and its oapl_rows."""
    if t is not None:
        return t, _rows(t, name, shape, dtype, index)
    t = like.new_empty(shape, dtype=dtype)
    return t, Rows(t.data_ptr(), shape[1])


def _gpu_of(t: torch.Tensor) -> int:
    """The index of the current GPU, on which t has to live."""
    index = t.get_device()
    if index < 0 or index != _current_gpu():
        _check_device(t)
    return index


def embed_fwd(E: torch.Tensor, tokens: torch.Tensor, *, scale: float = 1.0, out_dtype: Optional[torch.dtype] = None,
              out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """oapl_embed_fwd: [T, d], the rows of the embedding E [V, d] at `tokens`, scaled; in E's type or out_dtype (or out's)."""
    gpu = _gpu_of(E)
    if E.dim() != 2 or tokens.dim() != 1:
        raise ValueError("E must be [V, d] and tokens [T]")
    (V, d), T = E.shape, tokens.shape[0]
    if out is None:
        out = E.new_empty((T, d), dtype=out_dtype)
        rows = Rows(out.data_ptr(), d)
    elif out_dtype is not None and out.dtype is not out_dtype:
        raise TypeError(f"out must be {out_dtype}, got {out.dtype}")
    else:
        rows = _rows(out, "out", (T, d), out.dtype, gpu)
    rc = lib().oapl_embed_fwd(_flat(E, E.dtype, "E", gpu), _flat(tokens, torch.int32, "tokens", gpu), T, d, V, _dtype_code(E),
                              _dtype_code(out), scale, rows, _raw_stream(gpu))
    if rc != 0:
        raise OaplError(rc, "oapl_embed_fwd")
    return out


def embed_workspace_bytes(T: int, d: int, V: int) -> int:
    """oapl_embed_workspace_bytes."""
    return int(lib().oapl_embed_workspace_bytes(T, d, V))


class EmbedGrads(NamedTuple):
    dE: torch.Tensor              # [V, d] float32
    workspace: torch.Tensor


def embed_bwd(dout: torch.Tensor, tokens: torch.Tensor, V: Optional[int] = None, *, scale: float = 1.0,
              dE: Optional[torch.Tensor] = None, accumulate: bool = False, workspace: Optional[torch.Tensor] = None) -> EmbedGrads:
    """oapl_embed_bwd: the embedding's gradient from that of embed_fwd's output.

    A new tensor of V rows, or into dE: overwritten, or added to it (`accumulate`; the head's dW where the weights are shared).
    """
    gpu = _gpu_of(dout)
    if dout.dim() != 2 or tokens.shape != dout.shape[:1]:
        raise ValueError("dout must be [T, d] and tokens [T]")
    T, d = dout.shape
    if dE is None:
        if V is None or accumulate:
            raise ValueError("without dE there is nothing to add to, and V has to be given")
        dE = dout.new_empty((V, d), dtype=torch.float32)
    elif dE.dim() != 2 or dE.shape[1] != d or (V is not None and dE.shape[0] != V):
        raise ValueError("dE must be [V, d]")
    V = dE.shape[0]
    ws = _scratch(lib().oapl_embed_workspace_bytes(T, d, V), dout, workspace, "oapl_embed_workspace_bytes")
    rc = lib().oapl_embed_bwd(_rows(dout, "dout", dout.shape, dout.dtype, gpu), _flat(tokens, torch.int32, "tokens", gpu), T, d, V,
                              _dtype_code(dout), scale, 1 if accumulate else 0, _flat(dE, torch.float32, "dE", gpu), ws.data_ptr(),
                              ws.numel(), _raw_stream(gpu))
    if rc != 0:
        raise OaplError(rc, "oapl_embed_bwd")
    return EmbedGrads(dE, ws)


def residual_norm_workspace_bytes(T: int, d: int) -> int:
    """oapl_residual_norm_workspace_bytes."""
    return int(lib().oapl_residual_norm_workspace_bytes(T, d))


def _residual_norm_setup(x, y, gain, y_gain, gate):
    """(shape, the block's type, whether the gate is one a token, its oapl_rows, GPU)."""
    gpu = _gpu_of(x)
    if x.dim() != 2:
        raise ValueError("x must be [tokens, channels]")
    if y is None and gain is None:
        raise ValueError("there is neither a block's output to add nor a norm to take")
    if y is None and (y_gain is not None or gate is not None):
        raise ValueError("a gate and y_gain go with a block's output y")
    kind = (gain if y is None else y).dtype
    d = x.shape[1]
    if (gain is not None and gain.shape != (d,)) or (y_gain is not None and y_gain.shape != (d,)):
        raise ValueError("gains must have one value a channel")
    if gate is None:
        return x.shape, kind, 0, None, gpu
    if gate.dim() == 1:
        if gate.shape != (d,):
            raise ValueError("a gate that all tokens share must have one value a channel")
        return x.shape, kind, 0, Rows(_flat(gate, kind, "gate", gpu), 0), gpu
    return x.shape, kind, 1, _rows(gate, "gate", x.shape, kind, gpu), gpu


class ResidualNormResult(NamedTuple):
    x: torch.Tensor               # [T, d], the stream behind the block (x itself without one)
    out: Optional[torch.Tensor]   # [T, d], its norm


def residual_norm_fwd(x: torch.Tensor, y: Optional[torch.Tensor] = None, gain: Optional[torch.Tensor] = None, *,
                      y_gain: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None, scale: float = 1.0, eps: float = 1e-6,
                      x_out: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> ResidualNormResult:
    """oapl_residual_norm_fwd: a block's output y, normed (y_gain), gated and scaled, added to the residual stream x, and the norm
    (gain) of the sum.

    x may be float32 where y is bfloat16.  gate: [d], or [T, d] for one a token.  x_out may be x.
    """
    shape, kind, per_token, gates, gpu = _residual_norm_setup(x, y, gain, y_gain, gate)
    T, d = shape
    if (y is None and x_out is not None) or (gain is None and out is not None):
        raise ValueError("x_out goes with y, out with gain")
    y_rows = x_out_rows = out_rows = None
    if y is not None:
        y_rows = _rows(y, "y", shape, kind, gpu)
        x_out, x_out_rows = _result(x_out, "x_out", x, shape, x.dtype, gpu)
    if gain is not None:
        out, out_rows = _result(out, "out", x, shape, kind, gpu)
    rc = lib().oapl_residual_norm_fwd(
        _rows(x, "x", shape, x.dtype, gpu), y_rows, _flat(y_gain, kind, "y_gain", gpu), gates, per_token, _flat(gain, kind, "gain", gpu),
        T, d, _dtype_code(x), _dtype_code(gain if y is None else y), scale, eps, x_out_rows, out_rows, _raw_stream(gpu))
    if rc != 0:
        raise OaplError(rc, "oapl_residual_norm_fwd")
    return ResidualNormResult(x if y is None else x_out, out)


class ResidualNormGrads(NamedTuple):
    dx: torch.Tensor
    dy: Optional[torch.Tensor]
    dgain: Optional[torch.Tensor]     # [d] float32
    dy_gain: Optional[torch.Tensor]   # [d] float32
    dgate: Optional[torch.Tensor]     # [d] float32, or [T, d] in the gate's type
    workspace: Optional[torch.Tensor]


def residual_norm_bwd(x: torch.Tensor, y: Optional[torch.Tensor], dx_out: Optional[torch.Tensor], dout: Optional[torch.Tensor],
                      gain: Optional[torch.Tensor] = None, *, y_gain: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                      scale: float = 1.0, eps: float = 1e-6, dx: Optional[torch.Tensor] = None, dy: Optional[torch.Tensor] = None,
                      workspace: Optional[torch.Tensor] = None) -> ResidualNormGrads:
    """oapl_residual_norm_bwd: gradients of the stream in front of the block, of the block's output, the gains and the gate.

    x is the stream behind the block, residual_norm_fwd's result; dx_out and dout are the gradients of its two results (dx_out may
    be None, dout goes with gain).
    """
    shape, kind, per_token, gates, gpu = _residual_norm_setup(x, y, gain, y_gain, gate)
    T, d = shape
    if (gain is None) != (dout is None) or (y is None and dy is not None):
        raise ValueError("dout goes with gain, dy with y")
    y_rows = dy_rows = dout_rows = dgate_rows = dgate = None
    dx, dx_rows = _result(dx, "dx", x, shape, x.dtype, gpu)
    if y is not None:
        y_rows = _rows(y, "y", shape, kind, gpu)
        dy, dy_rows = _result(dy, "dy", x, shape, kind, gpu)
    if dout is not None:
        dout_rows = _rows(dout, "dout", shape, kind, gpu)
    if per_token:
        dgate, dgate_rows = _result(None, "dgate", x, shape, kind, gpu)
    dgain = None if gain is None else x.new_empty(d, dtype=torch.float32)
    dy_gain = None if y_gain is None else x.new_empty(d, dtype=torch.float32)
    shared = None if gate is None or per_token else x.new_empty(d, dtype=torch.float32)
    ws, ws_at, ws_bytes = None, None, 0
    if dgain is not None or dy_gain is not None or shared is not None:
        ws = _scratch(lib().oapl_residual_norm_workspace_bytes(T, d), x, workspace, "oapl_residual_norm_workspace_bytes")
        ws_at, ws_bytes = ws.data_ptr(), ws.numel()
    rc = lib().oapl_residual_norm_bwd(
        _rows(x, "x", shape, x.dtype, gpu), y_rows, _flat(y_gain, kind, "y_gain", gpu), gates, per_token, _flat(gain, kind, "gain", gpu),
        None if dx_out is None else _rows(dx_out, "dx_out", shape, x.dtype, gpu), dout_rows, T, d, _dtype_code(x),
        _dtype_code(gain if y is None else y), scale, eps, dx_rows, dy_rows, None if dgain is None else dgain.data_ptr(),
        None if dy_gain is None else dy_gain.data_ptr(), dgate_rows, None if shared is None else shared.data_ptr(), ws_at, ws_bytes,
        _raw_stream(gpu))
    if rc != 0:
        raise OaplError(rc, "oapl_residual_norm_bwd")
    return ResidualNormGrads(dx, dy, dgain, dy_gain, shared if dgate is None else dgate, ws)


def clip_workspace_bytes(n_tensors: int) -> int:
    """oapl_clip_workspace_bytes."""
    return int(lib().oapl_clip_workspace_bytes(n_tensors))


def _tensors(grads, out):
    """The oapl_tensor list of dense tensors on the current GPU, their number, and that GPU."""
    if len(grads) == 0:
        raise ValueError("there are no gradients")
    gpu = _gpu_of(grads[0])
    if out is not None and len(out) != len(grads):
        raise ValueError("out must have one tensor a gradient")
    # four words a tensor: its address, the result's, how many elements, the type (whose other half is padding)
    words = []
    for g, o in zip(grads, grads if out is None else out):
        kind, code = g.dtype, _CODES.get(g.dtype)
        if code is None or not (g.is_contiguous() and g.get_device() == gpu):
            _flat(g, kind, "a gradient", gpu)
            _dtype_code(g)
        at = to = g.data_ptr()
        if o is not g:
            if o.shape != g.shape:
                raise ValueError("out must have the gradients' shapes")
            to = _flat(o, kind, "out", gpu)
        words += (at, to, g.numel(), code)
    words = array.array("q", words)
    return words, len(grads), gpu


class GradNorm(NamedTuple):
    norm: torch.Tensor            # [1] float32
    workspace: Optional[torch.Tensor]


def grad_norm(grads, *, workspace: Optional[torch.Tensor] = None) -> GradNorm:
    """oapl_grad_norm: the norm of all gradients together (a list of contiguous tensors, float32 and bfloat16 mixed as they come)."""
    words, n, gpu = _tensors(grads, None)
    ws = _scratch(lib().oapl_clip_workspace_bytes(n), grads[0], workspace, "oapl_clip_workspace_bytes")
    norm = grads[0].new_empty(1, dtype=torch.float32)
    rc = lib().oapl_grad_norm(words.buffer_info()[0], n, norm.data_ptr(), ws.data_ptr(), ws.numel(), _raw_stream(gpu))
    if rc != 0:
        raise OaplError(rc, "oapl_grad_norm")
    return GradNorm(norm, ws)


def clip_grads(grads, max_norm: float, *, norm: Optional[torch.Tensor] = None, out=None,
               workspace: Optional[torch.Tensor] = None) -> GradNorm:
    """oapl_clip_grads: gradients scaled to max_norm where their common norm is larger (and finite), in place or into `out`.

    Returns their norm before that.  `norm`: a norm to go by instead, [1] float32 (of gradients that are spread over GPUs, say).
    """
    words, n, gpu = _tensors(grads, out)
    ws, given, made = None, None, None
    if norm is None:
        ws = _scratch(lib().oapl_clip_workspace_bytes(n), grads[0], workspace, "oapl_clip_workspace_bytes")
        norm = grads[0].new_empty(1, dtype=torch.float32)
        made = norm.data_ptr()
    else:
        if norm.numel() != 1:
            raise ValueError("norm must be one number")
        given = _flat(norm, torch.float32, "norm", gpu)
    rc = lib().oapl_clip_grads(words.buffer_info()[0], n, max_norm, given, made, None if ws is None else ws.data_ptr(),
                               0 if ws is None else ws.numel(), _raw_stream(gpu))
    if rc != 0:
        raise OaplError(rc, "oapl_clip_grads")
    return GradNorm(norm, ws)


def segmented_sum_f32(x: torch.Tensor, seq_offsets: torch.Tensor) -> torch.Tensor:
    """oapl_segmented_sum_f32: per-rollout sums in double."""
    dev = x.device
    n_seq = seq_offsets.shape[0] - 1
    out = torch.empty(n_seq, dtype=torch.float64, device=dev)
    rc = lib().oapl_segmented_sum_f32(_dev(x, torch.float32, "x", dev), _dev(seq_offsets, torch.int64, "seq_offsets", dev),
                                      n_seq, out.data_ptr(), _stream(dev))
    if rc != 0:
        raise OaplError(rc, "oapl_segmented_sum_f32")
    return out


def timing_enable(on: bool) -> None:
    rc = lib().oapl_timing_enable(1 if on else 0)
    if rc != 0:
        raise OaplError(rc, "oapl_timing_enable")


def timing_read():
    """{kernel name: (total milliseconds, launches)} since timing was enabled.  In small calls dH and dW are one launch, which
    counts as k_bwd_dw; k_bwd_dh then has none."""
    out = {}
    for i, name in enumerate(DENSE_KERNELS):
        ms = ctypes.c_double(0.0)
        n = ctypes.c_int64(0)
        rc = lib().oapl_timing_read(i, ctypes.byref(ms), ctypes.byref(n))
        if rc != 0:
            raise OaplError(rc, "oapl_timing_read")
        out[name] = (float(ms.value), int(n.value))
    return out
