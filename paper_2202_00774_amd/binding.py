"""ctypes binding of libsdgp.so: argument marshalling only.

Every function takes torch tensors that live on the GPU, hands their device
pointers and the current HIP stream to the C ABI, and raises ``SdgpError`` on a
non-zero status.  PyTorch is used for device memory and streams, nothing else.
"""
from __future__ import annotations

import ctypes
import functools
import os
import threading

import torch

F32, BF16 = 0, 1
RANDOM, GREEDY, GREEDY_ADJUSTED = 0, 1, 2

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "libsdgp.so")
_lock = threading.Lock()
_lib = None

EXPORTS = ("sdgp_prune", "sdgp_linear_bwd_data", "sdgp_conv_bwd_data", "sdgp_conv_bwd_data_workspace",
           "sdgp_conv_bwd_data_noalloc",
           "sdgp_channel_scales_workspace", "sdgp_channel_scales", "sdgp_prune_channel_rescaled", "sdgp_scale_filter",
           "sdgp_conv_bwd_data_channel_rescaled_workspace", "sdgp_conv_bwd_data_channel_rescaled",
           "sdgp_conv_bwd_data_compact_workspace", "sdgp_conv_bwd_data_compact",
           "sdgp_conv_bwd_data_grouped_workspace", "sdgp_conv_bwd_data_grouped",
           "sdgp_conv_fwd_workspace", "sdgp_conv_fwd", "sdgp_conv_bwd_weight_workspace", "sdgp_conv_bwd_weight",
           "sdgp_token_logprobs_workspace", "sdgp_token_logprobs", "sdgp_token_logprobs_bwd",
           "sdgp_block_norm", "sdgp_block_norm_bwd_workspace", "sdgp_block_norm_bwd", "sdgp_adamw_step",
           "sdgp_attention_workspace", "sdgp_attention", "sdgp_attention_bwd_workspace", "sdgp_attention_bwd",
           "sdgp_rotary", "sdgp_sequence_loss_workspace", "sdgp_policy_loss", "sdgp_policy_loss_bwd", "sdgp_preference_loss",
           "sdgp_preference_loss_bwd",
           "sdgp_peak_probe", "sdgp_status_string", "sdgp_version")


class SdgpError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where} failed with status {status}: {status_string(status)}")


def library_path() -> str:
    return _LIB_PATH


def load():
    """Loads libsdgp.so; raises if it has not been built (there is no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(_LIB_PATH):
                raise RuntimeError(f"{_LIB_PATH} is missing: build it with `python -m paper_2202_00774_amd.build`")
            lib = ctypes.CDLL(_LIB_PATH)
            i64, u64, i32, vp, sz = ctypes.c_int64, ctypes.c_uint64, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t
            lib.sdgp_prune.restype = i32
            lib.sdgp_prune.argtypes = [vp, i64, i64, i32, i32, i32, i32, u64, vp, vp, vp, vp]
            lib.sdgp_linear_bwd_data.restype = i32
            lib.sdgp_linear_bwd_data.argtypes = [vp, vp, vp, i64, i64, i64, i32, i32, i32, i32, u64, vp]
            lib.sdgp_conv_bwd_data.restype = i32
            lib.sdgp_conv_bwd_data.argtypes = [vp, vp, vp, i64, i64, i64, i64, i64, i32, i32, i32, i32, i32, i32, i32,
                                               i32, u64, vp, sz, vp]
            lib.sdgp_conv_bwd_data_noalloc.restype = i32
            lib.sdgp_conv_bwd_data_noalloc.argtypes = [vp, vp, vp, i64, i64, i64, i64, i64, i32, i32, i32, i32, i32, i32,
                                                       i32, i32, u64, vp]
            lib.sdgp_conv_bwd_data_workspace.restype = sz
            lib.sdgp_conv_bwd_data_workspace.argtypes = [i64, i64, i64, i64, i64, i32, i32, i32, i32, i32, i32, i32]
            lib.sdgp_channel_scales_workspace.restype = sz
            lib.sdgp_channel_scales_workspace.argtypes = [i64, i64, i32, i32, i32]
            lib.sdgp_channel_scales.restype = i32
            lib.sdgp_channel_scales.argtypes = [vp, i64, i64, i32, i32, i32, vp, vp, vp, sz, vp]
            lib.sdgp_prune_channel_rescaled.restype = i32
            lib.sdgp_prune_channel_rescaled.argtypes = [vp, i64, i64, i32, i32, i32, vp, vp, vp]
            lib.sdgp_scale_filter.restype = i32
            lib.sdgp_scale_filter.argtypes = [vp, vp, vp, i64, i64, i32, vp]
            lib.sdgp_conv_bwd_data_channel_rescaled_workspace.restype = sz
            lib.sdgp_conv_bwd_data_channel_rescaled_workspace.argtypes = [i64, i64, i64, i64, i64, i32, i32, i32, i32,
                                                                         i32, i32, i32]
            lib.sdgp_conv_bwd_data_channel_rescaled.restype = i32
            lib.sdgp_conv_bwd_data_channel_rescaled.argtypes = [vp, vp, vp, i64, i64, i64, i64, i64, i32, i32, i32, i32,
                                                               i32, i32, i32, vp, sz, vp]
            lib.sdgp_conv_bwd_data_compact_workspace.restype = sz
            lib.sdgp_conv_bwd_data_compact_workspace.argtypes = [i64, i64, i64, i64, i64, i32, i32, i32, i32, i32, i32, i32]
            lib.sdgp_conv_bwd_data_grouped_workspace.restype = sz
            lib.sdgp_conv_bwd_data_grouped_workspace.argtypes = [i64, i64, i64, i64, i64, i32, i32, i32, i32, i64, i32, i32, i32]
            lib.sdgp_conv_bwd_data_grouped.restype = i32
            lib.sdgp_conv_bwd_data_grouped.argtypes = [vp, vp, vp, i64, i64, i64, i64, i64, i32, i32, i32, i32, i64, i32, i32,
                                                       i32, i32, u64, vp, sz, vp]
            lib.sdgp_conv_bwd_data_compact.restype = i32
            lib.sdgp_conv_bwd_data_compact.argtypes = [vp, vp, vp, i64, i64, i64, i64, i64, i32, i32, i32, i32, i32, i32, i32,
                                                       i32, u64, vp, sz, vp]
            geom = [i64, i64, i64, i64, i64, i32, i32, i32, i32, i32]
            lib.sdgp_conv_fwd_workspace.restype = sz
            lib.sdgp_conv_fwd_workspace.argtypes = geom
            lib.sdgp_conv_fwd.restype = i32
            lib.sdgp_conv_fwd.argtypes = [vp, vp, vp] + geom + [vp, sz, vp]
            lib.sdgp_conv_bwd_weight_workspace.restype = sz
            lib.sdgp_conv_bwd_weight_workspace.argtypes = geom
            lib.sdgp_conv_bwd_weight.restype = i32
            lib.sdgp_conv_bwd_weight.argtypes = [vp, vp, vp] + geom + [vp, sz, vp]
            f32, f64 = ctypes.c_float, ctypes.c_double
            lib.sdgp_token_logprobs_workspace.restype = sz
            lib.sdgp_token_logprobs_workspace.argtypes = [i64, i64, i32, i32]
            lib.sdgp_token_logprobs.restype = i32
            lib.sdgp_token_logprobs.argtypes = [vp, i64, vp, i32, vp, vp, vp, vp, vp, i64, i64, i32, i32, f32, vp, sz, vp]
            lib.sdgp_token_logprobs_bwd.restype = i32
            lib.sdgp_token_logprobs_bwd.argtypes = [vp, i64, vp, i32, vp, vp, vp, vp, vp, i64, i64, i64, i32, f32, vp]
            lib.sdgp_block_norm.restype = i32
            lib.sdgp_block_norm.argtypes = [vp] * 8 + [i64, i64, i64, i32, i32, f32, f32, vp]
            lib.sdgp_block_norm_bwd_workspace.restype = sz
            lib.sdgp_block_norm_bwd_workspace.argtypes = [i64, i64, i64, i32]
            lib.sdgp_block_norm_bwd.restype = i32
            lib.sdgp_block_norm_bwd.argtypes = [vp] * 13 + [i64, i64, i64, i32, i32, f32, vp, sz, vp]
            lib.sdgp_adamw_step.restype = i32
            lib.sdgp_adamw_step.argtypes = [i32] + [vp] * 8 + [i32, i32, i32, f64, f64, f64, f64, f64, i64, vp, u64, vp]
            lib.sdgp_attention_workspace.restype = sz
            lib.sdgp_attention_workspace.argtypes = [i64, i64, i64, i64, i64, i32, i32]
            lib.sdgp_attention.restype = i32
            lib.sdgp_attention.argtypes = [vp] * 7 + [i64, vp, vp, i64, i64, i64, i64, i32, i32, i32, f32, vp, sz, vp]
            lib.sdgp_attention_bwd_workspace.restype = sz
            lib.sdgp_attention_bwd_workspace.argtypes = [i64, i64, i64, i64, i64, i32, i32]
            lib.sdgp_attention_bwd.restype = i32
            lib.sdgp_attention_bwd.argtypes = [vp] * 9 + [i64, vp, vp, vp, i64, i64, i64, i64, i32, i32, i32, f32, vp, sz, vp]
            lib.sdgp_rotary.restype = i32
            lib.sdgp_rotary.argtypes = [vp] * 6 + [i32, vp, vp, i32, i64, i64, i64, i64, i32, i32, i32, vp]
            lib.sdgp_sequence_loss_workspace.restype = sz
            lib.sdgp_sequence_loss_workspace.argtypes = [i64, i64]
            lib.sdgp_policy_loss.restype = i32
            lib.sdgp_policy_loss.argtypes = [vp] * 4 + [i32, vp, vp, i64, i64, f64, f64, f32, i32, vp, vp, vp, sz, vp]
            lib.sdgp_policy_loss_bwd.restype = i32
            lib.sdgp_policy_loss_bwd.argtypes = [vp] * 6 + [i32, vp, vp, i64, i64, f64, f64, f32, vp, vp]
            lib.sdgp_preference_loss.restype = i32
            lib.sdgp_preference_loss.argtypes = [vp] * 4 + [i64, i64, f64, f64, f64, i32, vp, vp, vp, vp, sz, vp]
            lib.sdgp_preference_loss_bwd.restype = i32
            lib.sdgp_preference_loss_bwd.argtypes = [vp] * 4 + [i64, i64, vp, vp]
            lib.sdgp_peak_probe.restype = i32
            lib.sdgp_peak_probe.argtypes = [i32, vp, vp, sz, i32, ctypes.POINTER(ctypes.c_double), vp]
            lib.sdgp_status_string.restype = ctypes.c_char_p
            lib.sdgp_status_string.argtypes = [i32]
            lib.sdgp_version.restype = i32
            lib.sdgp_version.argtypes = []
            _lib = lib
    return _lib


def status_string(status: int) -> str:
    return load().sdgp_status_string(int(status)).decode()


def version() -> int:
    return int(load().sdgp_version())


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported dtype {t.dtype}: float32 or bfloat16")


def _dev(t: torch.Tensor, name: str) -> torch.Tensor:
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


# The smallest calls are as long as their host side, so pointers and streams go to the library as plain integers
# (the argument types convert them) and the stream is asked for without building a Stream object around it.

def _ptr(t):
    return None if t is None else t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(t: torch.Tensor) -> int:
    if _raw_stream is not None:
        return _raw_stream(t.get_device())
    return torch.cuda.current_stream(t.device).cuda_stream


def sdgp_prune(dO: torch.Tensor, n: int, m: int, ranker: int, seed: int = 0, *, pruned: bool = True,
               compact: bool = False):
    """Alg. 1 on ``dO`` ([..., C], channels last).  Returns ``(pruned, vals, idx)``; entries not asked for are None."""
    _dev(dO, "dO")
    C = dO.shape[-1]
    rows = dO.numel() // C if C else 0
    out = torch.empty_like(dO) if pruned else None
    vals = idx = None
    if compact:
        if m < 1 or C % m:
            raise SdgpError(-3, "sdgp_prune")
        kshape = tuple(dO.shape[:-1]) + (C // m * n,)
        vals = torch.empty(kshape, dtype=dO.dtype, device=dO.device)
        idx = torch.empty(kshape, dtype=torch.uint8, device=dO.device)
    rc = load().sdgp_prune(_ptr(dO), rows, C, _dtype_code(dO), n, m, ranker, seed & (2**64 - 1), _ptr(out),
                           _ptr(vals), _ptr(idx), _stream(dO))
    if rc != 0:
        raise SdgpError(rc, "sdgp_prune")
    return out, vals, idx


def sdgp_linear_bwd_data(dO: torch.Tensor, W: torch.Tensor, n: int, m: int, ranker: int, seed: int = 0,
                         out: torch.Tensor | None = None) -> torch.Tensor:
    """dD = prune(dO) @ W for dO [rows, C_out], W [C_out, C_in]."""
    _dev(dO, "dO"), _dev(W, "W")
    if dO.dim() != 2 or W.dim() != 2 or W.shape[0] != dO.shape[1] or W.dtype != dO.dtype:
        raise ValueError("expected dO [rows, C_out] and W [C_out, C_in] of one dtype")
    rows, C_out = dO.shape
    C_in = W.shape[1]
    if out is None:
        out = dO.new_empty((rows, C_in))
    _dev(out, "out")
    rc = load().sdgp_linear_bwd_data(_ptr(dO), _ptr(W), _ptr(out), rows, C_out, C_in, _dtype_code(dO), n, m, ranker,
                                     seed & (2**64 - 1), _stream(dO))
    if rc != 0:
        raise SdgpError(rc, "sdgp_linear_bwd_data")
    return out


@functools.lru_cache(maxsize=1024)
def _need(query: str, *geometry) -> int:
    """Workspace bytes of a call: a pure function of its integers, asked of the library once for each layer."""
    return int(getattr(load(), query)(*geometry))


def conv_bwd_data_workspace(B, H, Wd, C_in, C_out, R, S, stride, pad, dtype_code, n, m) -> int:
    return int(load().sdgp_conv_bwd_data_workspace(B, H, Wd, C_in, C_out, R, S, stride, pad, dtype_code, n, m))


@functools.lru_cache(maxsize=1024)
def _conv_need(B, H, Wd, C_in, C_out, R, S, stride, pad, dt, n, m) -> int:
    """What sdgp_conv_bwd_data is given: nothing for the layers whose workspace no kernel reads, whatever the query says."""
    need = conv_bwd_data_workspace(B, H, Wd, C_in, C_out, R, S, stride, pad, dt, n, m)
    unread = dt == BF16 and R == S == stride == 1 and C_out % 32 != 0
    return 0 if unread and need != 2**64 - 1 else need


def sdgp_conv_bwd_data(dO: torch.Tensor, W: torch.Tensor, H: int, Wd: int, stride: int, pad: int, n: int, m: int,
                       ranker: int, seed: int = 0, out: torch.Tensor | None = None,
                       workspace: torch.Tensor | None = None) -> torch.Tensor:
    """dD [B,H,Wd,C_in] from dO [B,P,Q,C_out] (NHWC) and W [C_out,R,S,C_in]."""
    _dev(dO, "dO"), _dev(W, "W")
    if dO.dim() != 4 or W.dim() != 4 or W.shape[0] != dO.shape[3] or W.dtype != dO.dtype:
        raise ValueError("expected dO [B,P,Q,C_out] and W [C_out,R,S,C_in] of one dtype")
    B, P, Q, C_out = dO.shape
    _, R, S, C_in = W.shape
    if (H + 2 * pad - R) // stride + 1 != P or (Wd + 2 * pad - S) // stride + 1 != Q:
        raise ValueError("dO's spatial size does not match H, Wd, stride, pad")
    if out is None:
        out = dO.new_empty((B, H, Wd, C_in))
    _dev(out, "out")
    dt = _dtype_code(dO)
    need = _conv_need(B, H, Wd, C_in, C_out, R, S, stride, pad, dt, n, m)
    if need == 2**64 - 1:
        raise SdgpError(-3, "sdgp_conv_bwd_data_workspace")
    if need and (workspace is None or workspace.numel() * workspace.element_size() < need):
        try:
            workspace = torch.empty(need, dtype=torch.uint8, device=dO.device)
        except torch.OutOfMemoryError:
            if dt != F32:
                raise
            workspace = None    # (fp32 runs without, on another kernel)
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = load().sdgp_conv_bwd_data(_ptr(dO), _ptr(W), _ptr(out), B, H, Wd, C_in, C_out, R, S, stride, pad, dt, n, m,
                                   ranker, seed & (2**64 - 1), _ptr(workspace), wbytes, _stream(dO))
    if rc != 0:
        raise SdgpError(rc, "sdgp_conv_bwd_data")
    return out


def sdgp_conv_bwd_data_noalloc(dO: torch.Tensor, W: torch.Tensor, H: int, Wd: int, stride: int, pad: int, n: int, m: int,
                               ranker: int, seed: int, out: torch.Tensor) -> torch.Tensor:
    """sdgp_conv_bwd_data into the caller's ``out`` without a workspace: scratch comes from the library's own array."""
    _dev(dO, "dO"), _dev(W, "W"), _dev(out, "out")
    if dO.dim() != 4 or W.dim() != 4 or W.shape[0] != dO.shape[3] or W.dtype != dO.dtype:
        raise ValueError("expected dO [B,P,Q,C_out] and W [C_out,R,S,C_in] of one dtype")
    B, P, Q, C_out = dO.shape
    _, R, S, C_in = W.shape
    if (H + 2 * pad - R) // stride + 1 != P or (Wd + 2 * pad - S) // stride + 1 != Q:
        raise ValueError("dO's spatial size does not match H, Wd, stride, pad")
    if tuple(out.shape) != (B, H, Wd, C_in) or out.dtype != dO.dtype:
        raise ValueError("out must be [B,H,Wd,C_in] of dO's dtype")
    rc = load().sdgp_conv_bwd_data_noalloc(_ptr(dO), _ptr(W), _ptr(out), B, H, Wd, C_in, C_out, R, S, stride, pad,
                                           _dtype_code(dO), n, m, ranker, seed & (2**64 - 1), _stream(dO))
    if rc != 0:
        raise SdgpError(rc, "sdgp_conv_bwd_data_noalloc")
    return out


# ---------------------------------------------- Rescaled Magnitude, one factor per channel

_INVALID = 2**64 - 1


def _workspace(need: int, workspace, device, where: str):
    if need == _INVALID:
        raise SdgpError(-3, where)
    if workspace is None or workspace.numel() * workspace.element_size() < need:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=device)
    return workspace, workspace.numel() * workspace.element_size()


def sdgp_channel_scales(dO: torch.Tensor, n: int, m: int, *, sums: bool = False, workspace: torch.Tensor | None = None):
    """Per-channel factors of ``dO`` ([..., C]) under Magnitude n:m pruning: fp32 [C]; with ``sums`` also the two
    fp64 column sums as a [2, C] tensor (all |x|, kept |x|)."""
    _dev(dO, "dO")
    C = dO.shape[-1]
    rows = dO.numel() // C if C else 0
    dt = _dtype_code(dO)
    lib = load()
    workspace, wbytes = _workspace(_need("sdgp_channel_scales_workspace", rows, C, dt, n, m), workspace, dO.device,
                                   "sdgp_channel_scales_workspace")
    scale = torch.empty(C, dtype=torch.float32, device=dO.device)
    both = torch.empty((2, C), dtype=torch.float64, device=dO.device) if sums else None
    rc = lib.sdgp_channel_scales(_ptr(dO), rows, C, dt, n, m, _ptr(scale), _ptr(both), _ptr(workspace), wbytes, _stream(dO))
    if rc != 0:
        raise SdgpError(rc, "sdgp_channel_scales")
    return (scale, both) if sums else scale


def sdgp_prune_channel_rescaled(dO: torch.Tensor, n: int, m: int, scale: torch.Tensor | None = None) -> torch.Tensor:
    """Magnitude n:m pruning of ``dO`` with kept values multiplied by their channel's factor (computed when not given)."""
    _dev(dO, "dO")
    C = dO.shape[-1]
    rows = dO.numel() // C if C else 0
    if scale is None:
        scale = sdgp_channel_scales(dO, n, m)
    _dev(scale, "scale")
    if scale.dtype != torch.float32 or scale.numel() != C:
        raise ValueError("scale must be float32 [C]")
    out = torch.empty_like(dO)
    rc = load().sdgp_prune_channel_rescaled(_ptr(dO), rows, C, _dtype_code(dO), n, m, _ptr(scale), _ptr(out), _stream(dO))
    if rc != 0:
        raise SdgpError(rc, "sdgp_prune_channel_rescaled")
    return out


def sdgp_scale_filter(W: torch.Tensor, scale: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
    """``W[k, ...] * scale[k]`` for a filter whose first axis is C_out."""
    _dev(W, "W"), _dev(scale, "scale")
    C_out = W.shape[0]
    if scale.dtype != torch.float32 or scale.numel() != C_out:
        raise ValueError("scale must be float32 [C_out]")
    if out is None:
        out = torch.empty_like(W)
    _dev(out, "out")
    inner = W.numel() // C_out if C_out else 0
    rc = load().sdgp_scale_filter(_ptr(W), _ptr(scale), _ptr(out), C_out, inner, _dtype_code(W), _stream(W))
    if rc != 0:
        raise SdgpError(rc, "sdgp_scale_filter")
    return out


def sdgp_peak_probe(kind: int, a: torch.Tensor | None, b: torch.Tensor, nbytes: int = 0, iters: int = 1) -> float:
    """One launch of a measurement kernel (0 copy a -> b, 1 read a, 2 dense / 3 structured-sparse matrix instructions);
    returns the bytes or floating-point operations of the launch.  The caller times it."""
    _dev(b, "b")
    if a is not None:
        _dev(a, "a")
    work = ctypes.c_double(0.0)
    rc = load().sdgp_peak_probe(int(kind), _ptr(a) if a is not None else None, _ptr(b), int(nbytes), int(iters),
                                ctypes.byref(work), _stream(b))
    if rc != 0:
        raise SdgpError(rc, "sdgp_peak_probe")
    return work.value


def sdgp_conv_bwd_data_channel_rescaled(dO: torch.Tensor, W: torch.Tensor, H: int, Wd: int, stride: int, pad: int,
                                        n: int, m: int, out: torch.Tensor | None = None,
                                        workspace: torch.Tensor | None = None) -> torch.Tensor:
    """dD of a convolution from dO pruned by Magnitude and rescaled per channel, in one call."""
    _dev(dO, "dO"), _dev(W, "W")
    if dO.dim() != 4 or W.dim() != 4 or W.shape[0] != dO.shape[3] or W.dtype != dO.dtype:
        raise ValueError("expected dO [B,P,Q,C_out] and W [C_out,R,S,C_in] of one dtype")
    B, P, Q, C_out = dO.shape
    _, R, S, C_in = W.shape
    if (H + 2 * pad - R) // stride + 1 != P or (Wd + 2 * pad - S) // stride + 1 != Q:
        raise ValueError("dO's spatial size does not match H, Wd, stride, pad")
    if out is None:
        out = dO.new_empty((B, H, Wd, C_in))
    _dev(out, "out")
    dt = _dtype_code(dO)
    lib = load()
    need = _need("sdgp_conv_bwd_data_channel_rescaled_workspace", B, H, Wd, C_in, C_out, R, S, stride, pad, dt, n, m)
    workspace, wbytes = _workspace(need, workspace, dO.device, "sdgp_conv_bwd_data_channel_rescaled_workspace")
    rc = lib.sdgp_conv_bwd_data_channel_rescaled(_ptr(dO), _ptr(W), _ptr(out), B, H, Wd, C_in, C_out, R, S, stride, pad,
                                                 dt, n, m, _ptr(workspace), wbytes, _stream(dO))
    if rc != 0:
        raise SdgpError(rc, "sdgp_conv_bwd_data_channel_rescaled")
    return out


def sdgp_linear_bwd_data_channel_rescaled(dO: torch.Tensor, W: torch.Tensor, n: int, m: int) -> torch.Tensor:
    """The same for a linear layer (dO [rows, C_out], W [C_out, C_in]): a 1x1 convolution over rows pixels."""
    if dO.dim() != 2 or W.dim() != 2:
        raise ValueError("expected dO [rows, C_out] and W [C_out, C_in]")
    rows, C_out = dO.shape
    out = sdgp_conv_bwd_data_channel_rescaled(dO.view(rows, 1, 1, C_out), W.view(C_out, 1, 1, W.shape[1]), 1, 1, 1, 0, n, m)
    return out.view(rows, W.shape[1])


def sdgp_conv_bwd_data_compact(dO: torch.Tensor, W: torch.Tensor, H: int, Wd: int, stride: int, pad: int, n: int, m: int,
                               ranker: int, seed: int = 0, out: torch.Tensor | None = None,
                               workspace: torch.Tensor | None = None) -> torch.Tensor:
    """sdgp_conv_bwd_data through the compacted gradient: prune pass to (values, positions), then one AXPY per kept value."""
    _dev(dO, "dO"), _dev(W, "W")
    if dO.dim() != 4 or W.dim() != 4 or W.shape[0] != dO.shape[3] or W.dtype != dO.dtype:
        raise ValueError("expected dO [B,P,Q,C_out] and W [C_out,R,S,C_in] of one dtype")
    B, P, Q, C_out = dO.shape
    _, R, S, C_in = W.shape
    if (H + 2 * pad - R) // stride + 1 != P or (Wd + 2 * pad - S) // stride + 1 != Q:
        raise ValueError("dO's spatial size does not match H, Wd, stride, pad")
    if out is None:
        out = dO.new_empty((B, H, Wd, C_in))
    _dev(out, "out")
    dt = _dtype_code(dO)
    lib = load()
    need = _need("sdgp_conv_bwd_data_compact_workspace", B, H, Wd, C_in, C_out, R, S, stride, pad, dt, n, m)
    workspace, wbytes = _workspace(need, workspace, dO.device, "sdgp_conv_bwd_data_compact_workspace")
    rc = lib.sdgp_conv_bwd_data_compact(_ptr(dO), _ptr(W), _ptr(out), B, H, Wd, C_in, C_out, R, S, stride, pad, dt, n, m,
                                        ranker, seed & (2**64 - 1), _ptr(workspace), wbytes, _stream(dO))
    if rc != 0:
        raise SdgpError(rc, "sdgp_conv_bwd_data_compact")
    return out


def sdgp_conv_bwd_data_grouped(dO: torch.Tensor, W: torch.Tensor, H: int, Wd: int, stride: int, pad: int, groups: int,
                               n: int, m: int, ranker: int, seed: int = 0, out: torch.Tensor | None = None,
                               workspace: torch.Tensor | None = None) -> torch.Tensor:
    """sdgp_conv_bwd_data for a grouped convolution: dO [B,P,Q,C_out], W [C_out,R,S,C_in/groups] -> dD [B,H,Wd,C_in]."""
    _dev(dO, "dO"), _dev(W, "W")
    if dO.dim() != 4 or W.dim() != 4 or W.shape[0] != dO.shape[3] or W.dtype != dO.dtype:
        raise ValueError("expected dO [B,P,Q,C_out] and W [C_out,R,S,C_in/groups] of one dtype")
    B, P, Q, C_out = dO.shape
    _, R, S, cig = W.shape
    C_in = cig * groups
    if (H + 2 * pad - R) // stride + 1 != P or (Wd + 2 * pad - S) // stride + 1 != Q:
        raise ValueError("dO's spatial size does not match H, Wd, stride, pad")
    if out is None:
        out = dO.new_empty((B, H, Wd, C_in))
    _dev(out, "out")
    dt = _dtype_code(dO)
    lib = load()
    need = _need("sdgp_conv_bwd_data_grouped_workspace", B, H, Wd, C_in, C_out, R, S, stride, pad, groups, dt, n, m)
    workspace, wbytes = _workspace(need, workspace, dO.device, "sdgp_conv_bwd_data_grouped_workspace")
    rc = lib.sdgp_conv_bwd_data_grouped(_ptr(dO), _ptr(W), _ptr(out), B, H, Wd, C_in, C_out, R, S, stride, pad, groups, dt,
                                        n, m, ranker, seed & (2**64 - 1), _ptr(workspace), wbytes, _stream(dO))
    if rc != 0:
        raise SdgpError(rc, "sdgp_conv_bwd_data_grouped")
    return out


# ---------------------------------------------- the two other products of a layer's step (nothing is pruned)

def sdgp_conv_fwd(D: torch.Tensor, W: torch.Tensor, stride: int, pad: int, out: torch.Tensor | None = None,
                  workspace: torch.Tensor | None = None) -> torch.Tensor:
    """O [B,P,Q,C_out] from D [B,H,Wd,C_in] (NHWC) and W [C_out,R,S,C_in]."""
    _dev(D, "D"), _dev(W, "W")
    if D.dim() != 4 or W.dim() != 4 or W.shape[3] != D.shape[3] or W.dtype != D.dtype:
        raise ValueError("expected D [B,H,Wd,C_in] and W [C_out,R,S,C_in] of one dtype")
    B, H, Wd, C_in = D.shape
    C_out, R, S, _ = W.shape
    P, Q = (H + 2 * pad - R) // stride + 1, (Wd + 2 * pad - S) // stride + 1
    if out is None:
        out = torch.empty((B, max(P, 0), max(Q, 0), C_out), dtype=D.dtype, device=D.device)
    _dev(out, "out")
    dt = _dtype_code(D)
    lib = load()
    need = _need("sdgp_conv_fwd_workspace", B, H, Wd, C_in, C_out, R, S, stride, pad, dt)
    workspace, wbytes = _workspace(need, workspace, D.device, "sdgp_conv_fwd_workspace")
    rc = lib.sdgp_conv_fwd(_ptr(D), _ptr(W), _ptr(out), B, H, Wd, C_in, C_out, R, S, stride, pad, dt, _ptr(workspace), wbytes,
                           _stream(D))
    if rc != 0:
        raise SdgpError(rc, "sdgp_conv_fwd")
    return out


def sdgp_conv_bwd_weight(D: torch.Tensor, dO: torch.Tensor, R: int, S: int, stride: int, pad: int,
                         out: torch.Tensor | None = None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """dW [C_out,R,S,C_in] in float32 from D [B,H,Wd,C_in] and the unpruned dO [B,P,Q,C_out]."""
    _dev(D, "D"), _dev(dO, "dO")
    if D.dim() != 4 or dO.dim() != 4 or dO.shape[0] != D.shape[0] or dO.dtype != D.dtype:
        raise ValueError("expected D [B,H,Wd,C_in] and dO [B,P,Q,C_out] of one dtype")
    B, H, Wd, C_in = D.shape
    _, P, Q, C_out = dO.shape
    if (H + 2 * pad - R) // stride + 1 != P or (Wd + 2 * pad - S) // stride + 1 != Q:
        raise ValueError("dO's spatial size does not match D, R, S, stride, pad")
    if out is None:
        out = torch.empty((C_out, R, S, C_in), dtype=torch.float32, device=D.device)
    _dev(out, "out")
    if out.dtype != torch.float32 or tuple(out.shape) != (C_out, R, S, C_in):
        raise ValueError("out must be float32 [C_out,R,S,C_in]")
    dt = _dtype_code(D)
    lib = load()
    need = _need("sdgp_conv_bwd_weight_workspace", B, H, Wd, C_in, C_out, R, S, stride, pad, dt)
    workspace, wbytes = _workspace(need, workspace, D.device, "sdgp_conv_bwd_weight_workspace")
    rc = lib.sdgp_conv_bwd_weight(_ptr(D), _ptr(dO), _ptr(out), B, H, Wd, C_in, C_out, R, S, stride, pad, dt,
                                  _ptr(workspace), wbytes, _stream(D))
    if rc != 0:
        raise SdgpError(rc, "sdgp_conv_bwd_weight")
    return out


# ---------------------------------------------- around the pruned layers: the loss, the norms between blocks

def _row_stride(t: torch.Tensor, name: str) -> int:
    """The distance of two rows of ``t`` ([..., V], last stride 1, leading axes evenly spaced)."""
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if t.is_contiguous():
        return t.shape[-1]
    if t.dim() == 2 and t.stride(1) == 1 and t.stride(0) >= t.shape[1]:
        return t.stride(0)
    V = t.shape[-1]
    expect = None
    for size, stride in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if expect is None:
            ld, expect = stride, stride * size
        elif stride == expect:
            expect *= size
        else:
            raise ValueError(f"the rows of {name} must be evenly spaced")
    if expect is None:
        ld = V
    if (V > 1 and t.stride(-1) != 1) or ld < V:
        raise ValueError(f"{name} must have rows with stride 1 that do not overlap")
    return ld


def _beside(t: torch.Tensor, name: str, x: torch.Tensor) -> torch.Tensor:
    if t.get_device() != x.get_device():
        raise ValueError(f"{name} must live on the GPU of the other tensors")
    return _dev(t, name)


def _per_row(t: torch.Tensor, shape, name: str, dtypes, x: torch.Tensor) -> torch.Tensor:
    _beside(t, name, x)
    if t.shape != shape or t.dtype not in dtypes:
        raise ValueError(f"{name} must be {' or '.join(str(d) for d in dtypes)} {tuple(shape)}")
    return t


def _own_workspace(need: int, workspace, x: torch.Tensor, where: str):
    if workspace is not None:
        _beside(workspace, "workspace", x)
    return _workspace(need, workspace, x.device, where)


_FLOAT, _INTS = (torch.float32,), (torch.int64, torch.int32)


def sdgp_token_logprobs(logits: torch.Tensor, tokens: torch.Tensor | None, *, top: int = 0, scale: float = 1.0,
                        workspace: torch.Tensor | None = None):
    """Log probabilities of ``tokens`` ([...], < 0 for none) under softmax(scale * logits) ([..., V]), each row's entropy
    and its ``top`` best alternatives.  Returns ``(logp, entropy, top_logp, top_ids, stats)``; what is not asked for is
    None, ``stats`` is for ``sdgp_token_logprobs_bwd``."""
    if logits.dim() < 1:
        raise ValueError("expected logits [..., V]")
    ld, dt = _row_stride(logits, "logits"), _dtype_code(logits)
    shape, V = logits.shape[:-1], logits.shape[-1]
    rows = shape.numel()
    bits = 64
    if tokens is not None:
        _per_row(tokens, shape, "tokens", _INTS, logits)
        bits = 64 if tokens.dtype == torch.int64 else 32
    lib = load()
    need = _need("sdgp_token_logprobs_workspace", rows, V, dt, top)
    if need == _INVALID:
        raise SdgpError(-3, "sdgp_token_logprobs")
    wbytes = 0
    if need:
        workspace, wbytes = _own_workspace(need, workspace, logits, "sdgp_token_logprobs_workspace")
    entropy = logits.new_empty(shape, dtype=torch.float32)
    logp = None if tokens is None else torch.empty_like(entropy)
    stats = entropy.new_empty((*shape, 2))
    top_logp = top_ids = None
    if top:
        top_logp, top_ids = entropy.new_empty((*shape, top)), entropy.new_empty((*shape, top), dtype=torch.int64)
    rc = lib.sdgp_token_logprobs(_ptr(logits), ld, _ptr(tokens), bits, _ptr(logp), _ptr(entropy), _ptr(top_logp), _ptr(top_ids),
                                 _ptr(stats), rows, V, dt, top, scale, _ptr(workspace) if need else None, wbytes, _stream(logits))
    if rc != 0:
        raise SdgpError(rc, "sdgp_token_logprobs")
    return logp, entropy, top_logp, top_ids, stats


def sdgp_token_logprobs_bwd(logits: torch.Tensor, tokens: torch.Tensor | None, stats: torch.Tensor, entropy: torch.Tensor | None,
                            g_logp: torch.Tensor | None, g_entropy: torch.Tensor | None = None, *, scale: float = 1.0,
                            out: torch.Tensor | None = None) -> torch.Tensor:
    """dL/dlogits from dL/dlogp and dL/dentropy (fp32 [...], either may be None): what ``sdgp_linear_bwd_data`` takes as
    dO.  ``out`` may be ``logits`` itself."""
    ld, dt = _row_stride(logits, "logits"), _dtype_code(logits)
    shape, V = logits.shape[:-1], logits.shape[-1]
    if g_logp is None and g_entropy is None:
        raise ValueError("one of g_logp and g_entropy is needed")
    _per_row(stats, (*shape, 2), "stats", _FLOAT, logits)
    bits = 64
    if g_logp is not None:
        if tokens is None:
            raise ValueError("g_logp needs tokens")
        _per_row(g_logp, shape, "g_logp", _FLOAT, logits)
        _per_row(tokens, shape, "tokens", _INTS, logits)
        bits = 64 if tokens.dtype == torch.int64 else 32
    if g_entropy is not None:
        if entropy is None:
            raise ValueError("g_entropy needs entropy")
        _per_row(g_entropy, shape, "g_entropy", _FLOAT, logits)
        _per_row(entropy, shape, "entropy", _FLOAT, logits)
    if out is None:
        out = logits.new_empty(logits.shape)
    if out.shape != logits.shape or out.dtype != logits.dtype or out.get_device() != logits.get_device():
        raise ValueError("out must have the shape, dtype and GPU of logits")
    rc = load().sdgp_token_logprobs_bwd(_ptr(logits), ld, None if g_logp is None else _ptr(tokens), bits, _ptr(stats), _ptr(entropy), _ptr(g_logp),
                                        _ptr(g_entropy), _ptr(out), _row_stride(out, "out"), shape.numel(), V, dt, scale,
                                        _stream(logits))
    if rc != 0:
        raise SdgpError(rc, "sdgp_token_logprobs_bwd")
    return out


def _like(t, x: torch.Tensor, name: str):
    if t is not None:
        _beside(t, name, x)
        if t.shape != x.shape or t.dtype != x.dtype:
            raise ValueError(f"{name} must have the shape and dtype of the residual stream")


def _gate_and_weights(D: int, rows: int, x: torch.Tensor, gate, w_post, w_pre):
    """(groups, code of the weights' dtype) of checked arguments."""
    groups = 0
    if gate is not None:
        _beside(gate, "gate", x)
        if gate.shape[-1] != D or gate.dtype != x.dtype:
            raise ValueError("gate must be [..., D] of the residual stream's dtype")
        groups = gate.numel() // D
        if groups == 0 and rows or groups and rows % groups:
            raise ValueError("the rows must be a multiple of the gate's")
    wdt = F32
    for w, name in ((w_post, "w_post"), (w_pre, "w_pre")):
        if w is not None:
            _beside(w, name, x)
            if w.shape != (D,):
                raise ValueError(f"{name} must be [D]")
            wdt = _dtype_code(w)
    if w_post is not None and w_pre is not None and w_post.dtype != w_pre.dtype:
        raise ValueError("w_post and w_pre must have one dtype")
    return groups, wdt


def sdgp_block_norm(x: torch.Tensor, u: torch.Tensor | None = None, gate: torch.Tensor | None = None,
                    w_post: torch.Tensor | None = None, w_pre: torch.Tensor | None = None, *, residual_scale: float = 1.0,
                    eps: float = 1e-6, pre: bool = True):
    """y = residual_scale * x + gate * (rms_norm(u) * w_post) and h = rms_norm(y) * w_pre over the last axis, in one pass.

    ``u``: the block's output, None where there is none yet (y is then ``x`` itself).  ``gate``: [D], or [G, D] with row r
    of the flattened x using gate r // (rows / G).  ``pre=False``: no norm follows, h is None.  Returns ``(y, h, stats)``;
    ``stats`` is for ``sdgp_block_norm_bwd``."""
    _dev(x, "x")
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError("expected x [..., D]")
    _like(u, x, "u")
    if u is None and (gate is not None or w_post is not None or not pre):
        raise ValueError("gate and w_post belong to a block's output, and without one there is only the norm")
    if not pre and w_pre is not None:
        raise ValueError("w_pre is the weight of the norm that pre=False leaves out")
    D = x.shape[-1]
    rows = x.numel() // D
    groups, wdt = _gate_and_weights(D, rows, x, gate, w_post, w_pre)
    y = x if u is None else torch.empty_like(x)
    h = torch.empty_like(x) if pre else None
    stats = torch.empty((2, rows), dtype=torch.float32, device=x.device)
    rc = load().sdgp_block_norm(_ptr(x), _ptr(u), _ptr(gate), _ptr(w_post), _ptr(w_pre), None if u is None else _ptr(y), _ptr(h),
                                _ptr(stats), rows, D, groups, _dtype_code(x), wdt, residual_scale, eps, _stream(x))
    if rc != 0:
        raise SdgpError(rc, "sdgp_block_norm")
    return y, h, stats


def sdgp_block_norm_bwd(dy: torch.Tensor | None, dh: torch.Tensor | None, y: torch.Tensor, stats: torch.Tensor,
                        u: torch.Tensor | None = None, gate: torch.Tensor | None = None, w_post: torch.Tensor | None = None,
                        w_pre: torch.Tensor | None = None, *, residual_scale: float = 1.0, workspace: torch.Tensor | None = None):
    """Gradients of ``sdgp_block_norm``: ``(dx, du, dgate, dw_post, dw_pre)``, the weights' in fp32, None for what was not
    given.  ``dh`` is None exactly where the call left h out; ``dy`` None counts as 0."""
    _dev(y, "y")
    for t, name in ((dy, "dy"), (dh, "dh"), (u, "u")):
        _like(t, y, name)
    if dy is None and dh is None:
        raise ValueError("one of dy and dh is needed")
    if u is None and (gate is not None or w_post is not None) or dh is None and w_pre is not None:
        raise ValueError("gate and w_post belong to a block's output, w_pre to the norm behind it")
    D = y.shape[-1]
    rows = y.numel() // D
    _per_row(stats, (2, rows), "stats", _FLOAT, y)
    groups, wdt = _gate_and_weights(D, rows, y, gate, w_post, w_pre)
    dt = _dtype_code(y)
    lib = load()
    workspace, wbytes = _own_workspace(_need("sdgp_block_norm_bwd_workspace", rows, D, groups, dt), workspace, y,
                                       "sdgp_block_norm_bwd_workspace")
    dx = torch.empty_like(y)
    du = None if u is None else torch.empty_like(y)
    dgate = None if gate is None else torch.empty_like(gate)
    dw_post, dw_pre = (None if w is None else torch.empty(D, dtype=torch.float32, device=y.device) for w in (w_post, w_pre))
    rc = lib.sdgp_block_norm_bwd(_ptr(dy), _ptr(dh), _ptr(y), _ptr(u), _ptr(gate), _ptr(w_post), _ptr(w_pre), _ptr(stats), _ptr(dx),
                                 _ptr(du), _ptr(dgate), _ptr(dw_post), _ptr(dw_pre), rows, D, groups, dt, wdt, residual_scale,
                                 _ptr(workspace), wbytes, _stream(y))
    if rc != 0:
        raise SdgpError(rc, "sdgp_block_norm_bwd")
    return dx, du, dgate, dw_post, dw_pre


# ---------------------------------------------- packed sequences: attention, positions, losses of the log probabilities

_current_gpu = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _launch(name: str, x: torch.Tensor, *args) -> None:
    """Calls the library on the GPU of ``x``, whichever the current one is."""
    call = getattr(load(), name)
    if x.get_device() == _current_gpu():
        rc = call(*args, _stream(x))
    else:
        with torch.cuda.device(x.get_device()):
            rc = call(*args, _stream(x))
    if rc != 0:
        raise SdgpError(rc, name)


def _heads(t: torch.Tensor, name: str, packed: bool, x: torch.Tensor | None = None):
    """(distance of two tokens, of two heads) of ``t``, [T, heads, D] packed or [B, L, heads, D]."""
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if x is not None and (t.get_device() != x.get_device() or t.dtype != x.dtype):
        raise ValueError(f"{name} must have the dtype and the GPU of the other tensors")
    if t.dim() != (3 if packed else 4):
        raise ValueError(f"{name} must be {'[T, heads, D] with offsets' if packed else '[B, L, heads, D] without offsets'}")
    stride, shape = t.stride(), t.shape
    if shape[-1] > 1 and stride[-1] != 1:
        raise ValueError(f"the values of a head of {name} must have stride 1")
    if packed:
        return stride[0], stride[1]
    if shape[0] > 1 and shape[1] > 1 and stride[0] != shape[1] * stride[1]:
        raise ValueError(f"the tokens of {name} must be evenly spaced")
    return (stride[1] if shape[1] > 1 else stride[0]), stride[2]


def _offsets(offsets, name: str, x: torch.Tensor) -> torch.Tensor:
    _beside(offsets, name, x)
    if offsets.dtype != torch.int32 or offsets.dim() != 1 or offsets.numel() < 1:
        raise ValueError(f"{name} must be int32 [sequences + 1]")
    return offsets


def _attention_sizes(q, k, v, offsets, offsets_k, scale):
    """Checked arguments: (strides, offsets, offsets_k, sequences, Tq, Tk, H, Hk, D, dtype, scale)."""
    packed = offsets is not None
    strides = (*_heads(q, "q", packed), *_heads(k, "k", packed, q), *_heads(v, "v", packed, q))
    if v.shape != k.shape or k.shape[-1] != q.shape[-1] or (not packed and k.shape[0] != q.shape[0]):
        raise ValueError("k and v must have one shape, with q's head size and batch")
    H, D = q.shape[-2:]
    Hk = k.shape[-2]
    if Hk == 0 or H % Hk or H == 0:
        raise ValueError("the heads of q must be a multiple of those of k and v")
    if packed:
        _offsets(offsets, "offsets", q)
        if offsets_k is None:
            offsets_k = offsets
            if k.shape[0] != q.shape[0]:
                raise ValueError("k has other tokens than q: offsets_k is needed")
        elif _offsets(offsets_k, "offsets_k", q).numel() != offsets.numel():
            raise ValueError("offsets and offsets_k must be of one length")
        sequences, Tq, Tk = offsets.numel() - 1, q.shape[0], k.shape[0]
    else:
        if offsets_k is not None:
            raise ValueError("offsets_k belongs to offsets")
        sequences, Tq, Tk = q.shape[0], q.shape[0] * q.shape[1], k.shape[0] * k.shape[1]
    if scale is None:
        scale = D ** -0.5
    return (ctypes.c_int64 * 6)(*strides), offsets, offsets_k, sequences, Tq, Tk, H, Hk, D, _dtype_code(q), scale


def sdgp_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, offsets: torch.Tensor | None = None,
                   offsets_k: torch.Tensor | None = None, *, lengths: torch.Tensor | None = None, causal: bool = True,
                   scale: float | None = None, workspace: torch.Tensor | None = None):
    """``(o, lse)``: softmax attention, query head h of ``q`` on key head h // (H / Hk) of ``k`` and ``v``.

    With ``offsets`` (int32 [sequences + 1]) q is [T, H, D], k and v [T, Hk, D], sequences one behind the other; ``offsets_k``
    where the keys' differ.  Without, q is [B, L, H, D], k and v [B, Lk, Hk, D], and ``lengths`` (int32 [B]) says how many
    of the Lk keys there are (a cache).  Tokens and heads may be strided, a batch's tokens evenly: a cache is given whole, with
    ``lengths``.  Plans go by mean lengths: a long prompt and a few single tokens are faster as two calls.  ``causal``: the last query sees all keys, the one
    before all but the last, and so on.  ``scale``: D ** -0.5 by default."""
    strides, offsets, offsets_k, S, Tq, Tk, H, Hk, D, dt, scale = _attention_sizes(q, k, v, offsets, offsets_k, scale)
    if lengths is not None:
        if offsets is not None:
            raise ValueError("lengths are for keys without offsets")
        _per_row(lengths, (S,), "lengths", (torch.int32,), q)
    need = _need("sdgp_attention_workspace", S, Tq, Tk, H, Hk, D, dt)
    if need == _INVALID:
        raise SdgpError(-3, "sdgp_attention")
    wbytes = 0
    if need:
        workspace, wbytes = _own_workspace(need, workspace, q, "sdgp_attention_workspace")
    o, lse = q.new_empty(q.shape), q.new_empty(q.shape[:-1], dtype=torch.float32)
    _launch("sdgp_attention", q, _ptr(q), _ptr(k), _ptr(v), strides, _ptr(offsets), _ptr(offsets_k), _ptr(lengths), S, _ptr(o), _ptr(lse),
            Tq, Tk, H, Hk, D, dt, int(causal), scale, _ptr(workspace) if need else None, wbytes)
    return o, lse


def sdgp_attention_bwd(do: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor, lse: torch.Tensor,
                       offsets: torch.Tensor | None = None, offsets_k: torch.Tensor | None = None, *, causal: bool = True,
                       scale: float | None = None, workspace: torch.Tensor | None = None):
    """``(dq, dk, dv)`` from the gradient of ``o`` and what ``sdgp_attention`` took and returned."""
    strides, offsets, offsets_k, S, Tq, Tk, H, Hk, D, dt, scale = _attention_sizes(q, k, v, offsets, offsets_k, scale)
    for t, name in ((do, "do"), (o, "o")):
        _per_row(t, q.shape, name, (q.dtype,), q)
    _per_row(lse, q.shape[:-1], "lse", _FLOAT, q)
    need = _need("sdgp_attention_bwd_workspace", S, Tq, Tk, H, Hk, D, dt)
    if need == _INVALID:
        raise SdgpError(-3, "sdgp_attention_bwd")
    workspace, wbytes = _own_workspace(need, workspace, q, "sdgp_attention_bwd_workspace")
    dq, dk, dv = q.new_empty(q.shape), q.new_empty(k.shape), q.new_empty(k.shape)
    _launch("sdgp_attention_bwd", q, _ptr(do), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), strides, _ptr(offsets), _ptr(offsets_k), S,
            _ptr(dq), _ptr(dk), _ptr(dv), Tq, Tk, H, Hk, D, dt, int(causal), scale, _ptr(workspace), wbytes)
    return dq, dk, dv


def _tokens(t: torch.Tensor, name: str, x: torch.Tensor | None = None):
    """(distance of two tokens, of two heads) of ``t`` ([..., heads, D], the tokens evenly spaced)."""
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if x is not None and (t.get_device() != x.get_device() or t.dtype != x.dtype):
        raise ValueError(f"{name} must have the dtype and the GPU of the other tensors")
    if t.dim() < 2 or t.shape[-1] < 2:
        raise ValueError(f"expected {name} [..., heads, D]")
    stride, shape = t.stride(), t.shape
    if stride[-1] != 1:
        raise ValueError(f"the values of a head of {name} must have stride 1")
    token = expect = None
    for n, s in zip(reversed(shape[:-2]), reversed(stride[:-2])):
        if n == 1:
            continue
        if expect is not None and s != expect:
            raise ValueError(f"the tokens of {name} must be evenly spaced")
        token, expect = (s if token is None else token), s * n
    return (shape[-1] if token is None else token), stride[-2]


def _apart(a: torch.Tensor, b: torch.Tensor) -> bool:
    """Whether two tensors of heads share no memory: far from each other, or side by side in every token's values."""
    span = lambda t: sum((n - 1) * s for n, s in zip(t.shape, t.stride())) + 1  # noqa: E731
    size = a.element_size()
    if not a.numel() or not b.numel() or a.data_ptr() + span(a) * size <= b.data_ptr() or b.data_ptr() + span(b) * size <= a.data_ptr():
        return True
    (step, _), (other, _) = _tokens(a, ""), _tokens(b, "")
    if a.data_ptr() > b.data_ptr():
        a, b = b, a
    at = (b.data_ptr() - a.data_ptr()) // size
    wide = lambda t: (t.shape[-2] - 1) * t.stride(-2) + t.shape[-1]  # noqa: E731
    return step == other and at % step >= wide(a) and at % step + wide(b) <= step


def sdgp_rotary(q: torch.Tensor, k: torch.Tensor | None, positions: torch.Tensor, freqs: torch.Tensor, axes=None, *,
                interleaved: bool = False, inverse: bool = False, out=None):
    """``(q, k)`` turned by their positions; k may be None.

    ``q`` [..., H, D] and ``k`` [..., Hk, D] (tokens and heads may be strided), ``positions`` [...] or [..., axes] (int32 or
    int64), ``freqs`` fp32 [F], radians a position, 2 F <= D; values from 2 F on stay as they are.  ``axes``: how many of the
    F pairs each axis of the positions turns.  Pair i is (i, F + i), with ``interleaved`` (2 i, 2 i + 1).  ``inverse``: by
    the opposite angles, which takes gradients back.  ``out``: the pair of tensors to write, q and k themselves or others."""
    q_strides = _tokens(q, "q")
    tokens = q.shape[:-2]
    T, (H, D) = tokens.numel(), q.shape[-2:]
    _beside(positions, "positions", q), _beside(freqs, "freqs", q)
    if freqs.dtype != torch.float32 or freqs.dim() != 1 or not 1 <= 2 * freqs.numel() <= D:
        raise ValueError("freqs must be float32 [F], at most half a head's values")
    axes = (freqs.numel(),) if axes is None else tuple(int(n) for n in axes)
    if sum(axes) != freqs.numel() or any(n < 1 for n in axes) or len(axes) > 8:
        raise ValueError("axes are up to 8 numbers of pairs that add up to the frequencies")
    if positions.dtype not in _INTS or positions.shape != (*tokens, len(axes)) and (len(axes) > 1 or positions.shape != tokens):
        raise ValueError("positions must be int32 or int64, one for each token and axis")
    Hk, k_strides = 0, (0, 0)
    if k is not None:
        k_strides = _tokens(k, "k", q)
        Hk = k.shape[-2]
        if k.shape[:-2] != tokens or k.shape[-1] != D or Hk == 0:
            raise ValueError("k must have q's tokens and head size, and heads")
    if out is None:
        q_out = q.new_empty(q.shape)
        k_out = None if k is None else q.new_empty(k.shape)
    else:
        q_out, k_out = out
        if (k_out is None) != (k is None):
            raise ValueError("out holds a tensor for each of q and k")
    out_strides = []
    for y, x, name in ((q_out, q, "q"), (k_out, k, "k")):
        if x is None:
            out_strides += [0, 0]
            continue
        if out is None:
            out_strides += [x.shape[-2] * D, D]
            continue
        if y.shape != x.shape:
            raise ValueError("outputs must have the shapes of q and k")
        token, head = _tokens(y, "out", q)
        if not (y.data_ptr() == x.data_ptr() and y.stride() == x.stride() or _apart(y, x)):
            raise ValueError(f"the output for {name} must be {name} itself, or lie apart from it")
        if T > 1 and token < D or x.shape[-2] > 1 and head < D:
            raise ValueError("the heads of an output must not share memory")
        out_strides += [token, head]
    if out is not None and k is not None and not (_apart(q_out, k_out) and _apart(q_out, k) and _apart(k_out, q)):
        raise ValueError("the outputs for q and k must lie apart from each other and from the other input")
    if H == 0:
        raise ValueError("expected q with heads")
    _launch("sdgp_rotary", q, _ptr(q), _ptr(k), _ptr(q_out), _ptr(k_out), (ctypes.c_int64 * 8)(*q_strides, *k_strides, *out_strides),
            _ptr(positions), 64 if positions.dtype == torch.int64 else 32, _ptr(freqs), (ctypes.c_int32 * len(axes))(*axes), len(axes),
            T, H, Hk, D, _dtype_code(q), int(interleaved), int(inverse))
    return q_out, k_out


def _sequence_sizes(x: torch.Tensor, name: str, mask, offsets):
    """(T, sequences) of ``x``, [T] with offsets, [sequences, L] or [L] without; checks mask and offsets."""
    _dev(x, name)
    if x.dtype != torch.float32 or x.dim() != 1 and (x.dim() != 2 or offsets is not None):
        raise ValueError(f"{name} must be float32, [T] with offsets, [sequences, L] or [L] without")
    if mask is not None:
        _per_row(mask, x.shape, "mask", (torch.bool, torch.uint8), x)
    if offsets is not None:
        return x.numel(), _offsets(offsets, "offsets", x).numel() - 1
    return x.numel(), x.shape[0] if x.dim() == 2 else 1


def _policy_arguments(logp, old_logp, advantages, ref_logp, mask, offsets, clip, kl):
    T, S = _sequence_sizes(logp, "logp", mask, offsets)
    _per_row(old_logp, logp.shape, "old_logp", _FLOAT, logp)
    if ref_logp is not None:
        _per_row(ref_logp, logp.shape, "ref_logp", _FLOAT, logp)
    elif kl:
        raise ValueError("kl needs ref_logp")
    _beside(advantages, "advantages", logp)
    each = advantages.shape == logp.shape
    if advantages.dtype != torch.float32 or not each and advantages.shape not in ((S,), (S, 1)):
        raise ValueError("advantages must be float32, one for each token or one for each sequence")
    low, high = clip
    return (_ptr(old_logp), _ptr(ref_logp), _ptr(advantages), int(each), _ptr(mask), _ptr(offsets), S, T, low, high, kl), S, T


_AVERAGES = ("tokens", "sequences")


def sdgp_policy_loss(logp: torch.Tensor, old_logp: torch.Tensor, advantages: torch.Tensor, ref_logp: torch.Tensor | None = None,
                     mask: torch.Tensor | None = None, offsets: torch.Tensor | None = None, *, clip=(0.2, 0.2), kl: float = 0.0,
                     average: str = "tokens", workspace: torch.Tensor | None = None):
    """The clipped policy loss with a KL term: ``(loss, kl, clipped, weights)``.

    ``logp``, ``old_logp``, ``ref_logp``: fp32 [T] with ``offsets`` (int32 [sequences + 1]), [sequences, L] or [L] without.
    ``advantages``: of that shape, or [sequences] or [sequences, 1], the last also where packed tokens happen to be as many as
    their sequences.  ``mask``: bool or uint8, which tokens count.  The mean is over tokens, or
    with ``average="sequences"`` over the sequences' means.  ``kl`` and ``clipped`` are the mean divergence and the share of
    ratios that are cut; ``weights`` is for ``sdgp_policy_loss_bwd``."""
    if average not in _AVERAGES:
        raise ValueError('average is "tokens" or "sequences"')
    args, S, T = _policy_arguments(logp, old_logp, advantages, ref_logp, mask, offsets, clip, kl)
    workspace, wbytes = _own_workspace(_need("sdgp_sequence_loss_workspace", T, S), workspace, logp, "sdgp_sequence_loss_workspace")
    out, weights = logp.new_empty(3), logp.new_empty(S)
    _launch("sdgp_policy_loss", logp, _ptr(logp), *args, int(average == "sequences"), _ptr(out), _ptr(weights), _ptr(workspace), wbytes)
    return (*out.unbind(0), weights)


def _one(g: torch.Tensor, x: torch.Tensor) -> torch.Tensor:
    _beside(g, "g", x)
    if g.dtype != torch.float32 or g.numel() != 1:
        raise ValueError("g must be one float32")
    return g


def sdgp_policy_loss_bwd(g: torch.Tensor, weights: torch.Tensor, logp: torch.Tensor, old_logp: torch.Tensor, advantages: torch.Tensor,
                         ref_logp: torch.Tensor | None = None, mask: torch.Tensor | None = None, offsets: torch.Tensor | None = None, *,
                         clip=(0.2, 0.2), kl: float = 0.0, average: str = "tokens") -> torch.Tensor:
    """dL/dlogp from ``g`` = dL/dloss (one fp32 on the GPU) and what ``sdgp_policy_loss`` took and returned."""
    args, S, _ = _policy_arguments(logp, old_logp, advantages, ref_logp, mask, offsets, clip, kl)
    _one(g, logp), _per_row(weights, (S,), "weights", _FLOAT, logp)
    dlogp = torch.empty_like(logp)
    _launch("sdgp_policy_loss_bwd", logp, _ptr(g), _ptr(weights), _ptr(logp), *args, _ptr(dlogp))
    return dlogp


def sdgp_preference_loss(logp: torch.Tensor, ref_logp: torch.Tensor | None = None, mask: torch.Tensor | None = None,
                         offsets: torch.Tensor | None = None, *, beta: float = 0.1, margin: float = 0.0, smoothing: float = 0.0,
                         average: bool = False, workspace: torch.Tensor | None = None):
    """The loss of preferred sequences (0, 2, ..) against the rejected ones behind them (1, 3, ..): ``(loss, margins, weights)``.

    A sequence scores beta times the sum (``average``: the mean) of logp - ref_logp over its tokens that count; ``margins`` are
    the pairs' differences less ``margin``.  Shapes as for ``sdgp_policy_loss``; ``weights`` is for ``sdgp_preference_loss_bwd``."""
    T, S = _sequence_sizes(logp, "logp", mask, offsets)
    if S % 2:
        raise ValueError("sequences come in pairs")
    if ref_logp is not None:
        _per_row(ref_logp, logp.shape, "ref_logp", _FLOAT, logp)
    workspace, wbytes = _own_workspace(_need("sdgp_sequence_loss_workspace", T, S), workspace, logp, "sdgp_sequence_loss_workspace")
    loss, margins, weights = logp.new_empty(()), logp.new_empty(S // 2), logp.new_empty(S)
    _launch("sdgp_preference_loss", logp, _ptr(logp), _ptr(ref_logp), _ptr(mask), _ptr(offsets), S, T, beta, margin, smoothing, int(average),
            _ptr(loss), _ptr(margins), _ptr(weights), _ptr(workspace), wbytes)
    return loss, margins, weights


def sdgp_preference_loss_bwd(g: torch.Tensor, weights: torch.Tensor, logp: torch.Tensor, mask: torch.Tensor | None = None,
                             offsets: torch.Tensor | None = None) -> torch.Tensor:
    """dL/dlogp from ``g`` = dL/dloss (one fp32 on the GPU) and the forward call's ``weights``; of logp only the shape is used."""
    T, S = _sequence_sizes(logp, "logp", mask, offsets)
    _one(g, logp), _per_row(weights, (S,), "weights", _FLOAT, logp)
    dlogp = torch.empty_like(logp)
    _launch("sdgp_preference_loss_bwd", logp, _ptr(g), _ptr(weights), _ptr(mask), _ptr(offsets), S, T, _ptr(dlogp))
    return dlogp
