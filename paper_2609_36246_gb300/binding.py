"""Thin ctypes binding over libolive.so (include/olive.h), same entry names.

Every function here only marshals torch tensors into pointers and sizes and
calls the C ABI on the current torch CUDA stream; all computation happens in
the library's CUDA kernels.  There is no fallback: if libolive.so is missing
or fails to load, every call raises.
"""

from __future__ import annotations

import array
import ctypes
import functools
import operator
import os
import re

import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libolive.so")
HEADER = os.path.join(os.path.dirname(HERE), "include", "olive.h")

OLIVE_OK = 0
STATUS_NAMES = {
    0: "OLIVE_OK", 1: "OLIVE_ERR_INVALID_ARG", 2: "OLIVE_ERR_SHAPE", 3: "OLIVE_ERR_ALIGNMENT",
    4: "OLIVE_ERR_TOKEN_RANGE", 5: "OLIVE_ERR_OFFSETS", 6: "OLIVE_ERR_TIMEOUT",
    7: "OLIVE_ERR_UNSUPPORTED_DEVICE", 8: "OLIVE_ERR_CUDA", 9: "OLIVE_ERR_WORKSPACE",
    10: "OLIVE_ERR_BOUNDS",
}
REDUCE = {"sum": 0, "mean": 1}
DIRECTION = {"reverse": 0, "forward": 1}
DTYPE = {torch.bfloat16: 0, torch.float32: 1}
OP = {"logprob_fwd": 0, "loss_bwd": 1, "divergence": 2, "topk_fwd": 3, "splice_masked": 4,
      "topk_kl_bwd": 5, "loss_fwd_bwd": 6, "opd_stats": 7, "topk_kl_fwd_bwd": 8,
      "loss_fwd_bwd_slab": 9, "gated_mlp_fwd": 10, "gated_mlp_bwd": 11, "qk_norm_rope_bwd": 12,
      "grad_clip": 13, "row_norm_bwd": 14, "embedding_bwd": 15,
      "packed_attention_bwd": 16}
ACT = {"silu": 0, "gelu_tanh": 1}
NORM = {"layer": 0, "rms": 1}


class OliveError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)}")


_lib = None
_P = ctypes.c_void_p
_I = ctypes.c_int32
_F = ctypes.c_float
_S = ctypes.c_size_t
_L = ctypes.c_int64


def lib() -> ctypes.CDLL:
    """Loads libolive.so (raises if it is not built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise OliveError(8, f"libolive.so not found at {LIB_PATH}; build it with "
                            "paper_2609_36246_gb300.build.build()")
    _lib = _configure(ctypes.CDLL(LIB_PATH))
    return _lib


def use_library(path: str) -> ctypes.CDLL:
    """Makes every call of this module go through the library at `path`
    (e.g. the OLIVE_DEBUG build, paper_2609_36246_gb300.build.build(debug=True))
    and returns it; use_library(LIB_PATH) goes back to the release build."""
    global _lib
    _lib = _configure(ctypes.CDLL(path))
    return _lib


def _configure(L: ctypes.CDLL) -> ctypes.CDLL:
    L.olive_abi_version.restype = ctypes.c_int
    L.olive_abi_version.argtypes = []
    L.olive_status_clear.restype = ctypes.c_int
    L.olive_status_clear.argtypes = [_P, _P]
    L.olive_slab_rows.restype = _I
    L.olive_slab_rows.argtypes = [_I, _I]
    L.olive_status_string.restype = ctypes.c_char_p
    L.olive_status_string.argtypes = [ctypes.c_int]
    L.olive_workspace_size.restype = _S
    L.olive_workspace_size.argtypes = [ctypes.c_int, _I, _I, _I, _I, ctypes.c_int, ctypes.c_int]
    L.olive_splice_pack.restype = ctypes.c_int
    L.olive_splice_pack.argtypes = [_P, _P, _P, _P, _I, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P, _P]
    L.olive_token_logprob_fwd.restype = ctypes.c_int
    L.olive_token_logprob_fwd.argtypes = [_P, _P, _P, _P, _P, _I, _I, _I, _F, ctypes.c_int,
                                          _P, _P, _P, _P, _S, _P, _P]
    L.olive_token_loss_bwd.restype = ctypes.c_int
    L.olive_token_loss_bwd.argtypes = [_P, _P, _P, _P, _P, _I, _I, _I, _F, ctypes.c_int, _P, _P,
                                       _P, _P, ctypes.c_int, _P, _S, _P, _P]
    L.olive_token_divergence.restype = ctypes.c_int
    L.olive_token_divergence.argtypes = [_P, _P, _I, _P, _P, _I, _P, _P, _I, _I, _F, ctypes.c_int,
                                         _P, _P, _P, ctypes.c_int, _P, _S, _P, _P]
    L.olive_splice_pack_masked.restype = ctypes.c_int
    L.olive_splice_pack_masked.argtypes = [_P, _P, _P, _P, _P, _I, _I, _I, _P, _P, _P, _P, _P, _P,
                                           _P, _P, _S, _P, _P]
    L.olive_topk_compare.restype = ctypes.c_int
    L.olive_topk_compare.argtypes = [_P, _P, _I, _P, _P, _I, _I, _F, _I, _P, _P, _P, _P, _P, _P, _P,
                                     _P, _P]
    L.olive_scale.restype = ctypes.c_int
    L.olive_scale.argtypes = [_P, _P, _S, ctypes.c_int, _P, _P]
    L.olive_opd_token_stats.restype = ctypes.c_int
    L.olive_opd_token_stats.argtypes = [_P, _P, _I, _P, _P, _I, _P, _P, _I, _I, _F, ctypes.c_int, _I,
                                        _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _S, _P, _P]
    L.olive_token_loss_fwd_bwd.restype = ctypes.c_int
    L.olive_token_loss_fwd_bwd.argtypes = [_P, _P, _P, _P, _P, _I, _I, _I, _F, ctypes.c_int, _P, _P,
                                           _P, _P, _P, _P, ctypes.c_int, _P, _S, _P, _P]
    L.olive_token_loss_fwd_bwd_slab.restype = ctypes.c_int
    L.olive_token_loss_fwd_bwd_slab.argtypes = L.olive_token_loss_fwd_bwd.argtypes
    L.olive_topk_kl_fwd_bwd.restype = ctypes.c_int
    L.olive_topk_kl_fwd_bwd.argtypes = [_P, _P, _I, _P, _P, _I, _P, _P, _I, _I, _F, _I, _P, _P, _P,
                                        _P, _P, _P, _P, _P, _P, _P, _P, ctypes.c_int, _P, _S, _P,
                                        _P]
    L.olive_topk_kl_bwd.restype = ctypes.c_int
    L.olive_topk_kl_bwd.argtypes = [_P, _P, _P, _P, _I, _I, _I, _F, _I, _P, _P, _P, _P, _P, _P, _P,
                                    _P, ctypes.c_int, _P, _S, _P, _P]
    L.olive_token_topk_fwd.restype = ctypes.c_int
    L.olive_token_topk_fwd.argtypes = [_P, _P, _P, _P, _I, _I, _I, _F, _I, _P, _P, _P, _P, _P, _S,
                                       _P, _P]
    L.olive_token_logprob_fwd_noalloc.restype = ctypes.c_int
    L.olive_token_logprob_fwd_noalloc.argtypes = [_P, _P, _P, _P, _P, _I, _I, _I, _F, ctypes.c_int,
                                                  _P, _P, _P, _P, _P]
    view = [_P, _L, _L]
    heads = [_I, _I, _P, _P, _F, _P, _P, _P, _I, _I, _I, _I, ctypes.c_int]
    L.olive_packed_positions.restype = ctypes.c_int
    L.olive_packed_positions.argtypes = [_P, _I, _I, _P, _P]
    L.olive_qk_norm_rope_fwd.restype = ctypes.c_int
    L.olive_qk_norm_rope_fwd.argtypes = view * 2 + heads + view * 2 + [ctypes.c_int, _P, _P]
    L.olive_qk_norm_rope_bwd.restype = ctypes.c_int
    L.olive_qk_norm_rope_bwd.argtypes = (view * 4 + heads + view * 2 +
                                         [_P, _P, ctypes.c_int, _P, _S, _P, _P])
    L.olive_gated_mlp_fwd.restype = ctypes.c_int
    L.olive_gated_mlp_fwd.argtypes = [_P, _P, _P, _P, _P, _I, _I, _I, ctypes.c_int, _P, _P, _P, _S,
                                      _P, _P]
    L.olive_gated_mlp_bwd.restype = ctypes.c_int
    L.olive_gated_mlp_bwd.argtypes = [_P, _P, _P, _P, _P, _P, _I, _I, _I, ctypes.c_int, _P, _P, _P,
                                      _P, ctypes.c_int, _P, _S, _P, _P]
    L.olive_grad_clip.restype = ctypes.c_int
    L.olive_grad_clip.argtypes = [_P, _P, _P, _P, _I, _F, _P, _P, _S, _P]
    L.olive_grad_clip_apart.restype = ctypes.c_int
    L.olive_grad_clip_apart.argtypes = [_P, _P, _P, _P, _I]
    L.olive_embedding_fwd.restype = ctypes.c_int
    L.olive_embedding_fwd.argtypes = [_P, _P, _P, _I, _I, _I, _F, _P, ctypes.c_int, _P, _P]
    L.olive_embedding_bwd.restype = ctypes.c_int
    L.olive_embedding_bwd.argtypes = [_P, _P, _P, _I, _I, _I, _F, _P, ctypes.c_int, ctypes.c_int,
                                      ctypes.c_int, _P, _S, _P, _P]
    att = [_I, _I, _P, _I, _I, _I, _F, ctypes.c_int, _P, _F, _P]
    L.olive_packed_attention_fwd.restype = ctypes.c_int
    L.olive_packed_attention_fwd.argtypes = view * 3 + att + view + [_P, _P, _P]
    L.olive_packed_attention_bwd.restype = ctypes.c_int
    L.olive_packed_attention_bwd.argtypes = view * 5 + [_P] + att + view * 3 + [_P, _S, _P, _P]
    L.olive_row_norm_fwd.restype = ctypes.c_int
    L.olive_row_norm_fwd.argtypes = [_P, _P, _P, _P, _I, _I, _F, ctypes.c_int, _P, _P, _P,
                                     ctypes.c_int, _P]
    L.olive_row_norm_bwd.restype = ctypes.c_int
    L.olive_row_norm_bwd.argtypes = [_P, _P, _P, _P, _P, _I, _I, ctypes.c_int, _P, _P, _P,
                                     ctypes.c_int, _P, _S, _P]
    return L


def declared_symbols() -> list[str]:
    """Entry points declared with OLIVE_API in include/olive.h."""
    with open(HEADER) as f:
        text = f.read()
    return re.findall(r"OLIVE_API\s+[\w\s\*]*?\b(olive_\w+)\s*\(", text)


def _ptr(t):
    return None if t is None else t.data_ptr()


# The current device's index.  (torch.cuda.current_device() without its look at whether
# CUDA is initialised; what is asked for here follows a tensor that is on a device.)
_current = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream():
    # the handle of torch.cuda.current_stream() without the Stream object (2.8 us
    # of a call on the GB300's host)
    return torch._C._cuda_getCurrentRawStream(_current())


def _stream_of(device: int):
    return torch._C._cuda_getCurrentRawStream(device)


def _check(st: int, where: str):
    if st != OLIVE_OK:
        raise OliveError(st, where)


def _need(t, dtype, name):
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous CUDA {dtype} tensor")
    # the call goes to the current device's stream, where another device's address is a stray one
    if t.get_device() != _current():
        raise TypeError(f"{name} must be on the current CUDA device, {_current()}")


def new_status(device=None) -> torch.Tensor:
    dev = torch.device(device or "cuda")
    if dev.type != "cuda" or dev.index not in (None, torch.cuda.current_device()):
        return torch.zeros(1, dtype=torch.int32, device=dev)
    # a memset on the current stream (torch.zeros: 10.8 us of host time)
    st = torch.empty(1, dtype=torch.int32, device=dev)
    _check(lib().olive_status_clear(st.data_ptr(), _stream()), "olive_status_clear")
    return st


def status_bits(dev_status: torch.Tensor) -> list[str]:
    """Names of the error bits set in a device status word (synchronises)."""
    v = int(dev_status.item())
    return [STATUS_NAMES[c] for c in range(1, 11) if v & (1 << c)]


def olive_abi_version() -> int:
    return lib().olive_abi_version()


def olive_status_string(status: int) -> str:
    return lib().olive_status_string(status).decode()


def olive_workspace_size(op: str, T: int, d: int, V: int, d_t: int = 0, grad: bool = True,
                         grad_dtype=torch.bfloat16) -> int:
    return int(lib().olive_workspace_size(OP[op], T, d, d_t, V, int(grad), DTYPE[grad_dtype]))


def olive_slab_rows(T: int, V: int) -> int:
    """Rows of one G slab of the slab forms for T packed rows and V vocabulary
    entries (the library's rule, OLIVE_SLAB_ROWS included)."""
    return int(lib().olive_slab_rows(T, V))


def workspace(nbytes: int, device=None) -> torch.Tensor:
    return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device or "cuda")


def _pack_outputs(S: int, T_cap: int, dev, dev_status):
    out = {
        "ids": torch.empty(T_cap, dtype=torch.int32, device=dev),
        "targets": torch.empty(T_cap, dtype=torch.int32, device=dev),
        "loss_mask": torch.empty(T_cap, dtype=torch.uint8, device=dev),
        "cu_seqlens": torch.empty(S + 1, dtype=torch.int32, device=dev),
        "cut_offsets": torch.empty(max(S, 1), dtype=torch.int32, device=dev),
        "rows": torch.empty(T_cap, dtype=torch.int32, device=dev),
        "n_rows": torch.empty(1, dtype=torch.int32, device=dev),
    }
    out["dev_status"] = dev_status if dev_status is not None else new_status(dev)
    return out


def olive_splice_pack(prefix_ids, prefix_off, cont_ids, cont_off, V: int, T_cap: int,
                      dev_status=None) -> dict:
    """Packs the spliced sequences; returns the device outputs of olive.h."""
    for t, n in ((prefix_ids, "prefix_ids"), (prefix_off, "prefix_off"), (cont_ids, "cont_ids"),
                 (cont_off, "cont_off")):
        _need(t, torch.int32, n)
    S = prefix_off.numel() - 1
    dev = prefix_off.device
    out = _pack_outputs(S, T_cap, dev, dev_status)
    # empty id arrays still need a valid device address
    pid = prefix_ids if prefix_ids.numel() else torch.zeros(1, dtype=torch.int32, device=dev)
    cid = cont_ids if cont_ids.numel() else torch.zeros(1, dtype=torch.int32, device=dev)
    st = lib().olive_splice_pack(_ptr(pid), _ptr(prefix_off), _ptr(cid), _ptr(cont_off), S, V, T_cap,
                                 _ptr(out["ids"]), _ptr(out["targets"]), _ptr(out["loss_mask"]),
                                 _ptr(out["cu_seqlens"]), _ptr(out["cut_offsets"]),
                                 _ptr(out["rows"]), _ptr(out["n_rows"]), _ptr(out["dev_status"]),
                                 _stream())
    _check(st, "olive_splice_pack")
    return out


def olive_splice_pack_masked(prefix_ids, prefix_off, cont_ids, cont_off, cont_loss, V: int,
                             T_cap: int, dev_status=None) -> dict:
    """Multi-turn packing: cont_loss (uint8, one flag per continuation id)
    selects the teacher-action tokens that carry the loss."""
    for t, n in ((prefix_ids, "prefix_ids"), (prefix_off, "prefix_off"), (cont_ids, "cont_ids"),
                 (cont_off, "cont_off")):
        _need(t, torch.int32, n)
    _need(cont_loss, torch.uint8, "cont_loss")
    S = prefix_off.numel() - 1
    dev = prefix_off.device
    out = _pack_outputs(S, T_cap, dev, dev_status)
    pid = prefix_ids if prefix_ids.numel() else torch.zeros(1, dtype=torch.int32, device=dev)
    cid = cont_ids if cont_ids.numel() else torch.zeros(1, dtype=torch.int32, device=dev)
    cfl = cont_loss if cont_loss.numel() else torch.zeros(1, dtype=torch.uint8, device=dev)
    ws = workspace(olive_workspace_size("splice_masked", T_cap, 8, 1), dev)
    st = lib().olive_splice_pack_masked(_ptr(pid), _ptr(prefix_off), _ptr(cid), _ptr(cont_off),
                                        _ptr(cfl), S, V, T_cap, _ptr(out["ids"]),
                                        _ptr(out["targets"]), _ptr(out["loss_mask"]),
                                        _ptr(out["cu_seqlens"]), _ptr(out["cut_offsets"]),
                                        _ptr(out["rows"]), _ptr(out["n_rows"]), _ptr(ws), ws.numel(),
                                        _ptr(out["dev_status"]), _stream())
    _check(st, "olive_splice_pack_masked")
    return out


def olive_token_logprob_fwd(hidden, W, targets, rows, n_rows, inv_tau: float = 1.0,
                            reduction: str = "sum", ws=None, dev_status=None, out=None):
    """Per-token log-probs, lse and the Eq. (osd-ce) loss. Returns (logp, lse, loss)."""
    _need(hidden, torch.bfloat16, "hidden")
    _need(W, torch.bfloat16, "W")
    _need(targets, torch.int32, "targets")
    _need(rows, torch.int32, "rows")
    _need(n_rows, torch.int32, "n_rows")
    T, d = hidden.shape
    V = W.shape[0]
    if W.shape[1] != d:
        raise ValueError("hidden and W widths differ")
    dev = hidden.device
    if out is None:
        out = (torch.empty(T, dtype=torch.float32, device=dev),
               torch.empty(T, dtype=torch.float32, device=dev),
               torch.empty(1, dtype=torch.float32, device=dev))
    logp, lse, loss = out
    need = olive_workspace_size("logprob_fwd", T, d, V)
    if ws is None:
        ws = workspace(need, dev)
    ds = dev_status if dev_status is not None else new_status(dev)
    st = lib().olive_token_logprob_fwd(_ptr(hidden), _ptr(W), _ptr(targets), _ptr(rows), _ptr(n_rows),
                                       T, d, V, float(inv_tau), REDUCE[reduction], _ptr(logp),
                                       _ptr(lse), _ptr(loss), _ptr(ws), ws.numel(), _ptr(ds),
                                       _stream())
    _check(st, "olive_token_logprob_fwd")
    return logp, lse, loss


def olive_token_topk_fwd(hidden, W, rows, n_rows, K: int = 16, inv_tau: float = 1.0, ws=None,
                         dev_status=None):
    """Per-token lse, entropy and the K largest log-probs with their ids.

    Returns (lse [T], entropy [T], topk_logp [T, K], topk_ids [T, K])."""
    _need(hidden, torch.bfloat16, "hidden")
    _need(W, torch.bfloat16, "W")
    _need(rows, torch.int32, "rows")
    _need(n_rows, torch.int32, "n_rows")
    T, d = hidden.shape
    V = W.shape[0]
    dev = hidden.device
    lse = torch.empty(T, dtype=torch.float32, device=dev)
    ent = torch.empty(T, dtype=torch.float32, device=dev)
    tv = torch.empty(T, K, dtype=torch.float32, device=dev)
    ti = torch.empty(T, K, dtype=torch.int32, device=dev)
    if ws is None:
        ws = workspace(olive_workspace_size("topk_fwd", T, d, V), dev)
    ds = dev_status if dev_status is not None else new_status(dev)
    st = lib().olive_token_topk_fwd(_ptr(hidden), _ptr(W), _ptr(rows), _ptr(n_rows), T, d, V,
                                    float(inv_tau), int(K), _ptr(lse), _ptr(ent), _ptr(tv), _ptr(ti),
                                    _ptr(ws), ws.numel(), _ptr(ds), _stream())
    _check(st, "olive_token_topk_fwd")
    return lse, ent, tv, ti


def olive_topk_compare(h_t, W_t, rows, n_rows, s_ids, s_logp, t_ids, t_lse, inv_tau: float = 1.0,
                       dev_status=None, want_t_logp=False):
    """Top-K overlap ratio and top-K truncated reverse KL per masked row.

    Returns (overlap [T], kl_topk [T]), plus the teacher's log-probs at the
    student's top-K ids [T, K] when want_t_logp."""
    _need(h_t, torch.bfloat16, "h_t")
    _need(W_t, torch.bfloat16, "W_t")
    _need(s_ids, torch.int32, "s_ids")
    _need(t_ids, torch.int32, "t_ids")
    _need(s_logp, torch.float32, "s_logp")
    _need(t_lse, torch.float32, "t_lse")
    T, d_t = h_t.shape
    V = W_t.shape[0]
    K = s_ids.shape[1]
    dev = h_t.device
    ov = torch.empty(T, dtype=torch.float32, device=dev)
    kl = torch.empty(T, dtype=torch.float32, device=dev)
    tlp = torch.empty(T, K, dtype=torch.float32, device=dev) if want_t_logp else None
    ds = dev_status if dev_status is not None else new_status(dev)
    st = lib().olive_topk_compare(_ptr(h_t), _ptr(W_t), d_t, _ptr(rows), _ptr(n_rows), T, V,
                                  float(inv_tau), K, _ptr(s_ids), _ptr(s_logp), _ptr(t_ids),
                                  _ptr(t_lse), _ptr(ov), _ptr(kl), _ptr(tlp), _ptr(ds), _stream())
    _check(st, "olive_topk_compare")
    return (ov, kl, tlp) if want_t_logp else (ov, kl)


OPD_STATS_KEYS = ("kl", "s_lse", "t_lse", "s_entropy", "s_topk_logp", "s_topk_ids", "t_logp_s",
                  "overlap", "kl_topk")


def olive_opd_token_stats(h_s, W_s, h_t, W_t, rows, n_rows, K: int = 16, inv_tau: float = 1.0,
                          direction: str = "reverse", want=OPD_STATS_KEYS, ws=None,
                          dev_status=None) -> dict:
    """OPD's per-token KL, lse of both heads, student entropy and top-K lists,
    teacher log-probs at the student's top-K ids, top-K overlap and top-K KL
    from one sweep.  Returns a dict with the requested keys of OPD_STATS_KEYS."""
    for t, n in ((h_s, "h_s"), (W_s, "W_s"), (h_t, "h_t"), (W_t, "W_t")):
        _need(t, torch.bfloat16, n)
    _need(rows, torch.int32, "rows")
    _need(n_rows, torch.int32, "n_rows")
    T, d_s = h_s.shape
    d_t = h_t.shape[1]
    V = W_s.shape[0]
    if W_t.shape[0] != V or h_t.shape[0] != T:
        raise ValueError("student and teacher shapes disagree")
    dev = h_s.device
    shapes = {"s_topk_logp": (T, K), "s_topk_ids": (T, K), "t_logp_s": (T, K)}
    out = {}
    for k in OPD_STATS_KEYS:
        if k in want:
            dt = torch.int32 if k == "s_topk_ids" else torch.float32
            out[k] = torch.empty(shapes.get(k, (T,)), dtype=dt, device=dev)
    if ws is None:
        ws = workspace(olive_workspace_size("opd_stats", T, d_s, V, d_t=d_t), dev)
    ds = dev_status if dev_status is not None else new_status(dev)
    st = lib().olive_opd_token_stats(_ptr(h_s), _ptr(W_s), d_s, _ptr(h_t), _ptr(W_t), d_t,
                                     _ptr(rows), _ptr(n_rows), T, V, float(inv_tau),
                                     DIRECTION[direction], int(K),
                                     *[_ptr(out.get(k)) for k in OPD_STATS_KEYS],
                                     _ptr(ws), ws.numel(), _ptr(ds), _stream())
    _check(st, "olive_opd_token_stats")
    return out


def olive_topk_kl_bwd(h_s, W_s, rows, n_rows, s_lse, s_ids, s_logp, t_logp_s, kl_topk, grad_kl,
                      inv_tau: float = 1.0, grad_dtype=torch.bfloat16, ws=None, dev_status=None,
                      out=None):
    """Gradient of sum_t grad_kl[t] kl_topk[t] with respect to h_s and W_s,
    the student's top-K set held fixed.  Returns (d_h_s [T, d], d_W_s [V, d])."""
    _need(h_s, torch.bfloat16, "h_s")
    _need(W_s, torch.bfloat16, "W_s")
    _need(s_ids, torch.int32, "s_ids")
    for t, n in ((s_lse, "s_lse"), (s_logp, "s_logp"), (t_logp_s, "t_logp_s"), (kl_topk, "kl_topk"),
                 (grad_kl, "grad_kl")):
        _need(t, torch.float32, n)
    T, d = h_s.shape
    V = W_s.shape[0]
    K = s_ids.shape[1]
    dev = h_s.device
    if out is None:
        out = (torch.empty(T, d, dtype=grad_dtype, device=dev),
               torch.empty(V, d, dtype=grad_dtype, device=dev))
    dh, dw = out
    if ws is None:
        ws = workspace(olive_workspace_size("topk_kl_bwd", T, d, V, grad_dtype=grad_dtype), dev)
    ds = dev_status if dev_status is not None else new_status(dev)
    st = lib().olive_topk_kl_bwd(_ptr(h_s), _ptr(W_s), _ptr(rows), _ptr(n_rows), T, d, V,
                                 float(inv_tau), K, _ptr(s_lse), _ptr(s_ids), _ptr(s_logp),
                                 _ptr(t_logp_s), _ptr(kl_topk), _ptr(grad_kl), _ptr(dh), _ptr(dw),
                                 DTYPE[grad_dtype], _ptr(ws), ws.numel(), _ptr(ds), _stream())
    _check(st, "olive_topk_kl_bwd")
    return dh, dw


def olive_topk_kl_fwd_bwd(h_s, W_s, h_t, W_t, rows, n_rows, K, t_lse, grad_kl, t_ids=None,
                          inv_tau: float = 1.0, grad_dtype=torch.bfloat16, ws=None,
                          dev_status=None, out=None):
    """The student's top-K lists, the top-K KL against the teacher and its
    gradient in one sweep of the student's logits.  t_lse (and t_ids, for the
    overlap) come from olive_token_topk_fwd on the teacher.  Returns a dict
    with s_lse, s_ids, s_logp, t_logp_s, kl_topk, overlap (None without
    t_ids), d_h_s and d_W_s."""
    _need(h_s, torch.bfloat16, "h_s")
    _need(W_s, torch.bfloat16, "W_s")
    _need(h_t, torch.bfloat16, "h_t")
    _need(W_t, torch.bfloat16, "W_t")
    _need(t_lse, torch.float32, "t_lse")
    _need(grad_kl, torch.float32, "grad_kl")
    if t_ids is not None:
        _need(t_ids, torch.int32, "t_ids")
    T, ds = h_s.shape
    V = W_s.shape[0]
    dt = h_t.shape[1]
    dev = h_s.device
    if out is None:
        f = lambda *shape: torch.empty(*shape, dtype=torch.float32, device=dev)
        out = dict(s_lse=f(T), s_ids=torch.empty(T, K, dtype=torch.int32, device=dev),
                   s_logp=f(T, K), t_logp_s=f(T, K), kl_topk=f(T),
                   overlap=f(T) if t_ids is not None else None,
                   d_h_s=torch.empty(T, ds, dtype=grad_dtype, device=dev),
                   d_W_s=torch.empty(V, ds, dtype=grad_dtype, device=dev))
    if ws is None:
        ws = workspace(olive_workspace_size("topk_kl_fwd_bwd", T, ds, V, grad_dtype=grad_dtype), dev)
    st_buf = dev_status if dev_status is not None else new_status(dev)
    o = out
    st = lib().olive_topk_kl_fwd_bwd(
        _ptr(h_s), _ptr(W_s), ds, _ptr(h_t), _ptr(W_t), dt, _ptr(rows), _ptr(n_rows), T, V,
        float(inv_tau), K, _ptr(t_lse), _ptr(t_ids) if t_ids is not None else None, _ptr(grad_kl),
        _ptr(o["s_lse"]), _ptr(o["s_ids"]), _ptr(o["s_logp"]), _ptr(o["t_logp_s"]),
        _ptr(o["kl_topk"]), _ptr(o["overlap"]) if o["overlap"] is not None else None,
        _ptr(o["d_h_s"]), _ptr(o["d_W_s"]), DTYPE[grad_dtype], _ptr(ws), ws.numel(),
        _ptr(st_buf), _stream())
    _check(st, "olive_topk_kl_fwd_bwd")
    return out


def olive_token_loss_bwd(hidden, W, targets, rows, n_rows, lse, grad_loss, inv_tau: float = 1.0,
                         reduction: str = "sum", grad_dtype=torch.bfloat16, ws=None,
                         dev_status=None, out=None):
    """d loss/d hidden and d loss/d W. grad_loss is a 1-element fp32 CUDA tensor."""
    _need(hidden, torch.bfloat16, "hidden")
    _need(W, torch.bfloat16, "W")
    _need(lse, torch.float32, "lse")
    _need(grad_loss, torch.float32, "grad_loss")
    T, d = hidden.shape
    V = W.shape[0]
    dev = hidden.device
    if out is None:
        out = (torch.empty(T, d, dtype=grad_dtype, device=dev),
               torch.empty(V, d, dtype=grad_dtype, device=dev))
    dh, dw = out
    need = olive_workspace_size("loss_bwd", T, d, V, grad_dtype=grad_dtype)
    if ws is None:
        ws = workspace(need, dev)
    ds = dev_status if dev_status is not None else new_status(dev)
    st = lib().olive_token_loss_bwd(_ptr(hidden), _ptr(W), _ptr(targets), _ptr(rows), _ptr(n_rows),
                                    T, d, V, float(inv_tau), REDUCE[reduction], _ptr(lse),
                                    _ptr(grad_loss), _ptr(dh), _ptr(dw), DTYPE[grad_dtype],
                                    _ptr(ws), ws.numel(), _ptr(ds), _stream())
    _check(st, "olive_token_loss_bwd")
    return dh, dw


def olive_token_loss_fwd_bwd(hidden, W, targets, rows, n_rows, grad_loss, inv_tau: float = 1.0,
                             reduction: str = "sum", grad_dtype=torch.bfloat16, ws=None,
                             dev_status=None, out=None, slab: bool = False):
    """Forward and backward of one training step in one call (G on chip;
    slab=True: olive_token_loss_fwd_bwd_slab, G through an HBM slab).

    grad_loss is a 1-element fp32 CUDA tensor (the loss gradient, known before
    the call).  Returns (logp [T], lse [T], loss [1], d_hidden [T, d], d_W [V, d])."""
    _need(hidden, torch.bfloat16, "hidden")
    _need(W, torch.bfloat16, "W")
    _need(grad_loss, torch.float32, "grad_loss")
    T, d = hidden.shape
    V = W.shape[0]
    dev = hidden.device
    if out is None:
        out = (torch.empty(T, dtype=torch.float32, device=dev),
               torch.empty(T, dtype=torch.float32, device=dev),
               torch.empty(1, dtype=torch.float32, device=dev),
               torch.empty(T, d, dtype=grad_dtype, device=dev),
               torch.empty(V, d, dtype=grad_dtype, device=dev))
    logp, lse, loss, dh, dw = out
    if ws is None:
        op = "loss_fwd_bwd_slab" if slab else "loss_fwd_bwd"
        ws = workspace(olive_workspace_size(op, T, d, V, grad_dtype=grad_dtype), dev)
    ds = dev_status if dev_status is not None else new_status(dev)
    fn = lib().olive_token_loss_fwd_bwd_slab if slab else lib().olive_token_loss_fwd_bwd
    st = fn(_ptr(hidden), _ptr(W), _ptr(targets), _ptr(rows), _ptr(n_rows), T, d, V,
            float(inv_tau), REDUCE[reduction], _ptr(grad_loss), _ptr(logp), _ptr(lse), _ptr(loss),
            _ptr(dh), _ptr(dw), DTYPE[grad_dtype], _ptr(ws), ws.numel(), _ptr(ds), _stream())
    _check(st, "olive_token_loss_fwd_bwd_slab" if slab else "olive_token_loss_fwd_bwd")
    return logp, lse, loss, dh, dw


def olive_token_divergence(h_s, W_s, h_t, W_t, rows, n_rows, inv_tau: float = 1.0,
                           direction: str = "reverse", grad_kl=None, grad_dtype=torch.bfloat16,
                           ws=None, dev_status=None):
    """Per-token full-vocabulary KL; with grad_kl also d(sum g_t KL_t)/d h_s.

    Returns (kl [T] fp32, d_h_s or None)."""
    for t, n in ((h_s, "h_s"), (W_s, "W_s"), (h_t, "h_t"), (W_t, "W_t")):
        _need(t, torch.bfloat16, n)
    T, d_s = h_s.shape
    d_t = h_t.shape[1]
    V = W_s.shape[0]
    if W_t.shape[0] != V or h_t.shape[0] != T:
        raise ValueError("student and teacher shapes disagree")
    dev = h_s.device
    kl = torch.empty(T, dtype=torch.float32, device=dev)
    dhs = None
    if grad_kl is not None:
        _need(grad_kl, torch.float32, "grad_kl")
        dhs = torch.empty(T, d_s, dtype=grad_dtype, device=dev)
    need = olive_workspace_size("divergence", T, d_s, V, d_t=d_t, grad=grad_kl is not None)
    if ws is None:
        ws = workspace(need, dev)
    ds = dev_status if dev_status is not None else new_status(dev)
    st = lib().olive_token_divergence(_ptr(h_s), _ptr(W_s), d_s, _ptr(h_t), _ptr(W_t), d_t,
                                      _ptr(rows), _ptr(n_rows), T, V, float(inv_tau),
                                      DIRECTION[direction], _ptr(kl), _ptr(grad_kl), _ptr(dhs),
                                      DTYPE[grad_dtype], _ptr(ws), ws.numel(), _ptr(ds), _stream())
    _check(st, "olive_token_divergence")
    return kl, dhs


def olive_token_logprob_fwd_noalloc(hidden, W, targets, rows, n_rows, inv_tau: float = 1.0,
                                    reduction: str = "sum", dev_status=None, out=None):
    """olive_token_logprob_fwd without a workspace: scratch comes from the
    library's fixed device array (see include/olive.h for the size limit and
    the rule that overlapping calls must be serialised)."""
    _need(hidden, torch.bfloat16, "hidden")
    _need(W, torch.bfloat16, "W")
    T, d = hidden.shape
    V = W.shape[0]
    dev = hidden.device
    if out is None:
        out = (torch.empty(T, dtype=torch.float32, device=dev),
               torch.empty(T, dtype=torch.float32, device=dev),
               torch.empty(1, dtype=torch.float32, device=dev))
    logp, lse, loss = out
    ds = dev_status if dev_status is not None else new_status(dev)
    st = lib().olive_token_logprob_fwd_noalloc(_ptr(hidden), _ptr(W), _ptr(targets), _ptr(rows),
                                               _ptr(n_rows), T, d, V, float(inv_tau),
                                               REDUCE[reduction], _ptr(logp), _ptr(lse), _ptr(loss),
                                               _ptr(ds), _stream())
    _check(st, "olive_token_logprob_fwd_noalloc")
    return logp, lse, loss


def olive_scale(x, scale, out=None):
    """out = x * scale (scale: 1-element fp32 CUDA tensor); bf16 or fp32, in
    place when out is x."""
    if x.dtype not in DTYPE:
        raise TypeError("x must be bf16 or fp32")
    _need(x, x.dtype, "x")
    _need(scale, torch.float32, "scale")
    out = torch.empty_like(x) if out is None else out
    st = lib().olive_scale(_ptr(x), _ptr(out), x.numel(), DTYPE[x.dtype], _ptr(scale), _stream())
    _check(st, "olive_scale")
    return out


def olive_packed_positions(cu_seqlens, T_cap: int, out=None):
    """Position of every packed token inside its sequence (int32 [T_cap], 0
    behind the last one) from olive_splice_pack's cu_seqlens."""
    _need(cu_seqlens, torch.int32, "cu_seqlens")
    if out is None:
        out = torch.empty(T_cap, dtype=torch.int32, device=cu_seqlens.device)
    _need(out, torch.int32, "out")
    if out.numel() != T_cap:
        raise ValueError("out holds T_cap positions")
    st = lib().olive_packed_positions(_ptr(cu_seqlens), cu_seqlens.numel() - 1, T_cap, _ptr(out),
                                      _stream())
    _check(st, "olive_packed_positions")
    return out


# Small calls are bound by the host (a launch is 2.5 us on the GB300's, an attribute
# of a tensor 0.07): the calls below look at each tensor once, in one expression, and
# name what is wrong only when something is.
_BF16, _F32, _I32 = torch.bfloat16, torch.float32, torch.int32
_ptr_of, _numel_of, _device_of = torch.Tensor.data_ptr, torch.Tensor.numel, torch.Tensor.get_device
_is_dense, _dtype_of = torch.Tensor.is_contiguous, operator.attrgetter("dtype")


def _need_all(tensors, dtype, names):
    """_need for several tensors of one dtype at once; the current device's index."""
    try:
        for t in tensors:
            if t.dtype is not dtype:
                break
        else:
            cur, *more = set(map(_device_of, tensors))
            if cur >= 0 and not more and cur == _current() and all(map(_is_dense, tensors)):
                return cur
    except (TypeError, AttributeError):
        pass
    for t, n in zip(tensors, names):
        _need(t, dtype, n)
    return _current()


def _need_on(cur, t, dtype, name):
    """_need, the current device's index being known."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.get_device() != cur or not t.is_contiguous():
        _need(t, dtype, name)


def _need_given(cur, ws, dev_status):
    """The checks of a workspace and a status word that the caller brings."""
    if ws is not None:
        _need_on(cur, ws, ws.dtype, "ws")
    if dev_status is not None:
        _need_on(cur, dev_status, _I32, "dev_status")


@functools.lru_cache(maxsize=4096)
def _ws_bytes(op, T, d, V, grad, grad_dtype, d_t=0):
    return int(lib().olive_workspace_size(op, T, d, d_t, V, grad, grad_dtype))


def _bytes(n, dev):
    return torch.empty(n, dtype=torch.uint8, device=dev)


def _refuse_heads(t, T, H, D, dtype, name, cur):
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.get_device() != cur:
        raise TypeError(f"{name} must be a {dtype} tensor on the current CUDA device, {cur}")
    if t.shape != (T, H, D):
        raise ValueError(f"{name} must have the shape [{T}, {H}, {D}]")
    raise TypeError(f"{name}: the {D} values of a head must be contiguous")


def _heads(t, shape, dtype, name, cur):
    """Pointer, token stride and head stride of a view [T, H, D] with contiguous heads."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.shape != shape or t.get_device() != cur:
        _refuse_heads(t, *shape, dtype, name, cur)
    a, b, c = t.stride()
    if c != 1:
        _refuse_heads(t, *shape, dtype, name, cur)
    T, H, _ = shape
    # (the stride of a dimension of one entry means nothing)
    return t.data_ptr(), a if T > 1 else 0, b if H > 1 else 0


def _qk_args(q, k, w_q, w_k, cos, sin, positions, eps, interleaved):
    """Checks what the heads' forward and backward share; (views of q and k, the
    shared C arguments, their shapes, dtype, device and its index)."""
    if (not isinstance(q, torch.Tensor) or not isinstance(k, torch.Tensor) or not q.is_cuda or
            q.dtype not in DTYPE or q.dim() != 3 or k.dim() != 3):
        raise TypeError("q and k must be CUDA bf16 or fp32 tensors [T, heads, D]")
    cur = _need_all((w_q, w_k), q.dtype, ("w_q", "w_k"))
    sq, sk, dtype, dev = q.shape, k.shape, q.dtype, q.device
    T, Hq, D = sq
    if sk[0] != T or sk[2] != D:
        raise ValueError(f"k must have the shape [{T}, heads, {D}]")
    vq, vk = _heads(q, sq, dtype, "q", cur), _heads(k, sk, dtype, "k", cur)
    _need_on(cur, cos, _F32, "cos")
    _need_on(cur, sin, _F32, "sin")
    _need_on(cur, positions, _I32, "positions")
    if w_q.numel() != D or w_k.numel() != D:
        raise ValueError(f"w_q and w_k must hold {D} values")
    table = cos.shape
    if len(table) != 2 or table != sin.shape:
        raise ValueError("cos and sin must have the same shape [P, R/2]")
    if positions.numel() != T:
        raise ValueError(f"positions must hold {T} values")
    P, half = table
    common = (Hq, sk[1], w_q.data_ptr(), w_k.data_ptr(), eps, cos.data_ptr(), sin.data_ptr(),
              positions.data_ptr(), P, T, D, 2 * half, 1 if interleaved else 0)
    return vq, vk, common, sq, sk, dtype, dev, cur


def _qk_out(out, sq, sk, dtype, dev, cur):
    """The outputs and their views: contiguous ones where none are given."""
    if out is None:
        yq = torch.empty(sq, dtype=dtype, device=dev)
        yk = torch.empty(sk, dtype=dtype, device=dev)
        _, Hq, D = sq
        Hk = sk[1]
        return yq, yk, (yq.data_ptr(), Hq * D, D), (yk.data_ptr(), Hk * D, D)
    yq, yk = out
    return yq, yk, _heads(yq, sq, dtype, "q's output", cur), _heads(yk, sk, dtype, "k's output", cur)


def olive_qk_norm_rope_fwd(q, k, w_q, w_k, cos, sin, positions, eps: float = 1e-6,
                           interleaved: bool = False, dev_status=None, out=None):
    """RMS norm of every head of q [T, Hq, D] and k [T, Hk, D] (weights w_q, w_k
    [D]) and rotation by positions [T] with the tables cos, sin (fp32 [P, R/2];
    R <= D).  q and k may be views of one projection.  Returns (q_out, k_out),
    contiguous unless given as `out` (views, or q and k themselves)."""
    vq, vk, common, sq, sk, dtype, dev, cur = _qk_args(q, k, w_q, w_k, cos, sin, positions, eps, interleaved)
    yq, yk, oq, ok = _qk_out(out, sq, sk, dtype, dev, cur)
    _need_given(cur, None, dev_status)
    st = lib().olive_qk_norm_rope_fwd(*vq, *vk, *common, *oq, *ok, DTYPE[dtype], _ptr(dev_status),
                                      _stream_of(cur))
    if st:
        _check(st, "olive_qk_norm_rope_fwd")
    return yq, yk


def olive_qk_norm_rope_bwd(g_q, g_k, q, k, w_q, w_k, cos, sin, positions, eps: float = 1e-6,
                           interleaved: bool = False, ws=None, dev_status=None, out=None):
    """Gradients of olive_qk_norm_rope_fwd for its inputs q, k and the gradients
    g_q, g_k of its outputs.  Returns (d_q, d_k, dw_q, dw_k), the weights' in fp32;
    `out` takes (d_q, d_k), e.g. views of one projection's gradient."""
    vq, vk, common, sq, sk, dtype, dev, cur = _qk_args(q, k, w_q, w_k, cos, sin, positions, eps, interleaved)
    gq, gk = _heads(g_q, sq, dtype, "g_q", cur), _heads(g_k, sk, dtype, "g_k", cur)
    dq, dk, oq, ok = _qk_out(out, sq, sk, dtype, dev, cur)
    _need_given(cur, ws, dev_status)
    D = sq[2]
    dwq, dwk = torch.empty(D, dtype=_F32, device=dev), torch.empty(D, dtype=_F32, device=dev)
    if ws is None:
        ws = _bytes(_ws_bytes(12, 1, D, 1, 0, 0), dev)
    st = lib().olive_qk_norm_rope_bwd(*gq, *gk, *vq, *vk, *common, *oq, *ok, dwq.data_ptr(),
                                      dwk.data_ptr(), DTYPE[dtype], ws.data_ptr(), ws.numel(),
                                      _ptr(dev_status), _stream_of(cur))
    if st:
        _check(st, "olive_qk_norm_rope_bwd")
    return dq, dk, dwq, dwk


def _mlp_args(x, W_gate, W_up, W_down):
    cur = _need_all((x, W_gate, W_up, W_down), _BF16, ("x", "W_gate", "W_up", "W_down"))
    rows, wide = x.shape, W_gate.shape
    if len(rows) != 2:
        raise ValueError("x must have the shape [T, d]")
    T, d = rows
    f = wide[0]
    if wide != (f, d) or W_up.shape != wide or W_down.shape != (d, f):
        raise ValueError("W_gate and W_up must have the shape [f, d], W_down [d, f]")
    return T, d, f, cur


def olive_gated_mlp_fwd(x, W_gate, W_up, W_down, residual=None, act: str = "silu",
                        save: bool = False, ws=None, dev_status=None, out=None):
    """Gated feed-forward block on the rows of x [T, d] (bf16):
    (act(x W_gate^T) * (x W_up^T)) W_down^T (+ residual), act "silu" or
    "gelu_tanh".  Returns (y, saved): saved, with save=True, is what
    olive_gated_mlp_bwd takes (the pre-activations in 16 bits, 4 T f bytes), else
    None."""
    T, d, f, cur = _mlp_args(x, W_gate, W_up, W_down)
    dev = x.device
    if residual is not None:
        _need_on(cur, residual, _BF16, "residual")
        if residual.shape != x.shape:
            raise ValueError("residual must have the shape of x")
    if out is None:
        out = torch.empty((T, d), dtype=_BF16, device=dev)
    else:
        _need_on(cur, out, _BF16, "out")
        if out.shape != x.shape:
            raise ValueError("out must have the shape of x")
    _need_given(cur, ws, dev_status)
    saved = torch.empty((2, T, f), dtype=torch.int16, device=dev) if save else None
    if ws is None:
        ws = _bytes(_ws_bytes(10, T, d, f, 0, 0), dev)
    st = lib().olive_gated_mlp_fwd(x.data_ptr(), W_gate.data_ptr(), W_up.data_ptr(), W_down.data_ptr(),
                                   _ptr(residual), T, d, f, ACT[act], out.data_ptr(), _ptr(saved),
                                   ws.data_ptr(), ws.numel(), _ptr(dev_status), _stream_of(cur))
    if st:
        _check(st, "olive_gated_mlp_fwd")
    return out, saved


def olive_gated_mlp_bwd(dy, x, W_gate, W_up, W_down, saved, act: str = "silu",
                        grad_dtype=torch.bfloat16, need_dx: bool = True, need_dW: bool = True,
                        ws=None, dev_status=None, out=None):
    """Gradients of olive_gated_mlp_fwd (that of its residual is dy).  Returns
    (dx, dW_gate, dW_up, dW_down) of grad_dtype, None for what is not needed."""
    T, d, f, cur = _mlp_args(x, W_gate, W_up, W_down)
    dev = x.device
    _need_on(cur, dy, _BF16, "dy")
    _need_on(cur, saved, torch.int16, "saved")
    if dy.shape != x.shape or saved.shape != (2, T, f):
        raise ValueError("dy must have the shape of x, saved that of the forward")
    if out is None:
        dx = torch.empty((T, d), dtype=grad_dtype, device=dev) if need_dx else None
        dg = du = dd = None
        if need_dW:
            dg = torch.empty((f, d), dtype=grad_dtype, device=dev)
            du = torch.empty((f, d), dtype=grad_dtype, device=dev)
            dd = torch.empty((d, f), dtype=grad_dtype, device=dev)
    else:
        dx, dg, du, dd = out
        for t, shape in ((dx, (T, d)), (dg, (f, d)), (du, (f, d)), (dd, (d, f))):
            if t is not None:
                _need_on(cur, t, grad_dtype, "out")
                if t.shape != shape:
                    raise ValueError("out must have the shapes of x and the weights")
    kind = DTYPE[grad_dtype]
    _need_given(cur, ws, dev_status)
    if ws is None:
        ws = _bytes(_ws_bytes(11, T, d, f, 1, kind), dev)
    st = lib().olive_gated_mlp_bwd(dy.data_ptr(), x.data_ptr(), W_gate.data_ptr(), W_up.data_ptr(),
                                   W_down.data_ptr(), saved.data_ptr(), T, d, f, ACT[act], _ptr(dx),
                                   _ptr(dg), _ptr(du), _ptr(dd), kind, ws.data_ptr(), ws.numel(),
                                   _ptr(dev_status), _stream_of(cur))
    if st:
        _check(st, "olive_gated_mlp_bwd")
    return dx, dg, du, dd


def _grad_list(tensors, cur, what):
    """Pointers, element counts and dtypes of contiguous tensors on device `cur`."""
    try:
        kinds = list(map(DTYPE.__getitem__, map(_dtype_of, tensors)))
        fine = all(map(_is_dense, tensors)) and set(map(_device_of, tensors)) <= {cur}
    except (KeyError, AttributeError, TypeError):
        raise TypeError(f"{what} must be bf16 or fp32 tensors") from None
    if not fine:
        raise TypeError(f"{what} must be contiguous and on the current CUDA device")
    return list(map(_ptr_of, tensors)), list(map(_numel_of, tensors)), kinds


def olive_grad_clip(grads, max_norm: float, out="inplace", norm=None, ws=None):
    """The 2-norm over all elements of `grads` (bf16 or fp32 CUDA tensors,
    contiguous) as a 1-element fp32 tensor, and the gradients scaled by
    min(1, max_norm / (norm + 1e-6)): in place, into the list `out`, or not at
    all (out=None: only the norm).  What is written must not share memory with
    another gradient or output."""
    n = len(grads)
    cur = _current()
    src, num, kinds = _grad_list(grads, cur, "gradients")
    dst = None
    if out is not None:
        if isinstance(out, str):
            if out != "inplace":
                raise ValueError('out must be "inplace", None or a list of as many tensors as grads')
            dst = src
        else:
            if len(out) != n:
                raise ValueError('out must be "inplace", None or a list of as many tensors as grads')
            dst, sizes, types = _grad_list(out, cur, "out")
            if sizes != num or types != kinds:
                raise TypeError("out must be like the gradients")
    if norm is None:
        norm = torch.empty(1, dtype=_F32, device="cuda")
    else:
        _need_on(cur, norm, _F32, "norm")
    _need_given(cur, ws, None)
    if ws is None:
        ws = _bytes(_ws_bytes(13, max(n, 1), 0, 1, 0, 0), "cuda")
    # the four host arrays behind one another
    table = array.array("Q", src)
    table.extend(dst or ())
    table.extend(num)
    at, count = table.buffer_info()
    kind = array.array("i", kinds)
    lists = (at, at + 8 * n if dst is not None else None, at + 8 * (count - n), kind.buffer_info()[0], n)
    L = lib()
    # (blocks of one tensor would write what those of another read or write)
    if L.olive_grad_clip_apart(*lists):
        raise ValueError("a gradient that is scaled must not share memory with another (a tied one is listed once)")
    st = L.olive_grad_clip(*lists, max_norm, norm.data_ptr(), ws.data_ptr(), ws.numel(), _stream_of(cur))
    if st:
        _check(st, "olive_grad_clip")
    return norm


def _embedding_ids(cur, ids, n_ids, dev_status):
    _need_on(cur, ids, _I32, "ids")
    if n_ids is not None:
        _need_on(cur, n_ids, _I32, "n_ids")
        if n_ids.numel() != 1:
            raise ValueError("n_ids must hold one value")
    _need_given(cur, None, dev_status)


def olive_embedding_fwd(W, ids, scale: float = 1.0, n_ids=None, dev_status=None, out=None):
    """scale * W[ids] (W [V, d] bf16 or fp32, ids int32 [T]); rows from n_ids on
    (a device int32, e.g. cu_seqlens[-1:]) are 0."""
    if not isinstance(W, torch.Tensor) or W.dtype not in DTYPE or W.dim() != 2:
        raise TypeError("W must be a bf16 or fp32 tensor [V, d]")
    dtype = W.dtype
    cur = _need_all((W,), dtype, ("W",))
    _embedding_ids(cur, ids, n_ids, dev_status)
    T = ids.numel()
    V, d = W.shape
    if out is None:
        out = torch.empty((T, d), dtype=dtype, device=W.device)
    else:
        _need_on(cur, out, dtype, "out")
        if out.shape != (T, d):
            raise ValueError(f"out must have the shape [{T}, {d}]")
    st = lib().olive_embedding_fwd(W.data_ptr(), ids.data_ptr(), _ptr(n_ids), T, V, d, scale,
                                   out.data_ptr(), DTYPE[dtype], _ptr(dev_status), _stream_of(cur))
    if st:
        _check(st, "olive_embedding_fwd")
    return out


def olive_embedding_bwd(dy, ids, V: int, scale: float = 1.0, n_ids=None, grad_dtype=torch.bfloat16,
                        out=None, accumulate: bool = False, ws=None, dev_status=None):
    """Gradient [V, d] of olive_embedding_fwd's W for the gradient dy [T, d] of its
    output, or with `accumulate` added to `out` (an LM head's gradient that is also
    the embedding's).  Sums have a fixed order."""
    if not isinstance(dy, torch.Tensor) or dy.dtype not in DTYPE or dy.dim() != 2:
        raise TypeError("dy must be a bf16 or fp32 tensor [T, d]")
    cur = _need_all((dy,), dy.dtype, ("dy",))
    _embedding_ids(cur, ids, n_ids, dev_status)
    _need_given(cur, ws, None)
    T, d = dy.shape
    if ids.numel() != T:
        raise ValueError(f"ids must hold {T} values")
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs the gradient that is added to, out")
        out = torch.empty((V, d), dtype=grad_dtype, device=dy.device)
    else:
        grad_dtype = out.dtype
        if grad_dtype not in DTYPE:
            raise TypeError("out must be bf16 or fp32")
        _need_on(cur, out, grad_dtype, "out")
        if out.shape != (V, d):
            raise ValueError(f"out must have the shape [{V}, {d}]")
    if ws is None:
        ws = _bytes(_ws_bytes(15, T, d, V, 0, 0), dy.device)
    st = lib().olive_embedding_bwd(dy.data_ptr(), ids.data_ptr(), _ptr(n_ids), T, V, d, scale,
                                   out.data_ptr(), DTYPE[dy.dtype], DTYPE[grad_dtype],
                                   1 if accumulate else 0, ws.data_ptr(), ws.numel(),
                                   _ptr(dev_status), _stream_of(cur))
    if st:
        _check(st, "olive_embedding_bwd")
    return out


def _norm_args(x, w, name):
    """What the rows' norm's forward and backward share: T, d, dtype and the device's index."""
    if not isinstance(x, torch.Tensor) or x.dtype not in DTYPE or x.dim() != 2:
        raise TypeError(f"{name} must be a bf16 or fp32 tensor [T, d]")
    dtype = x.dtype
    cur = _need_all((x, w), dtype, (name, "w"))
    T, d = x.shape
    if w.shape != (d,):
        raise ValueError(f"w must have the shape [{d}]")
    return T, d, dtype, cur


def _like(cur, t, x, name):
    _need_on(cur, t, x.dtype, name)
    if t.shape != x.shape:
        raise ValueError(f"{name} must have the shape of the rows")
    return t


def olive_row_norm_fwd(x, w, b=None, residual=None, eps: float = 1e-6, kind: str = "layer",
                       save: bool = False, out=None, sum_out=None):
    """Norm of the rows of h = x (+ residual), [T, d] bf16 or fp32: kind "layer"
    (centred; the default here and in olive_row_norm_bwd) or "rms" (row_norm's, the
    autograd form's), weights w and bias b [d].  Returns (y, h, stats): h is x
    itself where there is no residual, stats (save=True) what olive_row_norm_bwd
    takes, else None."""
    T, d, dtype, cur = _norm_args(x, w, "x")
    dev = x.device
    if b is not None:
        _need_on(cur, b, dtype, "b")
        if b.shape != (d,):
            raise ValueError(f"b must have the shape [{d}]")
    y = torch.empty((T, d), dtype=dtype, device=dev) if out is None else _like(cur, out, x, "out")
    h = x
    if residual is not None:
        _like(cur, residual, x, "residual")
        h = torch.empty((T, d), dtype=dtype, device=dev) if sum_out is None else _like(cur, sum_out, x, "sum_out")
    elif sum_out is not None:
        raise ValueError("sum_out is the sum with a residual")
    stats = torch.empty((2, T), dtype=_F32, device=dev) if save else None
    st = lib().olive_row_norm_fwd(x.data_ptr(), _ptr(residual), w.data_ptr(), _ptr(b), T, d, eps,
                                  NORM[kind], y.data_ptr(), h.data_ptr() if residual is not None else None,
                                  _ptr(stats), DTYPE[dtype], _stream_of(cur))
    if st:
        _check(st, "olive_row_norm_fwd")
    return y, h, stats


def olive_row_norm_bwd(dy, h, w, stats, g_h=None, kind: str = "layer", need_db: bool = True, ws=None,
                       out=None):
    """Gradients of olive_row_norm_fwd for the rows h that it normed and the kind it was
    given ("layer" by default, as there): (dx, dw, db), dx that of x and of the residual,
    dw and db fp32 [d] (db None where it is not needed).  g_h, the gradient of h by other
    ways, is added to dx."""
    T, d, dtype, cur = _norm_args(h, w, "h")
    dev = h.device
    _like(cur, dy, h, "dy")
    if g_h is not None:
        _like(cur, g_h, h, "g_h")
    _need_on(cur, stats, _F32, "stats")
    if stats.shape != (2, T):
        raise ValueError("stats must be that of the forward")
    _need_given(cur, ws, None)
    dx = torch.empty((T, d), dtype=dtype, device=dev) if out is None else _like(cur, out, h, "out")
    dw = torch.empty(d, dtype=_F32, device=dev)
    db = torch.empty(d, dtype=_F32, device=dev) if need_db else None
    if ws is None:
        ws = _bytes(_ws_bytes(14, 1, d, 1, 0, 0), dev)
    st = lib().olive_row_norm_bwd(dy.data_ptr(), h.data_ptr(), w.data_ptr(), stats.data_ptr(), _ptr(g_h),
                                  T, d, NORM[kind], dx.data_ptr(), dw.data_ptr(), _ptr(db), DTYPE[dtype],
                                  ws.data_ptr(), ws.numel(), _stream_of(cur))
    if st:
        _check(st, "olive_row_norm_bwd")
    return dx, dw, db


def _att_args(q, k, v, cu_seqlens, scale, causal, prefix_end, cap, slopes):
    """Checks what the attention's forward and backward share; (views of q, k and v, the
    shared C arguments, their shapes, device and its index)."""
    if (not isinstance(q, torch.Tensor) or not isinstance(k, torch.Tensor) or not q.is_cuda or
            q.dtype is not _BF16 or q.dim() != 3 or k.dim() != 3):
        raise TypeError("q and k must be CUDA bf16 tensors [T, heads, D]")
    cur = _current()
    sq, sk = q.shape, k.shape
    T, Hq, D = sq
    Hk = sk[1]
    if sk[0] != T or sk[2] != D:
        raise ValueError(f"k must have the shape [{T}, heads, {D}]")
    vq, vk, vv = _heads(q, sq, _BF16, "q", cur), _heads(k, sk, _BF16, "k", cur), _heads(v, sk, _BF16, "v", cur)
    _need_on(cur, cu_seqlens, _I32, "cu_seqlens")
    S = cu_seqlens.numel() - 1
    if prefix_end is not None:
        _need_on(cur, prefix_end, _I32, "prefix_end")
        if prefix_end.numel() != S:
            raise ValueError(f"prefix_end must hold {S} values")
    if slopes is not None:
        _need_on(cur, slopes, _F32, "slopes")
        if slopes.numel() != Hq:
            raise ValueError(f"slopes must hold {Hq} values")
    common = (Hq, Hk, cu_seqlens.data_ptr(), S, T, D, D ** -0.5 if scale is None else scale,
              1 if causal else 0, _ptr(prefix_end), cap, _ptr(slopes))
    return vq, vk, vv, common, sq, sk, q.device, cur


def _att_out(out, shape, name, dev, cur):
    """An output and its view: a contiguous one where none is given."""
    if out is None:
        out = torch.empty(shape, dtype=_BF16, device=dev)
        return out, (out.data_ptr(), shape[1] * shape[2], shape[2])
    return out, _heads(out, shape, _BF16, name, cur)


def olive_packed_attention_fwd(q, k, v, cu_seqlens, scale=None, causal: bool = True, prefix_end=None,
                               cap: float = 0.0, slopes=None, dev_status=None, out=None):
    """Attention of packed tokens to their own sequence: q [T, Hq, D], k and v
    [T, Hk, D] (bf16; views will do), cu_seqlens int32 [S + 1].  scale is
    1 / sqrt(D) unless given; prefix_end (int32 [S], packed indices) ends what all
    rows of a sequence see; cap > 0 bends the scores by a tanh, slopes (fp32 [Hq])
    lower them with the distance.  Returns (o [T, Hq, D], lse fp32 [Hq, T]); rows
    behind the last sequence get 0 and -inf."""
    vq, vk, vv, common, sq, _, dev, cur = _att_args(q, k, v, cu_seqlens, scale, causal, prefix_end, cap, slopes)
    o, vo = _att_out(out, sq, "out", dev, cur)
    _need_given(cur, None, dev_status)
    lse = torch.empty((sq[1], sq[0]), dtype=_F32, device=dev)
    st = lib().olive_packed_attention_fwd(*vq, *vk, *vv, *common, *vo, lse.data_ptr(), _ptr(dev_status),
                                          _stream_of(cur))
    if st:
        _check(st, "olive_packed_attention_fwd")
    return o, lse


def olive_packed_attention_bwd(d_o, q, k, v, o, lse, cu_seqlens, scale=None, causal: bool = True,
                               prefix_end=None, cap: float = 0.0, slopes=None, ws=None, dev_status=None,
                               out=None):
    """Gradients (dq, dk, dv) of olive_packed_attention_fwd for its outputs o and lse
    and the gradient d_o of o; `out` takes them, e.g. views of one projection's
    gradient."""
    vq, vk, vv, common, sq, sk, dev, cur = _att_args(q, k, v, cu_seqlens, scale, causal, prefix_end, cap, slopes)
    vg, vo = _heads(d_o, sq, _BF16, "d_o", cur), _heads(o, sq, _BF16, "o", cur)
    _need_on(cur, lse, _F32, "lse")
    if lse.shape != (sq[1], sq[0]):
        raise ValueError(f"lse must have the shape [{sq[1]}, {sq[0]}]")
    dq, dk, dv = (None, None, None) if out is None else out
    (dq, oq), (dk, ok), (dv, ov) = (_att_out(t, s, n, dev, cur) for t, s, n in
                                    ((dq, sq, "dq"), (dk, sk, "dk"), (dv, sk, "dv")))
    _need_given(cur, ws, dev_status)
    if ws is None:
        ws = _bytes(_ws_bytes(16, sq[0], sq[2], sq[1], 0, 0, sk[1]), dev)
    st = lib().olive_packed_attention_bwd(*vg, *vq, *vk, *vv, *vo, lse.data_ptr(), *common, *oq, *ok, *ov,
                                          ws.data_ptr(), ws.numel(), _ptr(dev_status), _stream_of(cur))
    if st:
        _check(st, "olive_packed_attention_bwd")
    return dq, dk, dv


class FusedLMHeadCE(torch.autograd.Function):
    """Eq. (osd-ce) loss over the masked rows as an autograd op (gradients in
    the dtype of hidden; first derivatives only).  A status word given is the
    forward's and the backward's.

    With a gradient needed, the forward runs olive_token_loss_fwd_bwd with a
    unit loss gradient (each logit tile computed once) and the backward scales
    the stored gradients by the incoming one (olive_scale); otherwise, or with
    single_pass=False, it runs olive_token_logprob_fwd and the backward
    recomputes the logits (olive_token_loss_bwd)."""

    @staticmethod
    def forward(ctx, hidden, W, targets, rows, n_rows, inv_tau=1.0, reduction="sum",
                single_pass=True, dev_status=None):
        ctx.inv_tau, ctx.reduction, ctx.dev_status = inv_tau, reduction, dev_status
        ctx.single = bool(single_pass and (hidden.requires_grad or W.requires_grad))
        if ctx.single:
            one = torch.ones(1, dtype=torch.float32, device=hidden.device)
            _, _, loss, dh, dw = olive_token_loss_fwd_bwd(hidden, W, targets, rows, n_rows, one,
                                                          inv_tau, reduction, grad_dtype=hidden.dtype,
                                                          dev_status=dev_status)
            ctx.save_for_backward(dh, dw)
        else:
            _, lse, loss = olive_token_logprob_fwd(hidden, W, targets, rows, n_rows, inv_tau,
                                                   reduction, dev_status=dev_status)
            ctx.save_for_backward(hidden, W, targets, rows, n_rows, lse)
        return loss[0]

    @staticmethod
    @once_differentiable
    def backward(ctx, g):
        gl = g.reshape(1).to(torch.float32).contiguous()
        if ctx.single:
            dh1, dw1 = ctx.saved_tensors
            return (olive_scale(dh1, gl), olive_scale(dw1, gl), *[None] * 7)
        hidden, W, targets, rows, n_rows, lse = ctx.saved_tensors
        dh, dw = olive_token_loss_bwd(hidden, W, targets, rows, n_rows, lse, gl, ctx.inv_tau,
                                      ctx.reduction, grad_dtype=hidden.dtype,
                                      dev_status=ctx.dev_status)
        return (dh, dw, *[None] * 7)


def fused_lmhead_ce(hidden, W, targets, rows, n_rows, inv_tau=1.0, reduction="sum",
                    single_pass=True, dev_status=None):
    return FusedLMHeadCE.apply(hidden, W, targets, rows, n_rows, inv_tau, reduction, single_pass,
                               dev_status)


def _heads_gradient(g):
    """A gradient [T, heads, D] as the backward can read it.  Autograd hands over whatever
    view the next operation left (columns of a wider tensor, say), which need not start
    on 16 bytes nor have strides of whole 16 bytes: then a copy."""
    token, head, last = g.stride()
    fits = (last == 1 and g.data_ptr() % 16 == 0 and (g.shape[0] < 2 or token % 8 == 0) and
            (g.shape[1] < 2 or head % 8 == 0))
    return g if fits else g.clone(memory_format=torch.contiguous_format)


class QKNormRope(torch.autograd.Function):
    """Heads' norm and rotation as an autograd op (weights' gradients in the
    weights' type).  It has first derivatives only.  A status word given is the
    forward's and the backward's."""

    @staticmethod
    def forward(ctx, q, k, w_q, w_k, cos, sin, positions, eps=1e-6, interleaved=False,
                dev_status=None):
        ctx.save_for_backward(q, k, w_q, w_k, cos, sin, positions)
        ctx.eps, ctx.interleaved, ctx.dev_status = eps, interleaved, dev_status
        return olive_qk_norm_rope_fwd(q, k, w_q, w_k, cos, sin, positions, eps, interleaved,
                                      dev_status)

    @staticmethod
    @once_differentiable
    def backward(ctx, g_q, g_k):
        q, k, w_q, w_k, cos, sin, positions = ctx.saved_tensors
        dq, dk, dwq, dwk = olive_qk_norm_rope_bwd(_heads_gradient(g_q), _heads_gradient(g_k), q, k, w_q, w_k, cos, sin,
                                                  positions, ctx.eps, ctx.interleaved,
                                                  dev_status=ctx.dev_status)
        return (dq, dk, dwq.to(w_q.dtype), dwk.to(w_k.dtype), *[None] * 6)


def qk_norm_rope(q, k, w_q, w_k, cos, sin, positions, eps=1e-6, interleaved=False,
                 dev_status=None):
    return QKNormRope.apply(q, k, w_q, w_k, cos, sin, positions, eps, interleaved, dev_status)


class GatedMLP(torch.autograd.Function):
    """Gated feed-forward block as an autograd op (gradients in bf16; first
    derivatives only, but for the residual's).  The pre-activations are saved only
    where a gradient is needed.  A status word given is the forward's and the
    backward's."""

    @staticmethod
    def forward(ctx, x, W_gate, W_up, W_down, residual=None, act="silu", dev_status=None):
        needs = ctx.needs_input_grad
        ctx.act, ctx.need_dx, ctx.need_dW = act, needs[0], any(needs[1:4])
        ctx.dev_status = dev_status
        y, saved = olive_gated_mlp_fwd(x, W_gate, W_up, W_down, residual, act,
                                       save=ctx.need_dx or ctx.need_dW, dev_status=dev_status)
        if saved is not None:
            ctx.save_for_backward(x, W_gate, W_up, W_down, saved)
        return y

    @staticmethod
    def backward(ctx, dy):
        res = dy if ctx.needs_input_grad[4] else None
        if not (ctx.need_dx or ctx.need_dW):
            return None, None, None, None, res, None, None
        return (*GatedMLP._gradients(ctx, dy), res, None, None)

    @staticmethod
    @once_differentiable
    def _gradients(ctx, dy):
        if not dy.is_contiguous() or dy.data_ptr() % 16:
            dy = dy.clone(memory_format=torch.contiguous_format)
        x, W_gate, W_up, W_down, saved = ctx.saved_tensors
        return olive_gated_mlp_bwd(dy, x, W_gate, W_up, W_down, saved, ctx.act, need_dx=ctx.need_dx,
                                   need_dW=ctx.need_dW, dev_status=ctx.dev_status)


def _values_only(*tensors):
    """Whether a call is one for its values: autograd is off, and no tensor has a tangent
    (forward mode works where autograd is off; the Functions have none and say so)."""
    if torch.is_grad_enabled():
        return False
    # (asked of the tensors only where there is a level for tangents: 0.5 us each)
    return getattr(forward_ad, "_current_level", 0) < 0 or all(
        t is None or forward_ad.unpack_dual(t).tangent is None for t in tensors)


def gated_mlp(x, W_gate, W_up, W_down, residual=None, act="silu", dev_status=None):
    # (asked here: inside a Function autograd is off anyway, and a Parameter "needs" its
    # gradient under no_grad too; what is saved is 4 T f bytes)
    if _values_only(x, W_gate, W_up, W_down, residual):
        return olive_gated_mlp_fwd(x, W_gate, W_up, W_down, residual, act, dev_status=dev_status)[0]
    return GatedMLP.apply(x, W_gate, W_up, W_down, residual, act, dev_status)


def _whole(g):
    """A gradient as the calls read it: dense and on a 16-byte boundary, else a copy."""
    return g if g.is_contiguous() and g.data_ptr() % 16 == 0 else g.clone(memory_format=torch.contiguous_format)


class Embedding(torch.autograd.Function):
    """Embedding rows as an autograd op (the gradient in W's type; first derivatives
    only).  A status word given is the forward's and the backward's."""

    @staticmethod
    def forward(ctx, W, ids, scale=1.0, n_ids=None, dev_status=None):
        ctx.save_for_backward(ids, *(() if n_ids is None else (n_ids,)))
        ctx.V, ctx.scale, ctx.dtype, ctx.dev_status = W.shape[0], scale, W.dtype, dev_status
        return olive_embedding_fwd(W, ids, scale, n_ids, dev_status)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        ids, *n_ids = ctx.saved_tensors
        dW = olive_embedding_bwd(_whole(dy), ids, ctx.V, ctx.scale, n_ids[0] if n_ids else None, ctx.dtype,
                                 dev_status=ctx.dev_status)
        return dW, None, None, None, None


def embedding(W, ids, scale=1.0, n_ids=None, dev_status=None):
    return Embedding.apply(W, ids, scale, n_ids, dev_status)


class RowNorm(torch.autograd.Function):
    """Rows' norm as an autograd op (weights' gradients in the weights' type; first
    derivatives only): y, or with a residual (y, h) with h the sum.  Its kind is "rms"
    unless given, that of the direct calls "layer"."""

    @staticmethod
    def forward(ctx, x, w, b=None, residual=None, eps=1e-6, kind="rms"):
        y, h, stats = olive_row_norm_fwd(x, w, b, residual, eps, kind, save=True)
        ctx.save_for_backward(h, w, stats)
        ctx.kind, ctx.b_dtype, ctx.added = kind, None if b is None else b.dtype, residual is not None
        ctx.set_materialize_grads(False)
        return (y, h) if ctx.added else y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, g_h=None):
        if dy is None and g_h is None:
            return None, None, None, None, None, None
        h, w, stats = ctx.saved_tensors
        if dy is None:  # only the sum was used
            return g_h, None, None, g_h, None, None
        dx, dw, db = olive_row_norm_bwd(_whole(dy), h, w, stats, None if g_h is None else _whole(g_h), ctx.kind,
                                        ctx.b_dtype is not None)
        return (dx, dw.to(w.dtype), None if db is None else db.to(ctx.b_dtype), dx if ctx.added else None,
                None, None)


def row_norm(x, w, b=None, residual=None, eps=1e-6, kind="rms"):
    """RowNorm's form as a function: note its kind where none is given, "rms"."""
    # (nothing is kept for a backward where autograd is off)
    if _values_only(x, w, b, residual):
        y, h, _ = olive_row_norm_fwd(x, w, b, residual, eps, kind)
        return y if residual is None else (y, h)
    return RowNorm.apply(x, w, b, residual, eps, kind)


class PackedAttention(torch.autograd.Function):
    """Attention inside packed sequences as an autograd op (first derivatives only; none
    for the distance bias).  A status word given is the forward's and the backward's."""

    @staticmethod
    def forward(ctx, q, k, v, cu_seqlens, scale=None, causal=True, prefix_end=None, cap=0.0, slopes=None,
                dev_status=None):
        o, lse = olive_packed_attention_fwd(q, k, v, cu_seqlens, scale, causal, prefix_end, cap, slopes, dev_status)
        more = [t for t in (prefix_end, slopes) if t is not None]
        ctx.save_for_backward(q, k, v, o, lse, cu_seqlens, *more)
        ctx.given = (prefix_end is not None, slopes is not None)
        ctx.form, ctx.dev_status = (scale, causal, cap), dev_status
        return o

    @staticmethod
    @once_differentiable
    def backward(ctx, d_o):
        q, k, v, o, lse, cu, *more = ctx.saved_tensors
        scale, causal, cap = ctx.form
        prefix_end, slopes = (more.pop(0) if there else None for there in ctx.given)
        if d_o.shape[0] > 1 and d_o.stride(0) == 0:  # (one row for all tokens)
            d_o = d_o.clone(memory_format=torch.contiguous_format)
        dq, dk, dv = olive_packed_attention_bwd(_heads_gradient(d_o), q, k, v, o, lse, cu, scale, causal, prefix_end,
                                                cap, slopes, dev_status=ctx.dev_status)
        return (dq, dk, dv, *[None] * 7)


def packed_attention(q, k, v, cu_seqlens, scale=None, causal=True, prefix_end=None, cap=0.0, slopes=None,
                     dev_status=None):
    return PackedAttention.apply(q, k, v, cu_seqlens, scale, causal, prefix_end, cap, slopes, dev_status)


def _in_memory_order(g):
    """The same values with the dimensions in the order of their strides: contiguous,
    unless there are gaps.  (The values' order does not matter to clipping.)"""
    if g.is_contiguous():
        return g
    return g.permute(sorted(range(g.dim()), key=g.stride, reverse=True))


def clip_grad_norm_(parameters, max_norm):
    """olive_grad_clip in place on the gradients that the parameters (or the one
    parameter) hold."""
    if isinstance(parameters, torch.Tensor):
        parameters = (parameters,)
    # (a gradient that several entries hold is one: a tied parameter's counts and is scaled once)
    grads = {id(g): g for g in (p.grad for p in parameters) if g is not None}
    grads = [_in_memory_order(g) for g in grads.values()]
    flat = [g.contiguous() for g in grads]  # (itself, but for one with gaps: a copy, which goes back)
    norm = olive_grad_clip(flat, max_norm)
    for g, f in zip(grads, flat):
        if f is not g:
            g.copy_(f)
    return norm
