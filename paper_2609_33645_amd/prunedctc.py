"""Python binding of libprunedctc.so (C ABI in include/prunedctc.h).

Argument marshalling only: every step of the computation runs in the library's HIP
kernels.  PyTorch supplies device memory (outputs and workspace come from its caching
allocator) and the current stream.  If the library has not been built, every call
raises ``PrunedCTCError``; there is no fallback path.
"""
from __future__ import annotations

import ctypes
import functools
import math
import os
import threading
from array import array
from collections.abc import Iterable
from typing import Dict, List, Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libprunedctc.so")

PCTC_F32, PCTC_BF16 = 0, 1
STATUS = {0: "ok", -1: "invalid argument", -2: "bad label", -3: "bad length", -4: "workspace too small",
          -5: "HIP error", -6: "target too long"}
UTT_OK, UTT_NOT_ALIGNABLE, UTT_NONFINITE = 0, 1, 2
TOKEN_COUNTED, TOKEN_LEFT_OUT, TOKEN_NONFINITE = 0, 1, 2
MAX_TARGET = 1023
MAX_BEAMS = 32
MAX_CANDIDATES = 64


class PrunedCTCError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(msg)
        self.code = code


_lib = None


def lib() -> ctypes.CDLL:
    """Load the HIP library once.  torch is imported first so that the library binds to
    the HIP runtime torch already loaded."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise PrunedCTCError(-5, f"HIP library not built: {LIB_PATH} is missing "
                                 f"(run: python -m paper_2609_33645_amd.build)")
    L = ctypes.CDLL(LIB_PATH)
    c_i32, c_f, c_p, c_sz = ctypes.c_int32, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t
    i32p = ctypes.POINTER(ctypes.c_int32)
    L.pctc_workspace_size.argtypes = [c_i32, c_i32, i32p, i32p, c_i32, c_i32, c_f, c_i32]
    L.pctc_workspace_size.restype = c_sz
    L.pctc_workspace_size_ex.argtypes = [c_i32, c_i32, i32p, i32p, c_i32, c_i32, c_f, c_i32, c_i32]
    L.pctc_workspace_size_ex.restype = c_sz
    L.pctc_normaliser_chunk_columns.argtypes = [c_i32, c_i32, i32p, i32p, c_i32, c_i32, c_f, c_i32, c_i32]
    L.pctc_normaliser_chunk_columns.restype = c_i32
    L.pruned_ctc_fwd_bwd.argtypes = [c_i32, c_p, c_i32, c_p, c_i32, c_p, i32p, i32p, c_i32, c_i32, c_f, c_i32,
                                     c_p, c_p, c_p, c_p, c_p, c_p, c_sz, c_p]
    L.pruned_ctc_fwd_bwd.restype = c_i32
    L.pruned_ctc_fwd_bwd_ex.argtypes = [c_i32, c_p, c_i32, c_p, c_p, c_i32, c_p, i32p, i32p, c_i32, c_i32, c_f, c_i32,
                                        c_p, c_p, c_p, c_p, c_p, c_p, c_p, c_p, c_sz, c_p]
    L.pruned_ctc_fwd_bwd_ex.restype = c_i32
    L.pctc_lattice_leads.argtypes = [c_i32, c_i32, i32p, i32p, c_i32, c_i32, c_f]
    L.pctc_lattice_leads.restype = c_i32
    L.pctc_noalloc_scratch_bytes.argtypes = []
    L.pctc_noalloc_scratch_bytes.restype = c_sz
    L.pruned_ctc_fwd_bwd_noalloc.argtypes = [c_i32, c_p, c_i32, c_p, c_p, c_i32, c_p, i32p, i32p, c_i32, c_i32, c_f,
                                             c_i32, c_p, c_p, c_p, c_p, c_p, c_p, c_p, c_p]
    L.pruned_ctc_fwd_bwd_noalloc.restype = c_i32
    L.pctc_status_string.argtypes = [c_i32]
    L.pctc_status_string.restype = ctypes.c_char_p
    L.pctc_last_error.argtypes = []
    L.pctc_last_error.restype = ctypes.c_char_p
    L.pctc_union_scratch_bytes.argtypes = [c_i32]
    L.pctc_union_scratch_bytes.restype = c_sz
    L.pctc_union_remap.argtypes = [c_p, c_i32, c_i32, c_i32, c_p, c_p, c_p, c_p, c_p, c_p, c_p]
    L.pctc_union_remap.restype = c_i32
    L.pctc_lse_scratch_bytes.argtypes = [c_i32, c_i32]
    L.pctc_lse_scratch_bytes.restype = c_sz
    L.pctc_lse_select.argtypes = [c_i32, c_p, c_i32, c_i32, c_p, c_i32, c_p, c_p, c_i32, c_p, c_p, c_i32, c_p, c_p]
    L.pctc_lse_select.restype = c_i32
    L.pctc_dp_scratch_bytes.argtypes = [c_i32, i32p, i32p, c_f]
    L.pctc_dp_scratch_bytes.restype = c_sz
    L.pctc_ctc_dp.argtypes = [c_p, c_i32, c_i32, c_p, i32p, i32p, c_i32, c_f, c_p, c_p, c_p, c_p, c_p, c_p, c_p]
    L.pctc_ctc_dp.restype = c_i32
    L.pctc_greedy_workspace_size.argtypes = [c_i32, c_i32, c_i32]
    L.pctc_greedy_workspace_size.restype = c_sz
    L.pctc_greedy_workspace_size_ex.argtypes = [c_i32, c_i32, c_i32, c_i32, c_i32]
    L.pctc_greedy_workspace_size_ex.restype = c_sz
    L.pctc_greedy_decode.argtypes = [c_i32, c_p, c_i32, c_p, c_p, c_i32, i32p, c_i32, c_i32, c_p, c_p, c_p, c_p, c_sz,
                                     c_p]
    L.pctc_greedy_decode.restype = c_i32
    L.pctc_discarded_mass_scratch_bytes.argtypes = [c_i32, i32p, i32p]
    L.pctc_discarded_mass_scratch_bytes.restype = c_sz
    L.pctc_discarded_mass.argtypes = [c_p, c_i32, c_i32, c_p, i32p, i32p, c_i32, ctypes.POINTER(ctypes.c_float), c_i32,
                                      c_p, c_p, c_p]
    L.pctc_discarded_mass.restype = c_i32
    L.pctc_bwd_scratch_bytes.argtypes = [c_i32, c_i32, c_i32, c_i32, c_i32, c_i32]
    L.pctc_bwd_scratch_bytes.restype = c_sz
    L.pctc_bwd_chunk.argtypes = [c_i32, c_i32, c_i32, c_i32, c_i32]
    L.pctc_bwd_chunk.restype = c_i32
    L.pctc_head_bwd.argtypes = [c_i32, c_p, c_i32, c_i32, c_p, c_i32, c_p, c_p, c_i32, c_p, c_p, c_i32, c_p, c_p,
                                c_p, c_p]
    L.pctc_head_bwd.restype = c_i32
    L.pctc_grouped_workspace_size.argtypes = [c_i32, c_i32, c_i32, c_i32, c_i32, c_i32]
    L.pctc_grouped_workspace_size.restype = c_sz
    L.pctc_grouped_logprobs.argtypes = [c_i32, c_p, c_i32, c_i32, c_p, c_p, c_i32, c_p, c_i32, c_p, c_p, c_p, c_sz, c_p]
    L.pctc_grouped_logprobs.restype = c_i32
    L.pctc_grouped_backward.argtypes = [c_i32, c_p, c_i32, c_i32, c_p, c_p, c_i32, c_p, c_i32, c_p, c_p, c_p, c_i32,
                                        c_p, c_p, c_p, c_p, c_sz, c_p]
    L.pctc_grouped_backward.restype = c_i32
    L.pctc_frame_candidates_workspace_size.argtypes = [c_i32, c_i32, c_i32, c_i32, c_i32]
    L.pctc_frame_candidates_workspace_size.restype = c_sz
    L.pctc_frame_candidates.argtypes = [c_i32, c_p, c_i32, c_i32, c_p, c_p, c_i32, c_i32, c_i32, c_p, c_p, c_p, c_p, c_sz,
                                        c_p]
    L.pctc_frame_candidates.restype = c_i32
    L.pctc_frame_candidates_pass.argtypes = [c_i32, c_i32, c_i32, c_i32, c_i32, c_i32, i32p]
    L.pctc_frame_candidates_pass.restype = c_sz
    L.pctc_beam_state_bytes.argtypes = [c_i32, c_i32, c_i32]
    L.pctc_beam_state_bytes.restype = c_sz
    L.pctc_beam_reset.argtypes = [c_i32, c_i32, c_i32, c_p, c_sz, c_p]
    L.pctc_beam_reset.restype = c_i32
    L.pctc_beam_advance.argtypes = [c_p, c_p, c_p, c_i32, c_p, c_i32, c_i32, c_i32, c_f, c_p, c_p, c_sz, c_p, c_p]
    L.pctc_beam_advance.restype = c_i32
    L.pctc_beam_result.argtypes = [c_i32, c_i32, c_i32, c_p, c_sz, c_i32, c_p, c_p, c_p, c_p]
    L.pctc_beam_result.restype = c_i32
    L.pctc_beam_reorder.argtypes = [c_i32, c_p, c_p, c_p, c_p, c_i32, c_i32, c_p]
    L.pctc_beam_reorder.restype = c_i32
    L.pctc_beam_decode_workspace_size.argtypes = [c_i32, c_p, c_i32, c_i32, c_i32, c_i32, c_i32]
    L.pctc_beam_decode_workspace_size.restype = c_sz
    L.pctc_beam_decode.argtypes = [c_i32, c_p, c_i32, c_p, c_p, c_i32, c_p, c_i32, c_i32, c_i32, c_i32, c_f, c_i32, c_p,
                                   c_p, c_p, c_p, c_p, c_p, c_p, c_sz, c_p]
    L.pctc_beam_decode.restype = c_i32
    L.pctc_clip_workspace_size.argtypes = [c_i32]
    L.pctc_clip_workspace_size.restype = c_sz
    L.pctc_clip_grad_norm.argtypes = [c_i32, c_p, c_p, c_p, c_p, c_f, c_p, c_p, c_p, c_sz, c_p]
    L.pctc_clip_grad_norm.restype = c_i32
    c_i64, c_u64, c_d = ctypes.c_int64, ctypes.c_uint64, ctypes.c_double
    L.pctc_dropout.argtypes = [c_i32, c_p, c_p, c_p, c_i64, c_d, c_u64, c_u64, c_p, c_p]
    L.pctc_dropout.restype = c_i32
    L.pctc_embedding.argtypes = [c_i32, c_p, c_i32, c_i32, c_p, c_i32, c_i64, c_f, c_p, c_p]
    L.pctc_embedding.restype = c_i32
    L.pctc_embedding_backward_workspace_size.argtypes = [c_i64, c_i32]
    L.pctc_embedding_backward_workspace_size.restype = c_sz
    L.pctc_embedding_backward.argtypes = [c_i32, c_p, c_p, c_i32, c_i64, c_i32, c_i32, c_f, c_i32, c_p, c_i32, c_p, c_sz,
                                          c_p]
    L.pctc_embedding_backward.restype = c_i32
    L.pctc_gated_ffn_workspace_size.argtypes = [c_i32] * 6
    L.pctc_gated_ffn_workspace_size.restype = c_sz
    L.pctc_gated_ffn.argtypes = [c_i32, c_p, c_i32, c_i32, c_p, c_p, c_i32, c_p, c_i32, c_i32, c_p, c_p, c_p, c_p, c_sz,
                                 c_p]
    L.pctc_gated_ffn.restype = c_i32
    L.pctc_gated_ffn_backward.argtypes = [c_i32, c_p, c_p, c_i32, c_i32, c_p, c_p, c_p, c_p, c_i32, c_p, c_i32, c_i32,
                                          c_p, c_p, c_p, c_p, c_p, c_sz, c_p]
    L.pctc_gated_ffn_backward.restype = c_i32
    L.pctc_policy_workspace_size.argtypes = [c_i32] * 7
    L.pctc_policy_workspace_size.restype = c_sz
    L.pctc_policy_loss.argtypes = [c_i32, c_p, c_i32, c_i32, c_p, c_p, c_i32, c_p, c_p, c_p, c_p, c_p, c_f, c_f, c_f,
                                   c_i32, c_p, c_p, c_p, c_p, c_p, c_p, c_p, c_p, c_sz, c_p]
    L.pctc_policy_loss.restype = c_i32
    L.pctc_prof_enable.argtypes = [c_i32]
    L.pctc_prof_select.argtypes = [ctypes.c_char_p]
    L.pctc_prof_reset.argtypes = []
    L.pctc_prof_count.argtypes = []
    L.pctc_prof_count.restype = c_i32
    L.pctc_prof_get.argtypes = [c_i32, ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(ctypes.c_double),
                                ctypes.POINTER(ctypes.c_int64)]
    L.pctc_prof_get.restype = c_i32
    _lib = L
    return L


def _check(code: int, what: str) -> None:
    if code != 0:
        L = lib()
        detail = L.pctc_last_error().decode() if code == -5 else ""
        raise PrunedCTCError(code, f"{what}: {L.pctc_status_string(code).decode()} {detail}".strip())


def _host_i32(x) -> np.ndarray:
    if isinstance(x, torch.Tensor):
        x = x.detach().cpu().numpy()
    return np.ascontiguousarray(np.asarray(x, dtype=np.int32))


def _i32p(a: np.ndarray):
    return a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream) -> ctypes.c_void_p:
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return PCTC_BF16
    if t.dtype == torch.float32:
        return PCTC_F32
    raise PrunedCTCError(-1, f"unsupported dtype {t.dtype}")


def _workspace(nbytes: int, device) -> torch.Tensor:
    ws = torch.empty(max(int(nbytes), 256) + 256, dtype=torch.uint8, device=device)
    off = (-ws.data_ptr()) % 256
    return ws[off:off + max(int(nbytes), 256)]


def _bias_vector(bias: torch.Tensor, V: int, dev) -> torch.Tensor:
    if bias.numel() != V:
        raise PrunedCTCError(-1, f"bias must hold V = {V} values, got {bias.numel()}")
    return bias.reshape(V).to(device=dev, dtype=torch.float32).contiguous()


WS_NO_DW = 1  # workspace for calls without dW (frozen head)


def workspace_size(dtype: int, input_lengths, target_lengths, D: int, V: int, beam: float, chunk: int = 0,
                   want_dW: bool = True) -> int:
    T = _host_i32(input_lengths)
    U = _host_i32(target_lengths)
    return int(lib().pctc_workspace_size_ex(dtype, T.size, _i32p(T), _i32p(U), D, V, float(beam), chunk,
                                            0 if want_dW else WS_NO_DW))


def normaliser_chunk_columns(dtype: int, input_lengths, target_lengths, D: int, V: int, beam: float, chunk: int = 0,
                             want_dW: bool = True) -> int:
    """Vocabulary columns of the first backward chunk that the normaliser of a fused call writes
    itself (0: every chunk is recomputed); see pctc_normaliser_chunk_columns."""
    T = _host_i32(input_lengths)
    U = _host_i32(target_lengths)
    return int(lib().pctc_normaliser_chunk_columns(dtype, T.size, _i32p(T), _i32p(U), D, V, float(beam), chunk,
                                                   0 if want_dW else WS_NO_DW))


def lattice_leads(dtype: int, input_lengths, target_lengths, D: int, V: int, beam: float) -> bool:
    """Whether a fused call of this shape runs its lattice ungated beside the dense part of the
    backward (see pctc_lattice_leads)."""
    T = _host_i32(input_lengths)
    U = _host_i32(target_lengths)
    return bool(lib().pctc_lattice_leads(dtype, T.size, _i32p(T), _i32p(U), D, V, float(beam)))


def bwd_chunk(dtype: int, M: int, D: int, V: int, chunk: int = 0) -> int:
    """Vocabulary columns per backward step used for this problem (0 chunk = the default)."""
    return int(lib().pctc_bwd_chunk(int(dtype), int(M), int(D), int(V), int(chunk)))


def _grad_buffer(t: Optional[torch.Tensor], shape, dev) -> torch.Tensor:
    if t is None:
        return torch.empty(shape, dtype=torch.float32, device=dev)
    if t.dtype != torch.float32 or tuple(t.shape) != tuple(shape) or not t.is_contiguous() or t.device != dev:
        raise PrunedCTCError(-1, f"gradient buffer must be contiguous float32 {tuple(shape)} on {dev}")
    return t


def pruned_ctc_fwd_bwd(H: torch.Tensor, W: torch.Tensor, targets: torch.Tensor, input_lengths: Sequence[int],
                       target_lengths: Sequence[int], blank: int = 0, beam: float = math.inf, chunk: int = 0,
                       want_dH: bool = True, want_dW: bool = True, workspace: Optional[torch.Tensor] = None,
                       stream=None, dH_out: Optional[torch.Tensor] = None,
                       dW_out: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                       utt_weight: Optional[torch.Tensor] = None, want_db: bool = False) -> Dict[str, torch.Tensor]:
    """Loss and head gradients of Pruned CTC.  H [M, D] and W [V, D] are device tensors of
    the same dtype (bfloat16 or float32); targets is a device int32 tensor; the length
    arrays are host sequences.  Returns loss (float64 [1]), loss_per_utt, status, dH, dW
    and, with want_db, db.  dH_out / dW_out: optional preallocated float32 [M, D] / [V, D]
    gradient buffers.  bias: optional float32 [V] head bias (logits H W^T + b; a blank
    offset eta is added to bias[blank], and its gradient is db[blank]).  utt_weight:
    optional float32 [N] loss weights (loss = sum_n w_n L_n; loss_per_utt stays
    unweighted)."""
    L = lib()
    dt = _dtype_code(H)
    if W.dtype != H.dtype:
        raise PrunedCTCError(-1, "H and W must have the same dtype")
    if not (H.is_cuda and W.is_cuda and targets.is_cuda):
        raise PrunedCTCError(-1, "H, W and targets must be device tensors")
    H = H.contiguous()
    W = W.contiguous()
    targets = targets.to(torch.int32).contiguous()
    T = _host_i32(input_lengths)
    U = _host_i32(target_lengths)
    N = int(T.size)
    M, D = int(H.shape[0]), int(H.shape[1])
    V = int(W.shape[0])
    if W.shape[1] != D:
        raise PrunedCTCError(-1, "H and W widths differ")
    if int(T.sum()) != M:
        raise PrunedCTCError(-1, "sum of input lengths differs from the rows of H")
    if int(U.sum()) != int(targets.numel()):
        raise PrunedCTCError(-1, "sum of target lengths differs from the number of targets")
    dev = H.device
    nbytes = int(L.pctc_workspace_size_ex(dt, N, _i32p(T), _i32p(U), D, V, float(beam), chunk,
                                          0 if want_dW else WS_NO_DW))
    if nbytes == 0:
        code = -6 if (U > MAX_TARGET).any() else (-3 if ((T < 1).any() or (U < 0).any()) else -1)
        _check(code, "pruned_ctc_fwd_bwd")
    ws = workspace if workspace is not None else _workspace(nbytes, dev)
    # the library writes all three on success: one uninitialised allocation, split in views
    n1 = max(N, 1)
    small = torch.empty(8 + 8 * n1 + 4 * n1, dtype=torch.uint8, device=dev)
    loss = small[:8].view(torch.float64)
    loss_n = small[8:8 + 8 * n1].view(torch.float64)
    status = small[8 + 8 * n1:].view(torch.int32)
    dH = _grad_buffer(dH_out, (M, D), dev) if want_dH else None
    dW = _grad_buffer(dW_out, (V, D), dev) if want_dW else None
    db = torch.empty(V, dtype=torch.float32, device=dev) if want_db else None
    if bias is not None:
        bias = _bias_vector(bias, V, dev)
    if utt_weight is not None:
        utt_weight = utt_weight.to(device=dev, dtype=torch.float32).contiguous()
        if utt_weight.numel() != N:
            raise PrunedCTCError(-1, "utt_weight must have N entries")
    if bias is None and utt_weight is None and db is None:
        code = L.pruned_ctc_fwd_bwd(dt, _ptr(H), D, _ptr(W), V, _ptr(targets), _i32p(T), _i32p(U), N, int(blank),
                                    float(beam), int(chunk), _ptr(loss), _ptr(loss_n), _ptr(status), _ptr(dH),
                                    _ptr(dW), ctypes.c_void_p(ws.data_ptr()), ctypes.c_size_t(ws.numel()),
                                    _stream(stream))
    else:
        code = L.pruned_ctc_fwd_bwd_ex(dt, _ptr(H), D, _ptr(W), _ptr(bias), V, _ptr(targets), _i32p(T), _i32p(U), N,
                                       int(blank), float(beam), int(chunk), _ptr(utt_weight), _ptr(loss), _ptr(loss_n),
                                       _ptr(status), _ptr(dH), _ptr(dW), _ptr(db), ctypes.c_void_p(ws.data_ptr()),
                                       ctypes.c_size_t(ws.numel()), _stream(stream))
    _check(code, "pruned_ctc_fwd_bwd")
    return {"loss": loss, "loss_per_utt": loss_n[:N], "status": status[:N], "dH": dH, "dW": dW, "db": db,
            "workspace_bytes": nbytes}


def noalloc_scratch_bytes() -> int:
    """Size of the allocation-free entry point's per-device scratch array."""
    return int(lib().pctc_noalloc_scratch_bytes())


def pruned_ctc_fwd_bwd_noalloc(H: torch.Tensor, W: torch.Tensor, targets: torch.Tensor,
                               input_lengths: Sequence[int], target_lengths: Sequence[int], out: Dict[str, torch.Tensor],
                               blank: int = 0, beam: float = math.inf, chunk: int = 0,
                               bias: Optional[torch.Tensor] = None, utt_weight: Optional[torch.Tensor] = None,
                               stream=None) -> Dict[str, torch.Tensor]:
    """The fused call through pruned_ctc_fwd_bwd_noalloc: the library uses its own static
    scratch, and every output is a caller buffer passed in `out` (allocated beforehand):
    loss (float64 [1]), loss_per_utt (float64 [N]) and status (int32 [N]) or absent, and
    dH (float32 [M, D]), dW (float32 [V, D]), db (float32 [V]) or absent.  H, W, targets,
    bias and utt_weight must already be contiguous device tensors of the right dtypes (no
    conversion or copy is made here).  Returns `out`."""
    L = lib()
    dt = _dtype_code(H)
    T = _host_i32(input_lengths)
    U = _host_i32(target_lengths)
    N = int(T.size)
    for name, t in (("H", H), ("W", W), ("targets", targets), ("bias", bias), ("utt_weight", utt_weight)):
        if t is not None and not (t.is_cuda and t.is_contiguous()):
            raise PrunedCTCError(-1, f"{name} must be a contiguous device tensor")
    if targets.dtype != torch.int32 or W.dtype != H.dtype:
        raise PrunedCTCError(-1, "targets must be int32 and W of H's dtype")
    if bias is not None and bias.dtype != torch.float32 or utt_weight is not None and utt_weight.dtype != torch.float32:
        raise PrunedCTCError(-1, "bias and utt_weight must be float32")
    code = L.pruned_ctc_fwd_bwd_noalloc(dt, _ptr(H), int(H.shape[1]), _ptr(W), _ptr(bias), int(W.shape[0]),
                                        _ptr(targets), _i32p(T), _i32p(U), N, int(blank), float(beam), int(chunk),
                                        _ptr(utt_weight), _ptr(out["loss"]), _ptr(out.get("loss_per_utt")),
                                        _ptr(out.get("status")), _ptr(out.get("dH")), _ptr(out.get("dW")),
                                        _ptr(out.get("db")), _stream(stream))
    _check(code, "pruned_ctc_fwd_bwd_noalloc")
    return out


# ---- stage entry points ------------------------------------------------------------------

def union_remap(targets: torch.Tensor, blank: int, V: int, stream=None) -> Dict[str, torch.Tensor]:
    L = lib()
    targets = targets.to(torch.int32).contiguous()
    dev = targets.device
    Y = int(targets.numel())
    remap = torch.empty(V, dtype=torch.int32, device=dev)
    u_ids = torch.empty(1 + Y, dtype=torch.int32, device=dev)
    y_rel = torch.empty(max(Y, 1), dtype=torch.int32, device=dev)
    K = torch.zeros(1, dtype=torch.int32, device=dev)
    err = torch.zeros(1, dtype=torch.int32, device=dev)
    scratch = _workspace(int(L.pctc_union_scratch_bytes(int(V))), dev)
    code = L.pctc_union_remap(_ptr(targets), Y, int(blank), int(V), _ptr(remap), _ptr(u_ids), _ptr(y_rel), _ptr(K),
                              _ptr(err), ctypes.c_void_p(scratch.data_ptr()), _stream(stream))
    _check(code, "pctc_union_remap")
    k = int(K.item())
    return {"remap": remap, "u_ids": u_ids[:k], "y_rel": y_rel[:Y], "K": k}


def lse_select(H: torch.Tensor, W: torch.Tensor, u_ids: Optional[torch.Tensor] = None,
               stream=None) -> Dict[str, torch.Tensor]:
    """lambda [M] (float64) and, given the union u_ids, S [M, K] (float32)."""
    L = lib()
    dt = _dtype_code(H)
    H = H.contiguous()
    W = W.contiguous()
    M, D = int(H.shape[0]), int(H.shape[1])
    V = int(W.shape[0])
    dev = H.device
    lam = torch.empty(max(M, 1), dtype=torch.float64, device=dev)
    scratch = _workspace(int(L.pctc_lse_scratch_bytes(M, D)), dev)
    S = Kdev = None
    K = 1
    ldS = 1
    if u_ids is not None:
        u_ids = u_ids.to(torch.int32).contiguous()
        K = int(u_ids.numel())
        ldS = ((K + 3) // 4) * 4
        S = torch.zeros((max(M, 1), ldS), dtype=torch.float32, device=dev)
        Kdev = torch.tensor([K], dtype=torch.int32, device=dev)
    code = L.pctc_lse_select(dt, _ptr(H), M, D, _ptr(W), V, _ptr(u_ids), _ptr(Kdev), K, _ptr(lam), _ptr(S), ldS,
                             ctypes.c_void_p(scratch.data_ptr()), _stream(stream))
    _check(code, "pctc_lse_select")
    out = {"lam": lam[:M]}
    if S is not None:
        out["S"] = S[:M, :K]
    return out


def ctc_dp(S: torch.Tensor, y_rel: torch.Tensor, input_lengths, target_lengths, beam: float = math.inf,
           want_mask: bool = False, stream=None) -> Dict[str, torch.Tensor]:
    """Alignment stage on given selected-class scores S [M, K] (column 0 = blank)."""
    L = lib()
    T = _host_i32(input_lengths)
    U = _host_i32(target_lengths)
    N = int(T.size)
    M, K = int(S.shape[0]), int(S.shape[1])
    dev = S.device
    ldS = ((K + 3) // 4) * 4
    Sp = torch.zeros((max(M, 1), ldS), dtype=torch.float32, device=dev)
    Sp[:M, :K] = S.to(torch.float32)
    y_rel = y_rel.to(torch.int32).contiguous()
    G = torch.empty((max(M, 1), ldS), dtype=torch.float32, device=dev)
    g = torch.empty(max(M, 1), dtype=torch.float32, device=dev)
    loss_n = torch.zeros(max(N, 1), dtype=torch.float64, device=dev)
    status = torch.zeros(max(N, 1), dtype=torch.int32, device=dev)
    lattice = int(np.sum(T.astype(np.int64) * (2 * U.astype(np.int64) + 1)))
    mask = torch.zeros(max(lattice, 1), dtype=torch.uint8, device=dev) if want_mask else None
    nbytes = int(L.pctc_dp_scratch_bytes(N, _i32p(T), _i32p(U), float(beam)))
    scratch = _workspace(nbytes, dev)
    code = L.pctc_ctc_dp(_ptr(Sp), ldS, K, _ptr(y_rel), _i32p(T), _i32p(U), N, float(beam), _ptr(loss_n),
                         _ptr(status), _ptr(G), _ptr(g), _ptr(mask), ctypes.c_void_p(scratch.data_ptr()),
                         _stream(stream))
    _check(code, "pctc_ctc_dp")
    out = {"loss_per_utt": loss_n[:N], "status": status[:N], "G": G[:M, :K], "g": g[:M]}
    if mask is not None:
        out["mask"] = mask[:lattice]
    return out


def greedy_decode(H: torch.Tensor, W: torch.Tensor, input_lengths, blank: int = 0,
                  bias: Optional[torch.Tensor] = None, stream=None, to_host: bool = True) -> Dict[str, object]:
    """Framewise full-vocabulary argmax ids [M] and the collapsed token sequence of each
    utterance (a list of lists, only when to_host), plus the device buffers (tokens of
    utterance n at the offset of its first frame)."""
    L = lib()
    dt = _dtype_code(H)
    H = H.contiguous()
    W = W.contiguous()
    T = _host_i32(input_lengths)
    N = int(T.size)
    M, D = int(H.shape[0]), int(H.shape[1])
    V = int(W.shape[0])
    if int(T.sum()) != M:
        raise PrunedCTCError(-1, "sum of input lengths differs from the rows of H")
    dev = H.device
    if bias is not None:
        bias = _bias_vector(bias, V, dev)
    ids = torch.empty(max(M, 1), dtype=torch.int32, device=dev)
    tokens = torch.empty(max(M, 1), dtype=torch.int32, device=dev)
    lengths = torch.empty(max(N, 1), dtype=torch.int32, device=dev)
    ws = _workspace(int(L.pctc_greedy_workspace_size_ex(dt, N, M, D, V)), dev)
    code = L.pctc_greedy_decode(dt, _ptr(H), D, _ptr(W), _ptr(bias), V, _i32p(T), N, int(blank), _ptr(ids),
                                _ptr(tokens), _ptr(lengths), ctypes.c_void_p(ws.data_ptr()), ctypes.c_size_t(ws.numel()),
                                _stream(stream))
    _check(code, "pctc_greedy_decode")
    if not to_host:
        return {"ids": ids[:M], "tokens_dev": tokens[:M], "token_lengths": lengths[:N]}
    off = np.concatenate([[0], np.cumsum(T)]).astype(np.int64)
    tk = tokens.cpu().numpy()
    ln = lengths.cpu().numpy()[:N]
    seqs = [tk[off[n]:off[n] + ln[n]].tolist() for n in range(N)]
    return {"ids": ids[:M], "tokens": seqs, "token_lengths": lengths[:N]}


def discarded_mass(S: torch.Tensor, y_rel: torch.Tensor, input_lengths, target_lengths, beams: Sequence[float],
                   stream=None) -> torch.Tensor:
    """Discarded posterior mass delta [len(beams), N] (float64) of every utterance at every
    beam, on given selected-class scores S [M, K] (column 0 = blank)."""
    L = lib()
    T = _host_i32(input_lengths)
    U = _host_i32(target_lengths)
    N = int(T.size)
    M, K = int(S.shape[0]), int(S.shape[1])
    dev = S.device
    if S.dtype == torch.float32 and S.is_contiguous() and K % 4 == 0 and M > 0:
        ldS, Sp = K, S                     # already in the library's layout
    else:
        ldS = ((K + 3) // 4) * 4
        Sp = torch.zeros((max(M, 1), ldS), dtype=torch.float32, device=dev)
        Sp[:M, :K] = S.to(torch.float32)
    y_rel = y_rel.to(torch.int32).contiguous()
    b = np.ascontiguousarray(np.asarray(beams, np.float32))
    delta = torch.empty((max(len(b), 1), max(N, 1)), dtype=torch.float64, device=dev)
    nbytes = int(L.pctc_discarded_mass_scratch_bytes(N, _i32p(T), _i32p(U)))
    scratch = _workspace(nbytes, dev)
    code = L.pctc_discarded_mass(_ptr(Sp), ldS, K, _ptr(y_rel), _i32p(T), _i32p(U), N,
                                 b.ctypes.data_as(ctypes.POINTER(ctypes.c_float)), int(b.size), _ptr(delta),
                                 ctypes.c_void_p(scratch.data_ptr()), _stream(stream))
    _check(code, "pctc_discarded_mass")
    return delta[:len(b), :N]


def head_bwd(H: torch.Tensor, W: torch.Tensor, lam: torch.Tensor, G: torch.Tensor, g: torch.Tensor,
             remap: torch.Tensor, chunk: int = 0, want_dH: bool = True, want_dW: bool = True,
             stream=None) -> Dict[str, torch.Tensor]:
    L = lib()
    dt = _dtype_code(H)
    H = H.contiguous()
    W = W.contiguous()
    M, D = int(H.shape[0]), int(H.shape[1])
    V = int(W.shape[0])
    dev = H.device
    G = G.to(torch.float32).contiguous()
    ldG = int(G.shape[1])
    dH = torch.empty((M, D), dtype=torch.float32, device=dev) if want_dH else None
    dW = torch.empty((V, D), dtype=torch.float32, device=dev) if want_dW else None
    scratch = _workspace(int(L.pctc_bwd_scratch_bytes(dt, M, D, V, ldG, int(chunk))), dev)
    code = L.pctc_head_bwd(dt, _ptr(H), M, D, _ptr(W), V, _ptr(lam.to(torch.float64).contiguous()), _ptr(G), ldG,
                           _ptr(g.to(torch.float32).contiguous()), _ptr(remap.to(torch.int32).contiguous()),
                           int(chunk), _ptr(dH), _ptr(dW), ctypes.c_void_p(scratch.data_ptr()), _stream(stream))
    _check(code, "pctc_head_bwd")
    return {"dH": dH, "dW": dW}


# ---- grouped logits for a stock CTC -------------------------------------------------------

def grouped_logprobs(H: torch.Tensor, W: torch.Tensor, u_ids: torch.Tensor, bias: Optional[torch.Tensor] = None,
                     stream=None) -> Dict[str, torch.Tensor]:
    """log softmax of the grouped logits [M, K + 1] (float32: the K selected classes, then
    the merged "other" class) and the full normaliser lam [M] (float64)."""
    L = lib()
    dt = _dtype_code(H)
    H = H.contiguous()
    W = W.contiguous()
    M, D = int(H.shape[0]), int(H.shape[1])
    V = int(W.shape[0])
    dev = H.device
    u_ids = u_ids.to(device=dev, dtype=torch.int32).contiguous()
    K = int(u_ids.numel())
    if bias is not None:
        bias = _bias_vector(bias, V, dev)
    logp = torch.empty((M, K + 1), dtype=torch.float32, device=dev)
    lam = torch.empty(max(M, 1), dtype=torch.float64, device=dev)
    nbytes = int(L.pctc_grouped_workspace_size(dt, M, D, V, K, 0))
    if nbytes == 0:
        raise PrunedCTCError(-1, "pctc_grouped_workspace_size: invalid arguments")
    ws = _workspace(nbytes, dev)
    code = L.pctc_grouped_logprobs(dt, _ptr(H), M, D, _ptr(W), _ptr(bias), V, _ptr(u_ids), K, _ptr(logp), _ptr(lam),
                                   ctypes.c_void_p(ws.data_ptr()), ctypes.c_size_t(ws.numel()), _stream(stream))
    _check(code, "pctc_grouped_logprobs")
    return {"logp": logp, "lam": lam[:M]}


def grouped_backward(H: torch.Tensor, W: torch.Tensor, u_ids: torch.Tensor, logp: torch.Tensor, lam: torch.Tensor,
                     dlogp: torch.Tensor, bias: Optional[torch.Tensor] = None, chunk: int = 0,
                     want_dH: bool = True, want_dW: bool = True, want_db: bool = False,
                     stream=None) -> Dict[str, Optional[torch.Tensor]]:
    """dH, dW (and db) from the gradient of a loss w.r.t. the exported grouped log-probabilities."""
    L = lib()
    dt = _dtype_code(H)
    H = H.contiguous()
    W = W.contiguous()
    M, D = int(H.shape[0]), int(H.shape[1])
    V = int(W.shape[0])
    dev = H.device
    u_ids = u_ids.to(device=dev, dtype=torch.int32).contiguous()
    K = int(u_ids.numel())
    if tuple(logp.shape) != (M, K + 1) or tuple(dlogp.shape) != (M, K + 1):
        raise PrunedCTCError(-1, f"logp and dlogp must be [{M}, {K + 1}]")
    if bias is not None:
        bias = _bias_vector(bias, V, dev)
    logp = logp.to(torch.float32).contiguous()
    dlogp = dlogp.to(torch.float32).contiguous()
    lam = lam.to(torch.float64).contiguous()
    dH = torch.empty((M, D), dtype=torch.float32, device=dev) if want_dH else None
    dW = torch.empty((V, D), dtype=torch.float32, device=dev) if want_dW else None
    db = torch.empty(V, dtype=torch.float32, device=dev) if want_db else None
    nbytes = int(L.pctc_grouped_workspace_size(dt, M, D, V, K, int(chunk)))
    if nbytes == 0:
        raise PrunedCTCError(-1, "pctc_grouped_workspace_size: invalid arguments")
    ws = _workspace(nbytes, dev)
    code = L.pctc_grouped_backward(dt, _ptr(H), M, D, _ptr(W), _ptr(bias), V, _ptr(u_ids), K, _ptr(logp), _ptr(lam),
                                   _ptr(dlogp), int(chunk), _ptr(dH), _ptr(dW), _ptr(db),
                                   ctypes.c_void_p(ws.data_ptr()), ctypes.c_size_t(ws.numel()), _stream(stream))
    _check(code, "pctc_grouped_backward")
    return {"dH": dH, "dW": dW, "db": db}


class GroupedHead(torch.autograd.Function):
    """Autograd wrapper: grouped log-probabilities [M, K + 1] of the head H W^T (+ b), for a
    stock CTC loss over K + 1 classes.  The backward runs the library's recomputed backward;
    gradients are returned in the dtypes of H, W and b."""

    @staticmethod
    def forward(ctx, H, W, bias, u_ids):
        out = grouped_logprobs(H.detach(), W.detach(), u_ids, None if bias is None else bias.detach())
        ctx.save_for_backward(H, W, bias, u_ids, out["logp"], out["lam"])
        return out["logp"]

    @staticmethod
    def backward(ctx, dlogp):
        H, W, bias, u_ids, logp, lam = ctx.saved_tensors
        need = ctx.needs_input_grad
        r = grouped_backward(H.detach(), W.detach(), u_ids, logp, lam, dlogp,
                             bias=None if bias is None else bias.detach(), want_dH=need[0], want_dW=need[1],
                             want_db=bias is not None and need[2])
        dH = r["dH"].to(H.dtype) if r["dH"] is not None else None
        dW = r["dW"].to(W.dtype) if r["dW"] is not None else None
        db = r["db"].to(bias.dtype) if r["db"] is not None else None
        return dH, dW, db, None


def grouped_head(H: torch.Tensor, W: torch.Tensor, u_ids: torch.Tensor, bias: Optional[torch.Tensor] = None):
    return GroupedHead.apply(H, W, bias, u_ids)


# ---- readout with beams ------------------------------------------------------------------

_given: List[int] = []  # the threads whose running call was given a stream
_moved: Dict[int, int] = {}  # by thread: the device that was current before its running call made another so
_current_device = torch._C._cuda_getDevice  # (without the checks of torch.cuda.current_device)


def _sequence(x):
    """A tuple in the place of an iterable that could only be gone through once or is no plain sequence."""
    plain = isinstance(x, (torch.Tensor, np.ndarray, list, tuple, str, array)) or not isinstance(x, Iterable)
    return x if plain else tuple(x)


def _asynchronous(fn):
    """For calls that return before the device is done: with stream=..., the whole call, its
    allocations among it, is made on that stream, so that memory it lets go of is not handed out
    to another stream while the kernels still use it; nor is that of the caller's tensors.  What
    another stream writes into them the caller waits for.  Kernels go to the device of the tensors,
    whichever is current (see _raw_stream); `stream` must be one of it."""
    @functools.wraps(fn)
    def call(*args, stream=None, **kw):
        if stream is None:
            try:
                return fn(*args, **kw)
            finally:
                if _moved and threading.get_ident() in _moved:
                    torch.cuda.set_device(_moved.pop(threading.get_ident()))
        args, kw = [_sequence(x) for x in args], {k: _sequence(x) for k, x in kw.items()}
        _given.append(threading.get_ident())
        try:
            with torch.cuda.stream(stream):
                result = fn(*args, **kw)
        finally:
            _given.remove(threading.get_ident())
        for arg in (*args, *kw.values()):
            for t in arg if isinstance(arg, (list, tuple)) else (getattr(arg, "_state", arg),):  # (a search's)
                if isinstance(t, torch.Tensor) and t.is_cuda:
                    t.record_stream(stream)
        return result
    return call


def _raw_stream(dev: torch.device) -> int:
    """The handle of dev's current stream (without the stream object that current_stream makes, 2 us),
    for an _asynchronous call's launch.  A default stream's is the same on every device, and kernels go to
    the current device's: dev becomes the current one until the call is over."""
    index = dev.index
    if _current_device() != index:
        if threading.get_ident() in _given:
            raise PrunedCTCError(-1, f"stream must be one of {dev}, where the tensors are")
        _moved[threading.get_ident()] = torch.cuda.current_device()
        torch.cuda.set_device(index)
    return torch._C._cuda_getCurrentRawStream(index)


def _scratch(nbytes: int, dev: torch.device) -> torch.Tensor:
    """_workspace without its slice where the allocation is aligned already, as torch's are."""
    t = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    return t if t.data_ptr() % 256 == 0 else _workspace(nbytes, dev)


_I32 = np.dtype(np.int32)


def _counts(x):
    """Numbers of frames as an array of int32: whole numbers that it holds, nothing cut off."""
    if isinstance(x, torch.Tensor):
        x = x.detach().cpu().numpy()
    if isinstance(x, np.ndarray):
        x = x.tolist()
    try:
        return array("i", x)
    except TypeError:
        raise PrunedCTCError(-1, "numbers of frames must be whole numbers, one for each utterance") from None
    except OverflowError:
        raise PrunedCTCError(-3, "more frames than an utterance can have") from None


def _as(t: torch.Tensor, dtype: torch.dtype) -> torch.Tensor:
    return t if t.dtype is dtype and t.is_contiguous() else t.to(dtype).contiguous()


def _head_args(H: torch.Tensor, W: torch.Tensor, bias: Optional[torch.Tensor]):
    """Checked and contiguous H, W and bias of a readout, and the library's type code."""
    dt = _dtype_code(H)
    if W.dtype != H.dtype:
        raise PrunedCTCError(-1, "H and W must have the same dtype")
    if not (H.is_cuda and W.device == H.device):
        raise PrunedCTCError(-1, "H and W must be tensors of one device")
    if H.dim() != 2 or W.dim() != 2 or H.shape[1] != W.shape[1]:
        raise PrunedCTCError(-1, "H must be [M, D] and W [V, D]")
    if bias is not None:
        bias = _bias_vector(bias, int(W.shape[0]), H.device)
    return H.contiguous(), W.contiguous(), bias, dt


@_asynchronous
def frame_candidates(H: torch.Tensor, W: torch.Tensor, candidates: int, blank: int = 0,
                     bias: Optional[torch.Tensor] = None, *, stream=None) -> Dict[str, torch.Tensor]:
    """The most probable classes of every frame other than blank, by falling log probability over
    the full vocabulary: ids [M, C] (int32; -1 past the classes of non-zero probability), logp
    [M, C] and blank_logp [M] (float32)."""
    L = lib()
    H, W, bias, dt = _head_args(H, W, bias)
    M, D = H.shape
    V, C, dev = int(W.shape[0]), int(candidates), H.device
    nbytes = int(L.pctc_frame_candidates_workspace_size(dt, M, D, V, C))
    if nbytes == 0:
        _check(-1, "pctc_frame_candidates")
    ids = torch.empty((M, C), dtype=torch.int32, device=dev)
    logp = torch.empty((M, C), dtype=torch.float32, device=dev)
    blank_logp = torch.empty(M, dtype=torch.float32, device=dev)
    ws = _scratch(nbytes, dev)
    code = L.pctc_frame_candidates(dt, H.data_ptr(), M, D, W.data_ptr(), None if bias is None else bias.data_ptr(), V,
                                   int(blank), C, ids.data_ptr(), logp.data_ptr(), blank_logp.data_ptr(), ws.data_ptr(),
                                   ws.numel(), _raw_stream(dev))
    if code:
        _check(code, "pctc_frame_candidates")
    return {"ids": ids, "logp": logp, "blank_logp": blank_logp}


class BeamSearch:
    """CTC prefix beam search of N utterances (or live streams) with up to beam_size prefixes
    each, on candidate classes as frame_candidates gives them; the state stays on the device.

    max_frames bounds the frames an utterance may have in all (memory: 12 bytes a frame and
    beam).  token_bonus is added to a prefix's score per label (negative: a penalty).  Calls are
    asynchronous on the current stream (or `stream`), and one search's calls belong on one stream.

    In a captured graph an advance stays bound to the position of its capture (frames_done counts
    there, not at replays): capture one for each, and give result its max_tokens."""

    @_asynchronous
    def __init__(self, N: int, beam_size: int, max_frames: int, token_bonus: float = 0.0, device=None, *, stream=None):
        self.N, self.beam_size, self.max_frames = int(N), int(beam_size), int(max_frames)
        self.token_bonus = float(token_bonus)
        self.device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        if self.device.type != "cuda":
            raise PrunedCTCError(-1, "a search runs on a GPU")
        nbytes = int(lib().pctc_beam_state_bytes(self.N, self.beam_size, self.max_frames))
        if nbytes == 0:
            _check(-1, "pctc_beam_state_bytes")
        self._state = _workspace(nbytes, self.device)
        self.device = self._state.device
        self._mem = self._state.data_ptr(), self._state.numel()
        self._done = np.zeros(max(self.N, 1), np.int32)
        self._frames = np.zeros(max(self.N, 1), np.int32)
        self._host = self._frames.ctypes.data, self._done.ctypes.data
        self._ones = np.ones_like(self._frames)
        self._beams = torch.empty((self.N, self.beam_size), dtype=torch.int32, device=self.device)  # (a shape)
        self.reset()

    @property
    def frames_done(self) -> np.ndarray:
        """Frames that each utterance has had since the reset."""
        return self._done[:self.N].copy()

    @_asynchronous
    def reset(self, *, stream=None) -> None:
        """Starts every utterance anew with the empty prefix."""
        code = lib().pctc_beam_reset(self.N, self.beam_size, self.max_frames, *self._mem, _raw_stream(self.device))
        if code:
            _check(code, "pctc_beam_reset")
        self._done[:] = 0

    @_asynchronous
    def advance(self, ids: torch.Tensor, logp: torch.Tensor, blank_logp: torch.Tensor, frames: Sequence[int],
                *, stream=None) -> torch.Tensor:
        """frames[n] more frames of utterance n (0: none), packed utterance after utterance: ids and
        logp [sum frames, C], blank_logp [sum frames].  A row's classes are distinct and not blank, and
        their scores fall (a row in another order loses prefixes: sort it again after adding scores of
        your own); places with an id below 0 or a score of -inf or NaN, anywhere in a row, are left out.
        Returns parents [N, beam_size] (int32): the beam before the call that each beam descends from,
        -1 where there is no prefix (for beam_reorder)."""
        # (a live stream calls this every frame: an array of int32 is taken without a look at its values, a dot
        # product takes half of a sum, empty_like of empty)
        if type(frames) is not np.ndarray or frames.dtype is not _I32:
            frames = _counts(frames)
        if len(frames) != self.N:
            raise PrunedCTCError(-1, f"frames must have {self.N} entries")
        fr = self._frames
        fr[:self.N] = frames
        M, shape, dev = int(fr.dot(self._ones)), logp.shape, self.device
        if len(shape) != 2 or shape[0] != M or ids.shape != shape or blank_logp.shape != (M,):
            raise PrunedCTCError(-1, f"ids and logp must be [{M}, C] and blank_logp [{M}]")
        if ids.device != dev or logp.device != dev or blank_logp.device != dev:
            raise PrunedCTCError(-1, f"candidates must be on {dev}")
        ids, logp, blank_logp = _as(ids, torch.int32), _as(logp, torch.float32), _as(blank_logp, torch.float32)
        parents = torch.empty_like(self._beams)
        code = lib().pctc_beam_advance(ids.data_ptr(), logp.data_ptr(), blank_logp.data_ptr(), shape[1],
                                       self._host[0], self.N, self.beam_size, self.max_frames, self.token_bonus,
                                       self._host[1], *self._mem, parents.data_ptr(), _raw_stream(dev))
        if code:
            _check(code, "pctc_beam_advance")
        return parents

    @_asynchronous
    def result(self, max_tokens: Optional[int] = None, *, stream=None) -> Dict[str, torch.Tensor]:
        """The prefixes so far, best first: tokens [N, beam_size, max_tokens] (int32, -1 past the
        end; by default as many as the utterance with most frames so far could have),
        token_lengths [N, beam_size] (int32, -1: no prefix) and scores [N, beam_size] (float32)."""
        if max_tokens is None:
            max_tokens = int(self._done.max())
        tokens = torch.empty((self.N, self.beam_size, int(max_tokens)), dtype=torch.int32, device=self.device)
        lengths = torch.empty((self.N, self.beam_size), dtype=torch.int32, device=self.device)
        scores = torch.empty((self.N, self.beam_size), dtype=torch.float32, device=self.device)
        code = lib().pctc_beam_result(self.N, self.beam_size, self.max_frames, *self._mem, int(max_tokens),
                                      tokens.data_ptr(), lengths.data_ptr(), scores.data_ptr(), _raw_stream(self.device))
        _check(code, "pctc_beam_result")
        return {"tokens": tokens, "token_lengths": lengths, "scores": scores}


def _pointers(tensors) -> array:
    return array("Q", map(torch.Tensor.data_ptr, tensors))


def _at(a: Optional[array]) -> Optional[int]:
    """Address of a host array's values (the caller keeps the array until the call is over)."""
    return None if a is None else a.buffer_info()[0]


@_asynchronous
def beam_reorder(states: Sequence[torch.Tensor], parents: torch.Tensor, out: Optional[Sequence[torch.Tensor]] = None,
                 *, stream=None):
    """Per-beam state tensors [N, K, ...] of any type in the order of the surviving beams: state[n, k]
    becomes state[n, parents[n, k]] (a parent outside [0, K) leaves it).  In place, or into the
    tensors `out`; returns those written.  Tensors must be contiguous, and what is written must not
    overlap another tensor of the call (in place: no state twice in the list)."""
    dev = parents.device
    if parents.dim() != 2 or parents.dtype is not torch.int32 or not parents.is_cuda:
        raise PrunedCTCError(-1, "parents must be a device int32 [N, K]")
    N, K = parents.shape
    parents = parents.contiguous()
    dest = states if out is None else out
    if len(dest) != len(states):
        raise PrunedCTCError(-1, "out must have a tensor for each state")
    sizes = []
    for t, o in zip(states, dest):
        shape = t.shape
        if len(shape) < 2 or shape[0] != N or shape[1] != K:
            raise PrunedCTCError(-1, f"a state must be [{N}, {K}, ...]")
        if t.device != dev or not t.is_contiguous():
            raise PrunedCTCError(-1, f"states must be contiguous tensors on {dev}")
        if o is not t and (o.shape != shape or o.dtype is not t.dtype or o.device != dev or not o.is_contiguous()):
            raise PrunedCTCError(-1, f"out must be contiguous tensors of the states' shapes and types on {dev}")
        sizes.append(t.nbytes // (N * K) if N * K else 0)
    src, dst, nbytes = _pointers(states), None if out is None else _pointers(dest), array("q", sizes)
    code = lib().pctc_beam_reorder(len(sizes), _at(src), _at(dst), _at(nbytes), parents.data_ptr(), N, K,
                                   _raw_stream(dev))
    if code:
        _check(code, "pctc_beam_reorder")
    return list(dest)


@_asynchronous
def beam_decode(H: torch.Tensor, W: torch.Tensor, input_lengths, beam_size: int = 8, candidates: int = 16,
                blank: int = 0, bias: Optional[torch.Tensor] = None, token_bonus: float = 0.0,
                max_tokens: Optional[int] = None, *, stream=None) -> Dict[str, torch.Tensor]:
    """The beam_size best label sequences of each utterance under the head H W^T (+ bias): prefix beam
    search over each frame's `candidates` most probable classes and blank.  Returns tokens [N,
    beam_size, max_tokens] (by default the longest utterance's frames), token_lengths and scores [N,
    beam_size] (see BeamSearch.result), and the candidates ids, logp, blank_logp (see
    frame_candidates).  Asynchronous."""
    L = lib()
    H, W, bias, dt = _head_args(H, W, bias)
    T = np.array(_counts(input_lengths), np.int32)
    N, (M, D), V, K, C, dev = int(T.size), H.shape, int(W.shape[0]), int(beam_size), int(candidates), H.device
    if int(T.sum(dtype=np.int64)) != M:
        raise PrunedCTCError(-1, "sum of input lengths differs from the rows of H")
    Tp = T.ctypes.data
    nbytes = int(L.pctc_beam_decode_workspace_size(dt, Tp, N, D, V, K, C))
    if nbytes == 0:
        _check(-3 if (T < 1).any() else -1, "pctc_beam_decode")
    if max_tokens is None:
        max_tokens = int(T.max()) if N else 0
    most = int(max_tokens)
    i32, f32 = torch.int32, torch.float32
    out = {"tokens": torch.empty((N, K, most), dtype=i32, device=dev),
           "token_lengths": torch.empty((N, K), dtype=i32, device=dev),
           "scores": torch.empty((N, K), dtype=f32, device=dev), "ids": torch.empty((M, C), dtype=i32, device=dev),
           "logp": torch.empty((M, C), dtype=f32, device=dev), "blank_logp": torch.empty(M, dtype=f32, device=dev)}
    ws = _scratch(nbytes, dev)
    code = L.pctc_beam_decode(dt, H.data_ptr(), D, W.data_ptr(), None if bias is None else bias.data_ptr(), V, Tp, N,
                              int(blank), K, C, float(token_bonus), most, *map(torch.Tensor.data_ptr, out.values()),
                              ws.data_ptr(), ws.numel(), _raw_stream(dev))
    if code:
        _check(code, "pctc_beam_decode")
    return out


# ---- training step -----------------------------------------------------------------------

@_asynchronous
def clip_grad_norm(grads: Sequence[torch.Tensor], max_norm: float, out: Optional[Sequence[torch.Tensor]] = None,
                   *, stream=None) -> Dict[str, torch.Tensor]:
    """The global 2-norm over a list of float32 and bfloat16 gradients, and every gradient scaled by
    min(1, max_norm / (norm + 1e-6)), in place or into the tensors `out`.  Returns norm and scale
    (float32 [1], on the device).  A norm that is not finite scales by 1: test it before the step (one of
    finite values beyond float32's range is reported as infinite too, but clips).
    Tensors must be contiguous, and what is written must not overlap another tensor of the call (in place: no
    gradient twice in the list, unless max_norm is infinite)."""
    grads = list(grads)
    if not grads:
        raise PrunedCTCError(-1, "no gradients")
    dev = grads[0].device
    if dev.type != "cuda":
        raise PrunedCTCError(-1, "gradients must be device tensors")
    dest = grads if out is None else list(out)
    if len(dest) != len(grads):
        raise PrunedCTCError(-1, "out must have a tensor for each gradient")
    # list-wide checks (lists of hundreds of tensors are ordinary)
    T = torch.Tensor
    dtypes, sizes, devs = [g.dtype for g in grads], list(map(T.numel, grads)), set(map(T.get_device, grads))
    if not all(map(T.is_contiguous, grads)) or devs != {dev.index}:
        raise PrunedCTCError(-1, "gradients must be contiguous tensors of one device")
    if not set(dtypes) <= {torch.float32, torch.bfloat16}:
        raise PrunedCTCError(-1, "gradients must be float32 or bfloat16")
    if out is not None and (
            [o.dtype for o in dest] != dtypes or list(map(T.numel, dest)) != sizes
            or set(map(T.get_device, dest)) != devs or not all(map(T.is_contiguous, dest))):
        raise PrunedCTCError(-1, "out must be contiguous tensors of the gradients' types and sizes on their device")
    n = len(grads)
    L = lib()
    src, dst, counts = _pointers(grads), None if out is None else _pointers(dest), array("q", sizes)
    codes = array("i", [PCTC_F32 if d is torch.float32 else PCTC_BF16 for d in dtypes])
    nbytes = L.pctc_clip_workspace_size(n)
    ws = _scratch(nbytes, dev)
    res = torch.empty(2, dtype=torch.float32, device=dev)
    at = res.data_ptr()
    code = L.pctc_clip_grad_norm(n, _at(src), _at(dst), _at(counts), _at(codes), max_norm, at, at + 4, ws.data_ptr(),
                                 nbytes, _raw_stream(dev))
    if code:
        _check(code, "pctc_clip_grad_norm")
    norm, scale = res.split(1)
    return {"norm": norm, "scale": scale}


# ---- policy loss -------------------------------------------------------------------------

def _sizes_fit(*sizes: int) -> None:
    """The library's sizes are int32; ctypes would cut a larger one off."""
    if max(sizes) >= 2 ** 31 or min(sizes) < -2 ** 31:
        raise PrunedCTCError(-1, "a size does not fit 32 bits")


def _per_token(x: Optional[torch.Tensor], M: int, dev: torch.device, what: str) -> Optional[torch.Tensor]:
    if x is None:
        return None
    if x.numel() != M or x.device != dev or not x.dtype.is_floating_point:
        raise PrunedCTCError(-1, f"{what} must hold a value for each of the {M} rows of H, on {dev}")
    return _as(x.reshape(M), torch.float32)


@_asynchronous
def policy_loss(H: torch.Tensor, W: torch.Tensor, tokens: torch.Tensor, advantages: torch.Tensor,
                old_logp: Optional[torch.Tensor] = None, ref_logp: Optional[torch.Tensor] = None,
                weights: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, clip=(0.2, 0.2),
                kl_weight: float = 0.0, chunk: int = 0, want_dH: bool = True, want_dW: bool = True,
                want_db: bool = False, dH_out: Optional[torch.Tensor] = None, dW_out: Optional[torch.Tensor] = None,
                *, stream=None) -> Dict[str, torch.Tensor]:
    """Clipped policy loss with a KL term on the tokens that the head H W^T (+ bias) emits, row by row (see
    pctc_policy_loss), and its gradients; the rows x vocabulary logits are never stored.  tokens [M]
    int32 or int64, one outside [0, V) is left out (a prompt's places); advantages, old_logp (None: the
    policy itself sampled), ref_logp (None: no KL term) and weights (None: 1; the loss is their
    weighted sum) hold a value per row.  clip: how far below and above 1 the ratio counts (None: anywhere).
    Returns loss (float64 [1]), losses and logp (float32 [M]), status (int32 [M], TOKEN_*) and, of the type
    of H, dH [M, D], dW [V, D] and with want_db db [V].  dH_out / dW_out: the caller's tensors for them."""
    L = lib()
    _sizes_fit(*H.shape, *W.shape, int(chunk))
    H, W, bias, dt = _head_args(H, W, bias)
    (M, D), V, dev = H.shape, int(W.shape[0]), H.device
    if tokens.numel() != M or tokens.dtype not in (torch.int32, torch.int64) or tokens.device != dev:
        raise PrunedCTCError(-1, f"tokens must be int32 or int64, one for each of the {M} rows of H, on {dev}")
    if tokens.dtype is torch.int64:  # (nothing wraps into the vocabulary)
        tokens = tokens.clamp(-1, V)
    tokens = _as(tokens.reshape(M), torch.int32)
    adv, old, ref, w = (_per_token(x, M, dev, what) for x, what in (
        (advantages, "advantages"), (old_logp, "old_logp"), (ref_logp, "ref_logp"), (weights, "weights")))
    if adv is None:
        raise PrunedCTCError(-1, "no advantages")
    try:
        lo, hi = (math.inf, math.inf) if clip is None else map(float, clip)
    except (TypeError, ValueError):
        raise PrunedCTCError(-1, "clip must be None or how far below and above 1 the ratio counts") from None
    dH = _out(dH_out, (M, D), H.dtype, H, "dH_out") if want_dH else None
    dW = _out(dW_out, (V, D), H.dtype, H, "dW_out") if want_dW else None
    db = H.new_empty(V) if want_db else None
    nbytes = int(L.pctc_policy_workspace_size(dt, M, D, V, int(bias is not None), int(want_dH or want_dW or want_db),
                                              int(chunk)))
    if nbytes == 0:
        _check(-1, "pctc_policy_loss")
    loss = H.new_empty(1, dtype=torch.float64)
    losses, logp = H.new_empty((2, M), dtype=torch.float32).unbind()
    status = H.new_empty(M, dtype=torch.int32)
    ws = _scratch(nbytes, dev)
    at = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    code = L.pctc_policy_loss(dt, at(H), M, D, at(W), at(bias), V, at(tokens), at(adv), at(old), at(ref), at(w), lo,
                              hi, float(kl_weight), int(chunk), at(loss), at(losses), at(logp), at(status), at(dH),
                              at(dW), at(db), at(ws), ws.numel(), _raw_stream(dev))
    if code:
        _check(code, "pctc_policy_loss")
    return {"loss": loss, "losses": losses, "logp": logp, "status": status, "dH": dH, "dW": dW, "db": db}


# ---- below the head ----------------------------------------------------------------------

def _out(out: Optional[torch.Tensor], shape, dtype: torch.dtype, like: torch.Tensor, what: str = "out") -> torch.Tensor:
    """A new contiguous tensor, or the caller's, which must be one of that shape (on the device of `like`)."""
    dev = like.device
    if out is None:  # (half the time of torch.empty with a device; but what is not contiguous keeps its strides there)
        same = shape == like.shape and dtype is like.dtype and like.is_contiguous()
        return torch.empty_like(like) if same else like.new_empty(shape, dtype=dtype)
    if out.dtype is not dtype or tuple(out.shape) != tuple(shape) or out.device != dev or not out.is_contiguous():
        raise PrunedCTCError(-1, f"{what} must be contiguous {dtype} {tuple(shape)} on {dev}")
    return out


def _u64(x, what: str) -> int:
    if isinstance(x, float) or int(x) != x or not 0 <= int(x) < 2 ** 64:
        raise PrunedCTCError(-1, f"{what} must be a whole number below 2^64")
    return int(x)


@_asynchronous
def dropout(x: torch.Tensor, p: float, seed: int, offset=0, residual: Optional[torch.Tensor] = None,
            out: Optional[torch.Tensor] = None, *, stream=None) -> torch.Tensor:
    """Each value of x (bfloat16 or float32, any shape) zero with probability p, else times the inverse of
    the share kept, plus `residual`.  The mask is a function of seed, offset and the value's place alone
    (see pctc_dropout) and is not kept anywhere: the gradient of x is dropout(dy, p, seed, offset).  A call uses
    (x.numel() + 7) // 8 counters from offset on; calls that should differ take other offsets or seeds.
    offset: a whole number, or a device int64 tensor of one, which a captured graph reads at each replay.
    out may be x or residual."""
    if not x.is_cuda:
        raise PrunedCTCError(-1, "x must be a device tensor")
    dt, dev = _dtype_code(x), x.device
    x = x.contiguous()
    if residual is not None:
        if residual.dtype is not x.dtype or residual.shape != x.shape or residual.device != dev:
            raise PrunedCTCError(-1, "residual must be a tensor like x")
        residual = residual.contiguous()
    counter = None
    if isinstance(offset, torch.Tensor):
        if offset.dtype is not torch.int64 or offset.numel() != 1 or offset.device != dev:
            raise PrunedCTCError(-1, f"offset must be a whole number or an int64 tensor of one on {dev}")
        counter, offset = offset, 0
    y = _out(out, x.shape, x.dtype, x)
    code = lib().pctc_dropout(dt, x.data_ptr(), None if residual is None else residual.data_ptr(), y.data_ptr(),
                              x.numel(), float(p), _u64(seed, "seed"), _u64(offset, "offset"),
                              None if counter is None else counter.data_ptr(), _raw_stream(dev))
    if code:
        _check(code, "pctc_dropout")
    return y


def _token_args(tokens: torch.Tensor, dev: torch.device):
    if tokens.dtype not in (torch.int32, torch.int64) or tokens.device != dev:
        raise PrunedCTCError(-1, f"tokens must be int32 or int64 on {dev}")
    return tokens.contiguous(), 4 if tokens.dtype is torch.int32 else 8


@_asynchronous
def embedding(table: torch.Tensor, tokens: torch.Tensor, scale: float = 1.0, out: Optional[torch.Tensor] = None,
              *, stream=None) -> torch.Tensor:
    """Rows of table [V, D] (bfloat16 or float32) by token, times scale: [*tokens.shape, D].  A token outside
    [0, V) (a beam's -1 past its end) gives zeros.  tokens: int32 or int64, any shape."""
    if table.dim() != 2 or not table.is_cuda:
        raise PrunedCTCError(-1, "table must be a device tensor [V, D]")
    dt, dev, (V, D) = _dtype_code(table), table.device, table.shape
    _sizes_fit(V, D)
    table = table.contiguous()
    tokens, size = _token_args(tokens, dev)
    y = _out(out, (*tokens.shape, D), table.dtype, table)
    code = lib().pctc_embedding(dt, table.data_ptr(), V, D, tokens.data_ptr(), size, tokens.numel(), float(scale),
                                y.data_ptr(), _raw_stream(dev))
    if code:
        _check(code, "pctc_embedding")
    return y


@_asynchronous
def embedding_backward(dy: torch.Tensor, tokens: torch.Tensor, V: int, scale: float = 1.0,
                       out: Optional[torch.Tensor] = None, accumulate: bool = False,
                       dtype: Optional[torch.dtype] = None, *, stream=None) -> torch.Tensor:
    """Gradient of embedding()'s table [V, D] from dy [*tokens.shape, D]: the scaled sum of dy's rows for
    every class, summed in float in an order that the sizes fix.  New (in `dtype`, by default dy's), written
    into `out`, or with accumulate added to what `out` holds (the gradient that a loss left in the
    head tied to the table: float32 with a bfloat16 dy is ordinary)."""
    if not dy.is_cuda:
        raise PrunedCTCError(-1, "dy must be a device tensor")
    dt, dev = _dtype_code(dy), dy.device
    tokens, size = _token_args(tokens, dev)
    if dy.dim() < 1 or dy.shape[:-1] != tokens.shape:
        raise PrunedCTCError(-1, "dy must be [*tokens.shape, D]")
    V, D, N = int(V), int(dy.shape[-1]), tokens.numel()
    if accumulate and out is None:
        raise PrunedCTCError(-1, "accumulate needs out")
    kind = dtype if dtype is not None else dy.dtype if out is None else out.dtype
    if kind not in (torch.float32, torch.bfloat16):
        raise PrunedCTCError(-1, f"unsupported dtype {kind}")
    if V < 1 or D < 1:
        raise PrunedCTCError(-1, "V and D must be positive")
    _sizes_fit(V, D)
    dy = dy.contiguous()
    dW = _out(out, (V, D), kind, dy)
    L = lib()
    nbytes = L.pctc_embedding_backward_workspace_size(N, D)
    if nbytes == 0:
        _check(-1, "pctc_embedding_backward")
    ws = _scratch(nbytes, dev)
    code = L.pctc_embedding_backward(dt, dy.data_ptr(), tokens.data_ptr(), size, N, V, D, float(scale), _dtype_code(dW),
                                     dW.data_ptr(), int(bool(accumulate)), ws.data_ptr(), ws.numel(), _raw_stream(dev))
    if code:
        _check(code, "pctc_embedding_backward")
    return dW


_ACTIVATIONS = {"silu": 0, "gelu": 1}


def _ffn_args(x, w_gate, w_up, w_down, activation):
    """Checked and contiguous tensors of a gated block, its sizes, type code and activation's code."""
    dt, dev = _dtype_code(x), x.device
    if activation not in _ACTIVATIONS:
        raise PrunedCTCError(-1, f"activation must be one of {', '.join(_ACTIVATIONS)}")
    if not x.is_cuda or any(w.dtype is not x.dtype or w.device != dev for w in (w_gate, w_up, w_down)):
        raise PrunedCTCError(-1, "x and the weights must be tensors of one type on one device")
    if x.dim() < 1 or any(w.dim() != 2 for w in (w_gate, w_up, w_down)):
        raise PrunedCTCError(-1, "x must be [..., D] and the weights matrices")
    D, F, O = int(x.shape[-1]), int(w_gate.shape[0]), int(w_down.shape[0])
    if tuple(w_gate.shape) != (F, D) or w_up.shape != w_gate.shape or w_down.shape[1] != F:
        raise PrunedCTCError(-1, "w_gate and w_up must be [F, D], w_down [O, F]")
    M = x.numel() // D if D else 0
    _sizes_fit(M, D, F, O)
    return x.contiguous(), w_gate.contiguous(), w_up.contiguous(), w_down.contiguous(), (M, D, F, O), dt, \
        _ACTIVATIONS[activation]


@_asynchronous
def gated_ffn(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor,
              activation: str = "silu", keep: bool = False, out: Optional[torch.Tensor] = None,
              *, stream=None) -> Dict[str, Optional[torch.Tensor]]:
    """Gated feed-forward block y = (act(x w_gate^T) * (x w_up^T)) w_down^T of x [..., D], bfloat16 or float32,
    for activation "silu" or "gelu" (by the error function); D, F and O multiples of 8.  Returns y [..., O] and, with
    keep, gate and up [..., F] (float32), the two projections, which the backward reads (else None)."""
    L = lib()
    x, wg, wu, wd, (M, D, F, O), dt, act = _ffn_args(x, w_gate, w_up, w_down, activation)
    dev, lead = x.device, x.shape[:-1]
    nbytes = L.pctc_gated_ffn_workspace_size(dt, M, D, F, O, 0)
    if nbytes == 0:
        _check(-1, "pctc_gated_ffn")
    y = _out(out, (*lead, O), x.dtype, x)
    a, b = (x.new_empty((*lead, F), dtype=torch.float32) for _ in range(2)) if keep else (None, None)
    ws = _scratch(nbytes, dev)
    code = L.pctc_gated_ffn(dt, x.data_ptr(), M, D, wg.data_ptr(), wu.data_ptr(), F, wd.data_ptr(), O, act,
                            a.data_ptr() if keep else None, b.data_ptr() if keep else None, y.data_ptr(), ws.data_ptr(),
                            ws.numel(), _raw_stream(dev))
    if code:
        _check(code, "pctc_gated_ffn")
    return {"y": y, "gate": a, "up": b}


@_asynchronous
def gated_ffn_backward(dy: torch.Tensor, x: torch.Tensor, gate: torch.Tensor, up: torch.Tensor, w_gate: torch.Tensor,
                       w_up: torch.Tensor, w_down: torch.Tensor, activation: str = "silu", want_dx: bool = True,
                       want_dw: bool = True, *, stream=None) -> Dict[str, Optional[torch.Tensor]]:
    """Gradients of gated_ffn from dy [..., O] and the forward's x, gate and up: dx, dw_gate, dw_up and dw_down, of
    the type of x (None where not wanted)."""
    L = lib()
    x, wg, wu, wd, (M, D, F, O), dt, act = _ffn_args(x, w_gate, w_up, w_down, activation)
    dev, lead = x.device, x.shape[:-1]
    for t, n, kind, what in ((dy, O, x.dtype, "dy"), (gate, F, torch.float32, "gate"), (up, F, torch.float32, "up")):
        if t.dtype is not kind or t.device != dev or tuple(t.shape) != (*lead, n):
            raise PrunedCTCError(-1, f"{what} must be {kind} {(*lead, n)} on {dev}")
    dy, gate, up = dy.contiguous(), gate.contiguous(), up.contiguous()
    nbytes = L.pctc_gated_ffn_workspace_size(dt, M, D, F, O, 1)
    if nbytes == 0:
        _check(-1, "pctc_gated_ffn_backward")
    dx = torch.empty_like(x) if want_dx else None
    dws = [torch.empty_like(w) if want_dw else None for w in (wg, wu, wd)]
    ws = _scratch(nbytes, dev)
    at = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    code = L.pctc_gated_ffn_backward(dt, at(dy), at(x), M, D, at(gate), at(up), at(wg), at(wu), F, at(wd), O, act, at(dx),
                                     *map(at, dws), at(ws), ws.numel(), _raw_stream(dev))
    if code:
        _check(code, "pctc_gated_ffn_backward")
    return dict(zip(("dx", "dw_gate", "dw_up", "dw_down"), (dx, *dws)))


class Dropout(torch.autograd.Function):
    """Autograd wrapper of dropout().  The mask is made again in the backward, from the counters of the forward (a
    device tensor's value is copied: the caller may move it on before).  For this layer and those below, as
    for any operator: while a backward is captured into a graph, no autograd graph recorded outside the
    capture may still hold the same leaves."""

    @staticmethod
    def forward(ctx, x, p, seed, offset, residual):
        ctx.p, ctx.seed, ctx.has_residual = p, seed, residual is not None
        ctx.offset = offset.clone() if isinstance(offset, torch.Tensor) else offset
        return dropout(x.detach(), p, seed, ctx.offset, None if residual is None else residual.detach())

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        dx = dropout(dy, ctx.p, ctx.seed, ctx.offset) if ctx.needs_input_grad[0] else None
        return dx, None, None, None, dy if ctx.has_residual and ctx.needs_input_grad[4] else None


class Embedding(torch.autograd.Function):
    """Autograd wrapper of embedding(); the table's gradient has its type."""

    @staticmethod
    def forward(ctx, table, tokens, scale):
        ctx.save_for_backward(tokens)
        ctx.scale, ctx.V = scale, int(table.shape[0])
        return embedding(table.detach(), tokens, scale)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        (tokens,) = ctx.saved_tensors
        return embedding_backward(dy, tokens, ctx.V, ctx.scale) if ctx.needs_input_grad[0] else None, None, None


class GatedFFN(torch.autograd.Function):
    """Autograd wrapper of gated_ffn()."""

    @staticmethod
    def forward(ctx, x, w_gate, w_up, w_down, activation):
        r = gated_ffn(x.detach(), w_gate.detach(), w_up.detach(), w_down.detach(), activation,
                      keep=any(ctx.needs_input_grad[:4]))
        ctx.activation = activation
        ctx.save_for_backward(x, r["gate"], r["up"], w_gate, w_up, w_down)
        return r["y"]

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, gate, up, wg, wu, wd = (t.detach() for t in ctx.saved_tensors)
        need = ctx.needs_input_grad
        r = gated_ffn_backward(dy, x, gate, up, wg, wu, wd, ctx.activation, want_dx=need[0], want_dw=any(need[1:4]))
        return r["dx"], *(r[k] if n else None for k, n in zip(("dw_gate", "dw_up", "dw_down"), need[1:4])), None


def dropout_layer(x: torch.Tensor, p: float, seed: int, offset=0, residual: Optional[torch.Tensor] = None):
    """dropout() with gradients for x and residual."""
    return Dropout.apply(x, p, seed, offset, residual)


def embedding_layer(table: torch.Tensor, tokens: torch.Tensor, scale: float = 1.0):
    """embedding() with a gradient for the table."""
    return Embedding.apply(table, tokens, scale)


def gated_ffn_layer(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor,
                    activation: str = "silu"):
    """gated_ffn()'s y with gradients for x and the weights."""
    return GatedFFN.apply(x, w_gate, w_up, w_down, activation)


# ---- kernel timing -----------------------------------------------------------------------

def prof_enable(on: bool = True) -> None:
    lib().pctc_prof_enable(1 if on else 0)


def prof_select(name: Optional[str] = None) -> None:
    """Time only the kernels called `name` (None: all of them)."""
    lib().pctc_prof_select(name.encode() if name else None)


def prof_reset() -> None:
    lib().pctc_prof_reset()


def prof_read() -> Dict[str, Dict[str, float]]:
    L = lib()
    out = {}
    for i in range(L.pctc_prof_count()):
        name = ctypes.c_char_p()
        ms = ctypes.c_double()
        n = ctypes.c_int64()
        if L.pctc_prof_get(i, ctypes.byref(name), ctypes.byref(ms), ctypes.byref(n)):
            out[name.value.decode()] = {"total_ms": ms.value, "launches": int(n.value)}
    return out
