"""Python binding of the block-sparse attention path (argument marshalling only).

Every computation runs in the HIP kernels of libwavealign.so; torch supplies
device memory and the current HIP stream.
"""
from __future__ import annotations

import ctypes
import functools
import math
from typing import Optional

import torch

from . import _lib as L

_SKIP = {"auto": L.WA_SKIP_AUTO, "never": L.WA_SKIP_NEVER, "always": L.WA_SKIP_ALWAYS}
_DTYPE = {torch.bfloat16: L.WA_BF16, torch.float16: L.WA_F16, torch.float32: L.WA_F32}
_ROTARY_LAYOUT = {"half": L.WA_ROTARY_HALF, "interleaved": L.WA_ROTARY_INTERLEAVED}
_ROTARY_SCALING = {"none": L.WA_ROTARY_PLAIN, "linear": L.WA_ROTARY_LINEAR, "ntk": L.WA_ROTARY_NTK,
                   "yarn": L.WA_ROTARY_YARN}
_HEAD_ORDER = {"in-order": L.WA_HEADS_IN_ORDER, "interleaved": L.WA_HEADS_INTERLEAVED}


def _stream() -> ctypes.c_void_p:
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _dev(t: torch.Tensor, name: str) -> None:
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _mask_u8(mask: torch.Tensor, shape=None) -> torch.Tensor:
    """The mask as uint8, checked against the expected [B][H][M_B][N_B] shape (if given) before
    its placement, so that a mismatch is reported the same way on any device."""
    if mask.dtype not in (torch.bool, torch.uint8):
        raise ValueError("mask must be uint8 or bool")
    if mask.dim() != 4 or (shape is not None and tuple(mask.shape) != tuple(shape)):
        want = "[B][H][M_B][N_B]" if shape is None else str(tuple(shape))
        raise ValueError(f"mask must have shape {want}, got {tuple(mask.shape)}")
    if mask.shape[2] != mask.shape[3]:
        raise ValueError(f"mask must be square per head (M_B = N_B), got {tuple(mask.shape)}")
    return mask.view(torch.uint8) if mask.dtype == torch.bool else mask


def _check(t: Optional[torch.Tensor], name: str, dtype, shape=None, numel_min: Optional[int] = None) -> None:
    """dtype and shape (or minimum element count) of an optional tensor argument."""
    if t is None:
        return
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if numel_min is not None and t.numel() < numel_min:
        raise ValueError(f"{name} must hold at least {numel_min} elements, got {t.numel()}")


def _on_device(**tensors) -> None:
    """Placement and layout, checked once every shape is known to be right."""
    for name, t in tensors.items():
        if t is not None:
            _dev(t, name)


def _mask_dims(mask: torch.Tensor, seq_len: int, block: int):
    b, h = mask.shape[0], mask.shape[1]
    mb = -(-seq_len // block)
    return b, h, mb


def shape_of(batch: int, heads: int, seq_len: int, head_dim: int, block: int) -> L.WaShape:
    return L.WaShape(batch, heads, seq_len, head_dim, block)


def _workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(nbytes, 1), dtype=torch.uint8, device=device)


def wave_size(head_dim: int, block: int) -> int:
    lib = L.load()
    out = ctypes.c_int32(0)
    L.check(lib.wa_wave_size(head_dim, block, ctypes.byref(out)))
    return out.value


def default_skip_profile() -> L.WaSkipProfile:
    lib = L.load()
    p = L.WaSkipProfile()
    L.check(lib.wa_default_skip_profile(ctypes.byref(p)))
    return p


def perm_workspace_size(shape: L.WaShape) -> int:
    lib = L.load()
    n = ctypes.c_size_t(0)
    L.check(lib.wa_perm_workspace_size(ctypes.byref(shape), ctypes.byref(n)))
    return n.value


def _size(call: str, shape: L.WaShape) -> int:
    n = ctypes.c_size_t(0)
    L.check(getattr(L.load(), call)(ctypes.byref(shape), ctypes.byref(n)))
    return n.value


def _attn_workspace(workspace, call: str, shape: L.WaShape, device) -> torch.Tensor:
    """The given workspace if the call can run in it, else a new one with room for split rows."""
    need = _size(call, shape)
    if workspace is None or workspace.numel() < need:
        workspace = _workspace(need + _size("wa_attn_split_workspace_size", shape), device)
    return workspace


def attn_workspace_size(shape: L.WaShape) -> int:
    """Bytes for sparse_attn and sparse_attn_csr, with the room in which rows can be split."""
    return _size("wa_attn_workspace_size", shape) + _size("wa_attn_split_workspace_size", shape)


def mask_stats(mask: torch.Tensor, *, seq_len: int, block: int, head_dim: int = 128):
    """(row_nnz [B][H][M_B], col_cnt [B][H][N_B], head_stats [B][H][6]) as device tensors."""
    lib = L.load()
    b, h, mb = _mask_dims(mask, seq_len, block)
    mask = _mask_u8(mask, (b, h, mb, mb))
    _on_device(mask=mask)
    shape = shape_of(b, h, seq_len, head_dim, block)
    dev = mask.device
    row_nnz = torch.empty((b, h, mb), dtype=torch.int32, device=dev)
    col_cnt = torch.empty((b, h, mb), dtype=torch.int32, device=dev)
    stats = torch.empty((b, h, 6), dtype=torch.int64, device=dev)
    ws = _workspace(perm_workspace_size(shape), dev)
    L.check(lib.wa_mask_stats(_ptr(mask), ctypes.byref(shape), _ptr(row_nnz), _ptr(col_cnt), _ptr(stats),
                              _ptr(ws), ws.numel(), _stream()))
    return row_nnz, col_cnt, stats


def build_permutation(mask: torch.Tensor, *, seq_len: int, block: int, head_dim: int, wave: Optional[int] = None,
                      n_xcd: int = 8, iters: int = 10, seed: int = 0, skip: str = "auto",
                      profile: Optional[L.WaSkipProfile] = None, workspace: Optional[torch.Tensor] = None,
                      return_info: bool = False, out: Optional[torch.Tensor] = None,
                      flags_out: Optional[torch.Tensor] = None, seg_out: Optional[torch.Tensor] = None,
                      stage1_out: Optional[torch.Tensor] = None):
    """(perm int32 [B][H][M_B], seg_start int32 [B][H][n_xcd+1], head flags uint8 [B][H])
    (plus embedding and Stage-1 order if asked; stage1_out, if given, receives the Stage-1 order)."""
    lib = L.load()
    b, h, mb = _mask_dims(mask, seq_len, block)
    mask = _mask_u8(mask, (b, h, mb, mb))
    if skip not in _SKIP:
        raise ValueError(f"skip must be one of {sorted(_SKIP)}")
    _check(out, "out", torch.int32, (b, h, mb))
    _check(flags_out, "flags_out", torch.uint8, (b, h))
    _check(seg_out, "seg_out", torch.int32, (b, h, n_xcd + 1))
    _check(stage1_out, "stage1_out", torch.int32, (b, h, mb))
    _check(workspace, "workspace", torch.uint8)
    _on_device(mask=mask, out=out, flags_out=flags_out, seg_out=seg_out, stage1_out=stage1_out, workspace=workspace)
    shape = shape_of(b, h, seq_len, head_dim, block)
    dev = mask.device
    perm = torch.empty((b, h, mb), dtype=torch.int32, device=dev) if out is None else out
    flags = torch.empty((b, h), dtype=torch.uint8, device=dev) if flags_out is None else flags_out
    seg = torch.empty((b, h, n_xcd + 1), dtype=torch.int32, device=dev) if seg_out is None else seg_out
    emb = torch.empty((b, h, mb, 2), dtype=torch.int32, device=dev) if return_info else None
    s1 = torch.empty((b, h, mb), dtype=torch.int32, device=dev) if return_info and stage1_out is None else stage1_out
    params = L.WaPermParams(0 if wave is None else int(wave), int(n_xcd), int(iters), _SKIP[skip],
                            int(seed) & ((1 << 64) - 1),
                            ctypes.pointer(profile) if profile is not None else None)
    need = perm_workspace_size(shape)
    if workspace is None or workspace.numel() < need:
        workspace = _workspace(need, dev)
    L.check(lib.wa_build_permutation(_ptr(mask), ctypes.byref(shape), ctypes.byref(params), _ptr(perm), _ptr(seg),
                                     _ptr(flags), _ptr(emb), _ptr(s1), _ptr(workspace), workspace.numel(),
                                     _stream()))
    if return_info:
        return perm, seg, flags, emb, s1
    return perm, seg, flags


def compact_mask(mask: torch.Tensor, *, seq_len: int, block: int, head_dim: int = 128,
                 row_ptr: Optional[torch.Tensor] = None, col_idx: Optional[torch.Tensor] = None):
    """CSR lists: row_ptr int32 [B][H][M_B+1] (head-local offsets), col_idx int32 [B*H*M_B*N_B]."""
    lib = L.load()
    b, h, mb = _mask_dims(mask, seq_len, block)
    mask = _mask_u8(mask, (b, h, mb, mb))
    _check(row_ptr, "row_ptr", torch.int32, (b, h, mb + 1))
    _check(col_idx, "col_idx", torch.int32, numel_min=b * h * mb * mb)
    _on_device(mask=mask, row_ptr=row_ptr, col_idx=col_idx)
    shape = shape_of(b, h, seq_len, head_dim, block)
    if row_ptr is None:
        row_ptr = torch.empty((b, h, mb + 1), dtype=torch.int32, device=mask.device)
    if col_idx is None:
        col_idx = torch.empty((b * h * mb * mb,), dtype=torch.int32, device=mask.device)
    L.check(lib.wa_compact_mask(_ptr(mask), ctypes.byref(shape), _ptr(row_ptr), _ptr(col_idx), _stream()))
    return row_ptr, col_idx


def mask_producer_workspace_size(shape: L.WaShape) -> int:
    lib = L.load()
    n = ctypes.c_size_t(0)
    L.check(lib.wa_mask_producer_workspace_size(ctypes.byref(shape), ctypes.byref(n)))
    return n.value


def produce_block_mask(q: torch.Tensor, k: torch.Tensor, *, block: int, keep: int, diagonal: bool = True,
                       out: Optional[torch.Tensor] = None, codes_out: Optional[torch.Tensor] = None,
                       workspace: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Pooled-score top-k block mask uint8 [B][H][M_B][M_B] from q, k bf16 [B][H][N][d]. ``status``: an int32
    device tensor of one element the call zeroes and sets WA_PRODUCE_WAIT_EXPIRED in (nullable)."""
    lib = L.load()
    for t, nm in ((q, "q"), (k, "k")):
        _dev(t, nm)
        if t.dtype != torch.bfloat16:
            raise ValueError(f"{nm} must be bfloat16")
    if q.shape != k.shape or q.dim() != 4:
        raise ValueError("q and k must share one [B][H][N][d] shape")
    b, h, n, d = q.shape
    shape = shape_of(b, h, n, d, block)
    mb = -(-n // block)
    mask = torch.empty((b, h, mb, mb), dtype=torch.uint8, device=q.device) if out is None else out
    if mask.dtype != torch.uint8 or mask.numel() < b * h * mb * mb:
        raise ValueError("out must be a uint8 tensor of B*H*M_B*M_B elements")
    if codes_out is not None and (codes_out.dtype != torch.int8 or codes_out.numel() < 2 * b * h * mb * d):
        raise ValueError("codes_out must be an int8 tensor of 2*B*H*M_B*d elements")
    if status is not None and (status.dtype != torch.int32 or status.numel() < 1):
        raise ValueError("status must be an int32 tensor of at least one element")
    need = mask_producer_workspace_size(shape)
    if workspace is None or workspace.numel() < need:
        workspace = _workspace(need, q.device)
    L.check(lib.wa_produce_block_mask(_ptr(q), _ptr(k), ctypes.byref(shape), int(keep), 1 if diagonal else 0,
                                      _ptr(mask), _ptr(codes_out), _ptr(status), _ptr(workspace), workspace.numel(),
                                      _stream()))
    return mask


def check_perm(perm: torch.Tensor, *, seq_len: int, block: int, head_dim: int = 128,
               head_ok: Optional[torch.Tensor] = None) -> bool:
    """True if every perm[b][h] is a permutation of 0..M_B-1 (synchronises the current stream)."""
    lib = L.load()
    _dev(perm, "perm")
    if perm.dtype != torch.int32 or perm.dim() != 3:
        raise ValueError("perm must be an int32 [B][H][M_B] tensor")
    b, h, mb = perm.shape
    shape = shape_of(b, h, seq_len, head_dim, block)
    if -(-seq_len // block) != mb:
        raise ValueError("perm's last dimension must be ceil(seq_len / block)")
    n = ctypes.c_size_t(0)
    L.check(lib.wa_check_perm_workspace_size(ctypes.byref(shape), ctypes.byref(n)))
    ws = _workspace(n.value, perm.device)
    st = lib.wa_check_perm(_ptr(perm.contiguous()), ctypes.byref(shape), _ptr(head_ok), _ptr(ws), ws.numel(),
                           _stream())
    if st == L.WA_ERR_INVALID_PERM:
        return False
    L.check(st)
    return True


def _attn_args(q, k, v, block, v_transposed=False):
    """Shape of the call from q, k, v (checked before their placement); v may be the transposed
    [B][H][d][M_B*block] layout."""
    for t, nm in ((q, "q"), (k, "k"), (v, "v")):
        if t.dtype != torch.bfloat16:
            raise ValueError(f"{nm} must be bfloat16")
    if q.dim() != 4 or q.shape != k.shape:
        raise ValueError("q and k must share one [B][H][N][d] shape")
    b, h, n, d = q.shape
    if v_transposed:
        want = (b, h, d, -(-n // block) * block)
        if tuple(v.shape) != want:
            raise ValueError(f"vt must have shape {want} ([B][H][d][M_B*block]), got {tuple(v.shape)}")
    elif v.shape != q.shape:
        raise ValueError("q, k, v must share one [B][H][N][d] shape")
    return shape_of(b, h, n, d, block)


def _attn_outputs(q, out, status, return_lse):
    _check(out, "out", torch.bfloat16, tuple(q.shape))
    _check(status, "status", torch.int32, numel_min=1)
    if out is None or return_lse:
        _on_device(q=q)
    o = torch.empty_like(q) if out is None else out
    lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device) if return_lse else None
    return o, lse


def _order_args(q, block, perm, seg, n_xcd):
    b, h, n, _ = q.shape
    mb = -(-n // block)
    if not 1 <= int(n_xcd) <= 64:
        raise ValueError("n_xcd must lie in 1..64")
    _check(perm, "perm", torch.int32, (b, h, mb))
    _check(seg, "seg", torch.int32, (b, h, int(n_xcd) + 1))
    return b, h, mb


def _csr_args(row_ptr, col_idx, b, h, mb):
    if row_ptr is None or col_idx is None:
        raise ValueError("row_ptr and col_idx are required")
    _check(row_ptr, "row_ptr", torch.int32, (b, h, mb + 1))
    _check(col_idx, "col_idx", torch.int32, numel_min=b * h * mb * mb)


def sparse_attn(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, mask: torch.Tensor,
                perm: Optional[torch.Tensor] = None, seg: Optional[torch.Tensor] = None, *, block: int,
                scale: Optional[float] = None,
                n_xcd: int = 8, return_lse: bool = False, out: Optional[torch.Tensor] = None,
                workspace: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
    """O = block-sparse softmax attention of q over the kept KV blocks, in the original row order.
    `status` (int32, device) receives the call's WA_ATTN_* bits."""
    lib = L.load()
    shape = _attn_args(q, k, v, block)
    b, h, mb = _order_args(q, block, perm, seg, n_xcd)
    mask = _mask_u8(mask, (b, h, mb, mb))
    _check(workspace, "workspace", torch.uint8)
    o, lse = _attn_outputs(q, out, status, return_lse)
    _on_device(q=q, k=k, v=v, mask=mask, perm=perm, seg=seg, out=o, status=status, workspace=workspace)
    workspace = _attn_workspace(workspace, "wa_attn_workspace_size", shape, q.device)
    L.check(lib.wa_sparse_attn(_ptr(q), _ptr(k), _ptr(v), _ptr(mask), _ptr(perm), _ptr(seg), ctypes.byref(shape),
                               float(scale or 0.0), int(n_xcd), _ptr(o), _ptr(lse), _ptr(status), _ptr(workspace),
                               workspace.numel(), _stream()))
    return (o, lse) if return_lse else o


def sparse_attn_csr(q, k, v, row_ptr, col_idx, perm=None, seg=None, *, block: int, scale: Optional[float] = None,
                    n_xcd: int = 8, return_lse: bool = False, out: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
    """As sparse_attn, from the lists of compact_mask."""
    lib = L.load()
    shape = _attn_args(q, k, v, block)
    b, h, mb = _order_args(q, block, perm, seg, n_xcd)
    _csr_args(row_ptr, col_idx, b, h, mb)
    _check(workspace, "workspace", torch.uint8)
    o, lse = _attn_outputs(q, out, status, return_lse)
    _on_device(q=q, k=k, v=v, row_ptr=row_ptr, col_idx=col_idx, perm=perm, seg=seg, out=o, status=status,
               workspace=workspace)
    workspace = _attn_workspace(workspace, "wa_attn_workspace_size", shape, q.device)
    L.check(lib.wa_sparse_attn_csr(_ptr(q), _ptr(k), _ptr(v), _ptr(row_ptr), _ptr(col_idx), _ptr(perm), _ptr(seg),
                                   ctypes.byref(shape), float(scale or 0.0), int(n_xcd), _ptr(o), _ptr(lse),
                                   _ptr(status), _ptr(workspace), workspace.numel(), _stream()))
    return (o, lse) if return_lse else o


def transpose_v(v: torch.Tensor, *, block: int, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """V [B][H][N][d] -> V^T [B][H][d][M_B*block], zero past the last token (the layout of sparse_attn_vt)."""
    lib = L.load()
    if v.dtype != torch.bfloat16 or v.dim() != 4:
        raise ValueError("v must be a bfloat16 [B][H][N][d] tensor")
    b, h, n, d = v.shape
    want = (b, h, d, -(-n // block) * block)
    _check(out, "out", torch.bfloat16, want)
    _on_device(v=v, out=out)
    vt = torch.empty(want, dtype=torch.bfloat16, device=v.device) if out is None else out
    shape = shape_of(b, h, n, d, block)
    L.check(lib.wa_transpose_v(_ptr(v), ctypes.byref(shape), _ptr(vt), _stream()))
    return vt


def attn_vt_workspace_size(shape: L.WaShape) -> int:
    """Bytes for sparse_attn_vt, with the room in which rows can be split."""
    return _size("wa_attn_vt_workspace_size", shape) + _size("wa_attn_split_workspace_size", shape)


def sparse_attn_vt(q, k, vt, row_ptr, col_idx, perm=None, seg=None, *, block: int, scale: Optional[float] = None,
                   n_xcd: int = 8, head_order: str = "in-order", return_lse: bool = False,
                   out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                   status: Optional[torch.Tensor] = None):
    """As sparse_attn_csr with V given as V^T (transpose_v's layout); head_order is "in-order" (heads one
    after another in every queue) or "interleaved" (round-robin over the heads)."""
    lib = L.load()
    if head_order not in _HEAD_ORDER:
        raise ValueError(f"head_order must be one of {sorted(_HEAD_ORDER)}")
    shape = _attn_args(q, k, vt, block, v_transposed=True)
    b, h, mb = _order_args(q, block, perm, seg, n_xcd)
    _csr_args(row_ptr, col_idx, b, h, mb)
    _check(workspace, "workspace", torch.uint8)
    o, lse = _attn_outputs(q, out, status, return_lse)
    _on_device(q=q, k=k, vt=vt, row_ptr=row_ptr, col_idx=col_idx, perm=perm, seg=seg, out=o, status=status,
               workspace=workspace)
    workspace = _attn_workspace(workspace, "wa_attn_vt_workspace_size", shape, q.device)
    opts = L.WaAttnOptions(float(scale or 0.0), int(n_xcd), _HEAD_ORDER[head_order])
    L.check(lib.wa_sparse_attn_vt(_ptr(q), _ptr(k), _ptr(vt), _ptr(row_ptr), _ptr(col_idx), _ptr(perm), _ptr(seg),
                                  ctypes.byref(shape), ctypes.byref(opts), _ptr(o), _ptr(lse), _ptr(status),
                                  _ptr(workspace), workspace.numel(), _stream()))
    return (o, lse) if return_lse else o


def sparse_attn_vt_noalloc(q, k, vt, row_ptr, col_idx, perm=None, seg=None, *, block: int,
                           scale: Optional[float] = None, n_xcd: int = 8, head_order: str = "in-order",
                           lse: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                           status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """As sparse_attn_vt, for callers that cannot allocate: the library keeps the scheduler state in
    its static per-GPU scratch, so `out` (and `lse`, if wanted) must be given. Calls that overlap on
    one GPU race."""
    lib = L.load()
    if head_order not in _HEAD_ORDER:
        raise ValueError(f"head_order must be one of {sorted(_HEAD_ORDER)}")
    if out is None:
        raise ValueError("out is required (this entry point allocates nothing)")
    shape = _attn_args(q, k, vt, block, v_transposed=True)
    b, h, mb = _order_args(q, block, perm, seg, n_xcd)
    _csr_args(row_ptr, col_idx, b, h, mb)
    _check(out, "out", torch.bfloat16, tuple(q.shape))
    _check(lse, "lse", torch.float32, tuple(q.shape[:3]))
    _check(status, "status", torch.int32, numel_min=1)
    _on_device(q=q, k=k, vt=vt, row_ptr=row_ptr, col_idx=col_idx, perm=perm, seg=seg, out=out, lse=lse,
               status=status)
    opts = L.WaAttnOptions(float(scale or 0.0), int(n_xcd), _HEAD_ORDER[head_order])
    L.check(lib.wa_sparse_attn_vt_noalloc(_ptr(q), _ptr(k), _ptr(vt), _ptr(row_ptr), _ptr(col_idx), _ptr(perm),
                                          _ptr(seg), ctypes.byref(shape), ctypes.byref(opts), _ptr(out), _ptr(lse),
                                          _ptr(status), _stream()))
    return out


def _one_device(**tensors) -> int:
    """The device that all given tensors share; work is enqueued on that device's current stream."""
    index = -1
    for name, t in tensors.items():
        if t is None:
            continue
        if index < 0:
            index = t.get_device()
        if index < 0 or not t.is_cuda:
            raise ValueError(f"{name} must be a device tensor")
        if t.get_device() != index:
            raise ValueError(f"{name} is on {t.device}, the tensors before it on cuda:{index}")
    return index


def _call_on(index: int, call, *args) -> None:
    """The library call with device ``index`` current and its current stream as the last argument. The raw handles are asked
    for as torch's own extensions do: its stream and device objects take 3.5 us a call, these 0.3."""
    if index == torch._C._cuda_getDevice():
        L.check(call(*args, torch._C._cuda_getCurrentRawStream(index)))
        return
    with torch.cuda.device(index):
        L.check(call(*args, _stream()))


def rotary_frequencies(pairs: int, *, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                       original_len: float = 4096.0, beta_fast: float = 32.0, beta_slow: float = 1.0, device="cuda"):
    """(inv_freq float64 [pairs] on ``device``, scale) of one position axis for ``rotary``: base^(-i / pairs), for
    contexts ``factor`` times the trained length divided by it ("linear"), with a larger base ("ntk") or by the pair's
    turns over ``original_len`` ("yarn", linear in the turns, not in the pair's index; it also grows the values by scale). Axes are
    concatenated by the caller."""
    if scaling not in _ROTARY_SCALING:
        raise ValueError(f"scaling must be one of {sorted(_ROTARY_SCALING)}")
    freq, scale = (ctypes.c_double * max(int(pairs), 1))(), ctypes.c_double(1.0)
    how = L.WaRotaryScaling(_ROTARY_SCALING[scaling], float(factor), float(original_len), float(beta_fast),
                            float(beta_slow))
    L.check(L.load().wa_rotary_frequencies(int(pairs), float(base), ctypes.byref(how), freq, ctypes.byref(scale)))
    return torch.tensor(list(freq), dtype=torch.float64, device=device), scale.value


def rotary(q: torch.Tensor, k: Optional[torch.Tensor] = None, *, inv_freq: torch.Tensor,
           positions: Optional[torch.Tensor] = None, layout: str = "half", axis_pairs=None, scale: float = 1.0,
           backward: bool = False, out_q: Optional[torch.Tensor] = None, out_k: Optional[torch.Tensor] = None):
    """q (and k) [B][H][N][d] with the first 2 P columns of every head rotated by their tokens' positions; (q, k) in
    one launch. bfloat16, float16 or float32 of any strides with whole rows (a projection's [B][N][H][d] comes as
    ``x.transpose(1, 2)``); the result is contiguous, or written to out_q and out_k: any strides, the input itself for in place.

    inv_freq   float64 [P]: radians a position, from rotary_frequencies
    positions  int32 [N], [B][N] or [axes][1 or B][N]; None: token n is at n
    layout     "half" (pair i: columns i and i + P) or "interleaved" (2i and 2i + 1)
    axis_pairs pairs of each position axis (None: one axis)
    scale      factor of the rotated values
    backward   the transposed map: gradients of the outputs in, gradients of q and k out

    No autograd graph is recorded, also where q requires a gradient: the caller makes the backward call."""
    lib = L.load()
    if layout not in _ROTARY_LAYOUT:
        raise ValueError(f"layout must be one of {sorted(_ROTARY_LAYOUT)}")
    if k is None and out_k is not None:
        raise ValueError("out_k without k")
    if q.dim() != 4 or q.dtype not in _DTYPE:
        raise ValueError("q must be a bfloat16, float16 or float32 [B][H][N][d] tensor")
    b, _, n, d = q.shape
    if inv_freq.dtype != torch.float64 or inv_freq.dim() != 1 or not inv_freq.is_contiguous():
        raise ValueError("inv_freq must be a contiguous float64 vector")
    axis = [inv_freq.numel()] if axis_pairs is None else [int(x) for x in axis_pairs]
    axes = len(axis)
    if not 1 <= axes <= 3:
        raise ValueError("axis_pairs must name 1 to 3 axes")
    pos_batch = 1
    if positions is not None:
        ps = tuple(positions.shape)
        if (positions.dtype != torch.int32 or not positions.is_contiguous() or ps[-1:] != (n,)
                or not (ps[:-1] in ((axes, 1), (axes, b)) or axes == 1 and ps[:-1] in ((), (b,)))):
            raise ValueError(f"positions must be contiguous int32 [{axes}][1 or {b}][{n}] (of one axis also [{b}][{n}] or "
                             f"[{n}]), got {positions.dtype} {ps}")
        pos_batch = ps[-2] if len(ps) > 1 else 1
    outs, tensors = [], b""
    for x, o, name in ((q, out_q, "q"),) if k is None else ((q, out_q, "q"), (k, out_k, "k")):
        xb, xh, xn, xd = x.shape if x.dim() == 4 else (0, 0, 0, 0)
        if xb != b or xn != n or xd != d or x.dtype != q.dtype:
            raise ValueError(f"{name} must be a {q.dtype} tensor [{b}][H][{n}][{d}], got {x.dtype} {tuple(x.shape)}")
        if o is None:
            o = x.new_empty((b, xh, n, d))
        elif o.dtype != x.dtype or o.shape != x.shape:
            raise ValueError(f"out_{name} must be {x.dtype} of shape {tuple(x.shape)}, got {o.dtype} {tuple(o.shape)}")
        (s0, s1, s2, s3), (t0, t1, t2, t3) = x.stride(), o.stride()
        if d > 1 and (s3 != 1 or t3 != 1):
            raise ValueError(f"{name} and its output must have contiguous rows (last stride 1)")
        outs.append(o)
        tensors += L.ROTARY_TENSOR.pack(x.data_ptr(), o.data_ptr(), xh, s0, s1, s2, t0, t1, t2)
    index = _one_device(q=q, k=k, inv_freq=inv_freq, positions=positions, out_q=out_q, out_k=out_k)
    params = L.ROTARY_PARAMS.pack(b, n, d, _DTYPE[q.dtype], _ROTARY_LAYOUT[layout], inv_freq.numel(), axes,
                                  *(axis + [0, 0])[:3], pos_batch, 1 if backward else 0, float(scale))
    _call_on(index, lib.wa_rotary, params, tensors, len(outs), _ptr(inv_freq), _ptr(positions))
    return outs[0] if k is None else tuple(outs)


def diff_shape_of(batch: int, heads: int, kv_heads: int, q_len: int, kv_len: int, head_dim: int, value_dim: int,
                  block: int = 128) -> L.WaDiffShape:
    return L.WaDiffShape(batch, heads, kv_heads, q_len, kv_len, head_dim, value_dim, block)


def diff_attn_workspace_size(shape: L.WaDiffShape) -> int:
    """Bytes for diff_attn with or without a mask, 0 in some shapes: results of tiles computed in parts, about 135 MB at most."""
    return _size("wa_diff_attn_workspace_size", shape)


def _diff_args(q, k, v, lam, mask, block, causal, q_start, kv_lens):
    """(shape, mask as uint8) of a differential-attention call; q [B][2H][M][d], k [B][2Hk][N][d], v [B][Hk][N][dv]."""
    for t, nm in ((q, "q"), (k, "k"), (v, "v")):
        if t.dtype != torch.bfloat16 or t.dim() != 4:
            raise ValueError(f"{nm} must be a bfloat16 tensor of four dimensions")
    b, h2, m, d = q.shape
    hk, n, dv = v.shape[1:]
    if h2 % 2 or hk == 0 or (h2 // 2) % hk:
        raise ValueError(f"q must have two maps for each of a multiple of v's {hk} heads, got {h2}")
    if tuple(k.shape) != (b, 2 * hk, n, d) or v.shape[0] != b:
        raise ValueError(f"k must have shape {(b, 2 * hk, n, d)} and v {(b, hk, n, dv)}, got {tuple(k.shape)} and "
                         f"{tuple(v.shape)}")
    h = h2 // 2
    _check(lam, "lam", torch.float32, (h,))
    _check(q_start, "q_start", torch.int32, (b,))
    _check(kv_lens, "kv_lens", torch.int32, (b,))
    if q_start is not None and not causal:
        raise ValueError("q_start without causal")
    if mask is not None:
        if mask.dtype not in (torch.bool, torch.uint8):
            raise ValueError("mask must be uint8 or bool")
        want = (b, h, -(-m // block), -(-n // block))
        if tuple(mask.shape) != want:
            raise ValueError(f"mask must have shape {want}, got {tuple(mask.shape)}")
        mask = mask.view(torch.uint8) if mask.dtype == torch.bool else mask
    return diff_shape_of(b, h, hk, m, n, d, dv, block), mask


def _diff_scale(scale: Optional[float]) -> float:
    """The C ABI's softmax_scale, whose 0 is the default."""
    if scale is None:
        return 0.0
    value = ctypes.c_float(scale).value
    if not 0.0 < value < math.inf:
        raise ValueError(f"scale must be positive and finite in float32 (None: 1 / sqrt(d)), got {scale}")
    return value


def diff_attn(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, lam: torch.Tensor, mask: Optional[torch.Tensor] = None,
              *, block: int = 128, scale: Optional[float] = None, causal: bool = False,
              q_start: Optional[torch.Tensor] = None, kv_lens: Optional[torch.Tensor] = None, return_stats: bool = False,
              out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Differential attention: O = P_1 V - lam_h P_2 V bf16 [B][H][M][dv], P_m = softmax(scale Q_m K_m^T) over the kept keys.

    q, k, v   bfloat16 [B][2H][M][d], [B][2Hk][N][d], [B][Hk][N][dv] with dv = d or 2 d; the maps of head h are
              2h and 2h + 1, and H / Hk heads in a row share keys and values
    lam       float32 [H]
    mask      uint8 or bool [B][H][ceil(M/block)][ceil(N/block)] of kept blocks; None keeps all
    scale     positive; None: 1 / sqrt(d)
    causal    query i of sequence b sees the keys up to q_start[b] + i (q_start int32 [B]; None: N - M); what lies behind
              the last query's is not used
    kv_lens   int32 [B]: keys each sequence holds; what lies behind them is not used, all before has to be finite
    return_stats  also (maps, stats), which diff_attn_backward takes: each P_m V int16 [B][2H][M][dv] in steps of 1/32767 of
              its row's largest magnitude, and float32 [B][2H][M][3]: the log-sum-exp of the scaled scores, the step, and a
              factor of roundings

    No autograd graph is recorded, also where an input requires a gradient: the caller makes the backward call."""
    lib = L.load()
    softmax_scale = _diff_scale(scale)
    shape, mask = _diff_args(q, k, v, lam, mask, block, causal, q_start, kv_lens)
    want = (shape.batch, shape.heads, shape.q_len, shape.value_dim)
    _check(out, "out", torch.bfloat16, want)
    _check(workspace, "workspace", torch.uint8)
    _on_device(q=q, k=k, v=v, lam=lam, mask=mask, q_start=q_start, kv_lens=kv_lens, out=out, workspace=workspace)
    index = _one_device(q=q, k=k, v=v, lam=lam, mask=mask, q_start=q_start, kv_lens=kv_lens, out=out, workspace=workspace)
    need = diff_attn_workspace_size(shape)
    if need and (workspace is None or workspace.numel() < need):
        workspace = _workspace(need, q.device)
    o = q.new_empty(want) if out is None else out
    rows = (want[0], 2 * want[1], want[2])
    maps = q.new_empty((*rows, want[3]), dtype=torch.int16) if return_stats else None
    stats = q.new_empty((*rows, 3), dtype=torch.float32) if return_stats else None
    opts = L.WaDiffOptions(softmax_scale, 1 if causal else 0)
    _call_on(index, lib.wa_diff_attn, _ptr(q), _ptr(k), _ptr(v), _ptr(lam), _ptr(mask), _ptr(q_start), _ptr(kv_lens),
             ctypes.byref(shape), ctypes.byref(opts), _ptr(o), _ptr(maps), _ptr(stats), _ptr(workspace),
             0 if workspace is None else workspace.numel())
    return (o, maps, stats) if return_stats else o


def diff_attn_backward_workspace_size(shape: L.WaDiffShape) -> int:
    return _size("wa_diff_attn_backward_workspace_size", shape)


def diff_attn_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, lam: torch.Tensor,
                       mask: Optional[torch.Tensor], maps: torch.Tensor, stats: torch.Tensor, *, block: int = 128,
                       scale: Optional[float] = None, causal: bool = False,
                       q_start: Optional[torch.Tensor] = None, kv_lens: Optional[torch.Tensor] = None,
                       workspace: Optional[torch.Tensor] = None):
    """(dq, dk, dv bf16, dlam float32) from dout, the gradient of diff_attn's O: the other arguments as that call had
    them, maps and stats as it returned them with return_stats. Keys past kv_lens, or behind every query, get 0. Equal calls give equal bits."""
    lib = L.load()
    softmax_scale = _diff_scale(scale)
    shape, mask = _diff_args(q, k, v, lam, mask, block, causal, q_start, kv_lens)
    want = (shape.batch, shape.heads, shape.q_len, shape.value_dim)
    rows = (want[0], 2 * want[1], want[2])
    _check(dout, "dout", torch.bfloat16, want)
    _check(maps, "maps", torch.int16, (*rows, want[3]))
    _check(stats, "stats", torch.float32, (*rows, 3))
    _check(workspace, "workspace", torch.uint8)
    given = dict(dout=dout, q=q, k=k, v=v, lam=lam, mask=mask, maps=maps, stats=stats, q_start=q_start,
                 kv_lens=kv_lens, workspace=workspace)
    _on_device(**given)
    index = _one_device(**given)
    need = diff_attn_backward_workspace_size(shape)
    if workspace is None or workspace.numel() < need:
        workspace = _workspace(need, q.device)
    dq, dk, dv, dlam = (torch.empty_like(t) for t in (q, k, v, lam))
    opts = L.WaDiffOptions(softmax_scale, 1 if causal else 0)
    _call_on(index, lib.wa_diff_attn_backward, _ptr(dout), _ptr(q), _ptr(k), _ptr(v), _ptr(lam), _ptr(maps),
             _ptr(stats), _ptr(mask), _ptr(q_start), _ptr(kv_lens), ctypes.byref(shape), ctypes.byref(opts), _ptr(dq),
             _ptr(dk), _ptr(dv), _ptr(dlam), _ptr(workspace), workspace.numel())
    return dq, dk, dv, dlam


_SEQ_DTYPE = {torch.bfloat16: L.WA_BF16, torch.float16: L.WA_F16}
_I32 = torch.int32


def _rows(t: torch.Tensor, name: str, dtype, shape) -> bytes:
    """wa_token_rows of a tensor [T][H][d] with free strides and whole rows."""
    if t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{name} must be {dtype} of shape {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    s0, s1, s2 = t.stride()
    if s2 != 1:
        raise ValueError(f"{name} must have contiguous rows (last stride 1)")
    return L.TOKEN_ROWS.pack(t.data_ptr(), s0, s1)


def _int32(t: Optional[torch.Tensor], name: str, shape) -> None:
    """A contiguous int32 tensor; a None in ``shape`` takes any size."""
    if t is None:
        return
    if t.dtype is _I32 and t.is_contiguous():
        size = t.shape
        if size == shape or len(size) == len(shape) and all(w is None or n == w for n, w in zip(size, shape)):
            return
    want = "".join("[any]" if w is None else f"[{w}]" for w in shape)
    raise ValueError(f"{name} must be contiguous int32 {want}, got {t.dtype} {tuple(t.shape)} of strides {t.stride()}")


def _index(**tensors) -> int:
    """As _one_device, in less time where there is nothing to refuse (2.9 -> 1.0 us of seven tensors)."""
    given = [t for t in tensors.values() if t is not None]
    index = given[0].get_device()
    for t in given:
        if t.get_device() != index or index < 0:
            return _one_device(**tensors)
    return index


def _seq_args(q: torch.Tensor, kv_heads: int, starts: torch.Tensor, name: str = "q"):
    """(wa_seq_shape, tokens, heads, head_dim) of a call whose rows of queries are q [T][H][d]."""
    size, dtype = q.shape, _SEQ_DTYPE.get(q.dtype)
    if len(size) != 3 or dtype is None:
        raise ValueError(f"{name} must be a bfloat16 or float16 [T][H][d] tensor, got {q.dtype} {tuple(size)}")
    if starts.dtype is not _I32 or starts.dim() != 1 or not starts.is_contiguous():
        _int32(starts, "starts", (None,))
    t, h, d = size
    return L.SEQ_SHAPE.pack(starts.shape[0] - 1, t, h, kv_heads, d, dtype), t, h, d


@functools.lru_cache(maxsize=1024)
def _seq_size(call: str, shape: bytes, *more) -> int:
    n = ctypes.c_size_t(0)
    L.check(getattr(L.load(), call)(shape, *more, ctypes.byref(n)))
    return n.value


def _lse_step(dtype, d: int) -> int:
    return 1 + d // 4 if dtype == torch.bfloat16 else 1


def _room(workspace: Optional[torch.Tensor], need: int, device) -> torch.Tensor:
    _check(workspace, "workspace", torch.uint8)
    return _workspace(need, device) if workspace is None or workspace.numel() < need else workspace


def packed_attn_workspace_size(tokens: int, batch: int, heads: int, kv_heads: int, head_dim: int, dtype=torch.bfloat16) -> int:
    """Bytes for packed_attn and paged_attn of ``batch`` sequences with ``tokens`` queries in all."""
    return _seq_size("wa_seq_attn_workspace_size", L.SEQ_SHAPE.pack(batch, tokens, heads, kv_heads, head_dim, _SEQ_DTYPE[dtype]))


def packed_attn_backward_workspace_size(tokens: int, batch: int, heads: int, kv_heads: int, head_dim: int) -> int:
    return _seq_size("wa_packed_attn_backward_workspace_size",
                     L.SEQ_SHAPE.pack(batch, tokens, heads, kv_heads, head_dim, L.WA_BF16))


def packed_attn(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, starts: torch.Tensor, *, causal: bool = True,
                scale: Optional[float] = None, return_lse: bool = False, out: Optional[torch.Tensor] = None,
                workspace: Optional[torch.Tensor] = None):
    """Attention over packed sequences: O = softmax(scale Q K^T) V [T][H][d], each sequence over its own tokens.

    q, k, v   bfloat16 or float16 [T][H][d], [T][Hk][d], [T][Hk][d], d 64 or 128, of any strides (multiples of 8) with whole
              rows: parts of one projection's output will do; H / Hk heads in a row share keys and values
    starts    int32 [B + 1], ascending: sequence b has the rows starts[b] to starts[b + 1] - 1 and may be empty
    causal    each query sees the keys up to its own
    scale     positive; None: 1 / sqrt(d)
    return_lse  also what packed_attn_backward takes: float32 [H][T][1 + d / 4] (float16, which has no gradient: [H][T][1]), of
              which [..., 0] are the log-sum-exps of the scaled scores and the others hold, as bytes, what O lost in rounding
    out       as q, of any strides; None: a new contiguous tensor. Rows of no sequence keep what they hold (in a new
              tensor and in the log-sum-exps: anything)

    A sequence's keys and values have to be finite. No autograd graph is recorded: the caller makes the backward call."""
    lib = L.load()
    softmax_scale = _diff_scale(scale)
    if len(k.shape) != 3:
        raise ValueError(f"k must have shape [T][Hk][d], got {tuple(k.shape)}")
    shape, t, h, d = _seq_args(q, k.shape[1], starts)
    o = q.new_empty((t, h, d)) if out is None else out
    kv = (t, k.shape[1], d)
    rows = (_rows(q, "q", q.dtype, q.shape), _rows(k, "k", q.dtype, kv), _rows(v, "v", q.dtype, kv))
    to = _rows(o, "out", q.dtype, q.shape)
    index = _index(q=q, k=k, v=v, starts=starts, out=out, workspace=workspace)
    need = _seq_size("wa_seq_attn_workspace_size", shape)
    workspace = _room(workspace, need, q.device)
    lse = q.new_empty((h, t, _lse_step(q.dtype, d)), dtype=torch.float32) if return_lse else None
    _call_on(index, lib.wa_packed_attn, *rows, starts.data_ptr(), shape, L.SEQ_OPTIONS.pack(softmax_scale, 1 if causal else 0), to,
             _ptr(lse), workspace.data_ptr(), workspace.numel())
    return (o, lse) if return_lse else o


def packed_attn_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor,
                         lse: torch.Tensor, starts: torch.Tensor, *, causal: bool = True, scale: Optional[float] = None,
                         out=None, workspace: Optional[torch.Tensor] = None):
    """(dq, dk, dv) from dout, the gradient of packed_attn's O: the other arguments as that call had them, o and lse as it
    returned them. bfloat16 only. out: (dq, dk, dv) tensors of any strides (parts of one tensor will do); rows of no sequence
    keep what they hold (in new tensors: anything). Equal calls give equal bits."""
    lib = L.load()
    softmax_scale = _diff_scale(scale)
    if len(k.shape) != 3:
        raise ValueError(f"k must have shape [T][Hk][d], got {tuple(k.shape)}")
    shape, t, h, d = _seq_args(q, k.shape[1], starts)
    kv = (t, k.shape[1], d)
    bf = torch.bfloat16
    rows = [_rows(x, n, bf, w) for x, n, w in ((dout, "dout", q.shape), (q, "q", q.shape), (k, "k", kv), (v, "v", kv), (o, "o", q.shape))]
    if lse.dtype != torch.float32 or lse.shape != (h, t, _lse_step(bf, d)) or not lse.is_contiguous():
        raise ValueError(f"lse must be contiguous float32 [{h}][{t}][{_lse_step(bf, d)}], got {lse.dtype} {tuple(lse.shape)}")
    if out is None:
        out = (q.new_empty(q.shape), q.new_empty(kv), q.new_empty(kv))
    dq, dk, dv = out
    to = (_rows(dq, "dq", bf, q.shape), _rows(dk, "dk", bf, kv), _rows(dv, "dv", bf, kv))
    index = _index(dout=dout, q=q, k=k, v=v, o=o, lse=lse, starts=starts, dq=dq, dk=dk, dv=dv, workspace=workspace)
    workspace = _room(workspace, _seq_size("wa_packed_attn_backward_workspace_size", shape), q.device)
    _call_on(index, lib.wa_packed_attn_backward, *rows, lse.data_ptr(), starts.data_ptr(), shape,
             L.SEQ_OPTIONS.pack(softmax_scale, 1 if causal else 0), *to, workspace.data_ptr(), workspace.numel())
    return dq, dk, dv


def _pages(t: torch.Tensor, name: str, dtype, kv_heads: int, d: int) -> bytes:
    """wa_pages of a tensor [pages][Hk][page][d] with free strides and whole rows."""
    size = t.shape
    if t.dtype != dtype or len(size) != 4 or size[1] != kv_heads or size[3] != d:
        raise ValueError(f"{name} must be {dtype} [pages][{kv_heads}][page][{d}], got {t.dtype} {tuple(size)}")
    s0, s1, s2, s3 = t.stride()
    if s3 != 1:
        raise ValueError(f"{name} must have contiguous rows (last stride 1)")
    return L.PAGES.pack(t.data_ptr(), s0, s1, s2)


def _page_tables(tables: torch.Tensor, kv_lens: torch.Tensor, batch: int, n_pages: int, page: int) -> bytes:
    size, stride = tables.shape, tables.stride()
    if tables.dtype is not _I32 or len(size) != 2 or size[0] != batch or (size[1] > 1 and stride[1] != 1):
        raise ValueError(f"tables must be int32 [{batch}][pages] with contiguous rows, got {tables.dtype} {tuple(size)}")
    _int32(kv_lens, "kv_lens", (batch,))
    return L.PAGE_TABLES.pack(tables.data_ptr(), stride[0] if batch > 1 else 0, size[1], n_pages, page)


def paged_attn(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, tables: torch.Tensor, starts: torch.Tensor,
               kv_lens: torch.Tensor, *, causal: bool = True, scale: Optional[float] = None, return_lse: bool = False,
               out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
               workspace: Optional[torch.Tensor] = None):
    """Attention of new tokens over a paged cache: O [T][H][d]. Sequence b's n = starts[b + 1] - starts[b] queries (one, a chunk
    of a prompt, none) are its last n of kv_lens[b] tokens, whose keys and values lie in the pages already (page_store).

    q         bfloat16 or float16 [T][H][d], d 64 or 128, of any strides (multiples of 8) with whole rows
    k_pages, v_pages  as q [pages][Hk][page][d], page a power of two from 16 to 4096, of any strides with whole rows: a pool of
              both, or a layer of one, will do
    tables    int32 [B][any]: token i of sequence b lies in row i % page of page tables[b][i // page]
    starts    int32 [B + 1], ascending; kv_lens int32 [B]: tokens of each sequence, the new ones counted
    causal    query i of n sees the keys up to kv_lens[b] - n + i; else all kv_lens[b]. One that sees none gets 0
    status    int32 [1], to which WA_PAGE_BAD_INDEX (1) is added if a table names a page that there is not: its keys are left out
    return_lse  also float32 [H][T], the log-sum-exps of the scaled scores
    scale, out  as for packed_attn

    What lies behind a sequence's last token is not used; all before has to be finite."""
    lib = L.load()
    softmax_scale = _diff_scale(scale)
    if k_pages.dim() != 4:
        raise ValueError(f"k_pages must have shape [pages][Hk][page][d], got {tuple(k_pages.shape)}")
    n_pages, hk, page, _ = k_pages.shape
    shape, t, h, d = _seq_args(q, hk, starts)
    o = q.new_empty((t, h, d)) if out is None else out
    if v_pages.shape != k_pages.shape:
        raise ValueError(f"v_pages must have k_pages' shape {tuple(k_pages.shape)}, got {tuple(v_pages.shape)}")
    args = (_rows(q, "q", q.dtype, q.shape), _pages(k_pages, "k_pages", q.dtype, hk, d), _pages(v_pages, "v_pages", q.dtype, hk, d),
            _page_tables(tables, kv_lens, starts.shape[0] - 1, n_pages, page))
    to = _rows(o, "out", q.dtype, q.shape)
    _int32(status, "status", (1,))
    index = _index(q=q, k_pages=k_pages, v_pages=v_pages, tables=tables, starts=starts, kv_lens=kv_lens, out=out,
                   status=status, workspace=workspace)
    workspace = _room(workspace, _seq_size("wa_seq_attn_workspace_size", shape), q.device)
    lse = q.new_empty((h, t), dtype=torch.float32) if return_lse else None
    _call_on(index, lib.wa_paged_attn, *args, starts.data_ptr(), kv_lens.data_ptr(), shape,
             L.SEQ_OPTIONS.pack(softmax_scale, 1 if causal else 0), to, _ptr(lse), _ptr(status), workspace.data_ptr(),
             workspace.numel())
    return (o, lse) if return_lse else o


def page_store(k: torch.Tensor, v: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, tables: torch.Tensor,
               starts: torch.Tensor, kv_lens: torch.Tensor, *, status: Optional[torch.Tensor] = None) -> None:
    """Puts keys and values of new tokens into their pages: rows starts[b] to starts[b + 1] - 1 of k and v [T][Hk][d] (any
    strides, whole rows) are the last tokens of sequence b's kv_lens[b]. Pages, tables and status as for paged_attn."""
    lib = L.load()
    if k_pages.dim() != 4:
        raise ValueError(f"k_pages must have shape [pages][Hk][page][d], got {tuple(k_pages.shape)}")
    n_pages, hk, page, d = k_pages.shape
    shape, t, _, _ = _seq_args(k, hk, starts, "k")
    if v_pages.shape != k_pages.shape:
        raise ValueError(f"v_pages must have k_pages' shape {tuple(k_pages.shape)}, got {tuple(v_pages.shape)}")
    args = (_rows(k, "k", k.dtype, (t, hk, d)), _rows(v, "v", k.dtype, (t, hk, d)), _pages(k_pages, "k_pages", k.dtype, hk, d),
            _pages(v_pages, "v_pages", k.dtype, hk, d), _page_tables(tables, kv_lens, starts.shape[0] - 1, n_pages, page))
    _int32(status, "status", (1,))
    index = _index(k=k, v=v, k_pages=k_pages, v_pages=v_pages, tables=tables, starts=starts, kv_lens=kv_lens, status=status)
    _call_on(index, lib.wa_page_store, *args, starts.data_ptr(), kv_lens.data_ptr(), shape, _ptr(status))


def _page_state(refs, tables, lens, page: int) -> bytes:
    _int32(refs, "refs", (None,))
    _int32(tables, "tables", (None, None))
    _int32(lens, "lens", (tables.shape[0],))
    return L.PAGE_STATE.pack(refs.data_ptr(), tables.data_ptr(), lens.data_ptr(), refs.numel(), tables.shape[0], tables.shape[1], page)


def _page_sizes(refs, tables, page: int) -> bytes:
    return L.PAGE_STATE.pack(0, 0, 0, refs.numel(), tables.shape[0], tables.shape[1], page)


def _page_pool(pool: torch.Tensor, n_pages: int) -> bytes:
    if pool.dim() < 3 or pool.shape[1] != n_pages or not pool.is_contiguous():
        raise ValueError(f"pool must be contiguous [planes][{n_pages}][...], got {tuple(pool.shape)}")
    size = pool.element_size()
    for n in pool.shape[2:]:
        size *= n
    return L.PAGE_POOL.pack(pool.data_ptr(), size, pool.shape[0])


def page_workspace_size(n_pages: int, sequences: int, table_width: int, *, page: int, entries: int = 0) -> int:
    """Bytes for page_grow and page_compact, and for page_fork of ``entries`` children."""
    return _seq_size("wa_page_workspace_size", L.PAGE_STATE.pack(0, 0, 0, n_pages, sequences, table_width, page), entries)


def page_grow(refs: torch.Tensor, tables: torch.Tensor, lens: torch.Tensor, new_lens: torch.Tensor, *, page: int,
              status: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> None:
    """Grows sequence s to max(lens[s], new_lens[s]) tokens, in place: the pages it needs are the lowest free ones, in
    the order of the sequences. One that finds too few, or no room in its table, keeps its length and adds WA_PAGE_EXHAUSTED (2).

    refs      int32 [pages]: how many sequences hold each page; 0: free
    tables    int32 [S][any]; sequence s holds the first ceil(lens[s] / page) pages of its row
    lens, new_lens   int32 [S]: tokens
    page      tokens a page, a power of two
    status    int32 [1], to which bits are added"""
    lib = L.load()
    state = _page_state(refs, tables, lens, page)
    _int32(new_lens, "new_lens", (tables.shape[0],))
    _int32(status, "status", (1,))
    index = _index(refs=refs, tables=tables, lens=lens, new_lens=new_lens, status=status, workspace=workspace)
    workspace = _room(workspace, _seq_size("wa_page_workspace_size", _page_sizes(refs, tables, page), 0), refs.device)
    _call_on(index, lib.wa_page_grow, state, new_lens.data_ptr(), _ptr(status), workspace.data_ptr(), workspace.numel())


def page_fork(pool: torch.Tensor, refs: torch.Tensor, tables: torch.Tensor, lens: torch.Tensor, parents: torch.Tensor,
              children: torch.Tensor, *, page: int, status: Optional[torch.Tensor] = None,
              workspace: Optional[torch.Tensor] = None) -> None:
    """Makes sequence children[i] a copy of parents[i], in place: full pages are shared, a last one that is not full is copied to
    the lowest free page. Children are empty before and named once (else left out, WA_PAGE_BUSY, 4); one without a free
    page stays empty (WA_PAGE_EXHAUSTED, 2).

    pool      [planes][pages][...] contiguous, any type: keys and values of every layer; pages are multiples of 16 bytes
    parents, children   int32 [n]; refs, tables, lens, page, status   as for page_grow"""
    lib = L.load()
    state, at = _page_state(refs, tables, lens, page), _page_pool(pool, refs.numel())
    _int32(parents, "parents", (None,))
    n = parents.numel()
    _int32(children, "children", (n,))
    _int32(status, "status", (1,))
    index = _index(pool=pool, refs=refs, tables=tables, lens=lens, parents=parents, children=children, status=status,
                   workspace=workspace)
    workspace = _room(workspace, _seq_size("wa_page_workspace_size", _page_sizes(refs, tables, page), n), refs.device)
    _call_on(index, lib.wa_page_fork, state, at, parents.data_ptr(), children.data_ptr(), n, _ptr(status), workspace.data_ptr(),
             workspace.numel())


def page_free(refs: torch.Tensor, tables: torch.Tensor, lens: torch.Tensor, slots: torch.Tensor, *, page: int,
              status: Optional[torch.Tensor] = None) -> None:
    """Gives the pages of the sequences slots (int32 [n]) back, in place: refs go down, lens to 0; tables and contents stay."""
    lib = L.load()
    state = _page_state(refs, tables, lens, page)
    _int32(slots, "slots", (None,))
    _int32(status, "status", (1,))
    index = _index(refs=refs, tables=tables, lens=lens, slots=slots, status=status)
    _call_on(index, lib.wa_page_free, state, slots.data_ptr(), slots.numel(), _ptr(status))


def page_compact(pool: torch.Tensor, refs: torch.Tensor, tables: torch.Tensor, lens: torch.Tensor, *, page: int,
                 out_refs: Optional[torch.Tensor] = None, out_tables: Optional[torch.Tensor] = None,
                 used: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None) -> None:
    """Moves the pages in use to the front of the pool: of u in use those numbered u and above go, in order, to the free ones
    below u. out_refs and out_tables take the new state (None: in place); with their own, calls in flight may go on with the
    old one, since what a page held stays where it was until the page is dealt out again. used: int32 [1], u."""
    lib = L.load()
    state, at = _page_state(refs, tables, lens, page), _page_pool(pool, refs.numel())
    _int32(out_refs, "out_refs", refs.shape)
    _int32(out_tables, "out_tables", tables.shape)
    _int32(used, "used", (1,))
    _int32(status, "status", (1,))
    index = _index(pool=pool, refs=refs, tables=tables, lens=lens, out_refs=out_refs, out_tables=out_tables, used=used,
                   status=status, workspace=workspace)
    workspace = _room(workspace, _seq_size("wa_page_workspace_size", _page_sizes(refs, tables, page), 0), refs.device)
    _call_on(index, lib.wa_page_compact, state, at, _ptr(refs if out_refs is None else out_refs),
             _ptr(tables if out_tables is None else out_tables), _ptr(used), _ptr(status), workspace.data_ptr(), workspace.numel())


def page_copy(pool: torch.Tensor, source: torch.Tensor, target: torch.Tensor, *, status: Optional[torch.Tensor] = None) -> None:
    """Copies page source[i] to page target[i] (int32 [n]) in every plane of the pool; no page is both, or a target twice."""
    lib = L.load()
    at = _page_pool(pool, pool.shape[1] if pool.dim() > 1 else 0)
    _int32(source, "source", (None,))
    _int32(target, "target", (source.numel(),))
    _int32(status, "status", (1,))
    index = _index(pool=pool, source=source, target=target, status=status)
    _call_on(index, lib.wa_page_copy, at, pool.shape[1], source.data_ptr(), target.data_ptr(), source.numel(), _ptr(status))


def fp64_probe(a: torch.Tensor, b: torch.Tensor, c: torch.Tensor) -> torch.Tensor:
    lib = L.load()
    out = torch.empty((a.numel(), 6), dtype=torch.float64, device=a.device)
    L.check(lib.wa_fp64_probe(_ptr(a), _ptr(b), _ptr(c), _ptr(out), a.numel(), _stream()))
    return out


def xcc_probe(n_wg: int, device="cuda") -> torch.Tensor:
    lib = L.load()
    out = torch.full((n_wg,), -1, dtype=torch.int32, device=device)
    L.check(lib.wa_xcc_probe(_ptr(out), int(n_wg), _stream()))
    return out


def default_scale(head_dim: int) -> float:
    return 1.0 / math.sqrt(head_dim)
