"""Verification of drafted tokens against the target's logits (include/dlm.h).

The rule runs in libdlm.so's HIP kernels; nothing here waits for the device.
"""

from __future__ import annotations

from typing import NamedTuple

import torch

from . import _lib
from .cache import _DTYPES, _ints, _launch


class Verified(NamedTuple):
    """next int32 [n_seqs]: the token drawn after the kept ones (-1: none); keep int32 [rows]
    and keep_start int32 [n_seqs + 1]: the window rows kept, as PagedCache.commit takes them
    (-1 behind them)."""
    next: torch.Tensor
    keep: torch.Tensor
    keep_start: torch.Tensor


def _logits(t: torch.Tensor, name: str, rows: int, device: torch.device) -> int:
    """Elements from row to row of t [rows, vocab]."""
    if t.dim() != 2 or t.shape[0] != rows or t.dtype not in _DTYPES or t.device != device or t.shape[1] < 1:
        raise ValueError(f"{name} must be a bfloat16, float16 or float32 tensor [{rows}, vocab] on {device}")
    row, one = t.stride()
    if t.shape[1] > 1 and one != 1:
        raise ValueError(f"the logits of a row of {name} must lie next to each other")
    return row if rows > 1 else t.shape[1]


def _floats(t: torch.Tensor, name: str, n: int, device: torch.device) -> int:
    if t.dtype is not torch.float32 or t.device != device or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous float32 tensor of {n} values on {device}")
    return t.data_ptr()


def verify(row_start: torch.Tensor, tokens: torch.Tensor, target: torch.Tensor, u: torch.Tensor, u_next: torch.Tensor,
           parent: torch.Tensor | None = None, draft: torch.Tensor | None = None, temperature: float = 1.0,
           max_rows: int | None = None) -> Verified:
    """Which drafted tokens the target keeps, and the token after them.

    Windows of rows are packed (row_start int32 [n_seqs + 1]); row 0 of a window is the
    token drawn last, the others are drafted below it: row i below row parent[..] of its
    window (int32 [rows], an earlier one; None: row i - 1).  tokens int32 [rows]; target
    [rows, vocab]: the target's logits after each row; draft: those that each row's child
    was drawn from (chains only), None for drafted tokens that are certain.  u float32
    [rows], u_next float32 [n_seqs]: random numbers in [0, 1), one per drafted token and one
    per sequence.  temperature divides the logits (1e-30 to 1e30; 0: the largest decides).  max_rows: rows
    of the longest window (default and at most 1024).  No gradient passes through it.
    """
    lib, device = _lib.load(), target.device
    if device.type != "cuda":
        raise ValueError("target must be a device tensor")
    rows, n_seqs = tokens.numel(), row_start.numel() - 1
    starts, toks = _ints(row_start, "row_start", None, device), _ints(tokens, "tokens", rows, device)
    stride = _logits(target, "target", rows, device)
    vocab = target.shape[1]
    up = _ints(parent, "parent", rows, device)
    draft_ptr, draft_stride = None, 0
    if draft is not None:
        draft_stride = _logits(draft, "draft", rows, device)
        if draft.shape != target.shape or draft.dtype is not target.dtype:
            raise ValueError("draft must have target's shape and type")
        draft_ptr = draft.data_ptr() if rows else None
    up_ptr = up if rows else None
    u_ptr, u_next_ptr = _floats(u, "u", rows, device), _floats(u_next, "u_next", n_seqs, device)
    n = lib.dlm_verify_workspace_bytes(n_seqs, rows, vocab, 0 if draft is None else 1)
    if n == 0:
        raise ValueError(f"invalid sizes: {n_seqs} sequences, {rows} rows of {vocab} logits")
    ws = row_start.new_empty((n + 3) // 4)
    out = row_start.new_empty(2 * n_seqs + 1 + rows)
    nxt, keep_start, keep = out[:n_seqs], out[n_seqs:2 * n_seqs + 1], out[2 * n_seqs + 1:]
    _launch(lib.dlm_verify, "dlm_verify", device.index, n_seqs, starts, rows,
            min(1024, rows) if max_rows is None else int(max_rows), toks, up_ptr, _DTYPES[target.dtype], vocab,
            target.data_ptr(), stride, draft_ptr, draft_stride, temperature, u_ptr, u_next_ptr, nxt.data_ptr(),
            keep.data_ptr(), keep_start.data_ptr(), ws.data_ptr(), n)
    return Verified(nxt, keep, keep_start)
