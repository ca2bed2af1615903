"""Rotary positions and a paged key/value cache (include/dlm.h).

PyTorch supplies device memory and the stream; every operation runs in
libdlm.so's HIP kernels through the C ABI.  Nothing here waits for the device.
"""

from __future__ import annotations

import ctypes

import torch
from torch.autograd import forward_ad

from . import _lib
from ._lib import DlmCache, DlmNormGrads, DlmNormHeads, DlmRope, DlmRopeSpec, check

_DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
_SCALINGS = {None: 0, "linear": 1, "ntk": 2, "yarn": 3}


# A call is a few microseconds of work on the device: what happens on the host is
# kept to what checks and passes on the arguments.
_raw_stream = torch._C._cuda_getCurrentRawStream      # (device index) -> hipStream_t
_current_device = torch._C._cuda_getDevice


def _launch(fn, name: str, index: int, *args):
    """fn(*args, stream) with device `index` current; its refusals raise."""
    if _current_device() == index:
        status = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            status = fn(*args, _raw_stream(index))
    if status:
        check(status, name)


def _ints(t: torch.Tensor | None, name: str, n: int | None, device: torch.device) -> int | None:
    """Address of t, a contiguous int32 tensor of n elements on the device."""
    if t is None:
        return None
    if t.dtype is not torch.int32 or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor on {device}")
    if n is not None and t.numel() != n:
        raise ValueError(f"{name} must hold {n} values, has {t.numel()}")
    return t.data_ptr()


def _rows(t: torch.Tensor, name: str, heads: int | None, head_dim: int, device: torch.device):
    """(rows, heads, elements from row to row) of t [rows, heads, head_dim], whose heads
    lie next to each other."""
    shape = t.shape
    if len(shape) != 3 or shape[2] != head_dim or (heads is not None and shape[1] != heads) or t.device != device:
        raise ValueError(f"{name} must be [rows, {heads if heads is not None else 'heads'}, {head_dim}] on {device}, "
                         f"is {tuple(shape)} on {t.device}")
    n, h, _ = shape
    row, head, one = t.stride()
    if one != 1 or (h > 1 and head != head_dim):
        raise ValueError(f"the heads of {name} must lie next to each other")
    return n, h, row if n > 1 else h * head_dim           # a single row has any stride


def _mask_words(mask: torch.Tensor, rows: int) -> int:
    """Words per row of a mask; one of no words would have no address, which stands for
    no mask."""
    if mask.dim() != 2 or mask.shape[0] != rows or (rows and mask.shape[1] == 0):
        raise ValueError(f"mask must be int32 [{rows}, words] with at least one word")
    return mask.shape[1]


def _gain(t: torch.Tensor | None, name: str, head_dim: int, dtype: torch.dtype, device: torch.device):
    """(address, type) of a gain [head_dim] of the rows' type or float32."""
    if t is None:
        return None, _DTYPES[dtype]
    if t.shape != (head_dim,) or t.dtype not in (dtype, torch.float32) or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous tensor [{head_dim}] of type {dtype} or float32 on {device}")
    return t.data_ptr(), _DTYPES[t.dtype]


def _no_tangents(*tensors: torch.Tensor | None):
    """Refuse dual tensors of forward-mode differentiation: a kernel reads their values alone,
    and the result would say that its derivative is zero."""
    if forward_ad._current_level >= 0:                    # else nothing carries a tangent
        for t in tensors:
            if t is not None and forward_ad.unpack_dual(t).tangent is not None:
                raise ValueError("no forward-mode derivative (tangent) passes through a rotation")


class Rope:
    """Frequencies of rotary positions; a plain host structure, no device memory.

    head_dim values per head of which the first rot_dim (default all) are
    rotated, in pairs (i, i + rot_dim / 2) or, interleaved, (2 i, 2 i + 1).
    scaling: None, "linear", "ntk" or "yarn" for contexts `factor` times as long
    ("yarn": as original_len); scale: factor on the rotated values (0: the
    scaling's own).
    """

    def __init__(self, head_dim: int, rot_dim: int | None = None, theta: float = 10000.0, interleaved: bool = False,
                 scaling: str | None = None, factor: float = 1.0, original_len: int = 0, beta_slow: float = 1.0,
                 beta_fast: float = 32.0, scale: float = 0.0):
        if scaling not in _SCALINGS:
            raise ValueError(f"scaling must be one of {sorted(k for k in _SCALINGS if k)} or None")
        self.lib = _lib.load()
        spec = DlmRopeSpec(int(head_dim), int(head_dim if rot_dim is None else rot_dim), int(bool(interleaved)),
                           _SCALINGS[scaling], int(original_len), float(scale), float(theta), float(factor),
                           float(beta_slow), float(beta_fast))
        self.c = DlmRope()
        check(self.lib.dlm_rope_init(ctypes.byref(spec), ctypes.byref(self.c)), "dlm_rope_init")
        self._ref = ctypes.byref(self.c)
        self._head_dim = int(self.c.head_dim)

    @property
    def head_dim(self) -> int:
        return self._head_dim

    def apply(self, x: torch.Tensor, positions: torch.Tensor, out: torch.Tensor | None = None,
              transpose: bool = False) -> torch.Tensor:
        """x [rows, heads, head_dim] (any row and head strides) rotated to `positions`
        (int32 [rows]); into `out` (may be x).  transpose: the gradient with respect
        to x, given the gradient x of a rotation's result; autograd takes it by itself
        where x requires a gradient (`out` cannot be part of that; tangents of forward-mode
        differentiation are refused)."""
        _no_tangents(x, out)
        if torch.is_grad_enabled() and (x.requires_grad or (out is not None and out.requires_grad)):
            if out is not None:
                raise ValueError("a result in `out` carries no gradient: detach x and out, or leave out away")
            return _Rotation.apply(x, positions, self, transpose)
        return self._apply(x, positions, out, transpose)

    def _apply(self, x: torch.Tensor, positions: torch.Tensor, out: torch.Tensor | None, transpose: bool) -> torch.Tensor:
        shape, kind, device = x.shape, _DTYPES.get(x.dtype), x.device
        if len(shape) != 3 or shape[2] != self._head_dim or kind is None or device.type != "cuda":
            raise ValueError(f"x must be a bfloat16, float16 or float32 device tensor [rows, heads, {self._head_dim}]")
        if out is None:
            out = torch.empty(shape, dtype=x.dtype, device=device)
        elif out.shape != shape or out.dtype is not x.dtype or out.device != device:
            raise ValueError("out must have x's shape, type and device")
        xs, ys = x.stride(), out.stride()
        if xs[2] != 1 or ys[2] != 1:
            raise ValueError("the values of a head must lie next to each other")
        pos = _ints(positions, "positions", shape[0], device)
        _launch(self.lib.dlm_rope_apply, "dlm_rope_apply", device.index, self._ref, kind, shape[0], shape[1],
                x.data_ptr(), xs[0], xs[1], out.data_ptr(), ys[0], ys[1], pos, 1 if transpose else 0)
        return out


    # -------------------------------------------------------------- norms of heads
    def norm_apply(self, q: torch.Tensor, k: torch.Tensor | None, positions: torch.Tensor,
                   q_gain: torch.Tensor | None = None, k_gain: torch.Tensor | None = None, eps: float = 1e-6,
                   out: torch.Tensor | None = None, k_out: torch.Tensor | None = None):
        """Queries and keys [rows, heads, head_dim] (any row and head strides, each its own
        number of heads), each head over the root of its mean square, times its gain
        [head_dim] (their type or float32; None: ones), rotated to `positions`, in one
        launch: (queries, keys).  k None: queries alone.  out, k_out: results of queries and
        keys (may be q and k).  Gradients of q, k and the gains come by autograd (`out` and
        `k_out` cannot be part of that, nor a gradient of the gradient; tangents of forward-mode
        differentiation are refused)."""
        _no_tangents(q, k, q_gain, k_gain, out, k_out)
        given = [t for t in (out, k_out) if t is not None]
        if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (q, k, q_gain, k_gain, *given)):
            if given:
                raise ValueError("a result in `out` carries no gradient: detach the inputs and out, or leave out away")
            return _NormRotation.apply(q, k, positions, q_gain, k_gain, self, eps)
        return self._norm_apply(q, k, positions, q_gain, k_gain, eps, out, k_out)

    def _norm_set(self, x: torch.Tensor | None, gain: torch.Tensor | None, like: torch.Tensor, name: str) -> DlmNormHeads:
        """Rows, gain and type of a set of heads, its results still open."""
        if x is None:
            if gain is not None:
                raise ValueError(f"{name}_gain without {name}")
            return DlmNormHeads()
        shape = x.shape
        if len(shape) != 3 or shape[2] != self._head_dim or x.dtype not in _DTYPES or x.device.type != "cuda":
            raise ValueError(f"{name} must be a bfloat16, float16 or float32 device tensor [rows, heads, {self._head_dim}]")
        if x.dtype is not like.dtype or x.device != like.device or shape[0] != like.shape[0]:
            raise ValueError("q and k must have the same rows, type and device")
        row, head, one = x.stride()
        if one != 1:
            raise ValueError("the values of a head must lie next to each other")
        g, kind = _gain(gain, f"{name}_gain", self._head_dim, x.dtype, x.device)
        return DlmNormHeads(shape[1], kind, g, x.data_ptr(), row, head)

    def _norm_apply(self, q, k, positions, q_gain, k_gain, eps, out, k_out):
        sets = [self._norm_set(q, q_gain, q, "q"), self._norm_set(k, k_gain, q, "k")]
        if k is None and k_out is not None:
            raise ValueError("k_out without k")
        results = []
        for c, x, y, name in ((sets[0], q, out, "out"), (sets[1], k, k_out, "k_out")):
            if x is not None:
                if y is None:
                    y = torch.empty_like(x, memory_format=torch.contiguous_format)
                elif y.shape != x.shape or y.dtype is not x.dtype or y.device != x.device or y.stride(2) != 1:
                    raise ValueError(f"{name} must have its input's shape, type and device, a head's values next to each other")
                c.d_y = y.data_ptr()
                c.y_row_stride, c.y_head_stride = y.stride(0), y.stride(1)
            results.append(y)
        pos = _ints(positions, "positions", q.shape[0], q.device)
        _launch(self.lib.dlm_rope_norm, "dlm_rope_norm", q.device.index, self._ref, _DTYPES[q.dtype], q.shape[0],
                ctypes.byref(sets[0]), ctypes.byref(sets[1]), eps, pos)
        return tuple(results)

    def _norm_grad(self, q, k, positions, q_gain, k_gain, eps, dq, dk, needs):
        """Gradients of (q, k, q_gain, k_gain), given those of the results (None: none);
        needs: which are asked for."""
        device, kind = q.device, q.dtype
        rows, sets, grads, got = q.shape[0], [], [], []
        for x, gain, dy, name, need in ((q, q_gain, dq, "q", needs[2]), (k, k_gain, dk, "k", needs[3])):
            if x is None or dy is None:
                sets.append(DlmNormHeads())
                grads.append(DlmNormGrads())
                got.append((None, None))
                continue
            if dy.stride(2) != 1:                     # a head's values lie next to each other
                dy = dy.clone(memory_format=torch.contiguous_format)
            sets.append(self._norm_set(x, gain, q, name))
            dx = torch.empty_like(x, memory_format=torch.contiguous_format)
            dg = torch.empty_like(gain) if gain is not None and need else None
            grads.append(DlmNormGrads(dy.data_ptr(), dy.stride(0), dy.stride(1), dx.data_ptr(), dx.stride(0), dx.stride(1),
                                      None if dg is None else dg.data_ptr()))
            got.append((dx, dg, dy))
        n = self.lib.dlm_rope_norm_grad_workspace_bytes(self._ref)
        ws = positions.new_empty(n // 4)
        _launch(self.lib.dlm_rope_norm_grad, "dlm_rope_norm_grad", device.index, self._ref, _DTYPES[kind], rows,
                ctypes.byref(sets[0]), ctypes.byref(sets[1]), ctypes.byref(grads[0]), ctypes.byref(grads[1]), eps,
                positions.data_ptr(), ws.data_ptr(), n)
        return got[0][0], got[1][0], got[0][1], got[1][1]


class _NormRotation(torch.autograd.Function):
    """Norms of heads, then a rotation."""

    @staticmethod
    def forward(ctx, q, k, positions, q_gain, k_gain, rope, eps):
        ctx.save_for_backward(q, k, positions, q_gain, k_gain)
        ctx.rope, ctx.eps = rope, eps
        ctx.set_materialize_grads(False)
        return rope._norm_apply(q, k, positions, q_gain, k_gain, eps, None, None)

    @staticmethod
    def backward(ctx, dq, dk):
        if torch.is_grad_enabled():                   # create_graph: a gradient of it is refused
            return _NormRotation._final(ctx, dq, dk)
        return _NormRotation._gradients(ctx, dq, dk)

    @staticmethod
    def _gradients(ctx, dq, dk):
        q, k, positions, q_gain, k_gain = ctx.saved_tensors
        if dq is None and dk is None:
            return (None,) * 7
        _no_tangents(dq, dk)
        need = ctx.needs_input_grad
        gq, gk, gqg, gkg = ctx.rope._norm_grad(q, k, positions, q_gain, k_gain, ctx.eps, dq, dk,
                                               (need[0], need[1], need[3], need[4]))
        return gq, gk, None, gqg, gkg, None, None

    _final = staticmethod(torch.autograd.function.once_differentiable(lambda *a: _NormRotation._gradients(*a)))


class _Rotation(torch.autograd.Function):
    """A rotation is linear in x: its gradient is the rotation back, times the scale."""

    @staticmethod
    def forward(ctx, x, positions, rope, transpose):
        ctx.save_for_backward(positions)
        ctx.rope, ctx.transpose = rope, transpose
        return rope._apply(x, positions, None, transpose)

    @staticmethod
    def backward(ctx, grad):
        if grad.stride(-1) != 1:                      # a head's values lie next to each other
            grad = grad.clone(memory_format=torch.contiguous_format)
        return ctx.rope.apply(grad, ctx.saved_tensors[0], transpose=not ctx.transpose), None, None, None


class Share:
    """What groups of sequences have in common (PagedCache.share), for the attention of one
    pass."""

    __slots__ = ("cache", "epoch", "rows", "max_rows", "max_group_rows", "data")

    def __init__(self, cache: "PagedCache", rows: int, max_rows: int, max_group_rows: int, data: torch.Tensor):
        self.cache, self.epoch, self.data = cache, cache._epoch, data
        self.rows, self.max_rows, self.max_group_rows = rows, max_rows, max_group_rows


class PagedCache:
    """A paged key/value cache: n_pages pages of page_len tokens in n_layers layers,
    shared by n_seqs sequences of up to max_pages pages.

    k, v: [n_layers, n_pages, n_kv_heads, page_len, head_dim], allocated here
    unless given.  meta (int32) holds ref [n_pages], len [n_seqs] and table
    [n_seqs, max_pages], which are views of it.  Windows of rows are packed:
    row_start int32 [n_seqs + 1] on the device.  Calls on one cache share its
    workspaces: order them on one stream.  It serves: no gradient passes through
    append and attend.
    """

    def __init__(self, n_layers: int, n_pages: int, page_len: int, n_kv_heads: int, head_dim: int, n_seqs: int,
                 max_pages: int, dtype: torch.dtype = torch.bfloat16, device: str | torch.device = "cuda",
                 k: torch.Tensor | None = None, v: torch.Tensor | None = None):
        self.lib = _lib.load()
        device = torch.device(device)
        if device.type != "cuda":
            raise ValueError("a cache lives on a GPU")
        if device.index is None:
            device = torch.device("cuda", torch.cuda.current_device())
        self.device = device
        if dtype not in (torch.bfloat16, torch.float16):
            raise ValueError("dtype must be torch.bfloat16 or torch.float16")
        shape = (n_layers, n_pages, n_kv_heads, page_len, head_dim)
        c = DlmCache(_DTYPES[dtype], *(int(x) for x in (n_layers, n_pages, page_len, n_kv_heads, head_dim, n_seqs,
                                                        max_pages)))
        if self.lib.dlm_cache_workspace_bytes(ctypes.byref(c), 0, 0, 0) == 0:
            raise ValueError(f"invalid cache shape {shape}, {n_seqs} sequences of {max_pages} pages")
        for t, name in ((k, "k"), (v, "v")):
            if t is not None and (tuple(t.shape) != shape or t.dtype != dtype or t.device != device
                                  or not t.is_contiguous()):
                raise ValueError(f"{name} must be a contiguous {dtype} tensor {shape} on {device}")
        self.dtype = dtype
        self.k = torch.empty(shape, dtype=dtype, device=device) if k is None else k
        self.v = torch.empty(shape, dtype=dtype, device=device) if v is None else v
        self.meta = torch.empty(n_pages + n_seqs + n_seqs * max_pages, dtype=torch.int32, device=device)
        self.ref = self.meta[:n_pages]
        self.len = self.meta[n_pages:n_pages + n_seqs]
        self.table = self.meta[n_pages + n_seqs:].view(n_seqs, max_pages)
        c.d_k, c.d_v = self.k.data_ptr(), self.v.data_ptr()
        c.d_ref, c.d_len, c.d_table = self.ref.data_ptr(), self.len.data_ptr(), self.table.data_ptr()
        self.c = c
        self._ref = ctypes.byref(c)
        self._n_seqs, self._kv, self._hd, self._kind = int(n_seqs), int(n_kv_heads), int(head_dim), _DTYPES[dtype]
        self._ws, self._by_size = {}, {}
        self._epoch = 0                                   # of lengths and tables
        self.reset()

    # -------------------------------------------------------------- plumbing
    @property
    def n_seqs(self) -> int:
        return self._n_seqs

    def workspace(self, total_rows: int = 0, max_rows: int = 0, n_heads: int = 0) -> torch.Tensor:
        """Workspace of calls with these sizes; kept, so that captured graphs stay valid."""
        return self._workspace((total_rows, max_rows, n_heads), self.lib.dlm_cache_workspace_bytes)

    def _workspace(self, key: tuple, size, rounded: bool = False) -> torch.Tensor:
        """rounded: sizes that follow the rows go up to powers of two, so that all of them
        together stay below four times the largest need."""
        ws = self._ws.get(key)
        if ws is None:
            n = size(self._ref, *key)
            if n == 0:
                raise ValueError(f"invalid sizes: {key[0]} rows, {key[1]} at most, {key[-1]} heads")
            if rounded:
                n = 1 << (n - 1).bit_length()
            ws = self._by_size.get(n)
            if ws is None:
                ws = self._by_size[n] = torch.empty(n, dtype=torch.uint8, device=self.device)
            self._ws[key] = ws
        return ws

    def _call(self, name: str, *args):
        _launch(getattr(self.lib, name), name, self.device.index, self._ref, *args)

    def _change(self, name: str, *args):
        """A call that changes lengths or tables."""
        self._epoch += 1
        self._call(name, *args)

    def _starts(self, row_start: torch.Tensor) -> int:
        return _ints(row_start, "row_start", self._n_seqs + 1, self.device)

    # -------------------------------------------------------------- pages
    def reset(self):
        """Empty every sequence, free every page."""
        self._change("dlm_cache_reset")

    def reserve(self, row_start: torch.Tensor, total_rows: int | None = None) -> torch.Tensor:
        """Room for the windows' rows; ok int32 [n_seqs].  total_rows: rows that count
        (default: no bound but row_start's own)."""
        starts = self._starts(row_start)
        ok = torch.empty(self._n_seqs, dtype=torch.int32, device=self.device)
        ws = self.workspace()
        self._change("dlm_cache_reserve", starts, 1 << 24 if total_rows is None else int(total_rows), ok.data_ptr(),
                   ws.data_ptr(), ws.numel())
        return ok

    def commit(self, row_start: torch.Tensor, keep: torch.Tensor | None = None, keep_start: torch.Tensor | None = None,
               total_rows: int | None = None) -> torch.Tensor:
        """The kept rows of each window (default all) become its sequence's next tokens;
        ok int32 [n_seqs]."""
        starts = self._starts(row_start)
        kept = _ints(keep, "keep", None, self.device)
        kept_start = _ints(keep_start, "keep_start", self._n_seqs + 1, self.device)
        ok = torch.empty(self._n_seqs, dtype=torch.int32, device=self.device)
        n_keep = 0 if keep is None else keep.numel()
        if keep is not None and n_keep == 0:
            kept = starts                                 # an empty list has no address; nothing of it is read
        self._change("dlm_cache_commit", starts, 1 << 24 if total_rows is None else int(total_rows), kept, kept_start,
                   n_keep, ok.data_ptr())
        return ok

    def fork(self, src: torch.Tensor, dst: torch.Tensor) -> torch.Tensor:
        """Sequences dst become copies of src that share their pages; ok int32 [pairs]."""
        n = src.numel()
        a, b = _ints(src, "src", None, self.device), _ints(dst, "dst", n, self.device)
        ok = torch.empty(n, dtype=torch.int32, device=self.device)
        self._change("dlm_cache_fork", n, a, b, ok.data_ptr())
        return ok

    def truncate(self, new_len: torch.Tensor | None = None):
        """Keep at most new_len[s] tokens of sequence s (negative: leave it; None: 0 for all)."""
        self._change("dlm_cache_truncate", _ints(new_len, "new_len", self._n_seqs, self.device))

    def compact(self) -> torch.Tensor:
        """Move the pages in use to the lowest ids; int32 [1], how many there are."""
        used = torch.empty(1, dtype=torch.int32, device=self.device)
        ws = self.workspace()
        self._change("dlm_cache_compact", used.data_ptr(), ws.data_ptr(), ws.numel())
        return used

    # -------------------------------------------------------------- windows
    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor, row_start: torch.Tensor, max_rows: int,
               q: torch.Tensor | None = None, rope: Rope | None = None, positions: torch.Tensor | None = None,
               q_out: torch.Tensor | None = None, q_gain: torch.Tensor | None = None,
               k_gain: torch.Tensor | None = None, norm_eps: float | None = None) -> torch.Tensor | None:
        """Keys and values [rows, n_kv_heads, head_dim] of the windows into their reserved
        places; keys and queries rotated by `rope` to `positions` (default: the tokens'
        places).  Returns the rotated queries (in q_out if given).  norm_eps: keys and
        queries are normalised first, each head over the root of its mean square and times
        its gain [head_dim] (both of k's type or both float32; None: ones)."""
        device, kind = self.device, k.dtype
        starts = self._starts(row_start)
        T, _, ks = _rows(k, "k", self._kv, self._hd, device)
        Tv, _, vs = _rows(v, "v", self._kv, self._hd, device)
        if Tv != T or v.dtype is not kind or kind not in _DTYPES:
            raise ValueError("k and v must have the same rows and a floating type of 16 or 32 bits")
        pos = _ints(positions, "positions", T, device)
        heads = qs = qos = 0
        qp = qop = None
        if q is not None:
            Tq, heads, qs = _rows(q, "q", None, self._hd, device)
            if Tq != T or q.dtype is not kind:
                raise ValueError("q must have the rows and the type of k")
            if q_out is None:
                q_out = torch.empty(q.shape, dtype=self.dtype, device=device)
            To, _, qos = _rows(q_out, "q_out", heads, self._hd, device)
            if To != T or q_out.dtype is not self.dtype:
                raise ValueError("q_out must have q's rows and the cache's type")
            qp, qop = q.data_ptr(), q_out.data_ptr()
        call = (layer, starts, T, max_rows, _DTYPES[kind], k.data_ptr(), ks, v.data_ptr(), vs,
                None if rope is None else rope._ref, pos, heads, qp, qs, qop, qos)
        if norm_eps is None:
            if q_gain is not None or k_gain is not None:
                raise ValueError("gains without norm_eps")
            if T:
                self._call("dlm_cache_append", *call)
            return q_out
        qg, q_type = _gain(q_gain, "q_gain", self._hd, kind, device)
        kg, k_type = _gain(k_gain, "k_gain", self._hd, kind, device)
        if q_gain is not None and k_gain is not None and q_type != k_type:
            raise ValueError("q_gain and k_gain must have the same type")
        if T:
            self._call("dlm_cache_append_norm", *call, q_type if q_gain is not None else k_type, qg, kg, norm_eps)
        return q_out

    def share(self, row_start: torch.Tensor, groups: torch.Tensor, rows: int, max_rows: int,
              max_group_rows: int | None = None) -> Share:
        """What groups of sequences (int32 [n_seqs], a number per sequence in [0, n_seqs);
        others: by itself) have in common at the front of their tables, for attend in every
        layer of a pass: rows in all, at most max_rows of a sequence and max_group_rows of a
        group (default: all).  It stands until lengths or tables change (a group with more
        rows than it says shares nothing)."""
        starts = self._starts(row_start)
        group = _ints(groups, "groups", self._n_seqs, self.device)
        rows, max_rows = int(rows), int(max_rows)
        most = rows if max_group_rows is None else int(max_group_rows)
        n = self.lib.dlm_cache_share_bytes(self._ref, rows)
        if n == 0:
            raise ValueError(f"invalid number of rows: {rows}")
        data = groups.new_empty(n // 4)
        self._call("dlm_cache_share", starts, rows, max_rows, group, most, data.data_ptr(), n)
        return Share(self, rows, max_rows, most, data)

    def attend(self, layer: int, q: torch.Tensor, row_start: torch.Tensor, max_rows: int,
               mask: torch.Tensor | None = None, max_keys: int = 0, scale: float = 0.0,
               out: torch.Tensor | None = None, lse: torch.Tensor | None = None,
               share: Share | None = None) -> torch.Tensor:
        """Attention of the windows' rows q [rows, heads, head_dim] over their sequences'
        tokens and the window rows whose bits are set in mask (int32 [rows, words];
        None: all of them).  share: what groups of sequences have in common is read once for
        each group (made for these windows, lengths and tables)."""
        device = self.device
        starts = self._starts(row_start)
        T, heads, qs = _rows(q, "q", None, self._hd, device)
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=device)
        To, _, os = _rows(out, "out", heads, self._hd, device)
        if q.dtype is not self.dtype or out.dtype is not self.dtype or To != T:
            raise ValueError("q and out must have the cache's type and the same rows")
        words = 0
        if mask is not None:
            words = _mask_words(mask, T)
        bits = _ints(mask, "mask", None, device)
        if lse is not None and (lse.dtype is not torch.float32 or lse.shape != (T, heads) or not lse.is_contiguous()
                                or lse.device != device):
            raise ValueError("lse must be a contiguous float32 tensor [rows, heads]")
        if share is not None:
            if share.cache is not self or share.rows != T or share.max_rows != max_rows:
                raise ValueError("share was made for another cache or for other windows")
            if share.epoch != self._epoch:
                raise ValueError("lengths or tables have changed since share was made")
            if T:
                most = share.max_group_rows
                ws = self._workspace((T, max_rows, most, heads), self.lib.dlm_cache_shared_workspace_bytes, rounded=True)
                self._call("dlm_cache_attend_shared", layer, starts, T, max_rows, most, max_keys, share.data.data_ptr(),
                           4 * share.data.numel(), heads, q.data_ptr(), qs, bits, words, scale, out.data_ptr(), os,
                           None if lse is None else lse.data_ptr(), ws.data_ptr(), ws.numel())
            return out
        if T:
            ws = self.workspace(T, max_rows, heads)
            self._call("dlm_cache_attend", layer, starts, T, max_rows, max_keys, heads, q.data_ptr(), qs, bits, words, scale,
                       out.data_ptr(), os, None if lse is None else lse.data_ptr(), ws.data_ptr(), ws.numel())
        return out
