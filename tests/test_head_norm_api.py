"""CPU checks of what the norms of heads refuse; nothing is launched."""

from __future__ import annotations

import ctypes
import math

import pytest

from tests.test_cache_api import FAKE, _cache, _lib, _refused, _rope

NAN, INF = math.nan, math.inf


def _heads(L, **over):
    d = dict(n_heads=4, gain_dtype=0, d_gain=FAKE, d_x=FAKE, x_row_stride=256, x_head_stride=64, d_y=2 * FAKE,
             y_row_stride=256, y_head_stride=64)
    d.update(over)
    return L.DlmNormHeads(*(d[f] for f, _ in L.DlmNormHeads._fields_))


def _grads(L, **over):
    d = dict(d_dy=FAKE, dy_row_stride=256, dy_head_stride=64, d_dx=2 * FAKE, dx_row_stride=256, dx_head_stride=64,
             d_dgain=FAKE)
    d.update(over)
    return L.DlmNormGrads(*(d[f] for f, _ in L.DlmNormGrads._fields_))


BAD = [(dict(n_heads=-1), "n_heads"), (dict(n_heads=(1 << 24) + 1), "n_heads"), (dict(gain_dtype=1), "gain_dtype"),
       (dict(gain_dtype=3), "gain_dtype"), (dict(d_gain=FAKE + 1), "aligned"), (dict(gain_dtype=2, d_gain=FAKE + 2), "aligned"),
       (dict(d_x=None), "NULL"), (dict(d_x=FAKE + 1), "aligned"), (dict(x_row_stride=-1), "strides"),
       (dict(x_head_stride=-64), "strides")]
BAD_RESULT = [(dict(d_y=None), "NULL"), (dict(d_y=FAKE + 1), "aligned"), (dict(y_row_stride=-1), "strides"),
              (dict(y_row_stride=128), "overlap"), (dict(y_head_stride=32), "overlap"), (dict(y_head_stride=0), "overlap"),
              (dict(d_y=FAKE, y_row_stride=512), "in place")]
BAD_GRADS = [(dict(d_dy=None), "NULL"), (dict(d_dx=None), "NULL"), (dict(d_dy=FAKE + 1), "aligned"),
             (dict(d_dgain=FAKE + 1), "aligned"), (dict(dy_row_stride=-1), "strides"), (dict(dx_head_stride=0), "overlap"),
             (dict(d_dx=FAKE, dx_row_stride=512), "in place")]


@pytest.mark.parametrize("over,word", BAD + BAD_RESULT)
def test_forward_refusals(over, word):
    L, lib = _lib()
    r = _rope(L, lib)
    good, bad = _heads(L), _heads(L, **over)
    for q, k in ((bad, None), (good, bad)):
        k = None if k is None else ctypes.byref(k)
        _refused(lib, lib.dlm_rope_norm(ctypes.byref(r), 0, 3, ctypes.byref(q), k, 1e-6, FAKE, None), word)


@pytest.mark.parametrize("over,word", BAD + BAD_GRADS)
def test_gradient_refusals(over, word):
    L, lib = _lib()
    r = _rope(L, lib)
    mine = {f for f, _ in L.DlmNormHeads._fields_} & set(over)
    bad, bad_g = (_heads(L, **over), _grads(L)) if mine else (_heads(L), _grads(L, **over))
    big = 1 << 30
    for q, k, dq, dk in ((bad, None, bad_g, None), (_heads(L), bad, _grads(L), bad_g)):
        k, dk = (None, None) if k is None else (ctypes.byref(k), ctypes.byref(dk))
        _refused(lib, lib.dlm_rope_norm_grad(ctypes.byref(r), 0, 3, ctypes.byref(q), k, ctypes.byref(dq), dk, 1e-6, FAKE,
                                             FAKE, big, None), word)


def test_other_refusals():
    L, lib = _lib()
    r, q, g = _rope(L, lib), _heads(L), _grads(L)
    rp, qp, gp = ctypes.byref(r), ctypes.byref(q), ctypes.byref(g)
    n = lib.dlm_rope_norm_grad_workspace_bytes(rp)
    assert n > 0 and lib.dlm_rope_norm_grad_workspace_bytes(None) == 0
    assert lib.dlm_rope_norm_grad_workspace_bytes(ctypes.byref(L.DlmRope())) == 0
    for eps in (0.0, -1.0, NAN, INF):
        _refused(lib, lib.dlm_rope_norm(rp, 0, 3, qp, None, eps, FAKE, None), "eps")
        _refused(lib, lib.dlm_rope_norm_grad(rp, 0, 3, qp, None, gp, None, eps, FAKE, FAKE, n, None), "eps")
    for rope, dtype, rows, pos, word in ((None, 0, 3, FAKE, "rope"), (ctypes.byref(L.DlmRope()), 0, 3, FAKE, "rope"),
                                         (rp, 3, 3, FAKE, "dtype"), (rp, 0, -1, FAKE, "rows"), (rp, 0, 3, None, "pos"),
                                         (rp, 0, 3, FAKE + 2, "pos")):
        _refused(lib, lib.dlm_rope_norm(rope, dtype, rows, qp, None, 1e-6, pos, None), word)
        _refused(lib, lib.dlm_rope_norm_grad(rope, dtype, rows, qp, None, gp, None, 1e-6, pos, FAKE, n, None), word)
    _refused(lib, lib.dlm_rope_norm(rp, 0, 3, None, None, 1e-6, FAKE, None), "q is NULL")
    _refused(lib, lib.dlm_rope_norm_grad(rp, 0, 3, qp, None, None, None, 1e-6, FAKE, FAKE, n, None), "gradients")
    _refused(lib, lib.dlm_rope_norm_grad(rp, 0, 3, qp, None, gp, None, 1e-6, FAKE, None, n, None), "workspace")
    _refused(lib, lib.dlm_rope_norm_grad(rp, 0, 3, qp, None, gp, None, 1e-6, FAKE, FAKE + 64, n, None), "256-byte")
    _refused(lib, lib.dlm_rope_norm_grad(rp, 0, 3, qp, None, gp, None, 1e-6, FAKE, FAKE, n - 1, None), "small", -5)
    # results of both sets in one place
    far = _heads(L, d_y=3 * FAKE)
    _refused(lib, lib.dlm_rope_norm(rp, 0, 3, qp, qp, 1e-6, FAKE, None), "overlap")
    _refused(lib, lib.dlm_rope_norm_grad(rp, 0, 3, qp, ctypes.byref(far), gp, gp, 1e-6, FAKE, FAKE, n, None), "overlap")
    other = _grads(L, d_dx=5 * FAKE)
    _refused(lib, lib.dlm_rope_norm_grad(rp, 0, 3, qp, qp, gp, ctypes.byref(other), 1e-6, FAKE, FAKE, n, None), "overlap")
    # nothing to do
    assert lib.dlm_rope_norm(rp, 0, 0, qp, None, 1e-6, None, None) == 0
    none = _heads(L, n_heads=0, d_x=None, d_y=None)
    assert lib.dlm_rope_norm(rp, 0, 3, ctypes.byref(none), ctypes.byref(none), 1e-6, None, None) == 0
    quiet = _grads(L, d_dgain=None)
    assert lib.dlm_rope_norm_grad(rp, 0, 0, qp, None, ctypes.byref(quiet), None, 1e-6, None, FAKE, n, None) == 0


def test_append_refusals():
    L, lib = _lib()
    r = _rope(L, lib)

    def call(cache=None, layer=0, rows=4, max_rows=4, src=0, k=FAKE, ks=256, v=FAKE, vs=256, heads=0, q=None, qs=0, qo=None,
             qos=0, gain=0, qg=None, kg=None, eps=1e-6):
        c = cache or _cache(L)
        return lib.dlm_cache_append_norm(ctypes.byref(c), layer, FAKE, rows, max_rows, src, k, ks, v, vs, ctypes.byref(r), None,
                                         heads, q, qs, qo, qos, gain, qg, kg, eps, None)

    for eps in (0.0, -1.0, NAN, INF):
        _refused(lib, call(eps=eps), "eps")
    for kw, word in ((dict(cache=_cache(L, head_dim=96)), "head_dim"), (dict(layer=2), "layer"), (dict(rows=-1), "total_rows"),
                     (dict(max_rows=0), "max_rows"), (dict(src=1), "src_dtype"), (dict(k=None), "NULL"), (dict(ks=255), "k_stride"),
                     (dict(q=FAKE, heads=0), "n_heads"), (dict(q=FAKE, heads=8, qs=512), "q_out"), (dict(gain=1), "gain_dtype"),
                     (dict(kg=FAKE + 1), "aligned"), (dict(gain=2, qg=FAKE + 2), "aligned"),
                     (dict(cache=_cache(L, head_dim=128), ks=512, vs=512), "head_dim")):
        _refused(lib, call(**kw), word)
    assert call(rows=0) == 0
