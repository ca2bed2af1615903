"""CPU checks of sets of heads that are empty, and of inputs that carry a tangent; nothing is
launched."""

from __future__ import annotations

import ctypes

import pytest

from tests.test_cache_api import FAKE, _lib, _refused, _rope
from tests.test_head_norm_api import _grads, _heads


@pytest.mark.parametrize("over,grad,word", [(dict(gain_dtype=1), {}, "gain_dtype"), (dict(gain_dtype=3), {}, "gain_dtype"),
                                            (dict(), dict(d_dgain=FAKE + 1), "aligned"),
                                            (dict(gain_dtype=2), dict(d_dgain=FAKE + 2), "aligned")])
def test_the_gains_gradient_of_an_empty_set_is_checked(over, grad, word):
    L, lib = _lib()
    r = _rope(L, lib)
    empty = _heads(L, n_heads=0, **over)
    bad = _grads(L, **grad)
    n = lib.dlm_rope_norm_grad_workspace_bytes(ctypes.byref(r))
    other, other_g = _heads(L), _grads(L, d_dx=5 * FAKE, d_dgain=6 * FAKE)
    for q, k, dq, dk in ((empty, None, bad, None), (empty, other, bad, other_g), (other, empty, other_g, bad)):
        k, dk = (None, None) if k is None else (ctypes.byref(k), ctypes.byref(dk))
        _refused(lib, lib.dlm_rope_norm_grad(ctypes.byref(r), 0, 3, ctypes.byref(q), k, ctypes.byref(dq), dk, 1e-6, FAKE,
                                             FAKE, n, None), word)


def test_the_gains_gradients_of_two_sets_have_places_of_their_own():
    L, lib = _lib()
    r = _rope(L, lib)
    n = lib.dlm_rope_norm_grad_workspace_bytes(ctypes.byref(r))
    empty, full = _heads(L, n_heads=0), _heads(L)
    a, b = _grads(L), _grads(L, d_dx=5 * FAKE)
    for q, k in ((empty, full), (full, empty), (empty, empty)):
        _refused(lib, lib.dlm_rope_norm_grad(ctypes.byref(r), 0, 3, ctypes.byref(q), ctypes.byref(k), ctypes.byref(a),
                                             ctypes.byref(b), 1e-6, FAKE, FAKE, n, None), "overlap")
