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


@pytest.mark.parametrize("which", ["q", "k", "q_gain", "k_gain", "out", "k_out"])
@pytest.mark.parametrize("grad", [False, True])
def test_tangents_are_refused(which, grad):
    """A dual tensor's address leads to its values alone: the derivative would be lost."""
    import torch
    from torch.autograd import forward_ad
    from paper_2608_02625_amd import Rope
    rope = Rope(64)
    t = dict(q=torch.randn(3, 2, 64), k=torch.randn(3, 2, 64), q_gain=torch.ones(64), k_gain=torch.ones(64),
             out=torch.empty(3, 2, 64), k_out=torch.empty(3, 2, 64))
    if which not in ("out", "k_out"):
        t["out"] = t["k_out"] = None
    if grad:
        t["q"].requires_grad_()
    pos = torch.arange(3, dtype=torch.int32)
    with forward_ad.dual_level():
        t[which] = forward_ad.make_dual(t[which], torch.ones_like(t[which]))
        with pytest.raises(ValueError, match="tangent"):
            rope.norm_apply(t["q"], t["k"], pos, t["q_gain"], t["k_gain"], out=t["out"], k_out=t["k_out"])
        if which in ("q", "out"):
            with pytest.raises(ValueError, match="tangent"):
                rope.apply(t["q"], pos, out=t["out"])
        # without one the refusal is that of a tensor on the host
        with pytest.raises(ValueError, match="device tensor"):
            rope.norm_apply(torch.randn(3, 2, 64), None, pos)
