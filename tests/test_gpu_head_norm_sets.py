"""Sets of queries or keys that a call of Rope.norm_apply leaves empty, on the GPU."""

from __future__ import annotations

import pytest
import torch

from tests.gpu_util import need_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


@pytest.mark.parametrize("gain_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads,kv", [(0, 2), (3, 0), (0, 0), (0, None)])
def test_a_gain_without_heads_has_a_gradient_of_zeros(heads, kv, gain_dtype):
    """The sum over no heads, beside a set that has some."""
    from paper_2608_02625_amd import Rope
    g = torch.Generator(device="cuda").manual_seed(3)
    rope, hd, rows = Rope(64), 64, 11
    sets = [None if n is None else torch.randn(rows, n, hd, device="cuda", generator=g).bfloat16().requires_grad_() for n in (heads, kv)]
    gains = [None if n is None else torch.randn(hd, device="cuda", generator=g).to(gain_dtype).requires_grad_() for n in (heads, kv)]
    pos = torch.arange(rows, dtype=torch.int32, device="cuda")
    out = [t for t in rope.norm_apply(sets[0], sets[1], pos, gains[0], gains[1]) if t is not None]
    # What the allocator hands out next holds sevens.
    held = [torch.full((hd,), 7.0, dtype=gain_dtype, device="cuda") for _ in range(16)]
    del held
    leaves = [t for t in (*sets, *gains) if t is not None]
    got = torch.autograd.grad(out, leaves, [torch.ones_like(t) for t in out])
    n = len(leaves) // 2
    for count, dx, dg in zip((heads, kv), got[:n], got[n:]):
        assert dx.shape == (rows, count, hd)
        assert bool(dg.isfinite().all()) and bool(dg.any()) == (count > 0)


def test_tangents_are_refused_forwards_and_backwards():
    from torch.autograd import forward_ad
    from paper_2608_02625_amd import Rope
    rope = Rope(64)
    x = torch.randn(5, 2, 64, device="cuda", requires_grad=True)
    pos = torch.arange(5, dtype=torch.int32, device="cuda")
    for f in (lambda t: rope.norm_apply(t, None, pos)[0], lambda t: rope.apply(t, pos)):
        with forward_ad.dual_level():
            with pytest.raises(ValueError, match="tangent"):
                f(forward_ad.make_dual(x.detach(), torch.ones_like(x)))
            y = f(x)
            seed = forward_ad.make_dual(torch.ones_like(y), torch.ones_like(y))
            with pytest.raises(ValueError, match="tangent"):
                torch.autograd.grad(y, x, seed)
        y = f(x)
        assert torch.autograd.grad(y, x, torch.ones_like(y))[0].shape == x.shape
