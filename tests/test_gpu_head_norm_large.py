"""Norms of heads with the rotation at sizes where the gradient's workgroups walk over several
groups of rows, and where rows and pages go past the caches (128 MB and more), against the
formulas in float64 on the GPU.

Tolerances as in test_gpu_head_norm.py, but for the gain's gradient: at these sizes a lane adds
at most 64 float32 terms, and what lanes leave is added in float64, so the sum is within
(64 + what the terms are off) 2^-24 of the sum of its terms' magnitudes."""

from __future__ import annotations

import pytest
import torch

from tests.gpu_util import log, need_gpu
from tests.test_gpu_head_norm import BF, E, F32, HF, _rope, _rounding

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


def _turn(x, pos, rope, back=False):
    """x [rows, heads, hd] float64 rotated, and the sum of its pairs' magnitudes, scaled."""
    w, s, inter = rope
    n = len(w)
    ang = pos.double()[:, None] * torch.as_tensor(w, device=x.device)[None, :]
    c, d = s * ang.cos()[:, None], s * ang.sin()[:, None] * (-1 if back else 1)
    ia = torch.arange(0, 2 * n, 2, device=x.device) if inter else torch.arange(n, device=x.device)
    ib = ia + 1 if inter else ia + n
    y, mag = x.clone(), x.abs() * max(s, 1.0)
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * d, b * c + a * d
    mag[..., ia] = mag[..., ib] = max(s, 1.0) * (a.abs() + b.abs())
    return y, mag


def _normed(x, eps):
    x = x.double()
    r = 1.0 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    return x * r, r


def _close(got, want, tol, what):
    worst = ((got.double() - want).abs() / tol).max().item()
    assert worst <= 1.0, (what, worst)                # NaN: not
    return worst


def _rows(g, rows, heads, hd, dtype, odd):
    flat = torch.empty(rows * heads * hd + 1, dtype=dtype, device="cuda").normal_(generator=g)
    return flat[odd:rows * heads * hd + odd].view(rows, heads, hd)


@pytest.mark.parametrize("rows,heads,kv,hd,rot,interleaved,dtype,gain_dtype,odd", [
    (7001, 16, 4, 128, 128, False, BF, F32, 0), (20011, 16, 4, 128, 128, False, BF, BF, 0),
    (20011, 16, 4, 128, 96, True, HF, F32, 0), (7001, 16, 4, 128, 96, True, BF, F32, 0),
    (4099, 16, 16, 64, 48, True, F32, F32, 0), (9001, 16, 16, 64, 48, True, F32, F32, 0),
    (9001, 16, 16, 64, 64, False, F32, F32, 0), (30011, 1, 7, 64, 64, False, HF, HF, 0),
    (12001, 3, 1, 64, 64, False, BF, F32, 1), (12001, 3, 1, 64, 62, True, HF, F32, 1),
    (6001, 2, 2, 256, 256, True, F32, F32, 1), (6001, 2, 2, 255, 2, False, BF, BF, 0)])
def test_values_and_gradients(rows, heads, kv, hd, rot, interleaved, dtype, gain_dtype, odd):
    import paper_2608_02625_amd as P
    g = torch.Generator(device="cuda").manual_seed(rows + hd)
    rope, r = _rope(P, hd, rot, interleaved, **(dict(scaling="yarn", factor=4.0, original_len=512) if rot >= 32 else {}))
    eps = 1e-5
    xs = [_rows(g, rows, n, hd, dtype, odd).requires_grad_() for n in (heads, kv)]
    gains = [(1 + 0.3 * torch.randn(hd, device="cuda", generator=g)).to(gain_dtype).requires_grad_() for _ in range(2)]
    dys = [_rows(g, rows, n, hd, dtype, odd) for n in (heads, kv)]
    pos = torch.randint(-70000, 1 << 21, (rows,), device="cuda", generator=g, dtype=torch.int32)
    out = rope.norm_apply(xs[0], xs[1], pos, gains[0], gains[1], eps=eps)
    got = torch.autograd.grad(out, (*xs, *gains), dys)
    rel = hd / 2 + 6                                  # of r and of x r
    for i, (x, dy, n) in enumerate(zip(xs, dys, (heads, kv))):
        gain = gains[i].detach().double()
        total, size, worst = torch.zeros(hd, dtype=torch.float64, device="cuda"), 0.0, [0.0, 0.0]
        for a in range(0, rows, 4096):
            sl = slice(a, min(a + 4096, rows))
            xn, rr = _normed(x.detach()[sl], eps)
            y, mag = _turn(xn * gain, pos[sl], r)
            worst[0] = max(worst[0], _close(out[i].detach()[sl], y, (rel + 11) * E * mag + _rounding(y, dtype), f"{i} y"))
            u, umag = _turn(dy[sl].double(), pos[sl], r, True)
            h, hmag = u * gain, umag * gain.abs()
            dx = rr * (h - xn * (h * xn).mean(-1, keepdim=True))
            bx = E * rr * (hmag * (rel + 11) + xn.abs() * (hmag * xn.abs()).mean(-1, keepdim=True) * (hd + 3 * rel + 14))
            worst[1] = max(worst[1], _close(got[i][sl], dx, 1.01 * bx + _rounding(dx.abs() + bx, dtype), f"{i} dx"))
            total += (u * xn).sum((0, 1))
            size = size + (umag * xn.abs()).sum((0, 1))
        bg = E * size * (64 + rel + 11)
        w = _close(got[2 + i], total, 1.01 * bg + _rounding(total.abs() + bg, gain_dtype), f"{i} dgain")
        log(f"[{rows}x{n} heads of {hd}, {rot} rotated, {dtype}] y {worst[0]:.3f} dx {worst[1]:.3f} dgain {w:.3f} of the tolerance")


@pytest.mark.parametrize("dtype,src,seqs", [(BF, F32, 16), (BF, BF, 24), (HF, HF, 24)])
@pytest.mark.parametrize("rot,interleaved", [(128, False), (128, True), (64, True)])
def test_prompts_into_pages(dtype, src, seqs, rot, interleaved):
    """150 MB of prompts of up to 1024 tokens, ragged."""
    import paper_2608_02625_amd as P
    heads, kv, hd, page, top = 8, 2, 128, 64, 1024
    g = torch.Generator(device="cuda").manual_seed(rot)
    rope, r = _rope(P, hd, rot, interleaved, scaling="linear", factor=2.0)
    rows = [top - 3 * i for i in range(seqs)]
    starts = torch.tensor([sum(rows[:i]) for i in range(seqs + 1)], dtype=torch.int32, device="cuda")
    T = sum(rows)
    c = P.PagedCache(1, seqs * (top // page), page, kv, hd, seqs, top // page, dtype=dtype)
    assert bool(c.reserve(starts).all())
    c.k.fill_(7.0)
    c.v.fill_(7.0)
    t = torch.empty(T, (heads + 2 * kv) * hd, dtype=src, device="cuda").normal_(generator=g)
    q, k, v = [t[:, a * hd:b * hd].view(T, b - a, hd) for a, b in ((0, heads), (heads, heads + kv), (heads + kv, heads + 2 * kv))]
    gains = [1 + 0.2 * torch.randn(hd, device="cuda", generator=g) for _ in range(2)]
    got = c.append(0, k, v, starts, top, q=q, rope=rope, q_gain=gains[0], k_gain=gains[1], norm_eps=1e-6)
    at = torch.cat([torch.arange(n, device="cuda") for n in rows])
    seq = torch.cat([torch.full((n,), i, device="cuda") for i, n in enumerate(rows)])
    where = c.table[seq, at // page].long()
    keys, values = c.k[0][where, :, at % page], c.v[0][where, :, at % page]
    for x, gain, have, name in ((q, gains[0], got, "q"), (k, gains[1], keys, "k")):
        y, mag = _turn(_normed(x, 1e-6)[0] * gain.double(), at, r)
        w = _close(have, y, (hd / 2 + 17) * E * mag + _rounding(y, dtype), name)
        log(f"[{T} rows, {src} into {dtype}, {rot} rotated] {name} {w:.3f} of the tolerance")
    assert torch.equal(values, v.to(dtype))
    left = torch.ones(c.k.shape[1], page, dtype=torch.bool, device="cuda")
    left[where, at % page] = False                    # places of no token
    assert bool((c.k[0].transpose(1, 2)[left] == 7.0).all()) and bool((c.v[0].transpose(1, 2)[left] == 7.0).all())
