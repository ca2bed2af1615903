"""Norms of heads with the rotation (Rope.norm_apply), their gradients, and the form
that puts keys into pages, on the GPU against float64 references on the CPU.

Tolerances.  A rounding is off by at most half a step h of its type, relative.  With
e = 2^-24: a float32 sum of n terms is off by at most n e of the sum of their
magnitudes, whatever the order, so r = 1 / sqrt(mean + eps) is off by (n / 2 + 6) e
(the mean, one sum, one root, one quotient), relative.  A rotated value is within 8 e
(|a| + |b|) s of the formula for the a and b at hand.  A result is the formula's within
both, and its own rounding."""

from __future__ import annotations

import pytest
import torch

from tests import cache_ref as ref
from tests.gpu_util import log, need_gpu

pytestmark = pytest.mark.gpu

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
E = 2.0 ** -24


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


def _lib():
    import paper_2608_02625_amd as P
    return P


def _within(got, want, tol, what):
    got, want = got.detach().double().cpu(), want.double()
    bad = ~((got - want).abs() <= tol)
    worst = ((got - want).abs() / tol.clamp(min=1e-300)).nan_to_num(0).max().item() if got.numel() else 0.0
    log(f"[{what}] worst error {worst:.3f} of the tolerance")
    assert not bad.any(), (what, bad.nonzero()[:5].tolist(), got[bad][:5].tolist(), want[bad][:5].tolist())


def _swap(x, n, interleaved):
    """Every rotated value's partner in its pair; the others as they are."""
    ia = torch.arange(0, 2 * n, 2) if interleaved else torch.arange(n)
    ib = ia + 1 if interleaved else ia + n
    y = x.clone()
    y[..., ia], y[..., ib] = x[..., ib], x[..., ia]
    y[..., 2 * n:] = 0
    return y


def _forward(x, gain, pos, rope, eps):
    """(y, bound of the float32 error) in float64; rope: (w, scale, interleaved)."""
    w, s, inter = rope
    x, n = x.double(), x.shape[-1]
    r = 1.0 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    b = x * r * gain
    y = ref.rotate(b, pos, w, s, inter)
    mag = max(s, 1.0) * (b.abs() + _swap(b.abs(), len(w), inter))
    return y, (n / 2 + 6 + 3 + 8) * E * mag


def _backward(x, gain, pos, rope, eps, dy):
    """(dx, dgain, bounds of both) in float64, from the formula."""
    w, s, inter = rope
    x, dy, n = x.double(), dy.double(), x.shape[-1]
    r = 1.0 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    xn = x * r
    u = ref.rotate(dy, pos, w, s, inter, transpose=True)
    umag = max(s, 1.0) * (dy.abs() + _swap(dy.abs(), len(w), inter))
    h, hmag = u * gain, umag * gain.abs()
    mean = (h * xn).mean(-1, keepdim=True)
    mean_mag = (hmag * xn.abs()).mean(-1, keepdim=True)
    dx = r * (h - xn * mean)
    rel = n / 2 + 6                                   # of r, and of xn
    bx = E * r * (hmag * (rel + 8 + 3) + xn.abs() * mean_mag * (n + 3 * rel + 8 + 6))
    terms = x.shape[0] * x.shape[1]
    bg = E * (umag * xn.abs()).sum((0, 1)) * (terms + rel + 8 + 3)
    return dx, (u * xn).sum((0, 1)), bx, bg


def _rounding(y, dtype):
    return ref.half_step(dtype) * y.abs() + ref.half_subnormal(dtype) if dtype is not F32 else E * y.abs() + 2.0 ** -149


def _rope(P, hd, rot, interleaved, **kw):
    w, s = ref.frequencies(rot, kw.get("theta", 10000.0), kw.get("scaling"), kw.get("factor", 1.0), kw.get("original_len", 0))
    return P.Rope(hd, rot_dim=rot, interleaved=interleaved, **kw), (w, s, interleaved)


def _rows(g, rows, heads, kv, hd, dtype, layout):
    """q and k: tensors of their own, parts of one row, heads outermost, or at odd addresses."""
    if layout == "own":
        return [torch.randn(rows, n, hd, generator=g).to(dtype).cuda() for n in (heads, kv)]
    if layout == "packed":
        t = torch.randn(rows, (heads + 2 * kv) * hd, generator=g).to(dtype).cuda()
        return [t[:, :heads * hd].view(rows, heads, hd), t[:, heads * hd:(heads + kv) * hd].view(rows, kv, hd)]
    if layout == "heads":
        return [torch.randn(n, rows, hd, generator=g).to(dtype).cuda().transpose(0, 1) for n in (heads, kv)]
    t = torch.randn(rows * (heads + kv) * hd + 1, generator=g).to(dtype).cuda()[1:].view(rows, heads + kv, hd)
    return [t[:, :heads], t[:, heads:]]


SHAPES = [(1, 4, 4, 64, 64), (37, 16, 4, 128, 128), (130, 5, 3, 64, 48), (9, 7, 1, 96, 20), (21, 1, 2, 256, 256),
          (5, 3, 3, 2, 2), (11, 2, 2, 255, 2), (6, 20, 4, 128, 64), (3, 2, 1, 250, 2), (515, 2, 1, 32, 32)]


def _positions(g, rows):
    pos = torch.randint(-70000, 1 << 21, (rows,), generator=g, dtype=torch.int32)
    pos[0] = 0
    return pos


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,gain_dtype", [(BF, BF), (BF, F32), (HF, HF), (F32, F32)])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward_and_gradients(shape, dtype, gain_dtype, interleaved):
    P = _lib()
    rows, heads, kv, hd, rot = shape
    g = torch.Generator().manual_seed(rows * 131 + hd)
    kw = dict(scaling="yarn", factor=4.0, original_len=512) if rot >= 32 else {}
    rope, r = _rope(P, hd, rot, interleaved, **kw)
    for layout in ("own", "packed", "heads", "odd"):
        q, k = _rows(g, rows, heads, kv, hd, dtype, layout)
        gains = [(1 + 0.3 * torch.randn(hd, generator=g)).to(gain_dtype).cuda() for _ in range(2)]
        pos = _positions(g, rows)
        grads = [torch.randn(rows, n, hd, generator=g).to(dtype) for n in (heads, kv)]
        leaves = [t.detach().requires_grad_() for t in (q, k, *gains)]
        out = rope.norm_apply(leaves[0], leaves[1], pos.cuda(), leaves[2], leaves[3], eps=1e-5)
        got = torch.autograd.grad(out, leaves, [t.cuda() for t in grads])
        for i, x in enumerate((q, k)):
            gain = gains[i].cpu().double()
            y, tol = _forward(x.cpu(), gain, pos, r, 1e-5)
            name = f"{shape} {dtype} {layout} {'qk'[i]}"
            _within(out[i], y, tol + _rounding(y, dtype), name)
            dx, dg, bx, bg = _backward(x.cpu(), gain, pos, r, 1e-5, grads[i])
            _within(got[i], dx, bx * 1.01 + _rounding(dx.abs() + bx, dtype), name + " dx")
            _within(got[2 + i], dg, bg * 1.01 + _rounding(dg.abs() + bg, gain_dtype), name + " dgain")


@pytest.mark.parametrize("rows,heads,hd,rot", [(4, 3, 64, 64), (7, 2, 40, 24)])
def test_gradients_against_differences(rows, heads, hd, rot):
    P = _lib()
    g = torch.Generator().manual_seed(5)
    rope, r = _rope(P, hd, rot, False, scaling="linear", factor=2.0)
    x, gain = torch.randn(rows, heads, hd, generator=g), 1 + 0.2 * torch.randn(hd, generator=g)
    pos, dy = _positions(g, rows), torch.randn(rows, heads, hd, generator=g)
    leaves = [x.cuda().requires_grad_(), gain.cuda().requires_grad_()]
    out, none = rope.norm_apply(leaves[0], None, pos.cuda(), leaves[1])
    assert none is None
    dx, dg = torch.autograd.grad(out, leaves, dy.cuda())

    def loss(a, b):
        return (_forward(a, b, pos, r, 1e-6)[0] * dy.double()).sum()

    _, _, bx, bg = _backward(x, gain.double(), pos, r, 1e-6, dy)
    for _ in range(6):
        ex, eg = torch.randn(x.shape, generator=g).double(), torch.randn(hd, generator=g).double()
        # Fourth-order differences: the fifth derivative along a unit step is of the
        # loss's size, so their error is about 1e-3^4, and float64's over a step 1e-13.
        t = 1e-3
        f = [loss(x.double() + s * t * ex, gain.double() + s * t * eg) for s in (-2, -1, 1, 2)]
        slope = (f[0] - 8 * f[1] + 8 * f[2] - f[3]) / (12 * t)
        got = (dx.cpu().double() * ex).sum() + (dg.cpu().double() * eg).sum()
        tol = (bx * ex.abs()).sum() * 1.1 + (bg * eg.abs()).sum() * 1.1 + E * ((dx.cpu().abs() * ex.abs()).sum()
                                                                               + (dg.cpu().abs() * eg.abs()).sum()) + 1e-7 * abs(slope)
        assert abs(got - slope) <= tol, (got.item(), slope.item(), tol.item())


def test_no_gains_in_place_and_empty():
    P = _lib()
    g = torch.Generator().manual_seed(1)
    rope, r = _rope(P, 64, 64, False)
    q, k = _rows(g, 19, 4, 2, 64, BF, "packed")
    pos = _positions(g, 19)
    want = rope.norm_apply(q, k, pos.cuda())
    one = torch.ones(64, device="cuda")
    for a, b in zip(want, rope.norm_apply(q, k, pos.cuda(), one, one)):
        assert torch.equal(a, b)
    y, tol = _forward(q.cpu(), torch.ones(64).double(), pos, r, 1e-6)
    _within(want[0], y, tol + _rounding(y, BF), "no gain")
    a, b = rope.norm_apply(q, k, pos.cuda(), out=q, k_out=k)
    assert a is q and b is k and torch.equal(q, want[0]) and torch.equal(k, want[1])
    z = torch.zeros(0, 4, 64, dtype=BF, device="cuda", requires_grad=True)
    gain = torch.ones(64, device="cuda", requires_grad=True)
    out, _ = rope.norm_apply(z, None, torch.zeros(0, dtype=torch.int32, device="cuda"), gain)
    dz, dg = torch.autograd.grad(out, (z, gain), torch.zeros_like(out))
    assert dz.shape == z.shape and torch.equal(dg, torch.zeros_like(dg))
    zero = torch.zeros(3, 4, 64, dtype=HF, device="cuda")
    assert torch.equal(rope.norm_apply(zero, None, torch.arange(3, dtype=torch.int32, device="cuda"))[0], zero)


def test_a_row_does_not_change_another():
    """Infinities and NaN stay in the head that holds them."""
    P = _lib()
    g = torch.Generator().manual_seed(2)
    rope, _ = _rope(P, 128, 96, True)
    q, k = _rows(g, 40, 16, 4, 128, BF, "own")
    pos = _positions(g, 40).cuda()
    want = rope.norm_apply(q, k, pos)
    q[7, 3, 5], k[9, 1, 100] = float("nan"), float("inf")
    got = rope.norm_apply(q, k, pos)
    same = [(a == b).all(-1) for a, b in zip(got, want)]
    assert not same[0][7, 3] and not same[1][9, 1]
    assert int((~same[0]).sum()) == 1 and int((~same[1]).sum()) == 1


def test_only_one_result_is_used():
    P = _lib()
    g = torch.Generator().manual_seed(3)
    rope, _ = _rope(P, 64, 64, False)
    q, k = [t.requires_grad_() for t in _rows(g, 12, 4, 2, 64, F32, "own")]
    qg, kg = [torch.ones(64, device="cuda", requires_grad=True) for _ in range(2)]
    pos = _positions(g, 12).cuda()
    both = torch.autograd.grad([t.sum() for t in rope.norm_apply(q, k, pos, qg, kg)], (q, k, qg, kg))
    a, _ = rope.norm_apply(q, k, pos, qg, kg)
    one = torch.autograd.grad(a.sum(), (q, k, qg, kg), allow_unused=True)    # an expanded gradient: strides 0
    assert one[1] is None and one[3] is None and torch.equal(one[0], both[0])
    # Fewer heads are laid out otherwise over a workgroup, so the gain's 48 terms are added
    # in another order: both sums are within 48 e of the sum of the terms' magnitudes, and a
    # term is u x r with |u| <= |cos| + |sin| <= sqrt(2) for a gradient of ones.
    size = q.detach().abs() * (q.detach().square().mean(-1, keepdim=True) + 1e-6).rsqrt()
    assert ((one[2] - both[2]).abs() <= 2 * 48 * E * 2 ** 0.5 * 1.001 * size.sum((0, 1))).all()
    frozen, _ = rope.norm_apply(q, k.detach(), pos)
    assert torch.autograd.grad(frozen.sum(), q)[0].shape == q.shape
    with pytest.raises(RuntimeError):
        x, = torch.autograd.grad(rope.norm_apply(q, None, pos, qg)[0].square().sum(), q, create_graph=True)
        torch.autograd.grad(x.sum(), q)


def test_gradients_repeat_bit_for_bit_and_far_rows():
    P = _lib()
    g = torch.Generator(device="cuda").manual_seed(4)
    rope, r = _rope(P, 128, 128, False)
    x = torch.randn(9001, 5, 128, device="cuda", generator=g).to(BF).requires_grad_()
    gain = torch.ones(128, device="cuda", requires_grad=True)
    pos = torch.arange(9001, dtype=torch.int32, device="cuda")
    dy = torch.randn(9001, 5, 128, device="cuda", generator=g).to(BF)
    runs = [torch.autograd.grad(rope.norm_apply(x, None, pos, gain)[0], (x, gain), dy) for _ in range(3)]
    for a in runs[1:]:
        assert torch.equal(a[0], runs[0][0]) and torch.equal(a[1], runs[0][1])
    # offsets past 2^31 elements
    wide = torch.zeros((1 << 31) + (1 << 20), dtype=BF, device="cuda").view(-1, 1 << 20)
    far = wide[:, :256].view(wide.shape[0], 2, 128)
    far.normal_(generator=g)
    p = torch.arange(far.shape[0], dtype=torch.int32, device="cuda")
    near = far.contiguous()
    want, _ = rope.norm_apply(near, None, p)
    rope.norm_apply(far, None, p, out=far)
    assert torch.equal(far, want) and not wide[:, 256:].any()


def test_another_stream_and_a_graph():
    P = _lib()
    g = torch.Generator().manual_seed(6)
    rope, _ = _rope(P, 64, 64, False)
    q, k = _rows(g, 33, 8, 2, 64, BF, "packed")
    gains = [torch.randn(64, generator=g).cuda() for _ in range(2)]
    pos = _positions(g, 33).cuda()
    dy = [torch.randn(33, n, 64, generator=g).to(BF).cuda() for n in (8, 2)]

    def step():
        leaves = [t.detach().requires_grad_() for t in (q, k, *gains)]
        out = rope.norm_apply(leaves[0], leaves[1], pos, leaves[2], leaves[3])
        return [*out, *torch.autograd.grad(out, leaves, dy)]

    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for scale in (1.0, 2.0, -1.0):
        q.copy_(want[0] * scale)
        graph.replay()
        now = [t.clone() for t in held]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(now, step()))


@pytest.mark.parametrize("src", ["cache", "f32"])
@pytest.mark.parametrize("dtype,hd,page", [(BF, 128, 64), (HF, 64, 16)])
def test_append_normalises_keys_and_queries(dtype, hd, page, src):
    P = _lib()
    g = torch.Generator().manual_seed(8)
    kind = dtype if src == "cache" else F32
    rows, lens, heads, kv = [3, 0, 17, 1], [5, 9, 31, 0], 6, 2
    c = P.PagedCache(2, 16, page, kv, hd, 4, 4, dtype=dtype)
    fill = torch.tensor([0, 5, 14, 45, 45], dtype=torch.int32, device="cuda")
    c.reserve(fill)
    c.commit(fill)
    starts = torch.tensor([0, 3, 3, 20, 21], dtype=torch.int32, device="cuda")
    lens = c.len.tolist()
    assert lens == [5, 9, 31, 0] and bool(c.reserve(starts).all())
    T = 21
    for layout in ("packed", "odd"):
        c.k.fill_(7.0)
        c.v.fill_(-7.0)
        if layout == "packed":
            t = torch.randn(T, (heads + 2 * kv) * hd, generator=g).to(kind).cuda()
        else:
            t = torch.randn(T * (heads + 2 * kv) * hd + 1, generator=g).to(kind).cuda()[1:].view(T, -1)
        q, k, v = [t[:, a * hd:b * hd].view(T, b - a, hd) for a, b in ((0, heads), (heads, heads + kv), (heads + kv, heads + 2 * kv))]
        gains = [(1 + 0.2 * torch.randn(hd, generator=g)).to(kind).cuda() for _ in range(2)]
        at = torch.tensor([lens[s] + i for s in range(4) for i in range(rows[s])], dtype=torch.int32)
        for given in (None, torch.randint(0, 5000, (T,), generator=g, dtype=torch.int32)):
            pos = at if given is None else given
            rope, r = _rope(P, hd, hd, False)
            got = c.append(1, k, v, starts, 17, q=q, rope=rope, positions=None if given is None else given.cuda(),
                           q_gain=gains[0], k_gain=gains[1], norm_eps=1e-6)
            table = c.table.cpu()
            keys, values = c.k[1].cpu(), c.v[1].cpu()
            place = [(int(table[s, (lens[s] + i) // page]), (lens[s] + i) % page) for s in range(4) for i in range(rows[s])]
            for x, gain, have, name in ((q, gains[0], got, "q"),
                                        (k, gains[1], torch.stack([keys[p, :, o] for p, o in place]), "k")):
                y, tol = _forward(x.cpu(), gain.cpu().double(), pos, r, 1e-6)
                _within(have, y, tol + _rounding(y, dtype), f"append {dtype} {src} {layout} {name}")
            assert torch.equal(torch.stack([values[p, :, o] for p, o in place]), v.cpu().to(dtype))
            for p, o in place:
                keys[p, :, o], values[p, :, o] = 7.0, -7.0
            assert bool((keys == 7.0).all()) and bool((values == -7.0).all()) and bool((c.k[0] == 7.0).all())
        # norms alone, and a window without queries
        c.append(0, k, v, starts, 17, k_gain=gains[1], norm_eps=1e-6)
        have = torch.stack([c.k[0].cpu()[p, :, o] for p, o in place])
        y, tol = _forward(k.cpu(), gains[1].cpu().double(), torch.zeros(T), r, 1e-6)
        _within(have, y, tol + _rounding(y, dtype), "norms alone")
    # entries without a page and pages out of range drop their rows
    c.table[0, 5 // page] = -1
    c.table[2, 31 // page] = 99
    before = c.k.clone()
    c.append(0, k + 1, v, starts, 17, norm_eps=1e-6)
    changed = (before[0] != c.k[0]).any(-1).any(1)
    assert not bool(c.k[1].ne(before[1]).any())
    want = {(int(table[s, (lens[s] + i) // page]), (lens[s] + i) % page) for s, i in [(3, 0)] + [(2, i) for i in range(17)]
            if not (s == 2 and (31 + i) // page == 31 // page)}
    assert {tuple(x) for x in changed.nonzero().tolist()} == want


@pytest.mark.parametrize("dtype,src", [(BF, BF), (BF, F32), (HF, HF)])
@pytest.mark.parametrize("hd,rot,interleaved", [(64, 32, True), (128, 48, False), (128, 98, False), (64, 62, True), (64, 2, False)])
def test_append_of_partly_rotated_heads(hd, rot, interleaved, dtype, src):
    P = _lib()
    g = torch.Generator().manual_seed(rot)
    kw = dict(scaling="yarn", factor=4.0, original_len=512) if rot >= 32 else {}
    rope, r = _rope(P, hd, rot, interleaved, **kw)
    heads, kv, page, T = 3, 2, 32, 70
    c = P.PagedCache(1, 8, page, kv, hd, 2, 4, dtype=dtype)
    starts = torch.tensor([0, 40, 70], dtype=torch.int32, device="cuda")
    assert bool(c.reserve(starts).all())
    for off in (0, 1):                                # aligned, and at odd addresses
        t = torch.randn(T * (heads + 2 * kv) * hd + off, generator=g).to(src).cuda()[off:].view(T, -1)
        q, k, v = [t[:, a * hd:b * hd].view(T, b - a, hd) for a, b in ((0, heads), (heads, heads + kv), (heads + kv, heads + 2 * kv))]
        gains = [(1 + 0.2 * torch.randn(hd, generator=g)).cuda() for _ in range(2)]
        pos = torch.randint(0, 9000, (T,), generator=g, dtype=torch.int32)
        got = c.append(0, k, v, starts, 40, q=q, rope=rope, positions=pos.cuda(), q_gain=gains[0], k_gain=gains[1], norm_eps=1e-5)
        table = c.table.cpu()
        place = [(int(table[s, i // page]), i % page) for s, n in ((0, 40), (1, 30)) for i in range(n)]
        for x, gain, have in ((q, gains[0], got), (k, gains[1], torch.stack([c.k[0].cpu()[p, :, o] for p, o in place]))):
            y, tol = _forward(x.cpu(), gain.cpu().double(), pos, r, 1e-5)
            _within(have, y, tol + _rounding(y, dtype), f"append {hd} {rot} {dtype} {off}")
        assert torch.equal(torch.stack([c.v[0].cpu()[p, :, o] for p, o in place]), v.cpu().to(dtype))
