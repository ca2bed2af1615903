"""The paged cache and the rotary positions at the ends of their ranges, on the GPU:
row starts, lengths and bounds that break their rules, probabilities far below a row's
largest, heads and rows past 32-bit sums.  Tolerances as in tests/test_gpu_cache.py.
"""

from __future__ import annotations

import math

import pytest
import torch

from tests import cache_ref as ref
from tests.gpu_util import need_gpu
from tests.test_gpu_cache import BF, HF, _cache, _fill, _ints, _within

pytestmark = pytest.mark.gpu

INT_MAX, INT_MIN = (1 << 31) - 1, -(1 << 31)
SHIFT = 11                                            # of float16 probabilities, in powers of two


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


# ------------------------------------------------------------------ row starts

@pytest.mark.parametrize("dtype,H,KV,rows", [(BF, 4, 4, 30), (HF, 8, 4, 30), (BF, 16, 2, 30), (HF, 40, 1, 30)])
@pytest.mark.parametrize("starts", [[29, INT_MIN, 0], [INT_MAX, -2, 0], [INT_MAX, INT_MIN, INT_MAX], [5, -5, 30],
                                    [INT_MAX, INT_MAX - 1, INT_MIN], [0, INT_MIN + 7, INT_MIN], [5, 3, 30],
                                    [28, INT_MAX, 2]])
def test_row_starts_whose_difference_passes_32_bits(dtype, H, KV, rows, starts):
    """A start far from a falling or negative one behind it: a window has its rows where
    the second start lies above the first, and no rows otherwise; few and many rows."""
    for max_rows in (1, 4, rows):
        c, _ = _cache([64, 64], 16, KV, 64, dtype)
        c.k.normal_()
        c.v.normal_()
        c.len.fill_(20)
        q = torch.randn(rows, H, 64, device="cuda").to(dtype)
        mask = torch.full((rows, 1), -1, dtype=torch.int32, device="cuda")
        guard = torch.full((3 * rows, H, 64), 5.0, dtype=dtype, device="cuda")
        lse = torch.full((3 * rows, H), 5.0, device="cuda")
        s = _ints(starts)
        c.attend(0, q, s, max_rows, mask=mask, out=guard[rows:2 * rows], lse=lse[rows:2 * rows])
        want = torch.zeros(3 * rows, dtype=torch.bool)
        for a, e in zip(starts, starts[1:]):
            if a >= 0 and min(e, rows) > a:
                want[rows + a:rows + min(a + max_rows, e, rows)] = True
        assert torch.equal((guard != 5).any(-1).all(-1).cpu(), want) and torch.equal((lse != 5).all(-1).cpu(), want)
        assert (guard[~want.cuda()] == 5).all() and (lse[~want.cuda()] == 5).all()
        before = c.k.clone(), c.v.clone()
        c.append(0, q[:, :KV], q[:, :KV], s, max_rows)
        if not want.any():
            assert torch.equal(c.k, before[0]) and torch.equal(c.v, before[1])
        ok = c.reserve(s)
        assert set(ok.tolist()) <= {0, 1}


# ------------------------------------------------------------------ small probabilities

def _sink(dtype, n, gap, noise, at, rows, H, hd, page, max_keys):
    """One key `gap` above a long tail of (nearly) equal ones, with a value of zero, so
    that the result is the tail's.  Scores are exact; the tail's probabilities keep
    half a step each, or what float16 leaves of them: they are held times 2^SHIFT, so
    2^-(25 + SHIFT) of the largest one's weight (the sum's, at least) where they are
    subnormal, which is more than 14 + SHIFT powers of two below it."""
    g = torch.Generator().manual_seed(n + rows)
    c, table = _cache([n], page, 1, hd, dtype, seed=rows)
    k = torch.zeros(n, 1, hd)
    k[:, 0, 0] = (noise * torch.randn(n, generator=g)).clamp(-1, 1)
    k[at, 0, 0] = gap
    v = 1 + 0.5 * torch.randn(n, 1, hd, generator=g)
    v[at] = 0
    k, v = k.to(dtype), v.to(dtype)
    pages = table[0, :-(-n // page)].long()
    full = torch.zeros(len(pages) * page, 1, hd, dtype=dtype)
    for src, pool in ((k, c.k), (v, c.v)):
        full[:n] = src
        pool[0, pages.cuda()] = full.view(len(pages), page, 1, hd).transpose(1, 2).contiguous().cuda()
    c.len.copy_(_ints([n - rows]))
    q = torch.zeros(rows, H, hd, dtype=dtype)
    q[..., 0] = 1
    lse = torch.empty(rows, H, device="cuda")
    out = c.attend(0, q.cuda(), _ints([0, rows]), rows, scale=1.0, max_keys=max_keys, lse=lse)
    want, mag, want_lse = ref.attend(q, k, v, torch.ones(rows, n, dtype=torch.bool), 1.0)
    h = ref.half_step(dtype)
    low = dtype == HF and (gap + k[..., 0].abs().clamp(max=1).max().item()) * math.log2(math.e) > 14 + SHIFT
    tail = n * 2.0 ** -(25 + SHIFT) * v.double().abs().mean() if low else 0.0
    tol = h * want.abs() + (h + 1e-5) * mag + tail + ref.half_subnormal(dtype)
    what = f"sink {dtype} {n} keys {gap} below {at}, {rows} rows of {H} heads"
    _within(out, want, tol, what)
    _within(lse, want_lse, 1e-5 + 2.0 ** -22 * want_lse.abs(), what + " lse")


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("noise", [0.0, 0.25])
@pytest.mark.parametrize("gap", [9.0, 14.0, 16.0, 17.0, 17.5, 21.0])
@pytest.mark.parametrize("n,at,rows,H,hd,page,max_keys", [
    (131072, 0, 1, 1, 64, 64, 0), (131072, 5, 1, 4, 128, 128, 131072), (40000, 39000, 13, 4, 64, 16, 0),
    (131072, 70000, 40, 4, 128, 64, 131072), (20000, 3, 200, 2, 64, 32, 0), (900, 0, 1, 4, 64, 16, 900)])
def test_a_long_tail_far_below_one_key(dtype, gap, noise, n, at, rows, H, hd, page, max_keys):
    _sink(dtype, n, gap, noise, at, rows, H, hd, page, max_keys)


# ------------------------------------------------------------------ bounds on the keys

@pytest.mark.parametrize("dtype,H,KV,hd", [(BF, 4, 2, 64), (HF, 8, 2, 128)])
@pytest.mark.parametrize("rows", [1, 12, 70])
@pytest.mark.parametrize("length,max_keys,width", [(200, 161, 40), (200, 199, 40), (96, 40, 40), (3000, 2567, 400),
                                                   (190, 0, 11), (1 << 29, 0, 11), (176, 0, 11)])
def test_a_mask_does_not_bring_back_keys_behind_the_last(dtype, H, KV, hd, rows, length, max_keys, width):
    """Lengths above max_keys, or above what a table row (of an odd number of 16 keys)
    holds: keys from the bound on are seen by no row, with a mask as without one; rows
    of the window below it follow the mask."""
    page = 16
    room = width * page
    keys = min(length + rows, max_keys or room, room)
    g = torch.Generator().manual_seed(rows + max_keys)
    c, table = _cache([room], page, KV, hd, dtype, width=width, seed=rows)
    k, v = (torch.randn(room, KV, hd, generator=g).to(dtype) for _ in range(2))
    for src, pool in ((k, c.k), (v, c.v)):
        pool[0, table[0].long().cuda()] = src.view(width, page, KV, hd).transpose(1, 2).contiguous().cuda()
    c.len.copy_(_ints([length]))
    q = torch.randn(rows, H, hd, generator=g).to(dtype)
    mask = torch.randint(-2 ** 31, 2 ** 31 - 1, (rows, 3), generator=g, dtype=torch.int32)
    rs = _ints([0, rows])
    n = min(length, keys)
    bits = [[(int(mask[i, j // 32]) >> (j % 32)) & 1 for j in range(keys - n)] for i in range(rows)]
    see = torch.cat([torch.ones(rows, n, dtype=torch.bool), torch.tensor(bits, dtype=torch.bool).view(rows, keys - n)], 1)
    h = ref.half_step(dtype)
    for m, s in ((mask.cuda(), see), (None, torch.ones_like(see))):
        lse = torch.empty(rows, H, device="cuda")
        out = c.attend(0, q.cuda(), rs, rows, mask=m, max_keys=max_keys, lse=lse)
        want, mag, want_lse = ref.attend(q, k[:keys], v[:keys], s, hd ** -0.5)
        what = f"{rows} rows behind {length} tokens, {keys} keys"
        _within(out, want, h * want.abs() + (h + 2e-4) * mag + ref.half_subnormal(dtype), what)
        # float32 scores: hd 2^-24 of the sum of absolute products, below 64 here
        _within(lse, want_lse, torch.full_like(want_lse, 1e-3), what + " lse")


# ------------------------------------------------------------------ commit

@pytest.mark.parametrize("length", [1 << 30, (1 << 30) + 5, (1 << 30) + 64, (1 << 31) - 1, -1, -(1 << 31), 65])
@pytest.mark.parametrize("rows", [0, 4])
def test_commit_leaves_out_lengths_out_of_range_whole(length, rows):
    """A kept list with a length that no table row holds, with window rows and without:
    the sequence keeps its length, pages and tokens, and the ones beside it go through."""
    c, table = _cache([64, 64, 64], 16, 2, 64, BF, layers=2)
    c.k.copy_(torch.randn(c.k.shape, generator=torch.Generator().manual_seed(3)).to(BF))
    c.v.copy_(-c.k)
    c.len.copy_(_ints([10, length, 20]))
    before, k0 = c.meta.clone(), c.k.clone()
    rs = _ints([0, 8, 8 + rows, 12 + rows])
    keep, keep_start = _ints([0, 3, 5, 1, 3, 2]), _ints([0, 3, 5, 6])
    want_ok = [1, 1 if rows == 0 else 0, 1]
    assert c.commit(rs, keep=keep, keep_start=keep_start).tolist() == want_ok
    assert c.len.tolist() == [13, length, 21]
    n = c.ref.numel()
    assert torch.equal(c.table[1].cpu(), table[1]) and (c.ref[table[1].long().cuda()] == 1).all()
    assert c.table[0].tolist() == [int(table[0, 0]), -1, -1, -1]
    assert c.table[2].tolist() == [int(x) for x in table[2, :2]] + [-1, -1]
    want = k0.clone()
    for b, start, kept in ((0, 10, [0, 3, 5]), (2, 20, [2])):
        for i, x in enumerate(kept):
            t, f = start + i, start + x
            want[:, int(table[b, t // 16]), :, t % 16] = k0[:, int(table[b, f // 16]), :, f % 16]
    assert torch.equal(c.k, want) and torch.equal(c.v, -want)
    assert c.meta.numel() == before.numel() and c.ref.sum().item() == int((c.table >= 0).sum()) and n == c.ref.numel()


@pytest.mark.parametrize("kept,per", [([1, 3], 2), ([0, 1, 2, 3, 4], 5), ([3, 1], 2), ([], 0), ([0, 1, 2, 3], 4)])
def test_commit_of_tables_that_hold_any_ids(kept, per):
    """Ids below 0 or past the pool at a window's first token: left out, nothing moves and
    nothing is freed, whatever the id and the list."""
    ids = [-1, -2, -3, -16, -17, -18, -(1 << 31), 1 << 30, (1 << 31) - 1, 15, 16]
    c, table = _cache([32] * len(ids), 16, 1, 64, BF, spare=0)
    n = c.ref.numel()
    c.k.copy_(torch.randn(c.k.shape, generator=torch.Generator().manual_seed(5)).to(BF))
    c.v.copy_(-c.k)
    c.len.fill_(20)
    wild = [x for x in ids if not 0 <= x < n] + [-2 - (n - 1), -1 - n, -2 - n]
    wild = (wild + [-2] * len(ids))[:len(ids)]
    c.table[:, 1] = _ints(wild)
    k0, ref0, first = c.k.clone(), c.ref.clone(), c.table[:, 0].clone()
    rs = _ints([4 * b for b in range(len(ids) + 1)])
    keep = _ints(kept * len(ids))
    ok = c.commit(rs, keep=keep, keep_start=_ints([per * b for b in range(len(ids) + 1)]))
    assert ok.tolist() == [0] * len(ids) and c.len.tolist() == [20] * len(ids)
    assert torch.equal(c.ref, ref0) and torch.equal(c.table[:, 0], first) and torch.equal(c.k, k0)
    now = c.table[:, 1].tolist()
    assert all(a == b or (b == -1 and a < 0) for a, b in zip(wild, now))     # none stays none
    c.table[:, 1] = _ints(wild)
    for starts in ([-1] * (len(ids) + 1), [1 << 30] * (len(ids) + 1), [(-1) ** b * 3 for b in range(len(ids) + 1)]):
        ok = c.commit(rs, keep=keep, keep_start=_ints(starts))       # lists out of range
        assert ok.tolist() == [0] * len(ids) and c.len.tolist() == [20] * len(ids)
        assert torch.equal(c.ref, ref0) and torch.equal(c.table[:, 0], first) and torch.equal(c.k, k0)
    ok = c.commit(rs)                                  # without a list too
    assert ok.tolist() == [0] * len(ids) and torch.equal(c.ref, ref0)


def test_commit_frees_only_pages_that_entries_name():
    """Ids below 0 in entries behind an accepted window are none of the pool's pages."""
    c, table = _cache([64, 64], 16, 1, 64, BF)
    c.len.copy_(_ints([5, 5]))
    c.table[0, 1:] = _ints([-2, -5, -1 - c.ref.numel()])
    c.ref[table[0, 1:].long().cuda()] = 0
    held = c.ref.clone()
    ok = c.commit(_ints([0, 4, 8]), keep=_ints([2, 1, 3]), keep_start=_ints([0, 1, 3]))
    assert ok.tolist() == [1, 1] and c.len.tolist() == [6, 7]
    held[table[1, 1:].long().cuda()] -= 1
    assert torch.equal(c.ref, held)
    assert c.table.tolist() == [[int(table[b, 0]), -1, -1, -1] for b in range(2)]


# ------------------------------------------------------------------ rotary positions

@pytest.mark.parametrize("heads", [(1 << 31) - 1, (1 << 31) - 200])
def test_rotation_of_as_many_heads_as_a_call_may_name(heads):
    """Heads whose index passes 2^31 - 1 by the step to the next one end there (the
    results are 8.6 GB; one head is read for all)."""
    from paper_2608_02625_amd import Rope
    guard = 600
    x = torch.tensor([[[0.75, -1.5]]], dtype=BF, device="cuda").expand(1, heads, 2)
    buf = torch.full((heads + 2 * guard, 2), 5.0, dtype=BF, device="cuda")
    out = buf[guard:guard + heads].view(1, heads, 2)
    Rope(2).apply(x, _ints([3]), out=out)
    want = Rope(2).apply(x[:, :1], _ints([3]))[0, 0]
    assert (buf[:guard] == 5).all() and (buf[guard + heads:] == 5).all()
    for i in range(2):
        assert out[0, :, i].amin() == want[i] and out[0, :, i].amax() == want[i]


# ------------------------------------------------------------------ append

@pytest.mark.parametrize("dtype,src", [(BF, BF), (HF, torch.float32)])
def test_append_overwrites_no_token_of_another_sequence(dtype, src):
    """A pool without a free page: a copy that was cut back gets no page of its own, and
    its rows do not go over the tokens that its original counts; rows behind every
    sequence's tokens are written as ever, and queries come out whole."""
    from paper_2608_02625_amd import PagedCache, Rope
    page, KV, H, hd = 16, 2, 4, 64
    c = PagedCache(2, 3, page, KV, hd, 3, 4, dtype=dtype)
    c.k.zero_()
    c.v.zero_()
    first = torch.randn(40, KV, hd, device="cuda").to(src)
    rs = _ints([0, 40, 40, 40])
    assert c.reserve(rs).tolist() == [1, 1, 1]
    for layer in range(2):
        c.append(layer, first, -first, rs, 40)
    assert c.commit(rs).tolist() == [1, 1, 1]
    assert c.fork(_ints([0, 0]), _ints([1, 2])).tolist() == [1, 1]
    c.truncate(_ints([-1, 36, 30]))                   # 40, 36 and 30 tokens; the last page is shared by two of them
    rows = torch.randn(30, KV, hd, device="cuda").to(src)
    q = torch.randn(30, H, hd, device="cuda").to(src)
    rs = _ints([0, 0, 7, 14])                         # tokens 36 - 42 and 30 - 36
    assert c.reserve(rs).tolist() == [1, 0, 0]
    k0, v0, meta = c.k.clone(), c.v.clone(), c.meta.clone()
    rope = Rope(hd)
    got = [c.append(layer, rows, -rows, rs, 7, q=q, rope=rope) for layer in range(2)]
    assert torch.equal(c.meta, meta)
    p1, p2 = int(c.table[0, 1]), int(c.table[0, 2])
    want = k0.clone(), v0.clone()
    pos = torch.arange(36, 43, dtype=torch.int32, device="cuda")
    turned = rope.apply(rows[:7].contiguous(), pos).to(dtype) if src == dtype else None
    for layer in range(2):
        assert torch.equal(c.k[layer, p1], k0[layer, p1]) and torch.equal(c.v[layer, p1], v0[layer, p1])
        assert torch.equal(c.k[layer, p2, :, :8], k0[layer, p2, :, :8])     # tokens 32 - 39 of the first sequence
        assert torch.equal(c.v[layer, p2, :, :8], v0[layer, p2, :, :8])
        assert torch.equal(c.v[layer, p2, :, 8:11], -rows[4:7].to(dtype).transpose(0, 1))   # its tokens 40 - 42
        if turned is not None:
            assert torch.equal(c.k[layer, p2, :, 8:11], turned[4:7].transpose(0, 1))
        assert torch.equal(c.k[layer, p2, :, 11:], want[0][layer, p2, :, 11:])
    both = torch.cat([pos, torch.arange(30, 37, dtype=torch.int32, device="cuda")])
    w, scale = ref.frequencies(hd)
    turn = ref.rotate(q[:14].cpu(), both.cpu(), w, scale, False)
    for x in got:
        _within(x[:14], turn, ref.half_step(dtype) * turn.abs() + 2.0 ** -19 * 4 + ref.half_subnormal(dtype), "queries")


# ------------------------------------------------------------------ masks

def test_a_mask_of_no_words_is_refused():
    """It shows a row nothing, and is not the missing mask that shows it everything."""
    c, _ = _cache([40], 16, 2, 64, BF)
    q = torch.randn(4, 4, 64, device="cuda").to(BF)
    for rows in (1, 4):
        with pytest.raises(ValueError, match="mask"):
            c.attend(0, q[:rows], _ints([0, rows]), rows, mask=torch.empty(rows, 0, dtype=torch.int32, device="cuda"))
    from paper_2608_02625_amd import Refiner
    from workloads import WORKLOADS
    w = WORKLOADS["tiny"]
    model = Refiner(w.model.as_dict(), w.weight_seed)
    pages = model.cache(4, 16, 1, 4)
    tokens = torch.zeros(3, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="mask"):
        model.cache_step(pages, tokens, _ints([0, 3]), 3, mask=torch.empty(3, 0, dtype=torch.int32, device="cuda"))


# ------------------------------------------------------------------ a model's step

def test_a_step_of_no_rows():
    """Every sequence sits the pass out: nothing is computed, no token is invalid, and
    the same call may be captured."""
    from paper_2608_02625_amd import Refiner
    from workloads import WORKLOADS
    w = WORKLOADS["tiny"]
    model = Refiner(w.model.as_dict(), w.weight_seed)
    c = model.cache(4, 16, 2, 4)
    before = c.meta.clone()
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    rs, bad = _ints([0, 0, 0]), _ints([7])
    for kw in (dict(), dict(positions=none), dict(mask=none.view(0, 1)), dict(mask=none.view(0, 0)), dict(max_keys=5)):
        for max_rows in (0, 1, 9):
            bad.fill_(7)
            out = model.cache_step(c, none, rs, max_rows, n_invalid=bad, **kw)
            assert bad.item() == 0 and [x.numel() for x in out] == [0, 0, 0]
    assert c.attend(0, torch.empty(0, 4, c.k.shape[-1], dtype=BF, device="cuda"), rs, 0, mask=none.view(0, 0)).numel() == 0
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        model.cache_step(c, none, rs, 0, n_invalid=bad)
    for _ in range(3):
        bad.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert bad.item() == 0
    assert torch.equal(c.meta, before)
    with pytest.raises(ValueError):
        model.cache_step(c, none, rs, -1)


# ------------------------------------------------------------------ gradients of a rotation

@pytest.mark.parametrize("dtype", [BF, HF, torch.float32])
@pytest.mark.parametrize("interleaved,transpose", [(False, False), (True, False), (False, True)])
def test_rotation_under_autograd(dtype, interleaved, transpose):
    """The gradient is the formula's (the inner product with a fixed result), for a leaf, a
    broadcast row, a slice and a gradient of any layout; a second derivative is zero, and
    the gradient's own gradient is the rotation."""
    from paper_2608_02625_amd import Rope
    rows, heads, hd, rot = 7, 3, 64, 48
    g = torch.Generator().manual_seed(rot)
    rope = Rope(hd, rot, 10000.0, interleaved, "yarn", 4.0, 1024)
    pos = torch.tensor([0, 1, 5, 100, 4096, 131071, 7], dtype=torch.int32)
    w, scale = ref.frequencies(rot, 10000.0, "yarn", 4.0, 1024)
    up = torch.randn(rows, heads, hd, generator=g).to(dtype)
    h = ref.half_step(dtype)
    want = ref.rotate(up, pos, w, scale, interleaved, not transpose)
    # 2^-21 of the pair's magnitudes (below 16), times the scale, as in test_gpu_cache.py
    tol = h * want.abs() + ref.half_subnormal(dtype) + 2.0 ** -17 * scale
    leaf = torch.randn(rows, heads, hd, generator=g).to(dtype).cuda().requires_grad_()
    y = rope.apply(leaf, pos.cuda(), transpose=transpose)
    assert y.requires_grad and torch.equal(y.detach(), rope.apply(leaf.detach(), pos.cuda(), transpose=transpose))
    grads = {"plain": up.cuda(), "turned": up.cuda().permute(2, 0, 1).contiguous().permute(1, 2, 0)}
    for what, grad in grads.items():
        (got,) = torch.autograd.grad(y, leaf, grad, retain_graph=True)
        _within(got, want, tol, f"gradient {dtype} {what}")
    flat = torch.ones((), dtype=dtype, device="cuda").expand(rows, heads, hd)          # as from a sum
    (got,) = torch.autograd.grad(y, leaf, flat)
    ones = ref.rotate(torch.ones(rows, heads, hd), pos, w, scale, interleaved, not transpose)
    _within(got, ones, h * ones.abs() + ref.half_subnormal(dtype) + 2.0 ** -17 * scale, "gradient of a sum")
    one = torch.randn(1, heads, hd, generator=g).to(dtype).cuda().requires_grad_()      # one row for all positions
    (got,) = torch.autograd.grad(rope.apply(one.expand(rows, heads, hd), pos.cuda(), transpose=transpose), one, up.cuda())
    # torch adds the rows: seven roundings of sums below 32
    _within(got, want.sum(0, keepdim=True), tol.sum(0, keepdim=True) + 7 * 32 * h, "gradient of a shared row")
    wide = torch.randn(rows, heads * hd + 16, generator=g).to(dtype).cuda().requires_grad_()
    part = wide[:, 8:8 + heads * hd].view(rows, heads, hd)
    (got,) = torch.autograd.grad(rope.apply(part, pos.cuda(), transpose=transpose), wide, up.cuda())
    _within(got[:, 8:8 + heads * hd].view(rows, heads, hd), want, tol, "gradient of a slice")
    assert not got[:, :8].any() and not got[:, 8 + heads * hd:].any()
    again = up.cuda().requires_grad_()
    (first,) = torch.autograd.grad(rope.apply(leaf, pos.cuda(), transpose=transpose), leaf, again, create_graph=True)
    (got,) = torch.autograd.grad(first, again, leaf.detach())
    assert torch.equal(got, rope.apply(leaf.detach(), pos.cuda(), transpose=transpose))


def test_rotation_gradients_where_they_cannot_be():
    """`out` takes no part in autograd; without a graph nothing changes."""
    from paper_2608_02625_amd import Rope
    rope, pos = Rope(64), _ints([3, 4])
    leaf = torch.randn(2, 2, 64, device="cuda", requires_grad=True)
    plain = leaf.detach().clone()
    for x, out in ((leaf, torch.empty_like(plain)), (plain, (plain * 1).requires_grad_()), (leaf * 1, plain)):
        with pytest.raises(ValueError, match="out"):
            rope.apply(x, pos, out=out)
    with torch.no_grad():
        y = rope.apply(leaf, pos)
        assert not y.requires_grad and torch.equal(rope.apply(leaf, pos, out=torch.empty_like(plain)), y)
    assert not rope.apply(plain, pos).requires_grad
    for bad in (leaf[0], leaf.double()):
        with pytest.raises(ValueError):
            rope.apply(bad, pos)
    empty = torch.empty(0, 2, 64, device="cuda", requires_grad=True)
    rope.apply(empty, _ints([])).sum().backward()
    assert empty.grad.shape == (0, 2, 64)


def test_rotation_gradients_on_a_stream_and_in_a_graph():
    """The backward pass runs on the stream of the forward; captured, it replays to the
    eager gradient, with eager work in between."""
    from paper_2608_02625_amd import Rope
    rope, pos = Rope(128), torch.arange(33, dtype=torch.int32, device="cuda")
    x = torch.randn(33, 4, 128, device="cuda").to(BF)
    up = torch.randn(33, 4, 128, device="cuda").to(BF)
    want = rope.apply(up, pos, transpose=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        leaf = x.clone().requires_grad_()
        (got,) = torch.autograd.grad(rope.apply(leaf, pos), leaf, up)
    side.synchronize()
    assert torch.equal(got, want)
    del leaf, got
    leaf = x.clone().requires_grad_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        (got,) = torch.autograd.grad(rope.apply(leaf, pos), leaf, up)
    for _ in range(3):
        got.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        assert torch.equal(rope.apply(up, pos, transpose=True), want)
        torch.cuda.synchronize()


# ------------------------------------------------------------------ large scores

@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lens,rows,H,KV,hd", [([300, 50], [1, 1], 4, 2, 64), ([300, 50], [40, 40], 4, 2, 64),
                                               ([9000], [1], 4, 4, 64), ([7000, 40], [13, 5], 8, 2, 128),
                                               ([5000], [90], 4, 2, 64)])
def test_scores_of_thousands(dtype, lens, rows, H, KV, hd):
    """Both signs, whole and split over keys, held to the error of the scores at hand: a
    float32 product of hd values is summed by matrix instructions of 16 in a tree and one
    chain of hd / 16, so a value takes part in at most 4 + hd / 16 additions and the score
    is within (4 + hd / 16) 2^-24 of the sum of absolute products; the exponent's two
    roundings add 2^-23 of the row's maximum.  Probabilities and their sum are off by that
    much, relative, each; the log of the sum is, absolute."""
    g = torch.Generator().manual_seed(hd + rows[0])
    page = 16
    c, table = _cache([n + r for n, r in zip(lens, rows)], page, KV, hd, dtype, seed=2)
    ks, vs = _fill(c, table, lens, rows, KV, hd, dtype, g)
    c.len.copy_(_ints(lens))
    T = sum(rows)
    q = (300 * torch.randn(T, H, hd, generator=g)).to(dtype)
    sees = [torch.ones(n, n, dtype=torch.bool).tril() for n in rows]
    mask = ref.pack_mask(sees, (max(rows) + 31) // 32).cuda()
    lse = torch.empty(T, H, device="cuda")
    starts = [sum(rows[:b]) for b in range(len(rows) + 1)]
    out = c.attend(0, q.cuda(), _ints(starts), max(rows), mask=mask, scale=1.0, lse=lse, max_keys=max(lens) + max(rows))
    h = ref.half_step(dtype)
    for b, n in enumerate(rows):
        part = slice(starts[b], starts[b] + n)
        see = torch.cat([torch.ones(n, lens[b], dtype=torch.bool), sees[b]], 1)
        want, mag, want_lse = ref.attend(q[part], ks[b], vs[b], see, 1.0)
        keys = ks[b].double().repeat_interleave(H // KV, 1)
        total = torch.einsum("nhd,mhd->nhm", q[part].double().abs(), keys.abs()).masked_fill(~see[:, None], 0).amax(-1)
        e = (4 + hd / 16) * 2.0 ** -24 * total + 2.0 ** -23 * want_lse.abs() + 1e-5
        # At most 12 2^-24 of 128 * 300 * 0.64 * 1.6 = 39000 (the largest of thousands of sums
        # lies 1.6 times over their mean) and 2^-23 of 6000: a wrong factor between tiles or
        # parts, 2 at least, does not fit in.
        assert e.max() < 0.04
        what = f"scores of thousands {dtype} {rows[b]} rows behind {lens[b]}"
        _within(out[part], want, h * want.abs() + (h + 2 * e[..., None]) * mag + ref.half_subnormal(dtype), what)
        _within(lse[part], want_lse, e, what + " lse")


# ------------------------------------------------------------------ few rows

@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("H,KV,hd,page,lens,rows", [
    (16, 4, 128, 64, [3000, 17, 700], [1, 1, 1]), (16, 4, 64, 16, [900], [8]), (4, 4, 64, 32, [5000, 5], [32, 3]),
    (32, 1, 128, 128, [2000], [1]), (8, 8, 128, 16, [1, 40000], [1, 2])])
def test_probabilities_of_few_rows_lose_no_bits(dtype, H, KV, hd, page, lens, rows):
    """Up to 32 packed rows: the result is the formula's, rounded once.  A probability is
    taken in two terms, the second rounded to half a step h of at most h of it, so h^2 of
    the sum of p |v| is left, float16's 2^-36 of |v| per key, the float32 scores' error
    (hd 2^-24 of the sum of absolute products, below 2 hd 2^-24 sqrt(hd) for normal values)
    and the float32 sums' (1e-5)."""
    g = torch.Generator().manual_seed(hd + sum(rows))
    c, table = _cache([n + r for n, r in zip(lens, rows)], page, KV, hd, dtype, seed=3)
    ks, vs = _fill(c, table, lens, rows, KV, hd, dtype, g)
    c.len.copy_(_ints(lens))
    q = torch.randn(sum(rows), H, hd, generator=g).to(dtype)
    starts = [sum(rows[:b]) for b in range(len(rows) + 1)]
    out = c.attend(0, q.cuda(), _ints(starts), max(rows))
    h = ref.half_step(dtype)
    for b, n in enumerate(rows):
        part = slice(starts[b], starts[b] + n)
        want, mag, _ = ref.attend(q[part], ks[b], vs[b], torch.ones(n, lens[b] + n, dtype=torch.bool), hd ** -0.5)
        left = h * h + 2 * hd ** 1.5 * 2.0 ** -24 + 1e-5
        low = (lens[b] + n) * 2.0 ** -36 if dtype == HF else 0.0
        tol = h * want.abs() + left * mag + low + ref.half_subnormal(dtype)
        _within(out[part], want, tol, f"few rows {dtype} {H}/{KV}x{hd} behind {lens[b]}")
