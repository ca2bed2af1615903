"""Rotary positions and the paged cache on the GPU against plain float64
references on the CPU (tests/cache_ref.py).

Tolerances.  A rounding is off by at most half a step h of its type, relative.
Rotations: angles come from exact integer phases, sine and cosine are good to a
few 2^-24, so a value is within 2^-21 (|a| + |b|) s of the formula before it is
rounded once.  Attention: probabilities are rounded to the cache's type (h of the
sum of p |v|), the result once more (h of it); float32 scores of up to S differ by
at most hd 2^-24 S and their exponentials by as much, relative.
"""

from __future__ import annotations

import math
import random

import pytest
import torch

from tests import cache_ref as ref
from tests.gpu_util import log, need_gpu

pytestmark = pytest.mark.gpu

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


def _lib():
    import paper_2608_02625_amd as P
    return P


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _starts(rows):
    out = [0]
    for n in rows:
        out.append(out[-1] + n)
    return _ints(out)


def _within(got, want, tol, what):
    got, want = got.double().cpu(), want.double()
    bad = ~((got - want).abs() <= tol) & ~((got == want) | (got.isnan() & want.isnan()))
    worst = ((got - want).abs() / tol.clamp(min=1e-300)).nan_to_num(0).max().item() if got.numel() else 0.0
    log(f"[{what}] worst error {worst:.3f} of the tolerance")
    assert not bad.any(), (what, bad.nonzero()[:5].tolist(), got[bad][:5].tolist(), want[bad][:5].tolist())


# ------------------------------------------------------------------ rotary positions

POSITIONS = [0, 1, 2, 31, 4095, 65537, (1 << 20) + 3, (1 << 31) - 1, -1, -77777]


def _rotation_tol(x, w, scale, interleaved, want, dtype):
    """h of the result and 2^-21 of the pair's magnitudes."""
    mag = x.double().abs()
    both = mag.clone()
    n = len(w)
    ia = torch.arange(0, 2 * n, 2) if interleaved else torch.arange(n)
    ib = ia + 1 if interleaved else ia + n
    both[..., ia] = both[..., ib] = mag[..., ia] + mag[..., ib]
    return ref.half_step(dtype) * want.abs() + ref.half_subnormal(dtype) + 2.0 ** -21 * scale * both + 1e-12


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("hd,rot,heads,interleaved,scaling,layout", [
    (64, 64, 4, False, None, "plain"), (64, 64, 3, True, "linear", "plain"), (128, 128, 20, False, "yarn", "wide"),
    (128, 64, 5, True, "ntk", "heads"), (128, 50, 2, False, "yarn", "odd"), (80, 26, 3, True, None, "odd"),
    (256, 256, 1, False, "linear", "plain"), (256, 2, 2, True, None, "heads"), (2, 2, 7, False, None, "plain"),
    (128, 128, 6, False, None, "shared")])
def test_rotation(dtype, hd, rot, heads, interleaved, scaling, layout):
    P = _lib()
    g = torch.Generator().manual_seed(hd * 131 + rot + heads)
    rows = 37
    pos = torch.tensor([POSITIONS[i % len(POSITIONS)] + (i // 10) for i in range(rows)]).clamp(max=(1 << 31) - 1)
    pos = pos.to(torch.int32)
    host = torch.randn(rows, heads, hd, generator=g).to(dtype)
    if layout == "wide":                              # a slice of longer rows
        buf = torch.zeros(rows, heads * hd + 24, dtype=dtype, device="cuda")
        x = buf[:, 8:8 + heads * hd].view(rows, heads, hd)
    elif layout == "odd":                             # aligned to nothing but its elements
        buf = torch.zeros(rows * (heads * hd + 3) + 1, dtype=dtype, device="cuda")
        x = buf[1:1 + rows * (heads * hd + 3)].view(rows, heads * hd + 3)[:, :heads * hd].view(rows, heads, hd)
    elif layout == "heads":                           # heads outermost
        x = torch.zeros(heads, rows, hd, dtype=dtype, device="cuda").transpose(0, 1)
    elif layout == "shared":                          # one row for all positions
        x = torch.zeros(1, heads, hd, dtype=dtype, device="cuda").expand(rows, heads, hd)
        host = host[:1].expand(rows, heads, hd)
    else:
        x = torch.zeros(rows, heads, hd, dtype=dtype, device="cuda")
    (x[:1] if layout == "shared" else x).copy_(host[:1] if layout == "shared" else host)
    factor = 6.5 if scaling else 1.0
    rope = P.Rope(hd, rot, 10000.0, interleaved, scaling, factor, 2048)
    w, scale = ref.frequencies(rot, 10000.0, scaling, factor, 2048)
    # float32 angles of the reference: none; its own float64 product is good to
    # 2^-52 of a position's angle, 2^31 2^-52 = 5e-7 at the largest
    for back in (False, True):
        want = ref.rotate(host, pos, w, scale, interleaved, back)
        tol = _rotation_tol(host, w, scale, interleaved, want, dtype)
        got = rope.apply(x, pos.cuda(), transpose=back)
        _within(got, want, tol + 2e-6 * (pos.double().abs()[:, None, None] > 1e8) * scale * 8, f"rope {dtype} {layout} {back}")
        if layout != "shared":
            own = x.clone(memory_format=torch.preserve_format)
            assert rope.apply(own, pos.cuda(), out=own, transpose=back).data_ptr() == own.data_ptr()
            assert torch.equal(own, got)
            other = torch.empty(heads, rows, hd, dtype=dtype, device="cuda").transpose(0, 1)
            assert torch.equal(rope.apply(x, pos.cuda(), out=other, transpose=back), got)
    if layout == "wide":
        assert not buf[:, :8].any() and not buf[:, 8 + heads * hd:].any()


def test_rotation_of_more_rows_than_a_grid_has_places():
    """A workgroup a row, more rows than 2^32 threads along one axis hold; offsets past
    2^32 (the results are 9 GB)."""
    P = _lib()
    rows, hd = (1 << 24) + 3, 256
    x = torch.randn(1, 1, hd, generator=torch.Generator().manual_seed(4)).to(BF).cuda().expand(rows, 1, hd)
    pos = torch.arange(rows, dtype=torch.int32, device="cuda")
    out = torch.empty(rows * (hd + 1), dtype=BF, device="cuda").view(rows, hd + 1)[:, 1:].view(rows, 1, hd)
    P.Rope(hd, 2, interleaved=True).apply(x, pos, out=out)
    at = torch.tensor([0, 1, (1 << 20) - 1, 1 << 20, (1 << 23) + 5, rows - 2, rows - 1])
    w, scale = ref.frequencies(2)
    host = x[:1].cpu().expand(len(at), 1, hd)
    want = ref.rotate(host, at.to(torch.int32), w, scale, True)
    tol = _rotation_tol(host, w, scale, True, want, BF)
    _within(out[at.cuda()], want, tol, "rope of many rows")
    assert torch.equal(out[:, 0, 2:].amin(0), x[0, 0, 2:]) and torch.equal(out[:, 0, 2:].amax(0), x[0, 0, 2:])


def test_rotation_gradient_is_the_transpose():
    """d/dx of sum(g * rotate(x)), by differences and by the inner product."""
    P = _lib()
    rope = P.Rope(64, 48, 10000.0, True, "yarn", 4.0, 1024)
    gen = torch.Generator(device="cuda").manual_seed(5)
    x, g = (torch.randn(9, 3, 64, generator=gen, device="cuda") for _ in range(2))
    pos = _ints([0, 1, 5, 100, 1023, 4096, 30000, 131071, 7])
    grad = rope.apply(g, pos, transpose=True)
    for r, h, c in ((0, 0, 0), (3, 1, 10), (5, 2, 47), (7, 0, 46), (8, 1, 63)):
        d = torch.zeros_like(x)
        d[r, h, c] = 0.5
        # the map is linear, so a difference is exact but for float32 roundings of
        # values below 8: 2^-24 * 8 * a few terms
        diff = ((rope.apply(x + d, pos).double() - rope.apply(x - d, pos).double()) * g.double()).sum()
        assert abs(diff.item() - grad[r, h, c].item()) < 64 * 2.0 ** -21
    lhs = (rope.apply(x, pos).double() * g.double()).sum().item()
    rhs = (x.double() * grad.double()).sum().item()
    assert abs(lhs - rhs) < 9 * 3 * 64 * 8 * 2.0 ** -23


def test_rotation_edges():
    P = _lib()
    rope = P.Rope(128)
    e = torch.empty(0, 4, 128, dtype=BF, device="cuda")
    assert rope.apply(e, _ints([])).shape == (0, 4, 128)
    x = torch.randn(1, 1, 128, device="cuda").to(BF)
    assert torch.equal(rope.apply(x, _ints([0])), x)
    inf = x.clone()
    inf[0, 0, 3] = math.inf
    y = rope.apply(inf, _ints([0]))
    assert torch.isinf(y[0, 0, 3]) and torch.equal(y[0, 0, 70:], x[0, 0, 70:])
    for bad in (x[0], x.double(), x[..., :64], x.cpu()):
        with pytest.raises(ValueError):
            rope.apply(bad, _ints([0]))
    with pytest.raises(ValueError):
        rope.apply(x, torch.zeros(1, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        rope.apply(x, _ints([0, 1]))
    with pytest.raises(P.DlmError):
        P.Rope(128, rot_dim=3)


# ------------------------------------------------------------------ rows into pages

def _cache(rows_held, page, KV, hd, dtype, layers=1, width=None, spare=3, seed=0, shuffle=True):
    """A cache whose sequences hold pages for `rows_held` tokens each, in shuffled
    order; pools filled with a recognisable value."""
    P = _lib()
    need = [-(-n // page) for n in rows_held]
    n_pages = sum(need) + spare
    c = P.PagedCache(layers, n_pages, page, KV, hd, len(rows_held), width or max(1, max(need)), dtype=dtype)
    order = list(range(n_pages))
    if shuffle:
        random.Random(seed).shuffle(order)
    table = torch.full(tuple(c.table.shape), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        for e in range(n):
            table[b, e] = order[at]
            at += 1
    c.table.copy_(table)
    for p in order[:at]:
        c.ref[p] = 1
    c.k.fill_(-7.0)
    c.v.fill_(-9.0)
    return c, table


@pytest.mark.parametrize("dtype,src", [(BF, BF), (HF, HF), (BF, F32), (HF, F32)])
@pytest.mark.parametrize("H,KV,hd,page,rot,interleaved", [
    (16, 4, 128, 64, 128, False), (4, 4, 64, 16, 64, True), (7, 1, 64, 32, 24, False), (6, 3, 128, 128, 0, False),
    (10, 5, 64, 16, 50, True)])
def test_append(dtype, src, H, KV, hd, page, rot, interleaved):
    P = _lib()
    lens, rows = [0, 5, 33, 100, 7, 64], [3, 0, 70, 1, 130, 16]
    c, table = _cache([n + r for n, r in zip(lens, rows)], page, KV, hd, dtype, layers=2)
    c.len.copy_(_ints(lens))
    drop = (2, (lens[2] + 40) // page)                # a page that is not there: its rows are dropped
    table[drop] = -1
    drop2 = (4, 0)                                    # an id that is no page
    table[drop2] = c.ref.numel() + 5
    c.table.copy_(table)
    T, W = sum(rows), (H + 2 * KV) * hd
    g = torch.Generator().manual_seed(H * hd + page)
    qkv = torch.randn(T + 2, W, generator=g).to(src)  # two rows that no window covers
    dev = qkv.cuda()
    q = dev[:, :H * hd].view(T + 2, H, hd)
    k = dev[:, H * hd:(H + KV) * hd].view(T + 2, KV, hd)
    v = dev[:, (H + KV) * hd:].view(T + 2, KV, hd)
    pos = torch.randint(0, 1 << 17, (T + 2,), generator=g, dtype=torch.int32)
    rope = P.Rope(hd, rot, 10000.0, interleaved) if rot else None
    out = torch.full((T + 2, H, hd), 3.0, dtype=dtype, device="cuda")
    given = rot == 0 or page != 64                    # else: positions are the tokens' places
    got = c.append(1, k, v, _starts(rows), max(rows), q=q, rope=rope, positions=pos.cuda() if given else None, q_out=out)
    assert got is out
    if not given:
        pos = torch.tensor([n + i for n, r in zip(lens, rows) for i in range(r)] + [0, 0], dtype=torch.int32)
    w, scale = ref.frequencies(rot) if rot else ([], 1.0)
    hq = qkv[:, :H * hd].view(T + 2, H, hd)
    hk = qkv[:, H * hd:(H + KV) * hd].view(T + 2, KV, hd)
    hv = qkv[:, (H + KV) * hd:].view(T + 2, KV, hd)

    def turned(x):
        y = ref.rotate(x, pos, w, scale, interleaved) if rot else x.double()
        return y, (_rotation_tol(x, w, scale, interleaved, y, dtype) if rot else
                   ref.half_step(dtype) * y.abs() + ref.half_subnormal(dtype))
    want_q, tol_q = turned(hq)
    _within(out[:T], want_q[:T], tol_q[:T], "append q")
    assert (out[T:] == 3.0).all()
    want_k, tol_k = turned(hk)
    want_v = hv.to(dtype)
    K, V = c.k.cpu(), c.v.cpu()
    seen = torch.zeros(K.shape[1], page, dtype=torch.bool)
    t = 0
    for b, n in enumerate(rows):
        for i in range(n):
            e, at = (lens[b] + i) // page, (lens[b] + i) % page
            p = int(table[b, e])
            if 0 <= p < K.shape[1]:
                assert ((K[1, p, :, at].double() - want_k[t]).abs() <= tol_k[t]).all(), (b, i)
                assert torch.equal(V[1, p, :, at], want_v[t]), (b, i)
                seen[p, at] = True
            t += 1
    assert (K[0] == -7).all() and (V[0] == -9).all()  # the other layer
    assert (K[1].permute(0, 2, 1, 3)[~seen] == -7).all() and (V[1].permute(0, 2, 1, 3)[~seen] == -9).all()
    if src == dtype:                                  # queries in place
        own = q.clone()
        assert torch.equal(c.append(1, k, v, _starts(rows), max(rows), q=own, rope=rope,
                                    positions=pos.cuda() if given else None, q_out=own)[:T], out[:T])


def test_append_cuts_off_what_does_not_fit():
    """Rows past max_rows, past the table row, and starts out of range."""
    c, table = _cache([64, 64, 64], 16, 2, 64, BF)
    c.len.copy_(_ints([0, 60, 0]))
    k = torch.ones(40, 2, 64, dtype=BF, device="cuda")
    c.append(0, k, k * 2, _ints([0, 10, 20, 60]), 8)  # 10 rows cut to 8; 4 of 10 fit the row; 20 of 40 exist, 8 count
    got = (c.k[0, :, 0, :, 0] == 1).cpu()
    want = torch.zeros_like(got)
    want[table[0, 0], :8] = True
    want[table[1, 3], 12:] = True
    want[table[2, 0], :8] = True
    assert torch.equal(got, want)
    c.k.fill_(-7.0)
    c.append(0, k, k, _ints([-5, 3, 2, 2]), 8)        # a start below 0, one past its end, an empty one
    assert (c.k == -7).all()
    c.len.copy_(_ints([-3, 1 << 30, 0]))
    c.append(0, k, k, _ints([0, 4, 8, 8]), 8)
    assert (c.k == -7).all()


# ------------------------------------------------------------------ attention

def _fill(c, table, lens, rows, KV, hd, dtype, g):
    """Random K and V of every token of every sequence, in the pools and as lists."""
    ks, vs = [], []
    page = c.k.shape[3]
    K, V = c.k.cpu(), c.v.cpu()
    for b in range(len(lens)):
        n = lens[b] + rows[b]
        k, v = torch.randn(n, KV, hd, generator=g).to(dtype), torch.randn(n, KV, hd, generator=g).to(dtype)
        for e in range(-(-n // page)):
            p, m = int(table[b, e]), min(page, n - e * page)
            K[0, p, :, :m] = k[e * page:e * page + m].transpose(0, 1)
            V[0, p, :, :m] = v[e * page:e * page + m].transpose(0, 1)
        ks.append(k)
        vs.append(v)
    c.k.copy_(K)
    c.v.copy_(V)
    return ks, vs


def _see(kind, n, rng):
    see = torch.zeros(n, n, dtype=torch.bool)
    for i in range(n):
        if kind == "full":
            see[i] = True
        elif kind == "chain":
            see[i, :i + 1] = True
        elif kind == "tree":
            if i:
                see[i] = see[rng.randrange(max(0, i - 6), i)]
            see[i, i] = True
        elif kind == "blocks":
            see[i, i // 5 * 5:i // 5 * 5 + 5] = True
        elif kind == "random":                        # with empty rows
            if rng.random() < 0.7:
                see[i] = torch.tensor([rng.random() < 0.3 for _ in range(n)])
    return see


def _attend_case(dtype, H, KV, hd, page, lens, rows, kind, seed, scale=0.0, pad=0, spare=3, max_keys=None, q_mul=1.0):
    g = torch.Generator().manual_seed(seed)
    rng = random.Random(seed)
    c, table = _cache([n + r for n, r in zip(lens, rows)], page, KV, hd, dtype, seed=seed, spare=spare)
    # places that hold no token: values that would show in any result
    c.k.fill_(math.nan)
    c.v.fill_(math.nan)
    ks, vs = _fill(c, table, lens, rows, KV, hd, dtype, g)
    c.len.copy_(_ints(lens))
    T = sum(rows)
    q = (q_mul * torch.randn(T + 1, H, hd, generator=g)).to(dtype)
    sees = [_see(kind, n, rng) for n in rows]
    words = (max(rows) + 31) // 32 + (1 if seed % 2 else 0)
    mask = None if kind == "full" else torch.cat([ref.pack_mask(sees, words), torch.zeros(1, words, dtype=torch.int32)]).cuda()
    dq = torch.zeros(T + 1, H * hd + pad, dtype=dtype, device="cuda")
    dq[:, :H * hd] = q.view(T + 1, -1).cuda()
    dq = dq[:, :H * hd].view(T + 1, H, hd)
    out = torch.full((T + 1, H * hd + 2 * pad), 5.0, dtype=dtype, device="cuda")[:, :H * hd].view(T + 1, H, hd)
    lse = torch.full((T + 1, H), 5.0, device="cuda")
    got = c.attend(0, dq, _starts(rows), max(rows), mask=mask, scale=scale, out=out, lse=lse,
                   max_keys=max(n + r for n, r in zip(lens, rows)) if max_keys is None else max_keys)
    assert got is out
    s = scale or hd ** -0.5
    h = ref.half_step(dtype)
    t = 0
    for b, n in enumerate(rows):
        if n == 0:
            continue
        see = torch.cat([torch.ones(n, lens[b], dtype=torch.bool), sees[b]], 1)
        want, mag, want_lse = ref.attend(q[t:t + n], ks[b], vs[b], see, s)
        # largest score, and the sum of absolute products behind a score
        S = s * q[t:t + n].abs().double().amax() * ks[b].abs().double().amax() * hd if see.any() else 0.0
        e = hd * 2.0 ** -24 * float(S) / 4            # products are of random sign: a quarter of the worst case
        tol = h * want.abs() + (h + e + 1e-5) * mag + ref.half_subnormal(dtype)
        _within(out[t:t + n], want, tol, f"attend {dtype} {H}/{KV}x{hd} page {page} len {lens[b]} rows {n} {kind}")
        # -infinity where nothing is seen
        _within(lse[t:t + n], want_lse, (e + 1e-5) * torch.ones_like(want_lse) + 2.0 ** -22 * want_lse.abs().nan_to_num(0, 0, 0),
                "lse")
        dark = ~see.any(1)
        assert (out[t:t + n][dark.cuda()] == 0).all() and torch.isneginf(lse[t:t + n][dark.cuda()]).all()
        t += n
    assert (out[T:] == 5.0).all() and (lse[T:] == 5.0).all()
    return c, dq, mask, out, lse


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("H,KV,hd,page", [(4, 4, 64, 16), (16, 4, 128, 64), (6, 2, 128, 32), (5, 1, 64, 128), (40, 1, 64, 16)])
@pytest.mark.parametrize("lens,rows,kind", [
    ([0, 1, 31, 32, 33, 63, 64, 65], [1] * 8, "full"),
    ([0, 500, 3, 129], [1, 1, 0, 1], "chain"),
    ([0, 40, 17], [7, 5, 2], "tree"),
    ([30, 0, 100], [34, 65, 1], "tree"),
    ([0, 64, 15, 0], [33, 20, 40, 0], "random"),
    ([10, 70], [100, 130], "blocks"),
    ([0, 90], [200, 1], "full")])
def test_attend(dtype, H, KV, hd, page, lens, rows, kind):
    _attend_case(dtype, H, KV, hd, page, lens, rows, kind, seed=H + hd + page + len(lens), pad=8 * (H % 3))


@pytest.mark.parametrize("dtype,H,KV,hd,page,lens,rows,kind", [
    (BF, 16, 4, 128, 64, [20000], [1], "full"), (HF, 8, 8, 64, 16, [9000, 3], [3, 2], "tree"),
    (BF, 16, 4, 128, 32, [5000, 100, 0, 2500], [40, 9, 3, 0], "tree"), (BF, 4, 2, 64, 128, [12345], [70], "chain"),
    (HF, 4, 1, 128, 16, [4097, 4096, 4095], [1, 1, 1], "full")])
def test_attend_split_over_keys(dtype, H, KV, hd, page, lens, rows, kind):
    """Long sequences are split and joined; again gives the same bits, and a bound on
    the keys changes how, not what."""
    c, q, mask, out, lse = _attend_case(dtype, H, KV, hd, page, lens, rows, kind, seed=11)
    again = torch.empty_like(out)
    lse2 = torch.empty_like(lse)
    most = max(n + r for n, r in zip(lens, rows))
    c.attend(0, q, _starts(rows), max(rows), mask=mask, max_keys=most, out=again, lse=lse2)
    T = sum(rows)
    assert torch.equal(again[:T], out[:T]) and torch.equal(lse2[:T], lse[:T])
    c.attend(0, q, _starts(rows), max(rows), mask=mask, out=again)         # what the tables can hold
    h = ref.half_step(dtype)
    err = (again[:T].double() - out[:T].double()).abs()
    assert (err <= 4 * h * (out[:T].double().abs() + 1)).all()


@pytest.mark.parametrize("dtype,H,KV,hd,page,seqs,top,kind", [
    (BF, 4, 4, 64, 16, 130, 1, "full"), (HF, 4, 1, 128, 32, 1000, 2, "tree"), (BF, 8, 2, 64, 64, 70, 12, "tree"),
    (BF, 16, 4, 64, 16, 100, 30, "tree"), (HF, 16, 16, 64, 32, 11, 200, "blocks"), (BF, 8, 1, 128, 128, 90, 9, "random")])
def test_attend_batches(dtype, H, KV, hd, page, seqs, top, kind):
    """More sequences than lanes, ragged, some idle or empty; few and many rows each."""
    rng = random.Random(seqs)
    lens = [rng.choice([0, rng.randint(1, 40), rng.randint(1, 150)]) for _ in range(seqs)]
    rows = [rng.choice([0, 1, top, rng.randint(1, top)]) for _ in range(seqs)]
    rows[rng.randrange(seqs)] = top
    if seqs < 1000:
        lens[3] = 1500                                # one that is split, if it has rows
    _attend_case(dtype, H, KV, hd, page, lens, rows, kind, seed=seqs)


def test_row_starts_that_overlap_stay_in_bounds():
    """Falling row starts are not allowed; they reach no memory of others."""
    c, _ = _cache([300] * 64, 16, 4, 64, BF)
    c.k.normal_()
    c.v.normal_()
    c.len.fill_(100)
    q = torch.randn(200, 16, 64, device="cuda").to(BF)
    guard = torch.full((400, 16, 64), 5.0, dtype=BF, device="cuda")
    starts = _ints([0 if i % 2 == 0 else 200 for i in range(65)])
    c.attend(0, q, starts, 200, out=guard[100:300])
    assert (guard[:100] == 5).all() and (guard[300:] == 5).all()
    c.append(0, q[:, :4], q[:, :4], starts, 200)
    ok = c.reserve(starts)
    assert set(ok.tolist()) <= {0, 1}


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows", [1, 40])
def test_attend_extreme_scores(dtype, rows):
    """Scores of thousands, both signs: one key takes all, nothing overflows."""
    _attend_case(dtype, 4, 2, 64, 16, [300, 50], [rows, rows], "chain", seed=4, q_mul=300.0, scale=1.0)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("H,rows", [(4, 5), (8, 40)])
def test_what_a_row_does_not_see_does_not_change_it(dtype, H, rows):
    """Infinities and NaN in the keys and values of tree rows: rows that do not see
    them keep their bits, rows that do follow the formula."""
    lens, KV, hd, page = [45], 2, 64, 16
    c, q, mask, out, _ = _attend_case(dtype, H, KV, hd, page, lens, [rows], "tree", seed=21)
    clean = out.clone()
    rng = random.Random(21)
    see = _see("tree", rows, rng)
    for what, value in (("v", math.inf), ("v", -math.inf), ("v", math.nan), ("k", math.nan), ("k", math.inf)):
        j = 3
        pool = c.v if what == "v" else c.k
        t = lens[0] + j
        p = int(c.table[0, t // page])
        old = pool[0, p, :, t % page].clone()
        pool[0, p, :, t % page, 7] = value
        got = torch.empty_like(out)
        c.attend(0, q, _ints([0, rows]), rows, mask=mask, out=got)
        blind = ~see[:, j]
        assert blind.any() and see[:, j].any()
        assert torch.equal(got[:rows][blind.cuda()], clean[:rows][blind.cuda()]), (what, value)
        hit = got[:rows][see[:, j].cuda()]
        if what == "v":
            assert (hit[..., 7] == value).all() if not math.isnan(value) else hit[..., 7].isnan().all()
            rest = [i for i in range(hd) if i != 7]
            assert torch.equal(hit[..., rest], clean[:rows][see[:, j].cuda()][..., rest])
        elif math.isnan(value):
            assert hit.isnan().all()
        pool[0, p, :, t % page] = old
    # infinities of both signs in one value: their sum is no number
    for j, value in ((0, math.inf), (1, -math.inf)):
        t = lens[0] + j
        c.v[0, int(c.table[0, t // page]), :, t % page, 9] = value
    c.attend(0, q, _ints([0, rows]), rows, mask=mask, out=got)
    for i in range(rows):
        a, b = bool(see[i, 0]), bool(see[i, 1])
        x = got[i, :, 9]
        assert (x.isnan() if a and b else x == math.inf if a else x == -math.inf if b else x.isfinite()).all(), i


def test_missing_pages_are_seen_by_no_row():
    """A hole in a sequence (an id below 0 or past the pool) leaves its keys out."""
    for rows, H in ((1, 4), (50, 8)):
        for page, hole in ((16, 1), (16, 2), (32, 0), (64, 1)):
            g = torch.Generator().manual_seed(page + rows)
            c, table = _cache([150 + rows], page, 2, 64, BF, seed=page)
            ks, vs = _fill(c, table, [150], [rows], 2, 64, BF, g)
            c.len.copy_(_ints([150]))
            c.table[0, hole] = -1 if rows == 1 else c.ref.numel()
            q = torch.randn(rows, H, 64, generator=g).to(BF)
            out = c.attend(0, q.cuda(), _ints([0, rows]), rows)
            see = torch.ones(rows, 150 + rows, dtype=torch.bool)
            see[:, hole * page:(hole + 1) * page] = False
            want, mag, _ = ref.attend(q, ks[0], vs[0], see, 64 ** -0.5)
            h = ref.half_step(BF)
            _within(out, want, h * want.abs() + (h + 2e-4) * mag, f"hole {hole} of pages of {page}")
    c.table.fill_(-1)                                 # nothing at all
    out = c.attend(0, q.cuda(), _ints([0, rows]), rows)
    assert (out == 0).all()


@pytest.mark.parametrize("page,rows,H,kind", [(16, 1, 4, "full"), (16, 12, 8, "tree"), (16, 150, 8, "tree"), (32, 40, 8, "full"),
                                              (16, 300, 4, "blocks")])
def test_holes_anywhere_in_long_tables(page, rows, H, kind):
    """Holes at both ends of what a wave holds of a table row, next to each other, in
    single groups of 16 keys, in the window and in the last page."""
    g = torch.Generator().manual_seed(page + rows)
    rng = random.Random(rows)
    lens = [16 * 200 + 5, 16 * 70]
    counts = [rows, rows]
    c, table = _cache([n + rows for n in lens], page, 2, 64, BF, seed=page)
    c.k.fill_(math.nan)
    c.v.fill_(math.nan)
    ks, vs = _fill(c, table, lens, counts, 2, 64, BF, g)
    c.len.copy_(_ints(lens))
    q = torch.randn(2 * rows, H, 64, generator=g).to(BF)
    sees = [_see(kind, n, rng) for n in counts]
    mask = None if kind == "full" else ref.pack_mask(sees, (rows + 31) // 32).cuda()
    holes = [[0, 61, 62, 63, 64, 65, 99, 126], [5, (lens[1] + rows - 1) // page]]
    for b in range(2):
        for i, e in enumerate(holes[b]):
            if e * page < lens[b] + rows:
                c.table[b, e] = (-1, c.ref.numel(), -(1 << 31), (1 << 31) - 1)[i % 4]
    out = c.attend(0, q.cuda(), _starts(counts), rows, mask=mask, max_keys=max(lens) + rows)
    h = ref.half_step(BF)
    for b in range(2):
        see = torch.cat([torch.ones(rows, lens[b], dtype=torch.bool), sees[b]], 1)
        for e in holes[b]:
            see[:, e * page:(e + 1) * page] = False
        part = slice(b * rows, (b + 1) * rows)
        want, mag, _ = ref.attend(q[part], ks[b], vs[b], see, 64 ** -0.5)
        _within(out[part], want, h * want.abs() + (h + 2e-4) * mag + ref.half_subnormal(BF), f"holes {page} {rows} {b}")


def test_attend_cuts_off_what_does_not_fit():
    """Starts, lengths and row counts out of range reach no memory of others; rows in
    range are computed."""
    c, table = _cache([64, 64], 16, 2, 64, BF)
    c.k.normal_()
    c.v.normal_()
    q = torch.randn(30, 4, 64, device="cuda").to(BF)
    out = torch.full_like(q, 5.0)
    c.len.copy_(_ints([1 << 30, -8]))
    c.attend(0, q, _ints([0, 10, 99]), 12, out=out)   # lengths cut to the row, to 0; 20 of 89 rows exist, 12 count
    assert out[:22].isfinite().all() and (out[:22] != 5.0).any(-1).all() and (out[22:] == 5.0).all()
    out.fill_(5.0)
    c.attend(0, q, _ints([-4, 3, 2]), 12, out=out)
    assert (out == 5.0).all()
    full = c.attend(0, q, _ints([0, 30, 30]), 30)
    c.len.zero_()
    part = c.attend(0, q, _ints([0, 30, 30]), 30, max_keys=16)
    assert not torch.equal(full, part)


def test_attend_in_place_and_refusals():
    c, _ = _cache([200, 90], 32, 2, 128, BF)
    c.k.normal_()
    c.v.normal_()
    c.len.copy_(_ints([100, 90]))
    P = _lib()
    for rows, n in (([1, 0], 1), ([100, 0], 100)):
        q = torch.randn(n, 8, 128, device="cuda").to(BF)
        out = c.attend(0, q, _starts(rows), n)
        own = q.clone()
        assert torch.equal(c.attend(0, own, _starts(rows), n, out=own), out)
    rs = _starts([1, 0])
    q = torch.randn(1, 8, 128, device="cuda").to(BF)
    for kw in (dict(q=q.half()), dict(q=q.float()), dict(q=q[0]), dict(q=q[..., :64]), dict(q=q.cpu()),
               dict(row_start=rs.long()), dict(row_start=rs[:2]), dict(mask=torch.zeros(1, 1, device="cuda")),
               dict(mask=torch.zeros(2, 1, dtype=torch.int32, device="cuda")), dict(out=q[..., :64]),
               dict(lse=torch.zeros(1, 8, dtype=torch.float64, device="cuda"))):
        with pytest.raises(ValueError):
            c.attend(0, **dict(dict(q=q, row_start=rs, max_rows=1), **kw))
    for kw in (dict(layer=1), dict(max_rows=0), dict(scale=-1.0), dict(max_keys=-1)):
        with pytest.raises((P.DlmError, ValueError)):
            c.attend(**dict(dict(layer=0, q=q, row_start=rs, max_rows=1), **kw))
    with pytest.raises((P.DlmError, ValueError)):
        c.attend(0, torch.randn(1, 7, 128, device="cuda").to(BF), rs, 1)     # 7 heads over 2
    with pytest.raises(ValueError):
        P.PagedCache(1, 4, 16, 2, 64, 1, 2, device="cpu")
    with pytest.raises(ValueError):
        P.PagedCache(1, 4, 20, 2, 64, 1, 2)
    with pytest.raises(ValueError):
        P.PagedCache(1, 4, 16, 2, 64, 1, 2, k=torch.zeros(1, 4, 2, 16, 64, device="cuda"))
    e = torch.empty(0, 8, 128, dtype=BF, device="cuda")
    assert c.attend(0, e, _starts([0, 0]), 0).shape == e.shape


def test_pools_beyond_four_gigabytes():
    """Pages and layers whose byte offsets pass 2^32."""
    P = _lib()
    layers, pages, page, KV, hd = 2, 20000, 128, 8, 128          # 5.2 GB of keys a layer
    c = P.PagedCache(layers, pages, page, KV, hd, 1, 8)
    c.table[0, :4] = _ints([19999, 7, 19998, 16400])
    c.ref[_ints([19999, 7, 19998, 16400]).long()] = 1
    g = torch.Generator().manual_seed(9)
    n = 500
    k, v = (torch.randn(n, KV, hd, generator=g).to(BF) for _ in range(2))
    rs = _ints([0, n])
    c.append(1, k.cuda(), v.cuda(), rs, n)
    q = torch.randn(n, KV, hd, generator=g).to(BF)
    out = c.attend(1, q.cuda(), rs, n)
    want, mag, _ = ref.attend(q[:20], k, v, torch.ones(20, n, dtype=torch.bool), hd ** -0.5)
    h = ref.half_step(BF)
    _within(out[:20], want, h * want.abs() + (h + 2e-4) * mag, "far pages")
    assert c.commit(rs).tolist() == [1]
    f = c.compact()
    assert f.item() == 4 and sorted(c.table[0, :4].tolist()) == [0, 1, 2, 3]
    one = c.attend(1, q[:1].cuda(), _ints([0, 0]), 1)
    assert one.shape == (1, KV, hd)
    c.truncate(_ints([n - 1]))
    again = c.attend(1, q[:1].cuda(), _ints([0, 1]), 1)          # the last token is the window's
    _within(again, want[:1], h * want[:1].abs() + (h + 2e-4) * mag[:1], "far pages moved")


# ------------------------------------------------------------------ pages

def _state(c):
    return c.meta.tolist()


@pytest.mark.parametrize("seed,n_pages,page,n_seqs,width,layers,KV,hd,dtype", [
    (1, 12, 16, 4, 6, 1, 1, 64, BF), (2, 40, 16, 7, 9, 3, 2, 128, HF), (3, 300, 32, 64, 8, 2, 1, 64, BF),
    (4, 9, 128, 3, 4, 2, 3, 64, BF), (5, 5000, 16, 1000, 7, 1, 1, 64, BF)])
def test_pages_against_the_plain_reference(seed, n_pages, page, n_seqs, width, layers, KV, hd, dtype):
    """Long runs of passes, forks, truncations and compactions: tables, lengths and
    references equal the reference's, and so do the contents of every sequence."""
    P = _lib()
    rng = random.Random(seed)
    plain = ref.PlainCache(n_pages, page, n_seqs, width)
    c = P.PagedCache(layers, n_pages, page, KV, hd, n_seqs, width, dtype=dtype)
    assert _state(c) == plain.meta()
    c.k.zero_()
    c.v.zero_()
    serial = 1
    values = torch.randn(1 << 16, hd, generator=torch.Generator().manual_seed(seed)).to(dtype)
    for step in range(40 if n_seqs < 500 else 12):
        what = rng.choice(["pass", "pass", "pass", "fork", "truncate", "compact"]) if step else "pass"
        if what == "pass":
            rows = [rng.choice([0, 1, rng.randint(1, 3 * page)]) for _ in range(n_seqs)]
            if n_seqs > 500:
                rows = [r if rng.random() < 0.3 else 0 for r in rows]
            ok = c.reserve(_starts(rows))
            assert ok.tolist() == plain.reserve(rows), step
            assert _state(c) == plain.meta(), step
            T = sum(rows)
            base = serial
            serial += T
            first = [0]
            for n in rows:
                first.append(first[-1] + n)
            plain.append(rows, lambda b, i: base + first[b] + i)
            if T:
                ids = torch.arange(base, base + T) % (1 << 16)
                kv = values[ids].cuda().view(T, 1, hd).expand(T, KV, hd).contiguous()
                for layer in range(layers):
                    c.append(layer, kv * (layer + 1), kv * -(layer + 1), _starts(rows), max(rows))
            if rng.random() < 0.3:
                keep = None
            else:
                keep = [sorted(rng.sample(range(n), rng.randint(0, n))) for n in rows]
                for b, n in enumerate(rows):          # lists that do not rise, or leave the window
                    if n > 2 and rng.random() < 0.1:
                        keep[b] = rng.choice([[1, 1], [2, 0], [-1, 0], [0, n], list(range(n)) + [n]])
            if rng.random() < 0.3 and n_seqs > 1:     # a copy made between the pass's begin and its end
                s, d = rng.sample(range(n_seqs), 2)
                assert c.fork(_ints([s]), _ints([d])).tolist() == plain.fork([s], [d])
            want_ok = plain.commit(rows, keep)
            if keep is None:
                got = c.commit(_starts(rows))
            else:
                flat = [x for k in keep for x in k]
                got = c.commit(_starts(rows), keep=_ints(flat), keep_start=_starts([len(k) for k in keep]))
            assert got.tolist() == want_ok, (step, rows)
        elif what == "fork":
            m = rng.randint(0, min(6, n_seqs))
            src = [rng.randrange(-1, n_seqs + 1) for _ in range(m)]
            dst = [rng.randrange(-1, n_seqs + 1) for _ in range(m)]
            assert c.fork(_ints(src), _ints(dst)).tolist() == plain.fork(src, dst), step
        elif what == "truncate":
            new = [rng.choice([-1, 0, rng.randint(0, width * page)]) for _ in range(n_seqs)]
            c.truncate(_ints(new))
            plain.truncate(new)
        else:
            assert c.compact().item() == plain.compact(), step
        assert _state(c) == plain.meta(), (step, what)
    K, V = c.k.cpu(), c.v.cpu()
    n_checked = 0
    for b in range(n_seqs):
        for t, tag in enumerate(plain.contents(b)):
            p = plain.table[b][t // page]
            want = values[tag % (1 << 16)] if tag is not None else torch.zeros(hd, dtype=dtype)
            for layer in range(layers):
                for h in range(KV):
                    assert torch.equal(K[layer, p, h, t % page], want * (layer + 1)), (b, t, layer, h)
                    assert torch.equal(V[layer, p, h, t % page], want * -(layer + 1)), (b, t, layer, h)
            n_checked += 1
    log(f"[pages {seed}] {n_checked} tokens checked")
    c.truncate()
    assert not c.ref.any() and not c.len.any() and (c.table == -1).all()


def test_reserve_of_long_windows_and_whole_pools():
    """One sequence takes many pages at once; a pool is handed out to its last page; the
    next ones are refused whole."""
    P = _lib()
    n_pages = 9001
    c = P.PagedCache(1, n_pages, 16, 1, 64, 3, 8000)
    ok = c.reserve(_starts([16 * 7990 + 1, 16 * 1000, 16 * 20 + 5]))
    assert ok.tolist() == [1, 1, 0]
    assert c.table[0, :7991].tolist() == list(range(7991))
    assert c.table[1, :1000].tolist() == list(range(7991, 8991)) and (c.table[2] == -1).all()
    ok = c.reserve(_starts([1, 0, 160]))
    assert ok.tolist() == [1, 1, 1] and c.table[2, :10].tolist() == list(range(8991, 9001))
    assert c.reserve(_starts([0, 16 * 1000 + 1, 1])).tolist() == [1, 0, 1]
    assert c.reserve(_starts([16 * 8000 + 1, 0, 0])).tolist() == [0, 1, 1]       # past the table row
    assert (c.ref == 1).all()


def test_commit_bounds():
    """keep_start out of range, a start that falls, windows without their pages."""
    c, table = _cache([64, 64], 16, 1, 64, BF)
    before = _state(c)
    rs = _starts([8, 8])
    keep = _ints([0, 1, 2, 3, 4])
    for starts in ([0, 3, 6], [-1, 3, 5], [0, 5, 3], [2, 1, 0]):
        ok = c.commit(rs, keep=keep, keep_start=_ints(starts))
        good = [0 <= a <= b <= 5 for a, b in zip(starts, starts[1:])]
        assert [bool(x) for x in ok.tolist()] == good, starts
        c.meta.copy_(_ints(before))
    c.table[1, 0] = -1
    assert c.commit(rs).tolist() == [1, 0]
    assert c.len.tolist() == [8, 0]
    c.meta.copy_(_ints(before))
    c.len.copy_(_ints([60, -5]))
    assert c.commit(rs).tolist() == [0, 0] and c.len.tolist() == [60, -5]


def test_commit_judges_every_sequence_before_any_page_is_freed():
    """Windows that name each other's pages (tables written by hand): the first sequence
    of each pair keeps nothing and gives its page up; the second one's rows would move
    into that page, so it is left out, length and tokens."""
    P = _lib()
    B, page, hd = 512, 16, 64
    c = P.PagedCache(2, B // 2, page, 1, hd, B, 1)
    shared = torch.arange(B // 2, dtype=torch.int32).repeat_interleave(2)
    c.table.copy_(shared.view(B, 1))
    c.ref.fill_(2)
    c.k.copy_(torch.randn(c.k.shape, generator=torch.Generator().manual_seed(3)).to(BF))
    c.v.copy_(-c.k)
    k0 = c.k.clone()
    rs = _starts([4] * B)
    keep, starts = [], [0]
    for b in range(B):
        keep += [1, 3] if b % 2 else []
        starts.append(len(keep))
    ok = c.commit(rs, keep=_ints(keep), keep_start=_ints(starts))
    assert ok.tolist() == [1, 0] * (B // 2)
    assert c.len.tolist() == [0] * B and c.ref.tolist() == [1] * (B // 2)
    assert c.table[::2].flatten().tolist() == [-1] * (B // 2) and torch.equal(c.table[1::2, 0].cpu(), shared[::2])
    assert torch.equal(c.k, k0) and torch.equal(c.v, -k0)


# ------------------------------------------------------------------ together

@pytest.mark.parametrize("dtype", [BF, HF])
def test_a_tree_step_as_it_is_used(dtype):
    """Prompts, then steps of drafted trees of which a path is kept, on forked
    sequences: every result equals attention over the kept tokens alone."""
    P = _lib()
    rng = random.Random(8)
    g = torch.Generator().manual_seed(8)
    B, H, KV, hd, page, layers = 4, 8, 2, 64, 16, 2
    c = P.PagedCache(layers, 60, page, KV, hd, B, 12, dtype=dtype)
    rope = P.Rope(hd)
    w, _ = ref.frequencies(hd)
    kept = [([], [], []) for _ in range(B)]           # per sequence: k, v (layer 0) and positions so far
    h = ref.half_step(dtype)

    def step(rows, parents, pos, keep):
        T = sum(rows)
        rs = _starts(rows)
        assert c.reserve(rs).tolist() == [1] * B
        q, k, v = (torch.randn(T, n, hd, generator=g).to(dtype) for n in (H, KV, KV))
        flat = torch.tensor([p for s in pos for p in s], dtype=torch.int32)
        sees = []
        for b, n in enumerate(rows):
            see = torch.zeros(n, n, dtype=torch.bool)
            for i in range(n):
                if parents is None:
                    see[i] = True
                else:
                    if parents[b][i] >= 0:
                        see[i] = see[parents[b][i]]
                    see[i, i] = True
            sees.append(see)
        mask = None if parents is None else ref.pack_mask(sees, 1).cuda()
        for layer in range(layers):
            qr = c.append(layer, k.cuda() * (1 + layer), v.cuda(), rs, max(rows), q=q.cuda(), rope=rope, positions=flat.cuda())
            out = c.attend(layer, qr, rs, max(rows), mask=mask)
            if layer == 0:
                first = out
        kr, qr = ref.rotate(k, flat, w, 1.0, False).to(dtype), ref.rotate(q, flat, w, 1.0, False).to(dtype)
        t = 0
        for b, n in enumerate(rows):
            if n:
                ks = torch.stack(kept[b][0] + list(kr[t:t + n]))
                vs = torch.stack(kept[b][1] + list(v[t:t + n]))
                see = torch.cat([torch.ones(n, len(kept[b][0]), dtype=torch.bool), sees[b]], 1)
                want, mag, _ = ref.attend(qr[t:t + n], ks, vs, see, hd ** -0.5)
                # queries and keys are rounded on both sides; where they fall on different
                # neighbours (angles 2^-21 apart) a score moves by h of a product: 4 h
                _within(first[t:t + n], want, h * want.abs() + (6 * h + 1e-4) * mag, f"step of {n} rows")
                for i in keep[b]:
                    kept[b][0].append(kr[t + i])
                    kept[b][1].append(v[t + i])
            t += n
        if all(a == list(range(n)) for a, n in zip(keep, rows)):
            ok = c.commit(rs)
        else:
            ok = c.commit(rs, keep=_ints([i for a in keep for i in a]), keep_start=_starts([len(a) for a in keep]))
        assert ok.tolist() == [1] * B
        assert c.len.tolist() == [len(x[0]) for x in kept]

    rows = [20, 33, 0, 0]
    step(rows, None, [list(range(n)) for n in rows], [list(range(n)) for n in rows])
    assert c.fork(_ints([0, 1]), _ints([2, 3])).tolist() == [1, 1]
    for a, b in ((0, 2), (1, 3)):
        kept[b] = (list(kept[a][0]), list(kept[a][1]), [])
    for _ in range(4):
        rows = [rng.randint(1, 14) for _ in range(B)]
        parents = [[-1] + [rng.randrange(0, i) for i in range(1, n)] for n in rows]
        depth, keep = [], []
        for b, n in enumerate(rows):
            d = []
            for p in parents[b]:
                d.append(0 if p < 0 else d[p] + 1)
            depth.append([len(kept[b][0]) + x for x in d])
            path, i = [], rng.randrange(n)            # the path to some node
            while i >= 0:
                path.append(i)
                i = parents[b][i]
            keep.append(path[::-1])
        step(rows, parents, depth, keep)
    n = c.compact().item()
    assert (c.ref[:n] > 0).all() and not c.ref[n:].any()
    rows = [1, 1, 1, 1]
    step(rows, None, [[len(x[0])] for x in kept], [[0]] * B)


def test_captured_and_replayed():
    """A pass captured in a graph: replays equal the eager pass, with eager work in
    between."""
    P = _lib()
    B, H, KV, hd, page = 3, 8, 2, 128, 32
    lens, rows = [100, 700, 40], [1, 6, 40]
    c, _ = _cache([n for n in lens], page, KV, hd, BF, width=30, spare=40)
    c.k.normal_()
    c.v.normal_()
    c.len.copy_(_ints(lens))
    start = c.meta.clone()
    T = sum(rows)
    rope = P.Rope(hd, scaling="yarn", factor=4.0, original_len=512)
    src = torch.randn(T, (H + 2 * KV) * hd, device="cuda")
    q, k, v = src[:, :H * hd].view(T, H, hd), src[:, H * hd:(H + KV) * hd].view(T, KV, hd), src[:, (H + KV) * hd:].view(T, KV, hd)
    mask = torch.randint(-2 ** 31, 2 ** 31 - 1, (T, 2), device="cuda", dtype=torch.int32)
    keep, keep_start = _ints([0, 2, 5, 1, 9, 30]), _ints([0, 1, 3, 6])
    rs = _starts(rows)
    qo = torch.empty(T, H, hd, dtype=BF, device="cuda")
    out, lse = torch.empty_like(qo), torch.empty(T, H, device="cuda")
    pair = (_ints([0]), _ints([2]))

    def one():
        c.meta.copy_(start)
        ok = c.reserve(rs)
        c.append(0, k, v, rs, max(rows), q=q, rope=rope, q_out=qo)
        c.attend(0, qo, rs, max(rows), mask=mask, out=out, lse=lse)
        done = c.commit(rs, keep=keep, keep_start=keep_start)
        forked = c.fork(*pair)
        used = c.compact()
        return ok, done, forked, used

    pools = c.k.clone(), c.v.clone()
    oks = [t.clone() for t in one()]
    want = [t.clone() for t in (c.meta, c.k, c.v, out, lse)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = one()
    for _ in range(3):
        c.k.copy_(pools[0])
        c.v.copy_(pools[1])
        out.fill_(3.0)
        lse.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, oks):
            assert torch.equal(a, b)
        for a, b in zip((c.meta, c.k, c.v, out, lse), want):
            assert torch.equal(a, b)
        c.truncate()                                  # eager work on the same cache and workspaces
        c.reserve(rs)
        c.attend(0, qo, rs, max(rows), mask=mask)
        torch.cuda.synchronize()


def test_on_another_stream():
    c, _ = _cache([400, 70], 64, 4, 64, HF)
    c.k.normal_()
    c.v.normal_()
    c.len.copy_(_ints([380, 60]))
    q = torch.randn(30, 16, 64, device="cuda").half()
    rs = _starts([20, 10])
    want = c.attend(0, q, rs, 20)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = c.attend(0, q, rs, 20)
    s.synchronize()
    assert torch.equal(got, want)
