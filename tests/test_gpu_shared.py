"""Attention over shared prefixes (PagedCache.share, attend) on the GPU against float64
references on the CPU, whatever the tables share.

Tolerances as those of the plain attention: probabilities are rounded to the cache's type
(half a step h of the sum of p |v|), the result once more (h of it); float32 scores of up
to S differ by at most hd 2^-24 S and their exponentials by as much, relative; joining what
a prefix left adds a few 2^-24 of the sum of p |v|, within the 1e-5 of it that parts have."""

from __future__ import annotations

import math
import random

import pytest
import torch

from tests import cache_ref as ref
from tests.gpu_util import log, need_gpu
from tests.test_gpu_cache import _ints, _see, _starts, _within

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


class Case:
    """Sequences of groups (numbers; -1: by itself) with `whole` pages in common, their
    tokens on the CPU and in the pool, places without a token NaN.  Tables are so wide that
    a call without a bound on the keys shares, whatever the lengths."""

    def __init__(self, dtype, H, KV, hd, page, group, whole, lens, rows, kind="full", seed=0, width=0, layers=1):
        from paper_2608_02625_amd import PagedCache
        g, rng = torch.Generator().manual_seed(seed), random.Random(seed)
        self.dtype, self.H, self.KV, self.hd, self.page, self.rows, self.lens = dtype, H, KV, hd, page, rows, lens
        B = len(lens)
        need = [-(-(n + r) // page) for n, r in zip(lens, rows)]
        values = sum(rows) * H * hd
        width = max(max(need), 1) + width + int((48e6 + 1000 * values) / (4 * KV * hd)) // page + 1
        n_pages = sum(need) + 4
        order = list(range(n_pages))
        rng.shuffle(order)
        c = self.c = PagedCache(layers, n_pages, page, KV, hd, B, width, dtype=dtype)
        c.k.fill_(math.nan)
        c.v.fill_(math.nan)
        tables, front = torch.full((B, width), -1, dtype=torch.int32), {}
        k, v = c.k[0].cpu(), c.v[0].cpu()
        self.keys, self.values = [], []
        for b in range(B):
            mine = []
            if group[b] >= 0:
                have = front.setdefault(group[b], [])
                while len(have) < min(whole[group[b]], need[b]):
                    have.append(order.pop())
                mine = have[:min(whole[group[b]], need[b])]
            pages = mine + [order.pop() for _ in range(need[b] - len(mine))]
            tables[b, :len(pages)] = torch.tensor(pages, dtype=torch.int32)
            ks, vs = [torch.zeros(lens[b] + rows[b], KV, hd, dtype=dtype) for _ in range(2)]
            for e, p in enumerate(pages):
                n = min(page, lens[b] + rows[b] - e * page)
                fresh = torch.isnan(k[p, :, :n].float()).any(-1).any(0)
                for pool in (k, v):
                    pool[p, :, :n][:, fresh] = torch.randn(KV, int(fresh.sum()), hd, generator=g).to(dtype)
                ks[e * page:e * page + n], vs[e * page:e * page + n] = k[p, :, :n].transpose(0, 1), v[p, :, :n].transpose(0, 1)
            self.keys.append(ks)
            self.values.append(vs)
        c.k[0].copy_(k)
        c.v[0].copy_(v)
        c.table.copy_(tables)
        c.len.copy_(_ints(lens))
        self.group, self.starts = _ints(group), _starts(rows)
        T = self.T = sum(rows)
        self.q = torch.randn(T, H, hd, generator=g).to(dtype)
        self.sees = [_see(kind, n, rng) for n in rows]
        words = (max(rows) + 31) // 32
        self.mask = None if kind == "full" else ref.pack_mask(self.sees, words).cuda()
        self.kind = kind

    def run(self, max_group_rows=None, max_keys=0, check=True, gone=()):
        c, T, top = self.c, self.T, max(self.rows)
        share = c.share(self.starts, self.group, T, top, max_group_rows)
        out = torch.full((T + 2, self.H, self.hd), 5.0, dtype=self.dtype, device="cuda")
        lse = torch.full((T, self.H), 5.0, device="cuda")
        most = max_keys
        got = c.attend(0, self.q.cuda(), self.starts, top, mask=self.mask, max_keys=most, out=out[1:T + 1], lse=lse, share=share)
        assert (out[0] == 5.0).all() and (out[T + 1] == 5.0).all()
        if check:
            self.check(got, lse, most, gone)
        skip = share.data[4 * c.n_seqs:8 * c.n_seqs:4].tolist()
        return got, lse, skip

    def check(self, got, lse, most, gone):
        h, s, t = ref.half_step(self.dtype), self.hd ** -0.5, 0
        for b, n in enumerate(self.rows):
            if n == 0:
                continue
            see = torch.cat([torch.ones(n, self.lens[b], dtype=torch.bool), self.sees[b]], 1)
            see[:, most if most else see.shape[1]:] = False
            for i in range(see.shape[1]):
                if (b, i // self.page) in gone:
                    see[:, i] = False
            q = self.q[t:t + n]
            want, mag, want_lse = ref.attend(q, self.keys[b], self.values[b], see, s)
            S = s * q.abs().double().amax() * self.keys[b].abs().double().amax() * self.hd
            e = self.hd * 2.0 ** -24 * float(S) / 4   # products are of random sign: a quarter of the worst case
            tol = h * want.abs() + (h + e + 1e-5) * mag + ref.half_subnormal(self.dtype)
            _within(got[t:t + n], want, tol, f"shared {self.dtype} {self.H}/{self.KV}x{self.hd} page {self.page} seq {b}")
            _within(lse[t:t + n], want_lse, (e + 1e-5) * torch.ones_like(want_lse)
                    + 2.0 ** -22 * want_lse.abs().nan_to_num(0, 0, 0), "lse")
            t += n


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("H,KV,hd,page", [(4, 4, 64, 16), (16, 4, 128, 64), (6, 2, 128, 32), (5, 1, 64, 128)])
@pytest.mark.parametrize("tokens,tails,rows,kind", [
    (300, [1, 2, 40, 0], [1, 1, 1, 1], "full"),
    (130, [5, 0, 70, 200, 3], [3, 1, 0, 5, 2], "tree"),
    (513, [60, 61, 62], [7, 12, 1], "random"),
    (64, [0, 0], [1, 1], "full"),
    (31, [100, 100], [2, 2], "chain")])
def test_one_group(dtype, H, KV, hd, page, tokens, tails, rows, kind):
    whole = tokens // page
    case = Case(dtype, H, KV, hd, page, [2 % len(rows)] * len(rows), {2 % len(rows): whole}, [tokens + x for x in tails], rows, kind,
                seed=tokens + hd)
    _, _, skip = case.run()
    want = whole * page // 32 * 32
    for b, n in enumerate(rows):
        assert skip[b] == (want if n else 0)


@pytest.mark.parametrize("dtype,H,KV,hd,page,groups,members,tokens,tail,rows,kind", [
    (BF, 16, 4, 128, 64, 1, 40, 5000, 700, 1, "full"), (HF, 8, 8, 64, 16, 3, 7, 1500, 90, 2, "chain"),
    (BF, 32, 8, 128, 128, 2, 9, 2600, 300, 13, "tree"), (BF, 4, 1, 64, 32, 5, 30, 333, 40, 4, "tree"),
    (HF, 16, 4, 128, 64, 1, 12, 3000, 2500, 8, "random"), (BF, 4, 4, 64, 16, 200, 3, 70, 9, 1, "full"),
    (BF, 8, 1, 128, 32, 2, 6, 800, 100, 16, "tree"), (BF, 2, 2, 64, 16, 4, 3, 200, 60, 100, "blocks")])
def test_groups(dtype, H, KV, hd, page, groups, members, tokens, tail, rows, kind):
    """Several groups whose members lie anywhere, some idle, some alone; long prefixes are
    split and joined; again gives the same bits."""
    rng = random.Random(groups * 31 + members)
    group = [g for g in range(groups) for _ in range(members)] + [-1, -7, 1 << 30][:members % 4]
    rng.shuffle(group)
    prefix = [rng.randint(tokens // 2, tokens) for _ in range(groups)]
    lens = [(prefix[g] if 0 <= g < groups else rng.randint(0, tokens)) + rng.randint(0, tail) for g in group]
    n = [rng.choice([rows, rng.randint(1, rows), 0 if rng.random() < 0.2 else rows]) for _ in group]
    n[0] = rows
    group = [g if g < groups else -1 for g in group]
    case = Case(dtype, H, KV, hd, page, group, [p // page for p in prefix], lens, n, kind, seed=members)
    by_group = [sum(r for r, x in zip(n, group) if x == g) for g in range(groups)]
    got, lse, skip = case.run(max(by_group))
    for b, g in enumerate(group):
        alone = g < 0 or n[b] == 0 or sum(1 for x, r in zip(group, n) if x == g and r) < 2
        assert skip[b] == (0 if alone else prefix[g] // page * page // 32 * 32)
    again, lse2, _ = case.run(max(by_group), check=False)
    assert torch.equal(got, again) and torch.equal(lse, lse2)
    case.run()                                        # no bound but the rows
    case.run(max(by_group), max(a + b for a, b in zip(lens, n)))      # as it pays
    _, _, skip = case.run(max(by_group) - 1)          # the largest group has more rows than it says
    assert any(skip) == any(s for s, g in zip(case.run(max(by_group), check=False)[2], group)
                            if g >= 0 and by_group[g] < max(by_group))


def test_tables_that_share_less_than_their_groups_say():
    """Nothing in common, a shorter member, another page in the middle, a page missing."""
    page, hd = 32, 64
    base = dict(dtype=BF, H=4, KV=2, hd=hd, page=page, group=[1, 1, 1], whole={1: 6}, lens=[200, 210, 199], rows=[1, 2, 1])
    assert Case(**base).run()[2] == [192] * 3
    assert Case(**{**base, "lens": [200, 70, 199]}).run()[2] == [64] * 3
    assert Case(**{**base, "lens": [200, 0, 199]}).run()[2] == [0] * 3
    assert Case(**{**base, "lens": [200, 31, 199]}).run()[2] == [0] * 3
    assert Case(**{**base, "whole": {1: 0}}).run()[2] == [0] * 3
    case = Case(**base, width=3)
    a, b = case.c.table[1, 2].item(), case.c.table[1, 6].item()
    case.c.table[1, 2] = b                            # a page of its own in the middle of the prefix
    case.keys[1], case.values[1] = case.keys[1].clone(), case.values[1].clone()
    fill = [torch.randn(2, page, hd).to(BF) for _ in range(2)]
    case.c.k[0, b], case.c.v[0, b] = fill[0].cuda(), fill[1].cuda()
    for e in (2, 6):
        n = min(page, 212 - e * page)
        for have, x in ((case.keys, fill[0]), (case.values, fill[1])):
            have[1][e * page:e * page + n] = x[:, :n].transpose(0, 1)
    assert case.run()[2] == [64] * 3
    for bad in (-1, 1 << 20, a):
        case = Case(**base)
        old = case.c.table[:, 3].clone()
        if bad == a:
            case.c.table[0, 3] = -1
            gone = {(0, 3)}
        else:
            case.c.table[:, 3] = bad
            gone = {(s, 3) for s in range(3)}
        assert case.run(gone=gone)[2] == [96] * 3     # found page by page, up to the missing one
        case.c.table[:, 3] = old


def test_bounds_on_keys_and_row_starts():
    base = dict(dtype=BF, H=8, KV=2, hd=128, page=16, group=[0, 0, 0], whole={0: 20}, lens=[330, 350, 340], rows=[2, 1, 3])
    case = Case(**base)
    for most in (0, 353, 345, 330, 100, 33, 32, 5, 1):
        case.run(max_keys=most)
    # as many sequences as it takes to share under a bound below the prefix
    n, t = 60, 3000
    many = Case(BF, 16, 16, 64, 64, [0] * n, {0: 46}, [t + b for b in range(n)], [1] * n, seed=2)
    for most in (t + n + 1, 2999, 1985, 1024, 1000):
        many.run(max_keys=most)
    # Row starts that fall or overlap are not allowed; they reach no memory of others.
    guard = torch.full((400, 8, 128), 5.0, dtype=BF, device="cuda")
    q = torch.randn(200, 8, 128, device="cuda").to(BF)
    for starts in ([0, 200, 0, 200], [-5, 3, 900, 2], [0, 0, 200, 0], [200, 0, 0, 0]):
        for top in (16, 200):
            s = case.c.share(_ints(starts), case.group, 200, top)
            case.c.attend(0, q, _ints(starts), top, out=guard[100:300], share=s)
    # what another pass left in a share reaches no memory of others either
    s.data.fill_(1 << 30)
    case.c.attend(0, q, _ints([0, 2, 3, 6]), 200, out=guard[100:300], share=s)
    s = case.c.share(_ints([0, 2, 3, 6]), case.group, 200, 3)
    for word in (-1, 7, 1 << 30, -(1 << 31)):
        s.data.fill_(word)
        case.c.attend(0, q, _ints([0, 2, 3, 6]), 3, out=guard[100:300], share=s)
    assert (guard[:100] == 5).all() and (guard[300:] == 5).all()


def test_what_a_row_does_not_see_does_not_change_it():
    """Infinities and NaN in one sequence's own tokens stay in its rows; in the shared ones
    they are in every row."""
    case = Case(BF, 4, 2, 64, 16, [0] * 4, {0: 9}, [150, 160, 155, 170], [3, 1, 2, 1], "tree", seed=3)
    clean, _, skip = case.run()
    assert skip == [128] * 4
    p, c = case.c.table[1, 9].item(), case.c
    for value in (math.inf, math.nan):
        old = c.v[0, p, 0, 3, 5].clone()
        c.v[0, p, 0, 3, 5] = value
        got = case.run(check=False)[0]
        same = (got == clean).all(-1).all(-1)
        assert same.tolist() == [True] * 3 + [False] + [True] * 3
        assert bool((got[3, :2, 5].isnan() | got[3, :2, 5].isinf()).all()) and torch.equal(got[3, 2:], clean[3, 2:])
        c.v[0, p, 0, 3, 5] = old
        p0 = c.table[0, 2].item()
        old = c.v[0, p0, 1, 0, 7].clone()
        c.v[0, p0, 1, 0, 7] = value
        got = case.run(check=False)[0]
        assert not bool(got[:, 2:, 7].isfinite().any()) and torch.equal(got[:, :2], clean[:, :2])
        c.v[0, p0, 1, 0, 7] = old


def test_extreme_scores():
    for rows in (1, 9):
        case = Case(HF, 4, 2, 64, 16, [0] * 5, {0: 18}, [300, 320, 310, 290, 335], [rows] * 5, "chain", seed=5)
        case.q = (case.q * 100).to(HF)
        case.run()


def test_forks_as_they_are_used():
    """A prompt, copies of it that go on in different ways, a pass in every layer, in place,
    and refusals of what has become stale."""
    from paper_2608_02625_amd import PagedCache
    g = torch.Generator().manual_seed(9)
    H, KV, hd, page, L, B = 8, 2, 64, 16, 3, 4
    c = PagedCache(L, 64, page, KV, hd, B, 9000)      # so wide that a call without a bound on its keys shares
    groups = _ints([0] * B)
    keys, values = [[] for _ in range(B)], [[] for _ in range(B)]

    def append(rows):
        T = sum(rows)
        starts = _starts(rows)
        assert bool(c.reserve(starts).all())
        k, v = [torch.randn(L, T, KV, hd, generator=g).to(BF) for _ in range(2)]
        for layer in range(L):
            c.append(layer, k[layer].cuda(), v[layer].cuda(), starts, max(rows))
        t = 0
        for b, n in enumerate(rows):
            keys[b].append(k[:, t:t + n])
            values[b].append(v[:, t:t + n])
            t += n
        return starts, T

    starts, _ = append([75, 0, 0, 0])
    c.commit(starts)
    assert c.fork(_ints([0, 0, 0]), _ints([1, 2, 3])).tolist() == [1, 1, 1]
    for b in (1, 2, 3):
        keys[b], values[b] = list(keys[0]), list(values[0])
    for rows in ([1, 1, 1, 1], [2, 1, 0, 5], [30, 1, 1, 2]):
        starts, T = append(rows)
        share = c.share(starts, groups, T, max(rows))
        assert share.data[4 * B:8 * B:4].tolist() == [64 if n else 0 for n in rows]
        q = torch.randn(L, T, H, hd, generator=g).to(BF)
        for layer in range(L):
            x = q[layer].cuda()
            c.attend(layer, x, starts, max(rows), out=x, share=share)
            t = 0
            for b, n in enumerate(rows):
                if n:
                    k, v = torch.cat(keys[b], 1)[layer], torch.cat(values[b], 1)[layer]
                    see = torch.ones(n, k.shape[0], dtype=torch.bool)
                    want, mag, _ = ref.attend(q[layer, t:t + n], k, v, see, hd ** -0.5)
                    h = ref.half_step(BF)
                    _within(x[t:t + n], want, h * want.abs() + (h + 1e-4) * mag + 1e-30, f"layer {layer} sequence {b}")
                t += n
        with pytest.raises(ValueError):
            c.attend(0, q[0].cuda(), starts, max(rows) + 1, share=share)
        with pytest.raises(ValueError):
            c.attend(0, torch.cat([q[0], q[0]]).cuda(), starts, max(rows), share=share)
        c.commit(starts)
        with pytest.raises(ValueError):
            c.attend(0, q[0].cuda(), starts, max(rows), share=share)
    for bad in (groups.long(), groups[:2], groups.cpu()):
        with pytest.raises(ValueError):
            c.share(starts, bad, 5, 3)
    with pytest.raises(ValueError):
        c.share(starts, groups, -1, 3)


def test_captured_and_on_another_stream():
    case = Case(BF, 16, 4, 128, 64, [0, 1, 0, 1, 0, -1], [40, 3], [2600, 200, 2700, 250, 2650, 90], [2, 1, 1, 2, 1, 1], seed=13)
    want, _, skip = case.run()
    assert skip == [2560, 192, 2560, 192, 2560, 0]
    c, q, T = case.c, case.q.cuda(), case.T
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        share = c.share(case.starts, case.group, T, 2)
        got = c.attend(0, q, case.starts, 2, share=share)
    side.synchronize()
    assert torch.equal(got, want)
    out = torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        share = c.share(case.starts, case.group, T, 2)
        c.attend(0, q, case.starts, 2, out=out, share=share)
    for k in range(3):
        out.fill_(0)
        q.copy_(case.q.roll(k, 0))
        c.len.copy_(_ints([n - 70 * k if n > 300 else n for n in case.lens]))
        graph.replay()
        torch.cuda.synchronize()
        share = c.share(case.starts, case.group, T, 2)
        assert torch.equal(out, c.attend(0, q, case.starts, 2, share=share)), k
        log(f"[replay {k}] {share.data[24:48:4].tolist()}")
