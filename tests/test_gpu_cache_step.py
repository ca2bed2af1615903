"""A model's windows behind a paged cache (dlm_cache_step) against the float64
oracle: top-1 exact where the oracle's logit margin exceeds the exemption, max
logits within 2e-2 max-abs-relative, confidences within 2e-2, on rows whose router
gap exceeds 1e-2 at every block (the parity contract of the other passes)."""

from __future__ import annotations

import numpy as np
import pytest

from tests.gpu_util import HIDDEN_TOL, MARGIN, log, max_abs_rel, need_gpu
from workloads import WORKLOADS

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


def _i32(x):
    return _torch().tensor(np.ascontiguousarray(x, dtype=np.int32), device="cuda")


def _setup(name, **over):
    need_gpu()
    import oracle
    from paper_2608_02625_amd import Refiner
    w = WORKLOADS[name]
    shape = w.model.replace(**over) if over else w.model
    log(f"[cache step setup] {name} {over}")
    return shape, Refiner(shape.as_dict(), w.weight_seed), oracle.OracleWeights(shape, w.weight_seed)


@pytest.fixture(scope="module", params=[("tiny", dict(lm_head_scale=10.0)), ("small_moe", dict(n_layers=2)),
                                        ("mini_drafter", dict(n_layers=2, vocab=4096))], ids=lambda p: p[0])
def model(request):
    name, over = request.param
    if name == "mini_drafter":
        need_gpu()
        import oracle
        from paper_2608_02625_amd import Refiner
        from workloads import MODELS
        shape = MODELS[name].replace(**over)
        return shape, Refiner(shape.as_dict(), 3), oracle.OracleWeights(shape, 3)
    return _setup(name, **over)


def _starts(rows):
    return _i32(np.concatenate([[0], np.cumsum(rows)]))


def _oracle_rows(W, tokens, positions, limit, rows):
    """Reduction and smallest router gap of `rows` of one sequence."""
    import oracle
    x, infos, _ = oracle.forward(W, tokens[None], collect=True, positions=positions, key_limit=limit)
    red = oracle.lm_head_reduce(W, x[0, rows])
    gaps = [i["route_gap"][0, rows] for i in infos if i["route_gap"] is not None]
    red["gap"] = np.min(np.stack(gaps), axis=0) if gaps else np.full(len(rows), np.inf)
    return red


def _check(what, got, want, sharp):
    top1, conf, mx = (t.cpu().numpy() for t in got)
    keep = want["gap"] > MARGIN
    ok = keep & (want["margin"] > MARGIN * sharp)
    log(f"[{what}] {ok.sum()} of {len(ok)} top-1 compared; max logit {max_abs_rel(mx[keep], want['max_logit'][keep]):.2e}, "
        f"confidence {np.abs(conf - want['conf'])[keep].max():.2e}")
    assert keep.any()
    assert np.array_equal(top1[ok], want["top1"][ok]), what
    assert max_abs_rel(mx[keep], want["max_logit"][keep]) < HIDDEN_TOL, what
    assert np.abs(conf - want["conf"])[keep].max() < HIDDEN_TOL, what


def test_prompts_then_blocks(model):
    """Ragged prompts, then blocks of a draft, of which one sequence sits one out."""
    from oracle.draft import block_key_limit
    shape, R, W = model
    rng = np.random.default_rng(5)
    prompts, blk, sharp = [19, 64, 33], 16, shape.lm_head_scale
    B = len(prompts)
    seqs = [rng.integers(0, shape.vocab - 1, size=p + 3 * blk).astype(np.int32) for p in prompts]
    for s, p in zip(seqs, prompts):
        s[p + blk::3] = shape.mask_id                 # blocks in progress hold [MASK]
    c = R.cache(40, 16, B, 10)
    at = [0] * B
    for turn in range(4):
        rows = [p if turn == 0 else blk for p in prompts]
        if turn == 2:
            rows[1] = 0
        rs = _starts(rows)
        assert c.reserve(rs).tolist() == [1] * B
        toks = np.concatenate([s[a:a + n] for s, a, n in zip(seqs, at, rows)])
        got = R.cache_step(c, _i32(toks), rs, max(rows), max_keys=max(a + n for a, n in zip(at, rows)))
        t = 0
        for b, n in enumerate(rows):
            if n:
                end = at[b] + n
                want = _oracle_rows(W, seqs[b][:end], None, block_key_limit(prompts[b], end, blk),
                                    np.arange(at[b], end))
                _check(f"turn {turn} sequence {b}", [x[t:t + n] for x in got], want, sharp)
            t += n
        assert c.commit(rs).tolist() == [1] * B
        at = [a + n for a, n in zip(at, rows)]
        assert c.len.tolist() == at


def test_alternative_blocks_of_one_pass(model):
    """Three drafts of the next block in one window, each seeing itself and the prompt;
    one is kept, and the block after it sees that one."""
    from oracle.draft import block_key_limit
    shape, R, W = model
    rng = np.random.default_rng(6)
    P, blk, C, sharp = 37, 12, 3, shape.lm_head_scale
    prompt = rng.integers(0, shape.vocab - 1, size=P).astype(np.int32)
    alts = rng.integers(0, shape.vocab - 1, size=(C, blk)).astype(np.int32)
    c = R.cache(12, 32, 2, 6)
    rs = _i32([0, P, P])
    c.reserve(rs)
    R.cache_step(c, _i32(prompt), rs, P)
    assert c.commit(rs).tolist() == [1, 1]
    rs = _i32([0, C * blk, C * blk])
    assert c.reserve(rs).tolist() == [1, 1]
    pos = np.tile(P + np.arange(blk), C)
    words = np.zeros((C * blk, 2), dtype=np.uint32)
    for i in range(C * blk):
        for j in range(i // blk * blk, i // blk * blk + blk):
            words[i, j // 32] |= np.uint32(1 << (j % 32))
    got = R.cache_step(c, _i32(alts.reshape(-1)), rs, C * blk, positions=_i32(pos), mask=_i32(words.view(np.int32)))
    for a in range(C):
        seq = np.concatenate([prompt, alts[a]])
        want = _oracle_rows(W, seq, None, block_key_limit(P, P + blk, blk), np.arange(P, P + blk))
        _check(f"draft {a}", [x[a * blk:(a + 1) * blk] for x in got], want, sharp)
    assert c.commit(rs, keep=_i32(np.arange(2 * blk, 3 * blk)), keep_start=_i32([0, blk, blk])).tolist() == [1, 1]
    assert c.len.tolist() == [P + blk, 0]
    # the kept draft goes on in a second sequence too
    assert c.fork(_i32([0]), _i32([1])).tolist() == [1]
    rows = [5, 9]
    rs = _starts(rows)
    assert c.reserve(rs).tolist() == [1, 1]
    more = rng.integers(0, shape.vocab - 1, size=14).astype(np.int32)
    got = R.cache_step(c, _i32(more), rs, 9)
    t = 0
    for n in rows:
        seq = np.concatenate([prompt, alts[2], more[t:t + n]])
        want = _oracle_rows(W, seq, None, block_key_limit(P, len(seq), blk), np.arange(P + blk, P + blk + n))
        _check(f"{n} rows after it", [x[t:t + n] for x in got], want, sharp)
        t += n


def test_the_cache_step_agrees_with_the_drafting_step(model):
    """The same block through dlm_draft_step's own caches: equal up to the roundings."""
    torch = _torch()
    shape, R, W = model
    rng = np.random.default_rng(7)
    P, blk = 48, 16
    toks = rng.integers(0, shape.vocab - 1, size=(1, P + 2 * blk)).astype(np.int32)
    toks[0, P + blk + 1::2] = shape.mask_id
    c = R.cache(8, 16, 1, 8)
    for a, n in ((0, P), (P, blk)):
        rs = _i32([0, n])
        c.reserve(rs)
        R.cache_step(c, _i32(toks[0, a:a + n]), rs, n)
        c.commit(rs)
    rs = _i32([0, blk])
    c.reserve(rs)
    top1, conf, mx = R.cache_step(c, _i32(toks[0, P + blk:]), rs, blk)
    t1 = torch.empty(1, blk, dtype=torch.int32, device="cuda")
    cf, ml = (torch.empty(1, blk, dtype=torch.float32, device="cuda") for _ in range(2))
    R.draft_step(_i32(toks), P, blk, 1, 4, 2.0, top1=t1, conf=cf, max_logit=ml)
    err = (ml[0] - mx).abs().max() / mx.abs().max()
    log(f"max logits {err.item():.2e}, confidences {(cf[0] - conf).abs().max().item():.2e} apart")
    assert err < HIDDEN_TOL and (cf[0] - conf).abs().max() < HIDDEN_TOL


def test_tokens_rows_and_replays():
    """Invalid ids are counted and read as valid ones, rows behind the last window do
    not disturb others, and a captured step replays to the same bits."""
    torch = _torch()
    shape, R, _ = _setup("small_moe", n_layers=2)
    rng = np.random.default_rng(8)
    toks = rng.integers(0, shape.vocab - 1, size=40).astype(np.int32)
    c = R.cache(8, 16, 2, 4)
    rs = _i32([0, 20, 33])
    c.reserve(rs)
    bad = torch.empty(1, dtype=torch.int32, device="cuda")
    ref = [x.clone() for x in R.cache_step(c, _i32(toks[:33]), rs, 20, n_invalid=bad)]
    assert bad.item() == 0
    got = R.cache_step(c, _i32(toks), rs, 20, n_invalid=bad)
    for a, b in zip(got, ref):
        assert torch.equal(a[:33], b)
    wrong = toks[:33].copy()
    wrong[[3, 30]] = [-1, shape.vocab]
    got = R.cache_step(c, _i32(wrong), rs, 20, n_invalid=bad)
    assert bad.item() == 2 and all(x[13].isfinite() for x in got)
    src = _i32(toks[:33])
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        R.cache_step(c, src, rs, 20)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = R.cache_step(c, src, rs, 20)
    for _ in range(3):
        for x in out:
            x.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, ref):
            assert torch.equal(a, b)
        R.cache_step(c, _i32(wrong), rs, 20)          # eager work on the same workspace
        torch.cuda.synchronize()
    other = _setup("tiny")[1]
    with pytest.raises(ValueError):
        other.cache_step(c, src, rs, 20)              # a cache of another model
    for kw in (dict(tokens=src.long()), dict(row_start=rs[:2]), dict(positions=src[:3]),
               dict(mask=torch.zeros(2, 1, dtype=torch.int32, device="cuda")), dict(max_rows=0)):
        with pytest.raises(ValueError):
            R.cache_step(**dict(dict(cache=c, tokens=src, row_start=rs, max_rows=20), **kw))


def test_steps_of_many_sizes_share_workspaces_and_refuse_other_devices():
    """Packed rows come in any number: their workspaces are few.  Host tensors are
    refused before anything runs."""
    torch = _torch()
    shape, R, _ = _setup("tiny")
    c = R.cache(16, 16, 2, 4)
    toks = _i32(np.arange(100, dtype=np.int32) % shape.vocab)
    first = {}
    for rows in list(range(1, 41)) + [64, 100]:
        rs = _i32([0, (rows + 1) // 2, rows])
        c.truncate()
        assert c.reserve(rs).tolist() == [1, 1]
        out = R.cache_step(c, toks[:rows], rs, 50)
        first[rows] = [x.clone() for x in out]
    sizes = {ws.data_ptr(): ws.numel() for ws in R._ws.values()}
    assert len(sizes) <= 10 and sum(sizes.values()) <= 4 * max(sizes.values())
    for rows in (40, 1, 100, 7):                      # again, after others have used them
        rs = _i32([0, (rows + 1) // 2, rows])
        c.truncate()
        c.reserve(rs)
        assert all(torch.equal(a, b) for a, b in zip(R.cache_step(c, toks[:rows], rs, 50), first[rows]))
    rs = _i32([0, 2, 4])
    host = torch.zeros(4, dtype=torch.int32)
    for kw in (dict(tokens=host), dict(row_start=torch.tensor([0, 2, 4], dtype=torch.int32)), dict(positions=host),
               dict(mask=host.view(4, 1)), dict(n_invalid=host[:1])):
        with pytest.raises(ValueError):
            R.cache_step(**dict(dict(cache=c, tokens=toks[:4], row_start=rs, max_rows=2), **kw))


def test_top1_of_the_cache_step_and_the_drafting_step(model):
    """The same block both ways: equal top-1, and the oracle's, where its logit margin
    exceeds the exemption."""
    from oracle.draft import block_key_limit
    torch = _torch()
    shape, R, W = model
    rng = np.random.default_rng(9)
    P, blk = 48, 16
    for seed in range(3):
        toks = rng.integers(0, shape.vocab - 1, size=(1, P + blk)).astype(np.int32)
        toks[0, P + 1 + seed::2] = shape.mask_id
        c = R.cache(8, 16, 1, 8)
        for a, n in ((0, P), (P, blk)):
            rs = _i32([0, n])
            assert c.reserve(rs).tolist() == [1]
            top1, conf, mx = R.cache_step(c, _i32(toks[0, a:a + n]), rs, n)
            assert c.commit(rs).tolist() == [1]
        t1 = torch.empty(1, blk, dtype=torch.int32, device="cuda")
        R.draft_step(_i32(toks), P, blk, 0, 4, 2.0, top1=t1)
        want = _oracle_rows(W, toks[0], None, block_key_limit(P, P + blk, blk), np.arange(P, P + blk))
        _check(f"block {seed}", (top1, conf, mx), want, shape.lm_head_scale)
        sure = (want["gap"] > MARGIN) & (want["margin"] > MARGIN * shape.lm_head_scale)
        log(f"[draft step {seed}] {sure.sum()} of {blk} top-1 compared")
        assert sure.any()
        assert np.array_equal(t1[0].cpu().numpy()[sure], top1.cpu().numpy()[sure])
