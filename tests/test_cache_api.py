"""CPU checks of the rotary positions' and the paged cache's C ABI: frequencies,
sizes, refusals (nothing is launched), and the plain reference's own rules."""

from __future__ import annotations

import ctypes
import math
import random

import pytest

from tests.cache_ref import PlainCache, frequencies


def _lib():
    from paper_2608_02625_amd import _lib as L
    return L, L.load()


def _spec(L, **over):
    d = dict(head_dim=128, rot_dim=128, interleaved=0, scaling=0, original_len=0, scale=0.0, theta=10000.0, factor=1.0,
             beta_slow=1.0, beta_fast=32.0)
    d.update(over)
    return L.DlmRopeSpec(*(d[f] for f, _ in L.DlmRopeSpec._fields_))


@pytest.mark.parametrize("rot,theta,scaling,factor,original", [
    (128, 10000.0, None, 1.0, 0), (64, 500000.0, None, 1.0, 0), (2, 10000.0, None, 1.0, 0),
    (128, 10000.0, "linear", 4.0, 0), (96, 10000.0, "ntk", 8.0, 0), (128, 10000.0, "yarn", 8.0, 4096),
    (50, 500000.0, "yarn", 1.0, 8192), (256, 0.5, None, 1.0, 0)])
def test_phases_are_the_frequencies_in_turns(rot, theta, scaling, factor, original):
    L, lib = _lib()
    kind = {None: 0, "linear": 1, "ntk": 2, "yarn": 3}[scaling]
    r = L.DlmRope()
    spec = _spec(L, head_dim=256, rot_dim=rot, theta=theta, scaling=kind, factor=factor, original_len=original)
    assert lib.dlm_rope_init(ctypes.byref(spec), ctypes.byref(r)) == 0
    w, scale = frequencies(rot, theta, scaling, factor, original)
    assert (r.head_dim, r.rot_dim, r.interleaved) == (256, rot, 0)
    assert abs(r.scale - scale) <= 2 ** -24 * scale
    for i, x in enumerate(w):
        turns = x / (2 * math.pi)
        got = r.phase[i] / 2.0 ** 64
        # the reference's own powers and quotients are off by a few 2^-53
        assert abs(got - (turns - math.floor(turns))) <= 2 ** -48 * max(1.0, turns), i
    assert all(r.phase[i] == 0 for i in range(rot // 2, 128))


@pytest.mark.parametrize("over,word", [
    (dict(head_dim=0), "head_dim"), (dict(head_dim=258), "head_dim"), (dict(rot_dim=0), "rot_dim"),
    (dict(rot_dim=63), "rot_dim"), (dict(rot_dim=130), "rot_dim"), (dict(scaling=4), "scaling"),
    (dict(scaling=-1), "scaling"), (dict(theta=0.0), "theta"), (dict(theta=math.nan), "theta"),
    (dict(theta=math.inf), "theta"), (dict(scale=-1.0), "scale"), (dict(scale=math.nan), "scale"),
    (dict(scaling=1, factor=0.5), "factor"), (dict(scaling=1, factor=math.nan), "factor"),
    (dict(scaling=2, rot_dim=2, factor=2.0), "rot_dim"), (dict(scaling=3, factor=2.0), "original_len"),
    (dict(scaling=3, factor=2.0, original_len=64, beta_slow=32.0), "beta"),
    (dict(scaling=3, factor=2.0, original_len=64, beta_fast=math.inf), "beta")])
def test_rope_refusals(over, word):
    L, lib = _lib()
    r = L.DlmRope()
    r.rot_dim = 77
    spec = _spec(L, **over)
    assert lib.dlm_rope_init(ctypes.byref(spec), ctypes.byref(r)) == -1
    assert word.encode() in lib.dlm_last_error()
    assert r.rot_dim == 77                              # nothing written


FAKE = 1 << 20                                          # an address that no refused call may touch


def _cache(L, **over):
    d = dict(dtype=0, n_layers=2, n_pages=8, page_len=32, n_kv_heads=4, head_dim=64, n_seqs=3, max_pages=4, d_k=FAKE,
             d_v=FAKE, d_ref=FAKE, d_len=FAKE, d_table=FAKE)
    d.update(over)
    return L.DlmCache(*(d[f] for f, _ in L.DlmCache._fields_))


def _rope(L, lib, **over):
    r = L.DlmRope()
    spec = _spec(L, head_dim=64, rot_dim=64, **over)
    assert lib.dlm_rope_init(ctypes.byref(spec), ctypes.byref(r)) == 0
    return r


def _refused(lib, status, word, code=-1):
    assert status == code, (status, lib.dlm_last_error())
    assert word.encode() in lib.dlm_last_error(), lib.dlm_last_error()


BAD_CACHES = [(dict(dtype=2), "dtype"), (dict(head_dim=96), "head_dim"), (dict(page_len=48), "page_len"),
              (dict(page_len=256), "page_len"), (dict(page_len=0), "page_len"), (dict(n_layers=0), "n_layers"),
              (dict(n_pages=0), "n_pages"), (dict(n_pages=(1 << 20) + 1), "n_pages"), (dict(n_kv_heads=0), "n_kv_heads"),
              (dict(n_kv_heads=129), "n_kv_heads"), (dict(n_seqs=0), "n_seqs"), (dict(n_seqs=1025), "n_seqs"),
              (dict(max_pages=0), "max_pages"), (dict(max_pages=1 << 30), "max_pages")]
BAD_BUFFERS = [(dict(d_k=None), "NULL"), (dict(d_v=None), "NULL"), (dict(d_ref=None), "NULL"),
               (dict(d_len=None), "NULL"), (dict(d_table=None), "NULL"), (dict(d_k=FAKE + 64), "256-byte"),
               (dict(d_v=FAKE + 128), "256-byte"), (dict(d_table=FAKE + 2), "4-byte")]


def _calls(lib, c):
    big = 1 << 40
    return {
        "reset": lambda: lib.dlm_cache_reset(c, None),
        "reserve": lambda: lib.dlm_cache_reserve(c, FAKE, 4, None, FAKE, big, None),
        "append": lambda: lib.dlm_cache_append(c, 0, FAKE, 4, 4, 0, FAKE, 256, FAKE, 256, None, None, 0, None, 0, None, 0,
                                               None),
        "attend": lambda: lib.dlm_cache_attend(c, 0, FAKE, 4, 4, 0, 8, FAKE, 512, None, 0, 0.0, FAKE, 512, None, FAKE, big,
                                               None),
        "commit": lambda: lib.dlm_cache_commit(c, FAKE, 4, None, None, 0, None, None),
        "fork": lambda: lib.dlm_cache_fork(c, 1, FAKE, FAKE, None, None),
        "truncate": lambda: lib.dlm_cache_truncate(c, None, None),
        "compact": lambda: lib.dlm_cache_compact(c, None, FAKE, big, None),
    }


@pytest.mark.parametrize("over,word", BAD_CACHES + BAD_BUFFERS)
def test_every_call_refuses_an_unsound_cache(over, word):
    L, lib = _lib()
    c = _cache(L, **over)
    for name, call in _calls(lib, ctypes.byref(c)).items():
        _refused(lib, call(), word)
    if (over, word) in BAD_CACHES:
        assert lib.dlm_cache_workspace_bytes(ctypes.byref(c), 4, 4, 8) == 0
    for call in _calls(lib, None).values():
        _refused(lib, call(), "cache is NULL")


def test_append_refusals():
    L, lib = _lib()
    c, r = ctypes.byref(_cache(L)), _rope(L, lib)
    other = L.DlmRope()
    spec = _spec(L)
    assert lib.dlm_rope_init(ctypes.byref(spec), ctypes.byref(other)) == 0

    def call(layer=0, starts=FAKE, total=4, most=4, src=0, k=FAKE, ks=256, v=FAKE, vs=256, rope=None, heads=8, q=FAKE,
             qs=512, qo=FAKE, qos=512):
        return lib.dlm_cache_append(c, layer, starts, total, most, src, k, ks, v, vs, rope, None, heads, q, qs, qo, qos, None)

    for kw, word in [(dict(layer=-1), "layer"), (dict(layer=2), "layer"), (dict(starts=None), "row_start"),
                     (dict(total=-1), "total_rows"), (dict(most=-1), "max_rows"), (dict(most=0), "max_rows"),
                     (dict(total=(1 << 24) + 1), "total_rows"), (dict(src=1), "src_dtype"), (dict(src=7), "src_dtype"),
                     (dict(k=None), "NULL"), (dict(v=None), "NULL"), (dict(ks=255), "stride"), (dict(vs=0), "stride"),
                     (dict(k=FAKE + 1), "aligned"), (dict(src=2, v=FAKE + 2), "aligned"), (dict(heads=0), "n_heads"),
                     (dict(qo=None), "q_out"), (dict(qs=511), "q_stride"), (dict(qos=511), "q_stride"),
                     (dict(q=FAKE + 1), "aligned"), (dict(src=2), "in place"), (dict(qs=520), "in place"),
                     (dict(rope=ctypes.byref(L.DlmRope())), "dlm_rope_init"),
                     (dict(rope=ctypes.byref(other)), "head_dim")]:
        _refused(lib, call(**kw), word)
    assert call(total=0, most=0, rope=ctypes.byref(r)) == 0      # nothing to do


def test_append_and_rope_limits():
    """More work than a call may ask for; strides whose products pass 64 bits."""
    L, lib = _lib()
    many = ctypes.byref(_cache(L, n_seqs=1024))
    for heads, rows, q in ((16, 1 << 20, FAKE), (0, 1 << 24, None)):
        _refused(lib, lib.dlm_cache_append(many, 0, FAKE, rows, rows, 0, FAKE, 256, FAKE, 256, None, None, heads, q,
                                           heads * 64, q, heads * 64, None), "2^33")
    r = ctypes.byref(_rope(L, lib))
    for yr, yh in ((1 << 62, 1 << 62), ((1 << 63) - 1, 1 << 61)):
        _refused(lib, lib.dlm_rope_apply(r, 0, 1 << 30, 5, FAKE, 0, 0, 2 * FAKE, yr, yh, FAKE, 0, None), "overlap")


def test_attend_refusals():
    L, lib = _lib()
    c = ctypes.byref(_cache(L))
    need = lib.dlm_cache_workspace_bytes(c, 4, 4, 8)
    assert need > 0 and lib.dlm_cache_workspace_bytes(c, 4, 4, 6) == 0       # 6 heads over 4

    def call(layer=0, starts=FAKE, total=4, most=4, keys=0, heads=8, q=FAKE, qs=512, mask=None, words=0, scale=0.0,
             o=2 * FAKE, os=512, lse=None, ws=FAKE, size=need):
        return lib.dlm_cache_attend(c, layer, starts, total, most, keys, heads, q, qs, mask, words, scale, o, os, lse, ws,
                                    size, None)

    for kw, word in [(dict(layer=2), "layer"), (dict(starts=None), "row_start"), (dict(total=-1), "total_rows"),
                     (dict(most=0), "max_rows"), (dict(keys=-1), "max_keys"), (dict(heads=6), "n_heads"),
                     (dict(heads=0), "n_heads"), (dict(q=None), "NULL"), (dict(o=None), "NULL"), (dict(qs=504), "stride"),
                     (dict(os=8), "stride"), (dict(qs=516), "multiples of 8"), (dict(q=FAKE + 8), "16-byte"),
                     (dict(o=FAKE + 2), "16-byte"), (dict(o=FAKE, os=520), "in place"),
                     (dict(mask=FAKE, words=0), "mask"), (dict(mask=FAKE + 1, words=1), "mask"),
                     (dict(lse=FAKE + 2), "lse"), (dict(scale=-1.0), "scale"), (dict(scale=math.nan), "scale"),
                     (dict(scale=math.inf), "scale"), (dict(ws=None), "workspace"), (dict(ws=FAKE + 16), "256-byte")]:
        _refused(lib, call(**kw), word)
    _refused(lib, call(total=1 << 24, most=1 << 24, heads=1024, qs=65536, os=65536), "too large")
    many = ctypes.byref(_cache(L, n_seqs=1024))
    _refused(lib, lib.dlm_cache_attend(many, 0, FAKE, 1 << 20, 1 << 20, 0, 16, FAKE, 1024, None, 0, 0.0, FAKE, 1024, None,
                                       FAKE, 1 << 40, None), "2^33")
    _refused(lib, call(size=1024), "too small", -5)
    assert call(total=0, most=0) == 0


def test_page_call_refusals():
    L, lib = _lib()
    c = ctypes.byref(_cache(L))
    need = lib.dlm_cache_workspace_bytes(c, 0, 0, 0)
    assert need > 0
    _refused(lib, lib.dlm_cache_reserve(c, None, 4, None, FAKE, need, None), "row_start")
    _refused(lib, lib.dlm_cache_reserve(c, FAKE, -1, None, FAKE, need, None), "total_rows")
    _refused(lib, lib.dlm_cache_reserve(c, FAKE, 4, None, None, need, None), "workspace")
    _refused(lib, lib.dlm_cache_reserve(c, FAKE, 4, None, FAKE, need - 1, None), "too small", -5)
    _refused(lib, lib.dlm_cache_commit(c, None, 4, None, None, 0, None, None), "row_start")
    _refused(lib, lib.dlm_cache_commit(c, FAKE, 4, FAKE, None, 4, None, None), "go together")
    _refused(lib, lib.dlm_cache_commit(c, FAKE, 4, None, FAKE, 4, None, None), "go together")
    _refused(lib, lib.dlm_cache_commit(c, FAKE, 4, FAKE, FAKE, -1, None, None), "total_keep")
    _refused(lib, lib.dlm_cache_fork(c, -1, FAKE, FAKE, None, None), "n_pairs")
    _refused(lib, lib.dlm_cache_fork(c, 1025, FAKE, FAKE, None, None), "n_pairs")
    _refused(lib, lib.dlm_cache_fork(c, 1, None, FAKE, None, None), "NULL")
    assert lib.dlm_cache_fork(c, 0, None, None, None, None) == 0
    _refused(lib, lib.dlm_cache_compact(c, None, FAKE, need - 1, None), "too small", -5)


def test_rope_apply_refusals():
    L, lib = _lib()
    r = ctypes.byref(_rope(L, lib))

    def call(rope=r, dtype=0, rows=4, heads=2, x=FAKE, xr=128, xh=64, y=2 * FAKE, yr=128, yh=64, pos=FAKE):
        return lib.dlm_rope_apply(rope, dtype, rows, heads, x, xr, xh, y, yr, yh, pos, 0, None)

    for kw, word in [(dict(rope=None), "NULL"), (dict(rope=ctypes.byref(L.DlmRope())), "dlm_rope_init"),
                     (dict(dtype=3), "dtype"), (dict(rows=-1), "rows"), (dict(heads=-1), "heads"), (dict(x=None), "NULL"),
                     (dict(pos=None), "NULL"), (dict(x=FAKE + 1), "aligned"), (dict(dtype=2, y=FAKE + 2), "aligned"),
                     (dict(xr=-128), "strides"), (dict(yh=-64), "strides"), (dict(yr=0), "overlap"),
                     (dict(yh=32), "overlap"), (dict(yr=100), "overlap"), (dict(yr=64, yh=100), "overlap"),
                     (dict(y=FAKE, xr=256), "in place")]:
        _refused(lib, call(**kw), word)
    assert call(rows=0) == 0 and call(heads=0) == 0


def test_step_refusals():
    L, lib = _lib()
    from paper_2608_02625_amd.model import make_config
    from workloads import MODELS
    cfg = ctypes.byref(make_config(MODELS["tiny"]))
    c = _cache(L)
    assert lib.dlm_cache_step_workspace_bytes(cfg, ctypes.byref(c), 5, 5) > 0
    for over in (dict(dtype=1), dict(n_layers=3), dict(n_kv_heads=2), dict(head_dim=128), dict(page_len=5)):
        assert lib.dlm_cache_step_workspace_bytes(cfg, ctypes.byref(_cache(L, **over)), 5, 5) == 0, over
    for rows, most in ((0, 1), (-1, 1), (5, 0), (65537, 1)):
        assert lib.dlm_cache_step_workspace_bytes(cfg, ctypes.byref(c), rows, most) == 0
    assert lib.dlm_cache_step_workspace_bytes(cfg, None, 5, 5) == 0
    _refused(lib, lib.dlm_cache_step(None, ctypes.byref(c), FAKE, 4, 4, 0, FAKE, None, None, 0, FAKE, 1 << 40, None, None,
                                     None, None, None), "NULL")


def test_plain_reference_keeps_its_books():
    """Every page is named as often as its count says, sequences keep what they were
    given, and a copy does not see what its original writes later."""
    rng = random.Random(3)
    c = PlainCache(12, 4, 4, 6)
    want = {b: [] for b in range(4)}
    serial = 0
    for step in range(300):
        what = rng.choice(["pass", "pass", "fork", "truncate", "compact"])
        if what == "pass":
            rows = [rng.randint(0, 5) for _ in range(4)]
            ok = c.reserve(rows)
            rows = [n if o else 0 for n, o in zip(rows, ok)]
            names = {}

            def tag(b, i):
                return names.setdefault((b, i), (step, b, i))
            c.append(rows, tag)
            keep = [sorted(rng.sample(range(n), rng.randint(0, n))) for n in rows]
            assert c.commit(rows, keep) == [1] * 4
            for b in range(4):
                want[b] += [tag(b, i) for i in keep[b]]
        elif what == "fork":
            s, d = rng.sample(range(4), 2)
            assert c.fork([s], [d]) == [1]
            want[d] = list(want[s])
        elif what == "truncate":
            new = [rng.choice([-1, rng.randint(0, 20)]) for _ in range(4)]
            c.truncate(new)
            for b, n in enumerate(new):
                if n >= 0:
                    want[b] = want[b][:n]
        else:
            n = c.compact()
            assert all(r > 0 for r in c.ref[:n]) and not any(c.ref[n:])
        for b in range(4):
            assert c.contents(b) == want[b], (step, what, b)
        names_of = [p for row in c.table for p in row if p >= 0]
        assert [names_of.count(p) for p in range(12)] == c.ref
        serial += 1
    assert c.fork([0, 1], [2, 2]) == [0, 0] and c.fork([0, 2], [2, 3]) == [0, 1] and c.fork([1], [1]) == [0]


def test_step_limits():
    """What the cache's own calls refuse by size, a model's step refuses before anything
    is launched (its workspace has no size)."""
    L, lib = _lib()
    from paper_2608_02625_amd.model import make_config
    from workloads import MODELS
    wide = ctypes.byref(make_config(MODELS["tiny"].replace(n_heads=192, n_kv_heads=4)))
    for seqs, rows, most, fits in ((1024, 65535, 65535, False), (1024, 65535, 40000, True), (512, 65535, 65535, True),
                                   (1024, 65536, 1, True), (1024, 65537, 1, False)):
        c = _cache(L, n_seqs=seqs)
        n = lib.dlm_cache_step_workspace_bytes(wide, ctypes.byref(c), rows, most)
        assert (n > 0) == fits, (seqs, rows, most, n)
