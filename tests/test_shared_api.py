"""CPU checks of what shared-prefix attention refuses; nothing is launched."""

from __future__ import annotations

import ctypes
import math

import pytest

from tests.test_cache_api import BAD_BUFFERS, BAD_CACHES, FAKE, _cache, _lib, _refused

BIG = 1 << 40
SHARE = dict(d_row_start=FAKE, total_rows=6, max_rows=3, d_group=FAKE, max_group_rows=6, d_share=FAKE, share_bytes=BIG, stream=None)
ATTEND = dict(layer=0, d_row_start=FAKE, total_rows=6, max_rows=3, max_group_rows=6, max_keys=0, d_share=FAKE, share_bytes=BIG,
              n_heads=8, d_q=FAKE, q_stride=512, d_mask=None, mask_words=0, scale=0.0, d_o=FAKE, o_stride=512, d_lse=None,
              d_workspace=FAKE, workspace_bytes=BIG, stream=None)


def _share(lib, c, **over):
    return lib.dlm_cache_share(ctypes.byref(c), *{**SHARE, **over}.values())


def _attend(lib, c, **over):
    return lib.dlm_cache_attend_shared(ctypes.byref(c), *{**ATTEND, **over}.values())


@pytest.mark.parametrize("over,word", BAD_CACHES + BAD_BUFFERS)
def test_unsound_caches(over, word):
    L, lib = _lib()
    c = _cache(L, **over)
    _refused(lib, _share(lib, c), word)
    _refused(lib, _attend(lib, c), word)


@pytest.mark.parametrize("over,word", [
    (dict(d_row_start=None), "row_start"), (dict(total_rows=-1), "total_rows"), (dict(max_rows=-1), "max_rows"),
    (dict(max_rows=0), "max_rows"), (dict(total_rows=(1 << 24) + 1), "2^24"), (dict(max_group_rows=-1), "max_group_rows"),
    (dict(d_share=None), "share"), (dict(d_share=FAKE + 16), "256-byte")])
def test_refusals_of_both(over, word):
    L, lib = _lib()
    c = _cache(L)
    _refused(lib, _share(lib, c, **over), word)
    _refused(lib, _attend(lib, c, **over), word)


@pytest.mark.parametrize("over,word", [
    (dict(layer=2), "layer"), (dict(layer=-1), "layer"), (dict(n_heads=6), "n_heads"), (dict(n_heads=0), "n_heads"),
    (dict(max_keys=-1), "max_keys"), (dict(scale=-1.0), "scale"), (dict(scale=math.nan), "scale"), (dict(d_q=None), "NULL"),
    (dict(d_o=None), "NULL"), (dict(q_stride=511), "q_stride"), (dict(o_stride=516), "multiples of 8"), (dict(d_q=FAKE + 8), "16-byte"),
    (dict(d_o=FAKE, q_stride=520), "in place"), (dict(d_mask=FAKE, mask_words=0), "mask"), (dict(d_lse=FAKE + 2), "lse"),
    (dict(d_workspace=None), "workspace"), (dict(d_workspace=FAKE + 64), "256-byte")])
def test_attend_refusals(over, word):
    L, lib = _lib()
    _refused(lib, _attend(lib, _cache(L), **over), word)


def test_group_and_sizes():
    L, lib = _lib()
    c = _cache(L)
    cp = ctypes.byref(c)
    _refused(lib, _share(lib, c, d_group=None), "group")
    _refused(lib, _share(lib, c, d_group=FAKE + 2), "group")
    n = lib.dlm_cache_share_bytes(cp, 6)
    assert n >= 4 * 6 and lib.dlm_cache_share_bytes(cp, -1) == 0 and lib.dlm_cache_share_bytes(None, 6) == 0
    assert lib.dlm_cache_share_bytes(cp, (1 << 24) + 1) == 0
    _refused(lib, _share(lib, c, share_bytes=n - 1), "small", -5)
    _refused(lib, _attend(lib, c, share_bytes=n - 1), "small", -5)
    need = lib.dlm_cache_shared_workspace_bytes(cp, 6, 3, 6, 8)
    assert need >= lib.dlm_cache_workspace_bytes(cp, 6, 3, 8)
    _refused(lib, _attend(lib, c, workspace_bytes=need - 1), "small", -5)
    for bad in ((-1, 3, 6, 8), (6, -1, 6, 8), (6, 3, -1, 8), (6, 3, 6, 7)):
        assert lib.dlm_cache_shared_workspace_bytes(cp, *bad) == 0
    assert _attend(lib, c, total_rows=0, d_q=None, d_o=None) == 0
    # rows of a group times heads past what the list of units can count
    wide = _cache(L, n_seqs=1024)
    _refused(lib, _attend(lib, wide, total_rows=1 << 24, max_rows=1, max_group_rows=1 << 24), "n_seqs * n_heads * max_rows")
