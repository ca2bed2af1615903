"""CPU checks of what the verification of drafted tokens refuses; nothing is launched."""

from __future__ import annotations

import math

import pytest

from tests.test_cache_api import FAKE, _lib, _refused

ARGS = dict(n_seqs=2, d_row_start=FAKE, total_rows=6, max_rows=4, d_tokens=FAKE, d_parent=None, dtype=2, vocab=50, d_target=FAKE,
            target_stride=50, d_draft=None, draft_stride=0, temperature=1.0, d_u=FAKE, d_u_next=FAKE, d_next=FAKE, d_keep=FAKE,
            d_keep_start=FAKE, d_workspace=FAKE, workspace_bytes=1 << 40, stream=None)

BAD = [(dict(n_seqs=0), "n_seqs"), (dict(n_seqs=65536), "n_seqs"), (dict(total_rows=-1), "total_rows"),
       (dict(total_rows=(1 << 20) + 1), "total_rows"), (dict(max_rows=-1), "max_rows"), (dict(max_rows=0), "max_rows"),
       (dict(total_rows=2000, max_rows=1025), "max_rows"), (dict(vocab=0), "vocab"), (dict(vocab=(1 << 24) + 1), "vocab"),
       (dict(total_rows=1 << 20, vocab=1 << 24, target_stride=1 << 24), "2^31"), (dict(dtype=3), "dtype"),
       (dict(dtype=-1), "dtype"), (dict(temperature=-0.5), "temperature"), (dict(temperature=math.nan), "temperature"),
       (dict(temperature=math.inf), "temperature"), (dict(temperature=1e-31), "temperature"), (dict(temperature=1.1e30), "temperature"), (dict(d_row_start=None), "NULL"), (dict(d_tokens=None), "NULL"),
       (dict(d_target=None), "NULL"), (dict(d_u=None), "NULL"), (dict(d_u_next=None), "NULL"), (dict(d_next=None), "NULL"),
       (dict(d_keep=None), "NULL"), (dict(d_keep_start=None), "NULL"), (dict(d_parent=FAKE, d_draft=FAKE, draft_stride=50), "parent"),
       (dict(target_stride=49), "stride"), (dict(d_draft=FAKE, draft_stride=49), "stride"), (dict(d_target=FAKE + 2), "aligned"),
       (dict(d_draft=FAKE + 2, draft_stride=50), "aligned"), (dict(d_u=FAKE + 1), "aligned"), (dict(d_keep=FAKE + 2), "aligned"),
       (dict(d_row_start=FAKE + 2), "aligned"), (dict(d_workspace=None), "workspace"), (dict(d_workspace=FAKE + 8), "256-byte")]


@pytest.mark.parametrize("over,word", BAD)
def test_refusals(over, word):
    _, lib = _lib()
    _refused(lib, lib.dlm_verify(*{**ARGS, **over}.values()), word)


def test_workspace():
    _, lib = _lib()
    for draft in (0, 1):
        n = lib.dlm_verify_workspace_bytes(2, 6, 50, draft)
        assert n > 0
        over = dict(workspace_bytes=n - 1, d_draft=FAKE if draft else None, draft_stride=50)
        _refused(lib, lib.dlm_verify(*{**ARGS, **over}.values()), "small", -5)
    assert lib.dlm_verify_workspace_bytes(2, 6, 157184, 1) > lib.dlm_verify_workspace_bytes(2, 6, 157184, 0)
    for bad in ((0, 6, 50), (2, -1, 50), (2, 6, 0), (65536, 6, 50), (2, 1 << 20, 1 << 24)):
        assert lib.dlm_verify_workspace_bytes(*bad, 0) == 0


def test_step_logits_refusal():
    _, lib = _lib()
    for logits in (None, FAKE + 2):
        _refused(lib, lib.dlm_cache_step_logits(None, None, FAKE, 4, 4, 0, FAKE, None, None, 0, FAKE, 1 << 40, None, None, None,
                                                None, None, logits), "logits")
    _refused(lib, lib.dlm_cache_step_logits(None, None, FAKE, 4, 4, 0, FAKE, None, None, 0, FAKE, 1 << 40, None, None, None,
                                            None, None, FAKE), "model")
