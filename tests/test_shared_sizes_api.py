"""CPU checks of the sizes that shared-prefix attention takes; nothing is launched."""

from __future__ import annotations

import pytest

from tests.test_cache_api import _cache, _lib, _refused
from tests.test_shared_api import _attend


@pytest.mark.parametrize("rows,max_rows,group_rows", [(1 << 21, 128, 1 << 21), (1 << 22, 1000, 1 << 22), (1 << 23, 200, 1 << 23)])
def test_long_windows_share_nothing_and_have_no_bound_on_their_group(rows, max_rows, group_rows):
    """Their rows fill tiles by themselves: what the plain attention takes is taken (and asked
    for a workspace)."""
    L, lib = _lib()
    wide = _cache(L, n_seqs=1024)
    _refused(lib, _attend(lib, wide, total_rows=rows, max_rows=max_rows, max_group_rows=group_rows, workspace_bytes=0), "small", -5)
    # windows that could share have one
    _refused(lib, _attend(lib, wide, total_rows=rows, max_rows=2, max_group_rows=group_rows), "n_seqs * n_heads * max_rows")
