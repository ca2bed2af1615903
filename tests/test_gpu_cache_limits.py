"""The paged cache and the rotary positions at the ends of their ranges, on the GPU:
row starts, lengths and bounds that break their rules, probabilities far below a row's
largest, heads and rows past 32-bit sums.  Tolerances as in tests/test_gpu_cache.py.
"""

from __future__ import annotations

import pytest
import torch

from tests.gpu_util import need_gpu
from tests.test_gpu_cache import BF, HF, _cache, _ints

pytestmark = pytest.mark.gpu

INT_MAX, INT_MIN = (1 << 31) - 1, -(1 << 31)


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
