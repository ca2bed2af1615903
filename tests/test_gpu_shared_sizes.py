"""Attention over shared prefixes at the largest number of packed rows, most of them behind the
last sequence."""

from __future__ import annotations

import pytest
import torch

from tests.gpu_util import need_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


@pytest.mark.parametrize("rows", [1 << 24, (1 << 24) - 1])
def test_as_many_rows_as_a_call_takes(rows):
    """64 sequences of a row each in a batch padded to 2^24 rows: the bits of the plain attention
    where nothing is shared, its values where it is, and the other rows left as they were."""
    from paper_2608_02625_amd import PagedCache
    B, page, hd = 64, 128, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    c = PagedCache(1, 3 + B, page, 1, hd, B, (1 << 26) // page)          # wide: the sizes alone would share
    c.k.normal_(generator=g)
    c.v.normal_(generator=g)
    c.table.fill_(-1)
    c.table[:, :3] = torch.arange(3, dtype=torch.int32, device="cuda")
    c.table[:, 3] = torch.arange(3, 3 + B, dtype=torch.int32, device="cuda")
    c.len.copy_(torch.arange(3 * page, 3 * page + B, dtype=torch.int32, device="cuda"))
    starts = torch.arange(B + 1, dtype=torch.int32, device="cuda")
    q = torch.zeros(rows, 1, hd, dtype=torch.bfloat16, device="cuda")
    q[:B].normal_(generator=g)
    want = c.attend(0, q[:B], starts, 1)
    share = c.share(starts, torch.zeros(B, dtype=torch.int32, device="cuda"), rows, 1, B)
    assert share.data[4 * B:8 * B:4].tolist() == [3 * page] * B
    out = torch.full_like(q, 5.0)
    c.attend(0, q, starts, 1, out=out, share=share)
    assert bool((out[B:] == 5.0).all())
    # The same sum but for its order (1e-5 of a magnitude below 4) and two roundings of half a step.
    assert bool(((out[:B].float() - want.float()).abs() <= 2 * 2.0 ** -8 * want.float().abs() + 1e-4).all())
    if rows == 1 << 24:
        assert torch.equal(out[:B], want)
