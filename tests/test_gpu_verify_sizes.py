"""Verification of drafted tokens (verify) at sizes whose rows fill more than one axis of a
grid, and over windows that lie over each other, against the rule in float64 on the CPU
(test_gpu_verify.py: whole numbers, equal)."""

from __future__ import annotations

import numpy as np
import pytest
import torch

from tests.gpu_util import need_gpu
from tests.test_gpu_verify import BF, F32, _case, _run, _same, _want

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


@pytest.mark.parametrize("shape,dtype,V,rows", [("chain", F32, 5, [3, 7, 1, 0, 5] * 4200), ("tree", BF, 3, [33] * 2000)])
def test_rows_beyond_one_axis_of_the_grid(shape, dtype, V, rows):
    """67200 and 66000 rows of a workgroup each, of which 65536 lie along the first axis."""
    for temperature in (0.0, 0.8) if shape == "tree" else (0.8,):
        c = _case(7, rows, V, dtype, shape, temperature)
        _same(_run(c), _want(c))


@pytest.mark.parametrize("shape", ["chain", "certain", "tree"])
def test_windows_over_each_other(shape):
    """Each is verified as if it stood alone, whatever long path or rejected tokens another one
    finds in the same rows."""
    V, T = 40, 4000
    c = _case(9, [900, 450, T - 1350], V, F32, shape)
    c["u"][:] = 0.0                                   # whole chains are kept, but for a few rows
    if shape == "tree":                               # pairs of children, the first one unlikely, the second one kept
        local = np.concatenate([np.arange(n) for n in (900, 450, T - 1350)])
        c["parent"][:] = np.where(local % 2 == 1, local - 1, np.maximum(local - 2, -1))
        for i in np.flatnonzero(local % 2 == 1):
            c["tokens"][i] = int(c["target"][i - 1].argmin())
        c["u"][torch.from_numpy(local % 2 == 1)] = 1.0 - 2.0 ** -24
    else:
        c["u"][[1200, 1700]] = 1.0 - 2.0 ** -24
    c["u_next"] = torch.rand(8, generator=torch.Generator().manual_seed(1))
    for starts in ([0, 900, 450, 1200, 300, 1100, 1, 800, 0], [0, 700, 0, 700, 0, 650, 3, 703, 5], [5, 5, 4, 904, 4, 1000, 0, 9, 2]):
        c["starts"] = starts
        want = _want(c)
        assert len(want[1]) == T and max(b - a for a, b in zip(want[2], want[2][1:])) > (4 if shape == "tree" else 600)
        for _ in range(3):
            _same(_run(c), want)


def test_more_kept_rows_than_rows():
    """Windows over each other that keep more rows together than there are: cut off at the end."""
    c = _case(10, [600], 9, F32, "certain")
    c["u"][:] = 0.0
    c["u_next"] = torch.rand(4, generator=torch.Generator().manual_seed(2))
    c["starts"] = [0, 500, 100, 600, 50]
    keep, first = _want(c)[1:]
    assert first == [0, 500, 500, 1000, 1000]
    for _ in range(3):
        v = _run(c)
        assert v.keep.tolist() == keep[:600] and v.keep_start.tolist() == [min(x, 600) for x in first]
