"""Verification of drafted tokens (verify) at sizes whose rows fill more than one axis of a
grid, and over windows that lie over each other, against the rule in float64 on the CPU
(test_gpu_verify.py: whole numbers, equal)."""

from __future__ import annotations

import pytest

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
