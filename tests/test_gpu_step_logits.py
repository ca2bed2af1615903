"""A model's logits behind a cache against the vocabulary reduction of the same pass, on the GPU:
both are sums of the same products in the same order, so they are equal bit for bit."""

from __future__ import annotations

import pytest
import torch

from tests.gpu_util import need_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


@pytest.mark.parametrize("name", ["tiny", "small_moe"])
def test_the_largest_logit_is_the_reductions(name):
    from paper_2608_02625_amd import Refiner
    from workloads import WORKLOADS
    w = WORKLOADS[name]
    model = Refiner(w.model.as_dict(), w.weight_seed)
    g = torch.Generator(device="cuda").manual_seed(1)
    for seqs, n in ((1, 1), (3, 1), (1, 9), (4, 13), (16, 33), (2, 300)):
        cache = model.cache(seqs * 5, 64, seqs, 5)
        starts = torch.arange(0, seqs * n + 1, n, dtype=torch.int32, device="cuda")
        assert bool(cache.reserve(starts).all())
        tokens = torch.randint(0, w.model.vocab - 1, (seqs * n,), device="cuda", generator=g, dtype=torch.int32)
        held = torch.full((seqs * n + 2, w.model.vocab), 5.0, device="cuda")
        logits = held[1:-1]
        top1, _, largest = model.cache_step(cache, tokens, starts, n, logits=logits)
        assert torch.equal(largest, logits.max(1).values)
        first = (logits == largest[:, None]).int().argmax(1)
        assert torch.equal(top1.long(), first)
        assert bool((held[0] == 5.0).all()) and bool((held[-1] == 5.0).all())
