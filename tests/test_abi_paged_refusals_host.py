"""Refusals of the paged cache's entry points by value, before anything touches the GPU."""
import math

import pytest

from paper_2503_19950_amd import binding as B
from tests.test_abi_paged_host import _attn, _cache, _cfg, _step

inf, nan = math.inf, math.nan


@pytest.mark.parametrize("softcap", [inf, -inf, nan])
def test_softcaps_that_are_not_finite(softcap):
    cache, arrays = _cache((5, 5))
    for window in (0, 3):
        scores = B.lq_scores(softcap, window, None)
        assert _attn(_cfg(), cache, scores) == _step(_cfg(), cache, scores=scores) == B.LQ_ERR_SHAPE
    assert list(arrays[0]) == [5, 5]


@pytest.mark.parametrize("scale", [inf, -inf, nan])
def test_scales_that_are_not_finite(scale):
    cache, arrays = _cache((5, 5))
    for scores in (None, B.lq_scores(30.0, 0, None)):
        assert _attn(_cfg(), cache, scores, scale=scale) == _step(_cfg(), cache, scores=scores, scale=scale) == B.LQ_ERR_SHAPE
    assert list(arrays[0]) == [5, 5]
