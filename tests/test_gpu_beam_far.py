"""Beam selection with logits and scores next to the largest float, on the GPU; the order is test_host_beam_join's."""
import pytest
import torch

from test_gpu_beam import run
from test_host_beam_join import far_out, ordered

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("large", [1e31, 1e37, 1e38, 3e38])
@pytest.mark.parametrize("score", [1e36, -1e38, 3e38, -3e38])
def test_logits_and_scores_next_to_the_largest_float(large, score):
    for logits, scores in far_out(large, score):
        for n in (40, 3):
            t, p, _, _ = run(logits, scores, 4, n)
            assert list(zip(p, t)) == ordered(logits, scores, n)
