"""Scales of the logits that the attention cannot hold, refused before a GPU is touched."""
import pytest

import paper_2406_06237_b200 as ans
from test_batches_host import attend


@pytest.mark.parametrize("scale", [3e38, -3.4e38, float("inf"), float("nan")])
def test_a_scale_that_leaves_fp32_with_the_logarithm(scale):
    assert attend(scale=scale) == ans.ANS_ERR_INVALID_ARG
