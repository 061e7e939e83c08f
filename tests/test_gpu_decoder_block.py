"""The operators together, as examples/decoder_block.py uses them: compressed weights to a block's output."""
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("width,heads,prompt,tokens,bits", [(256, 4, 50, 5, 8), (256, 2, 1, 3, 8), (512, 4, 150, 2, 4)])
def test_block_follows_fp32(width, heads, prompt, tokens, bits):
    """e4m3 rows are off by up to 2^-4 of a value, 2^-5 or 3 % of it in the mean; the block's residual path carries
    half of the output's weight or more unchanged, so the norm of the deviation stays under 3 %.  A cache of 4 bits
    adds steps of 1/15 of a head's range, some 15 % of a value in the mean, to the attention's part: a
    mean over the sequence, at most a third of the output."""
    import decoder_block
    off, _, weight_bits = decoder_block.run(width, heads, prompt, tokens, bits)
    assert 0 < off < (0.03 if bits == 8 else 0.08)
    assert weight_bits < 5
