"""The example that runs append, attention and matrix-vector products as a block: a prompt, then decode steps."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("prompt,steps,seqs", [(200, 3, 1), (130, 2, 6)])
def test_decode_steps_after_a_prompt(prompt, steps, seqs):
    import attention_block
    block, attention = attention_block.run(prompt, steps, seqs)
    # Against the plain evaluation, which rounds nothing: the norm's output, the projection, the rotated queries, the
    # probabilities and the result are rounded to BF16 on the way, 2^-8 of each value at most (queries and norm act through scores
    # of a few units); rounding errors of independent signs add up to well below the sum of the five
    assert attention < 5 * 2 ** -8
    assert block < 6 * 2 ** -8
