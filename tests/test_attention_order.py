"""An order inside the prompt attention kernel that a run cannot show safely, read from its source."""
import os
import re

SOURCE = os.path.join(os.path.dirname(__file__), "..", "paper_2110_06037_gb300", "csrc", "attn_prompt.cuh")


def test_scores_wait_until_the_weights_in_their_place_have_been_read():
    """A tile's next scores are written over its weights in tensor memory, and products on different
    accumulators do not keep their order: between a product with the weights and the next scores lies a wait."""
    text = re.sub(r"//[^\n]*", "", open(SOURCE).read())
    loop = text[text.index("for (int j = 0; j < part.most; ++j)\n#pragma unroll"):]
    loop = loop[:loop.index("at += 2 * part.most")]
    read, wait, scores = loop.index("values(t, j)"), loop.index("must(&sh.pv[t]"), loop.index("scores(t, j + LA)")
    assert read < wait < scores
    assert "tc_fence_after()" in loop[wait:scores]
