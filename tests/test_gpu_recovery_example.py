"""The recovery operators as they are used together: slice an expert, train it against the whole one, evaluate."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_training_the_sliced_expert_brings_it_closer_to_the_whole_one():
    from recover_expert import recover
    lines = []
    r = recover(d_model=256, d_ff=512, vocab=2000, tokens=701, prune=0.37, steps=60, log=lines.append)
    assert r["kept"] == 512 - int(0.37 * 512)                     # an odd number of micro-experts is left: 323
    assert r["before"][0] > 0.0
    # on tokens the training did not see
    assert r["after"][0] < 0.9 * r["before"][0]
    assert abs(r["after"][1] - r["teacher_ppl"]) < abs(r["before"][1] - r["teacher_ppl"])
