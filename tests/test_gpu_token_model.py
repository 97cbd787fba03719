"""The token model example: trained through the operators, its loss falls to what the sequences leave
open (two free tokens and the place of the end), and the beams continue a sequence."""
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def test_the_model_learns_and_continues():
    import token_model
    losses, tokens, scores = token_model.main(300)
    assert all(x == x for x in losses)
    # 12.5 targets a sequence: two of log 46, then an end that may come at any step (at most log 2 each)
    assert sum(losses[-10:]) / 10 < 1.3 < 3.0 < losses[0]
    for n, (a, b) in enumerate(((9, 5), (41, 30))):
        assert (scores[n, :-1] >= scores[n, 1:]).all()
        for k in range(2):   # the two best go on alternating until they end, if they do
            row = tokens[n, k].tolist()
            for i, t in enumerate(row):
                if t == token_model.END:
                    assert all(x == token_model.END for x in row[i:])
                    break
                assert t == (a, b)[i % 2], row
