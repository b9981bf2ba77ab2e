"""The example that trains with the library's operators end to end: it learns, and the same seeds give the same bits."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("tokens,width,hidden,layers", [(512, 256, 1024, 2), (300, 200, 500, 1)])
def test_training_lowers_the_loss(tokens, width, hidden, layers):
    import torch

    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    import train_feed_forward as T

    losses = T.train(steps=120, tokens=tokens, width=width, hidden=hidden, layers=layers)
    assert all(x == x for x in losses)
    # a run that learned nothing would stay within noise (a few per cent) of its first losses
    assert sum(losses[-10:]) < 0.8 * sum(losses[:10])
    again = T.train(steps=3, tokens=tokens, width=width, hidden=hidden, layers=layers)
    assert again == losses[:3]                       # same seeds, same bits
