"""The example runs: a binarized layer and its head learn, and the head serves in 4 bits."""
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def test_train_and_serve():
    import train_and_serve
    first, last, same = train_and_serve.main(steps=60)
    assert last < first - 0.1                                     # ln 5000 = 8.5 to begin with
    assert same > 0.3                                             # one word in 5000 by chance
