"""The example runs, from a checkpoint to decoded tokens."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["tiny", "llama8b_1l"])
def test_resume_and_decode(name):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "resume_and_decode.py")
    spec = importlib.util.spec_from_file_location("resume_and_decode", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    got = example.run(name, steps=5, window=100)
    assert got["repaired_rows"] > 0 and got["repaired_finite"] and got["replays_agree"] and got["decoded"] == 5
    # Values are drawn with a spread near 1 (the checkpoint's with a few channels 8 times that): 16 codes over a row's
    # range are off by up to a fifteenth of it, and so is an average of them.
    assert 0.0 < got["worst_difference"] < 8.0
