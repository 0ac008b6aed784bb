"""examples/answer.py runs, and what it returns is attention over the evidence and the text alone: with 4-bit pages as
with 16-bit ones, up to the codes' rounding."""
import importlib.util
import os

import pytest
import torch

from tests.conftest import REPO

pytestmark = pytest.mark.gpu


def test_example_with_both_kinds_of_pages():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    spec = importlib.util.spec_from_file_location("answer_example", os.path.join(REPO, "examples", "answer.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    a, b = ex.run(bits=16, steps=5), ex.run(bits=4, steps=5)
    assert a[0] == b[0] and len(a[0]) >= 1
    assert len(a[2]) == 5
    for x, y in zip([a[1], *a[2]], [b[1], *b[2]]):
        assert bool(torch.isfinite(x.float()).all()) and bool(torch.isfinite(y.float()).all())
        # codes are off by up to half a step of about a third of a value's size: outputs, means over hundreds of tokens,
        # by about a tenth of theirs
        assert float((x.float() - y.float()).norm()) < 0.3 * float(x.float().norm())
