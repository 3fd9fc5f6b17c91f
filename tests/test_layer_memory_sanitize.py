"""Which ranges and views of the operators around the first LLM layer share memory, built with
g++ under AddressSanitizer and UndefinedBehaviorSanitizer, against sets of elements.  CPU only."""
import os
import shutil

import pytest

from tests.test_sanitize import CSRC, ROOT, _build_and_run


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_layer_memory_under_sanitizers(tmp_path):
    out = _build_and_run(tmp_path, "layer_memory_checks",
                         [os.path.join(ROOT, "tests", "sanitize", "layer_memory_driver.cpp"),
                          os.path.join(CSRC, "layer_plan.cpp")])
    assert "memory checks passed" in out
