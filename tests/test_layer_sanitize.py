"""The host planning of the operators around the first LLM layer (position spans, rotary
tables, views, gradient lists), built with g++ under AddressSanitizer and
UndefinedBehaviorSanitizer and driven on valid and invalid inputs.  CPU only."""
import os
import shutil

import pytest

from tests.test_sanitize import CSRC, ROOT, _build_and_run


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_layer_planning_under_sanitizers(tmp_path):
    out = _build_and_run(tmp_path, "layer_checks",
                         [os.path.join(ROOT, "tests", "sanitize", "layer_driver.cpp"),
                          os.path.join(CSRC, "layer_plan.cpp")])
    assert "layer checks passed" in out
