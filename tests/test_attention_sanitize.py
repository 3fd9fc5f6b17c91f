"""The host planning of the first LLM layer's attention (sequences, work items, cache checks),
built with g++ under AddressSanitizer and UndefinedBehaviorSanitizer and driven on valid and
invalid inputs.  CPU only."""
import os
import shutil

import pytest

from tests.test_sanitize import CSRC, ROOT, _build_and_run


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_attention_planning_under_sanitizers(tmp_path):
    out = _build_and_run(tmp_path, "attention_checks",
                         [os.path.join(ROOT, "tests", "sanitize", "attn_driver.cpp"),
                          os.path.join(CSRC, "attn_plan.cpp"), os.path.join(CSRC, "layer_plan.cpp")])
    assert "attention checks passed" in out
