"""The largest sizes that the first LLM layer's attention takes, on the host: built with g++ under
the sanitizers.  CPU only."""
import os
import shutil

import pytest

from tests.test_sanitize import CSRC, ROOT, _build_and_run


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_attention_limits_under_sanitizers(tmp_path):
    out = _build_and_run(tmp_path, "attention_limits",
                         [os.path.join(ROOT, "tests", "sanitize", "attn_limits_driver.cpp"),
                          os.path.join(CSRC, "attn_plan.cpp"), os.path.join(CSRC, "layer_plan.cpp")])
    assert "attention limits passed" in out
