"""The largest sizes that the first LLM layer's attention takes, on the host (built with g++ under
the sanitizers), and tensors of other dimensions than its calls take.  CPU only."""
import os
import shutil

import pytest
import torch

import paper_2607_03229_amd as mp
from tests.test_sanitize import CSRC, ROOT, _build_and_run


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_attention_limits_under_sanitizers(tmp_path):
    out = _build_and_run(tmp_path, "attention_limits",
                         [os.path.join(ROOT, "tests", "sanitize", "attn_limits_driver.cpp"),
                          os.path.join(CSRC, "attn_plan.cpp"), os.path.join(CSRC, "layer_plan.cpp")])
    assert "attention limits passed" in out


@pytest.mark.parametrize("shape", [(), (64,), (10, 64), (1, 10, 2, 64)], ids=str)
def test_other_dimensions_refused(shape):
    try:
        mp.load()
    except mp.MpipeError:
        pytest.skip("libmpipe.so is not built")
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype)
    cache = mp.KvCache(z(3, 2, 16, 64), z(3, 2, 16, 64))
    table, pos = z(10, 1, dtype=torch.int32), z(10, dtype=torch.int32)
    x, good = z(*shape), z(10, 2, 64)
    for call in (lambda: mp.op_cache_write(cache, x, good, table, pos),
                 lambda: mp.op_cache_write(cache, good, x, table, pos),
                 lambda: mp.op_cache_read(cache, table, pos, x, x.clone()),
                 lambda: mp.op_cache_attention(cache, x, table, pos, good, z(64)),
                 lambda: mp.op_cache_attention(cache, good, table, pos, x, z(64)),
                 lambda: mp.op_causal_attention_fwd(x, good, good.clone(), good, None, [0], [10])):
        with pytest.raises(mp.MpipeError):
            call()

def test_scratch_of_one_batch_serves_another():
    """The size is one up to 4095 sequences."""
    try:
        mp.load()
    except mp.MpipeError:
        pytest.skip("libmpipe.so is not built")
    size = {mp.op_cache_attention_scratch_bytes(n, 4, 2, 64) for n in (0, 1, 64, 4095)}
    assert len(size) == 1 and mp.op_cache_attention_scratch_bytes(5000, 4, 2, 64) > size.pop()
