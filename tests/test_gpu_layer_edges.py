"""Edges of the operators around the first LLM layer on the GPU, against float64 forms.
Tolerances are those of test_gpu_layer_ops.py, where they are derived; others beside their test."""
import numpy as np
import pytest

from tests import layer_ref as R
from tests.gpu_util import announce, torch_dev
from tests.test_gpu_layer_ops import (_cfg, _close, _filled, _mp, _norm_call, _np, _pos, _rand, _tdt,
                                      _untouched, _view, fp32_by_default)  # noqa: F401

pytestmark = pytest.mark.gpu


def test_grad_list_of_replaced_memory():
    """A tensor whose memory was replaced after its list was made is read and scaled where it is
    now; the memory it had stays."""
    torch, dev = torch_dev()
    mp = _mp()
    announce("grad list of replaced memory")
    a, b = torch.full((1000,), 3.0, device=dev), torch.full((40,), 2.0, device=dev)
    gl, old = mp.GradList([a, b]), a.data
    a.data = torch.full((2500,), 1.0, device=dev)
    sumsq = torch.empty(1, dtype=torch.float64, device=dev)
    scratch = torch.empty(mp.op_grad_scratch_bytes(gl), dtype=torch.uint8, device=dev)
    norms = torch.empty(2, device=dev)
    mp.op_grad_norm(gl, sumsq, norms, scratch)
    assert float(sumsq) == 2500 + 160 and float(norms[0]) == 50
    mp.op_grad_clip(gl, sumsq, 0.5 * 2660 ** 0.5)
    # the factor 0.5 off by three fp64 roundings comes out as 0.5 in fp32
    assert bool((a == 0.5).all()) and bool((b == 1).all()) and bool((old == 3).all())
