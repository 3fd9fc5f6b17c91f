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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_at_the_smallest_eps(dtype):
    """eps = 2^-126 on heads of zeros, of values whose squares are subnormal or nothing, and of
    ordinary ones."""
    torch, dev = torch_dev()
    mp = _mp()
    announce(f"norm at the smallest eps {dtype}")
    c, rows, d, eps = R.rope_cfg(64, [8, 4], rot=24), 6, 64, 2.0 ** -126
    gen = torch.Generator().manual_seed(71)
    p, pos = _pos(np.random.default_rng(7), 2, rows)
    x, dy = _rand(gen, (rows, 2, d), dtype), _rand(gen, (rows, 2, d), dtype)
    for r, scale in enumerate((0.0, 1e-24, 1e-20, 1e-19, 1e-10, 1.0)):
        x[r] *= scale
    g = 1 + 0.2 * _rand(gen, (d,), dtype)
    y, dx, dg = torch.empty_like(x), torch.empty_like(x), torch.empty(d, device=dev)
    scratch = torch.empty(mp.op_qk_norm_rope_scratch_bytes(rows, 2, 0, d), dtype=torch.uint8, device=dev)
    mp.op_qk_norm_rope_fwd(_cfg(c), x, None, g, None, eps, pos, y, None)
    mp.op_qk_norm_rope_bwd(_cfg(c), dy, None, x, None, g, None, eps, pos, dx, None, dg, None, scratch,
                           accumulate=False)
    xn, gn = _np(x), _np(g)
    r = 1.0 / np.sqrt((xn * xn).mean(-1, keepdims=True) + eps)
    _close(y, R.norm_rope(c, xn, gn, eps, p), R.partners(c, xn * r * gn), 2.0 ** -19, dtype, "forward")
    wx, wg, sx, sg = R.norm_rope_bwd(c, _np(dy), xn, gn, eps, p)
    _close(dx, wx, sx, 2.0 ** -18, dtype, "dx")
    _close(dg, wg, sg, 2.0 ** -19 + 12 * 2.0 ** -24, "f32", "dg")
    assert bool((y[0] == 0).all())
