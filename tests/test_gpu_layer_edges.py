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


@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
def test_clip_of_a_norm_far_above(dtype, out):
    """Factors below fp32's normal range and below all of it: the scaled gradient keeps fp32's
    precision (half a step of its product, half a step of a subnormal result)."""
    torch, dev = torch_dev()
    mp, gen = _mp(), torch.Generator().manual_seed(81)
    announce(f"clip of a norm far above {dtype}->{out}")
    for size, max_norm in ((1e38, 1.0), (1e38, 1e-3), (3e38, 1e-9), (3e38, 1e-30), (1e38, 1e-44)):
        ts = [torch.full((n,), size, device=dev).to(_tdt(dtype)) * torch.sign(
            torch.randn(n, generator=gen)).to(dev).to(_tdt(dtype)) for n in (1000, 77, 40001)]
        ts[0][::3] = 1e-3                    # and small ones among them, which vanish
        sumsq, _ = _norm_call(ts)
        ref = [_np(t) for t in ts]
        total = float(np.sqrt(sum((r * r).sum() for r in ref)))
        os = [torch.full((t.numel(),), float("nan"), device=dev, dtype=_tdt(out)) for t in ts]
        norm = torch.zeros(1, device=dev)
        mp.op_grad_clip(ts, sumsq, max_norm, norm, out=os)
        with np.errstate(over="ignore"):
            assert float(norm) == float(np.float32(total))
        f = max_norm / total
        half = 2.0 ** -24 if out == "f32" else 2.0 ** -24 + 2.0 ** -8
        step = 2.0 ** -150 if out == "f32" else 2.0 ** -134 + 2.0 ** -150    # of subnormals
        for r, o in zip(ref, os):
            # f is off by a few fp64 steps, the product by a rounding of its own
            assert bool((np.abs(_np(o) - r * f) <= (half + 1e-12) * np.abs(r * f) + step).all()), max_norm
        if dtype == out:
            mp.op_grad_clip(ts, sumsq, max_norm)
            assert all(torch.equal(a, b) for a, b in zip(ts, os))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("order", ["rows", "heads"])
def test_q_k_v_head_by_head(order, dtype):
    """[rows][heads][q | k | v][d] and [heads][rows][q | k | v][d], in place: the bits of dense
    tensors, and v as it was."""
    torch, dev = torch_dev()
    mp = _mp()
    announce(f"q, k, v head by head, {order} first, {dtype}")
    c, rows, heads, d = R.rope_cfg(64, [4, 6, 6], rot=32, pairing=1), 75, 5, 64
    cfg, gen = _cfg(c), torch.Generator().manual_seed(91)
    _, pos = _pos(np.random.default_rng(9), 3, rows)
    g = [1 + 0.2 * _rand(gen, (d,), dtype) for _ in range(2)]
    scratch = torch.empty(mp.op_qk_norm_rope_scratch_bytes(rows, heads, heads, d), dtype=torch.uint8, device=dev)

    def product():
        x = _rand(gen, (rows, heads, 3, d) if order == "rows" else (heads, rows, 3, d), dtype)
        v = x if order == "rows" else x.transpose(0, 1)
        return x, v[:, :, 0], v[:, :, 1], v[:, :, 2]

    def like(t):
        return torch.full(t.shape, float("nan"), dtype=t.dtype, device=dev)

    for f in (lambda q, k, qo, ko: mp.op_rope_axes(cfg, q, k, pos, qo, ko),
              lambda q, k, qo, ko: mp.op_qk_norm_rope_fwd(cfg, q, k, *g, 1e-6, pos, qo, ko)):
        x, q, k, v = product()
        want, keep = [like(q), like(k)], v.clone()
        f(q.contiguous(), k.contiguous(), *want)
        f(q, k, q, k)
        assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(v, keep)
    _, q, k, _ = product()
    _, dq, dk, dv = product()
    want, keep = [like(q), like(k)], dv.clone()
    gw, gg = ([torch.zeros(d, device=dev) for _ in range(2)] for _ in range(2))
    mp.op_qk_norm_rope_bwd(cfg, dq.contiguous(), dk.contiguous(), q.contiguous(), k.contiguous(), *g, 1e-6,
                           pos, *want, *gw, scratch)
    mp.op_qk_norm_rope_bwd(cfg, dq, dk, q, k, *g, 1e-6, pos, dq, dk, *gg, scratch)
    assert torch.equal(dq, want[0]) and torch.equal(dk, want[1]) and torch.equal(dv, keep)
    assert torch.equal(gg[0], gw[0]) and torch.equal(gg[1], gw[1])


@pytest.mark.parametrize("rows", [1, 2, 130])
def test_one_row_of_positions_for_all_axes(rows):
    """Positions of text: one row of them expanded to every axis, the bits of its copies."""
    torch, dev = torch_dev()
    mp = _mp()
    announce(f"one row of positions, {rows} rows")
    c, d = R.rope_cfg(128, [16, 24, 24], theta=1e6), 128
    cfg, gen = _cfg(c), torch.Generator().manual_seed(95)
    p, one = _pos(np.random.default_rng(9), 1, rows)
    copies, one = one.repeat(3, 1), one.expand(3, rows)
    assert one.stride(0) == 0
    q, k = _rand(gen, (rows, 6, d), "bf16"), _rand(gen, (rows, 2, d), "bf16")
    g = [_rand(gen, (d,), "bf16") for _ in range(2)]
    scratch = torch.empty(mp.op_qk_norm_rope_scratch_bytes(rows, 6, 2, d), dtype=torch.uint8, device=dev)
    got, want = [], []
    for out, pos in ((want, copies), (got, one)):
        o = [torch.empty_like(t) for t in (q, k) * 3] + [torch.empty(d, device=dev) for _ in range(2)]
        mp.op_rope_axes(cfg, q, k, pos, o[0], o[1])
        mp.op_qk_norm_rope_fwd(cfg, q, k, *g, 1e-6, pos, o[2], o[3])
        mp.op_qk_norm_rope_bwd(cfg, q, k, q, k, *g, 1e-6, pos, o[4], o[5], o[6], o[7], scratch, accumulate=False)
        out += o
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    _close(got[0], R.rotate(c, _np(q), np.repeat(p, 3, 0)), R.partners(c, _np(q)), 2.0 ** -22, "bf16", rows)
    with pytest.raises(mp.MpipeError):          # written positions have a row for every axis
        mp.op_seam_positions([0], [rows], [], [], one)
