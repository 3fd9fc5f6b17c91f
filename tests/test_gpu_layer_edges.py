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
    for size, max_norm in ((1e38, 1.0), (1e38, 1e-3), (3e38, 1e-9), (3e38, 1e-30), (1e38, 1e-37), (1e38, 1e-44),
                           (1e38, 0.0)):
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


# ---- the last lane of a head half filled ---------------------------------------------------------

# bf16 vectors of eight columns with an odd number of them behind the turned ones
HALF_FILLED = {
    "d40": R.rope_cfg(40, [4, 2, 2], rot=16),
    "d72_adjacent": R.rope_cfg(72, [8, 8], rot=32, pairing=1),
    "d104_interleaved": R.rope_cfg(104, [8, 8, 8], rot=48, order=1),
    "d248_adjacent": R.rope_cfg(248, [20, 50, 50], rot=240, pairing=1),
}


@pytest.mark.parametrize("layout", ["fused", "shifted"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", HALF_FILLED)
def test_half_filled_last_lane(name, dtype, layout):
    """Rotation both ways, norm and backward, out of place and in place: no column twice in the
    sums, none written twice with another value, none left out."""
    torch, dev = torch_dev()
    mp, c = _mp(), HALF_FILLED[name]
    cfg, d, axes, eps = _cfg(c), c["head_dim"], len(c["sections"]), float(np.float32(1e-6))
    rng, gen = np.random.default_rng(15), torch.Generator().manual_seed(16)
    for rows, hq, hk in ((1, 1, 1), (37, 7, 3), (130, 28, 4)):
        announce(f"half filled last lane {name} {dtype} {layout} rows={rows} heads={hq}+{hk}")
        p, pos = _pos(rng, axes, rows)
        x, dy = ([_filled(gen, (rows, h, d), dtype, layout)[0] for h in (hq, hk)] for _ in range(2))
        g = [1 + 0.2 * _rand(gen, (d,), dtype) for _ in range(2)]
        gg = [torch.full((d,), float("nan"), device=dev) for _ in range(2)]
        sc = torch.empty(mp.op_qk_norm_rope_scratch_bytes(rows, hq, hk, d), dtype=torch.uint8, device=dev)
        new = lambda: [_view(t.shape, dtype, layout) for t in x]
        turned, back, normed, dx = new(), new(), new(), new()
        v = lambda o: (o[0][0], o[1][0])
        mp.op_rope_axes(cfg, *x, pos, *v(turned))
        mp.op_rope_axes(cfg, *x, pos, *v(back), inverse=True)
        mp.op_qk_norm_rope_fwd(cfg, *x, *g, 1e-6, pos, *v(normed))
        mp.op_qk_norm_rope_bwd(cfg, *dy, *x, *g, 1e-6, pos, *v(dx), *gg, sc, accumulate=False)
        for z in range(2):
            xn, gn = _np(x[z]), _np(g[z])
            r = 1.0 / np.sqrt((xn * xn).mean(-1, keepdims=True) + eps)
            for o, inverse in ((turned, False), (back, True)):
                _close(o[z][0], R.rotate(c, xn, p, inverse), R.partners(c, xn), 2.0 ** -22, dtype, inverse)
            _close(normed[z][0], R.norm_rope(c, xn, gn, eps, p), R.partners(c, xn * r * gn), 2.0 ** -19,
                   dtype, "norm")
            wx, wg, sx, sg = R.norm_rope_bwd(c, _np(dy[z]), xn, gn, eps, p)
            _close(dx[z][0], wx, sx, 2.0 ** -18, dtype, "dx")
            n = min(rows * x[z].shape[1], 1200)
            _close(gg[z], wg, sg, 2.0 ** -19 + n * 2.0 ** -24, "f32", "dg")
            assert all(_untouched(*o[z]) for o in (turned, back, normed, dx))
        mp.op_qk_norm_rope_bwd(cfg, *dy, *x, *g, 1e-6, pos, *dy, None, None, sc)
        mp.op_qk_norm_rope_fwd(cfg, *x, *g, 1e-6, pos, *x)
        assert all(torch.equal(a, b[0]) for a, b in zip(x + dy, normed + dx))


# ---- the gains' gradient over large grids ----------------------------------------------------------

GAIN_CASES = [
    ("bf16", 33000, 28, 4, R.rope_cfg(128, [16, 24, 24], theta=1e6)),
    ("bf16", 60000, 28, 0, R.rope_cfg(128, [64])),
    ("f32", 17000, 28, 4, R.rope_cfg(128, [24, 20, 20], theta=1e6, order=1)),
    ("bf16", 90000, 1, 1, R.rope_cfg(128, [64])),              # eight angles a lane
    ("bf16", 120001, 2, 1, R.rope_cfg(64, [4, 6, 6], rot=32, pairing=1)),
    ("f32", 300007, 1, 2, R.rope_cfg(8, [4])),
    ("bf16", 20003, 9, 9, R.rope_cfg(256, [30, 45, 45], rot=240, pairing=1)),
    ("bf16", 9001, 65, 3, R.rope_cfg(16, [2, 2], rot=8)),
]


@pytest.mark.parametrize("case", GAIN_CASES, ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}-{c[3]}-{c[4]['head_dim']}")
def test_gain_gradient_counts_every_head_once(case):
    """Values of +-1 have a root-mean-square of 1, and at position 0 nothing turns: every term is
    a small whole number and every partial sum is exact (below 2^24), whatever the order.  One
    term lost or taken twice shows.  1 + eps is 1 in fp32."""
    torch, dev = torch_dev()
    mp = _mp()
    dtype, rows, hq, hk, c = case
    d, axes = c["head_dim"], len(c["sections"])
    announce(f"gains of {rows} rows, {hq}+{hk} heads of {d} {dtype}")
    gen = torch.Generator(device=dev).manual_seed(rows)

    def heads(h):
        if h == 0:
            return None, None
        x = torch.randint(0, 2, (rows, h, d), device=dev, generator=gen) * 2 - 1
        dy = torch.randint(1, 4, (rows, h, d), device=dev, generator=gen)
        dy *= torch.randint(0, 2, (rows, h, d), device=dev, generator=gen) * 2 - 1
        return x.to(_tdt(dtype)), dy.to(_tdt(dtype))

    (q, dq), (k, dk) = heads(hq), heads(hk)
    pos = torch.zeros((axes, rows), dtype=torch.int32, device=dev)
    g = [None if t is None else torch.ones(d, dtype=_tdt(dtype), device=dev) for t in (q, k)]
    base = [None if t is None else torch.randint(-99, 99, (d,), device=dev, generator=gen).float()
            for t in (q, k)]
    grad = [None if b is None else b.clone() for b in base]
    out = [None if t is None else torch.empty_like(t) for t in (q, k)]
    need = mp.op_qk_norm_rope_scratch_bytes(rows, hq, hk, d)
    scratch = torch.full((need // 4,), float("nan"), device=dev)
    mp.op_qk_norm_rope_bwd(_cfg(c), dq, dk, q, k, *g, 1e-12, pos, *out, *grad, scratch)
    for x, dy, b, got in zip((q, k), (dq, dk), base, grad):
        if x is not None:
            assert torch.equal(got.double(), b.double() + (x.double() * dy.double()).sum((0, 1)))
    if hk == 0:       # the largest grid: one side with more blocks than are resident at once
        assert int((~scratch.isnan()).sum()) // d > 768


@pytest.mark.parametrize("case", [GAIN_CASES[0], GAIN_CASES[2]],
                         ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}-{c[3]}-{c[4]['head_dim']}")
def test_gain_gradient_of_many_rows(case):
    """Ordinary values against float64 sums.  A wave takes at most 28 steps of heads here (1,280
    and 1,228 blocks of four waves for q), then 3 additions join its lanes, 2 its block's waves,
    12 a lane's blocks and 7 the lanes: no chain of more than 64.  A term is off by 2^-19 of its
    size.  Each side's bound is of its own sum of sizes."""
    torch, dev = torch_dev()
    mp = _mp()
    dtype, rows, hq, hk, c = case
    d, axes, half = c["head_dim"], len(c["sections"]), c["rot_dim"] // 2
    announce(f"gains of {rows} rows against float64, {hq}+{hk} heads of {d} {dtype}")
    gen = torch.Generator(device=dev).manual_seed(rows)
    p, pos = _pos(np.random.default_rng(rows), axes, rows)
    rand = lambda *s: torch.randn(s, device=dev, generator=gen).to(_tdt(dtype))
    x, dy = [rand(rows, h, d) for h in (hq, hk)], [rand(rows, h, d) for h in (hq, hk)]
    g, grad = [rand(d) for _ in range(2)], [torch.empty(d, device=dev) for _ in range(2)]
    out = [torch.empty_like(t) for t in x]
    scratch = torch.empty(mp.op_qk_norm_rope_scratch_bytes(rows, hq, hk, d), dtype=torch.uint8, device=dev)
    mp.op_qk_norm_rope_bwd(_cfg(c), *dy, *x, *g, 1e-6, pos, *out, *grad, scratch, accumulate=False)
    ang = torch.from_numpy(R.angles(c, p)).to(dev)[:, None]
    cos, sin = ang.cos(), ang.sin()
    for z in range(2):
        v, u = x[z].double(), dy[z].double()
        a, b = u[..., :half].clone(), u[..., half:].clone()      # whole heads in halves
        u[..., :half], u[..., half:] = a * cos + b * sin, b * cos - a * sin
        size = a.abs() + b.abs()
        v *= torch.rsqrt(v.square().mean(-1, keepdim=True) + 1e-6)
        want = (u * v).sum((0, 1))
        sizes = (torch.cat([size, size], -1) * v.abs()).sum((0, 1))
        err = (grad[z].double() - want).abs()
        assert bool((err <= (2.0 ** -19 + 64 * 2.0 ** -24) * sizes).all()), float((err / sizes).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,heads", [(1, 1), (3, 1), (5, 3), (67, 5)])
def test_an_infinite_output_gradient(rows, heads, dtype):
    """An infinity in the last row's last head of dy makes its pair's two columns of the gains'
    gradient infinite, of the formula's signs, and no other column anything but finite."""
    torch, dev = torch_dev()
    mp = _mp()
    announce(f"infinite output gradient {rows} rows {heads} heads {dtype}")
    c, d, eps = R.rope_cfg(128, [16, 24, 24], theta=1e6), 128, float(np.float32(1e-6))
    p, pos = _pos(np.random.default_rng(3), 3, rows)
    gen = torch.Generator().manual_seed(33)
    x, dy = _rand(gen, (rows, heads, d), dtype), _rand(gen, (rows, heads, d), dtype)
    dy[-1, -1, 5] = float("inf")
    g, dx, dg = torch.ones(d, device=dev, dtype=_tdt(dtype)), torch.empty_like(x), torch.empty(d, device=dev)
    sc = torch.empty(mp.op_qk_norm_rope_scratch_bytes(rows, heads, 0, d), dtype=torch.uint8, device=dev)
    mp.op_qk_norm_rope_bwd(_cfg(c), dy, None, x, None, g, None, 1e-6, pos, dx, None, dg, None, sc,
                           accumulate=False)
    with np.errstate(invalid="ignore"):
        _, want, _, _ = R.norm_rope_bwd(c, _np(dy), _np(x), _np(g), eps, p)
    assert sorted(np.flatnonzero(~np.isfinite(want)).tolist()) == [5, 69] and np.isinf(want[[5, 69]]).all()
    got = _np(dg)
    assert got[5] == want[5] and got[69] == want[69]
    assert np.isfinite(np.delete(got, [5, 69])).all()
