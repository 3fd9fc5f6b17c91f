"""Operators around the first LLM layer, without a GPU: every refusal comes from the host with
nothing launched, position plans are checked through the positions they end at, and the
reference backward is checked against differences."""
import ctypes as C
import math

import numpy as np
import pytest

import paper_2607_03229_amd as mp
from paper_2607_03229_amd import _binding as B
from tests import layer_ref as R

@pytest.fixture(autouse=True)
def fp32_by_default():
    """Tensors made without a type are fp32, whatever a test before left as torch's default."""
    torch = pytest.importorskip("torch")
    old = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(old)


FAKE = 0x100000     # never dereferenced: the call must fail on the host first


@pytest.fixture(scope="module")
def L():
    return B.load()


# ---- positions ----------------------------------------------------------------------------

def _positions(L, seq_row, seq_len, seq_pos, item_row, grid, step, n_rows=1000, pos=FAKE,
               ld=None):
    def arr(a, t):
        return None if a is None else np.ascontiguousarray(a, t)
    sr, sl, sp, ir = (arr(a, np.int64) for a in (seq_row, seq_len, seq_pos, item_row))
    g, st = arr(grid, np.int32), arr(step, np.int32)
    ptr = lambda a: None if a is None else a.ctypes.data
    return L.mpipe_op_seam_positions(ptr(sr), ptr(sl), ptr(sp), len(seq_row), ptr(ir), ptr(g),
                                     ptr(st), len(item_row), n_rows, pos,
                                     n_rows if ld is None else ld, None, None)


BAD_POSITIONS = {
    "sequence_past_the_rows": (-2, dict(seq_row=[990], seq_len=[11])),
    "negative_row": (-2, dict(seq_row=[-1], seq_len=[5])),
    "negative_length": (-2, dict(seq_row=[0], seq_len=[-5])),
    "sequences_overlap": (-2, dict(seq_row=[0, 9], seq_len=[10, 4])),
    "sequences_overlap_unordered": (-2, dict(seq_row=[9, 0], seq_len=[4, 10])),
    "negative_first_position": (-2, dict(seq_row=[0], seq_len=[5], seq_pos=[-1])),
    "position_beyond_int32": (-5, dict(seq_row=[0], seq_len=[5], seq_pos=[2 ** 31 - 4])),
    "item_in_no_sequence": (-2, dict(seq_row=[0], seq_len=[5], item_row=[5], grid=[[1, 2, 2]])),
    "item_between_sequences": (-2, dict(seq_row=[0, 20], seq_len=[5, 5], item_row=[10],
                                        grid=[[1, 2, 2]])),
    "item_across_the_end": (-2, dict(seq_row=[0], seq_len=[5], item_row=[2], grid=[[1, 4, 4]])),
    "items_overlap": (-2, dict(seq_row=[0], seq_len=[50], item_row=[2, 5],
                               grid=[[1, 4, 4], [1, 4, 4]])),
    "same_item_twice": (-2, dict(seq_row=[0], seq_len=[50], item_row=[2, 2],
                                 grid=[[1, 4, 4], [1, 4, 4]])),
    "odd_grid": (-2, dict(seq_row=[0], seq_len=[50], item_row=[2], grid=[[1, 3, 4]])),
    "no_slices": (-2, dict(seq_row=[0], seq_len=[50], item_row=[2], grid=[[0, 2, 4]])),
    "negative_step": (-2, dict(seq_row=[0], seq_len=[50], item_row=[2], grid=[[1, 2, 4]],
                               step=[-1])),
    "time_beyond_int32": (-5, dict(seq_row=[0], seq_len=[50], item_row=[2], grid=[[3, 2, 4]],
                                   step=[2 ** 30])),
    "null_positions": (-1, dict(seq_row=[0], seq_len=[5], pos=None)),
    "misaligned_positions": (-1, dict(seq_row=[0], seq_len=[5], pos=FAKE + 2)),
    "rows_closer_than_ld": (-1, dict(seq_row=[0], seq_len=[5], ld=999)),
}


@pytest.mark.parametrize("name", BAD_POSITIONS)
def test_positions_refused(L, name):
    status, kw = BAD_POSITIONS[name]
    kw = dict(dict(seq_pos=None, item_row=[], grid=np.zeros((0, 3)), step=None), **kw)
    assert _positions(L, **kw) == status
    assert B.last_error()


def test_refused_positions_write_no_next(L):
    nxt = np.full(1, -5, np.int64)
    a, n = np.zeros(1, np.int64), np.full(1, 4, np.int64)
    assert L.mpipe_op_seam_positions(a.ctypes.data, n.ctypes.data, None, 1, None, None, None, 0, 10,
                                     None, 10, nxt.ctypes.data, None) == -1
    assert nxt[0] == -5


def test_positions_of_nothing(L):
    """No sequences, or only empty ones: fine, and nothing is launched (the pointer is not
    looked at)."""
    none = dict(seq_pos=None, item_row=[], grid=np.zeros((0, 3)), step=None, pos=None)
    assert _positions(L, [], [], **none) == 0
    assert _positions(L, [4, 9], [0, 0], **none) == 0


# ---- rotary configurations and head views -----------------------------------------------------

def _heads(p=FAKE, row=1024, head=128, heads=8):
    return B._HEADS.pack(p or 0, row, head, heads, 0)


def _rope(L, cfg=None, dtype=1, rows=4, q=None, k=None, qo=None, ko=None, pos=FAKE * 2, ld=4):
    ref = lambda h: h
    cfg = mp.RopeCfg(128, [16, 24, 24]) if cfg is None else cfg
    q = _heads() if q is None else q
    qo = _heads(FAKE * 16) if qo is None else qo
    return L.mpipe_op_rope_axes(dtype, C.byref(cfg), rows, ref(q), ref(k), pos, ld, 0, ref(qo),
                                ref(ko), None)


def _cfg(**kw):
    base = dict(head_dim=128, sections=[16, 24, 24])
    base.update(kw)
    return mp.RopeCfg(**base)


BAD_CFG = {
    "sections_do_not_sum": (-1, dict(sections=[16, 24, 23])),
    "negative_section": (-1, dict(sections=[80, -16])),
    "head_dim_12": (-5, dict(head_dim=12, sections=[6])),
    "head_dim_264": (-5, dict(head_dim=264, sections=[132])),
    "rot_dim_above": (-5, dict(rot_dim=136, sections=[68])),
    "rot_dim_0": (-5, dict(rot_dim=0, sections=[0])),
    "rot_dim_20": (-5, dict(rot_dim=20, sections=[10])),
    "theta_1": (-1, dict(theta=1.0)),
    "theta_nan": (-1, dict(theta=math.nan)),
    "theta_inf": (-1, dict(theta=math.inf)),
    "order_2": (-1, dict(order=2)),
    "spectrum_2": (-1, dict(spectrum=2)),
    "pairing_2": (-1, dict(pairing=-1)),
    "interleaved_does_not_fit": (-1, dict(order=1, sections=[8, 28, 28])),
}


@pytest.mark.parametrize("name", BAD_CFG)
def test_rope_cfg_refused(L, name):
    status, kw = BAD_CFG[name]
    assert _rope(L, cfg=_cfg(**kw)) == status


def test_rope_cfg_sections():
    for bad in ([], [16] * 5):
        with pytest.raises(mp.MpipeError):
            mp.RopeCfg(128, bad)


BAD_VIEWS = {
    "bad_dtype": dict(dtype=2),
    "negative_rows": dict(rows=-1),
    "null_input": dict(q=_heads(None)),
    "null_output": dict(qo=_heads(None)),
    "misaligned": dict(q=_heads(FAKE + 1)),
    "negative_stride": dict(q=_heads(row=-1024)),
    "negative_heads": dict(q=_heads(heads=-1), qo=_heads(FAKE * 16, heads=-1)),
    "head_counts_differ": dict(qo=_heads(FAKE * 16, heads=4)),
    "output_rows_overlap": dict(qo=_heads(FAKE * 16, row=1000)),
    "output_heads_overlap": dict(qo=_heads(FAKE * 16, head=64)),
    "output_broadcast": dict(qo=_heads(FAKE * 16, row=0)),
    "stride_overflow": dict(q=_heads(row=2 ** 62)),
    "null_positions": dict(pos=None),
    "misaligned_positions": dict(pos=FAKE * 2 + 2),
    "ld_pos_below_rows": dict(ld=3),
    "in_place_shifted": dict(qo=_heads(FAKE + 256)),
    "in_place_other_strides": dict(q=_heads(row=128, head=512), qo=_heads(FAKE)),
    "k_output_over_q_output": dict(k=_heads(FAKE * 32), ko=_heads(FAKE * 16)),
    "k_output_over_q_input": dict(k=_heads(FAKE * 32), ko=_heads(FAKE)),
    "k_without_output": dict(k=_heads(FAKE * 32)),
}


@pytest.mark.parametrize("name", BAD_VIEWS)
def test_head_views_refused(L, name):
    assert _rope(L, **BAD_VIEWS[name]) == -1
    assert B.last_error()


def test_nothing_to_turn(L):
    assert _rope(L, rows=0, q=_heads(None), qo=_heads(None), pos=None) == 0
    assert _rope(L, q=_heads(None, heads=0), qo=_heads(None, heads=0), pos=None) == 0


def _norm(L, eps=1e-6, gains=(FAKE * 3, FAKE * 3), bwd=False, scratch=FAKE * 64, nbytes=1 << 30,
          grads=(FAKE * 5, FAKE * 5 + 1024), rows=4, dq_out=FAKE * 16):
    ref = lambda h: h
    cfg = mp.RopeCfg(128, [16, 24, 24])
    q, k, qo, ko = _heads(), _heads(FAKE * 8), _heads(dq_out), _heads(FAKE * 24)
    common = (gains[0], gains[1], eps, FAKE * 2, 4, ref(qo), ref(ko))
    if not bwd:
        return L.mpipe_op_qk_norm_rope_fwd(1, C.byref(cfg), rows, ref(q), ref(k), *common, None)
    dq, dk = _heads(FAKE * 32), _heads(FAKE * 40)
    return L.mpipe_op_qk_norm_rope_bwd(1, C.byref(cfg), rows, ref(dq), ref(dk), ref(q), ref(k),
                                       *common, *grads, 1, scratch, nbytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(eps=0.0), -1), (dict(eps=-1.0), -1), (dict(eps=math.nan), -1), (dict(eps=math.inf), -1),
    (dict(gains=(None, FAKE)), -1), (dict(gains=(FAKE, None)), -1), (dict(gains=(FAKE + 1, FAKE)), -1),
    (dict(bwd=True, eps=0.0), -1), (dict(bwd=True, scratch=None), -3), (dict(bwd=True, nbytes=64), -3),
    (dict(bwd=True, scratch=FAKE + 2), -1), (dict(bwd=True, grads=(FAKE * 5, FAKE * 5)), -1),
    (dict(bwd=True, grads=(FAKE * 5 + 2, FAKE)), -1),
    (dict(bwd=True, dq_out=FAKE * 40), -1),        # over dk: the other side's gradient
])
def test_norm_refused(L, kw, status):
    assert _norm(L, **kw) == status


def test_norm_scratch_query(L):
    assert mp.op_qk_norm_rope_scratch_bytes(0, 1, 1, 128) > 0
    for bad in ((-1, 1, 1, 128), (1, -1, 1, 128), (1, 1, 1, 0), (1, 1, 1, 264), (1 << 31, 1, 1, 128)):
        with pytest.raises(mp.MpipeError):
            mp.op_qk_norm_rope_scratch_bytes(*bad)


# ---- gradient lists ------------------------------------------------------------------------------

def _list(*ts):
    a = (B._GradTensor * max(len(ts), 1))()
    for x, (p, n, dt) in zip(a, ts):
        x.data, x.n, x.dtype = p, n, dt
    return a, len(ts)


GOOD = (FAKE, 1000, 0)
BAD_GRADS = {
    "bad_dtype": [(FAKE, 10, 2)],
    "negative_length": [(FAKE, -1, 0)],
    "null": [(None, 10, 0)],
    "misaligned_f32": [(FAKE + 2, 10, 0)],
    "misaligned_bf16": [(FAKE + 1, 10, 1)],
    "too_long": [(FAKE, 2 ** 60, 0)],
    "same_tensor_twice": [GOOD, GOOD],
    "overlap": [GOOD, (FAKE + 3996, 4, 0)],
    "overlap_unordered": [(FAKE + 3996, 4, 0), GOOD],
}


@pytest.mark.parametrize("name", BAD_GRADS)
def test_gradient_lists_refused(L, name):
    a, n = _list(*BAD_GRADS[name])
    assert L.mpipe_op_grad_scratch_bytes(a, n) == 0
    assert L.mpipe_op_grad_norm(a, n, FAKE * 8, None, FAKE * 9, 1 << 30, None) == -1
    assert L.mpipe_op_grad_clip(a, None, n, FAKE * 8, 1.0, None, None) == -1


@pytest.mark.parametrize("out", [
    [(FAKE * 4, 999, 0)],                                      # another length
    [(FAKE, 1000, 1)],                                         # over its input in another type
    [(FAKE + 4, 1000, 0)],                                     # shifted
    [(FAKE - 2000, 1000, 0)],
    [(FAKE * 4, 1000, 3)],
], ids=str)
def test_clip_outputs_refused(L, out):
    a, n = _list(GOOD)
    o, _ = _list(*out)
    assert L.mpipe_op_grad_clip(a, o, n, FAKE * 8, 1.0, None, None) == -1


def test_clip_outputs_of_two_refused(L):
    a, n = _list(GOOD, (FAKE * 2, 1000, 0))
    for out in ([(FAKE * 4, 1000, 0), (FAKE * 4 + 400, 1000, 0)],      # outputs share memory
                [(FAKE * 2, 1000, 0), (FAKE, 1000, 0)]):               # each other's input
        o, _ = _list(*out)
        assert L.mpipe_op_grad_clip(a, o, n, FAKE * 8, 1.0, None, None) == -1


def test_clip_arguments_refused(L):
    a, n = _list(GOOD)
    assert L.mpipe_op_grad_norm(a, n, None, None, FAKE * 9, 1 << 30, None) == -1
    assert L.mpipe_op_grad_norm(a, n, FAKE * 8 + 4, None, FAKE * 9, 1 << 30, None) == -1
    assert L.mpipe_op_grad_norm(a, n, FAKE * 8, None, FAKE * 9, 8, None) == -3
    assert L.mpipe_op_grad_norm(a, n, FAKE * 8, None, None, 1 << 30, None) == -3
    assert L.mpipe_op_grad_norm(a, n, FAKE * 8, None, FAKE * 9 + 4, 1 << 30, None) == -1
    assert L.mpipe_op_grad_clip(a, None, n, None, 1.0, None, None) == -1
    assert L.mpipe_op_grad_clip(a, None, n, FAKE * 8, 1.0, FAKE * 8 + 4, None) == -1
    assert L.mpipe_op_grad_clip(a, None, n, FAKE * 8, -1.0, None, None) == -1
    assert L.mpipe_op_grad_clip(a, None, n, FAKE * 8, math.nan, None, None) == -1
    assert L.mpipe_op_grad_norm(None, 3, FAKE * 8, None, FAKE * 9, 1 << 30, None) == -1


# ---- the binding's own checks ------------------------------------------------------------------

def test_binding_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    cfg = mp.RopeCfg(64, [32])
    q = torch.zeros(3, 2, 64)
    pos = torch.zeros(1, 3, dtype=torch.int32)
    with pytest.raises(mp.MpipeError, match="on the GPU"):
        mp.op_rope_axes(cfg, q, None, pos, torch.zeros_like(q), None)
    with pytest.raises(mp.MpipeError, match="on the GPU"):
        mp.op_grad_norm([q], torch.zeros(1, dtype=torch.float64), None, torch.zeros(4096))
    with pytest.raises(mp.MpipeError, match="on the GPU"):
        mp.op_seam_positions([0], [3], [], [], torch.zeros(3, 3, dtype=torch.int32))


@pytest.mark.parametrize("kw", [
    dict(q=(3, 2, 32)), dict(q_out=(3, 2, 32)), dict(q_out=(3, 3, 64)), dict(pos=(1, 4)),
    dict(pos=(2, 3)), dict(k=(3, 1, 64)), dict(k_out=(3, 1, 64)), dict(k=(4, 1, 64), k_out=(4, 1, 64)),
    dict(dtype="f64"), dict(out_dtype="bf16"), dict(pos_dtype="i64"),
], ids=str)
def test_binding_refuses_shapes(kw):
    torch = pytest.importorskip("torch")
    dts = {"f64": torch.float64, "f32": torch.float32, "bf16": torch.bfloat16}
    dt = dts[kw.get("dtype", "f32")]
    q = torch.zeros(kw.get("q", (3, 2, 64)), dtype=dt)
    qo = torch.zeros(kw.get("q_out", (3, 2, 64)), dtype=dts[kw["out_dtype"]] if "out_dtype" in kw else dt)
    k = torch.zeros(kw["k"], dtype=dt) if "k" in kw else None
    ko = torch.zeros(kw["k_out"], dtype=dt) if "k_out" in kw else None
    pos = torch.zeros(kw.get("pos", (1, 3)),
                      dtype=torch.int64 if "pos_dtype" in kw else torch.int32)
    with pytest.raises(mp.MpipeError):
        mp.op_rope_axes(mp.RopeCfg(64, [32]), q, k, pos, qo, ko)


def test_binding_refuses_lists():
    torch = pytest.importorskip("torch")
    with pytest.raises(mp.MpipeError):
        mp.GradList([torch.zeros(4, 4).t()[:, :2]])          # not contiguous
    with pytest.raises(mp.MpipeError):
        mp.GradList([torch.zeros(4, dtype=torch.float64)])
    with pytest.raises(mp.MpipeError):
        mp.op_seam_positions([0.5], [3], [], [], torch.zeros(3, 3, dtype=torch.int32))
    with pytest.raises(mp.MpipeError):
        mp.op_seam_positions([0], [3], [0], [[1, 2, 2 ** 40]], torch.zeros(3, 3, dtype=torch.int32))


# ---- the reference itself ------------------------------------------------------------------------

@pytest.mark.parametrize("kw", [dict(d=16, sections=[3, 5]), dict(d=24, sections=[2, 1, 1], rot=8, pairing=1),
                                dict(d=16, sections=[4, 2, 2], order=1, spectrum=1)])
def test_reference_backward_against_differences(kw):
    """Central differences of sum(dy * y) in every input and gain entry."""
    c = R.rope_cfg(**kw)
    rng = np.random.default_rng(5)
    d = c["head_dim"]
    x, dy = rng.standard_normal((2, 2, d)), rng.standard_normal((2, 2, d))
    g, pos = 1 + 0.3 * rng.standard_normal(d), rng.integers(0, 50, (len(c["sections"]), 2))
    dx, dg, _, _ = R.norm_rope_bwd(c, dy, x, g, 1e-3, pos)
    f = lambda x, g: float((dy * R.norm_rope(c, x, g, 1e-3, pos)).sum())
    h = 1e-5
    for arr, grad, other in ((x, dx, None), (g, dg, None)):
        for i in np.ndindex(arr.shape):
            keep = arr[i]
            arr[i] = keep + h
            up = f(x, g)
            arr[i] = keep - h
            down = f(x, g)
            arr[i] = keep
            # the cubic term: h^2 times a third derivative of order 10, and rounding 1e-16 / h
            assert abs((up - down) / (2 * h) - grad[i]) < 1e-7


def test_reference_rotation_is_the_encoders():
    """Two axes in blocks with a spectrum each are the encoder's 2D positions (oracle)."""
    import oracle
    rng = np.random.default_rng(2)
    heads, d = 3, 32
    y, x = oracle.positions(np.array([[1, 4, 6], [2, 2, 8]], np.int32))
    q = rng.standard_normal((len(y), heads * d))
    c = R.rope_cfg(d, [d // 4, d // 4], spectrum=1)
    for inverse in (False, True):
        want = oracle.rope2d(q, heads, d, y, x, inverse=inverse)
        got = R.rotate(c, q.reshape(-1, heads, d), np.stack([y, x]), inverse)
        assert np.abs(got.reshape(want.shape) - want).max() < 1e-12
