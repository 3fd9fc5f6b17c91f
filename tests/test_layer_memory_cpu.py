"""Buffers that the operators around the first LLM layer write, over others of the same call:
refused on the host with nothing launched.  The addresses are never dereferenced."""
import ctypes as C

import pytest

import paper_2607_03229_amd as mp
from paper_2607_03229_amd import _binding as B

KB, MB = 1 << 10, 1 << 20
ROWS, HEADS, D = 4, 8, 128          # bf16: a view is 8 KB, a gain 256 bytes, its gradient 512

# each buffer in a megabyte of its own
AT = {n: (i + 1) * MB for i, n in enumerate(
    ("q", "k", "dq", "dk", "q_out", "k_out", "q_gain", "k_gain", "q_grad", "k_grad", "pos", "scratch"))}


@pytest.fixture(scope="module")
def L():
    return B.load()


def _call(L, op, at):
    cfg = mp.RopeCfg(D, [16, 24, 24])
    h = lambda n: B._HEADS.pack(at[n], HEADS * D, D, HEADS, 0)
    pos, out = (at["pos"], ROWS), (h("q_out"), h("k_out"))
    if op == "rope":
        return L.mpipe_op_rope_axes(1, C.byref(cfg), ROWS, h("q"), h("k"), *pos, 0, *out, None)
    gains = (at["q_gain"], at["k_gain"], 1e-6)
    if op == "fwd":
        return L.mpipe_op_qk_norm_rope_fwd(1, C.byref(cfg), ROWS, h("q"), h("k"), *gains, *pos, *out, None)
    need = mp.op_qk_norm_rope_scratch_bytes(ROWS, HEADS, HEADS, D)
    return L.mpipe_op_qk_norm_rope_bwd(1, C.byref(cfg), ROWS, h("dq"), h("dk"), h("q"), h("k"), *gains,
                                       *pos, *out, at["q_grad"], at["k_grad"], 1, at["scratch"], need,
                                       None)


SHARED = [
    # gain gradients that share some or all of their elements
    ("bwd", "k_grad", "q_grad", 0), ("bwd", "k_grad", "q_grad", 4), ("bwd", "k_grad", "q_grad", 508),
    ("bwd", "q_grad", "k_grad", 256),
    # gain gradients in an output
    ("bwd", "q_grad", "q_out", 0), ("bwd", "q_grad", "k_out", 4 * KB), ("bwd", "k_grad", "q_out", 8 * KB - 4),
    ("bwd", "k_grad", "k_out", -508),
    # scratch over any other
    *[("bwd", "scratch", n, 0) for n in AT if n != "scratch"],
    ("bwd", "scratch", "q", 8 * KB - 4), ("bwd", "pos", "scratch", 64), ("bwd", "k_grad", "scratch", 1024),
    ("bwd", "q_gain", "scratch", 16),
    # what is read by every wave, in an output: positions (48 bytes) and gains
    *[(op, n, out, 4 * KB) for op in ("fwd", "bwd") for n in ("pos", "q_gain", "k_gain")
      for out in ("q_out", "k_out")],
    ("rope", "pos", "q_out", -44), ("rope", "pos", "k_out", 8 * KB - 4),
]


@pytest.mark.parametrize("op,name,over,shift", SHARED, ids=str)
def test_qk_buffers_that_share_memory(L, op, name, over, shift):
    at = dict(AT)
    at[name] = at[over] + shift
    assert _call(L, op, at) == -1
    assert "share" in B.last_error()


# ---- the norm of a gradient and its clip --------------------------------------------------------

def _list(*ts):
    a = (B._GradTensor * len(ts))()
    for x, (p, n, dt) in zip(a, ts):
        x.data, x.n, x.dtype = p, n, dt
    return a


GRADS = [(1 * MB, 1000, 0), (2 * MB, 0, 0), (3 * MB, 1000, 1)]     # 4000, 0 and 2000 bytes


@pytest.mark.parametrize("kw", [
    dict(norms=5 * MB), dict(norms=5 * MB - 8), dict(norms=5 * MB + 4),           # sumsq inside
    dict(scratch=5 * MB), dict(scratch=5 * MB - 64), dict(scratch=6 * MB), dict(scratch=6 * MB + 8),
    dict(scratch=1 * MB + 3992), dict(scratch=3 * MB - 8), dict(scratch=3 * MB + 1992),
    dict(sumsq=1 * MB + 3992), dict(sumsq=3 * MB), dict(norms=1 * MB), dict(norms=3 * MB - 8),
], ids=str)
def test_norm_buffers_that_share_memory(L, kw):
    at = dict(dict(sumsq=5 * MB, norms=6 * MB, scratch=7 * MB), **kw)
    a = _list(*GRADS)
    need = L.mpipe_op_grad_scratch_bytes(a, 3)
    assert L.mpipe_op_grad_norm(a, 3, at["sumsq"], at["norms"], at["scratch"], need, None) == -1
    assert "share" in B.last_error()


@pytest.mark.parametrize("kw", [
    dict(sumsq=1 * MB + 3992), dict(sumsq=3 * MB), dict(norm=1 * MB), dict(norm=3 * MB + 1996),
    dict(norm=5 * MB), dict(norm=5 * MB + 4),
    dict(out=True, sumsq=9 * MB), dict(out=True, norm=9 * MB + 3996), dict(out=True, norm=1 * MB),
    dict(out=True, norm=11 * MB + 4),
], ids=str)
def test_clip_buffers_that_share_memory(L, kw):
    at = dict(dict(sumsq=5 * MB, norm=6 * MB, out=False), **kw)
    a, o = _list(*GRADS), _list(*[(p + 8 * MB, n, 0) for p, n, _ in GRADS])
    assert L.mpipe_op_grad_clip(a, o if at["out"] else None, 3, at["sumsq"], 1.0, at["norm"], None) == -1
    assert "share" in B.last_error()


def test_grad_list_follows_its_tensors():
    """A list made once takes the memory that its tensors have at the call, not the freed one."""
    torch = pytest.importorskip("torch")
    f = dict(dtype=torch.float32)
    a, b = torch.zeros(1000, **f), torch.zeros(7, **f)
    gl = mp.GradList([a, b])
    small = mp.op_grad_scratch_bytes(gl)
    for change in (lambda: setattr(a, "data", torch.zeros(400_000, **f)),
                   lambda: a.set_(torch.zeros(300_000, **f)), lambda: a.resize_(500_000)):
        change()
        assert mp.op_grad_scratch_bytes(gl) == mp.op_grad_scratch_bytes([a, b]) > small
        assert (gl.array[0].data, gl.array[0].n) == (a.data_ptr(), a.numel())
        assert (gl.array[1].data, gl.array[1].n) == (b.data_ptr(), 7)
    a.data = torch.zeros(9, dtype=torch.bfloat16)
    assert mp.op_grad_scratch_bytes(gl) == small and gl.array[0].dtype == 1
    a.data = torch.zeros(8, 8, **f).t()
    for _ in range(2):                       # refused for as long as it is so
        with pytest.raises(mp.MpipeError, match="contiguous"):
            mp.op_grad_scratch_bytes(gl)
    a.data = torch.zeros(5, **f)
    mp.op_grad_scratch_bytes(gl)
    assert (gl.array[0].data, gl.array[0].n, gl.array[0].dtype) == (a.data_ptr(), 5, 0)
