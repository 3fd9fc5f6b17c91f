"""ctypes binding of libmpipe (include/mpipe.h, mpipe_ops.h, mpipe_sched.h, mpipe_derive.h).

Argument marshalling only: torch tensors provide device memory and the current
HIP stream; every step of the encoder runs in the library's kernels."""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import Dict, List, Optional, Sequence, Tuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libmpipe.so")

F32, BF16 = 0, 1
OK, NOOP_FROZEN = 0, 1
_STATUS = {0: "OK", 1: "NOOP_FROZEN", -1: "INVALID_ARG", -2: "BAD_METADATA", -3: "WORKSPACE",
           -4: "NO_TAPE", -5: "UNSUPPORTED", -6: "HIP"}


class MpipeError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"mpipe status {status} ({_STATUS.get(status, '?')}): {msg}")
        self.status = status


class EncoderCfg(C.Structure):
    _fields_ = [("in_chans", C.c_int32), ("patch", C.c_int32), ("temporal_patch", C.c_int32),
                ("hidden", C.c_int32), ("layers", C.c_int32), ("heads", C.c_int32),
                ("mlp", C.c_int32), ("merge", C.c_int32), ("llm_hidden", C.c_int32),
                ("dtype", C.c_int32), ("ln_eps", C.c_float), ("rope_theta", C.c_float)]

    @classmethod
    def from_config(cls, cfg) -> "EncoderCfg":
        """From any object with the encoder-config attributes (e.g. workload.EncoderConfig)."""
        dt = BF16 if getattr(cfg, "dtype", "bf16") in ("bf16", BF16) else F32
        return cls(cfg.in_chans, cfg.patch, cfg.temporal_patch, cfg.hidden, cfg.layers,
                   cfg.heads, cfg.mlp, cfg.merge, cfg.llm_hidden, dt, float(cfg.ln_eps),
                   float(cfg.rope_theta))


class RopeCfg(C.Structure):
    """mpipe_rope_cfg: which pairs of a head's columns turn by which axis' position, and how
    fast.  `sections`: pairs of each axis (their sum is rot_dim / 2); rot_dim defaults to
    head_dim.  The values are checked by the calls that take it."""
    _fields_ = [("head_dim", C.c_int32), ("rot_dim", C.c_int32), ("axes", C.c_int32),
                ("section", C.c_int32 * 4), ("order", C.c_int32), ("spectrum", C.c_int32),
                ("pairing", C.c_int32), ("theta", C.c_double)]

    def __init__(self, head_dim: int, sections: Sequence[int], rot_dim: Optional[int] = None,
                 theta: float = 10000.0, order: int = 0, spectrum: int = 0, pairing: int = 0):
        sections = [int(v) for v in sections]
        if not 1 <= len(sections) <= 4:
            raise MpipeError(-1, "one to four sections")
        super().__init__(int(head_dim), int(head_dim if rot_dim is None else rot_dim),
                         len(sections), (C.c_int32 * 4)(*sections), int(order), int(spectrum),
                         int(pairing), float(theta))


ROPE_BLOCKS, ROPE_INTERLEAVED = 0, 1
ROPE_ONE_SPECTRUM, ROPE_AXIS_SPECTRA = 0, 1
ROPE_HALVES, ROPE_ADJACENT = 0, 1


class _GradTensor(C.Structure):
    _fields_ = [("data", C.c_void_p), ("n", C.c_int64), ("dtype", C.c_int32),
                ("reserved", C.c_int32)]


_lib = None


def lib_path() -> str:
    return _LIB_PATH


def load():
    """Load libmpipe.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise MpipeError(-6, f"{_LIB_PATH} is missing: build it with paper_2607_03229_amd/build.py")
    L = C.CDLL(_LIB_PATH)
    P, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    st = C.c_int
    sig = {
        "mpipe_encoder_create": (st, [P, P]),
        "mpipe_encoder_destroy": (None, [P]),
        "mpipe_param_count": (i64, [P]),
        "mpipe_param_tensors": (i32, [P]),
        "mpipe_param_info": (st, [P, i32, C.c_char_p, i32, P, P, P]),
        "mpipe_encoder_sizes": (st, [P, P, i32, P, i32, i32, P, P, P, P]),
        "mpipe_encoder_regions": (st, [P, P, i32, P, i32, i32, i32, P, P, i32, P]),
        "mpipe_encoder_fwd": (st, [P, P, P, P, i32, P, i32, i32, P, P, sz, P, sz, P]),
        "mpipe_encoder_bwd": (st, [P, P, P, P, i32, P, i32, i32, P, sz, P, P, P, P, sz, P]),
        "mpipe_merge_scatter": (st, [P, i64, i32, i32, P, P, i64, P]),
        "mpipe_merge_gather": (st, [P, i64, i32, i32, P, i64, P, P]),
        "mpipe_merge_check_indices": (st, [P, i64, i64, P, P, P]),
        "mpipe_merge_check_indices_noalloc": (st, [P, i64, i64, P, P]),
        "mpipe_last_error": (C.c_char_p, []),
        "mpipe_profile_enable": (st, [P, i32]),
        "mpipe_encoder_set_side_stream": (st, [P, i32]),
        "mpipe_profile_read": (i32, [P, P, i32, P, i32, P, P, P]),
        "mpipe_op_gemm": (st, [i32, i32, i32, i32, i32, i32, P, i64, P, i64, P, i64, P, P, i64,
                               P, i64, i32, i32, i64, P]),
        "mpipe_op_gemm_kernel": (i32, [i32] * 7),
        "mpipe_op_splitk_reduce": (st, [P, i32, i64, i64, P, i64, P]),
        "mpipe_op_weight_grad_splits": (i32, [i64, i64, i64]),
        "mpipe_op_layernorm_fwd": (st, [i32, P, i64, i32, P, P, C.c_float, P, P, P, P]),
        "mpipe_op_layernorm_bwd": (st, [i32, P, P, P, P, P, i64, i32, P, P, P, P, P, P, P, sz, P]),
        "mpipe_op_rope": (st, [i32, P, i64, i32, i32, P, i32, C.c_float, i32, P, sz, P]),
        "mpipe_op_attention_fwd": (st, [i32, P, i64, i32, i32, P, i32, P, P, P, sz, P]),
        "mpipe_op_attention_bwd": (st, [i32, P, P, P, P, i64, i32, i32, P, i32, P, P, sz, P]),
        "mpipe_op_scratch_bytes": (sz, [i64, i32, i32, i32]),
        "mpipe_op_seam_positions": (st, [P, P, P, i32, P, P, P, i32, i64, P, i64, P, P]),
        "mpipe_op_rope_axes": (st, [i32, P, i64, P, P, P, i64, i32, P, P, P]),
        "mpipe_op_qk_norm_rope_fwd": (st, [i32, P, i64, P, P, P, P, C.c_float, P, i64, P, P, P]),
        "mpipe_op_qk_norm_rope_bwd": (st, [i32, P, i64, P, P, P, P, P, P, C.c_float, P, i64, P, P,
                                           P, P, i32, P, sz, P]),
        "mpipe_op_qk_norm_rope_scratch_bytes": (sz, [i64, i32, i32, i32]),
        "mpipe_op_grad_norm": (st, [P, i32, P, P, P, sz, P]),
        "mpipe_op_grad_scratch_bytes": (sz, [P, i32]),
        "mpipe_op_grad_clip": (st, [P, P, i32, P, C.c_double, P, P]),
        "mpipe_op_causal_attention_fwd": (st, [i32, i32, i64, i64, P, P, P, P, P, P, P, i32,
                                               C.c_float, P, P, i64, P]),
        "mpipe_op_causal_attention_bwd": (st, [i32, i32, i64, i64, P, P, P, P, P, P, i64, P, P, P,
                                               P, i32, C.c_float, P, P, P, P, sz, P]),
        "mpipe_op_causal_attention_scratch_bytes": (sz, [i64, i32, i64, i32, i32]),
        "mpipe_op_cache_write": (st, [P, i32, i64, P, P, P, i64, i32, i32, P, P, P, P]),
        "mpipe_op_cache_read": (st, [P, i32, i64, P, i64, i32, i32, P, P, P, P, P, P]),
        "mpipe_op_cache_attention": (st, [P, i32, i32, P, P, i64, i32, P, C.c_float, P, P, i64, P,
                                          sz, P]),
        "mpipe_op_cache_attention_scratch_bytes": (sz, [i32, i32, i32, i32]),
        "mpipe_encoder_cost": (st, [P, P, i32, P, i32, i32, C.c_double, C.c_double, P]),
        "mpipe_owner_map": (st, [P, i32, P, i32, i32, P, P, P]),
        "mpipe_schedule_valid": (st, [P, i32, i32, P]),
        "mpipe_derive": (st, [P, i32, i32, P, P, i32, i32, P, P]),
        "mpipe_derived_destroy": (None, [P]),
        "mpipe_derived_shape": (st, [P, P, P, P, P, P]),
        "mpipe_derived_placement": (st, [P, i32, P, P, P, P]),
        "mpipe_derived_owner": (st, [P, P]),
        "mpipe_derived_lists": (st, [P, P, P, P, P, P]),
        "mpipe_derived_nodes": (i32, [P, i32, P, i32]),
        "mpipe_event_costs": (st, [P, P, P, P, P, C.c_double, C.c_double, C.c_double, P]),
        "mpipe_makespan": (st, [P, P, P, P, P, P]),
        "mpipe_memory_peak": (st, [P, P, P]),
    }
    for name, (res, args) in sig.items():
        f = getattr(L, name)
        f.restype = res
        f.argtypes = args
    _lib = L
    return L


def last_error() -> str:
    v = load().mpipe_last_error()
    return v.decode() if v else ""


def _check(status: int, allow=(OK,)) -> int:
    if status not in allow:
        raise MpipeError(status, last_error())
    return status


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream=None) -> int:
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


def _host_i32(a) -> Tuple[np.ndarray, C.c_void_p]:
    arr = np.ascontiguousarray(np.asarray(a, dtype=np.int32))
    return arr, arr.ctypes.data_as(C.c_void_p)


# --------------------------------------------------------------------------
# Encoder handle
# --------------------------------------------------------------------------

class Encoder:
    """Handle over mpipe_encoder_*; all tensors are torch device tensors."""

    def __init__(self, cfg):
        self.L = load()
        self.ccfg = cfg if isinstance(cfg, EncoderCfg) else EncoderCfg.from_config(cfg)
        h = C.c_void_p()
        _check(self.L.mpipe_encoder_create(C.byref(self.ccfg), C.byref(h)))
        self._h = h

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            self.L.mpipe_encoder_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- parameter table --
    def param_count(self) -> int:
        return int(self.L.mpipe_param_count(C.byref(self.ccfg)))

    def param_table(self) -> List[Tuple[str, int, int, int]]:
        n = self.L.mpipe_param_tensors(C.byref(self.ccfg))
        buf = C.create_string_buffer(128)
        off, r, c = C.c_int64(), C.c_int64(), C.c_int64()
        out = []
        for i in range(n):
            _check(self.L.mpipe_param_info(C.byref(self.ccfg), i, buf, 128, C.byref(off),
                                           C.byref(r), C.byref(c)))
            out.append((buf.value.decode(), off.value, r.value, c.value))
        return out

    # -- sizes --
    def sizes(self, cu_seqlens, grid_thw, trainable: bool) -> Dict[str, int]:
        cu, cup = _host_i32(cu_seqlens)
        g, gp = _host_i32(np.asarray(grid_thw).reshape(-1, 3))
        ws, tp, nm, npch = C.c_size_t(), C.c_size_t(), C.c_int64(), C.c_int64()
        _check(self.L.mpipe_encoder_sizes(self._h, cup, max(len(cu) - 1, 0), gp, g.shape[0],
                                          int(trainable), C.byref(ws), C.byref(tp),
                                          C.byref(nm), C.byref(npch)))
        return {"workspace": ws.value, "tape": tp.value, "n_merged": nm.value,
                "n_patches": npch.value}

    def regions(self, cu_seqlens, grid_thw, trainable, which: int) -> np.ndarray:
        """int64 [n][2] (offset, bytes) of the workspace (which=0) or tape (1) ranges the
        step may write; at least 256 bytes after each range are never written."""
        cu, cup = _host_i32(cu_seqlens)
        g, gp = _host_i32(np.asarray(grid_thw).reshape(-1, 3))
        n = C.c_int32()
        args = (self._h, cup, max(len(cu) - 1, 0), gp, g.shape[0], int(trainable), which)
        _check(self.L.mpipe_encoder_regions(*args, None, None, 0, C.byref(n)))
        off, nb = np.zeros(n.value, np.int64), np.zeros(n.value, np.int64)
        _check(self.L.mpipe_encoder_regions(*args, off.ctypes.data_as(C.c_void_p),
                                            nb.ctypes.data_as(C.c_void_p), n.value, C.byref(n)))
        return np.stack([off, nb], axis=1)

    # -- fwd / bwd --
    def fwd(self, weights, patches, cu_seqlens, grid_thw, trainable: bool, merged, tape,
            workspace, stream=None) -> int:
        cu, cup = _host_i32(cu_seqlens)
        g, gp = _host_i32(np.asarray(grid_thw).reshape(-1, 3))
        tb = 0 if tape is None else tape.numel() * tape.element_size()
        wb = 0 if workspace is None else workspace.numel() * workspace.element_size()
        return _check(self.L.mpipe_encoder_fwd(
            self._h, _ptr(weights), _ptr(patches), cup, max(len(cu) - 1, 0), gp, g.shape[0],
            int(trainable), _ptr(merged), _ptr(tape), tb, _ptr(workspace), wb, _stream(stream)))

    def bwd(self, weights, patches, cu_seqlens, grid_thw, trainable: bool, tape, d_merged,
            d_weights, d_patches, workspace, stream=None) -> int:
        cu, cup = _host_i32(cu_seqlens)
        g, gp = _host_i32(np.asarray(grid_thw).reshape(-1, 3))
        tb = 0 if tape is None else tape.numel() * tape.element_size()
        wb = 0 if workspace is None else workspace.numel() * workspace.element_size()
        return _check(self.L.mpipe_encoder_bwd(
            self._h, _ptr(weights), _ptr(patches), cup, max(len(cu) - 1, 0), gp, g.shape[0],
            int(trainable), _ptr(tape), tb, _ptr(d_merged), _ptr(d_weights), _ptr(d_patches),
            _ptr(workspace), wb, _stream(stream)), allow=(OK, NOOP_FROZEN))

    # -- cost model --
    def cost(self, cu_seqlens, grid_thw, trainable, flops_per_second: float,
             bytes_per_second: float) -> Dict[str, float]:
        """W, D and the roofline seconds of this micro-batch's forward and backward slabs."""
        cu, cup = _host_i32(cu_seqlens)
        g, gp = _host_i32(np.asarray(grid_thw).reshape(-1, 3))
        out = (C.c_double * 6)()
        _check(self.L.mpipe_encoder_cost(self._h, cup, max(len(cu) - 1, 0), gp, g.shape[0],
                                         int(trainable), float(flops_per_second),
                                         float(bytes_per_second), out))
        keys = ("fwd_flops", "fwd_bytes", "fwd_seconds", "bwd_flops", "bwd_bytes", "bwd_seconds")
        return dict(zip(keys, list(out)))

    def set_side_stream(self, enable: Optional[bool]):
        """Backward weight-gradient work on the handle's internal stream or not; None (the
        default): on it where the micro-batch is large enough to gain."""
        _check(self.L.mpipe_encoder_set_side_stream(self._h,
                                                    -1 if enable is None else int(enable)))

    # -- kernel timing --
    def profile(self, enable: bool):
        _check(self.L.mpipe_profile_enable(self._h, int(enable)))

    def profile_read(self, stream=None) -> Dict[str, Tuple[int, float, float]]:
        cap, stride = 64, 64
        names = C.create_string_buffer(cap * stride)
        la = (C.c_int64 * cap)()
        ms = (C.c_double * cap)()
        fl = (C.c_double * cap)()
        n = self.L.mpipe_profile_read(self._h, _stream(stream), cap, names, stride, la, ms, fl)
        if n < 0:
            raise MpipeError(-6, "profile read failed")
        out = {}
        for i in range(n):
            nm = names.raw[i * stride:(i + 1) * stride].split(b"\0", 1)[0].decode()
            out[nm] = (int(la[i]), float(ms[i]), float(fl[i]))
        return out


# --------------------------------------------------------------------------
# Seam scatter / gather
# --------------------------------------------------------------------------

def _dt(t) -> int:
    import torch
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise MpipeError(-1, f"unsupported dtype {t.dtype}")


OWNER_GREEDY, OWNER_EXACT, OWNER_REFINED = 0, 1, 2


def owner_map(cost, warmup, method: int = OWNER_GREEDY):
    """ByMicrobatch owner: (owner [n_mb] int32, spill [n_ranks], max spill)."""
    c = np.ascontiguousarray(cost, dtype=np.float64)
    w = np.ascontiguousarray(warmup, dtype=np.float64)
    owner = np.zeros(c.shape[0], np.int32)
    spill = np.zeros(w.shape[0], np.float64)
    worst = C.c_double()
    _check(load().mpipe_owner_map(c.ctypes.data_as(C.c_void_p), c.shape[0],
                                  w.ctypes.data_as(C.c_void_p), w.shape[0], int(method),
                                  owner.ctypes.data_as(C.c_void_p),
                                  spill.ctypes.data_as(C.c_void_p), C.byref(worst)))
    return owner, spill, worst.value


# --------------------------------------------------------------------------
# Schedule algebra (host only)
# --------------------------------------------------------------------------

SK_1F1B, SK_GPIPE, SK_TRANSPOSE = 0, 1, 2
LAYOUT_SHARDED, LAYOUT_REPLICATED = 0, 1
COMM_NONE, COMM_GATHER, COMM_SCATTER, COMM_SEND, COMM_RECVGRAD = -1, 0, 1, 2, 3
GROUP_REPLICA, GROUP_DATA = 0, 1
EV_FWD, EV_BWD, EV_COLL, EV_DPREDUCE, EV_LOSS, EV_STEP_BARRIER = 0, 1, 2, 3, 4, 5
EDGE_ACTIVATION, EDGE_GRADIENT, EDGE_TURNAROUND, EDGE_ACCUMULATE, EDGE_SEQUENCE = 0, 1, 2, 3, 4
EVENT_FIELDS = ("kind", "region", "rank", "mb", "stage", "comm", "seam", "group")


def _vp(a: np.ndarray) -> C.c_void_p:
    return a.ctypes.data_as(C.c_void_p)


def schedule_valid(cut, n_layers: int, schedule) -> Tuple[bool, str]:
    """(valid, reason) for a (cut, schedule) pair."""
    c, cp = _host_i32(cut)
    s, sp = _host_i32(schedule)
    st = load().mpipe_schedule_valid(cp if c.size else None, s.size, int(n_layers), sp)
    return st == OK, ("" if st == OK else last_error())


class Derived:
    """derive(cut, schedule, model) read out into numpy arrays.

    layout, runs_bwd: [k]; slab_lo, slab_hi: [k, P]; owner: [M];
    seams: [k-1, 3] (left, fwd comm, bwd comm); reduces: [n, 2] (region, group);
    events: [n_events, 8] int32 with columns EVENT_FIELDS; edges: [n_edges, 3]
    (from, to, kind); nodes: list of P int32 arrays."""

    def __init__(self, cut, n_layers: int, schedule, trainable, n_ranks: int, n_mb: int,
                 owner=None):
        self.L = load()
        c, cp = _host_i32(cut)
        s, sp = _host_i32(schedule)
        t, tp = _host_i32(trainable)
        if t.size != s.size:
            raise MpipeError(-1, "one trainable bit per region")
        o, op = (None, None) if owner is None else _host_i32(owner)
        if o is not None and o.size != n_mb:
            raise MpipeError(-1, "one owner per micro-batch")
        h = C.c_void_p()
        _check(self.L.mpipe_derive(cp if c.size else None, s.size, int(n_layers), sp, tp,
                                   int(n_ranks), int(n_mb), op, C.byref(h)))
        self._h = h
        self.k, self.P, self.M = s.size, int(n_ranks), int(n_mb)
        ho, ne, nd, ns, nr = (C.c_int32() for _ in range(5))
        _check(self.L.mpipe_derived_shape(h, C.byref(ho), C.byref(ne), C.byref(nd),
                                          C.byref(ns), C.byref(nr)))
        self.has_order = bool(ho.value)
        self.layout = np.zeros(self.k, np.int32)
        self.runs_bwd = np.zeros(self.k, np.int32)
        self.slab_lo = np.zeros((self.k, self.P), np.int32)
        self.slab_hi = np.zeros((self.k, self.P), np.int32)
        for j in range(self.k):
            lay, rb = C.c_int32(), C.c_int32()
            _check(self.L.mpipe_derived_placement(h, j, C.byref(lay), C.byref(rb),
                                                  _vp(self.slab_lo[j]), _vp(self.slab_hi[j])))
            self.layout[j], self.runs_bwd[j] = lay.value, rb.value
        self.owner = np.zeros(self.M, np.int32)
        _check(self.L.mpipe_derived_owner(h, _vp(self.owner)))
        self.events = np.zeros((ne.value, 8), np.int32)
        self.edges = np.zeros((nd.value, 3), np.int32)
        self.seams = np.zeros((ns.value, 3), np.int32)
        red_r = np.zeros(nr.value, np.int32)
        red_g = np.zeros(nr.value, np.int32)
        _check(self.L.mpipe_derived_lists(h, _vp(self.events), _vp(self.edges), _vp(self.seams),
                                          _vp(red_r), _vp(red_g)))
        self.reduces = np.stack([red_r, red_g], axis=1) if nr.value else np.zeros((0, 2), np.int32)
        self.nodes = []
        for r in range(self.P):
            n = self.L.mpipe_derived_nodes(h, r, None, 0)
            if n < 0:
                raise MpipeError(-1, last_error())
            v = np.zeros(n, np.int32)
            self.L.mpipe_derived_nodes(h, r, _vp(v), n)
            self.nodes.append(v)

    def __del__(self):
        h = getattr(self, "_h", None)
        if h is not None and h.value:
            self.L.mpipe_derived_destroy(h)
            self._h = None

    def event_costs(self, fwd_cost, bwd_cost, seam_bytes, reduce_bytes, alpha: float,
                    beta: float, loss_cost: float) -> np.ndarray:
        """Cost of every event (Sec. 4.3); fwd_cost/bwd_cost [k, M] seconds of a whole
        region, seam_bytes [k-1, M], reduce_bytes [k]."""
        f = np.ascontiguousarray(fwd_cost, dtype=np.float64).reshape(-1)
        b = np.ascontiguousarray(bwd_cost, dtype=np.float64).reshape(-1)
        sb = np.ascontiguousarray(seam_bytes, dtype=np.float64).reshape(-1)
        rb = np.ascontiguousarray(reduce_bytes, dtype=np.float64).reshape(-1)
        if f.size != self.k * self.M or b.size != self.k * self.M or rb.size != self.k \
                or sb.size != (self.k - 1) * self.M:
            raise MpipeError(-1, "cost arrays do not match (k, M)")
        out = np.zeros(self.events.shape[0], np.float64)
        _check(self.L.mpipe_event_costs(self._h, _vp(f), _vp(b), _vp(sb) if sb.size else None,
                                        _vp(rb), float(alpha), float(beta), float(loss_cost),
                                        _vp(out)))
        return out

    def makespan(self, cost):
        """(T, bubble [P], start [n_events], finish [n_events])."""
        c = np.ascontiguousarray(cost, dtype=np.float64)
        if c.size != self.events.shape[0]:
            raise MpipeError(-1, "one cost per event")
        T = C.c_double()
        bub = np.zeros(self.P, np.float64)
        st = np.zeros(c.size, np.float64)
        fin = np.zeros(c.size, np.float64)
        _check(self.L.mpipe_makespan(self._h, _vp(c), C.byref(T), _vp(bub), _vp(st), _vp(fin)))
        return T.value, bub, st, fin

    def memory_peak(self, act_bytes) -> np.ndarray:
        a = np.ascontiguousarray(act_bytes, dtype=np.float64)
        if a.size != self.events.shape[0]:
            raise MpipeError(-1, "one byte count per event")
        out = np.zeros(self.P, np.float64)
        _check(self.L.mpipe_memory_peak(self._h, _vp(a), _vp(out)))
        return out


def merge_scatter(merged, placeholder_idx, embeds, stream=None) -> None:
    """embeds.view(-1, H)[idx[j]] = merged[j] (bit-exact, in place)."""
    H = merged.shape[-1]
    n_rows = embeds.numel() // H
    _check(load().mpipe_merge_scatter(_ptr(merged), merged.shape[0], H, _dt(merged),
                                      _ptr(placeholder_idx), _ptr(embeds), n_rows,
                                      _stream(stream)))


def merge_gather(d_embeds, placeholder_idx, d_merged, stream=None) -> None:
    """d_merged[j] = d_embeds.view(-1, H)[idx[j]]."""
    H = d_merged.shape[-1]
    n_rows = d_embeds.numel() // H
    _check(load().mpipe_merge_gather(_ptr(d_embeds), n_rows, H, _dt(d_embeds),
                                     _ptr(placeholder_idx), d_merged.shape[0], _ptr(d_merged),
                                     _stream(stream)))


def merge_check_indices(placeholder_idx, n_rows: int, marks, status, stream=None) -> None:
    _check(load().mpipe_merge_check_indices(_ptr(placeholder_idx), placeholder_idx.numel(),
                                            n_rows, _ptr(marks), _ptr(status), _stream(stream)))


def merge_check_indices_noalloc(placeholder_idx, n_rows: int, status, stream=None) -> None:
    """mpipe_merge_check_indices without a caller buffer (the library's built-in
    counters; n_rows <= CHECK_NOALLOC_MAX_ROWS)."""
    _check(load().mpipe_merge_check_indices_noalloc(_ptr(placeholder_idx),
                                                    placeholder_idx.numel(), n_rows,
                                                    _ptr(status), _stream(stream)))


CHECK_NOALLOC_MAX_ROWS = 1 << 20   # MPIPE_CHECK_NOALLOC_MAX_ROWS of include/mpipe.h


# --------------------------------------------------------------------------
# Kernel-level ops
# --------------------------------------------------------------------------

def op_scratch_bytes(N: int, heads: int, n: int, n_seg: int) -> int:
    return int(load().mpipe_op_scratch_bytes(N, heads, n, n_seg))


def op_gemm(dtype: int, layout: int, epilogue: int, M: int, N: int, K: int, A, lda: int, B,
            ldb: int, Cout, ldc: int, bias=None, aux=None, ld_aux: int = 0, C2=None,
            ldc2: int = 0, beta: int = 0, k_per_split: int = 0, split_stride: int = 0,
            stream=None) -> None:
    _check(load().mpipe_op_gemm(dtype, layout, epilogue, M, N, K, _ptr(A), lda, _ptr(B), ldb,
                                _ptr(Cout), ldc, _ptr(bias), _ptr(aux), ld_aux, _ptr(C2), ldc2,
                                beta, k_per_split, split_stride, _stream(stream)))


GEMM_KERNELS = ("general", "f32_32x32", "64x64", "64x128", "128x128", "large")


def gemm_kernel(dtype: int, layout: int, epilogue: int, M: int, N: int, K: int,
                k_per_split: int = 0) -> str:
    """The kernel op_gemm runs a product of dense, 16-byte aligned operands on."""
    k = int(load().mpipe_op_gemm_kernel(dtype, layout, epilogue, M, N, K, k_per_split))
    if k < 0:
        raise MpipeError(-1, "gemm_kernel: argument out of range")
    return GEMM_KERNELS[k]


def op_splitk_reduce(part, splits: int, M: int, N: int, out, ldo: int, stream=None) -> None:
    _check(load().mpipe_op_splitk_reduce(_ptr(part), splits, M, N, _ptr(out), ldo,
                                         _stream(stream)))


def gemm_split(M: int, N: int, K: int) -> int:
    """K splits of the backward's weight-gradient product dW[M][N] over K tokens."""
    return int(load().mpipe_op_weight_grad_splits(M, N, K))


def op_layernorm_fwd(dtype, X, rows, n, g, b, eps, Y, mean=None, rstd=None, stream=None):
    _check(load().mpipe_op_layernorm_fwd(dtype, _ptr(X), rows, n, _ptr(g), _ptr(b), eps, _ptr(Y),
                                         _ptr(mean), _ptr(rstd), _stream(stream)))


def op_layernorm_bwd(dtype, dY, X, mean, rstd, g, rows, n, dres, dX, dXt, grad_g, grad_b,
                     scratch, stream=None, colsum_dx=None):
    _check(load().mpipe_op_layernorm_bwd(dtype, _ptr(dY), _ptr(X), _ptr(mean), _ptr(rstd), _ptr(g),
                                         rows, n, _ptr(dres), _ptr(dX), _ptr(dXt), _ptr(grad_g),
                                         _ptr(grad_b), _ptr(colsum_dx), _ptr(scratch),
                                         scratch.numel() * scratch.element_size(),
                                         _stream(stream)))


def op_rope(dtype, qkv, rows, heads, head_dim, grid_thw, theta, inverse, scratch, stream=None):
    g, gp = _host_i32(np.asarray(grid_thw).reshape(-1, 3))
    _check(load().mpipe_op_rope(dtype, _ptr(qkv), rows, heads, head_dim, gp, g.shape[0], theta,
                                int(inverse), _ptr(scratch),
                                scratch.numel() * scratch.element_size(), _stream(stream)))


def op_attention_fwd(dtype, qkv, N, heads, head_dim, cu_seqlens, o, lse, scratch, stream=None):
    cu, cup = _host_i32(cu_seqlens)
    _check(load().mpipe_op_attention_fwd(dtype, _ptr(qkv), N, heads, head_dim, cup,
                                         max(len(cu) - 1, 0), _ptr(o), _ptr(lse), _ptr(scratch),
                                         scratch.numel() * scratch.element_size(),
                                         _stream(stream)))


def op_attention_bwd(dtype, qkv, o, d_o, lse, N, heads, head_dim, cu_seqlens, dqkv, scratch,
                     stream=None):
    cu, cup = _host_i32(cu_seqlens)
    _check(load().mpipe_op_attention_bwd(dtype, _ptr(qkv), _ptr(o), _ptr(d_o), _ptr(lse), N,
                                         heads, head_dim, cup, max(len(cu) - 1, 0), _ptr(dqkv),
                                         _ptr(scratch), scratch.numel() * scratch.element_size(),
                                         _stream(stream)))


# --------------------------------------------------------------------------
# The first LLM layer behind the seam, and the end of a trained step
# --------------------------------------------------------------------------

def _bad(msg: str) -> None:
    raise MpipeError(-1, msg)


def _launch(fn, dev: int, stream, *args) -> None:
    """fn(*args, stream) with GPU `dev` (of every tensor of the call) current, which it need
    not be before; the stream is that GPU's current one unless given."""
    import torch
    if dev < 0:
        _bad("tensors must be on the GPU")
    if stream is None:
        # the current stream's handle alone (0.1 us; a Stream object around it takes 1.1)
        handle = torch._C._cuda_getCurrentRawStream(dev)
    elif stream.device_index != dev:
        _bad("a stream of another device than the tensors'")
    else:
        handle = stream.cuda_stream
    here = torch.cuda.current_device()
    if here == dev:
        _check(fn(*args, handle))
        return
    torch.cuda.set_device(dev)
    try:
        _check(fn(*args, handle))
    finally:
        torch.cuda.set_device(here)


def _host_ints(a, name: str, dtype=np.int64) -> np.ndarray:
    """A list of whole numbers as the library reads it."""
    if type(a) is np.ndarray and a.dtype == dtype and a.ndim == 1:
        return a
    arr = np.asarray(a)
    if arr.ndim != 1 or not (arr.size == 0 or arr.dtype.kind in "iu"):
        _bad(f"{name}: a list of whole numbers")
    lim = np.iinfo(dtype)
    if arr.size and (int(arr.min()) < lim.min or int(arr.max()) > lim.max):
        _bad(f"{name}: a value beyond {lim.bits} bits")
    return arr.astype(dtype)


def op_seam_positions(seq_row, seq_len, item_row, grid_thw, pos, seq_pos=None, time_step=None,
                      stream=None) -> np.ndarray:
    """pos[:, row] (int32 [3][rows], rows adjacent) = the (time, height, width) position of
    every row of the sequences [seq_row, seq_row + seq_len); rows of none are left as they
    were.  Item i's merged rows start at row item_row[i] with the encoder's grid_thw[i].
    Returns the position behind each sequence's last row, which is `seq_pos` when it goes on."""
    import torch
    sr, sl = _host_ints(seq_row, "seq_row"), _host_ints(seq_len, "seq_len")
    sp = None if seq_pos is None else _host_ints(seq_pos, "seq_pos")
    ir = _host_ints(item_row, "item_row")
    g = _host_ints(np.asarray(grid_thw).reshape(-1), "grid_thw", np.int32)
    ts = None if time_step is None else _host_ints(time_step, "time_step", np.int32)
    if sl.size != sr.size or (sp is not None and sp.size != sr.size):
        _bad("seq_row, seq_len and seq_pos differ in length")
    if g.size != 3 * ir.size or (ts is not None and ts.size != ir.size):
        _bad("item_row, grid_thw and time_step differ in length")
    if (pos.dtype is not torch.int32 or pos.dim() != 2 or pos.shape[0] != 3 or
            (pos.shape[1] > 1 and pos.stride(1) != 1)):
        _bad("pos: int32 [3][rows], rows adjacent")
    nxt = np.zeros(sr.size, np.int64)
    # (the arrays' bytes: ctypes passes their address at once)
    _launch(load().mpipe_op_seam_positions, pos.get_device(), stream, sr.tobytes(), sl.tobytes(),
            None if sp is None else sp.tobytes(), sr.size, ir.tobytes(), g.tobytes(),
            None if ts is None else ts.tobytes(), ir.size, pos.shape[1], pos.data_ptr(),
            pos.stride(0), nxt.ctypes.data)
    return nxt


_HEADS = struct.Struct("PqqiI")    # mpipe_heads


def _qk(cfg, pos, q, k, q_more, k_more):
    """(torch dtype, rows, device, views of q and of q_more, of k and of k_more): q and k
    [rows][heads][head_dim] with any strides of rows and heads, either may be None, and what
    goes with each of the same shape.  A view is an mpipe_heads; None: no heads."""
    import torch
    one = q if q is not None else k
    if one is None:
        _bad("neither q nor k")
    rows, dtype, dev, views = one.shape[0], one.dtype, one.get_device(), []
    for x, more in ((q, q_more), (k, k_more)):
        if x is None:
            if any(y is not None for y in more):
                _bad("an output or gradient of q or k without its input")
            views.append((None,) * (1 + len(more)))
            continue
        shape = x.shape
        if len(shape) != 3 or shape[0] != rows or shape[2] != cfg.head_dim:
            _bad("q and k: [rows][heads][head_dim]")
        heads, v = shape[1], []
        for y in (x, *more):
            if y is None:
                _bad("q or k without its output or gradient")
            if y.dtype is not dtype or (y is not x and y.shape != shape):
                _bad("inputs, gradients and outputs differ in shape or dtype")
            rs, hs, cs = y.stride()
            if cs != 1:
                _bad("the columns of a head must be adjacent")
            if y.get_device() != dev:
                _bad("tensors on different devices")
            v.append(_HEADS.pack(y.data_ptr(), rs, hs, heads, 0))
        views.append(v)
    if (pos.dtype is not torch.int32 or pos.dim() != 2 or pos.shape[0] != cfg.axes or
            pos.shape[1] != rows or (rows > 1 and pos.stride(1) != 1)):
        _bad("pos: int32 [axes][rows], rows adjacent")
    if pos.get_device() != dev:
        _bad("tensors on different devices")
    return dtype, rows, dev, views[0], views[1]


def _vector(t, n: int, dtype, dev: int, what: str) -> int:
    """The address of a vector of n."""
    if t.dtype is not dtype or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        _bad(what)
    if t.get_device() != dev:
        _bad("tensors on different devices")
    return t.data_ptr()


def _buffer(t, dev: int) -> Tuple[Optional[int], int]:
    """Address and bytes of scratch."""
    if t is None:
        return None, 0
    if not t.is_contiguous():
        _bad("scratch must be contiguous")
    if t.get_device() != dev:
        _bad("tensors on different devices")
    return t.data_ptr(), t.numel() * t.element_size()


def _code(dtype) -> int:
    import torch
    if dtype is torch.bfloat16:
        return BF16
    if dtype is torch.float32:
        return F32
    raise MpipeError(-1, f"unsupported dtype {dtype}")


def op_rope_axes(cfg, q, k, pos, q_out, k_out, inverse: bool = False, stream=None) -> None:
    """q_out, k_out = q, k ([rows][heads][head_dim], any strides of rows and heads; k and
    k_out may be None) turned by pos (int32 [axes][rows], or one row of positions expanded to
    all axes); inverse turns back (the gradient).  An output may be its own input."""
    dtype, rows, dev, (q, qo), (k, ko) = _qk(cfg, pos, q, k, (q_out,), (k_out,))
    _launch(load().mpipe_op_rope_axes, dev, stream, _code(dtype), C.byref(cfg), rows, q, k,
            pos.data_ptr(), pos.stride(0), 1 if inverse else 0, qo, ko)


_GAIN = "gains: [head_dim] in the heads' dtype"
_GAIN_GRAD = "gain gradients: fp32 [head_dim]"


def op_qk_norm_rope_fwd(cfg, q, k, q_gain, k_gain, eps: float, pos, q_out, k_out,
                        stream=None) -> None:
    """The same behind a root-mean-square norm of every head with a gain [head_dim]."""
    dtype, rows, dev, (q, qo), (k, ko) = _qk(cfg, pos, q, k, (q_out,), (k_out,))
    gains = [None if g is None else _vector(g, cfg.head_dim, dtype, dev, _GAIN)
             for g in (q_gain, k_gain)]
    _launch(load().mpipe_op_qk_norm_rope_fwd, dev, stream, _code(dtype), C.byref(cfg), rows, q, k,
            *gains, eps, pos.data_ptr(), pos.stride(0), qo, ko)


def op_qk_norm_rope_scratch_bytes(rows: int, heads_q: int, heads_k: int, head_dim: int) -> int:
    n = int(load().mpipe_op_qk_norm_rope_scratch_bytes(rows, heads_q, heads_k, head_dim))
    if n == 0:
        _bad("op_qk_norm_rope_scratch_bytes: argument out of range")
    return n


def op_qk_norm_rope_bwd(cfg, dq, dk, q, k, q_gain, k_gain, eps: float, pos, dq_in, dk_in,
                        grad_q_gain, grad_k_gain, scratch, accumulate: bool = True,
                        stream=None) -> None:
    """Gradients of op_qk_norm_rope_fwd: dq_in, dk_in from dq, dk (they may be the same
    tensors) and the forward's q, k, gains, eps and positions; grad_q_gain, grad_k_gain (fp32
    [head_dim], may be None) are added to, or overwritten with accumulate=False.  scratch:
    op_qk_norm_rope_scratch_bytes."""
    import torch
    if (q is None and grad_q_gain is not None) or (k is None and grad_k_gain is not None):
        _bad("a gain's gradient without its heads")
    dtype, rows, dev, (q, dq, qi), (k, dk, ki) = _qk(cfg, pos, q, k, (dq, dq_in), (dk, dk_in))
    d, f32 = cfg.head_dim, torch.float32
    gains = [None if g is None else _vector(g, d, dtype, dev, _GAIN) for g in (q_gain, k_gain)]
    grads = [None if g is None else _vector(g, d, f32, dev, _GAIN_GRAD)
             for g in (grad_q_gain, grad_k_gain)]
    _launch(load().mpipe_op_qk_norm_rope_bwd, dev, stream, _code(dtype), C.byref(cfg), rows, dq,
            dk, q, k, *gains, eps, pos.data_ptr(), pos.stride(0), qi, ki, *grads,
            1 if accumulate else 0, *_buffer(scratch, dev))


class GradList:
    """The tensors of a gradient (fp32 or bf16, contiguous, one GPU) as the calls take them;
    it keeps them alive.  Made once for buffers that stay, or for every call.  A tensor whose
    memory was replaced since (`.data`, `set_`, a growing `resize_`) is taken with its new one."""

    def __init__(self, tensors):
        import torch
        self.address = torch.Tensor.data_ptr
        self.tensors = list(tensors)
        self.n = len(self.tensors)
        self.array = (_GradTensor * max(self.n, 1))()
        self._read()

    def _read(self):
        self.at = None      # read again by the next call if this one refuses a tensor
        self.dev = self.tensors[0].get_device() if self.n else None
        at, keep = [], []
        for a, t in zip(self.array, self.tensors):
            if not t.is_contiguous():
                _bad("gradients must be contiguous")
            if t.get_device() != self.dev:
                _bad("tensors on different devices")
            p = t.data_ptr()
            a.data, a.n, a.dtype = p, t.numel(), _code(t.dtype)
            at.append(p)
            keep.append(t.untyped_storage())
        # with the memory itself kept, no other tensor can come to lie at a known address
        self.at, self.keep = at, keep

    def now(self) -> "GradList":
        """The list with the tensors' present memory (1.2 us to see that 32 have not moved)."""
        if list(map(self.address, self.tensors)) != self.at:
            self._read()
        return self


def _grad_list(grads) -> GradList:
    return grads.now() if isinstance(grads, GradList) else GradList(grads)


def op_grad_scratch_bytes(grads) -> int:
    """Scratch of op_grad_norm for these tensors (a GradList or tensors)."""
    g = _grad_list(grads)
    n = int(load().mpipe_op_grad_scratch_bytes(g.array, g.n))
    if n == 0:
        raise MpipeError(-1, last_error())
    return n


def _result(t, n: int, dtype, dev: int, what: str) -> int:
    if t.dtype is not dtype or t.numel() != n or not t.is_contiguous():
        _bad(what)
    if t.get_device() != dev:
        _bad("tensors on different devices")
    return t.data_ptr()


def op_grad_norm(grads, sumsq, norms, scratch, stream=None) -> None:
    """sumsq (fp64 [1]) = the sum of squares over all of grads (a GradList or tensors);
    norms (fp32 [tensors], may be None) = each one's L2 norm."""
    import torch
    g, dev = _grad_list(grads), sumsq.get_device()
    if g.dev not in (None, dev):
        _bad("tensors on different devices")
    _launch(load().mpipe_op_grad_norm, dev, stream, g.array, g.n,
            _result(sumsq, 1, torch.float64, dev, "sumsq: fp64 [1]"),
            None if norms is None else _result(norms, g.n, torch.float32, dev,
                                               "norms: fp32 [tensors]"), *_buffer(scratch, dev))


def op_grad_clip(grads, sumsq, max_norm: float, norm=None, out=None, stream=None) -> None:
    """Scale grads to the norm max_norm where sqrt(sumsq) is above it (and finite): in place,
    or into `out` (tensors of the same lengths, fp32 or bf16, always written).  norm (fp32
    [1], may be None) = sqrt(sumsq)."""
    import torch
    g, o, dev = _grad_list(grads), None if out is None else _grad_list(out), sumsq.get_device()
    if g.dev not in (None, dev) or (o is not None and o.dev not in (None, dev)):
        _bad("tensors on different devices")
    if o is not None and o.n != g.n:
        _bad("grads and out differ in number")
    _launch(load().mpipe_op_grad_clip, dev, stream, g.array, None if o is None else o.array, g.n,
            _result(sumsq, 1, torch.float64, dev, "sumsq: fp64 [1]"), max_norm,
            None if norm is None else _result(norm, 1, torch.float32, dev, "norm: fp32 [1]"))


# --------------------------------------------------------------------------
# The first LLM layer's attention
# --------------------------------------------------------------------------

def _view(t, rows: int, d: int, dtype, dev: int, what: str) -> bytes:
    """An mpipe_heads of [rows][heads][d], any strides of rows and heads."""
    shape = t.shape
    if len(shape) != 3 or shape[0] != rows or shape[2] != d or t.dtype is not dtype:
        _bad(what)
    rs, hs, cs = t.stride()
    if cs != 1:
        _bad("the columns of a head must be adjacent")
    if t.get_device() != dev:
        _bad("tensors on different devices")
    return _HEADS.pack(t.data_ptr(), rs, hs, shape[1], 0)


def _lse(t, heads: int, rows: int, dev: int) -> Tuple[Optional[int], int]:
    import torch
    if t is None:
        return None, 0
    stride = t.stride()
    if (t.dtype is not torch.float32 or t.shape != (heads, rows) or
            (rows > 1 and stride[1] != 1)):
        _bad("lse: fp32 [heads of q][rows], rows adjacent")
    if t.get_device() != dev:
        _bad("tensors on different devices")
    return t.data_ptr(), stride[0] if heads > 1 else rows


def _sequence_lists(seq_row, seq_len, key_row, key_len):
    sr, sl = _host_ints(seq_row, "seq_row"), _host_ints(seq_len, "seq_len")
    if (key_row is None) != (key_len is None):
        _bad("key_row and key_len go together")
    kr = None if key_row is None else _host_ints(key_row, "key_row")
    kl = None if key_len is None else _host_ints(key_len, "key_len")
    n = sr.size
    if sl.size != n or (kr is not None and (kr.size != n or kl.size != n)):
        _bad("seq_row, seq_len, key_row and key_len differ in length")
    return (sr.tobytes(), sl.tobytes(), None if kr is None else kr.tobytes(),
            None if kl is None else kl.tobytes(), n)


_ATTN_Q = "q, o and their gradients: [rows][heads][head_dim] of one dtype"
_ATTN_K = "k, v and their gradients: [key rows][key heads][head_dim] in the dtype of q"


def _attn_shapes(q, k):
    of_q, of_k = q.shape, k.shape
    if len(of_q) != 3 or len(of_k) != 3:
        _bad(_ATTN_Q)
    return of_q[0], of_q[1], of_k[0], of_q[2], q.dtype, q.get_device()


def op_causal_attention_fwd(q, k, v, o, lse, seq_row, seq_len, key_row=None, key_len=None,
                            scale: Optional[float] = None, stream=None) -> None:
    """o ([rows][heads][head_dim]) = causal attention of q over k, v ([key rows][key heads]
    [head_dim], any strides of rows and heads), sequence s being the rows seq_row[s] .. +
    seq_len[s] and its keys key_row[s] .. + key_len[s] (the same rows unless given); they end
    together, so more keys are a prefix.  lse (fp32 [heads][rows], may be None) for the
    backward.  scale: head_dim ** -0.5 unless given.  Rows of no sequence are left as they
    were."""
    rq, hq, rk, d, dtype, dev = _attn_shapes(q, k)
    p, ld = _lse(lse, hq, rq, dev)
    _launch(load().mpipe_op_causal_attention_fwd, dev, stream, _code(dtype), d, rq, rk,
            _view(q, rq, d, dtype, dev, _ATTN_Q), _view(k, rk, d, dtype, dev, _ATTN_K),
            _view(v, rk, d, dtype, dev, _ATTN_K),
            *_sequence_lists(seq_row, seq_len, key_row, key_len),
            d ** -0.5 if scale is None else scale, _view(o, rq, d, dtype, dev, _ATTN_Q), p, ld)


def op_causal_attention_scratch_bytes(rows: int, heads: int, key_rows: int, key_heads: int,
                                      head_dim: int) -> int:
    n = int(load().mpipe_op_causal_attention_scratch_bytes(rows, heads, key_rows, key_heads,
                                                           head_dim))
    if n == 0:
        _bad("op_causal_attention_scratch_bytes: argument out of range")
    return n


def op_causal_attention_bwd(d_o, q, k, v, o, lse, seq_row, seq_len, dq, dk, dv, scratch,
                            key_row=None, key_len=None, scale: Optional[float] = None,
                            stream=None) -> None:
    """Gradients of op_causal_attention_fwd from d_o, the gradient of o, and what the forward took
    and gave: dq, dk, dv overwritten in the sequences' rows (they may be columns of one product).
    scratch: op_causal_attention_scratch_bytes."""
    rq, hq, rk, d, dtype, dev = _attn_shapes(q, k)
    if lse is None:
        _bad("the backward needs lse")
    p, ld = _lse(lse, hq, rq, dev)
    _launch(load().mpipe_op_causal_attention_bwd, dev, stream, _code(dtype), d, rq, rk,
            _view(d_o, rq, d, dtype, dev, _ATTN_Q), _view(q, rq, d, dtype, dev, _ATTN_Q),
            _view(k, rk, d, dtype, dev, _ATTN_K), _view(v, rk, d, dtype, dev, _ATTN_K),
            _view(o, rq, d, dtype, dev, _ATTN_Q), p, ld,
            *_sequence_lists(seq_row, seq_len, key_row, key_len),
            d ** -0.5 if scale is None else scale, _view(dq, rq, d, dtype, dev, _ATTN_Q),
            _view(dk, rk, d, dtype, dev, _ATTN_K), _view(dv, rk, d, dtype, dev, _ATTN_K),
            *_buffer(scratch, dev))


_KV_CACHE = struct.Struct("PPPPqiiii")    # mpipe_kv_cache
E4M3 = 2


class KvCache:
    """The pages of a key-value cache: k, v [pages][heads][page][head_dim] (contiguous; fp32,
    bf16 or torch.float8_e4m3fn, a page's tokens a power of two) and for 8 bits k_scale, v_scale,
    uint8 [pages][heads][page], which hold the exponent + 127 of each token's power of two.
    It keeps the tensors; their memory must stay where it is."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        import torch
        if k.dim() != 4 or v.shape != k.shape or v.dtype is not k.dtype:
            _bad("k and v: [pages][heads][page][head_dim] of one dtype")
        eight = k.dtype is torch.float8_e4m3fn
        self.dtype = E4M3 if eight else _code(k.dtype)
        if eight != (k_scale is not None) or eight != (v_scale is not None):
            _bad("scales go with 8-bit pages, and only with them")
        self.tensors = [t for t in (k, v, k_scale, v_scale) if t is not None]
        for t in self.tensors[2:]:
            if t.dtype is not torch.uint8 or t.shape != k.shape[:3]:
                _bad("scales: uint8 [pages][heads][page]")
        self.dev = k.get_device()
        for t in self.tensors:
            if not t.is_contiguous():
                _bad("the cache must be contiguous")
            if t.get_device() != self.dev:
                _bad("tensors on different devices")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.pages, self.heads, self.page, self.head_dim = k.shape

    def _now(self) -> bytes:
        return _KV_CACHE.pack(self.k.data_ptr(), self.v.data_ptr(),
                              0 if self.k_scale is None else self.k_scale.data_ptr(),
                              0 if self.v_scale is None else self.v_scale.data_ptr(), self.pages,
                              self.heads, self.page, self.head_dim, self.dtype)


def _table(table, dev: int) -> Tuple[int, int, int, int]:
    """Address, stride, sequences and width of page tables."""
    import torch
    if (table.dtype is not torch.int32 or table.dim() != 2 or
            (table.shape[1] > 1 and table.stride(1) != 1)):
        _bad("table: int32 [sequences][pages], a sequence's pages adjacent")
    if table.get_device() != dev:
        _bad("tensors on different devices")
    n, width = table.shape
    return table.data_ptr(), table.stride(0) if n > 1 else width, n, width


def _row_ints(t, rows: int, dev: int, what: str) -> Optional[int]:
    import torch
    return None if t is None else _vector(t, rows, torch.int32, dev, what)


def _cache_rows(cache, k, v, table, pos, seq, status):
    import torch
    what = "k and v: [rows][heads][head_dim] of one dtype"
    if k.dim() != 3:
        _bad(what)
    rows, d, dtype, dev = k.shape[0], cache.head_dim, k.dtype, cache.dev
    if pos is None:
        _bad("pos: int32 [rows]")
    return (rows, _code(dtype), _view(k, rows, d, dtype, dev, what),
            _view(v, rows, d, dtype, dev, what), _table(table, dev),
            _row_ints(seq, rows, dev, "seq: int32 [rows]"),
            _row_ints(pos, rows, dev, "pos: int32 [rows]"),
            None if status is None else _result(status, 1, torch.int32, dev, "status: int32 [1]"))


def op_cache_write(cache, k, v, table, pos, seq=None, status=None, stream=None) -> None:
    """Row i of k and v ([rows][heads][head_dim], fp32 or bf16, any strides of rows and heads)
    to token pos[i] of sequence seq[i] (int32; sequence i unless given), whose pages are
    table[seq[i]] (int32).  Rows with a negative pos or seq are left out; rows of a place
    outside the tables or the pool too, and status (int32 [1], may be None) becomes 1."""
    rows, code, kv, vv, tab, seq, pos, status = _cache_rows(cache, k, v, table, pos, seq, status)
    _launch(load().mpipe_op_cache_write, cache.dev, stream, cache._now(), code, rows, kv, vv,
            *tab, seq, pos, status)


def op_cache_read(cache, table, pos, k, v, seq=None, status=None, stream=None) -> None:
    """The other way: the keys and values of token pos[i] of sequence seq[i] into row i of k and
    v.  Rows left out keep what they held; rows of a bad place become NaN."""
    rows, code, kv, vv, tab, seq, pos, status = _cache_rows(cache, k, v, table, pos, seq, status)
    _launch(load().mpipe_op_cache_read, cache.dev, stream, cache._now(), code, rows, *tab, seq,
            pos, kv, vv, status)


def op_cache_attention(cache, q, table, lens, o, scratch, lse=None, scale: Optional[float] = None,
                       stream=None) -> None:
    """o[s] = attention of q[s] ([sequences][heads][head_dim]), the new token of sequence s, over
    its lens[s] (int32) tokens in the cache, the new one's own among them.  lse: fp32
    [heads][sequences], may be None.  scratch: op_cache_attention_scratch_bytes."""
    import torch
    if q.dim() != 3:
        _bad(_ATTN_Q)
    n, d, dtype, dev = q.shape[0], cache.head_dim, q.dtype, cache.dev
    at, ld, seqs, width = _table(table, dev)
    if seqs != n:
        _bad("table and q differ in sequences")
    p, ld_lse = _lse(lse, q.shape[1], n, dev)
    _launch(load().mpipe_op_cache_attention, dev, stream, cache._now(), _code(dtype), n,
            _view(q, n, d, dtype, dev, _ATTN_Q), at, ld, width,
            _vector(lens, n, torch.int32, dev, "lens: int32 [sequences]"),
            d ** -0.5 if scale is None else scale, _view(o, n, d, dtype, dev, _ATTN_Q), p, ld_lse,
            *_buffer(scratch, dev))


def op_cache_attention_scratch_bytes(seqs: int, heads: int, key_heads: int, head_dim: int) -> int:
    n = int(load().mpipe_op_cache_attention_scratch_bytes(seqs, heads, key_heads, head_dim))
    if n == 0:
        _bad("op_cache_attention_scratch_bytes: argument out of range")
    return n
