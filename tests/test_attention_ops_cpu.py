"""What the attention and cache calls refuse, on the host (no GPU: a refused call launches
nothing), and the float64 forms the GPU tests compare with."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2607_03229_amd as mp
from paper_2607_03229_amd import _binding as B
from tests import attn_ref as R

FAKE = 1 << 20          # addresses that only the checks look at, 16 MiB apart
STEP = 1 << 24


@pytest.fixture(scope="module")
def L():
    try:
        return mp.load()
    except mp.MpipeError:
        pytest.skip("libmpipe.so is not built")


def at(i):
    return FAKE + i * STEP


def heads(p, n=8, row=None, head=64):
    return B._HEADS.pack(p or 0, n * head if row is None else row, head, n, 0)


def ints(a):
    return None if a is None else np.asarray(a, np.int64).tobytes()


def fwd(L, dtype=1, d=64, rows_q=100, rows_k=100, q=None, k=None, v=None, seq_row=(0, 40),
        seq_len=(40, 60), key_row=None, key_len=None, n=None, scale=0.125, o=None, lse=at(9), ld=100):
    return L.mpipe_op_causal_attention_fwd(
        dtype, d, rows_q, rows_k, q or heads(at(0)), k or heads(at(1), 2), v or heads(at(2), 2),
        ints(seq_row), ints(seq_len), ints(key_row), ints(key_len),
        len(seq_row or ()) if n is None else n, scale, o or heads(at(3)), lse, ld, None)


BAD_FWD = {
    "bad_dtype": (-1, dict(dtype=2)),
    "head_dim_0": (-5, dict(d=0)),
    "head_dim_12": (-5, dict(d=12)),
    "head_dim_264": (-5, dict(d=264)),
    "scale_0": (-1, dict(scale=0.0)),
    "scale_negative": (-1, dict(scale=-1.0)),
    "scale_nan": (-1, dict(scale=math.nan)),
    "scale_inf": (-1, dict(scale=math.inf)),
    "negative_rows": (-1, dict(rows_q=-1)),
    "too_many_rows": (-5, dict(rows_k=2 ** 31)),
    "negative_sequences": (-1, dict(n=-1)),
    "null_lists": (-1, dict(seq_row=None, seq_len=None, n=2)),
    "key_row_alone": (-1, dict(key_row=(0, 40))),
    "key_len_alone": (-1, dict(key_len=(40, 60))),
    "negative_length": (-1, dict(seq_len=(40, -1))),
    "negative_first_row": (-1, dict(seq_row=(-1, 40))),
    "past_the_rows": (-1, dict(seq_len=(40, 61))),
    "row_overflow": (-1, dict(seq_row=(0, 2 ** 62), seq_len=(40, 2 ** 62))),
    "rows_shared": (-1, dict(seq_row=(0, 39))),
    "keys_past_the_rows": (-1, dict(key_row=(0, 41), key_len=(40, 60))),
    "fewer_key_rows": (-1, dict(rows_k=99)),
    "heads_not_a_multiple": (-1, dict(k=heads(at(1), 3), v=heads(at(2), 3))),
    "more_key_heads": (-1, dict(k=heads(at(1), 16), v=heads(at(2), 16))),
    "no_key_heads": (-1, dict(k=heads(at(1), 0), v=heads(at(2), 0))),
    "no_query_heads": (-1, dict(q=heads(at(0), 0), o=heads(at(3), 0))),
    "k_and_v_differ": (-1, dict(v=heads(at(2), 4))),
    "o_differs": (-1, dict(o=heads(at(3), 4))),
    "null_q": (-1, dict(q=heads(None))),
    "null_o": (-1, dict(o=heads(None))),
    "misaligned": (-1, dict(q=heads(at(0) + 1))),
    "negative_stride": (-1, dict(q=heads(at(0), row=-64))),
    "stride_overflow": (-1, dict(q=heads(at(0), row=2 ** 62))),
    "o_rows_overlap": (-1, dict(o=heads(at(3), row=500))),
    "o_heads_overlap": (-1, dict(o=heads(at(3), head=32))),
    "o_over_q": (-1, dict(o=heads(at(0)))),
    "o_over_k": (-1, dict(o=heads(at(1)))),
    "o_over_v": (-1, dict(o=heads(at(2) + 128))),
    "lse_misaligned": (-1, dict(lse=at(9) + 2)),
    "ld_lse_below_rows": (-1, dict(ld=99)),
    "lse_over_o": (-1, dict(lse=at(3))),
    "lse_over_q": (-1, dict(lse=at(0) - 400)),
}


@pytest.mark.parametrize("name", BAD_FWD)
def test_forward_refused(L, name):
    status, kw = BAD_FWD[name]
    assert fwd(L, **kw) == status
    assert B.last_error()


def test_nothing_to_attend_to(L):
    assert fwd(L, seq_row=(), seq_len=()) == 0
    assert fwd(L, seq_row=(0, 0), seq_len=(0, 0)) == 0
    none = heads(None, 0)
    assert fwd(L, q=none, k=none, v=none, o=none) == 0
    assert fwd(L, rows_q=0, rows_k=0, q=heads(None), k=heads(None, 2), v=heads(None, 2),
               o=heads(None), seq_row=(0,), seq_len=(0,)) == 0


def bwd(L, rows_k=100, d_o=None, q=None, k=None, v=None, o=None, lse=at(9), ld=100, dq=None,
        dk=None, dv=None, scratch=at(20), nbytes=1 << 20, seq_row=(0, 40), seq_len=(40, 60),
        key_row=None, key_len=None):
    return L.mpipe_op_causal_attention_bwd(
        1, 64, 100, rows_k, d_o or heads(at(4)), q or heads(at(0)), k or heads(at(1), 2),
        v or heads(at(2), 2), o or heads(at(3)), lse, ld, ints(seq_row), ints(seq_len),
        ints(key_row), ints(key_len), len(seq_row), 0.125, dq or heads(at(5)),
        dk or heads(at(6), 2), dv or heads(at(7), 2), scratch, nbytes, None)


BAD_BWD = {
    "null_lse": (-1, dict(lse=None)),
    "null_scratch": (-3, dict(scratch=None)),
    "small_scratch": (-3, dict(nbytes=64)),
    "misaligned_scratch": (-1, dict(scratch=at(20) + 8)),
    "keys_shared": (-1, dict(key_row=(0, 30), key_len=(40, 60))),
    "dq_over_d_o": (-1, dict(dq=heads(at(4)))),
    "dq_over_q": (-1, dict(dq=heads(at(0)))),
    "dq_over_o": (-1, dict(dq=heads(at(3)))),
    "dk_over_k": (-1, dict(dk=heads(at(1), 2))),
    "dk_over_dv": (-1, dict(dk=heads(at(7), 2))),
    "dk_over_dq": (-1, dict(dk=heads(at(5) + 64 * 2, 2))),
    "dv_over_lse": (-1, dict(lse=at(7))),
    "scratch_over_dq": (-1, dict(scratch=at(5))),
    "scratch_over_lse": (-1, dict(scratch=at(9))),
    "scratch_over_v": (-1, dict(scratch=at(2))),
    "dk_other_heads": (-1, dict(dk=heads(at(6), 4))),
    "null_dv": (-1, dict(dv=heads(None, 2))),
    "other_row_counts": (-1, dict(rows_k=160, dk=heads(at(5) + 100, 2), key_row=(0, 80), key_len=(80, 80))),
}


@pytest.mark.parametrize("name", BAD_BWD)
def test_backward_refused(L, name):
    status, kw = BAD_BWD[name]
    assert bwd(L, **kw) == status
    assert B.last_error()


def test_scratch_queries(L):
    assert mp.op_causal_attention_scratch_bytes(0, 0, 0, 0, 64) > 0
    for bad in ((-1, 1, 1, 1, 64), (1, 1, 2 ** 31, 1, 64), (1, 3, 1, 2, 64), (1, 1, 1, 2, 64),
                (1, 1, 1, 1, 60), (1, 2, 1, 0, 64)):
        with pytest.raises(mp.MpipeError):
            mp.op_causal_attention_scratch_bytes(*bad)
    assert mp.op_cache_attention_scratch_bytes(0, 1, 1, 8) > 0
    for bad in ((-1, 1, 1, 64), (1, 0, 1, 64), (1, 3, 2, 64), (1, 1, 1, 300), (1, 1, 0, 64)):
        with pytest.raises(mp.MpipeError):
            mp.op_cache_attention_scratch_bytes(*bad)


def cache(k=at(0), v=at(1), ks=None, vs=None, pages=10, heads=2, page=16, d=64, dtype=1):
    return B._KV_CACHE.pack(k or 0, v or 0, ks or 0, vs or 0, pages, heads, page, d, dtype)


def rows(L, c=None, dtype=1, n=5, k=None, v=None, table=at(4), ld=8, n_seq=3, width=8, seq=at(5),
         pos=at(6), status=at(7), read=False):
    c = c or cache()
    k, v = k or heads(at(2), 2), v or heads(at(3), 2)
    if read:
        return L.mpipe_op_cache_read(c, dtype, n, table, ld, n_seq, width, seq, pos, k, v, status, None)
    return L.mpipe_op_cache_write(c, dtype, n, k, v, table, ld, n_seq, width, seq, pos, status, None)


BAD_CACHE = {
    "dtype": (-1, dict(dtype=3)),
    "head_dim": (-5, dict(d=60)),
    "wide": (-5, dict(d=264)),
    "page_0": (-5, dict(page=0)),
    "page_24": (-5, dict(page=24)),
    "page_2_17": (-5, dict(page=1 << 17)),
    "no_heads": (-1, dict(heads=0)),
    "no_pages": (-1, dict(pages=0)),
    "negative_pages": (-1, dict(pages=-1)),
    "too_many_pages": (-1, dict(pages=1 << 31)),
    "null_k": (-1, dict(k=None)),
    "misaligned": (-1, dict(v=at(1) + 8)),
    "scales_for_bf16": (-1, dict(ks=at(8), vs=at(9))),
    "no_scales_for_e4m3": (-1, dict(dtype=2)),
    "one_scale": (-1, dict(dtype=2, ks=at(8))),
    "k_is_v": (-1, dict(v=at(0))),
    "scales_in_pages": (-1, dict(dtype=2, ks=at(0), vs=at(9))),
    "one_buffer_of_scales": (-1, dict(dtype=2, ks=at(8), vs=at(8))),
}
BAD_ROWS = {
    "dtype": (-1, dict(dtype=2)),
    "negative_rows": (-1, dict(n=-1)),
    "too_many_rows": (-5, dict(n=2 ** 30 + 1)),
    "negative_sequences": (-1, dict(n_seq=-1)),
    "negative_width": (-1, dict(width=-1)),
    "null_table": (-1, dict(table=None)),
    "misaligned_table": (-1, dict(table=at(4) + 2)),
    "ld_table": (-1, dict(ld=7)),
    "null_pos": (-1, dict(pos=None)),
    "misaligned_pos": (-1, dict(pos=at(6) + 1)),
    "misaligned_seq": (-1, dict(seq=at(5) + 2)),
    "misaligned_status": (-1, dict(status=at(7) + 2)),
    "other_heads": (-1, dict(k=heads(at(2), 4))),
    "null_rows": (-1, dict(v=heads(None, 2))),
    "rows_in_the_cache": (-1, dict(k=heads(at(0) + 64, 2))),
    "status_in_pos": (-1, dict(status=at(6))),
    "status_in_table": (-1, dict(status=at(4) + 4)),
    "status_in_cache": (-1, dict(status=at(1))),
    "status_in_rows": (-1, dict(status=at(2))),
}


@pytest.mark.parametrize("read", [False, True])
@pytest.mark.parametrize("name", BAD_CACHE)
def test_caches_refused(L, name, read):
    status, kw = BAD_CACHE[name]
    n = kw.get("heads", 2)
    assert rows(L, c=cache(**kw), read=read, k=heads(at(2), n), v=heads(at(3), n)) == status


@pytest.mark.parametrize("read", [False, True])
@pytest.mark.parametrize("name", BAD_ROWS)
def test_cache_rows_refused(L, name, read):
    status, kw = BAD_ROWS[name]
    assert rows(L, read=read, **kw) == status
    assert B.last_error()


def test_cache_rows_that_share(L):
    for kw in (dict(k=heads(at(3), 2)), dict(k=heads(at(6), 2)), dict(v=heads(at(5), 2)),
               dict(v=heads(at(4), 2))):
        assert rows(L, read=True, **kw) == -1
    for kw in (dict(pos=at(0)), dict(seq=at(1)), dict(table=at(0) + 256)):
        assert rows(L, **kw) == -1
    for read in (False, True):      # nothing to move
        assert rows(L, n=0, read=read, k=heads(None, 2), v=heads(None, 2), pos=None, table=None) == 0


def attend(L, c=None, dtype=1, n=3, q=None, table=at(4), ld=8, width=8, lens=at(5), scale=0.125,
           o=None, lse=at(6), ld_lse=3, scratch=at(10), nbytes=1 << 24):
    return L.mpipe_op_cache_attention(c or cache(), dtype, n, q or heads(at(2)), table, ld, width,
                                      lens, scale, o or heads(at(3)), lse, ld_lse, scratch, nbytes, None)


BAD_ATTEND = {
    "dtype": (-1, dict(dtype=2)),
    "types_differ": (-5, dict(dtype=0)),
    "cache_fp32": (-5, dict(c=cache(dtype=0))),
    "negative_sequences": (-1, dict(n=-1)),
    "negative_width": (-1, dict(width=-1)),
    "wide_table": (-5, dict(width=1 << 28, ld=1 << 28)),
    "scale": (-1, dict(scale=math.nan)),
    "heads": (-1, dict(q=heads(at(2), 3), o=heads(at(3), 3))),
    "o_heads": (-1, dict(o=heads(at(3), 4))),
    "no_heads": (-1, dict(q=heads(at(2), 0), o=heads(at(3), 0))),
    "null_table": (-1, dict(table=None)),
    "ld_table": (-1, dict(ld=7)),
    "null_lens": (-1, dict(lens=None)),
    "misaligned_lens": (-1, dict(lens=at(5) + 2)),
    "null_q": (-1, dict(q=heads(None))),
    "o_over_q": (-1, dict(o=heads(at(2)))),
    "lse_misaligned": (-1, dict(lse=at(6) + 1)),
    "ld_lse": (-1, dict(ld_lse=2)),
    "null_scratch": (-3, dict(scratch=None)),
    "small_scratch": (-3, dict(nbytes=1024)),
    "misaligned_scratch": (-1, dict(scratch=at(10) + 4)),
    "no_pages": (-1, dict(c=cache(pages=0))),
    "o_over_table": (-1, dict(o=heads(at(4)))),
    "o_over_lens": (-1, dict(o=heads(at(5)))),
    "o_over_cache": (-1, dict(o=heads(at(0)))),
    "lse_over_o": (-1, dict(lse=at(3))),
    "lse_over_lens": (-1, dict(lse=at(5))),
    "lse_over_cache": (-1, dict(lse=at(1))),
    "scratch_over_cache": (-1, dict(scratch=at(0))),
    "scratch_over_q": (-1, dict(scratch=at(2))),
    "scratch_over_lse": (-1, dict(scratch=at(6))),
    "scratch_over_table": (-1, dict(scratch=at(4))),
    "too_many": (-5, dict(n=1 << 21, ld_lse=1 << 21)),
}


@pytest.mark.parametrize("name", BAD_ATTEND)
def test_cache_attention_refused(L, name):
    status, kw = BAD_ATTEND[name]
    assert attend(L, **kw) == status
    assert B.last_error()


def test_no_sequences(L):
    assert attend(L, n=0, q=heads(None), o=heads(None), lens=None, table=None, scratch=None) == 0


# ---- the binding's own checks --------------------------------------------------------------

def test_binding_refuses(L):
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype)
    q, k = z(10, 4, 64), z(10, 2, 64)
    ok = dict(q=q, k=k, v=k.clone(), o=q.clone(), lse=None, seq_row=[0], seq_len=[10])
    bad = [dict(k=z(10, 2, 64, dtype=torch.float32)), dict(v=z(9, 2, 64)), dict(o=z(10, 4, 32)),
           dict(lse=z(4, 10)), dict(lse=z(4, 9, dtype=torch.float32)), dict(seq_len=[10, 1]),
           dict(seq_row=[0.5]), dict(q=z(10, 64)), dict(key_row=[0]),
           dict(q=z(10, 4, 128)[..., ::2]), dict(seq_row=[2 ** 70]), {}]   # last: not on the GPU
    for kw in bad:
        with pytest.raises(mp.MpipeError):
            mp.op_causal_attention_fwd(**dict(ok, **kw))
    f8 = torch.zeros(3, 2, 16, 64, dtype=torch.float8_e4m3fn)
    u8 = torch.zeros(3, 2, 16, dtype=torch.uint8)
    for args in ((f8, f8.clone()), (f8, f8.clone(), u8), (f8, f8.clone(), u8, u8[:2]),
                 (z(3, 2, 16, 64), z(3, 2, 16, 32)), (z(3, 2, 16, 64), z(3, 2, 16, 64), u8, u8.clone()),
                 (z(3, 2, 16, 64), z(3, 2, 64, 16).transpose(2, 3)), (z(3, 2, 16), z(3, 2, 16)),
                 (z(3, 2, 16, 64, dtype=torch.float16),) * 2):
        with pytest.raises(mp.MpipeError):
            mp.KvCache(*args)


# ---- the float64 forms ------------------------------------------------------------------------

def test_reference_attention_by_autograd():
    gen = torch.Generator().manual_seed(0)
    for lq, lk in ((7, 7), (5, 9), (6, 4), (3, 0)):
        q, k, v = (torch.randn(n, h, 8, generator=gen, dtype=torch.float64).requires_grad_()
                   for n, h in ((lq, 4), (lk, 2), (lk, 2)))
        g = torch.randn(lq, 4, 8, generator=gen, dtype=torch.float64)
        ref = R.attention(q.detach(), k.detach(), v.detach(), [(0, lq, 0, lk)], 0.3, g)
        lim = max(lk - lq, 0) - (lk - lq)        # first query that sees a key
        if lk:
            see = R.visible(lq, lk)[lim:]
            kk, vv = (x.repeat_interleave(2, 1) for x in (k, v))
            o = torch.nn.functional.scaled_dot_product_attention(
                q[lim:].transpose(0, 1), kk.transpose(0, 1), vv.transpose(0, 1), attn_mask=see,
                scale=0.3).transpose(0, 1)
            assert torch.allclose(ref["o"][0][lim:], o, atol=1e-12)
            s = torch.einsum("qhd,khd->hqk", q[lim:], kk) * 0.3
            s = s.masked_fill(~see, -math.inf)
            assert torch.allclose(ref["lse"][0][:, lim:], torch.logsumexp(s, 2), atol=1e-12)
            grads = torch.autograd.grad((o * g[lim:]).sum(), (q, k, v))
            for name, x in zip(("dq", "dk", "dv"), grads):
                assert torch.allclose(ref[name][0], x, atol=1e-12), name
        assert (ref["o"][0][:lim] == 0).all() and (ref["lse"][0][:, :lim] == -math.inf).all()


def test_reference_e4m3_by_torch():
    gen = torch.Generator().manual_seed(1)
    x = torch.randn(400, 64, generator=gen) * torch.exp(6 * torch.randn(400, 1, generator=gen))
    val, e = R.quantise(x)
    y = (x.double() * 2.0 ** -e.double()[:, None]).float()
    assert y.abs().max() <= 448 and (y.abs().amax(1) > 224).all()
    assert torch.equal(val, y.to(torch.float8_e4m3fn).double() * 2.0 ** e.double()[:, None])
    assert sorted(R.e4m3_values()) == R.e4m3_values() and len(R.e4m3_values()) == 127
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    assert torch.equal(codes, torch.tensor(R.e4m3_values(), dtype=torch.float64))
