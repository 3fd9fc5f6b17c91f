"""The first LLM layer's attention and its key-value cache on the GPU against float64 forms;
every bound counts the kernels' own roundings (attn_ref.py)."""
import math

import numpy as np
import pytest
import torch

from tests import attn_ref as R
import paper_2607_03229_amd as mp
from tests.gpu_util import announce

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float32
GUARD = 7.0     # what rows of no sequence hold, before and after


@pytest.fixture(autouse=True)
def float32_default():
    """Other test modules change torch's default type as they are imported."""
    old = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(old)


def normal(gen, *shape, dtype=BF):
    return torch.randn(shape, generator=gen).to(dtype)


def lay(x, layout, fill=GUARD):
    """x ([rows][heads][d], CPU) on the GPU in a layout of its own: the view, whole storage."""
    rows, heads, d = x.shape
    if layout == "plain":
        y = torch.full((rows, heads, d), fill, dtype=x.dtype, device="cuda")
    elif layout == "wide":          # columns of a wider product
        y = torch.full((rows, heads + 3, d), fill, dtype=x.dtype, device="cuda")[:, 2:2 + heads]
    elif layout == "heads_first":
        y = torch.full((heads, rows, d), fill, dtype=x.dtype, device="cuda").transpose(0, 1)
    elif layout == "odd":           # aligned to its elements only, odd strides
        y = torch.full((rows * (heads * (d + 1) + 1) + 1,), fill, dtype=x.dtype, device="cuda")
        y = y[1:].as_strided((rows, heads, d), (heads * (d + 1) + 1, d + 1, 1), 1)
    y.copy_(x)
    return y


def place(lens, gap=0, prefix=None, order=None):
    """Sequences one behind the other, `gap` rows between them: arrays and the reference's list."""
    prefix = prefix or [0] * len(lens)
    row, krow, seqs = gap, 0, []
    for n, p in zip(lens, prefix):
        m = max(n + p, 0)
        seqs.append((row, n, krow, m))
        row += n + gap
        krow += m
    seqs = [seqs[i] for i in (order or range(len(seqs)))]
    a = np.array(seqs, np.int64).reshape(-1, 4)
    return a, seqs, row, krow


def run(dtype, hq, hk, d, lens, prefix=None, gap=0, layout="plain", scale=None, seed=0, order=None,
        change=None, bwd=True, own_keys=True):
    """Forward and backward of one problem, checked; returns the outputs."""
    gen = torch.Generator().manual_seed(seed)
    a, seqs, rows, krows = place(lens, gap, prefix, order)
    if prefix is None:            # the keys are the queries' rows
        krows = rows
        a[:, 2:], seqs = a[:, :2], [(r, n, r, n) for r, n, _, _ in seqs]
    announce(f"attention {dtype} {hq}/{hk}x{d} lens {lens[:8]} prefix {prefix} gap {gap} {layout}")
    x = {"q": normal(gen, rows, hq, d, dtype=dtype), "k": normal(gen, krows, hk, d, dtype=dtype),
         "v": normal(gen, krows, hk, d, dtype=dtype), "d_o": normal(gen, rows, hq, d, dtype=dtype)}
    if change:
        change(x, seqs)
    scale = d ** -0.5 if scale is None else scale
    keys = dict(key_row=a[:, 2], key_len=a[:, 3]) if prefix is not None else {}
    g = {name: lay(t, layout) for name, t in x.items()}
    o = lay(torch.full_like(x["q"], GUARD), layout)
    lse = torch.full((hq, rows), GUARD, device="cuda")
    mp.op_causal_attention_fwd(g["q"], g["k"], g["v"], o, lse, a[:, 0], a[:, 1], scale=scale, **keys)
    ref = R.attention(x["q"], x["k"], x["v"], seqs, scale)
    R.check("o", o, ref["o"])
    R.check("lse", lse, ref["lse"])
    idle = torch.ones(rows, dtype=torch.bool)
    for r, n, _, _ in seqs:
        idle[r:r + n] = False
    assert (o.cpu()[idle] == GUARD).all() and (lse.cpu()[:, idle] == GUARD).all()
    out = {"o": o, "lse": lse}
    if not bwd:
        return out
    dq, dk, dv = (lay(torch.full_like(t, GUARD), layout) for t in (x["q"], x["k"], x["v"]))
    scratch = torch.empty(mp.op_causal_attention_scratch_bytes(rows, hq, krows, hk, d),
                          dtype=torch.uint8, device="cuda")
    mp.op_causal_attention_bwd(g["d_o"], g["q"], g["k"], g["v"], o, lse, a[:, 0], a[:, 1], dq, dk,
                               dv, scratch, scale=scale, **keys)
    ref = R.attention(x["q"], x["k"], x["v"], seqs, scale, x["d_o"], o.cpu())
    for name, t in (("dq", dq), ("dk", dk), ("dv", dv)):
        R.check(name, t, ref[name])
    kidle = torch.ones(krows, dtype=torch.bool)
    for _, _, r, n in seqs:
        kidle[r:r + n] = False
    assert (dq.cpu()[idle] == GUARD).all()
    assert (dk.cpu()[kidle] == GUARD).all() and (dv.cpu()[kidle] == GUARD).all()
    return dict(out, dq=dq, dk=dk, dv=dv)


# ---- causal attention ------------------------------------------------------------------------

LENS = [[1], [2, 1, 3], [15, 16, 17], [63, 64, 65], [127, 128, 129], [300], [257, 5, 700]]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("lens", LENS, ids=str)
def test_lengths(dtype, lens):
    run(dtype, 4, 2, 64, lens)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d", [8, 32, 40, 64, 72, 80, 96, 104, 128, 136, 200, 256])
def test_head_widths(dtype, d):
    run(dtype, 2, 1, d, [70, 131], gap=3)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("hq,hk", [(1, 1), (3, 3), (7, 1), (14, 2), (28, 4), (16, 8), (17, 1)])
def test_head_counts(dtype, hq, hk):
    run(dtype, hq, hk, 64, [90, 37])


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 80), (FP, 64)])
@pytest.mark.parametrize("layout", ["plain", "wide", "heads_first", "odd"])
def test_layouts(dtype, d, layout):
    run(dtype, 6, 2, d, [33, 0, 150], gap=5, layout=layout)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (FP, 64)])
@pytest.mark.parametrize("prefix", [[0, 5, 300], [64, 128, 1], [-1, -40, -500], [100, -20, 0]], ids=str)
def test_prefixes_and_queries_without_keys(dtype, d, prefix):
    run(dtype, 4, 2, d, [60, 77, 130], prefix=prefix, gap=2)


def test_keys_without_queries_and_queries_without_keys():
    for dtype in (BF, FP):
        out = run(dtype, 2, 2, 64, [0, 20, 0], prefix=[50, -20, 0])
        assert (out["dk"][:50] == 0).all() and (out["o"] == 0).all()
        assert (out["lse"] == -math.inf).all()


@pytest.mark.parametrize("dtype", [BF, FP])
def test_sequences_in_any_order(dtype):
    run(dtype, 4, 4, 64, [50, 200, 7, 90], order=[2, 0, 3, 1], gap=1)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (FP, 64)])
def test_long(dtype, d):
    run(dtype, 2, 1, d, [2500])


def test_many_sequences():
    """More than one launch's arguments hold."""
    run(BF, 2, 1, 64, [1 + i % 9 for i in range(500)], bwd=True)


@pytest.mark.parametrize("dtype,d", [(BF, 32), (BF, 64), (BF, 80), (BF, 128), (BF, 136), (FP, 64), (FP, 128)])
def test_few_key_heads(dtype, d):
    """Key tiles whose queries, of all heads of a group, go to several blocks: parts that begin and
    end inside a head, and keys that only a few of the last queries see."""
    run(dtype, 14, 2, d, [300, 5, 700])
    run(dtype, 16, 1, d, [129], prefix=[500])


@pytest.mark.parametrize("d", [48, 80, 104, 128])
def test_many_heads(d):
    """As many query tiles and key tiles as fill the chip by themselves."""
    run(BF, 28, 4, d, [700, 257, 300, 33], gap=2)
    run(BF, 16, 16, d, [100 + 11 * i for i in range(20)])


@pytest.mark.parametrize("dtype", [BF, FP])
def test_sharp_scores(dtype):
    """Weights near one hot, scores of thousands: maxima move by a lot from tile to tile."""
    def sharpen(x, seqs):
        x["q"] *= 8
        x["k"] *= 8
    # scores of up to 8 * 8 * 60 / 8: fp32 sums of them are off by 2^-24 of thousands
    run(dtype, 2, 1, 64, [300, 77], change=sharpen)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 72), (FP, 64)])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_values_behind_the_mask(dtype, d, value):
    """What a query does not see does not reach it, whatever it holds; keys likewise in the
    backward.  One sequence, a bad row in the middle of a tile."""
    n, at = 200, 100
    gen = torch.Generator().manual_seed(3)
    x = {s: normal(gen, n, h, d, dtype=dtype) for s, h in (("q", 4), ("k", 2), ("v", 2), ("d_o", 4))}
    clean = R.attention(x["q"], x["k"], x["v"], [(0, n, 0, n)], d ** -0.5)
    rows, lens = [0], [n]
    for spoilt in ("k", "v"):
        y = {s: t.clone() for s, t in x.items()}
        y[spoilt][at] = value
        g = {s: t.cuda() for s, t in y.items()}
        o, lse = torch.empty_like(g["q"]), torch.empty(4, n, device="cuda")
        announce(f"masked {spoilt} {value} {dtype} {d}")
        mp.op_causal_attention_fwd(g["q"], g["k"], g["v"], o, lse, rows, lens)
        R.check("o", o[:at], [t[:at] for t in clean["o"]])
        R.check("lse", lse[:, :at], [t[:, :at] for t in clean["lse"]])
        if spoilt == "v":
            R.check("lse", lse, clean["lse"])
            assert not torch.isfinite(o[at:].float()).any()
    # backward: clean forward, a bad row of what only some keys or queries see
    o = clean["o"][0].to(dtype)
    full = R.attention(x["q"], x["k"], x["v"], [(0, n, 0, n)], d ** -0.5, x["d_o"], o)
    lse = clean["lse"][0].float().cuda()
    scratch = torch.empty(mp.op_causal_attention_scratch_bytes(n, 4, n, 2, d), dtype=torch.uint8,
                          device="cuda")
    for spoilt in ("k", "v", "q", "d_o"):
        y = {s: t.clone() for s, t in x.items()}
        y[spoilt][at] = value
        g = {s: t.cuda() for s, t in y.items()}
        dq, dk, dv = (torch.empty_like(g[s]) for s in ("q", "k", "v"))
        announce(f"masked backward {spoilt} {value} {dtype} {d}")
        mp.op_causal_attention_bwd(g["d_o"], g["q"], g["k"], g["v"], o.cuda(), lse, rows, lens, dq,
                                   dk, dv, scratch)
        R.check("dq", dq[:at], [t[:at] for t in full["dq"]])
        if spoilt in ("q", "d_o"):       # row `at` counts for keys up to itself
            R.check("dk", dk[at + 1:], [t[at + 1:] for t in full["dk"]])
            R.check("dv", dv[at + 1:], [t[at + 1:] for t in full["dv"]])
            R.check("dq", dq[at + 1:], [t[at + 1:] for t in full["dq"]])


@pytest.mark.parametrize("dtype", [BF, FP])
def test_scores_of_minus_infinity(dtype):
    """Keys of weight 0: the whole first tiles of them, then ordinary ones; and a row that has
    nothing else, which is 0 / 0."""
    n, dead, d = 200, 150, 64
    gen = torch.Generator().manual_seed(4)
    q, k, v = (normal(gen, n, 2, d, dtype=dtype) for _ in range(3))
    q[..., 0] = 1.0
    k[:dead, :, 0] = -math.inf
    alive = k.clone()
    alive[..., 0] = k[-1, :, 0]
    o, lse = torch.empty(n, 2, d, dtype=dtype, device="cuda"), torch.empty(2, n, device="cuda")
    mp.op_causal_attention_fwd(q.cuda(), k.cuda(), v.cuda(), o, lse, [0], [n])
    ref = R.attention(q[dead:], torch.cat([k[dead:]]), v[dead:], [(0, n - dead, 0, n - dead)], d ** -0.5)
    R.check("o", o[dead:], ref["o"])
    R.check("lse", lse[:, dead:], ref["lse"])
    assert o[:dead].isnan().all() and (lse[:, :dead] == -math.inf).all()


@pytest.mark.parametrize("dtype", [BF, FP])
def test_gradients_by_differences(dtype):
    """The gradients against differences of a float64 loss along random directions: the loss is
    linear in d_o, so sum(dx * direction) is its slope."""
    gen = torch.Generator().manual_seed(6)
    n, hq, hk, d = 70, 4, 2, 64
    out = run(dtype, hq, hk, d, [n], seed=6)
    x = {s: normal(gen, n, h, d, dtype=dtype).double() for s, h in
         (("q", hq), ("k", hk), ("v", hk), ("d_o", hq))}
    loss = lambda q, k, v: (R.attention(q, k, v, [(0, n, 0, n)], d ** -0.5)["o"][0] * x["d_o"]).sum()
    gen2 = torch.Generator().manual_seed(7)
    bounds = R.attention(*(x[s].to(dtype) for s in ("q", "k", "v")), [(0, n, 0, n)], d ** -0.5,
                         x["d_o"].to(dtype), out["o"].cpu())
    for name in ("q", "k", "v"):
        u = torch.randn(x[name].shape, generator=gen2, dtype=torch.float64)
        h = 1e-5
        args = [dict(x, **{name: x[name] + s * h * u}) for s in (1, -1)]
        slope = (loss(*(args[0][s] for s in "qkv")) - loss(*(args[1][s] for s in "qkv"))) / (2 * h)
        got = (out["d" + name].double().cpu() * u).sum()
        bound = (bounds["d" + name][1] * u.abs()).sum() + 1e-6 * abs(slope) + 1e-6
        assert abs(got - slope) <= bound, (name, got, slope, bound)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_shared_keys_in_the_forward(dtype):
    """Two sequences of queries over one prefix."""
    gen = torch.Generator().manual_seed(8)
    q, k, v = normal(gen, 60, 4, 64, dtype=dtype), *(normal(gen, 100, 2, 64, dtype=dtype) for _ in range(2))
    o = torch.empty(60, 4, 64, dtype=dtype, device="cuda")
    seqs = [(0, 25, 0, 100), (25, 35, 0, 90)]
    a = np.array(seqs)
    mp.op_causal_attention_fwd(q.cuda(), k.cuda(), v.cuda(), o, None, a[:, 0], a[:, 1], a[:, 2], a[:, 3])
    R.check("o", o, R.attention(q, k, v, seqs, 0.125)["o"])


@pytest.mark.parametrize("dtype,d", [(BF, 128), (FP, 64)])
def test_the_same_bits(dtype, d):
    """A call again, forward and backward."""
    first = run(dtype, 6, 2, d, [130, 300, 65])
    again = run(dtype, 6, 2, d, [130, 300, 65])
    for name in first:
        assert torch.equal(first[name], again[name]), name


@pytest.mark.parametrize("dtype", [BF, FP])
def test_broadcast_inputs(dtype):
    """One row as every row's gradient, one head as every key head: as if they were written out."""
    rows, hq, hk, d = 333, 6, 3, 64
    gen = torch.Generator().manual_seed(3)
    q = normal(gen, rows, hq, d, dtype=dtype).cuda()
    k, v = (normal(gen, rows, 1, d, dtype=dtype).cuda().expand(rows, hk, d) for _ in range(2))
    d_o = normal(gen, 1, 1, d, dtype=dtype).cuda().expand(rows, hq, d)
    announce(f"broadcast {dtype}")

    def both(k, v, d_o):
        o, dq = torch.empty_like(q), torch.empty_like(q)
        dk, dv = (torch.empty(rows, hk, d, dtype=dtype, device="cuda") for _ in range(2))
        lse = torch.empty(hq, rows, device="cuda")
        scratch = torch.empty(mp.op_causal_attention_scratch_bytes(rows, hq, rows, hk, d),
                              dtype=torch.uint8, device="cuda")
        mp.op_causal_attention_fwd(q, k, v, o, lse, [0, 200], [190, 133])
        mp.op_causal_attention_bwd(d_o, q, k, v, o, lse, [0, 200], [190, 133], dq, dk, dv, scratch)
        return [t[r] for t in (o, dq, dk, dv) for r in (slice(0, 190), slice(200, 333))]
    for a, b in zip(both(k, v, d_o), both(k.contiguous(), v.contiguous(), d_o.contiguous())):
        assert torch.equal(a, b)


def test_offsets_past_32_bits():
    """Rows so far apart that elements lie behind 2^32 bytes and 2^31 elements."""
    rows, d = 1200, 64
    stride = (2 ** 31 // rows // 8 + 64) * 8
    gen = torch.Generator().manual_seed(9)
    x = [normal(gen, 40, 1, d) for _ in range(3)]
    big = torch.empty(rows * stride, dtype=BF, device="cuda")
    views = [big.as_strided((rows, 1, d), (stride, d, 1), 64 * i) for i in range(6)]
    for v, t in zip(views, x):
        v[-40:] = t.cuda()
    q, k, v, o, d_o, dq = views
    lse = torch.empty(1, rows, device="cuda")
    mp.op_causal_attention_fwd(q, k, v, o, lse, [rows - 40], [40])
    ref = R.attention(*x, [(0, 40, 0, 40)], 0.125)
    R.check("o", o[-40:], ref["o"])
    R.check("lse", lse[:, -40:], ref["lse"])
    d_o[-40:] = x[0].cuda()
    dk, dv = torch.empty(rows, 1, d, dtype=BF, device="cuda"), torch.empty(rows, 1, d, dtype=BF, device="cuda")
    scratch = torch.empty(mp.op_causal_attention_scratch_bytes(rows, 1, rows, 1, d),
                          dtype=torch.uint8, device="cuda")
    mp.op_causal_attention_bwd(d_o, q, k, v, o, lse, [rows - 40], [40], dq, dk, dv, scratch)
    ref = R.attention(*x, [(0, 40, 0, 40)], 0.125, x[0], o[-40:].cpu())
    for name, t in (("dq", dq), ("dk", dk), ("dv", dv)):
        R.check(name, t[-40:], ref[name])


# ---- the cache -------------------------------------------------------------------------------

def make_cache(n_pages, heads, page, d, dtype):
    if dtype == "e4m3":
        t = [torch.full((n_pages, heads, page, d), math.nan, device="cuda").to(torch.float8_e4m3fn)
             for _ in range(2)]
        s = [torch.full((n_pages, heads, page), 127, dtype=torch.uint8, device="cuda") for _ in range(2)]
        return mp.KvCache(*t, *s)
    return mp.KvCache(*(torch.full((n_pages, heads, page, d), math.nan, dtype=dtype, device="cuda")
                        for _ in range(2)))


def make_table(lens, page, extra=3, seed=0):
    need = [-(-n // page) for n in lens]
    gen = torch.Generator().manual_seed(seed)
    order = torch.randperm(sum(need) + extra, generator=gen).to(torch.int32)
    table = torch.full((len(lens), max(need + [1]) + 1), -1, dtype=torch.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    return table.cuda(), sum(need) + extra


def all_rows(lens, lo=None):
    lo = lo or [0] * len(lens)
    pos = torch.cat([torch.arange(a, n, dtype=torch.int32) for a, n in zip(lo, lens)])
    seq = torch.cat([torch.full((n - a,), i, dtype=torch.int32) for i, (a, n) in enumerate(zip(lo, lens))])
    return pos.cuda(), seq.cuda()


def stored(x, cache_dtype, out_dtype):
    if cache_dtype == "e4m3":
        return R.quantise(x)[0].to(out_dtype)
    return x.to(cache_dtype).to(out_dtype)


@pytest.mark.parametrize("page", [1, 4, 16, 64, 256])
@pytest.mark.parametrize("cache_dtype", [BF, FP, "e4m3"])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_write_and_read(dtype, cache_dtype, page):
    lens, heads = [1, 70, 0, 16, 33], 3
    for d in (8, 64, 72, 128, 256):
        table, pages = make_table(lens, page)
        cache = make_cache(pages, heads, page, d, cache_dtype)
        pos, seq = all_rows(lens)
        gen = torch.Generator().manual_seed(d)
        x = [torch.randn(len(pos), heads, d, generator=gen) *
             torch.exp(4 * torch.randn(len(pos), heads, 1, generator=gen)) for _ in range(2)]
        x = [t.to(dtype) for t in x]
        order = torch.randperm(len(pos), generator=gen).cuda()   # rows in any order
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        announce(f"cache {dtype} -> {cache_dtype} page {page} d {d}")
        mp.op_cache_write(cache, *(lay(t[order.cpu()], "wide") for t in x), table, pos[order],
                          seq=seq[order], status=status)
        for out_dtype in (BF, FP):
            k, v = (lay(torch.full_like(x[0], GUARD).to(out_dtype), "odd" if page == 4 else "plain")
                    for _ in range(2))
            mp.op_cache_read(cache, table, pos, k, v, seq=seq, status=status)
            for got, t in ((k, x[0]), (v, x[1])):
                assert torch.equal(got.cpu(), stored(t, cache_dtype, out_dtype))
        assert status.item() == 0
        # nothing else was touched
        used = torch.zeros(pages, page, dtype=torch.bool)
        for s, n in enumerate(lens):
            for i in range(n):
                used[int(table[s, i // page]), i % page] = True
        for t in (cache.k, cache.v):
            t = t.float().cpu()
            assert t.permute(0, 2, 1, 3)[~used].isnan().all()


def test_e4m3_roundings():
    """Every e4m3 value, every midpoint of two and its neighbours, at exponents of all sizes;
    zeros, infinities and NaN."""
    table = torch.tensor(R.e4m3_values())
    mid = (table[1:] + table[:-1]) / 2
    v = torch.cat([table, mid, mid * (1 + 2 ** -20), mid * (1 - 2 ** -20), torch.tensor([448.0])])
    v = torch.cat([v, -v])
    d = 256
    v = torch.cat([v, torch.zeros(-len(v) % (d - 1))]).view(-1, d - 1)
    rows = []
    for e in (-126, -125, -100, -20, -1, 0, 1, 60, 119):
        for top in (448.0, 449.0, 255.0):      # the head's largest, so its power of two is known
            t = torch.full((len(v), 1), top)
            rows.append(torch.cat([v.clamp(-top, top), t], 1) * 2.0 ** e)
    x = torch.cat(rows)
    x = torch.cat([x, torch.zeros(1, d), torch.full((1, d), math.nan), torch.full((1, d), math.inf)])
    odd = x[5].clone()
    odd[3], odd[4], odd[5] = math.inf, -math.inf, math.nan
    x = torch.cat([x, odd[None], torch.full((1, d), 2.0 ** -149), torch.full((1, d), 3.4e38)])[:, None]
    n = len(x)
    cache = make_cache(n, 1, 1, d, "e4m3")
    table_ = torch.arange(n, dtype=torch.int32, device="cuda")[None]
    pos, seq = all_rows([n])
    mp.op_cache_write(cache, x.cuda(), x.cuda(), table_, pos, seq=seq)
    k, v = torch.empty_like(x, device="cuda"), torch.empty_like(x, device="cuda")
    mp.op_cache_read(cache, table_, pos, k, v, seq=seq)
    val, e = R.quantise(x)
    val = val.float().double()     # as read: 3.4e38 = 255.8 * 2^120 is kept as 256 * 2^120 = 2^128
    assert torch.equal(cache.k_scale.view(-1).cpu().long(), e.view(-1) + 127)
    for got in (k, v):
        got = got.cpu().double()
        assert torch.equal(got.isnan(), val.isnan())
        assert torch.equal(got[~val.isnan()], val[~val.isnan()])


def test_rows_left_out_and_bad_places():
    page, d, heads = 8, 64, 2
    table = torch.tensor([[0, 5], [2, -1], [9, 1]], dtype=torch.int32, device="cuda")   # 5, 9: no such page
    cache = make_cache(4, heads, page, d, BF)
    pos = torch.tensor([0, -1, 3, 9, 8, 7, 16, 9, -5, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    seq = torch.tensor([0, 0, -1, 1, 0, 2, 0, 2, 7, 0], dtype=torch.int32, device="cuda")
    good = [0, 7]           # (0, 0) on page 0 and (2, 9) on page 1
    out = [1, 2, 8]         # padding
    x = torch.randn(10, heads, d, device="cuda").to(BF)
    for s, rows_, expect in ((pos[[0, 1, 2, 7]], [0, 1, 2, 7], 0), (pos, range(10), 1)):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        r = list(rows_)
        announce(f"bad places {expect}")
        mp.op_cache_write(cache, x[r], x[r], table, pos[r], seq=seq[r], status=status)
        assert status.item() == expect
        k, v = (torch.full((len(r), heads, d), GUARD, dtype=BF, device="cuda") for _ in range(2))
        status.zero_()
        mp.op_cache_read(cache, table, pos[r], k, v, seq=seq[r], status=status)
        assert status.item() == expect
        for i, row in enumerate(r):
            for t in (k, v):
                if row in good:
                    assert torch.equal(t[i], x[row])
                elif row in out:
                    assert (t[i] == GUARD).all()
                else:
                    assert t[i].isnan().all()
    held = torch.zeros(4, page, dtype=torch.bool)
    held[0, 0] = held[1, 1] = True
    assert cache.k.float().cpu().permute(0, 2, 1, 3)[~held].isnan().all()


# ---- attention over the cache ------------------------------------------------------------------

def decode(dtype, cache_dtype, hq, hk, d, page, lens, seed=0, lse=True, layout="plain"):
    gen = torch.Generator().manual_seed(seed)
    table, pages = make_table(lens, page, seed=seed)
    cache = make_cache(pages, hk, page, d, cache_dtype)
    pos, seq = all_rows([max(n, 0) for n in lens])
    x = [normal(gen, len(pos), hk, d, dtype=dtype) for _ in range(2)]
    if len(pos):
        mp.op_cache_write(cache, x[0].cuda(), x[1].cuda(), table, pos, seq=seq)
    q = normal(gen, len(lens), hq, d, dtype=dtype)
    o = lay(torch.full_like(q, GUARD), layout)
    stats = torch.full((hq, len(lens)), GUARD, device="cuda") if lse else None
    scratch = torch.empty(mp.op_cache_attention_scratch_bytes(len(lens), hq, hk, d),
                          dtype=torch.uint8, device="cuda")
    announce(f"decode {dtype} {cache_dtype} {hq}/{hk}x{d} page {page} lens {lens[:8]} of {len(lens)}")
    mp.op_cache_attention(cache, lay(q, layout), table,
                          torch.tensor(lens, dtype=torch.int32, device="cuda"), o, scratch, lse=stats)
    k, v = (stored(t, cache_dtype, FP).double() for t in x)
    seqs, at = [], 0
    for i, n in enumerate(lens):
        seqs.append((i, 1, at, max(n, 0)))
        at += max(n, 0)
    ref = R.attention(q, k, v, seqs, d ** -0.5)
    R.check("o", o, ref["o"])
    if lse:
        R.check("lse", stats, ref["lse"])
    return o, stats


CACHES = [(BF, BF), (BF, "e4m3"), (FP, FP), (FP, "e4m3")]


@pytest.mark.parametrize("dtype,cache_dtype", CACHES, ids=str)
@pytest.mark.parametrize("page", [1, 8, 16, 32, 64, 256])
def test_decode_pages(dtype, cache_dtype, page):
    decode(dtype, cache_dtype, 8, 2, 64, page, [1, 15, 16, 17, 31, 33, 127, 128, 129, 500])


@pytest.mark.parametrize("dtype,cache_dtype", CACHES, ids=str)
@pytest.mark.parametrize("d", [8, 40, 64, 80, 96, 128, 136, 256])
def test_decode_widths(dtype, cache_dtype, d):
    decode(dtype, cache_dtype, 4, 2, d, 16, [70, 300])


@pytest.mark.parametrize("dtype,cache_dtype", CACHES, ids=str)
@pytest.mark.parametrize("hq,hk", [(1, 1), (7, 7), (28, 4), (16, 1), (17, 1), (64, 2), (40, 1)])
def test_decode_heads(dtype, cache_dtype, hq, hk):
    decode(dtype, cache_dtype, hq, hk, 64, 16, [200, 3, 41])


@pytest.mark.parametrize("dtype,cache_dtype", CACHES, ids=str)
def test_decode_lengths(dtype, cache_dtype):
    decode(dtype, cache_dtype, 4, 2, 128, 32, [0, 1, 0, 5000, -3, 130, 0])
    decode(dtype, cache_dtype, 2, 1, 64, 32, [0])
    decode(dtype, cache_dtype, 2, 1, 64, 32, [20000], lse=False)


def test_decode_many_sequences():
    decode(BF, BF, 2, 1, 64, 16, [(i * 37) % 90 for i in range(700)])


@pytest.mark.parametrize("dtype,cache_dtype,hq,hk", [(BF, BF, 6, 3), (FP, "e4m3", 34, 2)])
def test_decode_more_heads_than_blocks(dtype, cache_dtype, hq, hk):
    """Most key heads lie in one block, some in two, those of one sequence in many."""
    lens = [(i * 61) % 400 for i in range(360)]
    lens[100] = 30000
    decode(dtype, cache_dtype, hq, hk, 64, 16, lens)


@pytest.mark.parametrize("layout", ["wide", "heads_first", "odd"])
def test_decode_layouts(layout):
    for dtype in (BF, FP):
        decode(dtype, dtype, 6, 2, 72, 16, [100, 20, 1], layout=layout)


def test_decode_bad_pages_and_lengths():
    """A page outside the pool or a length beyond the table makes its sequence NaN, no other."""
    for dtype, cache_dtype in CACHES:
        page, d = 16, 64
        cache = make_cache(6, 2, page, d, cache_dtype)
        table = torch.tensor([[0, 1, 2], [3, 77, 4], [4, -1, 5], [5, 1, 2], [0, -9, 2 ** 30]],
                             dtype=torch.int32, device="cuda")
        lens = torch.tensor([48, 33, 16, 49, 1000], dtype=torch.int32, device="cuda")
        pos = torch.arange(16, dtype=torch.int32, device="cuda").repeat(6)
        seq = torch.arange(6, dtype=torch.int32, device="cuda").repeat_interleave(16)
        x = [torch.randn(96, 2, d, device="cuda").to(dtype) for _ in range(2)]
        mp.op_cache_write(cache, *x, torch.arange(6, dtype=torch.int32, device="cuda")[:, None], pos, seq=seq)
        q = torch.randn(5, 4, d, device="cuda").to(dtype)
        o, lse = torch.empty_like(q), torch.empty(4, 5, device="cuda")
        scratch = torch.empty(mp.op_cache_attention_scratch_bytes(5, 4, 2, d), dtype=torch.uint8, device="cuda")
        announce(f"decode bad pages {dtype} {cache_dtype}")
        mp.op_cache_attention(cache, q, table, lens, o, scratch, lse=lse)
        k, v = (stored(t.cpu(), cache_dtype, FP).double() for t in x)
        ref = R.attention(q.cpu(), k, v, [(0, 1, 0, 48), (2, 1, 64, 16)], d ** -0.5)
        R.check("o", o, ref["o"])
        R.check("lse", lse, ref["lse"])
        for s in (1, 3, 4):
            assert o[s].isnan().all() and lse[:, s].isnan().all()


def test_decode_past_32_bits():
    """A pool of more than 2^31 values and 2^32 bytes; the pages in use are its last ones."""
    page, d, heads = 64, 128, 8
    pages = 2 ** 31 // (page * d * heads) + 40
    cache = mp.KvCache(*(torch.empty(pages, heads, page, d, dtype=BF, device="cuda") for _ in range(2)))
    n = 300
    table = torch.arange(pages - 5, pages, dtype=torch.int32, device="cuda").flip(0)[None]
    pos, seq = all_rows([n])
    gen = torch.Generator().manual_seed(1)
    x = [normal(gen, n, heads, d) for _ in range(2)]
    mp.op_cache_write(cache, x[0].cuda(), x[1].cuda(), table, pos, seq=seq)
    k, v = torch.empty_like(x[0], device="cuda"), torch.empty_like(x[0], device="cuda")
    mp.op_cache_read(cache, table, pos, k, v, seq=seq)
    assert torch.equal(k.cpu(), x[0]) and torch.equal(v.cpu(), x[1])
    q = normal(gen, 1, 16, d)
    o = torch.empty_like(q, device="cuda")
    scratch = torch.empty(mp.op_cache_attention_scratch_bytes(1, 16, heads, d), dtype=torch.uint8, device="cuda")
    mp.op_cache_attention(cache, q.cuda(), table, torch.tensor([n], dtype=torch.int32, device="cuda"), o, scratch)
    R.check("o", o, R.attention(q, *x, [(0, 1, 0, n)], d ** -0.5)["o"])


# ---- streams, graphs, and all of it together ----------------------------------------------------

def test_prompt_then_tokens():
    """A layer as it is used: heads normed and turned, the prompt's attention, its keys into the
    cache, then token by token over the cache; and the prompt's second half as a chunk over what
    the cache gives back.  Each token's output is the row of one causal pass over everything."""
    gen = torch.Generator().manual_seed(11)
    hq, hk, d, page = 8, 2, 128, 16
    total, prompt = [61, 130], [50, 120]
    rows = sum(total)
    start = [0, total[0]]
    x = normal(gen, rows, hq + 2 * hk, d).cuda()
    gains = [(1 + 0.1 * normal(gen, d).float()).to(BF).cuda() for _ in range(2)]
    pos = torch.cat([torch.arange(n, dtype=torch.int32) for n in total]).cuda()
    rope = mp.RopeCfg(d, [16, 24, 24], theta=1e6)
    q, k = (torch.empty(rows, h, d, dtype=BF, device="cuda") for h in (hq, hk))
    mp.op_qk_norm_rope_fwd(rope, x[:, :hq], x[:, hq:hq + hk], *gains, 1e-6,
                           pos.expand(3, rows), q, k)
    v = x[:, hq + hk:]
    whole = torch.empty_like(q)
    mp.op_causal_attention_fwd(q, k, v, whole, None, start, total)
    ref = R.attention(q.cpu(), k.cpu(), v.cpu(), [(s, n, s, n) for s, n in zip(start, total)], d ** -0.5)
    R.check("whole", whole, ref["o"])
    table, pages = make_table(total, page)
    cache = make_cache(pages, hk, page, d, BF)
    first = torch.cat([torch.arange(s, s + n) for s, n in zip(start, prompt)]).cuda()
    p_pos, p_seq = all_rows(prompt)
    mp.op_cache_write(cache, k[first], v[first], table, p_pos, seq=p_seq)
    scratch = torch.empty(mp.op_cache_attention_scratch_bytes(2, hq, hk, d), dtype=torch.uint8, device="cuda")
    for step in range(10):
        at = torch.tensor([s + n + step for s, n in zip(start, prompt)]).cuda()
        t_pos = torch.tensor([n + step for n in prompt], dtype=torch.int32, device="cuda")
        mp.op_cache_write(cache, k[at], v[at], table, t_pos)
        o = torch.empty(2, hq, d, dtype=BF, device="cuda")
        mp.op_cache_attention(cache, q[at], table, t_pos + 1, o, scratch)
        R.check("token", o, [t[at.cpu()] for t in ref["o"]])
    # the second sequence's last 40 rows as a chunk over the cache
    c_pos, c_seq = all_rows([0, total[1]])
    ck, cv = (torch.empty(total[1], hk, d, dtype=BF, device="cuda") for _ in range(2))
    mp.op_cache_read(cache, table, c_pos, ck, cv, seq=c_seq)
    assert torch.equal(ck, k[start[1]:]) and torch.equal(cv, v[start[1]:])
    o = torch.empty(40, hq, d, dtype=BF, device="cuda")
    mp.op_causal_attention_fwd(q[-40:], ck, cv, o, None, [0], [40], [0], [total[1]])
    R.check("chunk", o, [t[-40:] for t in ref["o"]])


@pytest.mark.parametrize("dtype,d", [(BF, 128), (FP, 64)])
def test_captured(dtype, d):
    """A step of training and one of serving in a graph each, which share a workspace; replayed
    with new inputs, lengths and pages, eager work of the same tensors between the replays."""
    hq, hk, n, page = 4, 2, 150, 16
    gen = torch.Generator().manual_seed(12)
    q, k, v, d_o = (normal(gen, n, h, d, dtype=dtype).cuda() for h in (hq, hk, hk, hq))
    outs = [torch.empty_like(t) for t in (q, q, k, v)]
    lse = torch.empty(hq, n, device="cuda")
    work = torch.empty(max(mp.op_causal_attention_scratch_bytes(n, hq, n, hk, d),
                           mp.op_cache_attention_scratch_bytes(2, hq, hk, d)), dtype=torch.uint8, device="cuda")
    row, ln = np.array([0, 100]), np.array([100, 50])

    def train():
        mp.op_causal_attention_fwd(q, k, v, outs[0], lse, row, ln)
        mp.op_causal_attention_bwd(d_o, q, k, v, outs[0], lse, row, ln, *outs[1:], work)

    cache = make_cache(40, hk, page, d, dtype)
    for t in (cache.k, cache.v):
        t.zero_()      # lengths grow over tokens that are never written
    table = torch.arange(40, dtype=torch.int32, device="cuda").view(2, 20)
    lens = torch.tensor([100, 50], dtype=torch.int32, device="cuda")
    tok = [torch.empty(2, h, d, dtype=dtype, device="cuda") for h in (hq, hk, hk, hq)]
    c_pos, c_seq = all_rows([100, 50])

    def serve():
        mp.op_cache_write(cache, tok[1], tok[2], table, lens - 1)
        mp.op_cache_attention(cache, tok[0], table, lens, tok[3], work)

    for t in tok:
        t.copy_(torch.randn(t.shape, generator=gen))
    mp.op_cache_write(cache, k, v, table, c_pos, seq=c_seq)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        train()
        serve()
    torch.cuda.synchronize()
    graphs = []
    for step in (train, serve):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        graphs.append(g)
    for turn in range(4):
        for t in (q, k, v, d_o, *tok[:3]):
            t.copy_(torch.randn(t.shape, generator=gen))
        lens += 7
        table.copy_(torch.randperm(40, generator=gen).to(torch.int32).view(2, 20))
        mp.op_cache_write(cache, k, v, table, c_pos, seq=c_seq)
        got = []
        for step, g in zip((train, serve), graphs):
            g.replay()
            torch.cuda.synchronize()
            a = [t.clone() for t in (*outs, lse, tok[3])]
            for t in (*outs, lse):
                t.zero_()
            step()
            torch.cuda.synchronize()
            b = [t.clone() for t in (*outs, lse, tok[3])]
            got.append((a, b))
        for x, y in zip(got[0][0][:5], got[0][1][:5]):
            assert torch.equal(x, y), turn
        assert torch.equal(got[1][0][5], got[1][1][5]) and got[1][0][5].isfinite().all(), turn


def test_on_another_stream():
    gen = torch.Generator().manual_seed(13)
    q, k, v = (normal(gen, 90, h, 64).cuda() for h in (4, 2, 2))
    o = torch.empty_like(q)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    mp.op_causal_attention_fwd(q, k, v, o, None, [0], [90], stream=s)
    s.synchronize()
    R.check("o", o, R.attention(q.cpu(), k.cpu(), v.cpu(), [(0, 90, 0, 90)], 0.125)["o"])
