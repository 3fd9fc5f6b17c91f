"""The first LLM layer's attention on the GPU at the largest sizes its calls take."""
import math

import pytest
import torch

import paper_2607_03229_amd as mp
from tests import attn_ref as R
from tests.gpu_util import announce

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(autouse=True)
def float32_default():
    """Other test modules change torch's default type as they are imported."""
    old = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(old)


@pytest.mark.parametrize("page", [16, 64])
def test_cache_of_as_many_tokens_as_a_length_counts(page):
    """Tables of up to 2^31 - page tokens, all in the pages of one sequence of four.  Queries of 0
    weigh all tokens alike, so the output is the mean of the values: the weights' sums are whole
    numbers, exact in fp32 up to 2^24, beyond which a wave's sum and the joins of at most 4096
    waves round by 2^-24 each; one rounding to bf16."""
    d, width = 64, 2 ** 31 // page - 1
    gen = torch.Generator().manual_seed(page)
    k, v = (torch.randint(-8, 9, (2, 1, page, d), generator=gen).to(BF) / 8 for _ in range(2))
    cache = mp.KvCache(k.cuda(), v.cuda())
    most = width * page
    lens = [most, 5, 2 ** 31 - 1, most - 7]       # the third is longer than its table
    table = torch.zeros(len(lens), width, dtype=torch.int32, device="cuda")
    table[1:, 0] = 1
    q = torch.zeros(len(lens), 1, d, dtype=BF, device="cuda")
    o = torch.full_like(q, 7.0)
    lse = torch.full((1, len(lens)), 7.0, device="cuda")
    scratch = torch.empty(mp.op_cache_attention_scratch_bytes(len(lens), 1, 1, d), dtype=torch.uint8,
                          device="cuda")
    announce(f"cache of {most} tokens, page {page}")
    mp.op_cache_attention(cache, q, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), o,
                          scratch, lse=lse)
    o, lse = o.double().cpu(), lse.double().cpu()
    assert o[2].isnan().all() and lse[0, 2].isnan()
    for s in (0, 1, 3):
        n = lens[s]
        count = torch.zeros(2, page, dtype=torch.float64)     # tokens in every place of the pages
        count[0] = n // page
        count[0, :n % page] += 1
        if s:                                                 # its first page is page 1
            first = min(n, page)
            count[1, :first] = 1
            count[0, :first] -= 1
        x = v.double()[:, 0]
        mean, size = ((count[..., None] * y).sum((0, 1)) / n for y in (x, x.abs()))
        assert ((o[s, 0] - mean).abs() <= 2.0 ** -8 * mean.abs() + 4096 * 2.0 ** -24 * size).all(), s
        assert abs(lse[0, s] - math.log(n)) <= 4096 * 2.0 ** -24 + 2.0 ** -22 * math.log(n), s


def test_more_threads_than_a_grid_holds():
    """65536 heads of 128 one-row sequences: blocks of 512 threads, 2^32 of them in one launch if it
    took all items.  All heads are alike, so one is the reference: a row's output is its only value,
    exactly, and the key head's gradients are 65536 times one head's, in sums of as many terms."""
    n, hq, d = 128, 65536, 128
    gen = torch.Generator().manual_seed(3)
    x = [torch.randn(n, 1, d, generator=gen).to(BF) for _ in range(4)]
    q, k, v, d_o = (t.cuda() for t in x)
    wide = lambda t: t.expand(n, hq, d)
    o = torch.full((n, hq, d), 7.0, dtype=BF, device="cuda")
    lse = torch.full((hq, n), 7.0, device="cuda")
    rows, lens = list(range(n)), [1] * n
    announce("65536 heads of 128 sequences")
    mp.op_causal_attention_fwd(wide(q), k, v, o, lse, rows, lens)
    ref = R.attention(*x[:3], [(i, 1, i, 1) for i in range(n)], d ** -0.5, x[3], x[2])
    assert torch.equal(o, wide(v))
    for h in (0, 1, hq // 2, hq - 1):
        R.check("lse", lse[h:h + 1], ref["lse"])
    assert torch.equal(lse, lse[:1].expand(hq, n))
    dq = torch.full_like(o, 7.0)
    dk, dv = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    scratch = torch.empty(mp.op_causal_attention_scratch_bytes(n, hq, n, 1, d), dtype=torch.uint8,
                          device="cuda")
    mp.op_causal_attention_bwd(wide(d_o), wide(q), k, v, o, lse, rows, lens, dq, dk, dv, scratch)
    for h in (0, 1, hq // 2, hq - 1):
        R.check("dq", dq[:, h:h + 1], ref["dq"])
    assert torch.equal(dq, dq[:, :1].expand(n, hq, d))
    many = hq * 2.0 ** -24
    for name, t in (("dk", dk), ("dv", dv)):
        value, bound = ref[name]
        R.check(name, t, (hq * value, hq * (bound + many * (value.abs() + bound))))


@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_more_sequences_than_any_batch(dtype):
    """200,000 sequences of one token or none: an output is its sequence's only value, or 0."""
    n, d = 200000, 64
    gen = torch.Generator().manual_seed(1)
    v = torch.randn(n, 1, 1, d, generator=gen).to(dtype).cuda()
    cache = mp.KvCache(torch.randn(n, 1, 1, d, generator=gen).to(dtype).cuda(), v)
    page = torch.randperm(n, generator=gen).to(torch.int32).cuda()
    lens = torch.randint(0, 2, (n,), generator=gen, dtype=torch.int32).cuda()
    q = torch.randn(n, 2, d, generator=gen).to(dtype).cuda()
    o, lse = torch.full_like(q, 7.0), torch.full((2, n), 7.0, device="cuda")
    scratch = torch.empty(mp.op_cache_attention_scratch_bytes(n, 2, 1, d), dtype=torch.uint8, device="cuda")
    announce(f"200,000 sequences {dtype}")
    mp.op_cache_attention(cache, q, page[:, None], lens, o, scratch, lse=lse)
    there = lens > 0
    want = torch.where(there[:, None], v[page.long(), 0, 0], torch.zeros(1, dtype=dtype, device="cuda"))
    assert torch.equal(o, want[:, None].expand(n, 2, d))
    assert (lse[:, ~there] == -math.inf).all() and lse[:, there].isfinite().all()


def test_time_grows_with_the_sequences_not_their_square():
    """Four times as many short sequences take about four times as long.  (Where each block of the join
    added up all lengths, 16384 took 13.6 times as long as 4096: 12.2 ms for 0.9.)"""
    heads, d, page = 8, 128, 16
    best = []
    for n in (4096, 16384):
        lens = torch.randint(10, 101, (n,), generator=torch.Generator().manual_seed(2), dtype=torch.int32)
        table = torch.arange(7 * n, dtype=torch.int32, device="cuda").view(n, 7)
        cache = mp.KvCache(*(torch.zeros(7 * n, heads, page, d, dtype=BF, device="cuda") for _ in range(2)))
        q = torch.randn(n, heads, d, device="cuda").to(BF)
        o, lens = torch.empty_like(q), lens.cuda()
        scratch = torch.empty(mp.op_cache_attention_scratch_bytes(n, heads, heads, d), dtype=torch.uint8,
                              device="cuda")
        times = []
        for _ in range(8):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            mp.op_cache_attention(cache, q, table, lens, o, scratch)
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        best.append(min(times))
        del cache
    assert best[1] <= 8 * best[0], best
