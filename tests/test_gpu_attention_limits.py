"""The first LLM layer's attention on the GPU at the largest sizes its calls take."""
import math

import pytest
import torch

import paper_2607_03229_amd as mp
from tests.gpu_util import announce

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float32


@pytest.mark.parametrize("page", [16, 64])
def test_cache_of_as_many_tokens_as_a_length_counts(page):
    """Tables of up to 2^31 - page tokens, all in the pages of one sequence of four.  Queries of 0
    weigh all tokens alike, so the output is the mean of the values: the weights' sums are whole
    numbers, exact in fp32 up to 2^24, beyond which a wave's sum and the joins of at most 3072
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
