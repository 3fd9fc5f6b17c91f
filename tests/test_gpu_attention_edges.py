"""The first LLM layer's attention on the GPU where its other tests do not look: infinities pinned
(attn_strict.py)."""

import pytest
import torch

from tests import attn_ref as R
from tests import attn_strict as S
from tests import test_gpu_attention_ops as G

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def strict(monkeypatch):
    """Every comparison of this module pins infinities; fp32 is torch's default type."""
    old = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    monkeypatch.setattr(R, "check", S.check)
    yield
    torch.set_default_dtype(old)


# ---- queries and sequences without keys ---------------------------------------------------------

@pytest.mark.parametrize("dtype,cache_dtype", G.CACHES, ids=str)
def test_tokens_of_empty_sequences(dtype, cache_dtype):
    G.decode(dtype, cache_dtype, 4, 2, 128, 32, [0, 1, 0, 5000, -3, 130, 0])
    G.decode(dtype, cache_dtype, 2, 1, 64, 32, [0])
    G.decode(dtype, cache_dtype, 2, 1, 64, 16, [(i * 37) % 90 for i in range(300)])
    lens = [(i * 61) % 400 for i in range(360)]
    lens[100] = 30000
    G.decode(dtype, cache_dtype, 6, 3, 64, 16, lens)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (BF, 96), (BF, 200), (FP, 64)])
@pytest.mark.parametrize("prefix", [[-1, -40, -500], [100, -20, 0], [-129, -64, -33]], ids=str)
def test_queries_without_keys(dtype, d, prefix):
    G.run(dtype, 4, 2, d, [60, 77, 330], prefix=prefix, gap=2)
