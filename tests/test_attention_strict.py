"""The strict comparison of the attention's tests, on the host."""
import math

import pytest
import torch

from tests import attn_ref as R
from tests import attn_strict as S

INF, NAN = math.inf, math.nan


def rejects(got, value, bound):
    t = lambda *x: torch.tensor(x, dtype=torch.float64)
    try:
        S.check("x", t(got), (t(value), t(bound)))
    except AssertionError:
        return True
    return False


@pytest.mark.parametrize("got,value,bound,bad", [
    (1.0, 1.0, 0.0, False), (1.1, 1.0, 0.2, False), (1.3, 1.0, 0.2, True), (NAN, 1.0, 0.2, True),
    (INF, 1.0, 0.2, True), (-INF, -INF, INF, False), (7.0, -INF, INF, True), (INF, -INF, INF, True),
    (NAN, -INF, INF, True), (7.0, -INF, NAN, True), (1.0, 1.0, INF, True), (1.0, 1.0, NAN, True),
    (7.0, NAN, NAN, False)])
def test_check(got, value, bound, bad):
    assert rejects(got, value, bound) == bad


def test_lse_of_sequences_without_keys_is_pinned():
    """What was never written (the tests' guard) is no lse of a sequence without keys."""
    gen = torch.Generator().manual_seed(0)
    q, k, v = (torch.randn(n, 2, 8, generator=gen) for n in (4, 3, 3))
    value, bound = R.attention(q, k, v, [(0, 1, 0, 0), (1, 3, 0, 2)], 0.3)["lse"]
    assert (value[:, :2] == -INF).all() and value[:, 2:].isfinite().all()
    S.check("lse", value, (value, bound))
    for i in (0, 1, 2):
        wrong = value.clone()
        wrong[1, i] = 7.0
        with pytest.raises(AssertionError):
            S.check("lse", wrong, (value, bound))
