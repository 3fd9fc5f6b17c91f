"""A comparison for the first LLM layer's attention that pins infinities too: attn_ref's bound of an
infinite lse is infinite itself, so that any finite result would lie within it."""
import torch


def check(name, got, want):
    """Every element within its bound, where the reference is infinite equal to it, and every bound a
    number where the reference is finite; rows that the reference leaves NaN are not looked at."""
    value, bound = want
    got = got.double().cpu()
    look = ~value.isnan()
    near = torch.where(value.isinf(), got == value, bound.isfinite() & ((got - value).abs() <= bound))
    bad = look & ~near
    if bad.any():
        i = tuple(torch.nonzero(bad)[0].tolist())
        raise AssertionError(f"{name}: {int(bad.sum())} of {int(look.sum())} off, first at {i}: "
                             f"{got[i].item()} for {value[i].item()} within {bound[i].item()}")
