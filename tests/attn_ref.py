"""Plain float64 forms of the first LLM layer's attention and its cache (torch on the CPU), and
how far a kernel may be from them: every rounding of its scheme counted at half a step.

A kernel's scores are fp32 sums of d products, so a score is off by at most (d + 2) 2^-24 scale
sum |q||k|, and a weight by that part of itself; sums over n keys or rows add n 2^-24 of their
terms' magnitudes.  bf16 kernels round weights and score gradients to bf16 before their second
products, 2^-8 of each; an output is rounded once, 2^-8 or 2^-24 of it."""
import math

import torch

F32 = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def visible(lq, lk):
    return torch.arange(lk)[None] <= torch.arange(lq)[:, None] + lk - lq


def attention(q, k, v, seqs, scale, d_o=None, o_in=None):
    """seqs: (first query, queries, first key, keys).  Returns {name: (value, bound)}, float64;
    rows of no sequence are NaN.  o_in: the o a backward is given (else the exact one)."""
    u = half_step(q.dtype)
    w_round = u if q.dtype == torch.bfloat16 else 0.0
    q, k, v = (x.double() for x in (q, k, v))
    hq, hk, d = q.shape[1], k.shape[1], q.shape[2]
    nan = lambda *s: torch.full(s, math.nan, dtype=torch.float64)
    res = {"o": (nan(*q.shape), nan(*q.shape)), "lse": (nan(hq, q.shape[0]), nan(hq, q.shape[0]))}
    if d_o is not None:
        d_o = d_o.double()
        for name, like in (("dq", q), ("dk", k), ("dv", v)):
            res[name] = (nan(*like.shape), nan(*like.shape))
    for r, n, kr, m in seqs:
        if d_o is not None:
            for name in ("dk", "dv"):
                for x in res[name]:
                    x[kr:kr + m] = 0.0
        if n == 0:
            continue
        see = visible(n, m)
        many = (max(m, n, d) + 8) * F32
        for h in range(hq):
            a, b, z = q[r:r + n, h], k[kr:kr + m, h // (hq // hk)], v[kr:kr + m, h // (hq // hk)]
            s = scale * a @ b.t()
            off = (d + 2) * F32 * scale * (a.abs() @ b.abs().t())
            s = torch.where(see, s, -math.inf)
            top = s.amax(1, keepdim=True) if m else torch.full((n, 1), -math.inf).double()
            e = torch.where(see, torch.exp(s - torch.where(top.isinf(), 0.0, top)), 0.0)
            tot = e.sum(1, keepdim=True)
            p = torch.where(tot > 0, e / tot, 0.0)
            zc = torch.where(see.any(0)[:, None], z, 0.0) if m else z
            o = p @ zc
            wide = torch.where(see, off, 0.0).amax(1, keepdim=True) if m else torch.zeros(n, 1).double()
            p_off = p * (2 * wide + w_round + many)       # weights: scores, rounding, the sum
            res["o"][0][r:r + n, h] = o
            res["o"][1][r:r + n, h] = p_off @ zc.abs() * (1 + u) + u * o.abs() + 1e-30
            lse = (top + torch.log(tot))[:, 0]
            res["lse"][0][h, r:r + n] = lse
            res["lse"][1][h, r:r + n] = wide[:, 0] + many + 8 * F32 * (1 + lse.abs())
            if d_o is None:
                continue
            g = d_o[r:r + n, h]
            dp, dp_off = g @ z.t(), many * (g.abs() @ z.abs().t())
            oo = o if o_in is None else o_in[r:r + n, h].double()
            delta = (g * oo).sum(1, keepdim=True)
            d_off = ((g * o).sum(1, keepdim=True) - delta).abs() + many * (g * oo).abs().sum(1, keepdim=True)
            true = (g * o).sum(1, keepdim=True)
            ds = p * (dp - true)
            ds_off = p * (d_off + dp_off) + p_off * (dp.abs() + true.abs()) + ds.abs() * (w_round + 4 * F32)
            kh = h // (hq // hk)
            res["dq"][0][r:r + n, h] = scale * ds @ b
            res["dq"][1][r:r + n, h] = (scale * (ds_off + many * ds.abs()) @ b.abs() * (1 + u) +
                                        u * (scale * ds @ b).abs() + 1e-30)
            res["dk"][0][kr:kr + m, kh] += scale * ds.t() @ a
            res["dk"][1][kr:kr + m, kh] += scale * (ds_off + many * ds.abs()).t() @ a.abs() * (1 + u)
            res["dv"][0][kr:kr + m, kh] += p.t() @ g
            res["dv"][1][kr:kr + m, kh] += (p_off + many * p).t() @ g.abs() * (1 + u)
        if d_o is not None:
            for name in ("dk", "dv"):
                res[name][1][kr:kr + m] += u * res[name][0][kr:kr + m].abs() + 1e-30
    return res


def check(name, got, want):
    """Every element within its bound; rows that the reference leaves NaN are not looked at."""
    value, bound = want
    got = got.double().cpu()
    look = ~value.isnan()
    same = (got == value) & look                  # infinities
    over = ((got - value).abs() > bound) & look & ~same
    bad = over | (got.isnan() & look)
    if bad.any():
        i = tuple(torch.nonzero(bad)[0].tolist())
        raise AssertionError(f"{name}: {int(bad.sum())} of {int(look.sum())} off, first at {i}: "
                             f"{got[i].item()} for {value[i].item()} within {bound[i].item()}")


# ---- the cache -----------------------------------------------------------------------------

def e4m3_values():
    """The 127 magnitudes of e4m3, in order."""
    out = [m * 2.0 ** -9 for m in range(8)]
    for e in range(1, 16):
        out += [(8 + m) * 2.0 ** (e - 10) for m in range(8) if not (e == 15 and m == 7)]
    return out


def quantise(x):
    """(values, exponents) of heads [..., d] of one token each: nearest e4m3 value, ties to the
    even code, of x / 2^e."""
    x = x.double()
    a = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1)
    e = torch.full(a.shape, -120, dtype=torch.int64)
    for i in range(-119, 121):
        e = torch.where(a > 448.0 * 2.0 ** (i - 1), i, e)
    f = torch.pow(2.0, e.double())[..., None]
    table = torch.tensor(e4m3_values(), dtype=torch.float64)
    y = torch.where(x.isfinite(), x / f, 0.0).abs()
    hi = torch.searchsorted(table, y.contiguous()).clamp(max=len(table) - 1)
    lo = (hi - 1).clamp(min=0)
    dl, dh = y - table[lo], table[hi] - y
    pick = torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    val = torch.where(x < 0, -table[pick], table[pick]) * f
    return torch.where(x.isfinite(), val, math.nan), e
