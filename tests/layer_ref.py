"""Plain float64 forms of the operators around the first LLM layer (numpy), and the sizes their
tests share.  A rotary configuration is a dict with the fields of RopeCfg."""
import numpy as np


def rope_cfg(d, sections, rot=None, theta=10000.0, order=0, spectrum=0, pairing=0):
    return dict(head_dim=d, sections=list(sections), rot_dim=d if rot is None else rot, theta=theta,
                order=order, spectrum=spectrum, pairing=pairing)


def pair_axes(c):
    """(axis, how many pairs of that axis come before) of every pair."""
    half, sec = c["rot_dim"] // 2, c["sections"]
    out, seen = [], [0] * len(sec)
    for i in range(half):
        if c["order"] == 1:
            a = i % len(sec)
            a = a if i // len(sec) < sec[a] else 0
        else:
            a = int(np.searchsorted(np.cumsum(sec), i, side="right"))
        out.append((a, seen[a]))
        seen[a] += 1
    assert seen == list(sec)
    return out


def angles(c, pos):
    """[rows][rot_dim / 2], reduced modulo one turn in extended precision."""
    half = c["rot_dim"] // 2
    out = np.zeros((pos.shape[1], half))
    for i, (a, n) in enumerate(pair_axes(c)):
        e = n / c["sections"][a] if c["spectrum"] == 1 else i / half
        f = np.longdouble(c["theta"]) ** np.longdouble(-e)
        x = pos[a].astype(np.longdouble) * f
        two_pi = np.longdouble("6.283185307179586476925286766559")
        out[:, i] = (x - two_pi * np.round(x / two_pi)).astype(np.float64)
    return out


def columns(c):
    """The two columns of every pair."""
    half = c["rot_dim"] // 2
    i = np.arange(half)
    return (2 * i, 2 * i + 1) if c["pairing"] == 1 else (i, i + half)


def rotate(c, x, pos, inverse=False):
    """x [rows][heads][d] float64."""
    ang = angles(c, pos)[:, None, :]
    cos, sin = np.cos(ang), np.sin(ang) * (-1.0 if inverse else 1.0)
    ia, ib = columns(c)
    y = x.copy()
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * cos - b * sin, b * cos + a * sin
    return y


def partners(c, x):
    """|a| + |b| for the columns of a pair, |x| elsewhere: the scale of a rotation's errors."""
    ia, ib = columns(c)
    m = np.abs(x)
    s = m[..., ia] + m[..., ib]
    m[..., ia] = m[..., ib] = s
    return m


def norm_rope(c, x, gain, eps, pos):
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return rotate(c, x * r * gain, pos)


def norm_rope_bwd(c, dy, x, gain, eps, pos):
    """(dx, dgain, scale of dx's errors, scale of dgain's errors)."""
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    u = rotate(c, dy, pos, inverse=True)
    ua = partners(c, dy)
    m = r * r * (gain * u * x).mean(-1, keepdims=True)
    ma = r * r * (np.abs(gain) * ua * np.abs(x)).mean(-1, keepdims=True)
    return (r * (gain * u - x * m), (u * x * r).sum((0, 1)),
            r * (np.abs(gain) * ua + np.abs(x) * ma), (ua * np.abs(x) * r).sum((0, 1)))


def seam_positions(seqs, items, pos):
    """seqs: (row, len, first position); items: (row, (t, gh, gw), step); pos int32 [3][rows],
    written in place.  Returns the next position of each sequence."""
    nxt = []
    for row, n, p in seqs:
        r = row
        starts = {i[0]: i for i in items if row <= i[0] < row + n}
        while r < row + n:
            if r in starts:
                _, (t, gh, gw), step = starts[r]
                h, w = gh // 2, gw // 2
                for tau in range(t):
                    for y in range(h):
                        for x in range(w):
                            pos[:, r] = (p + tau * step, p + y, p + x)
                            r += 1
                p += max((t - 1) * step + 1, h, w)
            else:
                pos[:, r] = p
                p += 1
                r += 1
        nxt.append(p)
    return nxt
