"""The attention of the first language-model layer behind the seam, on one GPU: cases with
inputs, their plain forms and a float64 reference.

  prompt   causal attention over whole prompts, grouped heads, sequences of different lengths;
           the keys of a sequence may begin before its queries (a chunk over its prefix)
  train    the same with its backward pass
  decode   attention of one new token of every sequence over a paged key-value cache
  cache    new keys and values written to the pages, in 8 bits or as they are, and the
           sequences read back as adjacent rows

`run` is one pass as a training or serving loop makes it: with `own` through the package's
entry points, without it in elementary torch operations."""
import math
import random

import numpy as np
import torch

own = False


def listed():
    def attend(name, op, seqs, length, hq, hk, d, dtype, **kw):
        return dict({"name": name, "op": op, "seqs": seqs, "len": length, "least": 0.5,
                     "hq": hq, "hk": hk, "d": d, "dtype": dtype, "prefix": 0, "padded": False},
                    **kw)

    def decode(name, seqs, length, hq, hk, d, page, dtype, cache, **kw):
        return dict({"name": name, "op": "decode", "seqs": seqs, "len": length, "least": 0.1,
                     "hq": hq, "hk": hk, "d": d, "page": page, "dtype": dtype, "cache": cache},
                    **kw)

    def cache(name, seqs, length, new, hk, d, page, dtype, cache):
        return {"name": name, "op": "cache", "seqs": seqs, "len": length, "new": new,
                "least": 0.5, "hk": hk, "d": d, "page": page, "dtype": dtype, "cache": cache}

    return [
        # serving: one short prompt of text
        attend("prompt_short", "prompt", 1, 77, 14, 2, 64, "bf16", least=1.0),
        # the frozen pass of a micro-batch: eight padded sequences of at most 8192 rows
        attend("prompt_batch", "prompt", 8, 8192, 28, 4, 128, "bf16", padded=True),
        # serving: the next 512 rows of four long prompts over what the cache gave back
        attend("prompt_chunk", "prompt", 4, 512, 32, 8, 128, "bf16", least=1.0, prefix=32256),
        # a small fp32 model, odd lengths
        attend("train_small_f32", "train", 5, 333, 6, 6, 64, "f32", least=0.1),
        # many short texts in one batch, the encoder's own head width
        attend("train_short", "train", 64, 700, 16, 16, 80, "bf16", least=0.03),
        # a trained micro-batch of eight sequences of at most 8192 rows
        attend("train_batch", "train", 8, 8192, 28, 4, 128, "bf16", padded=True),
        # serving: the next token of 8 short texts
        decode("decode_small", 8, 1000, 28, 4, 128, 16, "bf16", "bf16"),
        # serving: the next token of 64 running sequences
        decode("decode_batch", 64, 16384, 32, 8, 128, 32, "bf16", "bf16"),
        # serving: few sequences of long clips, the cache in 8 bits
        decode("decode_long", 4, 131072, 28, 4, 128, 64, "bf16", "e4m3", least=0.5),
        # 64 short sequences take one token each and are moved out of the cache
        cache("cache_tokens", 64, 512, 1, 8, 128, 16, "bf16", "e4m3"),
        # a chunk of four long prompts is written, and the prompts so far read for it
        cache("cache_chunk", 4, 32768, 2048, 4, 128, 64, "bf16", "bf16"),
        # whole prompts of a small fp32 model, narrow heads, into 8 bits and back
        cache("cache_prompt_f32", 3, 3001, 3001, 6, 40, 8, "f32", "e4m3"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))

    op = rng.choice(["prompt", "prompt", "train", "train", "decode", "decode", "cache"])
    hk = rng.choice([1, 2, 4, 8, rng.randint(1, 16)])
    d = rng.choice([32, 64, 80, 96, 128, 128, 128, 8 * rng.randint(1, 16)])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    least = rng.choice([0.05, 0.5, 1.0])
    if op in ("decode", "cache"):
        page = 2 ** rng.randint(0, 8)
        cache = rng.choice([dtype, "e4m3"])
        if op == "decode":
            length = log_int(1, 131072)
            hq = hk * rng.randint(1, 16)
            most = int(2.0e9 / (length * hk * d * (8 if cache == "f32" else 4)))
            hq = min(hq, 64 - 64 % hk)
            return {"op": op, "seqs": log_int(1, max(1, min(256, most))), "len": length,
                    "least": least, "hq": hq, "hk": hk, "d": d, "page": page, "dtype": dtype,
                    "cache": cache}
        length = log_int(1, 32768)
        most = int(1.3e8 / (length * hk * d * (2 if dtype == "bf16" else 4)))
        return {"op": op, "seqs": log_int(1, max(1, min(256, most))), "len": length,
                "new": log_int(1, length), "least": least, "hk": hk, "d": d, "page": page,
                "dtype": dtype, "cache": cache}
    hq = min(64, hk * rng.randint(1, 8))
    hq -= hq % hk
    # (the gradients of sequences of one row are zero: nothing to compare)
    length = log_int(8 if op == "train" else 1, 8192 if dtype == "bf16" else 2048)
    prefix = log_int(1, 8192) if op == "prompt" and rng.random() < 0.3 else 0
    # fp32 runs at a sixteenth of the bf16 rate; a backward costs two and a half forwards
    most = 3.0e12 / (4 * d * hq * length * (length / 2 + prefix))
    most = min(65536 * 32 // (length * hq), most / (16 if dtype == "f32" else 1))
    return {"op": op, "seqs": log_int(1, max(1, min(256, int(most)))), "len": length,
            "least": least, "hq": hq, "hk": hk, "d": d, "dtype": dtype, "prefix": prefix,
            "padded": rng.random() < 0.5}


# ---- inputs ------------------------------------------------------------------------------

def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _lengths(case):
    """Every sequence's rows, between `least` of the longest and the longest, which is there."""
    rng = random.Random(case["len"] * 31 + case["seqs"])
    lo = max(1, int(case["least"] * case["len"]))
    return [case["len"]] + [rng.randint(lo, case["len"]) for _ in range(case["seqs"] - 1)]


def _sequences(case):
    """(first query row, queries, first key row, keys) of every sequence, int64 arrays, and the
    rows of q and of k."""
    n = np.array(_lengths(case), np.int64)
    step = np.full_like(n, case["len"]) if case["padded"] else n
    keys = n + case["prefix"]
    kstep = step + case["prefix"]
    return (np.cumsum(step) - step, n, np.cumsum(kstep) - kstep, keys,
            int(step.sum()), int(kstep.sum()))


def _heads(case, seed):
    """q, k and v as columns of one product, or k and v apart where they reach further back; for
    training also the gradient of the output."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt, hq, hk, d = _dtype(case["dtype"]), case["hq"], case["hk"], case["d"]
    *_, rows, krows = _sequences(case)

    def normal(r, h):
        return torch.randn((r, h, d), device="cuda", generator=gen).to(dt)

    if case["prefix"]:
        q, k, v = normal(rows, hq), normal(krows, hk), normal(krows, hk)
    else:
        x = normal(rows, hq + 2 * hk)
        q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    return q, k, v, normal(rows, hq) if case["op"] == "train" else None


def _pages(case, gen):
    """The pool's pages and the sequences' tables: every page somewhere, a few left over."""
    page, n = case["page"], _lengths(case)
    width = -(-max(n) // page)
    need = [-(-x // page) for x in n]
    total = sum(need) + 7
    order = torch.randperm(total, device="cuda", generator=gen).to(torch.int32)
    table = torch.zeros((len(n), width), dtype=torch.int32, device="cuda")
    at = 0
    for s, x in enumerate(need):
        table[s, :x] = order[at:at + x]
        at += x
    return total, table


def _pool(case, total, gen):
    """One side of a cache that is in use: [pages][heads][page][d], and for 8 bits a byte a token
    and head, the scale's exponent + 127."""
    shape = (total, case["hk"], case["page"], case["d"])
    x = torch.empty(shape, dtype=_dtype(case["cache"]) if case["cache"] != "e4m3"
                    else torch.float8_e4m3fn, device="cuda")
    for part in x.split(max(1, (1 << 27) // (shape[1] * shape[2] * shape[3]))):
        r = torch.randn(part.shape, device="cuda", generator=gen)
        part.copy_((r * 64).clamp(-448, 448) if case["cache"] == "e4m3" else r)
    if case["cache"] != "e4m3":
        return x, None
    return x, torch.randint(119, 123, shape[:3], device="cuda", generator=gen, dtype=torch.uint8)


def _cached(case, seed):
    """Pages, tables, lengths, and q (decode) or the rows to write (cache)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    total, table = _pages(case, gen)
    k, ks = _pool(case, total, gen)
    v, vs = _pool(case, total, gen)
    s = {"k": k, "ks": ks, "v": v, "vs": vs, "table": table}
    n, dt, d = _lengths(case), _dtype(case["dtype"]), case["d"]
    if case["op"] == "decode":
        s["lens"] = torch.tensor(n, dtype=torch.int32, device="cuda")
        s["q"] = torch.randn((len(n), case["hq"], d), device="cuda", generator=gen).to(dt)
        return s
    new = [min(case["new"], x) for x in n]
    x = torch.randn((sum(new), 2 * case["hk"], d), device="cuda", generator=gen)
    x *= torch.exp(torch.randn((sum(new), 2 * case["hk"], 1), device="cuda", generator=gen))
    x = x.to(dt)
    s["k_new"], s["v_new"] = x[:, :case["hk"]], x[:, case["hk"]:]
    for name, lo in (("new", [a - b for a, b in zip(n, new)]), ("all", [0] * len(n))):
        s[name + "_pos"] = torch.cat([torch.arange(a, b, dtype=torch.int32)
                                      for a, b in zip(lo, n)]).cuda()
        s[name + "_seq"] = torch.cat([torch.full((b - a,), i, dtype=torch.int32)
                                      for i, (a, b) in enumerate(zip(lo, n))]).cuda()
    return s


def prepare(case, seed):
    dt = _dtype(case["dtype"])

    def out(*shape, dtype=dt):
        return torch.zeros(shape, dtype=dtype, device="cuda")

    if case["op"] in ("prompt", "train"):
        q, k, v, do = _heads(case, seed)
        row, n, krow, keys, rows, _ = _sequences(case)
        s = {"op": case["op"], "q": q, "k": k, "v": v, "do": do, "row": row, "len": n,
             "krow": krow, "keys": keys, "scale": case["d"] ** -0.5, "o": out(*q.shape),
             "lse": out(case["hq"], rows, dtype=torch.float32)}
        if do is not None:
            dx = out(rows, case["hq"] + 2 * case["hk"], case["d"])   # the product's gradient
            s["dq"], s["dk"], s["dv"] = dx.split([case["hq"], case["hk"], case["hk"]], 1)
            if own:
                import paper_2607_03229_amd as mp
                s["scratch"] = torch.empty(
                    mp.op_causal_attention_scratch_bytes(q.shape[0], case["hq"], k.shape[0],
                                                         case["hk"], case["d"]),
                    dtype=torch.uint8, device="cuda")
        return s
    s = dict(_cached(case, seed), op=case["op"], page=case["page"], scale=case["d"] ** -0.5)
    if case["op"] == "decode":
        s["o"] = out(*s["q"].shape)
        s["lse"] = out(case["hq"], case["seqs"], dtype=torch.float32)
    else:
        rows = s["all_pos"].numel()
        s["k_out"], s["v_out"] = (out(rows, case["hk"], case["d"]) for _ in range(2))
    if own:
        import paper_2607_03229_amd as mp
        s["cache"] = mp.KvCache(s["k"], s["v"], s["ks"], s["vs"])
        if case["op"] == "decode":
            s["scratch"] = torch.empty(
                mp.op_cache_attention_scratch_bytes(case["seqs"], case["hq"], case["hk"],
                                                    case["d"]), dtype=torch.uint8, device="cuda")
    return s


# ---- one pass ----------------------------------------------------------------------------

def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    import paper_2607_03229_amd as mp
    if s["op"] in ("prompt", "train"):
        seqs = dict(key_row=s["krow"], key_len=s["keys"], scale=s["scale"])
        mp.op_causal_attention_fwd(s["q"], s["k"], s["v"], s["o"], s["lse"], s["row"], s["len"],
                                   **seqs)
        if s["op"] == "prompt":
            return {"o": s["o"], "lse": s["lse"]}
        mp.op_causal_attention_bwd(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["row"],
                                   s["len"], s["dq"], s["dk"], s["dv"], s["scratch"], **seqs)
        return {"o": s["o"], "lse": s["lse"], "dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}
    if s["op"] == "decode":
        mp.op_cache_attention(s["cache"], s["q"], s["table"], s["lens"], s["o"], s["scratch"],
                              lse=s["lse"], scale=s["scale"])
        return {"o": s["o"], "lse": s["lse"]}
    mp.op_cache_write(s["cache"], s["k_new"], s["v_new"], s["table"], s["new_pos"],
                      seq=s["new_seq"])
    mp.op_cache_read(s["cache"], s["table"], s["all_pos"], s["k_out"], s["v_out"],
                     seq=s["all_seq"])
    return {"k": s["k_out"], "v": s["v_out"]}


def _plain(s):
    if s["op"] in ("prompt", "train"):
        return _plain_attention(s)
    if s["op"] == "decode":
        return _plain_decode(s)
    return {"k": _plain_cache(s, s["k"], s["ks"], s["k_new"], s["k_out"]),
            "v": _plain_cache(s, s["v"], s["vs"], s["v_new"], s["v_out"])}


def _plain_attention(s):
    """All sequences side by side, padded to the longest; blocks of queries so that the scores
    stay below 2^28 values."""
    q, k, v, do, dev = s["q"], s["k"], s["v"], s["do"], s["q"].device
    n, hq, hk, d = len(s["row"]), q.shape[1], k.shape[1], q.shape[2]
    row, nq, krow, nk = (torch.from_numpy(s[x]).to(dev) for x in ("row", "len", "krow", "keys"))
    most_q, most_k = int(s["len"].max()), int(s["keys"].max())
    at_q = torch.arange(most_q, device=dev)
    at_k = torch.arange(most_k, device=dev)
    in_q, in_k = at_q < nq[:, None], at_k < nk[:, None]
    rows_q = (row[:, None] + at_q)[in_q]

    def sides(x, rows, inside, heads):      # [n][hk][heads of a group][longest][d], fp32
        y = torch.zeros((*inside.shape, x.shape[1], d), device=dev)
        y[inside] = x[rows].float()
        return y.view(n, -1, hk, heads, d).permute(0, 2, 3, 1, 4).contiguous()

    rows_k = (krow[:, None] + at_k)[in_k]
    qf = sides(q, rows_q, in_q, hq // hk)
    kf, vf = sides(k, rows_k, in_k, 1)[:, :, 0], sides(v, rows_k, in_k, 1)[:, :, 0]
    of, lf = torch.empty_like(qf), torch.empty(qf.shape[:4], device=dev)
    if do is not None:
        dof = sides(do, rows_q, in_q, hq // hk)
        dqf, dkf, dvf = torch.empty_like(qf), torch.zeros_like(kf), torch.zeros_like(vf)
    kt, vt = kf.transpose(-1, -2).contiguous(), vf.transpose(-1, -2).contiguous()
    step = max(1, (1 << 28) // (n * hq * most_k))
    for i in range(0, most_q, step):
        qc = qf[:, :, :, i:i + step]
        c = qc.shape[3]

        def flat(x):
            return x.reshape(n, hk, -1, x.shape[-1])

        sc = (flat(qc) @ kt).view(n, hk, -1, c, most_k).mul_(s["scale"])
        seen = (at_k <= (at_q[i:i + c] + (nk - nq)[:, None])[..., None]) & in_k[:, None]
        sc.masked_fill_(~seen[:, None, None], -math.inf)
        top = sc.amax(-1, keepdim=True)
        p = sc.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        p /= total
        of[:, :, :, i:i + c] = (flat(p) @ vf).view(qc.shape)
        lf[:, :, :, i:i + c] = (top + total.log())[..., 0]
        if do is None:
            continue
        pd, dc = flat(p), flat(dof[:, :, :, i:i + c])
        dvf += pd.transpose(-1, -2) @ dc
        ds = dc @ vt
        ds -= (ds * pd).sum(-1, keepdim=True)
        ds.mul_(pd).mul_(s["scale"])
        dqf[:, :, :, i:i + c] = (ds @ kf).view(qc.shape)
        dkf += ds.transpose(-1, -2) @ flat(qc)

    def back(x, rows, inside, like):
        y = torch.zeros(like.shape, dtype=like.dtype, device=dev)
        y[rows] = x.permute(0, 3, 1, 2, 4).reshape(*inside.shape, -1, d)[inside].to(like.dtype)
        return y

    lse = torch.zeros((q.shape[0], hq), device=dev)
    lse[rows_q] = lf.permute(0, 3, 1, 2).reshape(*in_q.shape, hq)[in_q]
    out = {"o": back(of, rows_q, in_q, q), "lse": lse.t().contiguous()}
    if do is not None:
        out["dq"] = back(dqf, rows_q, in_q, q)
        out["dk"], out["dv"] = (back(x[:, :, None], rows_k, in_k, k) for x in (dkf, dvf))
    return out


def _values(x, scale, *at):
    """fp32 values of places of a pool."""
    if scale is None:
        return x[at].float()
    return (x.view(torch.uint8)[at].view(x.dtype).float() *
            torch.exp2(scale[at].float() - 127)[..., None])


def _plain_decode(s):
    q, table, lens = s["q"], s["table"].long(), s["lens"]
    n, hq, d = q.shape
    hk = s["k"].shape[1]

    def side(x, scale):     # [n][hk][tokens][d]
        y = _values(x, scale, table)
        return y.transpose(1, 2).reshape(n, hk, -1, d)

    k = side(s["k"], s["ks"])
    sc = (q.float().view(n, hk, -1, d) @ k.transpose(-1, -2).contiguous()) * s["scale"]
    seen = torch.arange(sc.shape[-1], device=q.device) < lens[:, None]
    sc.masked_fill_(~seen[:, None, None], -math.inf)
    top = sc.amax(-1, keepdim=True)
    p = (sc - top).exp()
    total = p.sum(-1, keepdim=True)
    o = (p / total) @ side(s["v"], s["vs"]).masked_fill_(~seen[:, None, :, None], 0.0)
    return {"o": o.reshape(n, hq, d).to(q.dtype),
            "lse": (top + total.log()).reshape(n, hq).t().contiguous()}


def _plain_cache(s, pool, scale, new, out):
    """New rows into the pages, then every row of the sequences out of them."""
    page, table = s["page"], s["table"].long()
    pos, seq = s["new_pos"].long(), s["new_seq"].long()
    at, off = table[seq, pos // page], pos % page
    x = new.float()
    if scale is None:
        pool[at, :, off] = x.to(pool.dtype)
    else:
        m, e = torch.frexp(x.abs().amax(-1))
        e = (e - 9 + (m > 0.875)).clamp(-120, 120)
        x = torch.ldexp(x, -e[..., None]).to(pool.dtype)
        pool.view(torch.uint8)[at, :, off] = x.view(torch.uint8)
        scale[at, :, off] = (e + 127).to(torch.uint8)
    pos, seq = s["all_pos"].long(), s["all_seq"].long()
    at, off = table[seq, pos // page], pos % page
    return _values(pool, scale, at, slice(None), off).to(out.dtype)


# ---- what a pass cannot do without -------------------------------------------------------

def work(case):
    size = {"bf16": 2, "f32": 4, "e4m3": 1}
    esz, d, hk = size[case["dtype"]], case["d"], case["hk"]
    if case["op"] in ("prompt", "train"):
        _, n, _, keys, *_ = _sequences(case)
        hq, rq, rk = case["hq"], int(n.sum()), int(keys.sum())
        pairs = int((n * (n + 1) // 2 + n * (keys - n)).sum())
        q, kv = rq * hq * d * esz, 2 * rk * hk * d * esz
        if case["op"] == "prompt":
            return {"bytes": 2 * q + kv + 4 * rq * hq, "flops": 4 * d * hq * pairs}
        # dq, dk, dv and the gradient of o beside them; scores made once and used twice
        return {"bytes": 4 * q + 2 * kv + 4 * rq * hq, "flops": 14 * d * hq * pairs}
    n = _lengths(case)
    row = 2 * hk * (d * size[case["cache"]] + (case["cache"] == "e4m3"))
    if case["op"] == "decode":
        q = case["seqs"] * case["hq"] * d * esz
        return {"bytes": sum(n) * row + 2 * q, "flops": 4 * d * case["hq"] * sum(n)}
    plain = 2 * hk * d * esz
    new = sum(min(case["new"], x) for x in n)
    return {"bytes": (new + sum(n)) * (row + plain), "flops": 2 * hk * d * (new + sum(n))}


# ---- the same in 64 bits -----------------------------------------------------------------

def exact(case, seed):
    if case["op"] in ("prompt", "train"):
        return _exact_attention(case, seed)
    s = _cached(case, seed)
    if case["op"] == "decode":
        return _exact_decode(case, s)
    return {"k": _exact_cache(case, s, "k"), "v": _exact_cache(case, s, "v")}


def _exact_attention(case, seed):
    q, k, v, do = _heads(case, seed)
    rows, hq, d = q.shape
    group = hq // case["hk"]
    o = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros((hq, rows), dtype=torch.float64, device="cuda")
    dq, dk, dv = (torch.zeros(x.shape, dtype=torch.float64, device="cuda") for x in (q, k, v))
    row, n, krow, keys, *_ = _sequences(case)
    for r, c, kr, kc in zip(row.tolist(), n.tolist(), krow.tolist(), keys.tolist()):
        hidden = torch.ones((c, kc), dtype=torch.bool, device="cuda").triu(kc - c + 1)
        for h in range(hq):
            a, b, z = (x[i:i + m, j].double() for x, i, m, j in
                       ((q, r, c, h), (k, kr, kc, h // group), (v, kr, kc, h // group)))
            w = torch.mm(a, b.t()) / math.sqrt(d)
            w[hidden] = -math.inf
            lse[h, r:r + c] = torch.logsumexp(w, 1)
            w = torch.softmax(w, 1)
            o[r:r + c, h] = torch.mm(w, z)
            if do is None:
                continue
            g = do[r:r + c, h].double()
            dv[kr:kr + kc, h // group] += torch.mm(w.t(), g)
            w *= torch.mm(g, z.t()) - (g * o[r:r + c, h]).sum(1)[:, None]
            dq[r:r + c, h] = torch.mm(w, b) / math.sqrt(d)
            dk[kr:kr + kc, h // group] += torch.mm(w.t(), a) / math.sqrt(d)
    out = {"o": o, "lse": lse}
    return out if do is None else dict(out, dq=dq, dk=dk, dv=dv)


def _exact_rows(case, s, side, i, n):
    """The first n tokens of sequence i, [n][hk][d] float64."""
    at = s["table"][i, :-(-n // case["page"])].long()
    if s[side + "s"] is None:
        x = s[side][at].double()
    else:
        x = s[side].view(torch.uint8)[at].view(s[side].dtype).double()
        x *= torch.exp2(s[side + "s"][at].double() - 127)[..., None]
    return x.permute(0, 2, 1, 3).reshape(-1, case["hk"], case["d"])[:n]


def _exact_decode(case, s):
    o = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty((case["hq"], case["seqs"]), dtype=torch.float64, device="cuda")
    group = case["hq"] // case["hk"]
    for i, n in enumerate(_lengths(case)):
        k, v = (_exact_rows(case, s, side, i, n) for side in ("k", "v"))
        for h in range(case["hk"]):
            heads = slice(h * group, (h + 1) * group)
            w = torch.mm(s["q"][i, heads].double(), k[:, h].t()) / math.sqrt(case["d"])
            lse[heads, i] = torch.logsumexp(w, 1)
            o[i, heads] = torch.mm(torch.softmax(w, 1), v[:, h])
    return {"o": o, "lse": lse}


def _exact_cache(case, s, side):
    new, at, parts = s[side + "_new"].double(), 0, []
    for i, n in enumerate(_lengths(case)):
        x, c = _exact_rows(case, s, side, i, n), min(case["new"], n)
        y = new[at:at + c]
        at += c
        if case["cache"] == "e4m3":
            y = _exact_e4m3(y)
        elif case["cache"] == "bf16":
            y = y.to(torch.bfloat16).double()
        x[n - c:] = y
        parts.append(x.to(_dtype(case["dtype"])).double())
    return torch.cat(parts)


def _exact_e4m3(x):
    """To the nearest value of 4 significant bits (ties to the even one) no finer than 2^-9,
    after a power of two that brings the largest of a head to 448 or less."""
    top = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top / 448.0))
    e += (top > 448.0 * torch.exp2(e)).double()
    e -= (top <= 448.0 * torch.exp2(e - 1)).double()
    e = e.clamp(-120, 120)
    y = x * torch.exp2(-e)
    unit = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / unit) * unit * torch.exp2(e)
