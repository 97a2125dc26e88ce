"""Timing cases of the operators beside the SPLA decode: the rotary position
embedding (rotate), the append that rotates the keys on the way (append_rope)
and the exact attention of new tokens over the cache (attend).

A case is a flat dict; keys by operator (op):
  all     dtype, batch, hq, hkv, d
  rotate  new (positions per sequence), lo, hi (tokens the shortest and longest
          sequence hold before), rot (rotated coordinates), pairs (half or
          interleaved), scaling, factor, fused (q and k are slices of one
          projection's rows), grad (the transposed map: a gradient)
  append  B (block size), new (tokens the longest sequence gets), least (the
          shortest), lo, hi (tokens held before), cap (capacity per sequence),
          paged, rot, pairs, scaling, factor
  attend  B, new (queries per sequence), lo, hi (tokens held, the new ones
          included), cap, paged, softcap (0: none), bias (by distance), doc
          (mean document length, 0: one document), prefix (tokens that every
          query sees, 0: none), ragged (sequences bring different counts)
With `own` false, run() computes the plain form in elementary torch operations
on the same cache buffers; with `own` true it calls the framework.
"""

import math

import torch

own = False

BASE = 500000.0  # rotary base
ORIG, LOW, HIGH = 8192, 1.0, 4.0  # context and band limits of scaling by parts


def _spla():
    from paper_2601_22379_amd import spla
    return spla


# ------------------------------------------------------------------- cases
def _rotate(name, batch, hq, hkv, d, new, lo, hi, dtype="bf16", rot=0, pairs="half",
            scaling="none", factor=1.0, fused=False, grad=False):
    c = dict(op="rotate", dtype=dtype, batch=batch, hq=hq, hkv=hkv, d=d, new=new, lo=lo, hi=hi,
             rot=rot or d, pairs=pairs, scaling=scaling, factor=factor, fused=fused, grad=grad)
    return dict(name=name, **c) if name else c


def _append(name, batch, hq, hkv, d, B, new, least, lo, hi, cap, paged=False, dtype="bf16", rot=0,
            pairs="half", scaling="none", factor=1.0):
    c = dict(op="append", dtype=dtype, batch=batch, hq=hq, hkv=hkv, d=d, B=B, new=new, least=least,
             lo=lo, hi=hi, cap=cap, paged=paged, rot=rot or d, pairs=pairs, scaling=scaling,
             factor=factor)
    return dict(name=name, **c) if name else c


def _attend(name, batch, hq, hkv, d, B, new, lo, hi, cap, paged=False, dtype="bf16", softcap=0.0,
            bias=False, doc=0, prefix=0, ragged=False):
    c = dict(op="attend", dtype=dtype, batch=batch, hq=hq, hkv=hkv, d=d, B=B, new=new, lo=lo, hi=hi,
             cap=cap, paged=paged, softcap=softcap, bias=bias, doc=doc, prefix=prefix,
             ragged=ragged)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # the token of one generating user: all latency
        _rotate("rotate_step", 1, 32, 8, 128, 1, 4100, 4100),
        # prompts straight from the projection's rows, context stretched fourfold
        _rotate("rotate_prompt_8k", 4, 32, 8, 128, 2048, 0, 6144, scaling="parts", factor=4.0,
                fused=True),
        # gradients of a short fp32 batch, half of each head rotated
        _rotate("rotate_grad_f32", 3, 8, 8, 64, 1001, 0, 0, dtype="f32", rot=32,
                pairs="interleaved", grad=True),
        # the step of a serving batch: a token for each of 16 conversations in a page pool
        _append("append_step_b16", 16, 32, 8, 128, 64, 1, 1, 500, 8000, 16384, paged=True),
        # prompts of uneven length into a page pool, stretched context
        _append("append_prompt_16k", 4, 32, 8, 128, 64, 16384, 11003, 0, 0, 32768, paged=True,
                scaling="parts", factor=4.0),
        # an odd fp32 chunk after short prefixes, part of each head rotated
        _append("append_chunk_f32", 2, 8, 4, 64, 32, 777, 130, 333, 1000, 4096, dtype="f32", rot=48,
                pairs="interleaved", scaling="linear", factor=2.0),
        # one token of one user in an ordinary conversation
        _attend("attend_step_4k", 1, 32, 8, 128, 64, 1, 4100, 4100, 32768),
        # a serving batch's step over long, uneven contexts in a page pool
        _attend("attend_step_b16_64k", 16, 32, 8, 128, 64, 1, 16000, 65000, 65536, paged=True),
        # a whole prompt
        _attend("attend_prompt_8k", 1, 32, 8, 128, 64, 8192, 8192, 8192, 8192),
        # a question after a long document, groups of five heads, capped scores
        _attend("attend_chunk_64k_cap", 1, 40, 8, 128, 64, 509, 66045, 66045, 131072, paged=True,
                softcap=30.0),
        # packed documents with a bias by distance, uneven chunks
        _attend("attend_docs_bias", 2, 32, 8, 128, 64, 4096, 3500, 5000, 8192, bias=True, doc=700,
                ragged=True),
        # a short fp32 chunk over a prefix that all of its queries see
        _attend("attend_prefix_f32", 2, 8, 4, 64, 32, 300, 1000, 1300, 2048, dtype="f32",
                prefix=1111, softcap=20.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["rotate", "append", "append", "attend", "attend", "attend"])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    d = 64 if rng.random() < (0.6 if dtype == "f32" else 0.25) else 128
    hkv = rng.choice([1, 2, 4, 8, 8])
    group = rng.choice([1, 2, 4, 4, 5, 6, 8, 8, 16])
    hq = hkv * group
    B = rng.choice([32, 64, 64, 128])
    rot = rng.choice([d, d, d // 2, 3 * d // 4, 2 * rng.randint(1, d // 2)])
    pairs = rng.choice(["half", "interleaved"])
    scaling, factor = rng.choice([("none", 1.0), ("linear", 4.0), ("base", 8.0), ("parts", 4.0)])
    if op == "rotate":
        batch = _log_int(rng, 1, 32)
        new = 1 if rng.random() < 0.3 else _log_int(rng, 2, max(2, 8192 * 32 // (batch * hq)))
        hi = _log_int(rng, 1, 1 << 20)
        return _rotate(None, batch, hq, hkv, d, new, rng.randint(0, hi), hi, dtype, rot, pairs,
                       scaling, factor, rng.random() < 0.5, rng.random() < 0.3)
    paged = rng.random() < 0.4
    if op == "append":
        batch = _log_int(rng, 1, 32)
        new = 1 if rng.random() < 0.3 else _log_int(rng, 2, 400000 // (batch * hkv))
        hi = 0 if rng.random() < 0.4 else _log_int(rng, 1, min(65536, 800000 // (batch * hkv)))
        least = rng.randint(1, new)
        cap = -(-(hi + new + rng.randint(0, hi + new)) // B) * B
        return _append(None, batch, hq, hkv, d, B, new, least, rng.randint(0, hi), hi, cap, paged,
                       dtype, rot, pairs, scaling, factor)
    if rng.random() < 0.45:  # a step, or a few tokens
        batch = _log_int(rng, 1, 32)
        new = 1 if rng.random() < 0.6 else rng.randint(2, 16)
        hi = _log_int(rng, new, max(new, min(1 << 19, 6000000 // (batch * hkv))))
    else:
        batch = _log_int(rng, 1, 4)
        new = _log_int(rng, 17, 4096)
        hi = _log_int(rng, new, max(new, min(131072, (1 << 28) // (batch * hq * new))))
    lo = rng.randint(max(1, hi // 4), hi)
    if dtype == "f32":
        hi, lo = min(hi, 8192), min(lo, 8192)
        new = min(new, 512, hi)
    cap = -(-(hi + rng.randint(0, hi)) // B) * B
    kind = rng.choice(["causal", "causal", "softcap", "bias", "doc", "prefix"])
    return _attend(None, batch, hq, hkv, d, B, new, lo, hi, cap, paged, dtype,
                   30.0 if kind == "softcap" else 0.0, kind == "bias",
                   _log_int(rng, 20, hi + 20) if kind == "doc" else 0,
                   rng.randint(1, hi) if kind == "prefix" else 0, rng.random() < 0.3)


# ------------------------------------------------------------------ inputs
def _frac(b):
    return (1.0 + b * 0.6180339887498949) % 1.0 if b else 1.0


def _spread(c, lo, hi):
    """Counts per sequence: spread unevenly over lo .. hi, the largest first."""
    return [int(round(lo + (hi - lo) * _frac(b))) for b in range(c["batch"])]


def _held(c):
    return _spread(c, c["lo"], c["hi"])


def _news(c):
    """New tokens per sequence."""
    if c["op"] == "append":
        return _spread(c, c["least"], c["new"])
    if not c.get("ragged"):
        n = [c["new"]] * c["batch"]
    else:
        n = _spread(c, (c["new"] + 1) // 2, c["new"])
    return [min(x, h) for x, h in zip(n, _held(c))] if c["op"] == "attend" else n


def _gen(seed, tag):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1000003 + tag * 7919) % (1 << 62))
    return g


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _randn(c, seed, tag, *shape):
    return torch.randn(shape, generator=_gen(seed, tag), device="cuda", dtype=_dtype(c))


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _encode_k(c, rows):
    """[..., B, d] token-major rows -> [..., B d] as the cache holds a block's keys."""
    B, d, lead = c["B"], c["d"], rows.shape[:-2]
    if c["dtype"] == "f32":
        return rows.reshape(lead + (B * d,))
    x = rows.reshape((-1, B // 32, 4, 2, 4, d // 32, 4, 8))  # token 8a + 4m + b, 32s + 8g + e
    return x.permute(0, 1, 3, 5, 6, 2, 4, 7).reshape(lead + (B * d,))


def _decode_k(c, slot):
    B, d, lead = c["B"], c["d"], slot.shape[:-1]
    if c["dtype"] == "f32":
        return slot.reshape(lead + (B, d))
    x = slot.reshape((-1, B // 32, 2, d // 32, 4, 4, 4, 8))
    return x.permute(0, 1, 5, 2, 6, 3, 4, 7).reshape(lead + (B, d))


def _encode_v(c, rows):
    B, d, lead = c["B"], c["d"], rows.shape[:-2]
    if c["dtype"] == "f32":
        return rows.transpose(-1, -2).reshape(lead + (B * d,))
    x = rows.reshape((-1, B // 32, 4, 8, d // 16, 16))  # token 8g + e, coordinate 16t + i
    return x.permute(0, 1, 4, 2, 5, 3).reshape(lead + (B * d,))


def _decode_v(c, slot):
    B, d, lead = c["B"], c["d"], slot.shape[:-1]
    if c["dtype"] == "f32":
        return slot.reshape(lead + (d, B)).transpose(-1, -2)
    x = slot.reshape((-1, B // 32, d // 16, 4, 16, 8))
    return x.permute(0, 1, 3, 5, 2, 4).reshape(lead + (B, d))


def _prefix_rows(c, seed, n):
    """Keys and values [batch, hkv, n, d] of the tokens held: a heavy-tailed offset per block."""
    b, h, d = c["batch"], c["hkv"], c["d"]
    nb = -(-n // 64)
    r = 0.25 * torch.rand((b, h, nb, 1, 1), generator=_gen(seed, 1), device="cuda")
    r = 0.25 * r.clamp_min(1e-4).pow(-1 / 1.5)
    u = torch.randn((b, h, nb, 1, d), generator=_gen(seed, 2), device="cuda")
    off = (r * u / u.norm(dim=-1, keepdim=True)).to(_dtype(c))
    k = _randn(c, seed, 3, b, h, nb, 64, d).add_(off)
    return k.view(b, h, nb * 64, d)[:, :, :n], _randn(c, seed, 4, b, h, n, d)


def _table(c, seed):
    """Pages of every block: of a shuffled pool, or in order (a contiguous cache)."""
    nb = c["cap"] // c["B"]
    n = c["batch"] * nb
    if c["paged"]:
        return torch.randperm(n, generator=_gen(seed, 5), device="cuda").int().view(-1, nb)
    return None


def _pages(c, table, pool, blocks):
    """[batch, hkv, n, B d] blocks of the cache buffer; blocks int64 [batch, n]."""
    b, h, bd, nb = c["batch"], c["hkv"], c["B"] * c["d"], c["cap"] // c["B"]
    if table is None:
        at = blocks[:, None, :, None].expand(b, h, blocks.shape[1], bd)
        return pool.view(b, h, nb, bd).gather(2, at)
    page = table.long().gather(1, blocks)
    return pool.view(b * nb, h, bd)[page].transpose(1, 2)


def _put_pages(c, table, pool, blocks, x):
    b, h, bd, nb = c["batch"], c["hkv"], c["B"] * c["d"], c["cap"] // c["B"]
    if table is None:
        at = blocks[:, None, :, None].expand(b, h, blocks.shape[1], bd)
        pool.view(b, h, nb, bd).scatter_(2, at, x)
    else:
        pool.view(b * nb, h, bd)[table.long().gather(1, blocks)] = x.transpose(1, 2)


def _phi(x):
    e = torch.exp(x - x.amax(-1, keepdim=True))
    return e / e.sum(-1, keepdim=True)


def _filled(c, seed):
    """The buffers of a cache that holds the prefix."""
    b, h, d, B, cap, dt = c["batch"], c["hkv"], c["d"], c["B"], c["cap"], _dtype(c)
    nb, lens = cap // B, _held(c)
    s = {"table": _table(c, seed), "lens": _ints(lens)}
    s["k"] = torch.zeros(b * h * cap * d, dtype=dt, device="cuda")
    s["v"] = torch.zeros_like(s["k"])
    n = -(-max(lens) // B) * B
    if n:
        k, v = _prefix_rows(c, seed, n)
        ok = torch.arange(n, device="cuda") < s["lens"][:, None]
        k, v = (x * ok[:, None, :, None] for x in (k, v))  # zeros past each sequence
        blocks = torch.arange(n // B, device="cuda").expand(b, n // B)
        _put_pages(c, s["table"], s["k"], blocks, _encode_k(c, k.view(b, h, -1, B, d)))
        _put_pages(c, s["table"], s["v"], blocks, _encode_v(c, v.view(b, h, -1, B, d)))
    nt = -(-nb // 64)
    s["stats"] = torch.zeros(b * h * nt * 2 * d * 64, device="cuda")
    s["state"] = torch.zeros(b * h * d * d, device="cuda")
    s["norm"] = torch.zeros(b * h * d, device="cuda")
    if n and c["op"] == "append":  # what an append updates
        cnt = (s["lens"][:, None] - blocks * B).clamp(0, B)
        _put_stats(c, s["stats"], blocks, k.view(b, h, -1, B, d), cnt)
        phi = _phi(k.float()) * ok[:, None, :, None]
        s["state"] = (phi.transpose(2, 3) @ v.float()).reshape(-1)
        s["norm"] = phi.sum(2).reshape(-1)
    return s


def _put_stats(c, stats, blocks, rows, cnt, keep=None):
    """Mean and sum of squared deviations of blocks (int64 [batch, n]) from their rows
    [batch, hkv, n, B, d], the first cnt [batch, n] of each; blocks with none stay."""
    b, h, d, n = c["batch"], c["hkv"], c["d"], blocks.shape[1]
    nt = -(-(c["cap"] // c["B"]) // 64)
    ok = (torch.arange(c["B"], device="cuda") < cnt[..., None])[:, None, :, :, None]
    x = rows.float()
    m = cnt.clamp_min(1)[:, None, :, None].float()
    mean = (x * ok).sum(3) / m
    m2 = ((x - mean[:, :, :, None]).square() * ok).sum(3)
    new = torch.stack([mean, m2], 3).view(b, h, n, 2, d // 4, 4)
    at = stats.view(b, h, nt, 2, d // 4, 64, 4).permute(0, 1, 2, 5, 3, 4, 6)
    bi = torch.arange(b, device="cuda")[:, None, None]
    hi = torch.arange(h, device="cuda")[None, :, None]
    ti, si = (blocks // 64)[:, None], (blocks % 64)[:, None]
    live = (cnt > 0)[:, None, :, None, None, None]
    at[bi, hi, ti, si] = torch.where(live, new, at[bi, hi, ti, si])


def _first_keys(c, seed):
    """First position each query sees (the start of its document), int32 [new, batch]."""
    if not c["doc"]:
        return None
    n = max(1, c["hi"] // c["doc"])
    cuts = torch.randint(0, c["hi"], (c["batch"], n), generator=_gen(seed, 9), device="cuda")
    cuts = torch.cat([torch.zeros_like(cuts[:, :1]), cuts.sort(1).values], 1)
    p = _positions(c).clamp_min(0).t().contiguous()  # [batch, new]
    at = torch.searchsorted(cuts, p, right=True) - 1
    return cuts.gather(1, at).t().contiguous().int()


def _positions(c):
    """Positions of the queries of an attend case, int64 [new, batch]."""
    first = [h - n for h, n in zip(_held(c), _news(c))]
    return torch.arange(c["new"], device="cuda")[:, None] + _ints(first).long()


def prepare(case, seed):
    c = case
    b, hq, hkv, d, T = c["batch"], c["hq"], c["hkv"], c["d"], c["new"]
    s = {"c": c}
    if c["op"] == "rotate":
        s["lens"] = _ints(_held(c))
        if c["fused"]:  # rows of a projection that gives q, k and v
            x = _randn(c, seed, 3, T, b, (hq + 2 * hkv) * d)
            s["q"] = x[..., :hq * d].view(T, b, hq, d)
            s["kn"] = x[..., hq * d:(hq + hkv) * d].view(T, b, hkv, d)
        else:
            s["q"], s["kn"] = _randn(c, seed, 3, T, b, hq, d), _randn(c, seed, 4, T, b, hkv, d)
        s["out"] = [torch.empty(x.shape, dtype=x.dtype, device="cuda") for x in (s["q"], s["kn"])]
    elif c["op"] == "append":
        s |= _filled(c, seed)
        s["kn"], s["vn"] = _randn(c, seed, 6, b, hkv, T, d), _randn(c, seed, 7, b, hkv, T, d)
        s["n"] = _ints(_news(c))
    else:
        s |= _filled(c, seed)
        s["q"] = _randn(c, seed, 6, T, b, hq, d) * 1.5
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros((T, b, hq), device="cuda")
        s["n"] = _ints(_news(c)) if c["ragged"] or min(_news(c)) < T else None
        s["slopes"] = None
        if c["bias"]:
            s["slopes"] = torch.exp2(-8.0 * torch.arange(1, hq + 1, device="cuda") / hq)
        s["first"] = _first_keys(c, seed)
        s["prefix"] = None
        if c["prefix"]:
            s["prefix"] = _ints(_spread(c, (c["prefix"] + 1) // 2, c["prefix"]))
    if c["op"] != "attend":
        s["turns"] = _turns(c)
    if c["op"] == "append":
        s["saved"] = [s["state"].clone(), s["norm"].clone(), s["lens"].clone()]
        nt = -(-(c["cap"] // c["B"]) // 64)  # statistics of the block each append starts in
        blk = s["lens"].long().clamp_max(c["cap"] - 1) // c["B"]
        at = torch.arange(s["stats"].numel(), device="cuda").view(b, hkv, nt, 2, d // 4, 64, 4)
        at = at.permute(0, 2, 5, 1, 3, 4, 6)[torch.arange(b, device="cuda"), blk // 64, blk % 64]
        s["stats_at"] = at.reshape(-1)
        s["saved"].append(s["stats"][s["stats_at"]])
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program of the framework keeps: its config, rotation and cache."""
    spla, c = _spla(), s["c"]
    B = c.get("B", 64)
    cap = c.get("cap", B)
    s["cfg"] = spla.make_config(c["batch"], c["hq"], c["hkv"], c["d"], B, 8, cap, c["dtype"],
                                kv_pages=c["batch"] * (cap // B) if c.get("paged") else 0)
    if c["op"] != "attend":
        s["rope"] = spla.make_rope(c["d"], c["rot"], c["pairs"], BASE, c["scaling"], c["factor"],
                                   ORIG, LOW, HIGH)
    if c["op"] != "rotate":
        s["cache"] = spla.SplaCache(s["cfg"], "cuda:0", block_table=s["table"])
        for mine, theirs in (("k", "k"), ("v", "v"), ("stats", "stats"), ("state", "state"),
                             ("norm", "norm"), ("lens", "seq_lens")):
            buf = getattr(s["cache"], theirs)
            buf.copy_(s[mine])
            s[mine] = buf


# --------------------------------------------------------------------- run
def run(s):
    op = s["c"]["op"]
    if op == "append":  # back to the tokens held before
        torch._foreach_copy_([s["state"], s["norm"], s["lens"]], s["saved"][:3])
        s["stats"].index_copy_(0, s["stats_at"], s["saved"][3])
    if own:
        return {"rotate": _own_rotate, "append": _own_append, "attend": _own_attend}[op](s)
    return {"rotate": _plain_rotate, "append": _plain_append, "attend": _plain_attend}[op](s)


def _own_rotate(s):
    return _spla().rotate(s["cfg"], s["rope"], q=s["q"], k=s["kn"], seq_lens=s["lens"],
                          q_out=s["out"][0], k_out=s["out"][1], transpose=s["c"]["grad"])


def _own_append(s):
    s["cache"].append_rope(s["rope"], s["kn"], s["vn"], s["n"])
    return s["k"], s["v"], s["state"], s["norm"], s["stats"], s["lens"]


def _own_attend(s):
    return s["cache"].attend(s["q"], s["out"], s["lse"], softcap=s["c"]["softcap"],
                             slopes=s["slopes"], first_key=s["first"], prefix_len=s["prefix"],
                             n_new=s["n"])


def _turns(c):
    """Radians per position of each pair, fp64."""
    r = c["rot"]
    i = torch.arange(r // 2, dtype=torch.float64, device="cuda")
    base = BASE
    if c["scaling"] == "base" and r > 2:
        base = BASE * c["factor"] ** (r / (r - 2))
    w = base ** (-2.0 * i / r)
    if c["scaling"] == "linear":
        w = w / c["factor"]
    if c["scaling"] == "parts":
        keep = ((ORIG * w / (2.0 * math.pi) - LOW) / (HIGH - LOW)).clamp(0.0, 1.0)
        w = w * (keep + (1.0 - keep) / c["factor"])
    return w


def _rotated(c, x, pos, w, sign=1.0):
    """x [..., d] rotated at positions pos (broadcast over x's leading dimensions): in fp64, so
    that values next to a rounding border fall on the right side, rounded once."""
    r = c["rot"]
    a = pos[..., None].double() * w
    cos, sin = torch.cos(a), sign * torch.sin(a)
    y = x[..., :r].double()
    if c["pairs"] == "half":
        x0, x1 = y[..., :r // 2], y[..., r // 2:]
        y = torch.cat([x0 * cos - x1 * sin, x1 * cos + x0 * sin], -1)
    else:
        x0, x1 = y[..., 0::2], y[..., 1::2]
        y = torch.stack([x0 * cos - x1 * sin, x1 * cos + x0 * sin], -1).flatten(-2)
    return torch.cat([y.to(x.dtype), x[..., r:]], -1)


def _plain_rotate(s):
    c = s["c"]
    pos = (torch.arange(c["new"], device="cuda")[:, None] + s["lens"])[..., None]
    sign = -1.0 if c["grad"] else 1.0
    return tuple(_rotated(c, x, pos, s["turns"], sign) for x in (s["q"], s["kn"]))


def _plain_append(s):
    c = s["c"]
    b, h, d, B, T = c["batch"], c["hkv"], c["d"], c["B"], c["new"]
    t = torch.arange(T, device="cuda")
    L0, n = s["lens"].long(), s["n"].long()
    rows = _rotated(c, s["kn"], (L0[:, None] + t)[:, None], s["turns"])
    # the blocks touched (sequences with fewer name their last one again)
    first, last = L0 // B, (L0 + n - 1).clamp_min(0) // B
    blocks = first[:, None] + torch.arange((T + B - 2) // B + 1, device="cuda")
    blocks = torch.minimum(blocks, torch.maximum(last, first)[:, None]).clamp_max(c["cap"] // B - 1)
    pos = blocks[:, :, None] * B + torch.arange(B, device="cuda")  # [b, nblk, B]
    src = pos - L0[:, None, None]
    new = ((src >= 0) & (src < n[:, None, None]))[:, None, :, :, None]
    src = src.clamp(0, T - 1).view(b, 1, -1, 1).expand(b, h, -1, d)
    shape = (b, h) + pos.shape[1:] + (d,)
    k = _decode_k(c, _pages(c, s["table"], s["k"], blocks))
    v = _decode_v(c, _pages(c, s["table"], s["v"], blocks))
    k = torch.where(new, rows.gather(2, src).view(shape), k)
    v = torch.where(new, s["vn"].gather(2, src).view(shape), v)
    _put_pages(c, s["table"], s["k"], blocks, _encode_k(c, k))
    _put_pages(c, s["table"], s["v"], blocks, _encode_v(c, v))
    cnt = ((L0 + n)[:, None] - blocks * B).clamp(0, B) * (n > 0)[:, None]
    _put_stats(c, s["stats"], blocks, k, cnt)
    phi = _phi(rows.float()) * (t < n[:, None])[:, None, :, None]
    s["state"] += (phi.transpose(2, 3) @ s["vn"].float()).reshape(-1)
    s["norm"] += phi.sum(2).reshape(-1)
    s["lens"] += s["n"]
    return s["k"], s["v"], s["state"], s["norm"], s["stats"], s["lens"]


def _plain_attend(s):
    c = s["c"]
    b, h, d, B, T, G = c["batch"], c["hkv"], c["d"], c["B"], c["new"], c["hq"] // c["hkv"]
    n = -(-max(_held(c)) // B)
    blocks = torch.arange(n, device="cuda").expand(b, n)
    k = _decode_k(c, _pages(c, s["table"], s["k"], blocks)).reshape(b, h, n * B, d).float()
    q = s["q"].view(T, b, h, G, d).permute(1, 2, 3, 0, 4).reshape(b, h, G * T, d).float()
    x = (q @ k.transpose(2, 3)).mul_(1.0 / math.sqrt(d)).view(b, h, G, T, n * B)
    del k
    if c["softcap"]:
        x = x.div_(c["softcap"]).tanh_().mul_(c["softcap"])
    j = torch.arange(n * B, device="cuda")
    L = s["lens"].long()
    bring = s["n"].long() if s["n"] is not None else torch.full_like(L, T)
    t = torch.arange(T, device="cuda")
    p = ((L - bring)[:, None] + t)[:, :, None]  # [b, T, 1]
    if s["slopes"] is not None:
        x = x.sub_(s["slopes"].view(1, h, G, 1, 1) * (p - j).abs().float()[:, None, None])
    see = (j <= p) & (j < L[:, None, None])
    if s["prefix"] is not None:
        see = (see | (j < s["prefix"][:, None, None])) & (j < L[:, None, None])
    if s["first"] is not None:
        see = see & (j >= s["first"].t()[:, :, None])
    x = x.masked_fill_(~see[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    x = x.sub_(torch.where(m == -math.inf, torch.zeros_like(m), m)).exp_()
    l = x.sum(-1, keepdim=True)
    v = _decode_v(c, _pages(c, s["table"], s["v"], blocks)).reshape(b, h, n * B, d).float()
    o = (x.view(b, h, G * T, n * B) @ v).view(b, h, G, T, d) / torch.where(l > 0, l, 1.0)
    o = o.permute(3, 0, 1, 2, 4).reshape(T, b, h * G, d).to(s["q"].dtype)
    lse = (m + l.log())[..., 0].permute(3, 0, 1, 2).reshape(T, b, h * G)
    live = (t[:, None] < bring)[:, :, None]  # rows past a sequence's own stay
    s["out"].copy_(torch.where(live[..., None], o, s["out"]))
    s["lse"].copy_(torch.where(live, lse, s["lse"]))
    return s["out"], s["lse"]


# ------------------------------------------------------------- what is due
def _visible(c):
    """Visible keys summed over the queries, and the keys read, per KV head."""
    pairs = keys = 0.0
    prefix = _spread(c, (c["prefix"] + 1) // 2, c["prefix"]) if c["prefix"] else [0] * c["batch"]
    for L, n, pre in zip(_held(c), _news(c), prefix):
        per = [min(L, max(p + 1, pre)) for p in range(L - n, L)]
        if c["doc"]:  # about half a document before each query
            per = [min(x, c["doc"] / 2 + 1) for x in per]
            keys += min(L, n + c["doc"] / 2)
        else:
            keys += L
        pairs += float(sum(per))
    return pairs, keys


def work(case):
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    b, hq, hkv, d, T = c["batch"], c["hq"], c["hkv"], c["d"], c["new"]
    if c["op"] == "rotate":
        n = b * T * (hq + hkv)
        return {"bytes": 2.0 * n * d * e, "flops": 3.0 * n * c["rot"]}
    if c["op"] == "append":
        tok = sum(_news(c)) * hkv
        units = sum((L + n - 1) // c["B"] - L // c["B"] + 1 for L, n in zip(_held(c), _news(c)))
        return {"bytes": 4.0 * tok * d * e + units * hkv * 2 * d * 4
                + 2.0 * b * hkv * (d + 1) * d * 4,
                "flops": tok * (2.0 * d * d + 3.0 * c["rot"] + 8.0 * d)}
    pairs, keys = _visible(c)
    rows = sum(_news(c)) * hq
    return {"bytes": 2.0 * keys * hkv * d * e + rows * (2.0 * d * e + 4),
            "flops": 4.0 * d * pairs * hq}


# ---------------------------------------------------- the same in 64 bits
def _angles64(c, pos):
    """Unit complex numbers of each pair at integer positions, computed from the definition."""
    r, out = c["rot"], []
    base = BASE * c["factor"] ** (r / (r - 2)) if c["scaling"] == "base" and r > 2 else BASE
    for i in range(r // 2):
        w = base ** (-2.0 * i / r)
        if c["scaling"] == "linear":
            w /= c["factor"]
        if c["scaling"] == "parts":
            n = ORIG * w / (2.0 * math.pi)
            keep = min(1.0, max(0.0, (n - LOW) / (HIGH - LOW)))
            w = keep * w + (1.0 - keep) * w / c["factor"]
        out.append(w)
    a = pos.double()[..., None] * torch.tensor(out, dtype=torch.float64, device="cuda")
    return torch.polar(torch.ones_like(a), a)


def _turn64(c, x, u):
    """Rows x [..., d] times the unit numbers u [..., rot / 2], as complex pairs."""
    r, y = c["rot"], x.double().clone()
    if c["pairs"] == "half":
        z = torch.complex(y[..., :r // 2], y[..., r // 2:r]) * u
        y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
    else:
        z = torch.complex(y[..., 0:r:2], y[..., 1:r:2]) * u
        y[..., 0:r:2], y[..., 1:r:2] = z.real, z.imag
    return y


def exact(case, seed):
    c, keep = case, own
    if c["op"] == "attend" and c["hq"] * c["batch"] * c["new"] * c["hi"] > 1 << 33:
        return None
    if c["op"] == "append" and c["batch"] * c["hkv"] * c["new"] * c["d"] > 1 << 27:
        return None
    globals()["own"] = False
    try:
        s = prepare(c, seed)
    finally:
        globals()["own"] = keep
    return {"rotate": _exact_rotate, "append": _exact_append, "attend": _exact_attend}[c["op"]](s)


def _exact_rotate(s):
    c = s["c"]
    pos = torch.arange(c["new"], device="cuda")[:, None] + s["lens"].long()
    u = _angles64(c, pos)[:, :, None]
    return tuple(_turn64(c, x, u.conj() if c["grad"] else u) for x in (s["q"], s["kn"]))


def _exact_append(s):
    c = s["c"]
    b, h, d, B = c["batch"], c["hkv"], c["d"], c["B"]
    k, v = s["k"].double(), s["v"].double()
    state, norm = s["state"].double().view(b, h, d, d), s["norm"].double().view(b, h, d)
    stats = s["stats"].double()
    nb = c["cap"] // B
    at = stats.view(b, h, -1, 2, d // 4, 64, 4).permute(0, 1, 2, 5, 3, 4, 6)
    for i, (L, n) in enumerate(zip(_held(c), _news(c))):
        pos = torch.arange(L, L + n, device="cuda")
        x = _turn64(c, s["kn"][i, :, :n], _angles64(c, pos))
        cached = x.to(_dtype(c)).double()
        y = s["vn"][i, :, :n].double()
        e = torch.softmax(cached, -1)
        state[i] += e.transpose(1, 2) @ y
        norm[i] += e.sum(1)
        for blk in range(L // B, (L + n - 1) // B + 1):
            one = torch.tensor([[blk]] * b, device="cuda")
            old = (_pages(c, s["table"], p, one)[i:i + 1, :, 0] for p in (k, v))
            old = [f(c, p)[0].clone() for f, p in zip((_decode_k, _decode_v), old)]
            t0, t1 = max(L, blk * B), min(L + n, (blk + 1) * B)
            full = old[0].clone()  # the keys as the cache holds them
            full[:, t0 - blk * B:t1 - blk * B] = cached[:, t0 - L:t1 - L]
            old[0][:, t0 - blk * B:t1 - blk * B] = x[:, t0 - L:t1 - L]
            old[1][:, t0 - blk * B:t1 - blk * B] = y[:, t0 - L:t1 - L]
            slot = [i, slice(None), blk] if s["table"] is None else [int(s["table"][i, blk])]
            shape = (b, h, nb, B * d) if s["table"] is None else (b * nb, h, B * d)
            k.view(shape)[tuple(slot)] = _encode_k(c, old[0])
            v.view(shape)[tuple(slot)] = _encode_v(c, old[1])
            full = full[:, :t1 - blk * B]
            mean = full.mean(1)
            m2 = (full - mean[:, None]).square().sum(1)
            at[i, :, blk // 64, blk % 64] = torch.stack([mean, m2], 1).view(h, 2, d // 4, 4)
    return k, v, state.reshape(-1), norm.reshape(-1), stats, None


def _exact_attend(s):
    c = s["c"]
    T, b, hq, d = s["q"].shape
    G, B = hq // c["hkv"], c["B"]
    out = torch.zeros((T, b, hq, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((T, b, hq), dtype=torch.float64, device="cuda")
    for i, (L, n) in enumerate(zip(_held(c), _news(c))):
        nb = -(-L // B)
        blocks = torch.arange(nb, device="cuda").expand(b, nb)
        K = _decode_k(c, _pages(c, s["table"], s["k"], blocks)[i]).reshape(c["hkv"], -1, d)
        V = _decode_v(c, _pages(c, s["table"], s["v"], blocks)[i]).reshape(c["hkv"], -1, d)
        p = torch.arange(L - n, L, device="cuda")[:, None]
        j = torch.arange(L, device="cuda")
        hide = j > p
        if s["prefix"] is not None:
            hide &= j >= s["prefix"][i]
        if s["first"] is not None:
            hide |= j < s["first"][:n, i, None]
        for m in range(hq):
            x = s["q"][:n, i, m].double() @ K[m // G, :L].double().t() / math.sqrt(d)
            if c["softcap"]:
                x = c["softcap"] * torch.tanh(x / c["softcap"])
            if s["slopes"] is not None:
                x = x - s["slopes"][m].double() * (p - j).abs()
            x = x.masked_fill(hide, -math.inf)
            lse[:n, i, m] = torch.logsumexp(x, -1)
            out[:n, i, m] = torch.softmax(x, -1) @ V[m // G, :L].double()
    return out, lse
