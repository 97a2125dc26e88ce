"""Attention over the 8-bit cache with a window: each way that a call may go (tiles of 128 rows,
tiles of 16, workgroups shared among sequences), which the tests see to themselves."""

import math

import pytest
import torch

import cache8_ref as C
import cache8_rule
from paper_2601_22379_amd import spla

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spla.lib()
    return torch.device("cuda:0")


def randn(dev, dtype, *shape, seed=0, scale=1.0):
    g = torch.Generator(device=dev).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=dev) * scale).to(DT[dtype])


def ints(dev, v):
    return torch.tensor(v, dtype=torch.int32, device=dev)


def filled(dev, dtype, lens, hq, hkv, d, cap, paged, B=64, nan=()):
    """A cache of sequences of `lens` tokens in buffers that held NaN, and the values it holds
    (fp64); nan: ("k" or "v", sequence, token, KV head, coordinate) that are NaN."""
    b, table, pages = len(lens), None, 0
    if paged:
        pages = b * (cap // B) + 1
        table = torch.randperm(pages, generator=torch.Generator().manual_seed(1))[:pages - 1]
        table = table.view(b, -1).int().to(dev)
    cache = spla.SplaCache8(spla.make_config(b, hq, hkv, d, B, 8, cap, dtype, kv_pages=pages), dev,
                            block_table=table)
    cache.k.fill_(0x7F)
    cache.v.fill_(0xFF)
    rows = {s: randn(dev, dtype, max(lens), b, hkv, d, seed=i) for i, s in enumerate("kv")}
    for s, i, t, h, c in nan:
        rows[s][t, i, h, c] = math.nan
    cache.append(rows["k"], rows["v"], ints(dev, lens))
    K, V = (x.double().permute(1, 2, 0, 3).contiguous() for x in cache.read(max(lens)))
    return cache, K, V


# name: dtype, d, hkv, group, lens, cap, T, window, sinks, paged
TILES = {
    "split": ("bf16", 128, 7, 4, [1200, 900], 1280, 300, 700, 5, True),
    "split_d64": ("bf16", 64, 4, 8, [2000], 2048, 513, 500, 3, False),
    "whole": ("bf16", 128, 16, 4, [700, 650, 641], 768, 640, 600, 1, False),
    "whole_d64": ("bf16", 64, 16, 4, [700, 650, 641], 768, 640, 97, 40, True),
    "short_window": ("bf16", 128, 4, 4, [1500], 1536, 1100, 33, 3, False),
    "short_window_d64": ("bf16", 64, 4, 4, [1500], 1536, 1100, 1, 1, True),
    "odd_group": ("bf16", 128, 6, 5, [1000, 333], 1024, 333, 450, 129, True),
    "f32": ("f32", 128, 8, 4, [1300, 701], 1344, 600, 700, 4, True),
    "f32_d64": ("f32", 64, 16, 4, [900, 800], 960, 777, 65, 2, False),
}
KINDS = ["window", "sinks", "softcap", "softcap_sinks", "softcap_large_sinks", "bias", "bias_sinks",
         "docs", "docs_sinks", "all"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", list(TILES))
def test_tiles_of_128(dev, name, kind):
    dtype, d, hkv, group, lens, cap, T, window, sinks, paged = TILES[name]
    b, hq = len(lens), hkv * group
    sinks = sinks if "sinks" in kind or kind == "all" else 0
    assert cache8_rule.plan(dtype, b, hkv, group, cap, T, window, sinks).tiles
    cache, K, V = filled(dev, dtype, lens, hq, hkv, d, cap, paged)
    q = randn(dev, dtype, T, b, hq, d, seed=3, scale=2.0)
    kw, ref = {}, {}
    if "softcap" in kind:  # bounds all scores / needs the running maximum
        kw["softcap"] = ref["softcap"] = 200.0 if "large" in kind else 30.0
    if kind == "all":
        kw["softcap"] = ref["softcap"] = 50.0
    if "bias" in kind or kind == "all":
        kw["slopes"] = ref["slopes"] = torch.exp2(-torch.arange(1.0, hq + 1, device=dev) * 8 / hq)
    if "docs" in kind or kind == "all":
        # the starts of documents of 1 to 150 tokens, and some queries that see nothing
        g = torch.Generator().manual_seed(5)
        f = torch.zeros((T, b), dtype=torch.int32)
        for i, L in enumerate(lens):
            starts = torch.cat([torch.zeros(1, dtype=torch.long),
                                torch.randint(1, 150, (L,), generator=g).cumsum(0)])
            pos = torch.arange(L - min(T, L), L)
            f[:len(pos), i] = starts[torch.searchsorted(starts, pos, right=True) - 1].int()
        f = torch.where(torch.rand((T, b), generator=g) < 0.02, f + 200, f)
        kw["first_key"], ref["first"] = f.to(dev), f
    news = [min(T, L) for L in lens]
    if kind == "all":
        news[-1] = T // 2
    out, lse = randn(dev, dtype, T, b, hq, d, seed=8), randn(dev, "f32", T, b, hq, seed=9)
    before = out.clone(), lse.clone()
    call = lambda o, l: cache.attend(q, o, l, n_new=ints(dev, news), window=window, sinks=sinks,  # noqa: E731
                                     **kw)
    call(out, lse)
    many = dtype == "bf16"
    C.check_attend(out, lse, q, K, V, lens, news, before=before, window=window, sinks=sinks,
                   coarse_cap=many, one_term=many, **ref)
    again = call(before[0].clone(), before[1].clone())
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)


def check_odd(out, lse, q, K, V, lens, T, window, sinks, one_term):
    """NaN among keys and values: a query that sees one among the keys is NaN, one that sees it
    among the values is NaN in that coordinate, and nothing else is."""
    hq, dev = q.shape[2], q.device
    G = hq // K.shape[1]
    hits = 0
    for i, L in enumerate(lens):
        n = min(T, L)
        pos, see = (t.to(dev) for t in C.visible(L, n, None, 0, window, sinks))
        for m in range(hq):
            k, v = K[i, m // G, :L], V[i, m // G, :L]
            lost = (see.double() @ torch.isnan(k).any(-1).double()) > 0
            hit = ((see.double() @ torch.isnan(v).double()) > 0) | lost[:, None]
            assert torch.equal(torch.isnan(out[:n, i, m]), hit), (i, m)
            assert torch.equal(torch.isnan(lse[:n, i, m]), lost), (i, m)
            ref, rl, tol, lt = C.attention(q[:n, i, m], torch.nan_to_num(k), torch.nan_to_num(v),
                                           pos, see, one_term=one_term)
            err = (out[:n, i, m].double() - ref).abs()
            assert bool((err <= tol)[~hit].all()), (i, m)
            assert bool(((lse[:n, i, m].double() - rl).abs() <= lt)[~lost].all()), (i, m)
            hits += int(hit.any(-1).sum()) - int(lost.sum())
    return hits


@pytest.mark.parametrize("keys", [False, True])
@pytest.mark.parametrize("sinks", [0, 5])
@pytest.mark.parametrize("name", ["split", "split_d64", "whole_d64", "short_window", "f32"])
def test_nan_in_tiles_of_128(dev, name, sinks, keys):
    """NaN that all queries, some, one or none see: in the sinks, before every window, inside
    windows and at the last token."""
    dtype, d, hkv, group, lens, cap, T, window, _, paged = TILES[name]
    assert cache8_rule.plan(dtype, len(lens), hkv, group, cap, T, window, sinks).tiles
    L = lens[0]
    nan = [("v", 0, 2, 0, 7), ("v", 0, 2, 1, 0), ("v", 0, L - T + 40, 0, d - 1),
           ("v", 0, L - 60, 2, 33), ("v", 0, L - 1, 1, 5), ("v", len(lens) - 1, lens[-1] // 2, 3, 9)]
    if L - T - window > 8:
        nan += [("v", 0, 6, 0, c) for c in range(d)]
    if keys:
        nan += [("k", 0, L - T // 2, 1, 3), ("k", 0, L - 1, 2, 4)]
    cache, K, V = filled(dev, dtype, lens, hkv * group, hkv, d, cap, paged, nan=nan)
    assert int(torch.isnan(V).sum()) == len([x for x in nan if x[0] == "v"])
    q = randn(dev, dtype, T, len(lens), hkv * group, d, seed=3)
    news = [min(T, x) for x in lens]
    out, lse = cache.attend(q, n_new=ints(dev, news), window=window, sinks=sinks)
    assert check_odd(out, lse, q, K, V, lens, T, window, sinks, dtype == "bf16") > 0


@pytest.mark.parametrize("dtype,T,cap", [("bf16", 1, 512), ("bf16", 16, 512), ("bf16", 60, 512),
                                         ("bf16", 150, 65536), ("f32", 3, 512),
                                         ("f32", 150, 65536)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (31, 4), (33, 200), (64, 1), (299, 4), (90, 2)])
def test_windows_in_tiles_of_16(dev, dtype, T, cap, window, sinks):
    """Windows of a large cache keep a call in tiles of 16 rows, whose weights have 16 bits."""
    lens = [300, 31, 150]
    p = cache8_rule.plan(dtype, 3, 2, 2, cap, T, window, sinks)
    assert p.rows == 16 and (cap == 512 or cache8_rule.plan(dtype, 3, 2, 2, 8 * cap, T).tiles)
    cache, K, V = filled(dev, dtype, lens, 4, 2, 128, cap, True)
    q = randn(dev, dtype, T, 3, 4, 128, seed=2, scale=2.0)
    news = [min(T, L) for L in lens]
    for kw in ({}, dict(softcap=7.0)):
        out, lse = cache.attend(q, n_new=ints(dev, news), window=window, sinks=sinks, **kw)
        C.check_attend(out, lse, q, K, V, lens, news, window=window, sinks=sinks, **kw)


@pytest.mark.parametrize("T,sinks", [(1, 5), (1, 0), (40, 5), (200, 5)])
def test_nan_in_tiles_of_16(dev, T, sinks):
    lens, window = [700, 120], 90
    assert cache8_rule.plan("bf16", 2, 4, 4, 1024, T, window, sinks).rows == 16
    nan = [("v", 0, 2, 0, 7), ("v", 0, 640, 1, 5), ("v", 0, 699, 2, 33), ("k", 0, 699, 3, 1),
           ("v", 1, 100, 0, 2)] + [("v", 0, 300, 0, c) for c in range(64)]
    cache, K, V = filled(dev, "bf16", lens, 16, 4, 64, 1024, True, nan=nan)
    q = randn(dev, "bf16", T, 2, 16, 64, seed=3)
    out, lse = cache.attend(q, n_new=ints(dev, [min(T, L) for L in lens]), window=window,
                            sinks=sinks)
    assert check_odd(out, lse, q, K, V, lens, T, window, sinks, False) > 0


# dtype, d, batch, hkv, group, T, longest, cap, window, sinks
SHARED = [("bf16", 128, 16, 8, 2, 1, 20000, 65536, 9000, 4),
          ("bf16", 64, 4, 8, 4, 4, 30000, 65536, 33000, 100),
          ("bf16", 128, 16, 2, 16, 1, 40000, 131072, 33000, 1),
          ("f32", 64, 5, 4, 1, 7, 50000, 262144, 52000, 4),
          ("f32", 64, 24, 4, 2, 2, 20000, 65536, 11000, 0),
          ("bf16", 64, 40, 1, 4, 9, 30000, 65536, 14000, 300),
          ("bf16", 128, 2, 4, 5, 12, 45000, 131072, 44000, 33)]


@pytest.mark.parametrize("dtype,d,b,hkv,group,T,top,cap,window,sinks", SHARED)
def test_windows_of_shared_workgroups(dev, dtype, d, b, hkv, group, T, top, cap, window, sinks):
    """Long windows of batches, some sequences within them and some past them: workgroups are
    shared by the lengths that the windows leave."""
    assert cache8_rule.plan(dtype, b, hkv, group, cap, T, window, sinks).shares > 0
    g = torch.Generator().manual_seed(b)
    lens = [int(x) for x in torch.randint(0, top // 6, (b,), generator=g)]
    lens[0], lens[-1] = top, min(lens[-1], 1)
    if b > 4:
        lens[b // 2], lens[1] = top, window // 2
    hq = hkv * group
    pages = sum(-(-L // 64) for L in lens) + 1  # as many as the sequences need
    table = torch.zeros((b, cap // 64), dtype=torch.int32)
    order, at = torch.randperm(pages, generator=g).int(), 0
    for i, L in enumerate(lens):
        n = -(-L // 64)
        table[i, :n] = order[at:at + n]
        at += n
    cache = spla.SplaCache8(spla.make_config(b, hq, hkv, d, 64, 8, cap, dtype, kv_pages=pages), dev,
                            block_table=table.to(dev))
    k, v = (randn(dev, dtype, top, b, hkv, d, seed=s) for s in (1, 2))
    cache.append(k, v, ints(dev, lens))
    del k, v
    K, V = (x.permute(1, 2, 0, 3) for x in cache.read(top))
    q = randn(dev, dtype, T, b, hq, d, seed=3, scale=2.0)
    news = [min(T, L) for L in lens]
    out, lse = randn(dev, dtype, T, b, hq, d, seed=8), randn(dev, "f32", T, b, hq, seed=9)
    before = out.clone(), lse.clone()
    kw = dict(n_new=ints(dev, news), window=window, sinks=sinks)
    cache.attend(q, out, lse, **kw)
    for i in range(b):  # (one sequence in 64 bits at a time)
        keep = before[0][:, i:i + 1], before[1][:, i:i + 1]
        C.check_attend(out[:, i:i + 1], lse[:, i:i + 1], q[:, i:i + 1], K[i:i + 1].double(),
                       V[i:i + 1].double(), lens[i:i + 1], news[i:i + 1], before=keep,
                       window=window, sinks=sinks)
    again = cache.attend(q, before[0].clone(), before[1].clone(), **kw)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)


def test_captured_windows_of_tiles(dev):
    """Windowed prompts of tiles of 128 rows, split and not, in two graphs that share a workspace,
    between eager calls."""
    dtype, d, hkv, group, lens, cap, T, window, sinks, paged = TILES["split"]
    cache, _, _ = filled(dev, dtype, lens, hkv * group, hkv, d, cap, paged)
    q, q2 = (randn(dev, dtype, t, 2, hkv * group, d, seed=5) for t in (T, 2 * T))
    assert cache8_rule.plan(dtype, 2, hkv, group, cap, 2 * T, window).tiles
    outs = [torch.empty_like(q), torch.empty_like(q2)]
    cache.attend(q2, window=window)
    cache.attend(q, window=window)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    with torch.cuda.graph(graphs[0]):
        cache.attend(q, outs[0], window=window, sinks=sinks)
    with torch.cuda.graph(graphs[1]):
        cache.attend(q2, outs[1], window=window)
    for i in range(4):
        q.copy_(randn(dev, dtype, *q.shape, seed=30 + i))
        q2.copy_(randn(dev, dtype, *q2.shape, seed=40 + i))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], cache.attend(q, window=window, sinks=sinks)[0])
        assert torch.equal(outs[1], cache.attend(q2, window=window)[0])
