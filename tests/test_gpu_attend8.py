"""Exact attention over the 8-bit cache on the GPU against the 64-bit form."""

import math

import pytest
import torch

import cache8_ref as C
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
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=dev) * scale).to(DT[dtype])


def ints(dev, v):
    return torch.tensor(v, dtype=torch.int32, device=dev)


def filled(dev, dtype, lens, hq, hkv, d, B, cap=None, paged=False, seed=1, garbage=False, **kw):
    """A cache of sequences of `lens` tokens and the values it holds (fp64); garbage: buffers full
    of NaN codes."""
    b, top = len(lens), max(max(lens), 1)
    cap = cap or -(-top // B) * B
    table, pages = None, 0
    if paged:
        pages = b * (cap // B) + 3
        table = torch.randperm(pages, generator=torch.Generator().manual_seed(seed))
        table = table[:b * (cap // B)].view(b, -1).int().to(dev)
    cfg = spla.make_config(b, hq, hkv, d, B, 8, cap, dtype, kv_pages=pages, **kw)
    cache = spla.SplaCache8(cfg, dev, block_table=table)
    if garbage:
        cache.k.fill_(0x7F)
        cache.v.fill_(0xFF)
        cache.scales.fill_(2.0 ** 100)
    k, v = (randn(dev, dtype, top, b, hkv, d, seed=seed + s) for s in (10, 20))
    cache.append(k, v, ints(dev, lens))
    # (what the cache holds is tested by itself)
    K, V = (x.double().permute(1, 2, 0, 3).contiguous() for x in cache.read(top))
    return cache, K, V


CASES = {
    # name: dtype, d, hq, hkv, B, lens, T, paged
    "one_token": ("bf16", 128, 4, 1, 32, [1], 1, False),
    "step_g4": ("bf16", 128, 8, 2, 64, [333, 1, 64, 65, 0], 1, True),
    "step_g16_d64": ("bf16", 64, 16, 1, 128, [2000, 31], 1, False),
    "step_g5_long": ("bf16", 128, 10, 2, 64, [20011], 1, True),
    "few_tokens_g8": ("bf16", 128, 16, 2, 32, [700, 33, 2], 3, False),
    "rows_17": ("bf16", 64, 3, 3, 64, [500, 17], 17, True),
    "chunk_g1": ("bf16", 128, 2, 2, 64, [300, 129], 129, False),
    "chunk_g5": ("bf16", 128, 5, 1, 64, [1000, 255, 100], 100, True),
    "chunk_g6_d64": ("bf16", 64, 6, 1, 32, [770], 257, False),
    "chunk_g16": ("bf16", 128, 16, 1, 128, [400, 64], 33, True),
    "prompt": ("bf16", 128, 4, 1, 64, [1100], 1100, False),
    "prompt_d64": ("bf16", 64, 8, 2, 64, [515, 515], 515, True),
    "long_prefix": ("bf16", 128, 8, 1, 64, [9001, 4500], 65, False),
    "f32_step": ("f32", 64, 4, 2, 32, [257, 1, 0], 1, False),
    "f32_chunk": ("f32", 128, 6, 2, 64, [300, 90], 77, True),
    "f32_g16": ("f32", 64, 16, 1, 128, [640], 9, False),
    "f32_long": ("f32", 128, 1, 1, 64, [5000], 2, False),
    "splits": ("bf16", 128, 8, 2, 64, [3001, 0, 5, 129], 4, True),
    "splits_rows_48": ("bf16", 64, 8, 2, 32, [2500, 40], 12, False),
    "splits_rows_96": ("bf16", 128, 8, 2, 64, [6100, 300], 24, False),
    "f32_rows": ("f32", 64, 8, 2, 32, [1000, 333, 40], 50, True),
    "f32_rows_splits": ("f32", 128, 8, 2, 64, [2501, 0, 90], 25, False),
    "f32_splits": ("f32", 128, 4, 2, 64, [2800, 1, 70], 8, True),
}


def tile_cap(dtype, hkv, group, B, b, T):
    """A capacity at which a call of T tokens goes by tiles of 128 rows (they are chosen by the
    work that there may be)."""
    pairs = 32768 if dtype == "bf16" else 98304
    steps = pairs // (-(-T * group // 16) * b * hkv) + 1
    return -(-steps * 32 // B) * B


KINDS = ["causal", "softcap", "bias", "docs", "prefix", "ragged", "window", "window_sinks",
         "window_docs", "window_prefix", "window_softcap", "window_bias", "softcap_large", "all"]


MANY = [n for n, c in CASES.items() if c[6] * c[2] // c[3] > 64]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name,wide", [(n, False) for n in CASES] + [(n, True) for n in MANY])
def test_against_64_bits(dev, name, wide, kind):
    dtype, d, hq, hkv, B, lens, T, paged = CASES[name]
    b = len(lens)
    cap = tile_cap(dtype, hkv, hq // hkv, B, b, T) if wide else None
    if cap is not None:
        cap = max(cap, -(-max(lens) // B) * B)
    cache, K, V = filled(dev, dtype, lens, hq, hkv, d, B, cap, paged=paged, garbage=True)
    q = randn(dev, dtype, T, b, hq, d, seed=3, scale=2.0)
    kw, ref = {}, {}
    if kind in ("softcap", "window_softcap", "all"):
        kw["softcap"] = ref["softcap"] = 7.0
    if kind == "softcap_large":
        kw["softcap"] = ref["softcap"] = 200.0
    if kind in ("bias", "window_bias", "all"):
        kw["slopes"] = ref["slopes"] = torch.exp2(-torch.arange(1.0, hq + 1, device=dev) * 8 / hq)
    if kind in ("docs", "window_docs", "all"):
        g = torch.Generator().manual_seed(5)
        f = torch.randint(-3, max(lens) + 2, (T, b), generator=g).int()
        f = torch.where(torch.rand((T, b), generator=g) < 0.3, torch.zeros_like(f), f)
        kw["first_key"], ref["first"] = f.to(dev), f
    if kind in ("prefix", "window_prefix", "all"):
        pre = [max(0, L * 2 // 3 - 5) if i != 1 else L + 9 for i, L in enumerate(lens)]
        kw["prefix_len"], ref["prefix"] = ints(dev, pre), pre
    news = [min(T, L) for L in lens]
    if kind in ("ragged", "all"):
        news = [min(L, (T + i) // (i + 1)) for i, L in enumerate(lens)]
        news[-1] = min(lens[-1], T)
    if kind.startswith("window") or kind == "all":
        w, s = {"window": (1, 0), "window_sinks": (40, 4), "window_docs": (33, 3),
                "window_prefix": (100, 37), "window_softcap": (90, 2), "window_bias": (65, 6),
                "all": (70, 1)}[kind]
        kw |= dict(window=w, sinks=s)
        ref |= dict(window=w, sinks=s)
    kw["n_new"] = ints(dev, news)
    out = randn(dev, dtype, T, b, hq, d, seed=8)
    lse = randn(dev, "f32", T, b, hq, seed=9)
    before = (out.clone(), lse.clone())
    got = cache.attend(q, out, lse, **kw)
    assert got[0] is out and got[1] is lse
    many = dtype == "bf16" and wide
    C.check_attend(out, lse, q, K, V, lens, news, before=before, coarse_cap=many, one_term=many,
                   **ref)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (31, 4), (32, 32), (33, 200), (64, 1),
                                          (299, 4), (300, 0), (301, 7), (2 ** 31 - 1, 2 ** 31 - 1),
                                          (0, 9)])
@pytest.mark.parametrize("dtype,T,wide", [("bf16", 1, False), ("bf16", 16, False),
                                          ("bf16", 150, False), ("bf16", 150, True),
                                          ("f32", 3, False), ("f32", 150, True)])
def test_windows(dev, dtype, T, wide, window, sinks):
    """Windows that end at, before and after borders of steps, blocks and sequences; sinks that
    touch and pass the window."""
    lens = [300, 31, 150]
    cap = tile_cap(dtype, 2, 2, 32, 3, T) if wide else 512
    cache, K, V = filled(dev, dtype, lens, 4, 2, 128, 32, cap=cap, paged=True)
    q = randn(dev, dtype, T, 3, 4, 128, seed=2, scale=2.0)
    news = [min(T, L) for L in lens]
    out, lse = cache.attend(q, n_new=ints(dev, news), window=window, sinks=sinks)
    many = dtype == "bf16" and wide
    C.check_attend(out, lse, q, K, V, lens, news, window=window, sinks=sinks, coarse_cap=many,
                   one_term=many)


@pytest.mark.parametrize("dtype,T,wide", [("bf16", 1, False), ("bf16", 70, False),
                                          ("bf16", 70, True), ("f32", 3, False),
                                          ("f32", 60, False), ("f32", 60, True)])
def test_unseen_nan_stays_out(dev, dtype, T, wide):
    """NaN in keys and values that a query does not see leave it alone; in values that it sees they
    reach it, and only that coordinate."""
    B, d, L = 32, 64, 200
    cap = tile_cap(dtype, 2, 2, B, 1, T) if wide else 224
    cfg = spla.make_config(1, 4, 2, d, B, 8, cap, dtype)
    cache = spla.SplaCache8(cfg, dev)
    k, v = (randn(dev, dtype, L, 1, 2, d, seed=s) for s in (1, 2))
    k[20:40] = math.nan  # hidden by the window of every query
    v[25:45] = math.inf
    v[L - 1, 0, 0, 5] = math.nan  # seen by the last query alone
    cache.append(k, v)
    K, V = (x.double().permute(1, 2, 0, 3) for x in cache.read(L))
    q = randn(dev, dtype, T, 1, 4, d, seed=3)
    out, lse = cache.attend(q, window=60, sinks=4)
    hit = torch.isnan(out)
    assert bool(hit[T - 1, 0, :2, 5].all()) and int(hit.sum()) == 2
    assert not torch.isnan(lse).any()
    out = torch.where(hit, torch.zeros_like(out), out)
    Kz, Vz = torch.nan_to_num(K), torch.nan_to_num(V)
    ok = out.clone()
    ok[T - 1, 0, :2, 5] = 0.0
    many = dtype == "bf16" and wide
    # the last query's hit coordinate is taken from the reference itself
    pos, see = C.visible(L, T, None, 0, 60, 4)
    for m in range(4):
        ref, _, tol, _ = C.attention(q[:, 0, m], Kz[0, m // 2], Vz[0, m // 2], pos.to(dev),
                                     see.to(dev), one_term=many)
        err = (ok[:, 0, m].double() - ref).abs()
        if m < 2:
            err[T - 1, 5] = 0.0
        assert bool((err <= tol).all()), (m, float((err / tol).max()))


def test_extreme_values(dev):
    """Blocks of very large and very small numbers side by side."""
    k = randn(dev, "bf16", 256, 1, 1, 128, seed=1)
    v = randn(dev, "bf16", 256, 1, 1, 128, seed=2)
    v[:64] *= 2.0 ** 90
    v[64:128] *= 2.0 ** -90
    k[128:192] *= 2.0 ** -60
    for T, wide in ((1, False), (40, False), (40, True)):
        cap = tile_cap("bf16", 1, 4, 64, 1, T) if wide else 256
        cache = spla.SplaCache8(spla.make_config(1, 4, 1, 128, 64, 8, cap, "bf16"), dev)
        cache.append(k, v)
        K, V = (x.double().permute(1, 2, 0, 3) for x in cache.read(256))
        q = randn(dev, "bf16", T, 1, 4, 128, seed=3)
        out, lse = cache.attend(q)
        C.check_attend(out, lse, q, K, V, [256], one_term=wide, coarse_cap=wide)
        out, lse = cache.attend(q, window=100, sinks=2)
        C.check_attend(out, lse, q, K, V, [256], one_term=wide, coarse_cap=wide, window=100,
                       sinks=2)


@pytest.mark.parametrize("T,cap", [(1, 2048), (5, 2048), (90, 2048), (90, 65536)])
def test_captured_replays(dev, T, cap):
    """One graph with an append and an attention, replayed between eager calls of other sizes;
    two graphs share the cache's workspace."""
    lens = [700, 300]
    cache, _, _ = filled(dev, "bf16", lens, 8, 2, 128, 64, cap=cap, paged=True)
    q, q2 = (randn(dev, "bf16", t, 2, 8, 128, seed=5) for t in (T, 2 * T))
    k = randn(dev, "bf16", T, 2, 2, 128, seed=6)
    outs = [torch.empty_like(q), torch.empty_like(q2)]
    cache.attend(q2)
    cache.attend(q)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    with torch.cuda.graph(graphs[0]):
        cache.append(k, k)
        cache.attend(q, outs[0], window=256, sinks=4)
    with torch.cuda.graph(graphs[1]):
        cache.attend(q2, outs[1])
    for i in range(4):
        q.copy_(randn(dev, "bf16", T, 2, 8, 128, seed=30 + i))
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], cache.attend(q, window=256, sinks=4)[0])
        assert torch.equal(outs[1], cache.attend(q2)[0])
    assert cache.seq_lens.tolist() == [L + 4 * T for L in lens]


@pytest.mark.parametrize("cap", [None, 65536])
def test_repeats_bit_for_bit(dev, cap):
    cache, _, _ = filled(dev, "bf16", [5000, 1234], 8, 2, 128, 64, cap)
    for T in (1, 9, 200):
        q = randn(dev, "bf16", T, 2, 8, 128, seed=5)
        a, la = cache.attend(q, window=2000, sinks=4)
        for _ in range(3):
            o, l = cache.attend(q, window=2000, sinks=4)
            assert torch.equal(a, o) and torch.equal(la, l)


def test_window_counts_are_refused(dev):
    cache, _, _ = filled(dev, "bf16", [40], 2, 1, 64, 32)
    q = randn(dev, "bf16", 1, 1, 2, 64)
    for window, sinks in ((-1, 0), (4, -1), (2 ** 31, 0), (2 ** 32 + 4, 0), (4, 2 ** 32)):
        with pytest.raises(ValueError):
            cache.attend(q, window=window, sinks=sinks)


def test_other_stream(dev):
    cache, K, V = filled(dev, "bf16", [900], 8, 2, 128, 64)
    q = randn(dev, "bf16", 1, 1, 8, 128, seed=5)
    ref, _ = cache.attend(q)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        out, _ = cache.attend(q)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(out, ref)


def test_served_sequence(dev):
    """Prompts, chunks and single tokens of a dense layer, from the projection's rows on: norms
    and rotation in one pass, the quantising append, attention with a window and sinks; then the
    prefix handed to a 16-bit cache."""
    import rope_attend_ref as R
    b, hq, hkv, d, B, cap = 2, 8, 2, 128, 64, 512
    nb = cap // B
    table = torch.randperm(b * nb, generator=torch.Generator().manual_seed(2)).view(b, nb).int()
    cfg = spla.make_config(b, hq, hkv, d, B, 8, cap, "bf16", kv_pages=b * nb)
    cache = spla.SplaCache8(cfg, dev, block_table=table.to(dev))
    rope = spla.make_rope(d, base=10000.0)
    w = R.frequencies(d)
    wq, wk = (1.0 + 0.2 * randn(dev, "f32", d, seed=s) for s in (50, 51))
    K, V = C.Held(b, hkv, d, B, cap), C.Held(b, hkv, d, B, cap)
    for i, n in enumerate([[150, 100], [33, 40], [1, 1], [1, 1], [1, 0], [64, 3]]):
        T = max(n)
        x = randn(dev, "bf16", T, b, (hq + 2 * hkv) * d, seed=60 + i, scale=1.5)
        q = x[..., :hq * d].view(T, b, hq, d)
        k = x[..., hq * d:(hq + hkv) * d].view(T, b, hkv, d)
        v = x[..., (hq + hkv) * d:].view(T, b, hkv, d)
        start = list(K.lens)
        pos = torch.arange(T)[:, None] + torch.tensor(start)
        qr, kr = cache.norm_rotate(rope, q, k, wq, wk)
        for got, rows, weight in ((qr, q, wq), (kr, k, wk)):
            ref = C.norm_rotate(rows, weight, 1e-6, pos[..., None].to(dev), w)
            # (fp32 steps of a pair's size, see test_gpu_norm_rotate.tolerance)
            tol = 1.001 * 2.0 ** -8 * ref.abs() + 2.0 ** -19 * ref.abs().amax(-1, keepdim=True)
            assert bool(((got.double() - ref).abs() <= tol).all())
        cache.append(kr, v, ints(dev, n))
        K.append(kr.cpu(), n, start)
        V.append(v.cpu(), n, start)
        for window, sinks in ((0, 0), (48, 4)):
            out, lse = cache.attend(qr, n_new=ints(dev, n), window=window, sinks=sinks)
            C.check_attend(out, lse, qr, K.x, V.x, K.lens, n, window=window, sinks=sinks)
    # handed on: a 16-bit cache that attends alike
    k, v = cache.read(max(K.lens))
    cfg16 = spla.make_config(b, hq, hkv, d, B, 8, cap, "bf16")
    other = spla.SplaCache(cfg16, dev)
    other.append(k.permute(1, 2, 0, 3).contiguous(), v.permute(1, 2, 0, 3).contiguous(),
                 cache.seq_lens)
    q = randn(dev, "bf16", b, hq, d, seed=90)
    out8, lse8 = cache.attend(q)
    C.check_attend(out8[None], lse8[None], q[None], K.x, V.x, K.lens)
    out16, lse16 = other.attend(q)
    C.check_attend(out16[None], lse16[None], q[None], K.x, V.x, K.lens)


def test_tile_rule_is_the_librarys(dev):
    """The capacities that tile_cap gives do reach the tiles of 128 rows: their workspaces have
    room for records of 128 rows."""
    for dtype, T in (("bf16", 70), ("f32", 60)):
        cap = tile_cap(dtype, 2, 2, 32, 1, T)
        small, large = (spla.attend8_workspace_bytes(
            spla.make_config(1, 4, 2, 64, 32, 8, c, dtype), T) for c in (cap - 64, cap))
        rows = 128 * -(-T * 2 // 128) * 2  # of the call
        split = min(128, 768 // (rows // 128), cap // 512)
        assert large >= rows * split * 66 * 4 and large != small


@pytest.mark.parametrize("T,group,window", [(1, 4, 300), (17, 4, 128), (40, 2, 2000)])
def test_windows_of_long_caches(dev, T, group, window):
    """A cache with room for much more than the window: splits and tiles by the window, after
    and before calls without one in the same workspace."""
    lens = [3000, 700]
    cache, K, V = filled(dev, "bf16", lens, 2 * group, 2, 128, 64, cap=262144)
    q = randn(dev, "bf16", T, 2, 2 * group, 128, seed=2, scale=2.0)
    many = T * group > 64
    for _ in range(2):
        out, lse = cache.attend(q, window=window, sinks=4)
        C.check_attend(out, lse, q, K, V, lens, window=window, sinks=4, one_term=many)
        out, lse = cache.attend(q)
        C.check_attend(out, lse, q, K, V, lens, one_term=many)
        out, lse = cache.attend(q, window=window, prefix_len=ints(dev, [2500, 0]))
        C.check_attend(out, lse, q, K, V, lens, window=window, prefix=[2500, 0], one_term=many)


@pytest.mark.parametrize("kind", ["causal", "window", "docs", "ragged"])
@pytest.mark.parametrize("dtype,d,b,hkv,group,T,top,cap", [
    ("bf16", 128, 16, 8, 2, 1, 8192, 8192), ("bf16", 64, 4, 8, 4, 4, 9000, 65536),
    ("bf16", 128, 16, 2, 16, 1, 12000, 32768), ("f32", 64, 5, 4, 1, 7, 3000, 106496),
    ("bf16", 64, 40, 1, 4, 9, 2000, 32768), ("bf16", 128, 2, 4, 5, 12, 2500, 32768)])
def test_shared_lengths(dev, dtype, d, b, hkv, group, T, top, cap, kind):
    """Batches whose long sequences take more workgroups than their short ones."""
    g = torch.Generator().manual_seed(b)
    lens = [int(x) for x in torch.randint(0, top // 8, (b,), generator=g)]
    lens[0], lens[-1], lens[b // 2] = top, min(lens[-1], 1), top if b > 4 else lens[b // 2]
    cfg = spla.make_config(b, hkv * group, hkv, d, 64, 8, cap, dtype)
    # the workspace has room for 512 shares: counters, a record of 16 rows for each
    assert spla.attend8_workspace_bytes(cfg, T) >= 768 * 128 + 512 * 16 * (d + 2) * 4
    cache, K, V = filled(dev, dtype, lens, hkv * group, hkv, d, 64, cap)
    q = randn(dev, dtype, T, b, hkv * group, d, seed=3, scale=2.0)
    news = [min(T, L) for L in lens]
    kw, ref = {}, {}
    if kind == "window":
        kw = ref = dict(window=700, sinks=4)
    if kind == "docs":
        f = torch.randint(0, top, (T, b), generator=g).int()
        kw, ref = dict(first_key=f.to(dev)), dict(first=f)
    if kind == "ragged":
        news = [min(L, i % (T + 1)) for i, L in enumerate(lens)]
    out = randn(dev, dtype, T, b, hkv * group, d, seed=8)
    lse = randn(dev, "f32", T, b, hkv * group, seed=9)
    before = (out.clone(), lse.clone())
    cache.attend(q, out, lse, n_new=ints(dev, news), **kw)
    C.check_attend(out, lse, q, K, V, lens, news, before=before, **ref)
    again = cache.attend(q, before[0].clone(), before[1].clone(), n_new=ints(dev, news), **kw)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)
