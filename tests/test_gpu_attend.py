"""Exact attention over the cache on the GPU against the 64-bit form."""

import ctypes

import numpy as np
import pytest
import torch

import rope_attend_ref as R
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


def filled(dev, dtype, lens, hq, hkv, d, B, cap=None, paged=False, seed=1, garbage=False, **kw):
    """A cache of sequences of `lens` tokens and its rows; garbage: buffers that held NaN."""
    b, top = len(lens), max(max(lens), 1)
    cap = cap or -(-top // B) * B
    table, pages = None, 0
    if paged:
        pages = b * (cap // B) + 3
        table = torch.randperm(pages, generator=torch.Generator().manual_seed(seed))
        table = table[:b * (cap // B)].view(b, -1).int().to(dev)
    cfg = spla.make_config(b, hq, hkv, d, B, 8, cap, dtype, kv_pages=pages, **kw)
    cache = spla.SplaCache(cfg, dev, block_table=table)
    if garbage:
        cache.k.fill_(float("nan"))
        cache.v.fill_(float("nan"))
    K, V = (randn(dev, dtype, b, hkv, top, d, seed=seed + s) for s in (10, 20))
    cache.append(K, V, torch.tensor(lens, dtype=torch.int32, device=dev))
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
    # keys in many splits, joined by a launch of their own; short sequences beside a long one
    "splits": ("bf16", 128, 8, 2, 64, [3001, 0, 5, 129], 4, True),
    "splits_rows_48": ("bf16", 64, 8, 2, 32, [2500, 40], 12, False),
    "splits_rows_96": ("bf16", 128, 8, 2, 64, [6100, 300], 24, False),
    "f32_rows": ("f32", 64, 8, 2, 32, [1000, 333, 40], 50, True),
    "f32_rows_splits": ("f32", 128, 8, 2, 64, [2501, 0, 90], 25, False),
    "f32_splits": ("f32", 128, 4, 2, 64, [2800, 1, 70], 8, True),
}
KINDS = ["causal", "softcap", "bias", "docs", "prefix", "ragged", "all"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", list(CASES))
def test_attend(dev, name, kind):
    dtype, d, hq, hkv, B, lens, T, paged = CASES[name]
    b = len(lens)
    cache, K, V = filled(dev, dtype, lens, hq, hkv, d, B, cap=-(-(max(lens) + 70) // B) * B,
                         paged=paged, garbage=kind != "causal")
    q = randn(dev, dtype, T, b, hq, d, seed=5, scale=1.5)
    rng = np.random.default_rng(list(CASES).index(name))
    kw, ref = {}, {}
    if kind in ("softcap", "all"):
        kw["softcap"] = ref["softcap"] = 5.0
    if kind in ("bias", "all"):
        ref["slopes"] = kw["slopes"] = torch.exp2(-8.0 * torch.arange(1, hq + 1, device=dev) / hq)
    if kind in ("docs", "all"):
        # documents, and queries that see nothing (first key past their own position)
        first = np.zeros((T, b), np.int32)
        for i, L in enumerate(lens):
            cuts = np.sort(np.append(rng.integers(0, max(L, 1), 5), 0))
            p = np.maximum(np.arange(L - T, L), 0)
            first[:, i] = cuts[np.searchsorted(cuts, p, side="right") - 1]
            first[rng.integers(0, T), i] = rng.choice([L, 1 << 30, max(L - 1, 0)])
        first[0, 0] = -5
        ref["first"] = kw["first_key"] = torch.from_numpy(first).to(dev)
    if kind in ("prefix", "all"):
        ref["prefix"] = [int(x) for x in rng.integers(0, max(lens) + 2, b)]
        kw["prefix_len"] = torch.tensor(ref["prefix"], dtype=torch.int32, device=dev)
    news = None
    if kind in ("ragged", "all"):  # counts past the chunk and below zero are clamped
        news = [int(x) for x in rng.integers(0, T + 1, b)]
        news[0] = T + 3
        if b > 1:
            news[-1] = -1
        kw["n_new"] = torch.tensor(news, dtype=torch.int32, device=dev)
    out, lse = randn(dev, dtype, T, b, hq, d, seed=7), torch.randn(T, b, hq, device=dev)
    before = (out.clone(), lse.clone())
    cache.attend(q, out, lse, **kw)
    torch.cuda.synchronize()
    R.check_attend(out, lse, q, K, V, lens, news, before=before, **ref)
    again, lse2 = cache.attend(q, before[0].clone(), before[1].clone(), **kw)
    assert torch.equal(again, out) and torch.equal(lse2, lse)


def test_scale_and_three_dimensions(dev):
    cache, K, V = filled(dev, "bf16", [200, 90], 8, 2, 128, 64, softmax_scale=0.3)
    q = randn(dev, "bf16", 2, 8, 128)
    out, lse = cache.attend(q)
    assert out.shape == (2, 8, 128) and lse.shape == (2, 8)
    R.check_attend(out[None], lse[None], q[None], K, V, [200, 90], scale=0.3)


@pytest.mark.parametrize("softcap", [2.0 ** -10, 41.0, 42.0, 1024.0])
@pytest.mark.parametrize("dtype,T", [("bf16", 9), ("bf16", 100), ("f32", 9), ("f32", 40)])
def test_caps(dev, dtype, T, softcap):
    """The smallest and the largest cap, and those on the two sides of the one up to which
    weights need no maximum; scores up to a few hundred."""
    cache, K, V = filled(dev, dtype, [400, 333], 8, 2, 128, 64)
    q = randn(dev, dtype, T, 2, 8, 128, seed=3, scale=30.0)
    for slopes in (None, torch.linspace(0.0, 1.0, 8, device=dev)):
        out, lse = cache.attend(q, softcap=softcap, slopes=slopes)
        R.check_attend(out, lse, q, K, V, [400, 333], softcap=softcap, slopes=slopes,
                       cap_series=dtype == "f32" or T * 4 <= 64)


@pytest.mark.parametrize("size", [2.0 ** 70, 2.0 ** -30])
@pytest.mark.parametrize("softcap", [0.0, 41.0, 42.0])
@pytest.mark.parametrize("dtype,T", [("bf16", 9), ("bf16", 100), ("f32", 9), ("f32", 40)])
def test_large_and_small_values(dev, dtype, T, softcap, size):
    """Queries against the keys' mean direction: scores at both ends of the cap."""
    cache, K, V = filled(dev, dtype, [400, 333], 8, 2, 128, 64)
    cache.reset()
    K, V = K + 2.0, V * size
    cache.append(K, V, torch.tensor([400, 333], dtype=torch.int32, device=dev))
    q = randn(dev, dtype, T, 2, 8, 128, seed=3)
    q[:, :, ::2] = 1.0
    q[:, :, 1::2] = -1.0
    out, lse = cache.attend(q, softcap=softcap)
    R.check_attend(out, lse, q, K, V, [400, 333], softcap=softcap,
                   cap_series=dtype == "f32" or T * 4 <= 64)


@pytest.mark.parametrize("dtype,T", [("bf16", 12), ("bf16", 70), ("f32", 30)])
def test_more_queries_than_tokens_and_first_keys_outside(dev, dtype, T):
    lens = [5, 40, 0, 700]
    cache, K, V = filled(dev, dtype, lens, 4, 1, 64, 32)
    q = randn(dev, dtype, T, 4, 4, 64, seed=5)
    for pre in (None, [4, 0, 3, 900]):
        dev_pre = None if pre is None else torch.tensor(pre, dtype=torch.int32, device=dev)
        out, lse = cache.attend(q, prefix_len=dev_pre)
        R.check_attend(out, lse, q, K, V, lens, prefix=pre)
    g = torch.Generator().manual_seed(T)
    first = torch.randint(-50, 750, (T, 4), generator=g).int().to(dev)
    first[0, 0], first[1, 0] = -(1 << 31), (1 << 31) - 1
    out, lse = cache.attend(q, first_key=first)
    R.check_attend(out, lse, q, K, V, lens, first=first)


@pytest.mark.parametrize("T", [1, 30])
def test_sequences_that_share_pages(dev, T):
    cache, K, V = filled(dev, "bf16", [300, 192], 4, 1, 128, 64, paged=True)
    cache.block_table[1, :3] = cache.block_table[0, :3]
    K[1, :, :192], V[1, :, :192] = K[0, :, :192], V[0, :, :192]
    q = randn(dev, "bf16", T, 2, 4, 128, seed=6)
    out, lse = cache.attend(q)
    R.check_attend(out, lse, q, K, V, [300, 192])


@pytest.mark.parametrize("dtype,T", [("bf16", 40), ("bf16", 2), ("bf16", 300), ("f32", 40)])
def test_what_a_query_does_not_see_does_not_matter(dev, dtype, T):
    """Infinities and NaN in keys and values behind a query's own position, or in another
    document, leave its result as it was; queries that see them get what the formula gives."""
    L = 611
    cache, K, V = filled(dev, dtype, [L], 4, 2, 128, 64)
    q = randn(dev, dtype, T, 1, 4, 128, seed=3)
    clean, clean_lse = cache.attend(q)
    first = torch.zeros(T, 1, dtype=torch.int32, device=dev)
    first[1:] = 100  # all but the first query: the document from token 100 on
    doc, doc_lse = cache.attend(q, first_key=first)
    bad = V.clone()
    bad[0, 0, 50, 3], bad[0, 1, 51, 70] = float("inf"), float("nan")
    bad[0, 1, L - 1, 5], bad[0, 1, L - 1, 6] = float("-inf"), float("nan")
    worse = K.clone()
    worse[0, :, 20] = float("nan")
    worse[0, 0, L - 1, 9] = float("inf") * q[T - 1, 0, 0, 9].sign()  # head 0's score: + infinity
    cache.reset()
    cache.append(worse, bad)
    out, lse = cache.attend(q, first_key=first)
    torch.cuda.synchronize()
    # neither the first document nor the last token
    assert torch.equal(out[1:T - 1], doc[1:T - 1]) and torch.equal(lse[1:T - 1], doc_lse[1:T - 1])
    assert bool(torch.isnan(out[0]).all()) and bool(torch.isnan(lse[0]).all())  # NaN key seen
    assert bool(torch.isnan(out[T - 1, 0, 0]).all())  # an infinite score: inf - inf
    # the last token's values alone (finite keys)
    cache.reset()
    cache.append(K, bad)
    out, lse = cache.attend(q, first_key=first)
    last, keep = out[T - 1, 0], doc[T - 1, 0]
    assert bool((last[2:, 5] == float("-inf")).all()) and bool(torch.isnan(last[2:, 6]).all())
    rest = [c for c in range(128) if c not in (5, 6)]
    assert torch.equal(last[:, rest], keep[:, rest]) and torch.equal(lse, doc_lse)
    assert bool((out[0, 0, :2, 3] == float("inf")).all())
    assert bool(torch.isnan(out[0, 0, 2:, 70]).all())
    assert torch.equal(clean_lse[0], lse[0])


def test_offsets_past_32_bits(dev):
    """Pages beyond 2^32 elements of the pool, and a contiguous cache as long."""
    B, d = 128, 128
    pages = (1 << 32) // (B * d) + 40
    cfg = spla.make_config(2, 4, 1, d, B, 8, 512, "bf16", kv_pages=pages)
    table = torch.tensor([[pages - 1, 5, pages - 7, 0], [3, pages - 2, pages - 30, 9]],
                         dtype=torch.int32, device=dev)
    cache = spla.SplaCache(cfg, dev, block_table=table)
    lens = [500, 259]
    K, V = (randn(dev, "bf16", 2, 1, 500, d, seed=s) for s in (1, 2))
    rope = spla.make_rope(d)
    n = torch.tensor(lens, dtype=torch.int32, device=dev)
    _, kr = spla.rotate(cfg, rope, k=K.permute(2, 0, 1, 3).contiguous())
    cache.append_rope(rope, K, V, n)
    assert cache.device_errors() == 0
    kr = kr.permute(1, 2, 0, 3).contiguous()
    for T in (1, 50, 300):
        q = randn(dev, "bf16", T, 2, 4, d, seed=T)
        out, lse = cache.attend(q)
        R.check_attend(out, lse, q, kr, V, lens)
    del cache
    torch.cuda.empty_cache()
    # the last sequence of a contiguous cache starts at element 2^32
    cfg = spla.make_config(9, 1, 1, d, B, 8, 1 << 22, "bf16")
    cache = spla.SplaCache(cfg, dev)
    K, V = (randn(dev, "bf16", 9, 1, 200, d, seed=s) for s in (3, 4))
    cache.append(K, V)
    for T in (1, 130):
        q = randn(dev, "bf16", T, 9, 1, d, seed=T)
        out, lse = cache.attend(q)
        R.check_attend(out, lse, q, K, V, [200] * 9)


def test_a_page_out_of_range_reads_inside_the_pool(dev):
    """As the decode, page 0 stands in for such an entry: other sequences are not touched."""
    cache, K, V = filled(dev, "bf16", [300, 200], 4, 1, 128, 64, paged=True)
    q = randn(dev, "bf16", 5, 2, 4, 128)
    out, lse = cache.attend(q)
    cache.block_table[0, 2] = 1 << 20
    cache.block_table[0, 3] = -1
    bad, bad_lse = cache.attend(q)
    assert torch.equal(bad[:, 1], out[:, 1]) and torch.equal(bad_lse[:, 1], lse[:, 1])


@pytest.mark.parametrize("T", [1, 30, 200])
def test_streams_and_graphs(dev, T):
    cache, K, V = filled(dev, "bf16", [700, 350], 8, 2, 128, 64, cap=2048)
    q = randn(dev, "bf16", T, 2, 8, 128)
    want, want_lse = cache.attend(q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        out, lse = cache.attend(q, torch.empty_like(q), torch.empty_like(want_lse))
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.attend(q, out, lse)
    # another graph on the same workspace, and eager calls of other sizes in between
    two = torch.cuda.CUDAGraph()
    out2, lse2 = torch.empty_like(q), torch.empty_like(lse)
    with torch.cuda.graph(two):
        cache.attend(q, out2, lse2, softcap=7.0)
    big = randn(dev, "bf16", 350, 2, 8, 128, seed=8)
    for i in range(4):
        q.copy_(randn(dev, "bf16", T, 2, 8, 128, seed=30 + i))
        cache.append(K[:, :, :7 + i].contiguous(), V[:, :, :7 + i].contiguous())
        graph.replay()
        two.replay()
        cache.attend(big)
        torch.cuda.synchronize()
        for got, lg, kw in ((out, lse, {}), (out2, lse2, dict(softcap=7.0))):
            want, want_lse = cache.attend(q, **kw)
            assert torch.equal(got, want) and torch.equal(lg, want_lse), i


def test_without_options_and_lse(dev):
    """The C call with NULL options and no log-sum-exp."""
    cache, K, V = filled(dev, "bf16", [500, 70], 8, 2, 128, 64)
    for T in (1, 20, 100):
        q = randn(dev, "bf16", T, 2, 8, 128, seed=T)
        want, _ = cache.attend(q)
        out = torch.empty_like(q)
        ws = torch.zeros(spla.attend_workspace_bytes(cache.cfg, T), dtype=torch.uint8, device=dev)
        assert spla.lib().spla_attend(
            ctypes.byref(cache.cfg), ctypes.byref(cache._struct), T, q.data_ptr(), None,
            out.data_ptr(), None, ws.data_ptr(), ws.numel(),
            torch.cuda.current_stream().cuda_stream) == 0
        assert torch.equal(out, want)


@pytest.mark.parametrize("T", [1, 4, 100])
def test_two_caches_on_two_streams(dev, T):
    """Calls in flight at once, each on its own cache and workspace."""
    caches = [filled(dev, "bf16", [3000, 900 + 64 * i], 8, 2, 128, 64, cap=4096, seed=i + 1)[0]
              for i in range(2)]
    qs = [randn(dev, "bf16", T, 2, 8, 128, seed=9 + i) for i in range(2)]
    want = [c.attend(q) for c, q in zip(caches, qs)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [(torch.empty_like(w[0]), torch.empty_like(w[1])) for w in want]
    torch.cuda.synchronize()
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                caches[i].attend(qs[i], *got[i])
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1])


@pytest.mark.parametrize("T", [12, 90])
def test_bias_with_a_prefix(dev, T):
    """Keys on both sides of the query, with steep slopes."""
    lens = [700, 130]
    cache, K, V = filled(dev, "bf16", lens, 8, 2, 128, 64)
    q = randn(dev, "bf16", T, 2, 8, 128, seed=2)
    slopes = torch.linspace(0.0, 2.0, 8, device=dev)
    for prefix in (None, [700, 100]):
        pre = None if prefix is None else torch.tensor(prefix, dtype=torch.int32, device=dev)
        out, lse = cache.attend(q, slopes=slopes, prefix_len=pre)
        R.check_attend(out, lse, q, K, V, lens, slopes=slopes, prefix=prefix)


@pytest.mark.parametrize("T", [1, 40])
def test_sliding_window_on_a_cache_with_selection_windows(dev, T):
    """Negative slopes too: scores that grow with the distance."""
    lens = [1500, 64]
    cache, K, V = filled(dev, "bf16", lens, 8, 2, 128, 64, sel_window=32, sel_stride=16)
    q = randn(dev, "bf16", T, 2, 8, 128, seed=2)
    pos = torch.tensor(lens) - T + torch.arange(T)[:, None]
    first = (pos - 127).int().to(dev)
    slopes = torch.linspace(-0.05, 0.05, 8, device=dev)
    out, lse = cache.attend(q, first_key=first, slopes=slopes)
    R.check_attend(out, lse, q, K, V, lens, first=first, slopes=slopes)


def test_served_sequence(dev):
    """The operators together, as a dense layer of a served model uses them: uneven prompt
    chunks, then steps, rotated by their positions, into a paged cache; every output against
    the whole sequence in 64 bits. The SPLA decode and prefill of the same rotated rows, while
    they still select every block, are the same attention."""
    b, hq, hkv, d, B = 2, 10, 2, 128, 64
    cfg = spla.make_config(b, hq, hkv, d, B, 16, 1024, "bf16", kv_pages=40)
    table = torch.randperm(40)[:32].view(2, 16).int().to(dev)
    cache = spla.SplaCache(cfg, dev, block_table=table)
    kw = dict(base=500000.0, scaling="parts", factor=4.0, orig_len=256.0, low=1.0, high=4.0)
    rope, w = spla.make_rope(d, 128, "half", **kw), R.frequencies(128, **kw)
    gamma = torch.ones(hq, d, device=dev)
    ks, vs, lens = [[], []], [[], []], [0, 0]
    for T, counts in ((300, [300, 211]), (129, [1, 129]), (1, [1, 1]), (1, [1, 1]), (2, [2, 1])):
        x = randn(dev, "bf16", T, b, (hq + 2 * hkv) * d, seed=T + counts[1])
        q, k, v = x.split([hq * d, hkv * d, hkv * d], -1)
        n = torch.tensor(counts, dtype=torch.int32, device=dev)
        qr, _ = cache.rotate(rope, q=q.view(T, b, hq, d))
        rows = [t.view(T, b, hkv, d).permute(1, 2, 0, 3).contiguous() for t in (k, v)]
        cache.append_rope(rope, *rows, n)
        out, lse = cache.attend(qr, n_new=n)
        for i in range(b):
            c = counts[i]
            pos = torch.arange(lens[i], lens[i] + c, device=dev)
            ks[i].append(R.turn(rows[0][i, :, :c], pos, w).float().to(torch.bfloat16))
            vs[i].append(rows[1][i, :, :c])
            lens[i] += c
            K, V = torch.cat(ks[i], 1), torch.cat(vs[i], 1)
            want = R.turn(q.view(T, b, hq, d)[:c, i], pos[:, None], w).float().to(torch.bfloat16)
            assert torch.equal(want, qr[:c, i])
            R.check_attend(out[:c, i:i + 1], lse[:c, i:i + 1], qr[:c, i:i + 1], K[None], V[None],
                           [lens[i]])
        if T == 1:  # all of the at most 9 blocks are selected: the decode is exact attention
            dec, _ = cache.decode(qr[0], gamma)
            diff = (dec.float() - out[0].float()).abs().amax(-1)
            # both round weights and result to bf16: 2^-8 of the largest value each, twice
            size = torch.cat([V.abs().amax().float().view(1) for V in
                              (torch.cat(x, 1) for x in vs)]).max()
            assert bool((diff <= 2 * 2 * 2.0 ** -8 * size).all())
    assert cache.seq_lens.cpu().tolist() == lens and cache.device_errors() == 0
