"""Rotary positions on the GPU against the 64-bit formula, and the append that
rotates on the way against an append of the rotated rows."""

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


def config(batch=2, hq=8, hkv=2, d=128, B=64, cap=1024, dtype="bf16", **kw):
    return spla.make_config(batch, hq, hkv, d, B, 8, cap, dtype, **kw)


def randn(dev, dtype, *shape, seed=0):
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device=dev).to(DT[dtype])


SHAPES = [  # dtype, d, rot, layout, T, batch, hq, hkv
    ("bf16", 128, 128, "half", 1, 1, 32, 8),
    ("bf16", 128, 128, "interleaved", 7, 3, 5, 1),
    ("bf16", 128, 64, "half", 300, 4, 8, 2),          # four rows per workgroup, part rotated
    ("bf16", 128, 96, "interleaved", 1031, 1, 4, 4),
    ("bf16", 128, 128, "half", 1100, 1, 32, 8),       # one row per workgroup, many rows
    ("bf16", 64, 64, "half", 33, 2, 16, 1),
    ("bf16", 64, 30, "half", 5, 2, 4, 2),             # pair by pair
    ("bf16", 64, 2, "interleaved", 9, 1, 3, 3),
    ("f32", 128, 128, "half", 6, 2, 4, 2),
    ("f32", 128, 126, "interleaved", 11, 2, 2, 2),
    ("f32", 64, 32, "half", 513, 3, 4, 1),
    ("f32", 64, 64, "interleaved", 1, 5, 1, 1),
]


@pytest.mark.parametrize("case", SHAPES, ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("transpose", [False, True])
def test_rotate(dev, case, transpose):
    dtype, d, rot, layout, T, b, hq, hkv = case
    cfg = config(b, hq, hkv, d, dtype=dtype)
    kw = dict(base=500000.0, scaling="parts", factor=4.0, orig_len=8192.0, low=1.0, high=4.0)
    rope = spla.make_rope(d, rot, layout, gain=1.25, **kw)
    w = R.frequencies(rot, **kw)
    q, k = randn(dev, dtype, T, b, hq, d, seed=1), randn(dev, dtype, T, b, hkv, d, seed=2)
    lens = torch.tensor([1000003 * (i + 1) // 3 for i in range(b)], dtype=torch.int32, device=dev)
    pos = torch.arange(T, device=dev)[:, None] + lens
    qo, ko = spla.rotate(cfg, rope, q, k, seq_lens=lens, transpose=transpose)
    for got, x in ((qo, q), (ko, k)):
        R.check_turned(got, x, pos[..., None], w, layout=layout, gain=1.25, transpose=transpose)
    # keys alone, in place, at positions given one by one
    pos = torch.randint(-(1 << 31), (1 << 31) - 1, (T, b), device=dev).int()
    pos[0, 0] = 0
    k2 = k.clone()
    none, got = spla.rotate(cfg, rope, k=k2, k_out=k2, positions=pos, transpose=transpose)
    assert none is None and got is k2
    R.check_turned(k2, k, pos[..., None], w, layout=layout, gain=1.25, transpose=transpose)


def test_more_rows_than_a_launch_holds(dev):
    """Over 2^22 workgroups and 2^31 elements, in place."""
    cfg, rope, w = config(1, 8, 8, 64), spla.make_rope(64, 22), R.frequencies(22)
    T = (1 << 22) + 5
    base = randn(dev, "bf16", 1009, 1, 8, 64, seed=4)
    x = base.repeat(-(-T // 1009), 1, 1, 1)[:T]
    spla.rotate(cfg, rope, q=x, q_out=x)
    t = torch.cat([torch.arange(0, 40), torch.arange((1 << 22) - 40, T)]).to(dev)
    R.check_turned(x[t], base[t % 1009], t[:, None, None], w)


def test_rotate_strided_rows(dev):
    """q and k as slices of one projection's rows, into rows of another width; nothing
    outside the rows is written, and 3-dimensional tensors are one position."""
    cfg, rope = config(3, 8, 2), spla.make_rope(128, 64)
    x = randn(dev, "bf16", 5, 3, 12 * 128)
    q, k = x[..., :1024].view(5, 3, 8, 128), x[..., 1024:1280].view(5, 3, 2, 128)
    wide = torch.full((5, 3, 16 * 128), 7.0, dtype=torch.bfloat16, device=dev)
    qo, ko = wide[..., 256:1280].view(5, 3, 8, 128), wide[..., 1280:1536].view(5, 3, 2, 128)
    pos = (torch.arange(15, device=dev) * 77).view(5, 3).int()
    spla.rotate(cfg, rope, q, k, positions=pos, q_out=qo, k_out=ko)
    w = R.frequencies(64)
    R.check_turned(qo, q, pos[..., None], w)
    R.check_turned(ko, k, pos[..., None], w)
    assert bool((wide[..., :256] == 7).all()) and bool((wide[..., 1536:] == 7).all())
    one, _ = spla.rotate(cfg, rope, q[2].contiguous(), positions=pos[2])
    assert one.shape == (3, 8, 128) and torch.equal(one, qo[2])
    empty, _ = spla.rotate(cfg, rope, q[:0])
    assert empty.shape == (0, 3, 8, 128)


@pytest.mark.parametrize("layout,rot", [("half", 64), ("interleaved", 22)])
def test_rotate_gradient(dev, layout, rot):
    """transpose=True is the gradient: against autograd of the 64-bit formula and against
    differences (exact for a linear map, up to the rounding of each fp32 result)."""
    cfg = config(2, 4, 2, 64, dtype="f32")
    rope = spla.make_rope(64, rot, layout, gain=0.7)
    w = R.frequencies(rot)
    x, g = randn(dev, "f32", 9, 2, 4, 64, seed=3), randn(dev, "f32", 9, 2, 4, 64, seed=4)
    pos = torch.arange(9, device=dev)[:, None].expand(9, 2).int().contiguous() * 1000
    dx, _ = spla.rotate(cfg, rope, g, positions=pos, transpose=True)
    leaf = x.double().requires_grad_(True)
    (R.turn(leaf, pos[..., None], w, layout, 0.7) * g.double()).sum().backward()
    size = g.double().abs().amax(-1, keepdim=True)
    assert bool(((dx.double() - leaf.grad).abs()
                 <= 2.0 ** -24 * 1.01 * leaf.grad.abs() + size * 2.0 ** -35).all())
    e = randn(dev, "f32", 9, 2, 4, 64, seed=5)
    up, _ = spla.rotate(cfg, rope, x + e, positions=pos)
    y, _ = spla.rotate(cfg, rope, x, positions=pos)
    step = ((x + e).double() - x.double())
    lhs = ((up.double() - y.double()) * g.double()).sum()
    rhs = (dx.double() * step).sum()
    # each of the three fp32 results is off by half a step of its size at most
    bound = 2.0 ** -24 * (((up.double().abs() + y.double().abs()) * g.double().abs()).sum()
                          + (dx.double().abs() * step.abs()).sum()) * 1.01
    assert abs(lhs - rhs) <= bound


def test_rotate_on_another_stream_and_in_a_graph(dev):
    cfg, rope = config(2, 8, 2), spla.make_rope(128)
    q, lens = randn(dev, "bf16", 4, 2, 8, 128), torch.tensor([5, 9], dtype=torch.int32, device=dev)
    want, _ = spla.rotate(cfg, rope, q, seq_lens=lens)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(q)
    with torch.cuda.stream(s):
        spla.rotate(cfg, rope, q, seq_lens=lens, q_out=out)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(out, want)
    out.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        spla.rotate(cfg, rope, q, seq_lens=lens, q_out=out)
    for shift in (0, 100, 7):
        lens.add_(shift)
        graph.replay()
        torch.cuda.synchronize()
        want, _ = spla.rotate(cfg, rope, q, seq_lens=lens)
        assert torch.equal(out, want)


# ------------------------------------------------------------ rotating append
APPENDS = {  # dtype, d, hkv, B, paged, windows, rot, layout, slabs of (tokens, counts)
    "bf16_d128": ("bf16", 128, 2, 64, False, (0, 0), 128, "half",
                  [(200, [200, 3, 0]), (1, None), (130, [0, 130, 77]), (1, [1, 0, 1])]),
    "bf16_d128_paged": ("bf16", 128, 1, 32, True, (0, 0), 96, "interleaved",
                        [(1, None), (95, [95, 1, 31]), (64, None)]),
    "bf16_d128_windows": ("bf16", 128, 2, 64, False, (32, 16), 128, "half",
                          [(100, [100, 99, 1]), (1, None), (33, None)]),
    "bf16_d64": ("bf16", 64, 3, 128, True, (0, 0), 30, "half",
                 [(257, [257, 0, 5]), (1, None), (2, None)]),
    "f32_d64": ("f32", 64, 2, 32, False, (0, 0), 64, "interleaved",
                [(77, [77, 32, 33]), (1, None), (40, None)]),
    "f32_d128_paged": ("f32", 128, 1, 64, True, (0, 0), 128, "half",
                       [(1, None), (70, [1, 70, 69])]),
    "bf16_d128_part": ("bf16", 128, 2, 128, True, (0, 0), 48, "half",
                       [(300, [300, 129, 2]), (50, None)]),
    "bf16_d128_pairs": ("bf16", 128, 2, 64, False, (0, 0), 112, "interleaved",
                        [(130, [130, 65, 0]), (64, None)]),
    "bf16_d128_odd": ("bf16", 128, 1, 64, False, (0, 0), 90, "half", [(130, [130, 65, 0])]),
    "bf16_d128_long": ("bf16", 128, 1, 64, False, (0, 0), 128, "half", [(5000, [5000, 4097, 64])]),
}


@pytest.mark.parametrize("name", list(APPENDS))
def test_append_rope(dev, name):
    """Cache contents after rotating appends: the rotated rows, and the statistics, state and
    lengths that an append of those rows gives, bit for bit but for the state, whose sums are
    taken in another order: within the bounds below."""
    dtype, d, hkv, B, paged, win, rot, layout, slabs = APPENDS[name]
    b, cap = 3, -(-(sum(s[0] for s in slabs) + 5) // B) * B
    pages, table, extra = 0, None, {}
    if paged:
        pages = b * (cap // B) + 5
        table = torch.randperm(pages, generator=torch.Generator().manual_seed(3))
        table = table[:b * (cap // B)].view(b, -1).int().to(dev)
    cfg = config(b, hkv * 2, hkv, d, B, cap, dtype, sel_window=win[0], sel_stride=win[1],
                 kv_pages=pages)
    kw = dict(base=500000.0, scaling="linear", factor=2.0)
    rope, w = spla.make_rope(d, rot, layout, **kw), R.frequencies(rot, **kw)
    one, two = (spla.SplaCache(cfg, dev, block_table=table) for _ in range(2))
    shift = torch.tensor([0, 1000000, -7], dtype=torch.int32, device=dev)
    lens, rows, vals = [0] * b, [[] for _ in range(b)], [[] for _ in range(b)]
    for i, (T, counts) in enumerate(slabs):
        k, v = (randn(dev, dtype, b, hkv, T, d, seed=10 * i + x) for x in (1, 2))
        n = None if counts is None else torch.tensor(counts, dtype=torch.int32, device=dev)
        one.append_rope(rope, k, v, n, pos_shift=shift)
        # the same rows rotated by themselves (position-major), then appended
        pos = torch.arange(T, device=dev)[:, None] + two.seq_lens + shift
        _, kr = spla.rotate(cfg, rope, k=k.permute(2, 0, 1, 3).contiguous(),
                            positions=pos.int().contiguous())
        two.append(kr.permute(1, 2, 0, 3).contiguous(), v, n)
        for s in range(b):
            c = T if counts is None else counts[s]
            p = torch.arange(lens[s], lens[s] + c, device=dev) + int(shift[s])
            rows[s].append((k[s, :, :c], p))
            vals[s].append(v[s, :, :c])
            lens[s] += c
    torch.cuda.synchronize()
    assert one.device_errors() == 0 and one.seq_lens.cpu().tolist() == lens
    for x, y in ((one.k, two.k), (one.v, two.v), (one.stats, two.stats)):
        assert torch.equal(x, y)
    K, V = one.k_logical(), one.v_logical()
    S, z = one.state_logical()
    mean, m2 = one.stats_logical()
    for s in range(b):
        at = 0
        for x, p in rows[s]:
            R.check_turned(K[s, :, at:at + len(p)], x, p, w, layout=layout)
            at += len(p)
        assert torch.equal(V[s, :, :at], torch.cat(vals[s], 1))
        # S = sum phi(k)^T v: phi to fp32's bits, its exponent (up to 8) rounded twice and the
        # exponential, sum and quotient within a few steps: 2^-19; fp32 sums of the terms
        phi = torch.softmax(K[s, :, :at].double(), -1)
        tol = 2.0 ** -19 + (at + 64) * 2.0 ** -24
        vd = V[s, :, :at].double()
        assert bool(((S[s].double() - phi.transpose(1, 2) @ vd).abs()
                     <= tol * (phi.transpose(1, 2) @ vd.abs()) + 1e-30).all())
        assert bool(((z[s].double() - phi.sum(1)).abs() <= tol * phi.sum(1)).all())
        us, ul = (win[1], win[0]) if win[1] else (B, B)
        for u in range(-(-at // us)):  # every unit: the slabs' roundings to fp32 add up
            x = K[s, :, u * us:min(u * us + ul, at)].double()
            mu = x.mean(1)
            top = x.abs().amax(1) + 1e-30
            assert bool(((mean[s, :, u].double() - mu).abs() <= top * 2.0 ** -22).all())
            want = (x - mu[:, None]).square().sum(1)
            # rounded means of earlier slabs move the sum by their rounding times the spread
            assert bool(((m2[s, :, u].double() - want).abs()
                         <= 2.0 ** -20 * (want + x.shape[1] * top * top)).all())


def test_append_rope_at_the_capacity_and_a_bad_page(dev):
    """Tokens past the capacity are dropped and flagged, as are rows whose page is none."""
    rope = spla.make_rope(128)
    cfg = config(1, 2, 1, 128, 32, 64)
    cache = spla.SplaCache(cfg, dev)
    k, v = (randn(dev, "bf16", 1, 1, 40, 128, seed=s) for s in (1, 2))
    for _ in range(3):
        cache.append_rope(rope, k[:, :, :30].contiguous(), v[:, :, :30].contiguous())
    torch.cuda.synchronize()
    assert cache.seq_lens.item() == 64 and cache.device_errors() == spla.DEVERR_CAPACITY
    pos = torch.arange(64, device=dev)
    x = torch.cat([k[0, 0, :30]] * 3)[:64]
    R.check_turned(cache.k_logical()[0, 0], x, pos, R.frequencies(128))
    table = torch.tensor([[3, 9]], dtype=torch.int32, device=dev)  # block 1: no such page
    paged = spla.SplaCache(config(1, 2, 1, 128, 32, 64, kv_pages=4), dev, block_table=table)
    paged.append_rope(rope, k, v)
    torch.cuda.synchronize()
    assert paged.device_errors() == spla.DEVERR_PAGE and paged.seq_lens.item() == 40
    R.check_turned(paged.k_logical()[0, 0, :32], k[0, 0, :32], pos[:32], R.frequencies(128))
    assert bool((paged.k.view(4, -1)[:3] == 0).all())


def test_append_rope_in_a_graph(dev):
    """Captured once, replayed with other rows and growing lengths, eager work in between."""
    cfg, rope = config(2, 4, 2, 128, 64, 512), spla.make_rope(128)
    for T in (1, 20):
        one, two = spla.SplaCache(cfg, dev), spla.SplaCache(cfg, dev)
        k, v = (randn(dev, "bf16", 2, 2, T, 128, seed=s) for s in (1, 2))
        n = torch.tensor([T, T - 1], dtype=torch.int32, device=dev)
        one.append_rope(rope, k, v, n)  # workspaces come before the capture
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            one.append_rope(rope, k, v, n)
        one.reset()
        for i in range(4):
            k.copy_(randn(dev, "bf16", 2, 2, T, 128, seed=20 + i))
            graph.replay()
            two.append_rope(rope, k, v, n)
            torch.cuda.synchronize()
            for x, y in ((one.k, two.k), (one.v, two.v), (one.stats, two.stats),
                         (one.state, two.state), (one.norm, two.norm),
                         (one.seq_lens, two.seq_lens)):
                assert torch.equal(x, y), (T, i)


def test_binding_refuses(dev):
    cfg, rope = config(2, 4, 2), spla.make_rope(128)
    cache = spla.SplaCache(cfg, dev)
    k = randn(dev, "bf16", 2, 2, 6, 128)
    n = torch.ones(2, dtype=torch.int32, device=dev)
    for a in ((k[:, :1], k), (k, k[:, :, :5]), (k.float(), k), (k[..., ::2], k[..., ::2]),
              (k.cpu(), k), (k.transpose(0, 1), k), (k[0], k[0])):
        with pytest.raises(ValueError):
            cache.append_rope(rope, *a)
    for kw in (dict(n_new=n.long()), dict(n_new=n[:1]), dict(pos_shift=n.float()),
               dict(pos_shift=n.cpu())):
        with pytest.raises(ValueError):
            cache.append_rope(rope, k, k, **kw)
    with pytest.raises(spla.SplaError):
        cache.append_rope(spla.make_rope(64), k, k)
    q = randn(dev, "bf16", 3, 2, 4, 128)
    f = torch.zeros(3, 2, dtype=torch.int32, device=dev)
    for a, kw in (((q[:, :1],), {}), ((q.float(),), {}), ((q.cpu(),), {}), ((q[0, 0],), {}),
                  ((q,), dict(out=q[:2])), ((q,), dict(lse=f.float())), ((q,), dict(n_new=f)),
                  ((q,), dict(first_key=f[:2])), ((q,), dict(first_key=f.t())),
                  ((q,), dict(slopes=f[0].float())), ((q,), dict(prefix_len=n.long())),
                  ((q.transpose(0, 1),), {})):
        with pytest.raises(ValueError):
            cache.attend(*a, **kw)
    for kw in (dict(softcap=-1.0), dict(softcap=float("nan")), dict(out=q)):
        with pytest.raises(spla.SplaError):
            cache.attend(q, **kw)
    assert cache.attend(q[:0])[0].shape == (0, 2, 4, 128)
