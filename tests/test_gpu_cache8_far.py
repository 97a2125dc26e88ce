"""The 8-bit cache and the per-head norms where offsets pass 32 bits: a capacity of 4M tokens, and
rows that lie 2 GiB apart."""

import pytest
import torch

import cache8_ref as C
import rope_attend_ref as R
from paper_2601_22379_amd import spla

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spla.lib()
    return torch.device("cuda:0")


def randn(dev, *shape, seed=0, scale=1.0):
    g = torch.Generator(device=dev).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=dev) * scale).bfloat16()


@pytest.mark.parametrize("paged", [False, True])
def test_far_tokens(dev, paged):
    """Sequences whose tokens so far are taken as held: what an append adds at the far end, the
    read-back, and attention over a window that starts behind them."""
    hkv, group, d, B, cap = 10, 2, 128, 128, 1 << 22
    nb, start = cap // B, [cap - 1024, cap - 1000]
    pages, table = 0, None
    if paged:  # the last pages of a pool of 8 GiB
        pages = 1 << 16
        table = torch.full((2, nb), pages - 64, dtype=torch.int32)
        table[0, -16:] = torch.arange(pages - 32, pages - 16)
        table[1, -16:] = torch.arange(pages - 16, pages)
        table = table.to(dev)
    cfg = spla.make_config(2, hkv * group, hkv, d, B, 8, cap, "bf16", kv_pages=pages)
    assert spla.cache8_bytes(cfg)[0] > 1 << 33
    cache = spla.SplaCache8(cfg, dev, block_table=table)
    cache.seq_lens.copy_(torch.tensor(start))
    T = 700
    k, v = randn(dev, T, 2, hkv, d, seed=1), randn(dev, T, 2, hkv, d, seed=2)
    n = [T, T - 5]
    cache.append(k, v, torch.tensor(n, dtype=torch.int32, device=dev))
    lens = [s + m for s, m in zip(start, n)]
    assert cache.seq_lens.tolist() == lens and cache.device_errors() == 0
    K, V = C.Held(2, hkv, d, B, 1024), C.Held(2, hkv, d, B, 1024)
    here = [s - (cap - 1024) for s in start]  # in the last 1024 tokens
    K.lens, V.lens = list(here), list(here)
    K.append(k.cpu(), n, here)
    V.append(v.cpu(), n, here)
    got = cache.read(1024, torch.full((2,), cap - 1024, dtype=torch.int32, device=dev))
    for x, held in zip(got, (K, V)):
        for i in range(2):
            want = held.x[i].transpose(0, 1).clone()
            want[here[i] + n[i]:] = 0.0
            assert torch.equal(x[:, i].cpu().double(), want)
    lengths = [h + m for h, m in zip(here, n)]
    for rows, window in ((1, 600), (40, 300), (300, 350)):
        q = randn(dev, rows, 2, hkv * group, d, seed=3)
        out, lse = cache.attend(q, window=window)
        C.check_attend(out, lse, q, K.x, V.x, lengths, window=window)


def test_rows_far_apart(dev):
    T, b, hq, hkv, d = 2, 2, 4, 2, 64
    wide = torch.zeros(T, b, 1 << 30, dtype=torch.bfloat16, device=dev)
    x = randn(dev, T, b, (hq + 2 * hkv) * d, seed=1)
    wide[..., :x.shape[-1]] = x
    cut = lambda y: (y[..., :hq * d].view(T, b, hq, d),  # noqa: E731
                     y[..., hq * d:(hq + hkv) * d].view(T, b, hkv, d),
                     y[..., (hq + hkv) * d:(hq + 2 * hkv) * d].view(T, b, hkv, d))
    (q, k, v), near = cut(wide), [y.contiguous() for y in cut(x)]
    cfg, rope = spla.make_config(b, hq, hkv, d, 32, 8, 64, "bf16"), spla.make_rope(d)
    w = 1.0 + 0.1 * torch.randn(d, device=dev)
    a, c = (spla.norm_rotate(cfg, rope, r[0], r[1], w, w) for r in ((q, k), near))
    assert torch.equal(a[0], c[0]) and torch.equal(a[1], c[1])
    ref = C.norm_rotate(near[0], w, 1e-6, torch.arange(T, device=dev)[:, None, None],
                        R.frequencies(d))
    assert bool(((a[0].double() - ref).abs() <= 2.0 ** -7 * ref.abs().amax(-1, keepdim=True)).all())
    g = [randn(dev, *y.shape, seed=4 + i) for i, y in enumerate(near[:2])]
    a, c = (spla.norm_rotate_grad(cfg, rope, r[0], r[1], *g, w, w) for r in ((q, k), near))
    for y, z in zip(a, c):
        assert torch.equal(y, z)
    one, two = (spla.SplaCache8(cfg, dev) for _ in range(2))
    one.append(k, v)
    two.append(*near[1:])
    assert torch.equal(one.k, two.k) and torch.equal(one.v, two.v)
    spla.norm_rotate(cfg, rope, q, k, w, w, q_out=q, k_out=k)  # written far apart, too
    want = spla.norm_rotate(cfg, rope, near[0], near[1], w, w)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    assert torch.equal(v, near[2]) and not wide[..., x.shape[-1]:x.shape[-1] + 4096].any()
