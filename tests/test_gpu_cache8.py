"""Appends to the 8-bit cache and its read-back on the GPU against the 64-bit form: bit for bit."""

import ctypes
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


def randn(dtype, *shape, seed=0, scale=1.0):
    g = torch.Generator()
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(DT[dtype])


def table_of(dev, b, nb, seed=3):
    pages = b * nb + 3
    t = torch.randperm(pages, generator=torch.Generator().manual_seed(seed))[:b * nb]
    return t.view(b, nb).int().to(dev), pages


def make(dev, dtype, b, hkv, d, B, cap, paged=False, hq=None):
    table, pages = table_of(dev, b, cap // B) if paged else (None, 0)
    cfg = spla.make_config(b, hq or hkv, hkv, d, B, 8, cap, dtype, kv_pages=pages)
    return spla.SplaCache8(cfg, dev, block_table=table)


def ints(dev, v):
    return torch.tensor(v, dtype=torch.int32, device=dev)


def same(got, want, dtype):
    """Every number equal, NaN included; want fp64, representable in dtype."""
    w = want.to(DT[dtype])
    assert torch.equal(torch.nan_to_num(w.double(), nan=1e300), torch.nan_to_num(want, nan=1e300))
    g = got.cpu()
    assert torch.equal(torch.isnan(g), torch.isnan(w))
    assert torch.equal(torch.nan_to_num(g), torch.nan_to_num(w))


def check_read(cache, K, V, lens, dtype, first=None, n=None):
    n = max(lens) + 3 if n is None else n
    f = None if first is None else ints(cache.device, first)
    k, v = cache.read(n, f)
    for b, L in enumerate(lens):
        p = torch.arange(n) + (0 if first is None else first[b])
        ok = (p >= 0) & (p < L)
        at = p.clamp(0, K.cap - 1)
        for got, held in ((k, K), (v, V)):
            want = (held.x[b][:, at] * 1.0).transpose(0, 1).clone()
            want[~ok] = 0.0
            same(got[:, b], want, dtype)


CASES = {
    # name: dtype, b, hkv, d, B, cap, paged, appends (tokens per sequence, one list per call)
    "one": ("bf16", 1, 1, 128, 64, 64, False, [[1]]),
    "tokens": ("bf16", 2, 2, 128, 64, 128, True, [[1, 1]] * 40),
    "tokens_f32": ("f32", 3, 1, 64, 32, 96, False, [[1, 0, 1]] * 37),
    "chunks": ("bf16", 3, 2, 128, 64, 512, True, [[100, 1, 0], [1, 63, 64], [77, 200, 1], [1, 1, 1]]),
    "chunks_d64": ("bf16", 2, 3, 64, 128, 640, False, [[130, 127], [1, 2], [300, 1], [33, 129]]),
    "chunks_f32": ("f32", 2, 2, 128, 128, 512, False, [[5, 200], [123, 1], [130, 60]]),
    "chunks_f32_d64": ("f32", 2, 1, 64, 64, 512, True, [[63, 65], [2, 1], [250, 31]]),
    "small_blocks": ("bf16", 2, 1, 128, 32, 1024, True, [[1000, 31], [7, 900], [1, 1]]),
    "full": ("bf16", 2, 1, 64, 64, 256, False, [[256, 100], [0, 156]]),
}


@pytest.mark.parametrize("growing", [False, True])
@pytest.mark.parametrize("name", list(CASES))
def test_append_and_read(dev, name, growing):
    dtype, b, hkv, d, B, cap, paged, appends = CASES[name]
    cache = make(dev, dtype, b, hkv, d, B, cap, paged)
    K, V = C.Held(b, hkv, d, B, cap), C.Held(b, hkv, d, B, cap)
    cache.k.random_(0, 255)  # whatever the buffers held
    cache.scales.fill_(float("nan"))
    for i, n in enumerate(appends):
        T = max(max(n), 1)
        scale = 4.0 ** (i % 7) if growing else 1.0
        k = randn(dtype, T, b, hkv, d, seed=10 * i, scale=scale)
        v = randn(dtype, T, b, hkv, d, seed=10 * i + 1, scale=0.3 / scale)
        start = list(K.lens)
        K.append(k, n, start)
        V.append(v, n, start)
        cache.append(k.to(dev), v.to(dev), ints(dev, n))
        assert cache.seq_lens.tolist() == K.lens
    assert not cache.counters.any()
    assert cache.device_errors() == 0
    check_read(cache, K, V, K.lens, dtype)
    check_read(cache, K, V, K.lens, dtype, first=[L - 50 for L in K.lens], n=70)
    nb = [-(-L // B) for L in K.lens]
    if not paged:  # the powers of two themselves
        got = cache.scales.view(b, hkv, cap // B, 2).cpu().double()
        for i, n in enumerate(nb):
            assert torch.equal(got[i, :, :n, 0], 2.0 ** K.e[i, :, :n].double())
            assert torch.equal(got[i, :, :n, 1], 2.0 ** V.e[i, :, :n].double())


def test_every_bf16_number(dev):
    """All 65536 bf16 numbers, at scales that they reach by themselves or with a larger one."""
    d, B = 128, 32
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = x.view(16, 32, 1, 1, d)
    for big in (None, 3.0e38, 448.0, 1.0, 2.0 ** -90):
        cache = make(dev, "bf16", 1, 1, d, B, 512)
        rows = x.clone()
        if big is not None:
            rows = torch.where(rows.abs() <= big, rows, torch.zeros_like(rows))
            rows[:, 0, 0, 0, 0] = big
        rows = rows.view(512, 1, 1, d)
        K = C.Held(1, 1, d, B, 512)
        K.append(rows, [512], [0])
        cache.append(rows.to(dev), rows.to(dev))
        check_read(cache, K, K, [512], "bf16")


def test_codes_of_a_scale(dev):
    """fp32 numbers on and beside every tie of two codes, under the scale 1."""
    v = C.code_values()[:0x7F]
    mid = (v[1:] + v[:-1]) / 2
    x = torch.cat([v, mid, mid * (1 + 2.0 ** -20), mid * (1 - 2.0 ** -20)])
    x = torch.cat([x, -x]).float()
    rows = torch.zeros(32 * 64)
    rows[:len(x)] = x
    rows[-1] = 448.0
    rows = rows.view(32, 1, 1, 64)
    cache = make(dev, "f32", 1, 1, 64, 32, 32)
    cache.append(rows.to(dev), rows.to(dev))
    assert torch.equal(cache.scales.cpu(), torch.ones(2))
    k, _ = cache.read(32)
    same(k, C.to_codes(rows.double()), "f32")


def test_odd_numbers(dev):
    """Infinities and NaN become NaN and leave the scale alone; zeros keep their sign."""
    k = randn("f32", 40, 1, 2, 64, seed=5)
    k[3, 0, 0, 7], k[4, 0, 0, 8], k[5, 0, 1, 9] = math.inf, math.nan, -math.inf
    k[6, 0, 0, 10] = -0.0
    cache = make(dev, "f32", 1, 2, 64, 32, 64)
    K = C.Held(1, 2, 64, 32, 64)
    K.append(k, [40], [0])
    cache.append(k.to(dev), k.to(dev))
    check_read(cache, K, K, [40], "f32")
    got, _ = cache.read(40)
    assert math.copysign(1.0, got[6, 0, 0, 10].item()) == -1.0


def test_rows_of_wider_ones(dev):
    """Rows that are slices of a projection's, and every other row of a batch twice as large."""
    b, hq, hkv, d, T = 3, 8, 2, 128, 21
    x = randn("bf16", T, b, (hq + 2 * hkv) * d, seed=1).to(dev)
    k = x[..., hq * d:(hq + hkv) * d].view(T, b, hkv, d)
    v = x[..., (hq + hkv) * d:].view(T, b, hkv, d)
    one, two = (make(dev, "bf16", b, hkv, d, 64, 128, hq=hq) for _ in range(2))
    one.append(k, v)
    two.append(k.contiguous(), v.contiguous())
    assert torch.equal(one.k, two.k) and torch.equal(one.v, two.v)
    one.append(k[0], v[0])  # one token, without T
    two.append(k[:1].contiguous(), v[:1].contiguous())
    assert torch.equal(one.k, two.k) and torch.equal(one.v, two.v)
    assert one.seq_lens.tolist() == [T + 1] * b


def test_capacity_and_pages(dev):
    cache = make(dev, "bf16", 2, 1, 64, 32, 64)
    k = randn("bf16", 50, 2, 1, 64, seed=2)
    K = C.Held(2, 1, 64, 32, 64)
    K.append(k, [50, 20], [0, 0])
    cache.append(k.to(dev), k.to(dev), ints(dev, [50, 20]))
    assert cache.device_errors() == 0
    K.append(k, [50, 44], [50, 20])
    cache.append(k.to(dev), k.to(dev), ints(dev, [50, 44]))
    assert cache.device_errors() == spla.DEVERR_CAPACITY
    assert cache.seq_lens.tolist() == [64, 64]
    check_read(cache, K, K, [64, 64], "bf16")
    cache.clear_device_errors()
    cache.append(k[:1].to(dev), k[:1].to(dev))  # full: nothing, by the single token's way too
    assert cache.device_errors() == spla.DEVERR_CAPACITY and cache.seq_lens.tolist() == [64, 64]
    # a page out of range: its rows are not written, the others are
    paged = make(dev, "bf16", 2, 1, 64, 32, 64, paged=True)
    paged.block_table[1, 0] = 7
    paged.block_table[0, 1] = -1
    paged.append(k.to(dev), k.to(dev))
    assert paged.device_errors() == spla.DEVERR_PAGE
    assert paged.seq_lens.tolist() == [50, 50]
    got, _ = paged.read(32)
    K = C.Held(2, 1, 64, 32, 64)
    K.append(k, [50, 50], [0, 0])
    same(got[:, 0], K.x[0, :, :32].transpose(0, 1).clone(), "bf16")


def test_capacity_of_long_appends(dev):
    """Appends whose length a launch of its own advances, past the capacity."""
    cache = make(dev, "bf16", 2, 2, 128, 32, 256, paged=True)
    K = C.Held(2, 2, 128, 32, 256)
    for i, n in enumerate([[200, 130], [200, 126], [5, 256]]):
        k = randn("bf16", 256 if i == 2 else 200, 2, 2, 128, seed=30 + i)
        start = list(K.lens)
        K.append(k, n, start)
        cache.append(k.to(dev), k.to(dev), ints(dev, n))
        assert cache.seq_lens.tolist() == K.lens
        assert cache.device_errors() == (0 if i == 0 else spla.DEVERR_CAPACITY)
    assert K.lens == [256, 256]
    check_read(cache, K, K, K.lens, "bf16")


def test_neighbours_stay(dev):
    """An append writes the blocks it touches and nothing else."""
    cache = make(dev, "bf16", 2, 2, 128, 64, 256)
    cache.k.fill_(0x55)
    cache.v.fill_(0x33)
    cache.scales.fill_(3.0)
    k = randn("bf16", 70, 2, 2, 128, seed=4)
    cache.append(k.to(dev), k.to(dev), ints(dev, [70, 0]))
    kb, vb = (x.view(2, 2, 4, 64 * 128) for x in (cache.k, cache.v))
    assert bool((kb[1] == 0x55).all()) and bool((vb[1] == 0x33).all())
    assert bool((kb[0, :, 2:] == 0x55).all()) and bool((vb[0, :, 2:] == 0x33).all())
    s = cache.scales.view(2, 2, 4, 2)
    assert bool((s[1] == 3.0).all()) and bool((s[0, :, 2:] == 3.0).all())


@pytest.mark.parametrize("T", [1, 3, 300])
def test_captured_appends(dev, T):
    """A captured append replayed with eager ones between the replays."""
    b, hkv, d, B, cap = 3, 2, 128, 64, 2048
    cache, plain = (make(dev, "bf16", b, hkv, d, B, cap, paged=True) for _ in range(2))
    k, v = randn("bf16", T, b, hkv, d, seed=6).to(dev), randn("bf16", T, b, hkv, d, seed=7).to(dev)
    n = ints(dev, [T, T, max(T - 1, 0)])
    cache.append(k, v, n)
    plain.append(k, v, n)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.append(k, v, n)
    for i in range(4):
        k.copy_(randn("bf16", T, b, hkv, d, seed=20 + i, scale=2.0 ** i))
        graph.replay()
        plain.append(k, v, n)
        if i % 2:
            cache.append(k, v, n)
            plain.append(k, v, n)
        torch.cuda.synchronize()
        assert torch.equal(cache.seq_lens, plain.seq_lens)
        total = int(cache.seq_lens.max())
        for x, y in zip(cache.read(total), plain.read(total)):
            assert torch.equal(x, y)


def test_reset_and_empty(dev):
    cache = make(dev, "bf16", 2, 1, 128, 64, 128)
    k = randn("bf16", 5, 2, 1, 128, seed=8).to(dev)
    cache.append(k[:0], k[:0])
    assert cache.seq_lens.tolist() == [0, 0]
    kk, vv = cache.read(4)
    assert not kk.any() and not vv.any() and cache.read(0)[0].shape[0] == 0
    cache.append(k, k)
    cache.reset()
    assert cache.seq_lens.tolist() == [0, 0] and not cache.read(5)[0].any()


def test_far_positions(dev):
    """first at the ends of int32."""
    cache = make(dev, "bf16", 2, 1, 64, 32, 64)
    k = randn("bf16", 40, 2, 1, 64, seed=9)
    cache.append(k.to(dev), k.to(dev))
    got, _ = cache.read(70, ints(dev, [2 ** 31 - 1, -2 ** 31]))
    assert not got.any()


def test_read_one_of_two(dev):
    cache = make(dev, "bf16", 1, 2, 128, 64, 64)
    k = randn("bf16", 33, 1, 2, 128, seed=11).to(dev)
    cache.append(k, k * 2)
    kk, vv = cache.read(33)
    for which in range(2):
        out = torch.full_like(kk, 7.0)
        st = torch.cuda.current_stream().cuda_stream
        assert spla.lib().spla_read8(ctypes.byref(cache.cfg), ctypes.byref(cache.struct), 33, None,
                                     None if which else out.data_ptr(),
                                     out.data_ptr() if which else None, st) == 0
        assert torch.equal(out, (kk, vv)[which])
