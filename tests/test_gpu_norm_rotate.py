"""Per-head norms with the rotation in the same pass, and their gradients, on the GPU against
the 64-bit forms and against differences."""

import ctypes

import pytest
import torch

import cache8_ref as C
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


def ints(dev, v):
    return torch.tensor(v, dtype=torch.int32, device=dev)


CASES = {
    # name: dtype, d, hq, hkv, T, batch, rot, layout, weights (None, "shared", "head"), gain
    "token": ("bf16", 128, 4, 1, 1, 1, 128, "half", "shared", 1.0),
    "token_f32": ("f32", 64, 1, 1, 1, 3, 64, "interleaved", "head", 1.0),
    "rows": ("bf16", 128, 32, 8, 37, 2, 128, "half", "shared", 1.0),
    "interleaved": ("bf16", 128, 10, 2, 21, 3, 128, "interleaved", "head", 0.7),
    "part": ("bf16", 128, 8, 8, 33, 1, 48, "half", "shared", 1.0),
    "part_interleaved_d64": ("bf16", 64, 16, 1, 50, 2, 16, "interleaved", "head", 1.3),
    "odd_part": ("bf16", 128, 6, 2, 19, 2, 70, "half", "head", 1.0),
    "odd_part_d64": ("bf16", 64, 5, 1, 23, 2, 6, "interleaved", "shared", 1.0),
    "two": ("f32", 64, 3, 3, 11, 2, 2, "half", "shared", 1.0),
    "plain": ("bf16", 128, 8, 2, 9, 4, 128, "half", None, 1.0),
    "f32": ("f32", 128, 8, 2, 40, 3, 128, "half", "shared", 1.0),
    "f32_part": ("f32", 128, 4, 4, 40, 1, 72, "interleaved", "head", 1.0),
    "f32_odd": ("f32", 128, 5, 1, 13, 2, 90, "half", "head", 1.0),
    "many_d64": ("bf16", 64, 8, 2, 1100, 2, 64, "half", "shared", 1.0),
    "many_heads": ("bf16", 128, 80, 16, 30, 2, 128, "half", "head", 1.0),
    "many_rows": ("bf16", 128, 4, 4, 1500, 3, 128, "half", "shared", 1.0),
}


def inputs(dev, name, scale=2.0):
    dtype, d, hq, hkv, T, b, rot, layout, kind, gain = CASES[name]
    cfg = spla.make_config(b, hq, hkv, d, 64, 8, 64, dtype)
    rope = spla.make_rope(d, rot, layout, gain=gain)
    q, k, gq, gk = (randn(dev, dtype, T, b, h, d, seed=s, scale=scale if s < 3 else 1.0)
                    for s, h in ((1, hq), (2, hkv), (3, hq), (4, hkv)))
    wq = wk = None
    if kind:
        wq, wk = (1.0 + 0.4 * randn(dev, "f32", *((h, d) if kind == "head" else (d,)), seed=9 + h)
                  for h in (hq, hkv))
    pos = torch.arange(T, device=dev)[:, None] + torch.arange(b, device=dev) * 1000 + 3
    return cfg, rope, q, k, gq, gk, wq, wk, pos.int().contiguous()


def tolerance(dtype, ref, x, angle):
    """One rounding to fp32 and one to the type, and fp64 steps: d + 16 of the head's largest, and
    of the angle in turns. bf16 rows are computed in fp32: each of a pair's two products is off by
    at most 8 steps of 2^-24 (root 2, r, x r, w, cosine, product, sum) of itself, and a product is
    at most the head's largest |w x r| gain, which the turned head's largest is at least 1 / sqrt 2
    of (a turn keeps a pair's length)."""
    size = ref.abs().amax(-1, keepdim=True) * 2.0 ** 0.5
    own = 16 * 2.0 ** -24 if dtype == "bf16" else 0.0
    return ((C.HALF[DT[dtype]] + 2.0 ** -24) * ref.abs() * 1.001
            + size * (own + 2.0 ** -52 * (8 * angle + x.shape[-1] + 16)))


def check(got, ref, dtype, angle):
    tol = tolerance(dtype, ref, ref, angle)
    err = (got.double() - ref).abs()
    assert bool((err <= tol).all()), float((err / tol).max())


@pytest.mark.parametrize("eps", [1e-6, 0.0, 0.5])
@pytest.mark.parametrize("name", list(CASES))
def test_forward(dev, name, eps):
    dtype, d, hq, hkv, T, b, rot, layout, kind, gain = CASES[name]
    cfg, rope, q, k, _, _, wq, wk, pos = inputs(dev, name)
    w = R.frequencies(rot)
    keep = q.clone(), k.clone()
    qo, ko = spla.norm_rotate(cfg, rope, q, k, wq, wk, eps=eps, positions=pos)
    assert torch.equal(q, keep[0]) and torch.equal(k, keep[1])
    for got, x, weight in ((qo, q, wq), (ko, k, wk)):
        ref = C.norm_rotate(x, weight, eps, pos[..., None], w, layout=layout, gain=gain)
        check(got, ref, dtype, float(pos.max()) + 1)
    # one of the two alone, in place
    spla.norm_rotate(cfg, rope, q=q, q_weight=wq, eps=eps, positions=pos, q_out=q)
    assert torch.equal(q, qo)
    spla.norm_rotate(cfg, rope, k=k, k_weight=wk, eps=eps, positions=pos, k_out=k)
    assert torch.equal(k, ko)


@pytest.mark.parametrize("name", list(CASES))
def test_gradients(dev, name):
    dtype, d, hq, hkv, T, b, rot, layout, kind, gain = CASES[name]
    cfg, rope, q, k, gq, gk, wq, wk, pos = inputs(dev, name)
    w, eps = R.frequencies(rot), 1e-5
    dq, dk, dwq, dwk = spla.norm_rotate_grad(cfg, rope, q, k, gq, gk, wq, wk, eps, positions=pos)
    assert (dwq is None) == (wq is None) == (dwk is None)
    for dx, dw, x, g, weight in ((dq, dwq, q, gq, wq), (dk, dwk, k, gk, wk)):
        ref, rw = C.norm_rotate_grad(x, g, weight, eps, pos[..., None], w, layout=layout, gain=gain)
        # steps of the gradient's two terms, which may cancel; bf16 rows in fp32: u by 8 steps of
        # its size as in the forward pass, n by 6, their products' mean by 16 more (a sum of d
        # terms over lanes and by fives and sixes within them), the last two operations by 2:
        # 40 in all of (1 + n^2) |u| r
        y, n, r = C.norm(x, weight, eps)
        u = R.turn(g, pos[..., None], w, layout=layout, gain=gain, transpose=True)
        size = (u if weight is None else u * weight.double()).abs().amax(-1, keepdim=True) * r
        size = size * (1 + n.abs().amax(-1, keepdim=True))
        steps = 2.0 ** -52 * (8 * (float(pos.max()) + 1) + 2 * d + 32)
        own = 40 * 2.0 ** -24 if dtype == "bf16" else 0.0
        tol = (C.HALF[DT[dtype]] + 2.0 ** -24) * ref.abs() * 1.001 + size * (steps + own)
        err = (dx.double() - ref).abs()
        assert bool((err <= tol).all()), float((err / tol).max())
        if weight is None:
            continue
        terms = (u * n).abs().flatten(0, -3).sum(0)
        if weight.dim() == 1:
            rw, terms = rw.sum(0), terms.sum(0)
        assert dw.shape == weight.shape and dw.dtype is torch.float32
        # bf16 rows: g by 8 steps of a pair's size, n by 6, the sum of up to 19 terms by 19
        pairs = (g.double().abs().amax(-1, keepdim=True) * 2.0 ** 0.5 * abs(gain) * n.abs())
        pairs = pairs.flatten(0, -3).sum(0)
        pairs = pairs.sum(0) if weight.dim() == 1 else pairs
        tol = 2.0 ** -24 * rw.abs() * 1.001 + terms * 2.0 ** -52 * (
            8 * (float(pos.max()) + 1) + d + T * b * hq) + pairs * (
                33 * 2.0 ** -24 if dtype == "bf16" else 0.0)
        assert bool(((dw.double() - rw).abs() <= tol).all())
    # the same bits again, and in place of the rows or of the gradients
    again = spla.norm_rotate_grad(cfg, rope, q, k, gq, gk, wq, wk, eps, positions=pos, q_out=gq,
                                  k_out=k)
    assert again[0] is gq and again[1] is k
    for x, y in zip(again, (dq, dk, dwq, dwk)):
        assert x is y is None or torch.equal(x, y)


def test_gradients_are_differences(dev):
    """fp64 central differences of the 64-bit form along random directions, and the kernel's
    gradients along the same ones."""
    cfg, rope, q, k, gq, gk, wq, wk, pos = inputs(dev, "f32")
    w, eps, h = R.frequencies(128), 1e-5, 1e-6
    dq, _, dwq, _ = spla.norm_rotate_grad(cfg, rope, q, k, gq, gk, wq, wk, eps, positions=pos)

    def loss(x, weight):
        y, _, _ = C.norm(x, weight, eps)
        return (R.turn(y, pos[..., None], w) * gq.double()).sum()

    for seed in range(3):
        vx, vw = randn(dev, "f32", *q.shape, seed=70 + seed).double(), randn(
            dev, "f32", *wq.shape, seed=80 + seed).double()
        x, wt = q.double(), wq.double()
        for num, got in ((loss(x + h * vx, wt) - loss(x - h * vx, wt), (dq.double() * vx).sum()),
                         (loss(x, wt + h * vw) - loss(x, wt - h * vw), (dwq.double() * vw).sum())):
            num = num / (2 * h)
            # differences: h^2 and roundings of a sum of 123k terms over h; the kernel's fp32
            assert abs(float(num - got)) <= 1e-4 * (1.0 + abs(float(num)))


def test_rows_of_wider_ones(dev):
    """Slices of a projection's rows, gradients into slices of one buffer; lengths as positions."""
    b, hq, hkv, d, T = 3, 6, 2, 128, 17
    cfg = spla.make_config(b, hq, hkv, d, 64, 8, 64, "bf16")
    rope = spla.make_rope(d)
    x = randn(dev, "bf16", T, b, (hq + 2 * hkv) * d, seed=1)
    q, k = x[..., :hq * d].view(T, b, hq, d), x[..., hq * d:(hq + hkv) * d].view(T, b, hkv, d)
    lens = ints(dev, [5, 0, 70000])
    wq = 1 + 0.1 * randn(dev, "f32", d, seed=5)
    a = spla.norm_rotate(cfg, rope, q, k, wq, None, seq_lens=lens)
    c = spla.norm_rotate(cfg, rope, q.contiguous(), k.contiguous(), wq, None, seq_lens=lens)
    assert torch.equal(a[0], c[0]) and torch.equal(a[1], c[1])
    g = torch.full((T, b, (hq + 2 * hkv) * d), 7.0, dtype=torch.bfloat16, device=dev)
    out = g[..., :hq * d].view(T, b, hq, d), g[..., hq * d:(hq + hkv) * d].view(T, b, hkv, d)
    gq, gk = randn(dev, "bf16", T, b, hq, d, seed=2), randn(dev, "bf16", T, b, hkv, d, seed=3)
    spla.norm_rotate_grad(cfg, rope, q, k, gq, gk, wq, None, seq_lens=lens, q_out=out[0],
                          k_out=out[1])
    ref = spla.norm_rotate_grad(cfg, rope, q.contiguous(), k.contiguous(), gq, gk, wq, None,
                                seq_lens=lens)
    assert torch.equal(out[0], ref[0]) and torch.equal(out[1], ref[1])
    assert bool((g[..., (hq + hkv) * d:] == 7.0).all())


def test_extremes(dev):
    """Heads whose squares pass fp32, zeros, infinities and NaN; each head by itself."""
    cfg = spla.make_config(1, 6, 1, 64, 64, 8, 64, "f32")
    rope = spla.make_rope(64)
    q = randn(dev, "f32", 1, 1, 6, 64, seed=1)
    q[0, 0, 0] *= 1e36
    q[0, 0, 1] *= 1e-30
    q[0, 0, 2] = 0.0
    q[0, 0, 3, 5] = float("inf")
    q[0, 0, 4, 6] = float("nan")
    k = q[:, :, 5:6].contiguous()
    qo, ko = spla.norm_rotate(cfg, rope, q, k, eps=1e-6)
    ref = C.norm(q, None, 1e-6)[0]  # position 0: no turn
    for h in (0, 1, 2, 5):
        assert bool(((qo[0, 0, h].double() - ref[0, 0, h]).abs() <= 2.0 ** -23 * ref[0, 0, h].abs()
                     + 1e-44).all()), h
    assert torch.isnan(qo[0, 0, 3]).any() and torch.isnan(qo[0, 0, 4]).all()
    assert torch.equal(ko[0, 0, 0], qo[0, 0, 5])
    zero, _ = spla.norm_rotate(cfg, rope, q=q, eps=0.0)
    assert torch.isnan(zero[0, 0, 2]).all()


def test_no_rows(dev):
    cfg, rope, q, k, gq, gk, wq, wk, pos = inputs(dev, "rows")
    e = q[:0], k[:0]
    out = spla.norm_rotate(cfg, rope, *e, wq, wk)
    assert out[0].shape[0] == 0
    for a, c in ((wq, wk), (torch.ones(32, 128, device=dev), torch.ones(8, 128, device=dev))):
        g = spla.norm_rotate_grad(cfg, rope, *e, *e, a, c)
        assert g[0].shape[0] == 0 and not g[2].any() and not g[3].any()
        assert g[2].shape == a.shape and g[3].shape == c.shape
    # the library, which needs no workspace for that
    dw = torch.ones(128, device=dev)
    st = torch.cuda.current_stream().cuda_stream
    assert spla.lib().spla_norm_rotate_grad(
        ctypes.byref(cfg), ctypes.byref(rope), 0, None, None, None, None, 0, 1e-6, *[None, 0] * 6,
        None, dw.data_ptr(), None, 0, st) == 0
    assert not dw.any()


def test_captured_replays(dev):
    cfg, rope, q, k, gq, gk, wq, wk, pos = inputs(dev, "rows")
    spla.norm_rotate_grad(cfg, rope, q, k, gq, gk, wq, wk, positions=pos)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = spla.norm_rotate(cfg, rope, q, k, wq, wk, positions=pos)
        g = spla.norm_rotate_grad(cfg, rope, q, k, gq, gk, wq, wk, positions=pos)
    for i in range(4):
        q.copy_(randn(dev, "bf16", *q.shape, seed=40 + i))
        gk.copy_(randn(dev, "bf16", *gk.shape, seed=50 + i))
        graph.replay()
        torch.cuda.synchronize()
        ye = spla.norm_rotate(cfg, rope, q, k, wq, wk, positions=pos)
        ge = spla.norm_rotate_grad(cfg, rope, q, k, gq, gk, wq, wk, positions=pos)
        for a, b in zip(y + g, ye + ge):
            assert torch.equal(a, b)


def test_autograd_counts_writes(dev):
    """In place is a write that autograd sees; rows and weights that it would record are
    refused."""
    cfg, rope, q, k, gq, gk, wq, wk, pos = inputs(dev, "rows")
    before = q._version
    spla.norm_rotate(cfg, rope, q=q, q_weight=wq, positions=pos, q_out=q)
    assert q._version > before
    before = gq._version
    spla.norm_rotate_grad(cfg, rope, q=q, q_grad=gq, q_weight=wq, positions=pos, q_out=gq)
    assert gq._version > before
    wq.requires_grad_()
    with pytest.raises(ValueError):
        spla.norm_rotate(cfg, rope, q=q, q_weight=wq, positions=pos)
    with torch.no_grad():
        spla.norm_rotate(cfg, rope, q=q, q_weight=wq, positions=pos)


def test_one_weights_gradient(dev):
    """The library with the gradient of one weight only."""
    cfg, rope, q, k, gq, gk, wq, wk, pos = inputs(dev, "rows")
    ref = spla.norm_rotate_grad(cfg, rope, q, k, gq, gk, wq, wk, positions=pos)
    T, b = q.shape[:2]
    ws = torch.empty(spla.norm_rotate_grad_workspace_bytes(cfg, T), dtype=torch.uint8, device=dev)
    dq, dk, dw = torch.empty_like(q), torch.empty_like(k), torch.empty_like(wk)
    rows = lambda x: (x.data_ptr(), x.shape[2] * 128)  # noqa: E731
    st = torch.cuda.current_stream().cuda_stream
    assert spla.lib().spla_norm_rotate_grad(
        ctypes.byref(cfg), ctypes.byref(rope), T, pos.data_ptr(), None, wq.data_ptr(), wk.data_ptr(),
        0, 1e-6, *rows(q), *rows(gq), *rows(dq), *rows(k), *rows(gk), *rows(dk), None,
        dw.data_ptr(), ws.data_ptr(), ws.numel(), st) == 0
    assert torch.equal(dw, ref[3]) and torch.equal(dq, ref[0]) and torch.equal(dk, ref[1])
