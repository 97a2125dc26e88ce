"""Exact attention at the ends of the value range, and the precision of capped scores, on the
GPU against the 64-bit form."""

import math

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


def held(dev, dtype, K, V, cap, hq):
    """A cache with softmax_scale 1 that holds K, V [b, hkv, L, d]."""
    b, hkv, L, d = K.shape
    cfg = spla.make_config(b, hq, hkv, d, 32, 2, cap, dtype, n_sink=0, n_local=0,
                           softmax_scale=1.0)
    cache = spla.SplaCache(cfg, dev)
    cache.append(K, V)
    return cache


# 16 heads on one KV head. Tiles of 16 rows: the four wavefronts' joint, the last workgroup's
# join of 8 splits, the join in a launch of its own (32 splits); many rows: unsplit and split.
FORMS = [("bf16", 1, 100, 128), ("bf16", 1, 1000, 1024), ("bf16", 1, 4000, 4096),
         ("bf16", 7, 500, 512), ("bf16", 7, 4000, 4096),
         ("f32", 1, 100, 128), ("f32", 1, 1000, 1024), ("f32", 1, 4000, 4096),
         ("f32", 7, 50, 64), ("f32", 7, 1000, 1024)]


@pytest.mark.parametrize("last", [True, False])
@pytest.mark.parametrize("kind", ["plain", "bias", "cap"])
@pytest.mark.parametrize("form", FORMS, ids=lambda f: "-".join(map(str, f)))
def test_large_values_of_vanishing_weight(dev, form, kind, last):
    """Keys whose scores lie more than 126 bits under the highest, with values of 2^97, beside
    values of 2^-30 at the highest scores (seen last, or first): what the former add is below
    2^97 e^-120 = 2^-76, and the outputs are the mean of the latter."""
    dtype, T, L, cap = form
    K = torch.zeros(1, 1, L, 128, dtype=DT[dtype], device=dev)
    V = randn(dev, dtype, 1, 1, L, 128, seed=1)
    top = torch.zeros(L, dtype=torch.bool, device=dev)
    top[L - T - 3 if last else 0:L if last else 5] = True
    K[0, 0, top, 0] = 140.0
    V *= torch.where(top, 2.0 ** -30, 2.0 ** 95)[:, None].to(DT[dtype])
    cache = held(dev, dtype, K, V, cap, 16)
    q = torch.zeros(T, 1, 16, 128, dtype=DT[dtype], device=dev)
    q[..., 0] = 1.0
    kw = {}
    if kind == "bias":
        kw["slopes"] = torch.linspace(0.0, 2.0 ** -10, 16, device=dev)
    if kind == "cap":
        kw["softcap"] = 200.0
    out, lse = cache.attend(q, **kw)
    R.check_attend(out, lse, q, K, V, [L], scale=1.0, cap_series=True, **kw)
    assert float(out.abs().max()) < 2.0 ** -26


@pytest.mark.parametrize("softcap,size", [(0.0, 2.0 ** 95), (42.0, 2.0 ** 95), (41.0, 2.0 ** 73),
                                          (5.0, 2.0 ** 73)])
@pytest.mark.parametrize("form", FORMS, ids=lambda f: "-".join(map(str, f)))
def test_largest_values(dev, form, softcap, size):
    """Values up to the documented 2^97 (2^75 with a small cap) leave every sum finite."""
    dtype, T, L, cap = form
    K, V = randn(dev, dtype, 1, 1, L, 128, seed=2), randn(dev, dtype, 1, 1, L, 128, seed=3)
    K[..., 0] = 8.0
    V = V.abs() * size
    cache = held(dev, dtype, K, V, cap, 16)
    q = randn(dev, dtype, T, 1, 16, 128, seed=4)
    q[..., 0] = 40.0  # scores at the upper end of the cap
    out, lse = cache.attend(q, softcap=softcap)
    assert bool(torch.isfinite(out).all())
    R.check_attend(out, lse, q, K, V, [L], scale=1.0, softcap=softcap,
                   cap_series=dtype == "f32" or T == 1)


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("softcap", [20.0, 64.0, 65.0, 200.0, 1024.0])
@pytest.mark.parametrize("form", [("bf16", 1), ("bf16", 40), ("f32", 1), ("f32", 40)],
                         ids=lambda f: "-".join(map(str, f)))
def test_capped_scores(dev, form, softcap, bias):
    """Queries that see one key each (products of one coordinate: exact): the log-sum-exp is the
    capped score, off by c 2^-21 at most, for caps above 64 also by 2^-18 of itself, and four
    fp32 roundings. The bias of a query's own position is none."""
    dtype, T = form
    L = 300
    K = torch.zeros(1, 1, L, 128, dtype=DT[dtype], device=dev)
    size = torch.exp2(torch.linspace(-12.0, 1.0, L, device=dev)) * softcap
    K[0, 0, :, 0] = (size * randn(dev, "f32", L, seed=6)).to(DT[dtype])
    K = K[:, :, torch.randperm(L, generator=torch.Generator().manual_seed(7)).to(dev)].contiguous()
    V = randn(dev, dtype, 1, 1, L, 128, seed=8)
    cache = held(dev, dtype, K, V, 320, 16)
    q = torch.zeros(T, 1, 16, 128, dtype=DT[dtype], device=dev)
    q[..., 0] = 1.0
    pos = torch.arange(L - T, L, device=dev)
    kw = dict(slopes=torch.linspace(0.5, 2.0, 16, device=dev)) if bias else {}
    out, lse = cache.attend(q, softcap=softcap, first_key=pos.int()[:, None].contiguous(), **kw)
    want = softcap * torch.tanh(K[0, 0, pos, 0].double() / softcap)[:, None, None]
    tol = torch.full_like(want, softcap * 2.0 ** -21)
    if softcap > 64.0:
        tol = torch.minimum(tol, want.abs() * 2.0 ** -18)
    tol = tol + want.abs() * 2.0 ** -22
    assert bool(((lse.double() - want).abs() <= tol).all()), float(
        ((lse.double() - want).abs() / tol).max())
    # (in bf16 the weight, e to a difference of references, may be rounded beside the output)
    v = V[0, 0, pos][:, None, None].double()
    assert bool(((out.double() - v).abs() <= v.abs() * 2.01 * 2.0 ** -8).all())


@pytest.mark.parametrize("kind", ["plain", "bias", "cap", "prefix"])
@pytest.mark.parametrize("T,L,cap", [(1, 100, 128), (2, 1000, 1024), (4, 4000, 4096), (4, 37, 64)])
def test_weights_of_few_rows(dev, T, L, cap, kind):
    """bf16 values that cancel in pairs, so that the rounding of a weight shows: weights of few
    rows are products of two bf16 terms, off by 2^-16."""
    K, V = randn(dev, "bf16", 1, 1, L, 128, seed=11), randn(dev, "bf16", 1, 1, L, 128, seed=12)
    q = randn(dev, "bf16", 1, 1, 16, 128, seed=13, scale=0.1).expand(T, 1, 16, 128).contiguous()
    kw, prefix = {}, 0
    if kind == "bias":
        kw["slopes"] = torch.full((16,), 2.0 ** -8, device=dev)
    if kind == "cap":
        kw["softcap"] = 3.0
    if kind == "prefix":
        prefix = L
    dot = q[0, 0, 0].double() @ K[0, 0].double().t()
    x = 3.0 * torch.tanh(dot / 3.0) if kind == "cap" else dot
    if kind == "bias":  # relative to any position after both
        x = x + torch.arange(L, device=dev) * 2.0 ** -8
    n = L // 2 * 2
    V[0, 0, 1:n:2] = (-V[0, 0, 0:n:2].double() * torch.exp(x[0:n:2] - x[1:n:2])[:, None]).bfloat16()
    cache = held(dev, "bf16", K, V, cap, 16)
    q[:, :, 1:] = q[:, :, :1]
    pre = torch.tensor([L], dtype=torch.int32, device=dev) if prefix else None
    out, lse = cache.attend(q, prefix_len=pre, **kw)
    pos, lo, hi = (t.to(dev) for t in R.visible(L, T, T, None, prefix))
    slope = float(kw["slopes"][0]) if kind == "bias" else 0.0
    ref, rl, tol, lt = R.attention(q[:, 0, 0], K[0, 0], V[0, 0], pos, 1.0, kw.get("softcap", 0.0),
                                   slope, lo, hi, True)
    j = torch.arange(L, device=dev)
    xs = x[None] - (slope * pos[:, None] if slope else 0.0)
    p = torch.exp(xs - rl[:, None]) * ((j >= lo[:, None]) & (j < hi[:, None]))
    pv = p @ V[0, 0].double().abs()
    tol = tol - pv * 2.0 ** -8 + pv * 2.0 ** -16
    for m in range(16):
        err = (out[:, 0, m].double() - ref).abs()
        assert bool((err <= tol).all()), (m, float((err / tol).max()))
