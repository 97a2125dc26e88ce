"""Attention over the 8-bit cache by queries at the ends of their type."""

import math

import pytest
import torch

import cache8_ref as C
from paper_2601_22379_amd import spla

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
BF16_MAX = torch.finfo(torch.bfloat16).max
F32_MAX = torch.finfo(torch.float32).max


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spla.lib()
    return torch.device("cuda:0")


def randn(dev, *shape, seed=0):
    return torch.randn(shape, generator=torch.Generator(device=dev).manual_seed(seed), device=dev)


# few rows (tiles of 16) and, at a large capacity, many (tiles of 128)
FORMS = [("bf16", 128, 3, 256), ("bf16", 128, 150, 131072), ("f32", 64, 3, 256),
         ("f32", 128, 3, 256), ("f32", 64, 150, 524288), ("f32", 128, 150, 524288)]


@pytest.mark.parametrize("dtype,d,T,cap", FORMS)
def test_largest_finite(dev, dtype, d, T, cap):
    """Finite queries up to the type's largest, over keys and a scale that keep the scores small."""
    L, scale = 250, 2.0 ** -28
    cfg = spla.make_config(1, 4, 2, d, 64, 8, cap, dtype, softmax_scale=scale)
    cache = spla.SplaCache8(cfg, dev)
    k = randn(dev, L, 1, 2, d, seed=1) * 2.0 ** -100
    v = randn(dev, L, 1, 2, d, seed=2)
    cache.append(k.to(DT[dtype]), v.to(DT[dtype]))
    K, V = (x.double().permute(1, 2, 0, 3).contiguous() for x in cache.read(L))
    q = randn(dev, T, 1, 4, d, seed=3)
    big = F32_MAX if dtype == "f32" else BF16_MAX
    # (between bf16's largest and fp32's, a number rounds to a bf16 infinity)
    for i, x in enumerate((big, -big, BF16_MAX, -(BF16_MAX + big) / 2, big * (1 - 2.0 ** -20))):
        q[:, 0, i % 4, 5 + 11 * i] = x
    q = q.to(DT[dtype])
    q = torch.where(torch.isfinite(q), q, torch.full_like(q, BF16_MAX))
    out, lse = cache.attend(q)
    many = dtype == "bf16" and T > 64
    C.check_attend(out, lse, q, K, V, [L], scale=scale, one_term=many)


@pytest.mark.parametrize("softcap", [5.0, 50.0, 200.0])
@pytest.mark.parametrize("dtype,d,T,cap", FORMS)
def test_infinite_under_a_cap(dev, dtype, d, T, cap, softcap):
    """An infinite score is the cap itself: +-c by the sign of the key's number."""
    L = 250
    cfg = spla.make_config(1, 4, 2, d, 64, 8, cap, dtype)
    cache = spla.SplaCache8(cfg, dev)
    k = randn(dev, L, 1, 2, d, seed=1)
    k = torch.where(k < 0, k - 0.25, k + 0.25)  # none of them zero
    v = randn(dev, L, 1, 2, d, seed=2)
    cache.append(k.to(DT[dtype]), v.to(DT[dtype]))
    K, V = (x.double().permute(1, 2, 0, 3).contiguous() for x in cache.read(L))
    q = randn(dev, T, 1, 4, d, seed=3).to(DT[dtype])
    at = {0: (7, math.inf), 2: (d - 3, -math.inf)}  # head: coordinate, value
    for m, (c, x) in at.items():
        q[:, 0, m, c] = x
    q[0, 0, 1, 3], q[0, 0, 3, 4] = math.inf, math.nan  # a row of its own each
    out, lse = cache.attend(q, softcap=softcap)
    see = torch.arange(L, device=dev) <= torch.arange(L - T, L, device=dev)[:, None]
    # weights 1 and e^-2c: a capped score is off by c 2^-21, and by 2^-22 of its own size and of the
    # maximum's, exp2 by 2^-21, the sums by L 2^-24; weights enter their product in 24 bits (fp32),
    # 16 (bf16) or 8 (bf16, many rows); the output is rounded once
    many = dtype == "bf16" and T > 64
    eps = softcap * (2.0 ** -20 + 2.0 ** -21) + 2.0 ** -20 + L * 2.0 ** -24
    own = 2.0 ** -24 if dtype == "f32" else 2.0 ** -8 if many else 2.0 ** -16
    for m, (c, x) in at.items():
        s = softcap * torch.sign(K[0, m // 2, :, c]) * math.copysign(1.0, x)
        s = s.expand(T, L).masked_fill(~see, -math.inf)
        ref_lse = torch.logsumexp(s, -1)
        p = torch.exp(s - ref_lse[:, None])
        ref = p @ V[0, m // 2]
        tol = (p @ V[0, m // 2].abs()) * (2 * eps + own) + C.HALF[DT[dtype]] * ref.abs() + 1e-30
        err = (out[:, 0, m].double() - ref).abs()
        assert bool((err <= 1.01 * tol).all()), (m, float((err / tol).max()))
        le = (lse[:, 0, m].double() - ref_lse).abs()
        assert bool((le <= eps + 2.0 ** -22 * (softcap + 7.0)).all()), float(le.max())
    assert torch.isnan(out[0, 0, 3]).all() and torch.isnan(lse[0, 0, 3])
    assert torch.isfinite(out[:, 0, 1]).all() and torch.isfinite(out[1:, 0, 3]).all()


@pytest.mark.parametrize("dtype,d,T,cap", FORMS)
def test_odd_rows_stay_by_themselves(dev, dtype, d, T, cap):
    """NaN in a query, or infinities without a cap: no other query changes by a bit."""
    L = 250
    cfg = spla.make_config(1, 4, 2, d, 64, 8, cap, dtype)
    cache = spla.SplaCache8(cfg, dev)
    cache.append(*(randn(dev, L, 1, 2, d, seed=s).to(DT[dtype]) for s in (1, 2)))
    q = randn(dev, T, 1, 4, d, seed=3).to(DT[dtype])
    want, wl = cache.attend(q)
    odd = torch.zeros(T, 1, 4, dtype=torch.bool, device=dev)
    for t, m, x in ((0, 1, math.nan), (1, 2, math.inf), (T - 1, 3, -math.inf)):
        q[t, 0, m, 9] = x
        odd[t, 0, m] = True
    out, lse = cache.attend(q)
    assert torch.isnan(out[odd]).all()
    assert torch.equal(out[~odd], want[~odd]) and torch.equal(lse[~odd], wl[~odd])
