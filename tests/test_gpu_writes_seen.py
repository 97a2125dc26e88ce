"""Outputs that the caller hands in: autograd has to see that they were written, whatever tensor
names the memory."""

import pytest
import torch

from paper_2601_22379_amd import spla

pytestmark = pytest.mark.gpu

B, HQ, HKV, D, T = 2, 4, 2, 64, 3


def rows(h, seed=0, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((T, B, h, D), generator=g, device="cuda").to(dtype)


def kept(x):
    """A product that keeps x for its backward pass."""
    w = torch.ones_like(x, requires_grad=True)
    return (x * w).sum()


def stale(z):
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.backward()


@pytest.fixture(scope="module")
def cfg():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return spla.make_config(B, HQ, HKV, D, 32, 8, 64, "bf16")


@pytest.fixture(scope="module")
def rope():
    return spla.make_rope(D)


@pytest.mark.parametrize("call", ["rotate", "norm_rotate"])
@pytest.mark.parametrize("how", ["buffer", "view", "slices"])
def test_rotations(cfg, rope, call, how):
    fn = getattr(spla, call)
    q, k = rows(HQ), rows(HKV, 1)
    if how == "buffer":  # memory of the caller's that is not the input's
        qo, ko = rows(HQ, 2), rows(HKV, 3)
        zs = kept(qo), kept(ko)
        fn(cfg, rope, q, k, q_out=qo, k_out=ko)
    elif how == "view":  # in place, under another name
        zs = kept(q), kept(k)
        fn(cfg, rope, q, k, q_out=q.view(T, B, HQ, D), k_out=k.view(T, B, HKV, D))
    else:  # slices of one projection's rows
        x = torch.randn(T, B, (HQ + HKV) * D, device="cuda").bfloat16()
        zs = kept(x),
        fn(cfg, rope, q, k, q_out=x[..., :HQ * D].view(T, B, HQ, D),
           k_out=x[..., HQ * D:].view(T, B, HKV, D))
    for z in zs:
        stale(z)
    z = kept(q)  # what is only read stays usable
    fn(cfg, rope, q, k)
    z.backward()


@pytest.mark.parametrize("how", ["buffer", "view"])
def test_gradients(cfg, rope, how):
    q, k, gq, gk = rows(HQ), rows(HKV, 1), rows(HQ, 2), rows(HKV, 3)
    if how == "buffer":
        outs = rows(HQ, 4), rows(HKV, 5)
        zs = [kept(x) for x in outs]
    else:
        outs = gq.view(gq.shape), k.view(k.shape)
        zs = [kept(gq), kept(k)]
    spla.norm_rotate_grad(cfg, rope, q, k, gq, gk, q_out=outs[0], k_out=outs[1])
    for z in zs:
        stale(z)


def test_caches(cfg):
    k = rows(HKV, 1)
    c8, c16 = spla.SplaCache8(cfg), spla.SplaCache(cfg)
    c8.append(k, k)
    c16.append(k.permute(1, 2, 0, 3).contiguous(), k.permute(1, 2, 0, 3).contiguous())
    q = rows(HQ, 2)
    for cache in (c8, c16):
        out, lse = rows(HQ, 3), torch.randn(T, B, HQ, device="cuda")
        zs = kept(out), kept(lse), kept(out[1:])
        cache.attend(q, out, lse)
        for z in zs:
            stale(z)
    ko, vo = rows(HKV, 4), rows(HKV, 5)
    zs = kept(ko), kept(vo)
    c8.read(T, k_out=ko, v_out=vo)
    for z in zs:
        stale(z)


def test_under_inference_mode(cfg, rope):
    """Tensors without a count of writes are written all the same, inside the mode and outside."""
    with torch.inference_mode():
        q, k, out, lse = rows(HQ), rows(HKV, 1), rows(HQ, 2), torch.empty(T, B, HQ, device="cuda")
        ko, vo = rows(HKV, 2), rows(HKV, 3)
    for inside in (True, False):
        with torch.inference_mode(inside):
            want = spla.norm_rotate(cfg, rope, q, k)
            got = spla.norm_rotate(cfg, rope, q, k, q_out=out, k_out=ko)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            spla.rotate(cfg, rope, q, k, q_out=out, k_out=ko)
            cache = spla.SplaCache8(cfg)
            cache.append(k, k)
            cache.attend(q, out, lse)
            assert torch.equal(out, cache.attend(q)[0])
            cache.read(T, k_out=ko, v_out=vo)
            assert torch.equal(ko, vo)
