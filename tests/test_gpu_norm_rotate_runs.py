"""Per-head norms with the rotation over many rows: gradients whose workgroups go through their
run of rows several times and turn their fp32 sums to fp64 on the way, forward passes whose last
workgroup has fewer rows than the others."""

import pytest
import torch

import cache8_ref as C
import rope_attend_ref as R
from paper_2601_22379_amd import spla

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
RUNS = 512  # runs of rows that a call's workgroups take, at most


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spla.lib()
    return torch.device("cuda:0")


def randn(dev, dtype, *shape, seed=0, scale=1.0):
    g = torch.Generator(device=dev).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=dev) * scale).to(DT[dtype])


def rounds(dtype, d, heads, rot, rows):
    """(rows that a workgroup takes at once, rounds of the longest run, rows that a thread has summed
    ahead of the last round): by the sizes of norm_rotate_grad_kernel."""
    elem = 2 if dtype == "bf16" else 4
    lanes = d * elem // 32 if rot % (32 // elem) == 0 else d // 2
    at_once = min(256 // min(256, heads * lanes), 32)
    per = at_once * max(1, min(4, 32 // at_once))
    n = -(-(-(-rows // RUNS)) // per)
    return at_once, n, (n - 1) * (per // at_once)


CASES = {
    # name: dtype, d, hq, hkv, T, batch, rot, layout, rows at once, rounds
    "two_chunks": ("bf16", 128, 32, 8, 5201, 2, 128, "half", 1, 6),
    "one_chunk": ("bf16", 128, 24, 8, 3469, 3, 128, "interleaved", 1, 6),
    "eight_at_once": ("bf16", 128, 3, 1, 33301, 2, 128, "half", 8, 5),
    "nine_at_once": ("bf16", 64, 6, 1, 17011, 5, 64, "interleaved", 9, 7),
    "many_at_once": ("bf16", 64, 1, 1, 300007, 1, 64, "half", 32, 19),
    "odd_part": ("bf16", 128, 4, 4, 10403, 1, 70, "half", 1, 6),
    "odd_part_small": ("bf16", 64, 2, 1, 9777, 2, 6, "interleaved", 2, 5),
    "part": ("bf16", 128, 8, 8, 20011, 1, 48, "half", 2, 5),
    "f32": ("f32", 64, 8, 2, 6511, 4, 64, "half", 3, 5),
    "f32_two_chunks": ("f32", 128, 16, 4, 10999, 1, 128, "interleaved", 1, 6),
    "f32_odd": ("f32", 128, 3, 1, 10601, 1, 90, "half", 1, 6),
}


@pytest.mark.parametrize("kind", ["shared", "head"])
@pytest.mark.parametrize("name", list(CASES))
def test_gradients_of_long_runs(dev, name, kind):
    dtype, d, hq, hkv, T, b, rot, layout, once, n_rounds = CASES[name]
    *sizes, held = rounds(dtype, d, hq + hkv, rot, T * b)
    assert sizes == [once, n_rounds] and held >= 16 and T * b % RUNS
    cfg = spla.make_config(b, hq, hkv, d, 64, 8, 64, dtype)
    rope, w, eps = spla.make_rope(d, rot, layout, gain=0.9), R.frequencies(rot), 1e-5
    # values of one sign mostly, so that the sums do not hide what a run leaves out
    q, k, gq, gk = (randn(dev, dtype, T, b, h, d, seed=s) + 0.5
                    for s, h in ((1, hq), (2, hkv), (3, hq), (4, hkv)))
    wq, wk = (1.0 + 0.4 * randn(dev, "f32", *((h, d) if kind == "head" else (d,)), seed=9 + h)
              for h in (hq, hkv))
    pos = (torch.arange(T, device=dev)[:, None] + torch.arange(b, device=dev) * 1000).int()
    dq, dk, dwq, dwk = spla.norm_rotate_grad(cfg, rope, q, k, gq, gk, wq, wk, eps, positions=pos)
    far = float(pos.max()) + 1
    for dx, dw, x, g, weight in ((dq, dwq, q, gq, wq), (dk, dwk, k, gk, wk)):
        rw = torch.zeros(x.shape[2:], dtype=torch.float64, device=dev)
        pairs, terms = torch.zeros_like(rw), torch.zeros_like(rw)
        for t in range(0, T, 8192):  # the 64-bit form of so many rows at a time
            p, xs, gs = pos[t:t + 8192, :, None], x[t:t + 8192], g[t:t + 8192]
            ref, part = C.norm_rotate_grad(xs, gs, weight, eps, p, w, layout=layout, gain=0.9)
            _, n, r = C.norm(xs, weight, eps)
            u = R.turn(gs, p, w, layout=layout, gain=0.9, transpose=True)
            # as for short runs: the rows' gradients by 40 steps of (1 + n^2) |u| r (bf16 rows in
            # fp32), fp64 steps and one rounding
            size = (u * weight.double()).abs().amax(-1, keepdim=True) * r
            size = size * (1 + n.abs().amax(-1, keepdim=True))
            steps = 2.0 ** -52 * (8 * far + 2 * d + 32)
            tol = ((C.HALF[DT[dtype]] + 2.0 ** -24) * ref.abs() * 1.001
                   + size * (steps + (40 * 2.0 ** -24 if dtype == "bf16" else 0.0)))
            assert bool(((dx[t:t + 8192].double() - ref).abs() <= tol).all())
            rw += part
            terms += (u * n).abs().flatten(0, 1).sum(0)
            pairs += (gs.double().abs().amax(-1, keepdim=True) * 2.0 ** 0.5 * 0.9
                      * n.abs()).flatten(0, 1).sum(0)
        if kind == "shared":
            rw, terms, pairs = rw.sum(0), terms.sum(0), pairs.sum(0)
        # bf16 rows: g by 8 steps of a pair's size, n by 6, a sum of up to 18 terms by 18; then
        # fp64 sums and one rounding
        tol = 2.0 ** -24 * rw.abs() * 1.001 + terms * 2.0 ** -52 * (8 * far + d + T * b * hq)
        tol = tol + pairs * (32 * 2.0 ** -24 if dtype == "bf16" else 0.0)
        err = (dw.double() - rw).abs()
        assert bool((err <= tol).all()), float((err / tol).max())
    again = spla.norm_rotate_grad(cfg, rope, q, k, gq, gk, wq, wk, eps, positions=pos)
    for x, y in zip(again, (dq, dk, dwq, dwk)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype,d,hq,hkv,T,b", [
    ("bf16", 128, 4, 4, 1025, 1), ("bf16", 128, 16, 8, 347, 3), ("bf16", 64, 8, 2, 1031, 1),
    ("bf16", 64, 3, 1, 257, 6), ("f32", 128, 8, 2, 1027, 1), ("f32", 64, 8, 8, 205, 5)])
def test_last_rows(dev, dtype, d, hq, hkv, T, b):
    """Rows by fours whose number is no multiple of four: all of them and nothing behind them."""
    assert T * b >= 1024 and T * b % 4
    cfg, rope = spla.make_config(b, hq, hkv, d, 64, 8, 64, dtype), spla.make_rope(d)
    q, k = randn(dev, dtype, T, b, hq, d, seed=1), randn(dev, dtype, T, b, hkv, d, seed=2)
    wq, wk = (1.0 + 0.4 * randn(dev, "f32", d, seed=s) for s in (3, 4))
    pos = (torch.arange(T, device=dev)[:, None] + torch.arange(b, device=dev) * 77).int()
    bufs = [torch.full((T + 2, b, h, d), 7.0, dtype=DT[dtype], device=dev) for h in (hq, hkv)]
    spla.norm_rotate(cfg, rope, q, k, wq, wk, positions=pos, q_out=bufs[0][1:-1],
                     k_out=bufs[1][1:-1])
    for buf, x, weight in ((bufs[0], q, wq), (bufs[1], k, wk)):
        assert bool((buf[0] == 7.0).all()) and bool((buf[-1] == 7.0).all())
        ref = C.norm_rotate(x, weight, 1e-6, pos[..., None], R.frequencies(d))
        size = ref.abs().amax(-1, keepdim=True) * 2.0 ** 0.5
        own = 16 * 2.0 ** -24 if dtype == "bf16" else 0.0
        steps = 2.0 ** -52 * (8 * (float(pos.max()) + 1) + d + 16)
        tol = (C.HALF[DT[dtype]] + 2.0 ** -24) * ref.abs() * 1.001 + size * (own + steps)
        assert bool(((buf[1:-1].double() - ref).abs() <= tol).all())
