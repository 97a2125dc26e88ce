"""Plain 64-bit forms of the rotary positions and of exact attention, and the
error bounds the GPU tests hold the kernels to (not collected by pytest)."""

from __future__ import annotations

import math

import numpy as np
import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}  # half a rounding step


def frequencies(rot, base=10000.0, scaling="none", factor=1.0, orig_len=0.0, low=1.0, high=32.0):
    """Radians per position of each pair."""
    out = []
    for i in range(rot // 2):
        b = base * factor ** (rot / (rot - 2)) if scaling == "base" and rot > 2 else base
        w = b ** (-2.0 * i / rot)
        if scaling == "linear":
            w /= factor
        if scaling == "parts":
            turns = orig_len * w / (2.0 * math.pi)
            c = min(1.0, max(0.0, (turns - low) / (high - low)))
            w = c * w + (1.0 - c) * w / factor
        out.append(w)
    return np.array(out)


def turn(x, pos, w, layout="half", gain=1.0, transpose=False):
    """x [..., d] (torch) rotated at pos [...] -> fp64."""
    x = x.double()
    w = torch.as_tensor(w, dtype=torch.float64, device=x.device)
    r = 2 * len(w)
    a = pos.double()[..., None].to(x.device) * w
    cos, sin = gain * torch.cos(a), gain * torch.sin(a) * (-1.0 if transpose else 1.0)
    y = x.clone()
    i0 = slice(0, r // 2) if layout == "half" else slice(0, r, 2)
    i1 = slice(r // 2, r) if layout == "half" else slice(1, r, 2)
    y[..., i0] = x[..., i0] * cos - x[..., i1] * sin
    y[..., i1] = x[..., i1] * cos + x[..., i0] * sin
    return y


def check_turned(got, x, pos, w, **kw):
    """got: one rounding to fp32 and one to its type away from the 64-bit rotation, whose angle
    is off by a few fp64 steps of its size in turns."""
    assert got.shape == x.shape
    if not x.numel():
        return
    ref = turn(x, pos, w, **kw)
    r = 2 * len(w)
    size = x.double().abs().amax(-1, keepdim=True) * abs(kw.get("gain", 1.0))
    angle = pos.double().abs().max().item() * float(np.max(w)) + 1.0
    tol = (HALF[got.dtype] + 2.0 ** -24) * ref.abs() * 1.001 + size * (8.0 * angle * 2.0 ** -52)
    err = (got.double() - ref).abs()
    assert bool((err[..., :r] <= tol[..., :r]).all()), float((err - tol)[..., :r].max())
    assert torch.equal(got[..., r:], x[..., r:])


def attention(q, k, v, pos, scale=None, softcap=0.0, slope=0.0, lo=None, hi=None,
              cap_series=False):
    """One head in fp64: q [T, d], k, v [L, d], visible keys lo[t] .. hi[t] - 1.
    Returns out, lse and bounds on the error of each (see bounds in the body)."""
    dt = q.dtype
    q, k, v = q.double(), k.double(), v.double()
    T, d = q.shape
    L = k.shape[0]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    j = torch.arange(L, device=q.device)
    see = (j >= lo[:, None]) & (j < hi[:, None])
    dot = q @ k.t() * scale
    capped = softcap * torch.tanh(dot / softcap) if softcap else dot
    x = capped - slope * (pos[:, None] - j).abs()
    x = x.masked_fill(~see, -math.inf)
    lse = torch.logsumexp(x, -1) if L else torch.full((T,), -math.inf, device=q.device).double()
    p = torch.exp(x - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)[:, None])
    p = p.masked_fill(~see, 0.0)
    out = p @ torch.where(torch.isfinite(v), v, torch.zeros_like(v))
    # error of a score: d + 4 fp32 roundings of the sum's terms, 4 of the score's own size and of
    # the running maximum's (scaling, bias, difference to it), tanh within 2^-21, with
    # cap_series (fp32, and few rows) also within 2^-18 of itself (below 1/4 six roundings, above
    # that 2^-21 of four times itself), exp2 within 2 steps. A weight is off by that share of itself; bf16 weights are rounded once more; the
    # sums of L weights take fp32 roundings; the output is rounded once.
    top = x.amax(-1, keepdim=True) if L else torch.zeros((T, 1), device=q.device)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    xa = torch.where(see, x, torch.zeros_like(x)).abs()
    eps = (2.0 ** -24 * (d + 4) * scale * (q.abs() @ k.abs().t()) + 2.0 ** -22 * (xa + top.abs())
           + 2.0 ** -21)
    cap = torch.full_like(x, softcap * 2.0 ** -21)
    eps = eps + (torch.minimum(cap, 2.0 ** -18 * capped.abs()) if cap_series else cap)
    eps = torch.where(see, eps, torch.zeros_like(eps))
    steps = min(L, 4096) * 2.0 ** -24
    pe = p * (eps + steps)
    va = torch.where(torch.isfinite(v), v, torch.zeros_like(v)).abs()
    tol = pe @ va + out.abs() * (pe.sum(-1, keepdim=True) + HALF[dt]) * 1.01 + 1e-30
    if dt == torch.bfloat16:
        tol = tol + (p @ va) * HALF[dt]
    lse_tol = pe.sum(-1) * 1.01 + 2.0 ** -22 * (torch.where(lse == -math.inf, 0.0, lse).abs() + 1.0)
    return out, lse, tol, lse_tol


def visible(L, n, T, first=None, prefix=0):
    """(pos, lo, hi) of the n queries of a sequence of L tokens, int64 [n]."""
    pos = torch.arange(L - n, L)
    hi = torch.clamp(torch.maximum(pos + 1, torch.full_like(pos, prefix)), max=L)
    lo = torch.zeros_like(pos) if first is None else first[:n].long().clamp_min(0)
    none = lo >= hi
    lo[none] = hi[none] = 0
    return pos, lo, hi


def check_attend(out, lse, q, K, V, lens, news=None, scale=None, softcap=0.0, slopes=None,
                 first=None, prefix=None, before=None, cap_series=False):
    """out, lse of a call against the 64-bit form. K, V [b, h, max, d]; q [T, b, hq, d];
    before: (out, lse) ahead of the call, which rows without a query keep."""
    T, b, hq, d = q.shape
    G = hq // K.shape[1]
    dev = q.device
    for i in range(b):
        L = lens[i]
        n = T if news is None else min(max(news[i], 0), T)
        pos, lo, hi = (t.to(dev) for t in visible(
            L, n, T, None if first is None else first[:, i].cpu(), 0 if prefix is None else
            prefix[i]))
        for m in range(hq):
            ref, rl, tol, lt = attention(q[:n, i, m], K[i, m // G, :L], V[i, m // G, :L], pos,
                                         scale, softcap, 0.0 if slopes is None else
                                         float(slopes[m]), lo, hi, cap_series)
            err = (out[:n, i, m].double() - ref).abs()
            assert bool((err <= tol).all()), (i, m, float((err / tol).max()), float(err.max()))
            gone = rl == -math.inf
            assert torch.equal(lse[:n, i, m] == -math.inf, gone), (i, m)
            le = (lse[:n, i, m].double() - rl).abs()[~gone]
            assert bool((le <= lt[~gone]).all()), (i, m, float(le.max()))
        if before is not None:
            assert torch.equal(out[n:, i], before[0][n:, i])
            assert torch.equal(lse[n:, i], before[1][n:, i])
