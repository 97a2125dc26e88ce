"""Plain 64-bit forms of the 8-bit cache, of attention over it and of the per-head norms, and the
error bounds the GPU tests hold the kernels to (not collected by pytest)."""

from __future__ import annotations

import math

import torch

import rope_attend_ref as R

HALF = R.HALF
E_MIN, E_MAX = -100, 119


def code_values():
    """The 256 numbers of e4m3 from its definition, fp64 (NaN at magnitude 0x7F)."""
    out = []
    for c in range(256):
        s, e, m = c >> 7, c >> 3 & 15, c & 7
        x = math.nan if c & 0x7F == 0x7F else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out.append(-x if s else x)
    return torch.tensor(out, dtype=torch.float64)


def to_codes(x):
    """fp64 x to the nearest number of e4m3 (ties to the even code), as fp64: by search in the
    list of numbers. Finite magnitudes past 448 give 448, infinities and NaN give NaN."""
    x = x.double()
    v = code_values()[:0x7F].to(x.device)  # 0 .. 448, ascending with the code
    a = x.abs().clamp_max(448.0)
    hi = torch.searchsorted(v, a.contiguous()).clamp_max(len(v) - 1)
    lo = (hi - 1).clamp_min(0)
    up = (v[hi] - a) < (a - v[lo])
    tie = (v[hi] - a) == (a - v[lo])
    pick = torch.where(up | (tie & (hi % 2 == 0)) | (v[hi] == a), v[hi], v[lo])
    return torch.where(torch.isfinite(x), torch.copysign(pick, x), torch.full_like(x, math.nan))


def exponent(amax):
    e = E_MIN
    while e < E_MAX and amax > 448.0 * 2.0 ** e:
        e += 1
    return e


class Held:
    """What an 8-bit cache of one config holds, in fp64: appended to like the cache."""

    def __init__(self, batch, hkv, d, B, cap):
        self.B, self.cap = B, cap
        self.x = torch.zeros((batch, hkv, cap, d), dtype=torch.float64)  # the values held
        self.e = torch.full((batch, hkv, cap // B), E_MIN)
        self.lens = [0] * batch

    def append(self, rows, n, start):
        """rows [T, batch, hkv, d] (cpu), the first n[b] of sequence b, to tokens start[b] .."""
        for b in range(rows.shape[1]):
            L = start[b]
            k = min(max(n[b], 0), rows.shape[0], self.cap - L)
            for blk in range(L // self.B, -(-(L + k) // self.B)):
                t0, t1 = max(L, blk * self.B), min(L + k, (blk + 1) * self.B)
                if t0 >= t1:
                    continue
                for h in range(rows.shape[2]):
                    new = rows[t0 - L:t1 - L, b, h].double()
                    had = t0 - blk * self.B
                    fin = new[torch.isfinite(new)].abs()
                    e = exponent(float(fin.max()) if fin.numel() else 0.0)
                    if had:
                        e = max(e, int(self.e[b, h, blk]))
                    s = 2.0 ** e
                    old = self.x[b, h, blk * self.B:t0]
                    self.x[b, h, blk * self.B:t0] = to_codes(old / s) * s
                    self.x[b, h, t0:t1] = to_codes(new / s) * s
                    self.e[b, h, blk] = e
            self.lens[b] = L + k


def visible(L, n, first=None, prefix=0, window=0, sinks=0):
    """(pos [n], see [n, L]) of the n queries of a sequence of L tokens."""
    pos = torch.arange(L - n, L)
    j = torch.arange(L)
    p = pos[:, None]
    f = torch.zeros_like(p) if first is None else first[:n, None].long().clamp_min(0)
    see = (j >= f) & ((j <= p) | (j < prefix))
    if window:
        see &= (j > p - window) | (j < f + sinks)
    return pos, see


def attention(q, k, v, pos, see, scale=None, softcap=0.0, slope=0.0, coarse_cap=False,
              one_term=False):
    """One head in fp64: q [T, d] over the values k, v [L, d] held, see [T, L]. Returns out, lse
    and bounds on the error of each."""
    dt = q.dtype
    q, k, v = q.double(), k.double(), v.double()
    T, d = q.shape
    L = k.shape[0]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    j = torch.arange(L, device=q.device)
    dot = q @ k.t() * scale
    capped = softcap * torch.tanh(dot / softcap) if softcap else dot
    x = (capped - slope * (pos[:, None] - j).abs()).masked_fill(~see, -math.inf)
    lse = torch.logsumexp(x, -1) if L else torch.full((T,), -math.inf, device=q.device).double()
    p = torch.exp(x - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)[:, None])
    p = p.masked_fill(~see, 0.0)
    vf = torch.where(torch.isfinite(v), v, torch.zeros_like(v))
    out = p @ vf
    # Keys and values are exact. A score's error: fp32 roundings of the sum (d terms of each of
    # up to 3 parts of the query: 3 d + 4 at 2^-24 of the terms' magnitudes), 4 of the score's own
    # size and of the running maximum's, the cap within c 2^-21 (few rows, and caps above 64: and
    # within 2^-18 of itself), exp2 within 2 steps. A weight is off by that share of itself;
    # the sums of L weights take fp32 roundings; the output is rounded once. A weight enters its
    # product in bf16 terms: half a step of bf16 is finfo.eps / 2 = 2^-8 of a number, so one term
    # leaves up to 2^-8 of the weight, a second one 2^-8 of that rest, 2^-16, a third 2^-24.
    top = x.amax(-1, keepdim=True) if L else torch.zeros((T, 1), device=q.device)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    xa = torch.where(see, x, torch.zeros_like(x)).abs()
    eps = (2.0 ** -24 * (3 * d + 4) * scale * (q.abs() @ k.abs().t())
           + 2.0 ** -22 * (xa + top.abs()) + 2.0 ** -21)
    if softcap:
        cap = torch.full_like(x, softcap * 2.0 ** -21)
        eps = eps + (cap if coarse_cap else torch.minimum(cap, 2.0 ** -18 * capped.abs()))
    eps = torch.where(see, eps, torch.zeros_like(eps))
    pe = p * (eps + min(L, 4096) * 2.0 ** -24)
    weight = 2.0 ** -24 if dt == torch.float32 else 2.0 ** -8 if one_term else 2.0 ** -16
    va = vf.abs()
    tol = (pe + p * weight) @ va * 1.01 + out.abs() * (pe.sum(-1, keepdim=True) + HALF[dt]) * 1.01
    tol = tol + 1e-30
    lse_tol = pe.sum(-1) * 1.01 + 2.0 ** -22 * (torch.where(lse == -math.inf, 0.0, lse).abs() + 1.0)
    return out, lse, tol, lse_tol


def check_attend(out, lse, q, K, V, lens, news=None, scale=None, softcap=0.0, slopes=None,
                 first=None, prefix=None, window=0, sinks=0, before=None, coarse_cap=False,
                 one_term=False):
    """out, lse of a call against the 64-bit form. K, V fp64 [b, h, max, d], the values held;
    q [T, b, hq, d]; before: (out, lse) ahead of the call, which rows without a query keep."""
    T, b, hq, d = q.shape
    G = hq // K.shape[1]
    dev = q.device
    K, V = K.to(dev), V.to(dev)
    for i in range(b):
        L = lens[i]
        n = T if news is None else min(max(news[i], 0), T)
        pos, see = (t.to(dev) for t in visible(
            L, n, None if first is None else first[:, i].cpu(), 0 if prefix is None else prefix[i],
            window, sinks))
        for m in range(hq):
            ref, rl, tol, lt = attention(q[:n, i, m], K[i, m // G, :L], V[i, m // G, :L], pos, see,
                                         scale, softcap, 0.0 if slopes is None else
                                         float(slopes[m]), coarse_cap, one_term)
            err = (out[:n, i, m].double() - ref).abs()
            assert bool((err <= tol).all()), (i, m, float((err / tol).max()), float(err.max()))
            gone = rl == -math.inf
            assert torch.equal(lse[:n, i, m] == -math.inf, gone), (i, m)
            assert not bool(out[:n, i, m][gone].any()), (i, m)
            le = (lse[:n, i, m].double() - rl).abs()[~gone]
            assert bool((le <= lt[~gone]).all()), (i, m, float(le.max()))
        if before is not None:
            assert torch.equal(out[n:, i], before[0][n:, i])
            assert torch.equal(lse[n:, i], before[1][n:, i])


def norm(x, weight, eps):
    """fp64 heads normed: (w x r, x r, r)."""
    x = x.double()
    r = (x.square().mean(-1, keepdim=True) + eps) ** -0.5
    w = torch.ones(x.shape[-1], dtype=torch.float64, device=x.device) if weight is None else \
        weight.double()
    return x * r * w, x * r, r


def norm_rotate(x, weight, eps, pos, w, **kw):
    return R.turn(norm(x, weight, eps)[0], pos, w, **kw)


def norm_rotate_grad(x, g, weight, eps, pos, w, **kw):
    """(dx, dw [.., heads, d] summed over the rows) in fp64, from the formulas."""
    y, n, r = norm(x, weight, eps)
    g = R.turn(g, pos, w, transpose=True, **kw)
    u = g if weight is None else g * weight.double()
    dx = r * (u - n * (u * n).mean(-1, keepdim=True))
    return dx, (g * n).flatten(0, -3).sum(0)
