"""The 8-bit cache and the per-head norms on the CPU: sizes, refusals before anything is
enqueued, the binding's checks, the documented layout."""

import ctypes
import math

import pytest
import torch

import cache8_ref as C
from paper_2601_22379_amd import spla


def cfg(**kw):
    base = dict(batch=4, n_q_heads=32, n_kv_heads=8, head_dim=128, block_size=64, top_k=32,
                max_seq_len=131072, dtype="bf16")
    base.update(kw)
    return spla.make_config(**base)


@pytest.mark.parametrize("libname", ["hip", "host"])
def test_sizes(libname):
    lib = spla.lib() if libname == "hip" else spla.host_lib()
    b = spla.cache8_bytes(cfg(), lib)
    assert b == [4 * 8 * 131072 * 128] * 2 + [4 * 8 * 2048 * 8, 16, 4 * 32 * 4]
    assert b[0] * 2 == spla.cache_bytes(cfg(), lib)[0]  # half a bf16 cache's
    assert spla.cache8_bytes(cfg(dtype="f32"), lib) == b
    pg = spla.cache8_bytes(cfg(kv_pages=1000), lib)
    assert pg == [1000 * 8 * 64 * 128] * 2 + [1000 * 8 * 8, 16, 512]
    assert spla.attend8_workspace_bytes(cfg(), 0, lib) >= 0
    assert spla.attend8_workspace_bytes(cfg(), 1, lib) % 256 == 0
    assert spla.norm_rotate_grad_workspace_bytes(cfg(), 0, lib) == 0
    one = spla.norm_rotate_grad_workspace_bytes(cfg(), 1, lib)
    assert one == 4 * 40 * 128 * 8  # a record of fp64 sums per position, up to a number of runs
    assert spla.norm_rotate_grad_workspace_bytes(cfg(), 1 << 30, lib) < 1 << 30
    for fn in (lib.spla_attend8_workspace_bytes, lib.spla_norm_rotate_grad_workspace_bytes):
        n = ctypes.c_size_t(0)
        assert fn(ctypes.byref(cfg()), -1, ctypes.byref(n)) == -1
        assert fn(ctypes.byref(cfg()), 1, None) == -1
        assert fn(None, 1, ctypes.byref(n)) == -1
    n = ctypes.c_size_t(0)
    assert lib.spla_attend8_workspace_bytes(ctypes.byref(cfg()), 131073, ctypes.byref(n)) == -3
    assert lib.spla_cache8_bytes(ctypes.byref(cfg()), None) == -1
    assert lib.spla_cache8_bytes(ctypes.byref(cfg(head_dim=96)), (ctypes.c_size_t * 5)()) == -2


def cache8(**kw):
    c = spla.SplaCache8Struct(*([4096] * 5), None, None)
    for k, v in kw.items():
        setattr(c, k, v)
    return ctypes.byref(c)


def test_cache_calls_refuse():
    lib, c = spla.lib(), ctypes.byref(cfg())
    paged = ctypes.byref(cfg(kv_pages=64))
    row = 8 * 128
    for bad in (dict(k_codes=None), dict(v_codes=None), dict(scales=None), dict(seq_lens=None),
                dict(counters=None), dict(k_codes=4097), dict(v_codes=4104),
                dict(block_table=4096)):
        assert lib.spla_append8(c, cache8(**bad), 1, 4096, row, 4096, row, None, None) == -1
        assert lib.spla_read8(c, cache8(**bad), 1, None, 4096, 8192, None) == -1
        assert lib.spla_attend8(c, cache8(**bad), 1, 4096, None, 8192, None, None, 0, None) == -1
        assert lib.spla_reset8(c, cache8(**bad), None) == -1
    assert lib.spla_append8(paged, cache8(), 1, 4096, row, 4096, row, None, None) == -1
    assert lib.spla_append8(None, cache8(), 1, 4096, row, 4096, row, None, None) == -1
    assert lib.spla_append8(c, None, 1, 4096, row, 4096, row, None, None) == -1
    # rows: missing, misaligned, strides that hold no row or are no multiple of 16 bytes
    for k, ks, v, vs in ((None, row, 4096, row), (4096, row, None, row), (4100, row, 4096, row),
                         (4096, row - 8, 4096, row), (4096, row, 4096, row + 4),
                         (4096, -row, 4096, row)):
        assert lib.spla_append8(c, cache8(), 1, k, ks, v, vs, None, None) == -1
    assert lib.spla_append8(c, cache8(), -1, 4096, row, 4096, row, None, None) == -1
    assert lib.spla_append8(c, cache8(), 131073, 4096, row, 4096, row, None, None) == -3
    assert lib.spla_append8(c, cache8(), 0, None, 0, None, 0, None, None) == 0
    for args in ((-1, None, 4096, 8192), (1, None, None, None), (1, None, 4100, 8192),
                 (1, None, 4096, 8200), (1, None, 4096, 4096)):
        assert lib.spla_read8(c, cache8(), *args, None) == -1
    assert lib.spla_read8(c, cache8(), 0, None, None, None, None) == 0


def test_attend8_refuses():
    lib, c = spla.lib(), ctypes.byref(cfg())

    def call(n=1, q=4096, out=8192, ws=4096, size=1 << 40, **kw):
        o = spla.SplaAttend8Opts(spla.SplaAttendOpts(kw.pop("softcap", 0.0)))
        for k, v in kw.items():
            setattr(o, k, v)
        return lib.spla_attend8(c, cache8(), n, q, ctypes.byref(o), out, None, ws, size, None)

    assert call(n=-1) == -1 and call(n=131073) == -3 and call(n=0) == 0
    assert call(window=-1) == -1 and call(window=4, sinks=-1) == -1
    for cap in (-1.0, 2.0 ** -11, 1025.0, math.nan, math.inf):
        assert call(softcap=cap) == -1
    assert call(q=None) == -1 and call(out=None) == -1 and call(out=4096) == -1
    assert call(q=4100) == -1 and call(out=8200) == -1
    assert call(ws=None) == -4 and call(size=16) == -4 and call(ws=4100) == -4


def test_norm_refuses():
    lib, cf = spla.lib(), cfg()
    c, rope = ctypes.byref(cf), spla.make_rope(128)
    r = ctypes.byref(rope)
    q, k = 32 * 128, 8 * 128
    ok = dict(rope=r, n=1, wq=None, wk=None, per=0, eps=1e-6, q=4096, qs=q, qo=8192, qos=q, k=4096,
              ks=k, ko=8192, kos=k)

    def fwd(**kw):
        a = ok | kw
        return lib.spla_norm_rotate(c, a["rope"], a["n"], None, None, a["wq"], a["wk"], a["per"],
                                    a["eps"], a["q"], a["qs"], a["qo"], a["qos"], a["k"], a["ks"],
                                    a["ko"], a["kos"], None)

    def bwd(gq=4096, gqs=q, gk=4096, gks=k, dwq=None, dwk=None, ws=None, size=0, **kw):
        a = ok | kw
        return lib.spla_norm_rotate_grad(c, a["rope"], a["n"], None, None, a["wq"], a["wk"],
                                         a["per"], a["eps"], a["q"], a["qs"], gq, gqs, a["qo"],
                                         a["qos"], a["k"], a["ks"], gk, gks, a["ko"], a["kos"], dwq,
                                         dwk, ws, size, None)

    bad = [dict(rope=None), dict(rope=ctypes.byref(spla.make_rope(64))), dict(n=-1), dict(per=2),
           dict(eps=-1e-9), dict(eps=math.nan), dict(eps=math.inf), dict(wq=4100), dict(wk=4104),
           dict(q=None), dict(qo=None), dict(k=None), dict(ko=None), dict(q=4100), dict(ko=8200),
           dict(qs=q - 8), dict(kos=k + 4), dict(q=8192, qos=q + 8),
           dict(q=None, qo=None, k=None, ko=None)]
    for b in bad:
        assert fwd(**b) == -1, b
        assert bwd(**b) == -1, b
    assert fwd(n=0) == 0 and bwd(n=0) == 0
    for b in (dict(gq=None), dict(gk=None), dict(gq=4100), dict(gks=k - 8), dict(gq=8192, gqs=q + 8),
              dict(q=None, qo=None, gq=None, dwq=4096, ws=4096, size=1 << 30)):
        assert bwd(**b) == -1, b
    assert bwd(dwq=4096) == -4 and bwd(dwk=4096, ws=4096, size=100) == -4
    assert bwd(dwk=4096, ws=4100, size=1 << 30) == -4


def test_binding_refuses():
    """Shapes, types and devices, on CPU tensors: nothing reaches the library."""
    cf = spla.make_config(2, 4, 2, 64, 32, 8, 64, "bf16")
    rope = spla.make_rope(64)
    q, k = (torch.zeros(3, 2, h, 64, dtype=torch.bfloat16) for h in (4, 2))
    w = torch.ones(64)
    bad = [dict(), dict(q=q[0, 0]), dict(q=q.float()), dict(q=q[:, :1]), dict(q=q, k=k[:2]),
           dict(q=q, k=q), dict(q=q, q_out=k), dict(k=k, q_out=q), dict(q=q, q_weight=w.half()),
           dict(q=q, q_weight=w[:32]), dict(q=q, k=k, q_weight=w, k_weight=torch.ones(2, 64)),
           dict(q=q, q_weight=torch.ones(4, 128)[:, ::2]),
           dict(q=q, q_weight=w.clone().requires_grad_()), dict(q=q.clone().requires_grad_()),
           dict(q=q, positions=torch.zeros(3, 2)), dict(q=q, seq_lens=torch.zeros(3).int()),
           dict(q=q.transpose(2, 3).contiguous().transpose(2, 3)), dict(q=q, k=k)]
    for kw in bad:  # (the last one: not on a GPU)
        with pytest.raises(ValueError):
            spla.norm_rotate(cf, rope, **kw)
    bad = [dict(q=q), dict(q_grad=q), dict(q=q, q_grad=q, k_weight=w),
           dict(q=q, q_grad=q, k_grad=k), dict(q=q, q_grad=q, k_out=k),
           dict(q=q, q_grad=k), dict(q=q, q_grad=q.float()), dict(q=q, q_grad=q)]
    for kw in bad:
        with pytest.raises(ValueError):
            spla.norm_rotate_grad(cf, rope, **kw)


def layout(d, which, t, c):
    """Byte of number (t, c) of a slot as include/spla.h documents it."""
    tt, step = t % 32, t // 32
    if which == "k":
        chunk = (tt // 4 % 2 * (d // 64) + c // 64) * 64 + c // 16 % 4 * 16 + 4 * (tt // 8) + tt % 4
        return step * 32 * d + 16 * chunk + c % 16
    chunk = c // 32 * 64 + tt // 8 * 16 + c % 16
    return step * 32 * d + 16 * chunk + 8 * (c // 16 % 2) + tt % 8


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("which", ["k", "v"])
def test_layout_is_one_to_one(d, which):
    at = {layout(d, which, t, c) for t in range(128) for c in range(d)}
    assert at == set(range(128 * d))


def test_reference_codes():
    """The reference's own rounding, pinned by the definition."""
    v = C.code_values()
    assert v[0x7E] == 448.0 and v[1] == 2.0 ** -9 and v[0x38] == 1.0 and math.isnan(v[0xFF])
    x = torch.tensor([1.0625, 1.1875, 464.0, 1e30, 2.0 ** -10, 2.0 ** -10 * 1.001, 3 * 2.0 ** -10,
                      -17.0, -19.0, math.inf])
    want = [1.0, 1.25, 448.0, 448.0, 0.0, 2.0 ** -9, 2.0 ** -8, -16.0, -20.0]
    got = C.to_codes(x)
    assert got[:-1].tolist() == want and math.isnan(got[-1])
    fin = v[torch.isfinite(v)]
    assert torch.equal(C.to_codes(fin), fin)
    assert [C.exponent(a) for a in (0.0, 448.0, 448.1, 1.75, 1.0, 3.4e38)] == [
        -100, 0, 1, -8, -8, 119]
