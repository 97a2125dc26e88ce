"""Rotary positions and exact attention on the CPU: the rotation's frequencies,
workspace sizes, and the calls that the host checks refuse before any launch."""

import ctypes
import math

import pytest
import torch

import rope_attend_ref as R
from paper_2601_22379_amd import spla


def _lib(name):
    return spla.lib() if name == "hip" else spla.host_lib()


def _cfg(**kw):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, block_size=64, top_k=8,
                max_seq_len=4096, dtype="bf16")
    base.update(kw)
    return spla.make_config(**base)


FAKE = spla.SplaCacheStruct(*([256] * 6), None)


@pytest.mark.parametrize("libname", ["hip", "host"])
@pytest.mark.parametrize("kw", [
    dict(rot=128), dict(rot=2), dict(rot=50, base=5e5), dict(rot=64, scaling="linear", factor=4.0),
    dict(rot=128, scaling="base", factor=8.0), dict(rot=2, scaling="base", factor=8.0),
    dict(rot=128, base=5e5, scaling="parts", factor=8.0, orig_len=8192.0, low=1.0, high=4.0),
])
def test_frequencies(libname, kw):
    rot = kw["rot"]
    r = spla.make_rope(128, rot_dim=rot, library=_lib(libname),
                       **{k: v for k, v in kw.items() if k != "rot"})
    want = R.frequencies(**kw) / (2.0 * math.pi)
    got = list(r.turns)[:rot // 2]
    # pow, and up to four products, each within a few fp64 steps; the exponent's rounding is
    # magnified by ln(base) <= 16
    assert all(abs(g - w) <= 2.0 ** -47 * w for g, w in zip(got, want))
    assert list(r.turns)[rot // 2:] == [0.0] * (64 - rot // 2)
    assert (r.head_dim, r.rot_dim, r.gain) == (128, rot, 1.0)


@pytest.mark.parametrize("kw,want", [
    (dict(head_dim=96), -2), (dict(rot_dim=3), -1), (dict(rot_dim=0), -1), (dict(rot_dim=130), -1),
    (dict(layout=2), -1), (dict(scaling=4), -1), (dict(scaling=-1), -1), (dict(base=1.0), -1),
    (dict(base=float("nan")), -1), (dict(base=float("inf")), -1), (dict(gain=float("inf")), -1),
    (dict(scaling="linear", factor=0.5), -1), (dict(scaling="base", factor=float("nan")), -1),
    (dict(scaling="parts", factor=2.0, orig_len=0.0), -1),
    (dict(scaling="parts", factor=2.0, orig_len=100.0, low=4.0, high=4.0), -1),
])
def test_rotations_refused(kw, want):
    for name in ("hip", "host"):
        with pytest.raises(spla.SplaError) as e:
            spla.make_rope(**{"head_dim": 128, "library": _lib(name), **kw})
        assert e.value.status == want
    assert spla.host_lib().spla_rope_init(None, None) == -1


def test_workspace_sizes():
    for lib in (spla.lib(), spla.host_lib()):
        c = _cfg()
        ap = spla.append_workspace_bytes(c, 100, lib)
        assert spla.append_rope_workspace_bytes(c, 100, lib) >= ap
        for n in (0, 1, 17, 4096):
            assert spla.attend_workspace_bytes(c, n, lib) % 256 == 0
        for f in (spla.append_rope_workspace_bytes, spla.attend_workspace_bytes):
            for n, want in ((-1, -1), (4097, -3)):
                with pytest.raises(spla.SplaError) as e:
                    f(c, n, lib)
                assert e.value.status == want
    # sizes are products of 64-bit numbers: 1 M tokens of 64 sequences of 16 KV heads
    big = _cfg(batch=64, n_q_heads=16, n_kv_heads=16, max_seq_len=1 << 20)
    assert spla.append_rope_workspace_bytes(big, 1 << 20) > 64 * 16 * (1 << 20) * 128 * 2
    # the partial results stay small whatever the shape
    assert all(spla.attend_workspace_bytes(big, n) < 256 << 20 for n in (1, 16, 4096, 1 << 20))


def _rotate(cfg, rope, n=1, q=256, qs=1024, qo=512, qos=1024, k=None, ks=0, ko=None, kos=0, tr=0):
    return spla.lib().spla_rotate(ctypes.byref(cfg), ctypes.byref(rope) if rope else None, n, None,
                                  None, q, qs, qo, qos, k, ks, ko, kos, tr, None)


def test_rotate_refuses():
    c, r = _cfg(), spla.make_rope(128)
    assert _rotate(c, r, n=0) == 0
    assert _rotate(c, r, n=-1) == -1
    assert _rotate(c, None) == -1
    assert _rotate(c, spla.make_rope(64)) == -1            # another head size
    assert _rotate(c, spla.SplaRope()) == -1               # never initialised
    assert _rotate(_cfg(n_q_heads=9), r) == -1
    assert _rotate(c, r, tr=2) == -1
    assert _rotate(c, r, q=None, qo=None) == -1            # nothing to rotate
    assert _rotate(c, r, qo=None) == -1 and _rotate(c, r, q=None) == -1
    assert _rotate(c, r, ko=256) == -1 and _rotate(c, r, k=256, ks=256) == -1
    assert _rotate(c, r, q=264) == -1 and _rotate(c, r, qo=520) == -1   # 8-byte aligned
    assert _rotate(c, r, qs=1023) == -1 and _rotate(c, r, qs=1028) == -1  # short; 8 bytes over
    assert _rotate(c, r, qos=1016) == -1
    assert _rotate(c, r, qo=256, qos=2048) == -1           # in place with another stride
    assert _rotate(c, r, k=256, ks=255, ko=512, kos=256) == -1


def test_append_rope_refuses():
    lib, c, r = spla.lib(), _cfg(), spla.make_rope(128)

    def call(cfg=c, cache=FAKE, rope=r, k=256, v=256, n=4, ws=256, size=1 << 40):
        return lib.spla_append_rope(ctypes.byref(cfg), ctypes.byref(cache) if cache else None,
                                    ctypes.byref(rope) if rope else None, k, v, n, None, None, ws,
                                    size, None)
    assert call(n=0) == 0
    assert call(n=-1) == -1 and call(n=4097) == -3
    assert call(k=None) == -1 and call(v=None) == -1 and call(k=264) == -1 and call(v=258) == -1
    assert call(rope=None) == -1 and call(rope=spla.make_rope(64)) == -1
    assert call(cache=None) == -1 and call(cache=spla.SplaCacheStruct()) == -1
    assert call(ws=None) == -4 and call(ws=264) == -4 and call(size=16) == -4
    assert call(cfg=_cfg(kv_pages=64)) == -1               # a pool without its table
    assert call(cfg=_cfg(top_k=2)) == -1


def test_attend_refuses():
    lib, c = spla.lib(), _cfg()

    def call(cfg=c, cache=FAKE, n=4, q=256, out=512, ws=256, size=1 << 40, cap=0.0):
        o = spla.SplaAttendOpts(cap, 0.0, None, None, None, None)
        return lib.spla_attend(ctypes.byref(cfg), ctypes.byref(cache) if cache else None, n, q,
                               ctypes.byref(o), out, None, ws, size, None)
    assert call(n=0) == 0 and call(n=0, q=None, out=None) == 0
    assert call(n=-1) == -1 and call(n=4097) == -3
    assert call(q=None) == -1 and call(out=None) == -1 and call(out=256) == -1
    assert call(q=264) == -1 and call(out=520) == -1
    assert call(cache=None) == -1 and call(cache=spla.SplaCacheStruct()) == -1
    for bad in (-1.0, float("nan"), float("inf"), 2.0 ** -11, 1025.0, 1e-40):
        assert call(cap=bad) == -1
    need = spla.attend_workspace_bytes(c, 4)
    assert need > 0
    assert call(ws=None) == -4 and call(ws=264) == -4 and call(size=need - 1) == -4
    assert call(cfg=_cfg(kv_pages=64)) == -1 and call(cfg=_cfg(head_dim=96)) == -2


def test_binding_checks_rows():
    c, r = _cfg(), spla.make_rope(128)
    q = torch.zeros(3, 2, 8, 128, dtype=torch.bfloat16)
    for bad in (dict(q=q[:, :, :7]), dict(q=q.float()), dict(q=q[:, :1]), dict(),
                dict(q=q.transpose(0, 1).contiguous().transpose(0, 1)),  # rows not evenly spaced
                dict(q=q, q_out=q[:2]), dict(k_out=q), dict(q=q, k=q[:2, :, :2]),
                dict(q=q, seq_lens=torch.zeros(2)), dict(q=q, positions=torch.zeros(5).int()),
                dict(q=q[..., ::2])):
        with pytest.raises(ValueError):
            spla.rotate(c, r, **bad)


def test_rows_on_the_host_are_refused():
    q = torch.zeros(3, 2, 8, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        spla.rotate(_cfg(), spla.make_rope(128), q=q)


def test_a_workspace_does_not_grow_in_a_capture(monkeypatch):
    """A fill recorded by the capture would leave the counters of other calls undefined until
    the first replay."""
    cache = object.__new__(spla.SplaCache)
    cache.cfg, cache.device = _cfg(), torch.device("cpu")
    cache._ws_sizes, cache._outgrown = {}, []

    def sizes(cfg, n):
        return 256 * n
    monkeypatch.setattr(spla, "_aligned_workspace",
                        lambda n, device: torch.empty(n, dtype=torch.uint8))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    ws = cache._workspace("attend", 4, sizes, None)
    assert ws.numel() >= 1024 and not ws.any()
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    assert cache._workspace("attend", 3, sizes, ws) is ws
    with pytest.raises(RuntimeError):
        cache._workspace("attend", 5, sizes, ws)
    with pytest.raises(RuntimeError):
        cache._workspace("rope", 1, sizes, None)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    assert cache._workspace("attend", 5, sizes, ws).numel() >= 1280 and cache._outgrown[0] is ws


def _growing(monkeypatch, capturing):
    """A cache's workspaces on the CPU: (cache, sizes) with 256 bytes per token."""
    cache = object.__new__(spla.SplaCache)
    cache.cfg, cache.device = _cfg(), torch.device("cpu")
    cache._ws_sizes, cache._outgrown = {}, []
    monkeypatch.setattr(spla, "_aligned_workspace",
                        lambda n, device: torch.empty(n, dtype=torch.uint8))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing[0])
    return cache, lambda cfg, n: 256 * n


def test_outgrown_workspaces_are_let_go(monkeypatch):
    """Prompts that get longer one by one: one workspace is kept, of at most half as much again
    as the largest call needs, made anew a few times only."""
    cache, sizes = _growing(monkeypatch, [False])
    ws, made = None, 0
    for n in range(1, 400):
        new = cache._workspace("rope", n, sizes, ws)
        made, ws = made + (new is not ws), new
        assert 256 * n <= ws.numel() <= 256 * n * 3 // 2
    assert cache._outgrown == [] and made <= 18  # log(400) / log(1.5), and the first small ones


def test_captured_workspaces_are_kept(monkeypatch):
    """A graph names the workspace of its capture: that one stays, the others do not."""
    on = [False]
    cache, sizes = _growing(monkeypatch, on)
    ws = cache._workspace("rope", 4, sizes, None)
    on[0] = True
    assert cache._workspace("rope", 4, sizes, ws) is ws
    assert cache._workspace("rope", 3, sizes, ws) is ws
    on[0] = False
    big = cache._workspace("rope", 100, sizes, ws)
    bigger = cache._workspace("rope", 1000, sizes, big)
    assert bigger is not big is not ws
    assert len(cache._outgrown) == 1 and cache._outgrown[0] is ws


@pytest.mark.parametrize("libname", ["hip", "host"])
def test_workspace_of_one_rotation(libname):
    """Keys that are rotated in registers need no room for the rotated rows; the query for any
    rotation is the largest."""
    lib, rows = _lib(libname), 2 * 2 * 1000 * 128 * 2
    for kw, rot, saved in ((dict(), 128, rows), (dict(), 48, rows), (dict(), 40, 0), (dict(), 2, 0),
                           (dict(head_dim=64), 64, 0), (dict(dtype="f32"), 128, 0),
                           (dict(sel_window=32, sel_stride=16), 128, 0)):
        c = _cfg(**kw)
        rope = spla.make_rope(c.head_dim, rot, library=lib)
        got = spla.append_rope_workspace_bytes(c, 1000, lib, rope)
        assert got + saved == spla.append_rope_workspace_bytes(c, 1000, lib)
        assert got % 256 == 0 and got >= spla.append_workspace_bytes(c, 1000, lib)
    n = ctypes.c_size_t(0)
    for bad in (spla.SplaRope(), spla.make_rope(64, library=lib)):
        assert lib.spla_append_rope_workspace_bytes_ex(ctypes.byref(_cfg()), ctypes.byref(bad), 4,
                                                       ctypes.byref(n)) == -1
    assert lib.spla_append_rope_workspace_bytes_ex(ctypes.byref(_cfg()), None, 4, None) == -1


def test_positions_of_another_shape_are_refused():
    """Position ids as [batch, T] have the right count, and would turn rows by others' angles."""
    c, r = _cfg(), spla.make_rope(128)
    q = torch.zeros(3, 2, 8, 128, dtype=torch.bfloat16)
    ids = torch.arange(6).int()
    for bad in (ids.view(2, 3), ids, ids.view(3, 2, 1)):
        with pytest.raises(ValueError, match="positions"):
            spla.rotate(c, r, q=q, positions=bad)
    with pytest.raises(ValueError, match="positions"):
        spla.rotate(c, r, q=q[0], positions=ids[:2].view(2, 1))
    for bad in (ids[:2].view(2, 1), ids[:2].view(1, 2)):
        with pytest.raises(ValueError, match="seq_lens"):
            spla.rotate(c, r, q=q, seq_lens=bad)
    for ok in (dict(q=q, positions=ids.view(3, 2)), dict(q=q[0], positions=ids[:2]),
               dict(q=q[0], positions=ids[:2].view(1, 2)),
               dict(q=q, seq_lens=ids[:2])):
        with pytest.raises(ValueError, match="on a GPU"):  # all else is right
            spla.rotate(c, r, **ok)


def test_rows_that_record_a_gradient_are_refused():
    """The results lie outside autograd's graph, and a rotation in place would change a tensor
    that a recorded product has kept."""
    c, r = _cfg(), spla.make_rope(128)
    q = torch.zeros(3, 2, 8, 128, dtype=torch.bfloat16)
    k, leaf = q[:, :, :2].contiguous(), q.clone().requires_grad_(True)
    for bad in (dict(q=leaf), dict(q=leaf * 2), dict(q=q, q_out=leaf), dict(q=leaf, q_out=leaf),
                dict(q=q, k=k.clone().requires_grad_(True)), dict(k=k, k_out=leaf[:, :, :2])):
        with pytest.raises(ValueError, match="gradient"):
            spla.rotate(c, r, **bad)
        with pytest.raises(ValueError, match="on a GPU"), torch.no_grad():  # all else is right
            spla.rotate(c, r, **bad)
    with pytest.raises(ValueError, match="on a GPU"):
        spla.rotate(c, r, q=leaf.detach(), transpose=True)


def test_a_device_without_an_index_is_the_one_it_named_then(monkeypatch):
    """A cache made on "cuda" stays on the device that was current, whichever is later: its calls
    launch there, and its workspaces lie there."""
    at = [3]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: at[0])
    device = spla._indexed("cuda")
    at[0] = 5
    assert device == torch.device("cuda:3") and device.index == 3
    assert spla._indexed("cuda:1") == torch.device("cuda:1")
    assert spla._indexed(torch.device("cuda")) == torch.device("cuda:5")
    assert spla._indexed("cpu") == torch.device("cpu")
