"""The rotating append in a workspace of just the bytes its rotation needs."""

import ctypes

import pytest
import torch

from paper_2601_22379_amd import spla

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,rot,dtype,T", [(128, 128, "bf16", 700), (128, 32, "bf16", 65),
                                           (128, 40, "bf16", 700), (64, 64, "bf16", 130),
                                           (64, 48, "f32", 77), (128, 128, "bf16", 1)])
def test_exact_workspace(d, rot, dtype, T):
    dev = torch.device("cuda:0")
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    cfg = spla.make_config(2, 4, 2, d, 64, 8, 1024, dtype)
    one, two = spla.SplaCache(cfg, dev), spla.SplaCache(cfg, dev)
    rope = spla.make_rope(d, rot)
    g = torch.Generator(device=dev)
    g.manual_seed(T)
    k, v = (torch.randn(2, 2, T, d, generator=g, device=dev).to(dt) for _ in range(2))
    need = spla.append_rope_workspace_bytes(cfg, T, rope=rope)
    ws = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device=dev)
    ws[:need] = 0
    for _ in range(1 if T > 500 else 3):
        one.append_rope(rope, k, v)
        assert spla.lib().spla_append_rope(
            ctypes.byref(cfg), ctypes.byref(two.struct), ctypes.byref(rope), k.data_ptr(),
            v.data_ptr(), T, None, None, ws.data_ptr(), need,
            torch.cuda.current_stream().cuda_stream) == 0
    assert bool((ws[need:] == 0xA5).all())
    for x, y in ((one.k, two.k), (one.v, two.v), (one.stats, two.stats), (one.state, two.state),
                 (one.norm, two.norm), (one.seq_lens, two.seq_lens)):
        assert torch.equal(x, y)
    assert spla.lib().spla_append_rope(
        ctypes.byref(cfg), ctypes.byref(two.struct), ctypes.byref(rope), k.data_ptr(), v.data_ptr(),
        T, None, None, ws.data_ptr(), need - 1, torch.cuda.current_stream().cuda_stream) == -4
    two.append_rope(rope, k[:, :, :1].contiguous(), v[:, :, :1].contiguous())
    assert two._rope_ws.numel() == spla.append_rope_workspace_bytes(cfg, 1, rope=rope)


def test_default_device():
    """A cache made without naming a device, from a page table on the current one."""
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(1, 8)
    cache = spla.SplaCache(spla.make_config(1, 4, 2, 128, 64, 8, 512, "bf16", kv_pages=8),
                           block_table=table)
    assert cache.device == table.device == cache.seq_lens.device
    k = torch.randn(1, 2, 70, 128, device="cuda").bfloat16()
    cache.append_rope(spla.make_rope(128), k, k)
    out, lse = cache.attend(torch.zeros(1, 4, 128, dtype=torch.bfloat16, device="cuda"))
    # equal weights: fp32 sums of 70 of them, the result rounded once (2^-8 of the largest)
    want = k.float().mean(2).repeat_interleave(2, 1)
    assert bool(((out.float() - want).abs() <= 2.0 ** -8 * k.abs().max().float()).all())
    assert bool((lse.cpu() - torch.log(torch.tensor(70.0))).abs().max() < 1e-5)
