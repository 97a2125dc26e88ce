"""Blocks of an 8-bit cache whose block table entry names no page: the read-back."""

import ctypes

import pytest
import torch

import cache8_ref as C
from paper_2601_22379_amd import spla

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spla.lib()
    return torch.device("cuda:0")


@pytest.mark.parametrize("dtype,d,B", [("bf16", 128, 32), ("bf16", 64, 128), ("f32", 64, 64),
                                       ("f32", 128, 32)])
def test_no_rows_of_another_sequence(dev, dtype, d, B):
    """A block without a page is held by nobody: the read-back gives zeros for it and says so in
    the error word, and never the rows of page 0, another sequence's."""
    b, hkv, nb = 3, 2, 4
    cap = nb * B
    pages = b * nb
    table = torch.arange(pages, dtype=torch.int32).view(b, nb)  # page 0: sequence 0's first block
    bad = {(0, 2): -1, (1, 0): pages, (1, 3): 2 ** 31 - 1, (2, 1): -2 ** 31}
    for at, p in bad.items():
        table[at] = p
    cfg = spla.make_config(b, hkv, hkv, d, B, 8, cap, dtype, kv_pages=pages)
    cache = spla.SplaCache8(cfg, dev, block_table=table.to(dev))
    g = torch.Generator().manual_seed(1)
    k, v = ((torch.randn((cap, b, hkv, d), generator=g) + 3.0).to(DT[dtype]) for _ in range(2))
    lens = [cap, cap - 5, cap - B + 1]
    K, V = C.Held(b, hkv, d, B, cap), C.Held(b, hkv, d, B, cap)
    K.append(k, lens, [0] * b)
    V.append(v, lens, [0] * b)
    cache.append(k.to(dev), v.to(dev), torch.tensor(lens, dtype=torch.int32, device=dev))
    assert cache.device_errors() == spla.DEVERR_PAGE and cache.seq_lens.tolist() == lens
    for (i, blk) in bad:
        K.x[i, :, blk * B:(blk + 1) * B] = 0.0
        V.x[i, :, blk * B:(blk + 1) * B] = 0.0
    for first in ([0] * b, [7, B - 3, 1 - B]):
        cache.clear_device_errors()
        got = cache.read(cap + 3, torch.tensor(first, dtype=torch.int32, device=dev))
        for x, held in zip(got, (K, V)):
            for i in range(b):
                at = torch.arange(cap + 3) + first[i]
                ok = (at >= 0) & (at < lens[i])
                want = held.x[i][:, at.clamp(0, cap - 1)].transpose(0, 1).clone()
                want[~ok] = 0.0
                assert torch.equal(x[:, i].cpu().double(), want), (first, i)
        assert cache.device_errors() == spla.DEVERR_PAGE
    # nothing of a bad block is asked for: no error
    cache.clear_device_errors()
    cache.read(B, torch.tensor([0, B, 0], dtype=torch.int32, device=dev))
    assert cache.device_errors() == 0
    # no error word, and one of the two arrays
    out = torch.full((cap, b, hkv, d), 7.0, dtype=DT[dtype], device=dev)
    c = cache.struct
    plain = spla.SplaCache8Struct(c.k_codes, c.v_codes, c.scales, c.seq_lens, c.counters, None,
                                  c.block_table)
    assert spla.lib().spla_read8(ctypes.byref(cfg), ctypes.byref(plain), cap, None, None,
                                 out.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
    assert cache.device_errors() == 0
    assert not out[:B, 1].any() and torch.equal(out[:lens[2]], cache.read(lens[2])[1])
