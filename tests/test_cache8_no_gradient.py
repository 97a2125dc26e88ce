"""The 8-bit cache's calls record nothing for autograd: rows that it would record are refused (on
CPU tensors: nothing reaches the library)."""

import pytest
import torch

from paper_2601_22379_amd import spla


@pytest.fixture
def launched(monkeypatch):
    calls = []
    monkeypatch.setattr(spla, "_launch", lambda fn, where, *rest: calls.append(where))
    monkeypatch.setattr(spla, "_aligned_workspace",
                        lambda n, device: torch.empty(n, dtype=torch.uint8))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    return calls


def rows(h, leaf=False):
    x = torch.zeros(3, 2, h, 64, dtype=torch.bfloat16)
    return x.requires_grad_() if leaf else x


def test_rows_that_record_a_gradient_are_refused(launched):
    cache = spla.SplaCache8(spla.make_config(2, 4, 2, 64, 32, 8, 64, "bf16"), "cpu")
    q, k, lse = rows(4), rows(2), torch.zeros(3, 2, 4)
    slopes = torch.zeros(4)
    ql, kl, ll, sl = rows(4, True), rows(2, True), lse.clone().requires_grad_(), \
        slopes.clone().requires_grad_()
    calls = [lambda: cache.append(kl, k), lambda: cache.append(k, kl),
             lambda: cache.append(kl * 2, k), lambda: cache.append(k[0], kl[0]),
             lambda: cache.attend(ql), lambda: cache.attend(ql * 2), lambda: cache.attend(ql[0]),
             lambda: cache.attend(q, out=ql), lambda: cache.attend(q, lse=ll),
             lambda: cache.attend(q, slopes=sl),
             lambda: cache.read(3, k_out=kl), lambda: cache.read(3, v_out=kl)]
    for call in calls:
        with pytest.raises(ValueError, match="no gradient is recorded"):
            call()
    assert launched == []
    with torch.no_grad():  # asked for: the numbers alone
        for call in calls:
            call()
    assert len(launched) == len(calls)
    cache.append(kl.detach(), k)
    cache.attend(q, q.clone(), lse, slopes=slopes)
    cache.read(3, k_out=k)
    assert len(launched) == len(calls) + 3
