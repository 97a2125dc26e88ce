"""Rotations in place beside autograd."""

import pytest
import torch

from paper_2601_22379_amd import spla

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("which", ["q", "k", "both"])
def test_in_place_is_seen_by_autograd(which):
    """A product has kept rows that are then rotated in place: its gradient would be that of
    other rows, so its backward pass refuses, as after any operation of torch in place."""
    cfg, rope = spla.make_config(2, 4, 4, 128, 64, 8, 1024, "bf16"), spla.make_rope(128)
    q, k = (torch.randn(3, 2, 4, 128, device="cuda").bfloat16() for _ in range(2))
    for rows, name in ((q, "q"), (k, "k")):
        w = torch.ones(128, device="cuda", dtype=torch.bfloat16, requires_grad=True)
        z = (rows * w).sum()
        kw = {}
        if which in ("q", "both"):
            kw.update(q=q, q_out=q)
        if which in ("k", "both"):
            kw.update(k=k, k_out=k)
        spla.rotate(cfg, rope, **kw)
        if which in (name, "both"):
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                z.backward()
        else:
            z.backward()
            want = rows.double().sum((0, 1, 2))
            # 24 terms, summed in fp32 at least once and rounded to bf16 at each of three axes
            tol = 4 * 2.0 ** -8 * rows.double().abs().sum((0, 1, 2))
            assert bool(((w.grad.double() - want).abs() <= tol).all())


def test_in_place_under_inference_mode():
    cfg, rope = spla.make_config(2, 4, 4, 128, 64, 8, 1024, "bf16"), spla.make_rope(128)
    with torch.inference_mode():
        q = torch.randn(3, 2, 4, 128, device="cuda").bfloat16()
        want, _ = spla.rotate(cfg, rope, q)
        spla.rotate(cfg, rope, q, q_out=q)
        assert torch.equal(q, want)
    spla.rotate(cfg, rope, q, q_out=q)  # a tensor of inference mode outside it
