"""scaled_matmul with scales over the whole range of fp32: the terms are what has to be in range, not the product of two scales.

Tolerance: test_gpu_block_ops' (roundings of the result and of the sums, relative), and half a step of the smallest numbers for each
block's term and for the result.
"""
import numpy as np
import pytest
import torch

from oracle import block_oracle as blk
from tests.test_gpu_block_ops import SIMT, _built, handle, np64, operands, product_bound  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("flags", [0, SIMT])
@pytest.mark.parametrize("m", [1, 3, 30, 60, 100, 300])
def test_scales_whose_product_is_out_of_range(handle, dtype, flags, m):
    """Three kinds of rows side by side.  Even blocks of channels: ordinary scales, products below the normal numbers whose terms are normal,
    large ones.  Odd blocks, whose weights' scale is 3e38: a scale of 1e-38, zero, and one that takes the product to infinity where
    the row's values are zeros."""
    n, k = 200, 391
    x = operands(m, n, k, dtype, seed=m, bias=False, add=False)
    g = torch.Generator().manual_seed(m)
    some = torch.exp(0.5 * torch.randn(m, 4, generator=g))
    kind = (torch.arange(m) + (0 if m > 1 else 1)) % 3
    even = torch.tensor([1.0, 2.0 ** -126, 2.0 ** 90])[kind]
    odd = torch.tensor([1e-38, 0.0, 2.0 ** 100])[kind]
    scale = some.double() * torch.stack([even, odd, even, odd], 1).double()
    x["a_scale"] = scale.float().cuda()
    sw = torch.tensor([1.37 * 2.0 ** -12, 3e38, 1.9 * 2.0 ** -12, 2.9e38])
    x["w_scale"] = torch.stack([sw, sw.flip(0).roll(1, 0).flip(0).roll(1, 0)]).cuda().contiguous()
    a = x["a"].float()
    wide = torch.zeros(m, k, dtype=torch.bool, device=a.device)
    wide[:, 128:256], wide[:, 384:] = True, True
    a[wide & (kind == 2).to(a.device)[:, None]] = 0
    room = torch.zeros(m, 400, dtype=x["a"].dtype, device=a.device)
    room[:, :k] = a.to(x["a"].dtype)
    x["a"] = room[:, :k]
    want, size = blk.scaled_matmul(*(np64(x[i]) for i in ("a", "a_scale", "w", "w_scale", "bias", "add")))
    got = np64(handle(dtype, flags=flags).scaled_matmul(**x))
    assert np.isfinite(want).all() and (np.abs(want) < 3e38).all()
    least = 4 * 2.0 ** -150 + (2.0 ** -134 if dtype == "bf16" else 2.0 ** -150)
    off = np.abs(got - want) / (product_bound(want, size, dtype, k) + least)
    assert np.isfinite(got).all() and off.max() <= 1, (off.max(1), kind)


def test_signs_and_what_is_not_finite(handle):
    """Negative scales; an infinite or NaN scale reaches what it scales and nothing else."""
    for m in (5, 100, 300):
        x = operands(m, 150, 256, "f32", seed=m, bias=False, add=False)
        x["a_scale"] = x["a_scale"] * torch.where(torch.arange(m) % 2 == 0, -1e-30, 1e20).cuda()[:, None]
        x["w_scale"] = x["w_scale"] * torch.tensor([-1e-11, 1e-11]).cuda()[None]
        want, size = blk.scaled_matmul(*(np64(x[i]) for i in ("a", "a_scale", "w", "w_scale", "bias", "add")))
        vda = handle("f32")
        got = np64(vda.scaled_matmul(**x))
        assert (np.abs(got - want) <= product_bound(want, size, "f32", 256) + 6 * 2.0 ** -150).all()
        first = vda.scaled_matmul(**x)
        x["a_scale"][3, 1], x["a_scale"][4, 0] = float("inf"), float("nan")
        bad = vda.scaled_matmul(**x)
        rest = [i for i in range(m) if i not in (3, 4)]
        assert not bad[3:5].isfinite().any() and bad[rest].equal(first[rest])
