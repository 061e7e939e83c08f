"""Tokens added behind a scale that others have chosen, which is no power of two: code = rint(x / scale) to the last tie."""
import math
from fractions import Fraction

import pytest
import torch

from batch_helpers import BF16, fill_cache, ints
from paper_2406_06237_b200.runtime import BlockCache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, BF16])
@pytest.mark.parametrize("scale", [0.3, 1.0 / 127, 0.0123456, 3.0, 1.9999999, 1.0000001, 7e-12, 5e20, 2.0 ** 126 * 1.7, 0.25])
def test_codes_at_and_beside_ties(dtype, scale):
    scale = float(torch.tensor(scale))
    n, heads, dim = 15, 2, 128
    steps = torch.arange(n * heads * dim, dtype=torch.float64) % 253 - 126               # -126 .. 126
    near = ((steps + 0.5 * torch.where(steps < 0, 1, -1)) * scale).float()
    near = torch.where(near.isfinite(), near, 0.0)
    bits = near.view(torch.int32)
    x = torch.cat([(bits + k).view(torch.float32).view(n, heads, dim)[k + 2::5] for k in (-2, -1, 0, 1, 2)])
    if dtype is BF16:
        x = near.view(n, heads, dim)
    x = x.to(dtype)
    holds = 127 * 2.0 ** (math.frexp(scale)[1] - 1)      # 127 steps of the power of two below: what the scale is kept for
    x = torch.where(x.isfinite() & (x.double().abs() <= holds), x, 0)
    arrays = fill_cache(2, heads, 16, dim)
    arrays[1][:], arrays[3][:] = scale, scale
    cache = BlockCache.wrap(*arrays)
    cache.write(x.cuda(), -x.cuda(), ints([[1]]), ints([1 + n]), ints([0, n]))
    assert cache.read_status() == 0 and (arrays[1][1] == scale).all()
    exact = Fraction(scale)
    want = torch.tensor([round(Fraction(float(v)) / exact) for v in x.flatten()], dtype=torch.int8).view(n, heads, dim).transpose(0, 1)
    assert torch.equal(arrays[0][1, :, 1:].cpu(), want) and torch.equal(arrays[2][1, :, 1:].cpu(), -want)
