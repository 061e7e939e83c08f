"""Adapters of rows that are not finite, at ranks that the kernels round up."""
import pytest
import torch

from batch_helpers import BF16, F64, ints, sums
from paper_2406_06237_b200.runtime import Adapters

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rank", [1, 8, 16, 24, 50, 100])
@pytest.mark.parametrize("new", [[1, 1, 1], [20, 7, 40]])
@pytest.mark.parametrize("n_in,n_out", [(256, 96), (100, 33)])
def test_an_infinity_gives_what_the_definition_gives(rank, new, n_in, n_out):
    """With positive A and B, an infinity in x is an infinity of its sign in all of the row's outputs, and one of each sign is NaN."""
    g = torch.Generator(device="cuda").manual_seed(rank)

    def positive(*shape):
        return (0.1 + torch.rand(shape, device="cuda", generator=g)).to(BF16)

    rows, starts = sums(new)[-1], sums(new)
    a, b, x, y = positive(3, rank, n_in), positive(3, n_out, rank), positive(rows, n_in), positive(rows, n_out)
    x[0, 5] = float("inf")
    x[starts[1], 0] = -float("inf")
    x[rows - 1, 3], x[rows - 1, n_in - 1] = float("inf"), -float("inf")
    f = Adapters(a, b)
    got = f(x, y, ints([2, 0, 1]), ints(starts))
    want = torch.cat([y[r0:r1].to(F64) + (x[r0:r1].to(F64) @ a[i].to(F64).T) @ b[i].to(F64).T for i, r0, r1 in zip((2, 0, 1), starts, starts[1:])])
    assert want[0].isposinf().all() and want[starts[1]].isneginf().all() and want[rows - 1].isnan().all()
    odd = ~want.isfinite()
    assert torch.equal(got.to(F64)[odd].nan_to_num(7.0, 5.0, -5.0), want[odd].nan_to_num(7.0, 5.0, -5.0))
    assert got[~odd].isfinite().all() and f.read_status() == 0


@pytest.mark.parametrize("new", [[1, 1], [20, 7]])
@pytest.mark.parametrize("sign", [1, -1])
def test_a_sum_above_the_largest_bf16_number_stays_finite(new, sign):
    """h = 3.3895e38 + 1e36 is an fp32 number that bf16 rounds to infinity; out is h 2^-100 within 2^-17 of it and one rounding to fp32."""
    rows, starts = sums(new)[-1], sums(new)
    a, b = torch.zeros(1, 16, 64, dtype=BF16, device="cuda"), torch.zeros(1, 32, 16, dtype=BF16, device="cuda")
    a[0, 3, :2], b[0, :, 3] = 1, 2.0 ** -100
    x = torch.zeros(rows, 64, dtype=BF16, device="cuda")
    x[:, 0], x[:, 1] = sign * torch.finfo(BF16).max, sign * 1e36
    got = Adapters(a, b)(x, torch.zeros(rows, 32, device="cuda"), ints([0, 0]), ints(starts)).to(F64)
    want = x[:, :2].to(F64).sum(1, keepdim=True) * 2.0 ** -100
    assert ((got - want).abs() <= (2.0 ** -17 + 2.0 ** -24) * want.abs()).all()
