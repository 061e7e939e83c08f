"""The norm over the whole range of its types: rows whose squares pass the largest fp32 number or vanish under the smallest."""
import pytest
import torch

from paper_2406_06237_b200.runtime import RmsNorm
from test_gpu_norm import BF16, E4M3, F32, check

pytestmark = pytest.mark.gpu

# widths and row counts that reach every kernel: warps and blocks on a row, rings, rows off 16 bytes
SIZES = [(13, 7), (13, 64), (26, 250), (13, 512), (13, 1024), (2600, 1024), (9100, 251), (13, 8192), (1300, 8192), (1537, 2047), (910, 16381), (13, 16384),
         (13, 32761), (13, 32768)]


def rows_of(kind, rows, width, dtype, seed):
    """Row i is of the i-th kind of size, over and over; x and its residual.  None of the rows is all zeros."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, r = torch.randn(rows, width, device="cuda", generator=g), torch.randn(rows, width, device="cuda", generator=g)
    x[:, 0] = x[:, 0].abs() + 0.5                         # and no row of one value cancels
    r[:, 0] = r[:, 0].abs() + 0.5
    for i, size in enumerate(kind):
        s = torch.full((width,), 1.0, device="cuda")
        if isinstance(size, tuple):                       # a part of the row in one size, the rest in another; or one value apart
            s[:] = size[1]
            s[:(width + 1) // 2 if len(size) == 2 else 1] = size[0]
        else:
            s[:] = size
        x[i::len(kind)] *= s
        r[i::len(kind)] *= s
    return x.to(dtype), r.to(dtype)


LARGE = [1e37, 1.0, 1e18, 2e19, 1e17, (3e37, 1.0), (1.0, 3e37), (3e37, 1.0, "one"), (1e37, 1e-16), 5e18, 1e-3, 3e36, 1e30]
SMALL = [1e-36, 1.0, 1e-23, 1e-20, 1e-30, (1e-16, 1.0), (1.0, 1e-16), (1e-36, 0.0, "one"), (1e-20, 0.0), 1e-18, 1e-15, (1e-30, 1e-37), 1e-10]


@pytest.mark.parametrize("out_dtype", [BF16, F32, E4M3])
@pytest.mark.parametrize("x_dtype", [BF16, F32])
@pytest.mark.parametrize("rows,width", SIZES)
def test_large_rows(rows, width, x_dtype, out_dtype):
    """Values up to the type's largest, whose products with the weight pass it too; the result is of ordinary size."""
    x, r = rows_of(LARGE, rows, width, x_dtype, rows + width)
    w = torch.randn(width, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).to(BF16) + 4
    for eps in (1e-5, 0.0):
        f = RmsNorm(w, eps, out_dtype)
        check(x, r, w, eps, *f(x, r), out_dtype)
        check(x, None, w, eps, *f(x), out_dtype)


@pytest.mark.parametrize("out_dtype", [BF16, F32, E4M3])
@pytest.mark.parametrize("x_dtype", [BF16, F32])
@pytest.mark.parametrize("rows,width", SIZES)
def test_small_rows_without_an_eps(rows, width, x_dtype, out_dtype):
    x, r = rows_of(SMALL, rows, width, x_dtype, rows + width)
    w = torch.randn(width, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    for eps in (0.0, 1e-36):
        f = RmsNorm(w, eps, out_dtype)
        check(x, r, w, eps, *f(x, r), out_dtype)
        check(x, None, w, eps, *f(x), out_dtype)


@pytest.mark.parametrize("out_dtype", [F32, E4M3])
@pytest.mark.parametrize("x_dtype", [BF16, F32])
@pytest.mark.parametrize("rows,width", [(13, 1000), (1300, 4100), (1300, 4096), (2600, 64)])
@pytest.mark.parametrize("target", ["x", "residual"])
def test_rows_summed_in_place(target, rows, width, x_dtype, out_dtype):
    """In fp32 the stored sum is the sum.  In bf16 it is rounded: rows in range do not see that, the others are the norm
    of the stored sum."""
    for kind, eps in ((LARGE, 1e-6), (SMALL, 0.0)):
        x, r = rows_of(kind, rows, width, x_dtype, 3)
        f = RmsNorm(None, eps, out_dtype, device="cuda")
        want = f(x, r)
        h = x + r if x_dtype is F32 else x.float() + r.float()
        squares = h.double().square().sum(1)
        got = f(x, r, summed={"x": x, "residual": r}[target])
        assert torch.equal(got[2], want[2])
        again = (squares > 2.0 ** 128 * 0.98) | ((squares < 2.0 ** -100 * 1.02) if eps == 0 else squares < 0)
        assert 0 < int(again.sum()) < rows
        if x_dtype is F32:
            again[:] = False
        assert torch.equal(got[0][~again].view(torch.uint8), want[0][~again].view(torch.uint8))
        if out_dtype is E4M3:
            assert torch.equal(got[1][~again], want[1][~again])
        if again.any():
            check(got[2][again], None, None, eps, got[0][again], got[1][again] if out_dtype is E4M3 else None, None, out_dtype)


def test_matrices_not_equally_aligned():
    x, r = rows_of(LARGE, 130, 515, BF16, 4)
    room = torch.empty(130, 520, device="cuda", dtype=BF16)
    off = room[:, 2:517]
    off.copy_(r)
    f = RmsNorm(None, 1e-6, F32, device="cuda")
    check(x, r, None, 1e-6, *f(x, off), F32)


@pytest.mark.parametrize("width", [64, 1000, 8192, 32768])
def test_zeros_nan_and_inf_beside_them(width):
    """What has no ordinary result keeps it: 0 / 0, a NaN's row, an infinite value's row."""
    x = torch.randn(8, width, device="cuda") * 1e30
    x[0] = 0
    x[1, width // 2] = float("nan")
    x[2, 3] = float("inf")
    x[3, 3] = -float("inf")
    for eps in (0.0, 1e-6):
        y, (q, s, _) = RmsNorm(None, eps, F32, device="cuda")(x)[0], RmsNorm(None, eps, E4M3, device="cuda")(x)
        assert y[0].isnan().all() if eps == 0 else (y[0] == 0).all()
        assert y[1].isnan().all() and q[1].float().isnan().all() and s[1].isnan()
        for i in (2, 3):
            assert y[i, 3].isnan() and (y[i, :3] == 0).all() and (y[i, 4:] == 0).all() and s[i].isnan() and q[i].float().isnan().all()
        check(x[4:], None, None, eps, y[4:], None, None, F32)
