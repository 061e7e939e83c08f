"""The norm against its formula in 64 bits."""
import pytest
import torch

import paper_2406_06237_b200 as ans
from operator_helpers import rounds_from
from paper_2406_06237_b200.runtime import RmsNorm

pytestmark = pytest.mark.gpu
BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn

# Sum of squares: up to 40 terms a thread and 10 steps of a tree, each within 2^-24 of a sum of positive
# numbers, so 50 * 2^-24, halved by the root; eight more roundings up to y: under 2^-18 in all.
FP32 = 2.0 ** -18


def formula(x, r, w, eps):
    h = x.double() + (0 if r is None else r.double())
    y = h / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    return h, y if w is None else y * w.double()


def check(x, r, w, eps, out, scales, summed, out_dtype):
    h, y = formula(x, r, w, eps)
    if r is not None:
        assert rounds_from(summed, h, 2.0 ** -24 * h.abs() + 1e-38).all()
    if out_dtype is not E4M3:
        assert rounds_from(out, y, FP32 * y.abs() + 1e-37).all()
        return
    top = (y.abs().amax(1) / 448).clamp(min=2.0 ** -126)
    assert ((scales.double() - top).abs() <= FP32 * top).all()
    s = scales.double()[:, None]
    # three bits after the leading one: half a step is 2^-4 of a value, or half of the smallest step, 2^-9
    assert ((out.float().double() * s - y).abs() <= (2.0 ** -4 + 2 * FP32) * y.abs() + (2.0 ** -10 + 1e-6) * s).all()
    assert (out.float().abs() <= 448).all()


@pytest.mark.parametrize("out_dtype", [BF16, F32, E4M3])
@pytest.mark.parametrize("x_dtype", [BF16, F32])
@pytest.mark.parametrize("rows,width", [(1, 1), (1, 8192), (3, 7), (5, 8), (9, 250), (17, 256), (8, 1000), (7, 1024), (33, 1030),
                                        (2, 2047), (4, 4096), (3, 8200), (2, 16384), (2, 16385), (2, 32761), (2, 32768)])
def test_rows(rows, width, x_dtype, out_dtype):
    g = torch.Generator(device="cuda").manual_seed(rows * 40000 + width)
    x = (3 * torch.randn(rows, width, device="cuda", generator=g)).to(x_dtype)
    r = torch.randn(rows, width, device="cuda", generator=g).to(x_dtype)
    w = torch.randn(width, device="cuda", generator=g).to(BF16 if width % 2 else F32)
    for residual, weight in ((r, w), (None, w), (r, None), (None, None)):
        f = RmsNorm(weight, 1e-5, out_dtype, device="cuda")
        got = f(x, residual)
        assert (got[1] is not None) == (out_dtype is E4M3) and (got[2] is not None) == (residual is not None)
        check(x, residual, weight, 1e-5, *got, out_dtype)


@pytest.mark.parametrize("out_dtype", [BF16, F32, E4M3])
@pytest.mark.parametrize("x_dtype", [BF16, F32])
@pytest.mark.parametrize("rows,width", [(9000, 64), (9001, 250), (7000, 500), (5003, 1024), (3000, 2048), (2001, 4096), (1201, 8192), (701, 12000),
                                        (701, 16384), (1000, 8201), (901, 16381), (3001, 2047), (700, 1111)])
def test_many_rows(rows, width, x_dtype, out_dtype):
    """Row counts at which blocks take row after row, some of them one more than others."""
    g = torch.Generator(device="cuda").manual_seed(rows + width)
    x = (3 * torch.randn(rows, width, device="cuda", generator=g)).to(x_dtype)
    r = torch.randn(rows, width, device="cuda", generator=g).to(x_dtype)
    w = torch.randn(width, device="cuda", generator=g).to(F32 if rows % 2 else BF16)
    f = RmsNorm(w, 1e-5, out_dtype)
    for residual in (r, None):
        check(x, residual, w, 1e-5, *f(x, residual), out_dtype)


@pytest.mark.parametrize("out_dtype", [BF16, E4M3])
@pytest.mark.parametrize("offset,stride", [(0, 520), (3, 515), (8, 513), (5, 700)])
@pytest.mark.parametrize("width", [513, 512, 40])
def test_strides_and_places(width, offset, stride, out_dtype):
    """Rows anywhere in larger buffers: equally far from 16 bytes, and not; nothing beside them is written."""
    g = torch.Generator(device="cuda").manual_seed(width + stride)
    rows = 11

    def view(dtype, off, st):
        room = torch.full((rows * st + off + width,), 7, device="cuda").to(dtype)
        return room, room[off:off + rows * st].view(rows, st)[:, :width]

    for r_off, r_stride in ((offset, stride), (offset + 1, stride), (offset, stride + 1)):
        if r_stride < width or stride < width:
            continue
        _, x = view(BF16, offset, stride)
        _, r = view(BF16, r_off, r_stride)
        x.copy_(torch.randn(rows, width, device="cuda", generator=g))
        r.copy_(torch.randn(rows, width, device="cuda", generator=g))
        w = torch.randn(width + 1, device="cuda", generator=g).to(BF16)[1:]
        (oroom, out), (sroom, summed) = view(out_dtype, offset, stride), view(BF16, offset, stride)
        f = RmsNorm(w.clone() if r_off == offset else w, 1e-6, out_dtype)
        got = f(x, r, out=out, summed=summed)
        check(x, r, w, 1e-6, *got, out_dtype)
        for room, t in ((oroom, out), (sroom, summed)):
            t.zero_() if t.dtype is not E4M3 else t.view(torch.uint8).zero_()
            assert int((room.float() == 7).sum()) == room.numel() - rows * width


@pytest.mark.parametrize("target", ["x", "residual"])
def test_sum_in_place(target):
    x, r = torch.randn(5, 4096, device="cuda").to(BF16), torch.randn(5, 4096, device="cuda").to(BF16)
    f = RmsNorm(torch.ones(4096, device="cuda"), out_dtype=E4M3)
    want = f(x, r)
    got = f(x, r, summed={"x": x, "residual": r}[target])
    assert torch.equal(got[2], want[2]) and torch.equal(got[0].view(torch.uint8), want[0].view(torch.uint8)) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("width", [64, 1000, 8192])
def test_zeros_nan_inf_and_small_rows(width):
    x = torch.randn(6, width, device="cuda")
    x[0] = 0
    x[1, width // 2] = float("nan")
    x[2, 3] = float("inf")
    x[3] *= 1e-38                                    # y is far under what 448 * 2^-126 stands for
    x[4, 1:] = 0                                     # one large value
    f8, f32 = RmsNorm(None, 1e-6, E4M3, device="cuda"), RmsNorm(None, 1e-6, F32, device="cuda")
    q, s, _ = f8(x)
    y = f32(x)[0]
    assert (y[0] == 0).all() and (q[0].float() == 0).all() and s[0] == 2.0 ** -126
    assert y[1].isnan().all() and q[1].float().isnan().all() and s[1].isnan()
    assert y[2, 3].isnan() and (y[2, :3] == 0).all() and s[2].isnan() and q[2].float().isnan().all()
    for i in (3, 4, 5):
        assert ((q[i].float() * s[i] - y[i]).abs() <= y[i].abs() * (2.0 ** -4 + FP32) + s[i] * 2.0 ** -9.99).all()
    z = RmsNorm(None, 0.0, F32, device="cuda")(x[:1])[0]
    assert z.isnan().all()                           # 0 / 0


def test_many_rows_and_streams():
    """More rows than a grid's second dimension holds, on a stream of its own."""
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        x = torch.randn(70001, 64, device="cuda").to(BF16)
        got = RmsNorm(None, 1e-6, F32, device="cuda")(x)[0]
    st.synchronize()
    check(x, None, None, 1e-6, got, None, None, F32)


def test_empty():
    f = RmsNorm(None, device="cuda")
    assert f(torch.empty(0, 64, device="cuda"))[0].shape == (0, 64)
    assert f(torch.empty(3, 0, device="cuda"))[0].shape == (3, 0)


def test_refusals():
    x = torch.randn(4, 64, device="cuda")
    f = RmsNorm(torch.ones(64, device="cuda"), out_dtype=E4M3)
    for bad in (x[:, :32], x.double(), x.cpu(), x.t(), x[0], x[:1].expand(4, 64)):
        with pytest.raises(ValueError):
            f(bad)
    for kw in (dict(residual=x.to(BF16)), dict(out=x), dict(scales=x[0]), dict(summed=x), dict(residual=x, summed=x[:2])):
        with pytest.raises(ValueError):
            f(x, **kw)
    with pytest.raises(ValueError):
        RmsNorm(torch.ones(64, device="cuda"))(x, scales=torch.empty(4, device="cuda"))
    with pytest.raises(ValueError):
        RmsNorm(torch.ones(64, device="cuda"), out_dtype=torch.int8)
    with pytest.raises(RuntimeError):
        RmsNorm(torch.ones(64))
    with pytest.raises(ans.AnsError):
        RmsNorm(None, device="cuda")(torch.zeros(1, 32769, device="cuda"))
    with pytest.raises(ans.AnsError):
        RmsNorm(None, -1.0, device="cuda")(x)
