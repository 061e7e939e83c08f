"""The product with its epilogue against its formula in 64 bits."""
import math

import pytest
import torch

import paper_2406_06237_b200 as ans
from operator_helpers import rounds_from
from paper_2406_06237_b200.runtime import Linear, symbols_to_e4m3

pytestmark = pytest.mark.gpu
BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


def integers(shape, most, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-most, most + 1, shape, device="cuda", generator=g).float().to(dtype)


# every tile form, its edges, and lengths of K around a stage (64 bf16 or 128 e4m3) and a split of it
SIZES = [(1, 1, 1), (1, 128, 64), (2, 130, 65), (16, 257, 512), (17, 64, 1000), (31, 1000, 2048), (33, 129, 130), (64, 128, 4096),
         (65, 300, 200), (100, 1000, 2048), (128, 256, 128), (129, 128, 256), (333, 1000, 2048), (500, 2500, 72), (777, 3001, 264),
         (1100, 2048, 640), (2047, 1025, 1024), (1030, 8200, 4096), (4100, 600, 128), (100, 2048, 8192)]


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_sums_are_exact(m, n, k, dtype):
    """Whole numbers whose sums stay under 2^24: fp32 sums of any order are exact, so any lost, doubled or
    misplaced element shows."""
    x, w = integers((m, k), 8, dtype, m + n), integers((n, k), 8, dtype, k)
    f = Linear(w)
    y = f(x, out_dtype=F32)
    assert torch.equal(y, (x.double() @ w.double().T).float())
    assert f.read_status() == 0


ACTS = {
    "none": lambda v: v, "relu": lambda v: v.clamp(min=0), "gelu": lambda v: v * torch.special.ndtr(v),
    "gelu_tanh": lambda v: v * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)), "silu": lambda v: v * torch.sigmoid(v),
}


@pytest.mark.parametrize("out_dtype", [BF16, F32])
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("m,n,k", [(1, 200, 96), (5, 515, 1024), (90, 259, 512), (600, 2052, 320)])
def test_epilogue(m, n, k, dtype, act, out_dtype):
    g = torch.Generator(device="cuda").manual_seed(m + n + k)
    x = torch.randn(m, k, device="cuda", generator=g).to(dtype)
    w = torch.randn(n, k, device="cuda", generator=g).to(dtype)
    xs = torch.rand(m, device="cuda", generator=g) + 0.5
    ws = (torch.rand(n, device="cuda", generator=g) + 0.5) / math.sqrt(k)
    bias = torch.randn(n, device="cuda", generator=g)
    res = torch.randn(m, n, device="cuda", generator=g).to(out_dtype)
    sums = x.double() @ w.double().T
    # fp32 sums of k products: at most k + 8 roundings of 2^-23 (the tensor cores may truncate) of the sum of magnitudes
    slack = (k + 8) * 2.0 ** -23 * (x.double().abs() @ w.double().abs().T)
    for use in ((1, 1, 1, 1), (0, 0, 0, 0), (1, 0, 1, 0), (0, 1, 0, 1)):
        scale = (xs.double()[:, None] if use[0] else 1) * (ws.double() if use[1] else torch.ones((), device="cuda").double() / math.sqrt(k))
        f = Linear(w, scales=ws if use[1] else 1 / math.sqrt(k), bias=bias if use[2] else None, activation=act)
        y = f(x, x_scales=xs if use[0] else None, residual=res if use[3] else None, out_dtype=out_dtype)
        v = sums * scale + (bias.double() if use[2] else 0)
        want = ACTS[act](v) + (res.double() if use[3] else 0)
        # the activations' slopes are at most 1.13; they and the scales cost some 2^-20 of their values in fp32
        tol = 1.13 * slack * scale + 2.0 ** -20 * (v.abs() + want.abs() + (res.double().abs() if use[3] else 0)) + 1e-30
        assert rounds_from(y, want, tol).all(), use
        assert f.read_status() == 0


@pytest.mark.parametrize("m,n,k", [(3, 131, 64), (70, 260, 200), (513, 2051, 136)])
@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_strides_and_places(m, n, k, dtype):
    """Rows in larger buffers filled with NaN; outputs at odd places; residual in place."""
    pad = 48
    def room(rows, cols, dt, off):
        t = torch.full((rows, cols + pad), float("nan"), device="cuda").to(dt)
        return t[:, off:off + cols], t
    x, _ = room(m, k, dtype, 16)
    w, _ = room(n, k, dtype, 32)
    x.copy_(integers((m, k), 4, dtype, 1)); w.copy_(integers((n, k), 4, dtype, 2))
    want = (x.double() @ w.double().T)
    for off in (0, 1, 4):
        for dt in (F32, BF16):
            y, whole = room(m, n, dt, off)
            y.copy_(integers((m, n), 3, dt, 3))
            expect = (want + y.double()).to(dt)
            f = Linear(w)
            assert f(x, residual=y, out=y) is y
            assert torch.equal(y, expect)
            assert int(whole.isnan().sum()) == m * pad
    # x at an odd place, and with rows that do not start on 16 bytes
    for off, cols in ((1, k), (8, k), (0, k - 3), (5, k - 7)):
        odd = torch.full((m, k + 21), float("nan"), device="cuda").to(dtype)[:, off:off + cols]
        odd.copy_(x[:, :cols])
        assert torch.equal(Linear(w[:, :cols])(odd, out_dtype=F32), (odd.double() @ w[:, :cols].double().T).float())
    # a K that is no multiple of 16 bytes, contiguous: copied
    x2, w2 = integers((m, k + 1), 4, dtype, 4), integers((n, k + 1), 4, dtype, 5)
    assert torch.equal(Linear(w2)(x2, out_dtype=F32), (x2.double() @ w2.double().T).float())


def test_nan_and_inf_stay_in_their_rows():
    x, w = integers((20, 256), 4, BF16, 1), integers((200, 256), 4, BF16, 2)
    x[3, 17], x[7, 200] = float("nan"), float("inf")
    y = Linear(w, activation="relu")(x, out_dtype=F32)
    assert y[3].isnan().all()
    ok = torch.tensor([i for i in range(20) if i not in (3, 7)], device="cuda")
    assert torch.equal(y[ok], (x[ok].double() @ w.double().T).clamp(min=0).float())
    assert not y[7].isfinite()[w[:, 200] > 0].any()


def test_empty_and_k_zero():
    assert Linear(torch.empty(5, 0, device="cuda").to(BF16), bias=torch.arange(5.0), activation="silu")(
        torch.empty(70, 0, device="cuda").to(BF16), out_dtype=F32).sub(torch.nn.functional.silu(torch.arange(5.0, device="cuda"))).abs().max() < 1e-6
    assert Linear(torch.empty(0, 64, device="cuda").to(BF16))(torch.empty(3, 64, device="cuda").to(BF16)).shape == (3, 0)
    assert Linear(torch.empty(9, 64, device="cuda").to(BF16))(torch.empty(0, 64, device="cuda").to(BF16)).shape == (0, 9)


@pytest.mark.parametrize("m", [1, 40, 300])
def test_same_every_time_and_on_a_stream(m):
    x, w = torch.randn(m, 2048, device="cuda").to(BF16), torch.randn(2500, 2048, device="cuda").to(BF16)
    f = Linear(w)
    first = f(x)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        others = [f(x) for _ in range(5)]
    st.synchronize()
    assert all(torch.equal(first, o) for o in others)


def test_captured_in_a_graph():
    x, w = integers((24, 512), 4, BF16, 1), integers((640, 512), 4, BF16, 2)
    f, y = Linear(w), torch.empty(24, 640, device="cuda")
    f(x, out=y)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        f(x, out=y)
    x.copy_(integers((24, 512), 4, BF16, 9))
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, (x.double() @ w.double().T).float())


def test_symbols_to_e4m3():
    q = torch.randint(0, 16, (64, 64), dtype=torch.uint8, device="cuda")
    assert torch.equal(symbols_to_e4m3(q, 7).float(), q.float() - 7)
    with pytest.raises(ValueError):
        symbols_to_e4m3(q + 20, 3)                   # 17 and more: not all exact


def test_refusals():
    w = torch.randn(64, 128, device="cuda").to(BF16)
    x = torch.randn(4, 128, device="cuda").to(BF16)
    f = Linear(w)
    for bad in (x.float(), x[:, :64], x.cpu(), x[0]):
        with pytest.raises(ValueError):
            f(bad)
    for kw in (dict(x_scales=torch.ones(3, device="cuda")), dict(residual=torch.zeros(4, 64, device="cuda")), dict(out_dtype=torch.float16),
               dict(out=torch.empty(4, 65, device="cuda")), dict(out=torch.empty(64, 4, device="cuda").t()),
               dict(out=torch.empty(1, 64, device="cuda").expand(4, 64))):
        with pytest.raises(ValueError):
            f(x, **kw)
    for kw in (dict(activation="tanh"), dict(scales=torch.ones(3)), dict(bias=torch.ones(3))):
        with pytest.raises(ValueError):
            Linear(w, **kw)
    with pytest.raises(ValueError):
        Linear(w.float())
    with pytest.raises(RuntimeError):
        Linear(w.cpu())
    d = ans.binding.ans_product_desc.from_buffer_copy(f._desc)
    y = torch.empty(4, 64, device="cuda")
    d.d_x, d.x_stride, d.m, d.d_y, d.y_stride, d.y_dtype = x.data_ptr(), 128, 4, y.data_ptr(), 64, ans.ANS_F32
    ans.binding.ans_product(d, f.status.data_ptr())
    for field, value in (("d_x", x.data_ptr() + 2), ("d_x", x.data_ptr() + 1), ("x_stride", 127), ("x_stride", 132), ("w_stride", 0), ("y_stride", 63), ("d_y", None),
                         ("d_y", y.data_ptr() + 2), ("dtype", ans.ANS_F32), ("y_dtype", ans.ANS_E4M3), ("activation", 5), ("k", 1 << 23), ("m", 1 << 31)):
        e = ans.binding.ans_product_desc.from_buffer_copy(d)
        setattr(e, field, value)
        with pytest.raises(ans.AnsError):
            ans.binding.ans_product(e, f.status.data_ptr())
    with pytest.raises(ans.AnsError):
        ans.binding.ans_product(d, None)
    torch.cuda.synchronize()
