"""What a handle keeps between calls, and what it reads anew."""
import numpy as np
import pytest
import torch

import paper_2406_06237_b200 as ans
from paper_2406_06237_b200.runtime import DeviceBatch, Linear, pack_layer

pytestmark = pytest.mark.gpu
BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


def integers(shape, most, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-most, most + 1, shape, device="cuda", generator=g).float().to(dtype)


def product(x, w):
    """Whole numbers with sums under 2^24: exact in fp32."""
    return (x.double() @ w.double().T).float()


# n, k, the weight's first element in its buffer, its rows' distance (0: k)
PLACES = [(128, 256, 0, 0), (128, 256, 1, 0), (65, 131, 0, 0), (300, 2047, 0, 0), (1, 33, 3, 0), (1000, 64, 8, 0), (200, 100, 0, 104), (200, 100, 5, 203),
          (3001, 520, 0, 521)]


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("n,k,off,stride", PLACES)
def test_a_weight_written_again_is_read_again(n, k, off, stride, dtype):
    """Wherever the weight lies: a call multiplies by what its buffer holds when the stream gets there."""
    stride = stride or k
    room = torch.full((off + n * stride,), 9.0, device="cuda").to(dtype)
    w = room.as_strided((n, k), (stride, 1), off)
    for m in (1, 70):
        x = integers((m, k), 4, dtype, m)
        f = Linear(w)
        for seed in range(3):
            w.copy_(integers((n, k), 4, dtype, seed))
            assert torch.equal(f(x, out_dtype=F32), product(x, w))
        assert f.read_status() == 0


def test_a_transposed_weight_is_read_again():
    base = torch.empty(300, 77, device="cuda", dtype=BF16)
    f, x = Linear(base.t()), integers((5, 300), 4, BF16, 1)
    for seed in range(2):
        base.copy_(integers((300, 77), 4, BF16, seed))
        assert torch.equal(f(x, out_dtype=F32), product(x, base.t()))


def test_a_broadcast_weight():
    """Strides of zero: one column for all, one row for all."""
    x = integers((5, 300), 4, BF16, 1)
    for w in (integers((77, 1), 4, BF16, 2).expand(77, 300), integers((1, 300), 4, BF16, 2).expand(77, 300)):
        for settled in (False, True):
            assert torch.equal(Linear(w, settled=settled)(x, out_dtype=F32), product(x, w))


@pytest.mark.parametrize("k", [64, 67])
def test_a_weight_written_between_replays(k):
    w, x, y = integers((130, k), 4, BF16, 1), integers((20, k), 4, BF16, 2), torch.empty(20, 130, device="cuda")
    f = Linear(w)
    f(x, out=y)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        f(x, out=y)
    for seed in (5, 6):
        w.copy_(integers((130, k), 4, BF16, seed))
        g.replay()
        assert torch.equal(y, product(x, w))


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("n,k,off,stride", PLACES)
def test_a_settled_weight_anywhere(n, k, off, stride, dtype):
    stride = stride or k
    w = torch.empty(off + n * stride, device="cuda").to(dtype).as_strided((n, k), (stride, 1), off)
    w.copy_(integers((n, k), 4, dtype, 1))
    f = Linear(w, settled=True)
    for m in (1, 70):
        x = integers((m, k), 4, dtype, m)
        assert torch.equal(f(x, out_dtype=F32), product(x, w))


def vectors(n):
    """Tensors of n values in every form that is not the one the kernel reads."""
    return {"fp32": torch.empty(n, device="cuda"), "bf16": torch.empty(n, device="cuda", dtype=BF16), "double": torch.empty(n, device="cuda", dtype=torch.float64),
            "strided": torch.empty(n, 3, device="cuda")[:, 1]}


@pytest.mark.parametrize("form", ["fp32", "bf16", "double", "strided"])
def test_bias_and_scales_written_again_are_read_again(form):
    n, k = 203, 64
    w, x = integers((n, k), 4, BF16, 1), integers((9, k), 4, BF16, 2)
    bias, scales = vectors(n)[form], vectors(n)[form]
    f = Linear(w, scales=scales, bias=bias)
    for seed in range(3):
        bias.copy_(integers((n,), 9, F32, seed))
        scales.copy_(2.0 ** integers((n,), 3, F32, seed + 7))
        assert torch.equal(f(x, out_dtype=F32), product(x, w) * scales.float() + bias.float())
    settled = Linear(w, scales=scales, bias=bias, settled=True)
    assert torch.equal(settled(x, out_dtype=F32), product(x, w) * scales.float() + bias.float())


def test_one_scale_for_all():
    n, k = 130, 64
    w, x = integers((n, k), 4, BF16, 1), integers((9, k), 4, BF16, 2)
    scale = torch.full((1,), 0.5, device="cuda")
    f = Linear(w, scales=scale)
    for value in (0.25, 4.0):
        scale.fill_(value)
        assert torch.equal(f(x, out_dtype=F32), product(x, w) * value)
    # numbers and tensors of another device are taken when the handle is made
    there = torch.full((n,), 2.0)
    by_number, by_host = Linear(w, scales=0.5, bias=there), Linear(w, scales=there, bias=torch.ones(n, dtype=torch.int32))
    there.zero_()
    assert torch.equal(by_number(x, out_dtype=F32), product(x, w) * 0.5 + 2) and torch.equal(by_host(x, out_dtype=F32), product(x, w) * 2 + 1)


@pytest.mark.parametrize("k", [64, 67])
def test_tensors_that_require_a_gradient_are_taken_by_their_values(k):
    w, x, bias = integers((130, k), 4, BF16, 1), integers((9, k), 4, BF16, 2), integers((130,), 4, BF16, 3)
    want = product(x, w) + bias.float()
    y = Linear(w.requires_grad_(), bias=bias.requires_grad_())(x.requires_grad_(), out_dtype=F32)
    assert torch.equal(y, want) and not y.requires_grad


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("n,k,off,stride", PLACES)
def test_rows_and_weight_off_16_bytes_together(n, k, off, stride, dtype):
    """Both are laid out by one launch, X behind W; what lies between the rows is never used."""
    stride = stride or k
    w = torch.full((off + n * stride + 40,), float("nan"), device="cuda").to(dtype).as_strided((n, k), (stride, 1), off)
    w.copy_(integers((n, k), 4, dtype, 1))
    f = Linear(w)
    for m in (1, 2, 33, 300):
        for x_off, x_stride in ((0, k + (-k) % 16), (1, k + 3), (0, k)):
            x = torch.full((x_off + m * x_stride,), float("nan"), device="cuda").to(dtype).as_strided((m, k), (x_stride, 1), x_off)
            x.copy_(integers((m, k), 4, dtype, m))
            assert torch.equal(f(x, out_dtype=F32), product(x, w))
    assert f.read_status() == 0


@pytest.mark.parametrize("n,k", [(130, 256), (130, 255), (64, 2047)])
def test_a_weight_decoded_again_behind_its_handle(n, k):
    """The handle is made before the weight is decoded; every decode into the buffer is multiplied by."""
    symbols = [np.random.default_rng(seed).integers(0, 16, n * k).astype(np.uint8) for seed in range(3)]
    batches = [DeviceBatch([pack_layer(s, 16, 8, 4096, 32, ans.ANS_LAYOUT_QUADS, 4, 8, 0.25, ans.ANS_BF16)]) for s in symbols]
    weight = torch.zeros(n * k, device="cuda", dtype=BF16)
    f, x = Linear(weight.view(n, k)), integers((40, k), 4, BF16, 1)
    for s, b in zip(symbols, batches):
        b.decode()
        weight.copy_(b.output(0))
        y = f(x, out_dtype=F32)
        want = torch.from_numpy((s.astype(np.float32) - 8) * 0.25).cuda().view(n, k)
        assert torch.equal(y, product(x, want)) and b.read_status() == 0
    own = Linear(batches[0].output(0).view(n, k))           # and in the decoder's own buffer
    batches[0].out_sets[0][0].zero_()
    assert not own(x, out_dtype=F32).any()
    batches[0].decode()
    assert torch.equal(own(x, out_dtype=F32), product(x, torch.from_numpy((symbols[0].astype(np.float32) - 8) * 0.25).cuda().view(n, k)))
