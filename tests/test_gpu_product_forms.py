"""The product's forms one by one: which sizes take which, and sums, epilogue and places in the forms that prompts take."""
import math

import pytest
import torch

import paper_2406_06237_b200 as ans
from operator_helpers import rounds_from
from paper_2406_06237_b200.runtime import Linear
from test_gpu_product import ACTS, BF16, E4M3, F32, integers

pytestmark = pytest.mark.gpu
CODE = {BF16: ans.ANS_BF16, E4M3: ans.ANS_E4M3}


def form(m, n, k, dtype):
    return ans.binding.ans_product_form(m, n, k, CODE[dtype])


# Pairs of SMs: m, n, k, type, tokens of a tile.  Up to four tiles a pair (74 pairs on a B200), last tiles of a few tokens and
# features, 5 to 129 stages of K, the last one in part.
WHOLE = [(700, 4100, 520, BF16, 256), (1030, 5130, 1030, BF16, 256), (2050, 8200, 520, BF16, 256), (1537, 5130, 4104, BF16, 256),
         (700, 4100, 520, E4M3, 256), (1030, 5130, 1030, E4M3, 256), (2050, 8200, 520, E4M3, 256), (3000, 5130, 4104, E4M3, 256),
         (1030, 4100, 2056, BF16, 512), (3000, 5130, 4104, BF16, 512), (3000, 8200, 4104, BF16, 512), (5200, 2600, 4104, BF16, 512),
         (1100, 4100, 4112, E4M3, 512), (3000, 5130, 8208, E4M3, 512), (5200, 2600, 8208, E4M3, 512)]
ONE_OF_EACH = [WHOLE[1], WHOLE[5], WHOLE[9], WHOLE[13]]


@pytest.mark.parametrize("m,n,k,dtype,tokens", WHOLE)
def test_sums_in_pairs_are_exact(m, n, k, dtype, tokens):
    assert form(m, n, k, dtype) == (tokens, 0)
    x, w = integers((m, k), 8, dtype, m + n), integers((n, k), 8, dtype, k)
    want = (x.double() @ w.double().T).float()
    f = Linear(w)
    y = torch.empty(m, n, device="cuda")
    for _ in range(4):                                   # launches whose ends overlap
        y.fill_(float("nan"))
        f(x, out=y)
        f(x, out=y)
        assert torch.equal(y, want)
    assert f.read_status() == 0


@pytest.mark.parametrize("out_dtype", [BF16, F32])
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("m,n,k,dtype,tokens", ONE_OF_EACH)
def test_epilogue_in_pairs(m, n, k, dtype, tokens, act, out_dtype):
    """As for the other forms, with the bounds derived there."""
    assert form(m, n, k, dtype) == (tokens, 0)
    g = torch.Generator(device="cuda").manual_seed(m + n + k)
    x = torch.randn(m, k, device="cuda", generator=g).to(dtype)
    w = torch.randn(n, k, device="cuda", generator=g).to(dtype)
    xs = torch.rand(m, device="cuda", generator=g) + 0.5
    ws = (torch.rand(n, device="cuda", generator=g) + 0.5) / math.sqrt(k)
    bias = torch.randn(n, device="cuda", generator=g)
    res = torch.randn(m, n, device="cuda", generator=g).to(out_dtype)
    sums = x.double() @ w.double().T
    slack = (k + 8) * 2.0 ** -23 * (x.double().abs() @ w.double().abs().T)
    for use in ((1, 1, 1, 1), (0, 0, 0, 0), (1, 0, 1, 0), (0, 1, 0, 1)):
        scale = (xs.double()[:, None] if use[0] else 1) * (ws.double() if use[1] else torch.ones((), device="cuda").double() / math.sqrt(k))
        f = Linear(w, scales=ws if use[1] else 1 / math.sqrt(k), bias=bias if use[2] else None, activation=act)
        y = f(x, x_scales=xs if use[0] else None, residual=res if use[3] else None, out_dtype=out_dtype)
        v = sums * scale + (bias.double() if use[2] else 0)
        want = ACTS[act](v) + (res.double() if use[3] else 0)
        tol = 1.13 * slack * scale + 2.0 ** -20 * (v.abs() + want.abs() + (res.double().abs() if use[3] else 0)) + 1e-30
        assert rounds_from(y, want, tol).all(), use
        assert f.read_status() == 0


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("off,stride", [(0, 0), (1, 3), (4, 4), (3, 1), (0, 2)])
@pytest.mark.parametrize("m,n,k,dtype,tokens", ONE_OF_EACH)
def test_residual_in_place_in_pairs(m, n, k, dtype, tokens, off, stride, dt):
    """Outputs at odd places and strides, the residual in the same place, NaN around them."""
    pad = 16 + stride
    whole = torch.full((m, n + pad), float("nan"), device="cuda").to(dt)
    y = whole[:, off:off + n]
    y.copy_(integers((m, n), 3, dt, 3))
    x, w = integers((m, k), 4, dtype, 1), integers((n, k), 4, dtype, 2)
    expect = (x.double() @ w.double().T + y.double()).to(dt)
    f = Linear(w)
    assert f(x, residual=y, out=y) is y
    assert torch.equal(y, expect)
    assert int(whole.isnan().sum()) == m * pad
    other = integers((m, n + 3), 3, dt, 4)[:, 2:2 + n]
    assert torch.equal(f(x, residual=other, out=y), (x.double() @ w.double().T + other.double()).to(dt))
    assert int(whole.isnan().sum()) == m * pad and f.read_status() == 0


@pytest.mark.parametrize("m,n,k,dtype,tokens", ONE_OF_EACH)
def test_the_same_every_time_in_pairs(m, n, k, dtype, tokens):
    x, w = torch.randn(m, k, device="cuda").to(dtype), torch.randn(n, k, device="cuda").to(dtype)
    f = Linear(w, activation="gelu")
    first = f(x)
    assert all(torch.equal(first, f(x)) for _ in range(5))


# Clusters: tokens of a tile and the CTAs that share its K
SPLIT = [(1, 40000, 512, 16, 2), (5, 2500, 4104, 16, 8), (16, 9000, 2056, 16, 4), (30, 520, 8192, 16, 8), (20, 20000, 1024, 32, 1), (40, 9000, 1024, 32, 2),
         (30, 9000, 4096, 32, 4), (17, 4000, 4096, 32, 8), (64, 20000, 512, 64, 1), (60, 5000, 4096, 64, 4), (100, 2050, 8200, 64, 8), (600, 2052, 320, 128, 1),
         (100, 9000, 1024, 128, 2), (300, 1030, 2056, 128, 4)]


@pytest.mark.parametrize("m,n,k,tokens,parts", SPLIT)
def test_sums_in_clusters_are_exact(m, n, k, tokens, parts):
    assert form(m, n, k, BF16) == (tokens, parts)
    x, w = integers((m, k), 8, BF16, m + n), integers((n, k), 8, BF16, k)
    bias, res = integers((n,), 8, F32, 3), integers((m, n), 8, F32, 4)
    y = Linear(w, bias=bias)(x, residual=res, out_dtype=F32)
    assert torch.equal(y, (x.double() @ w.double().T + bias.double() + res.double()).float())


def test_every_form_is_tested():
    """The sizes of this file and their forms: every tile there is, and every way to deal K."""
    forms = {form(m, n, k, dtype) for m, n, k, dtype, _ in WHOLE} | {form(*c[:3], BF16) for c in SPLIT}
    assert {t for t, _ in forms} == {16, 32, 64, 128, 256, 512} and {p for _, p in forms} == {0, 1, 2, 4, 8}
