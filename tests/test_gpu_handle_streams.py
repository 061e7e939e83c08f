"""Handles made on one stream, used on others, and dropped while their calls run."""
import pytest
import torch

from paper_2406_06237_b200.runtime import Linear, PagedCache, RmsNorm

pytestmark = pytest.mark.gpu
BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


def integers(shape, most, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-most, most + 1, shape, device="cuda", generator=g).float().to(dtype)


class Work:
    """Some milliseconds of work for the current stream."""

    def __init__(self):
        self.a, self.b = torch.randn(8192, 8192, device="cuda").to(BF16), torch.empty(8192, 8192, device="cuda", dtype=BF16)

    def __call__(self, times=8):
        for _ in range(times):
            torch.matmul(self.a, self.a, out=self.b)


@pytest.fixture(scope="module")
def work():
    return Work()


@pytest.mark.parametrize("settled", [False, True])
@pytest.mark.parametrize("k", [512, 515])
def test_a_product_on_another_stream_than_its_makers(work, k, settled):
    w, x = integers((700, k), 4, E4M3, 1), integers((40, k), 4, E4M3, 2)
    want = (x.double() @ w.double().T).float() * 0.5 + 3
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        work()
        f = Linear(w, scales=0.5, bias=torch.full((700,), 3.0), settled=settled)
        with torch.cuda.stream(other):
            y = f(x, out_dtype=F32)
            assert f.read_status() == 0
        torch.cuda.synchronize()
        assert torch.equal(y, want)


def test_a_cache_on_another_stream_than_its_makers(work):
    """The cache's zeros are in place before anything is written on another stream."""
    heads, dim, tokens = 4, 64, 500
    k, v = integers((tokens, heads, dim), 100, BF16, 1), integers((tokens, heads, dim), 100, BF16, 2)
    slots = torch.randperm(640, device="cuda")[:tokens]
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    work()
    c = PagedCache(40, 16, heads, dim)
    with torch.cuda.stream(other):
        c.write(k, v, slots)
    torch.cuda.synchronize()
    d = PagedCache(40, 16, heads, dim)
    d.write(k, v, slots)
    for f in ("k_codes", "k_scales", "k_zeros", "v_codes", "v_scales", "v_zeros"):
        assert torch.equal(getattr(c, f), getattr(d, f)), f
    assert c.k_codes.any() and c.read_status() == 0


@pytest.mark.parametrize("k", [512, 515])
def test_a_product_dropped_while_it_runs(work, k):
    """The handle's scales and its laid out weight go back to the maker's stream only when the call is done with them."""
    w, x = integers((700, k), 4, BF16, 1), integers((40, k), 4, BF16, 2)
    want = (x.double() @ w.double().T).float() * 0.5
    other = torch.cuda.Stream()
    for _ in range(5):
        f = Linear(w.clone(), scales=0.5, settled=True)
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            work()
            y = f(x, out_dtype=F32)
        del f
        others = [torch.full((n,), float("nan"), device="cuda") for n in (700, 700, 64, 64, 700 * 260, 700 * 256)]
        torch.cuda.synchronize()
        assert torch.equal(y, want)
        del others


def test_a_cache_dropped_while_it_runs(work):
    heads, dim, tokens = 4, 64, 640
    k = integers((tokens, heads, dim), 100, BF16, 1)
    tables, starts = torch.arange(40, device="cuda", dtype=torch.int32)[None], torch.tensor([0, tokens], device="cuda", dtype=torch.int32)
    slots = torch.arange(tokens, device="cuda")
    other = torch.cuda.Stream()
    want = None
    for _ in range(4):
        c = PagedCache(40, 16, heads, dim)
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            work()
            c.write(k, k, slots)
            got = c.read(tables, starts, tokens)
        sizes = [t.numel() for t in (c.k_codes, c.k_codes, c.k_zeros, c.k_zeros)]
        del c
        others = [torch.full((n,), 255, device="cuda", dtype=torch.uint8) for n in sizes]
        torch.cuda.synchronize()
        want = got[0] if want is None else want
        assert torch.equal(got[0], want) and torch.equal(got[1], want)
        assert ((want - k).abs() <= 1.5 * 200 / 255 + 0.5).all()      # a step and a half, and bf16's rounding of values up to 100
        del others


def test_a_norm_on_two_streams(work):
    x, weight = torch.randn(300, 4096, device="cuda").to(BF16), torch.rand(4096, device="cuda") + 0.5
    f = RmsNorm(weight, out_dtype=E4M3)
    want = f(x)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            work(2)
            got.append(f(x))
    del f, weight
    junk = torch.full((4096,), float("nan"), device="cuda")
    torch.cuda.synchronize()
    for q, s, _ in got:
        assert torch.equal(q.view(torch.uint8), want[0].view(torch.uint8)) and torch.equal(s, want[1])
    assert junk.isnan().all()
