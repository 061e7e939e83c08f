"""Weights that are settled: read before the work queued ahead of a call is done, while all else of the call waits for it."""
import pytest
import torch

from paper_2406_06237_b200.runtime import Linear, RmsNorm

pytestmark = pytest.mark.gpu
BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


def integers(shape, most, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-most, most + 1, shape, device="cuda", generator=g).float().to(dtype)


# Stages of K (128 bytes) around a ring (3 to 5 stages in these forms) and its multiples, dealt over 1, 2, 4 and 8 CTAs by
# the number of tiles of features.
@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("n", [130, 1100, 4000, 9000, 40000])
@pytest.mark.parametrize("m", [1, 16, 30, 64, 100])
def test_sums_are_exact(m, n, dtype):
    """Whole numbers with sums under 2^24; two calls back to back, the second with other rows."""
    per = 64 if dtype is BF16 else 128
    for k in {per * s - d for s, d in ((1, 0), (2, 7), (3, 0), (4, 0), (5, 0), (5, 1), (6, 0), (8, 0), (11, 3), (24, 0), (41, 0), (64, 5))}:
        if n * k > 1 << 26:
            continue
        x, z, w = integers((m, k), 8, dtype, m + n), integers((m, k), 8, dtype, k), integers((n, k), 8, dtype, k + 1)
        f = Linear(w, settled=True)
        y, u = f(x, out_dtype=F32), f(z, out_dtype=F32)
        assert torch.equal(y, (x.double() @ w.double().T).float()), k
        assert torch.equal(u, (z.double() @ w.double().T).float()), k
        assert f.read_status() == 0


@pytest.mark.parametrize("m", [1, 20, 60, 120, 300])
def test_a_chain_behind_long_work(m):
    """A long product writes the rows that two settled products, one behind the other, multiply, and the residual they add:
    all of it in buffers that hold the last trip's values until then."""
    width, hidden = 2048, 5000
    w0, w1, w2 = (integers(s, 2, BF16, i) for i, s in enumerate(((width, 8192), (hidden, width), (width, hidden))))
    long = Linear(w0)
    buffers = [torch.empty(m + 2048, width, device="cuda", dtype=BF16), torch.empty(m, hidden, device="cuda", dtype=BF16),
               torch.empty(m, width, device="cuda", dtype=BF16)]
    results = {}
    for settled in (False, True):
        f, g = Linear(w1, scales=1 / 256, settled=settled), Linear(w2, scales=1 / 256, activation="silu", settled=settled)
        for trip in range(12):
            x = torch.randn(m + 2048, 8192, device="cuda", generator=torch.Generator("cuda").manual_seed(trip)).to(BF16)
            torch.cuda.synchronize()
            a = long(x, out=buffers[0])
            b = f(a[:m], out=buffers[1])
            c = g(b, residual=a[:m], out=buffers[2])
            results[settled, trip] = a[:m].clone(), b.clone(), c.clone()
            assert f.read_status() == 0 and g.read_status() == 0
    for trip in range(12):
        for plain, early in zip(results[False, trip], results[True, trip]):
            assert torch.equal(plain, early)


@pytest.mark.parametrize("m", [1, 40])
def test_scales_of_the_rows_written_just_ahead(m):
    """Norm, 8-bit product, norm, 8-bit product: rows and their scales come from the launch right ahead."""
    width = 4096
    w = [integers((width, width), 7, E4M3, i) for i in range(2)]
    norm = RmsNorm(None, out_dtype=E4M3, device="cuda")
    room = [torch.empty(m, width, device="cuda", dtype=t) for t in (E4M3, BF16)] + [torch.empty(m, device="cuda")]
    results = {}
    for settled in (False, True):
        f = [Linear(v, scales=1 / 256, settled=settled) for v in w]
        for trip in range(12):
            x = torch.randn(m, width, device="cuda", generator=torch.Generator("cuda").manual_seed(trip)).to(BF16) * (trip + 1)
            torch.cuda.synchronize()
            for g in f:
                rows, scales, _ = norm(x, out=room[0], scales=room[2])
                x = g(rows, x_scales=scales, residual=x, out=room[1])
            results[settled, trip] = x.clone()
            assert all(g.read_status() == 0 for g in f)
    for trip in range(12):
        assert torch.equal(results[False, trip], results[True, trip])


@pytest.mark.parametrize("m", [1, 16, 60])
def test_in_a_graph(m):
    w, x, y = integers((1000, 2048), 4, BF16, 1), integers((m, 2048), 4, BF16, 2), torch.empty(m, 1000, device="cuda")
    z = torch.empty_like(x)
    f = Linear(w, settled=True)
    f(x, out=y)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        z.copy_(x)
        f(z, out=y)
    for seed in (5, 6, 7):
        x.copy_(integers((m, 2048), 4, BF16, seed))
        g.replay()
        assert torch.equal(y, (x.double() @ w.double().T).float())
