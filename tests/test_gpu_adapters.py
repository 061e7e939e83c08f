"""Low-rank adapters against their definition in 64 bits."""
import pytest
import torch

from batch_helpers import BF16, F64, ints, sums
from operator_helpers import rounds_from
from paper_2406_06237_b200 import binding as B
from paper_2406_06237_b200.runtime import Adapters

pytestmark = pytest.mark.gpu
F32, E4M3 = torch.float32, torch.float8_e4m3fn


def make(count, rank, n_in, n_out, rows, x_dtype=BF16, y_dtype=BF16, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=g)

    x = normal(rows, n_in).to(x_dtype)
    xs = 0.5 + torch.rand(rows, device="cuda", generator=g) if x_dtype is E4M3 else None
    a, b = (normal(count, rank, n_in) / n_in ** 0.5).to(BF16), normal(count, n_out, rank).to(BF16)
    return x, xs, a, b, 0.5 + torch.rand(count, device="cuda", generator=g), normal(rows, n_out).to(y_dtype)


def definition(x, xs, a, b, scales, y, which, starts):
    """(result, error before the last rounding).  h = x A^T is summed in fp32 in groups of 16, in up to n_in / 16 + 16 additions, each
    off by at most 2^-22 of the sum of magnitudes; two factors round it by 2^-24 each; as two bf16 numbers it is within
    2^-17; its product with B is 2 rank / 16 additions more and one with y, each within 2^-22 of the magnitudes."""
    out, slack = y.to(F64), torch.zeros(y.shape, dtype=F64, device=y.device)
    for s, i in enumerate(which):
        r0, r1 = starts[s], starts[s + 1]
        if i < 0 or r0 == r1:
            continue
        f = scales[i].to(F64) if scales is not None else torch.ones((), dtype=F64, device=y.device)
        u, w, v = x[r0:r1].to(F64), a[i].to(F64), b[i].to(F64)
        if xs is not None:
            u = u * xs[r0:r1, None].to(F64)
        h, mass = f * (u @ w.T), f * (u.abs() @ w.abs().T)
        out[r0:r1] += h @ v.T
        off = (2.0 ** -17 + 2.0 ** -23) * h.abs() + (x.shape[1] / 16 + 16) * 2.0 ** -22 * mass
        slack[r0:r1] = off @ v.abs().T + (2 * a.shape[1] / 16 + 3) * 2.0 ** -22 * (mass @ v.abs().T + y[r0:r1].to(F64).abs())
    return out, slack


def check(x, xs, a, b, scales, y, which, starts, out=None):
    f = Adapters(a, b, scales)
    was = y.clone()
    got = f(x, y, ints(which), ints(starts), x_scales=xs, out=out)
    assert f.read_status() == 0
    want, slack = definition(x, xs, a, b, scales, was, which, starts)
    n = starts[-1]
    ok = rounds_from(got[:n], want[:n], slack[:n])
    assert ok.all(), (int((~ok).sum()), ok.numel(), float((got[:n].double() - want[:n]).abs().max()))
    for s, i in enumerate(which):
        if i < 0:
            assert torch.equal(got[starts[s]:starts[s + 1]], was[starts[s]:starts[s + 1]])
    return got


@pytest.mark.parametrize("rank", [1, 4, 8, 16, 24, 32, 50, 64, 128])
@pytest.mark.parametrize("n_in,n_out", [(512, 768), (1000, 1000), (333, 257), (64, 8), (2048, 70)])
@pytest.mark.parametrize("new", [[1] * 9, [70, 0, 5, 16, 129]])
def test_shapes(rank, n_in, n_out, new):
    starts = sums(new)
    which = [(3 * s) % 5 if s != 2 else -1 for s in range(len(new))]
    check(*make(5, rank, n_in, n_out, starts[-1]), which, starts)


@pytest.mark.parametrize("x_dtype", [BF16, E4M3])
@pytest.mark.parametrize("y_dtype", [BF16, F32])
@pytest.mark.parametrize("rank,n_in,n_out,new", [(16, 1024, 1024, [1, 1, 1]), (32, 4096, 2048, [100, 33]), (64, 640, 1500, [17, 40, 3]), (8, 100, 60, [5, 50]), (128, 2048, 512, [20])])
def test_types(x_dtype, y_dtype, rank, n_in, n_out, new):
    starts = sums(new)
    check(*make(3, rank, n_in, n_out, starts[-1], x_dtype, y_dtype), list(range(len(new))), starts)


def test_large_and_many():
    new = [200, 1, 64, 333]
    check(*make(4, 16, 8192, 8192, sum(new)), [3, 0, 0, 2], sums(new))
    new = [1] * 200
    check(*make(50, 16, 2048, 1024, 200), [(7 * s) % 51 - 1 for s in range(200)], sums(new))


def test_without_scales_in_place_and_strided():
    new = [30, 2]
    x, _, a, b, _, y = make(2, 16, 256, 200, 32)
    want = check(x, None, a, b, None, y, [1, 0], sums(new))
    packed = torch.zeros(32, 900, dtype=BF16, device="cuda")
    packed[:, 1:201], packed[:, 301:557] = y, x
    view = packed[:, 1:201]
    got = check(packed[:, 301:557], None, a, b, None, view, [1, 0], sums(new), out=view)         # nothing on 16 bytes, in place
    assert torch.equal(got, want) and (packed[:, 201:301] == 0).all() and (packed[:, 0] == 0).all()
    got = check(x, None, a, b, None, y, [1, 0], sums(new), out=y)
    assert got is y and torch.equal(got, want)


def test_padding_rows_and_ids_that_are_none():
    x, _, a, b, scales, y = make(3, 8, 128, 96, 20)
    f = Adapters(a, b, scales)
    out = torch.full_like(y, 5.0)
    f(x, y, ints([2, 0]), ints([0, 3, 7]), out=out)
    assert f.read_status() == 0 and (out[7:] == 5).all() and not (out[:7] == 5).all()
    f(x, y, ints([3, 0]), ints([0, 3, 7]), out=out)
    assert f.read_status() == B.ANS_STATUS_BAD_PAGE and torch.equal(out[:3], y[:3])
    f(x, y, ints([1, 0]), ints([0, 3, 21]), out=out)
    assert f.read_status() == B.ANS_STATUS_BAD_PAGE
    f(x, y, ints([-2, -1]), ints([0, 3, 7]), out=out)
    assert f.read_status() == 0 and torch.equal(out[:7], y[:7])
    assert f(x[:0], y[:0], ints([0]), ints([0, 0])).shape == (0, 96)


def test_nan_and_infinity_stay_in_their_rows():
    x, _, a, b, scales, y = make(2, 16, 256, 64, 40)
    f = Adapters(a, b, scales)
    want = f(x, y, ints([0, 1]), ints([0, 20, 40]))
    x[3, 7], x[25, 0] = float("nan"), float("inf")
    got = f(x, y, ints([0, 1]), ints([0, 20, 40]))
    rows = torch.ones(40, dtype=torch.bool, device="cuda")
    rows[[3, 25]] = False
    assert torch.equal(got[rows], want[rows]) and got[3].isnan().all() and not got[25].isfinite().any()


def test_graph_and_repeats():
    x, _, a, b, scales, y = make(6, 16, 1024, 512, 80)
    f = Adapters(a, b, scales)
    which, starts = ints([0, 1, 5]), ints([0, 1, 50, 80])
    want = f(x, y, which, starts)
    for _ in range(4):
        assert torch.equal(f(x, y, which, starts), want)
    out = torch.empty_like(y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f(x, y, which, starts, out=out)
    which.copy_(ints([4, -1, 2]))
    starts.copy_(ints([0, 30, 31, 80]))
    a.mul_(-1)                                           # weights are read anew by each call
    graph.replay()
    assert torch.equal(out, f(x, y, which, starts)) and not torch.equal(out, want)
    want, slack = definition(x, None, a, b, scales, y, [4, -1, 2], [0, 30, 31, 80])
    assert rounds_from(out, want, slack).all() and f.read_status() == 0


def test_room_that_is_too_small_is_refused():
    x, _, a, b, scales, y = make(3, 16, 512, 256, 40)
    f = Adapters(a, b, scales)
    f(x, y, ints([0, 2]), ints([0, 9, 40]))
    torch.cuda.synchronize()
    d = f._desc
    for size, place in ((d.room_bytes - 1, d.d_room), (d.room_bytes, None)):
        d.room_bytes, d.d_room = size, place
        with pytest.raises(B.AnsError) as e:
            B.ans_adapters(d, f._status)
        assert e.value.code == B.ANS_ERR_BUFFER_TOO_SMALL


@pytest.mark.parametrize("rank,n_in,n_out", [(16, 512, 1024), (32, 1100, 300), (100, 64, 512)])
@pytest.mark.parametrize("seqs", [3, 256, 257, 700])
def test_shares_of_ragged_requests(rank, n_in, n_out, seqs):
    """Blocks have parts of several requests' tiles: requests of many sizes, without rows, without adapters, out beside y and over it."""
    new = [(7 * s * s + 3 * s) % (1 + 4000 // seqs) for s in range(seqs)]
    new[seqs // 2] += 300
    which = [(5 * s) % 9 - 1 if s % 4 else -1 for s in range(seqs)]
    x, _, a, b, scales, y = make(8, rank, n_in, n_out, sum(new) + 40)
    got = check(x, None, a, b, scales, y, which, sums(new))
    for _ in range(3):
        over = y.clone()
        assert check(x, None, a, b, scales, over, which, sums(new), out=over) is over
        assert torch.equal(over[:sum(new)], got[:sum(new)]) and torch.equal(over[sum(new):], y[sum(new):])
