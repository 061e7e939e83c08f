"""Launches that overlap their ends keep the stream's order: an operator behind decode calls that wait for nothing."""
import numpy as np
import pytest
import torch

import paper_2406_06237_b200 as ans
from paper_2406_06237_b200.runtime import DeviceBatch, Linear, RmsNorm, pack_layer

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def packed(n, layout, seed):
    rng = np.random.default_rng(seed)
    sym = np.clip(np.rint(rng.laplace(0, 1.2, n)) + 8, 0, 15).astype(np.uint8)
    return pack_layer(sym, 16, 8, 4096, 32, layout, 4, 8, 0.25, ans.ANS_BF16), (sym.astype(np.float32) - 8) * 0.25


@pytest.mark.parametrize("layout", [ans.ANS_LAYOUT_QUADS, ans.ANS_LAYOUT_STRIPS])
def test_an_operator_behind_two_idle_decodes(layout):
    """A long product, a short and a long decode that wait for nothing (inputs settled, outputs idle), then a norm of
    the product's output and a product with each decoded matrix: all of them have to see finished work."""
    long, _ = packed(4096 * 4096, layout, 1)
    short, w_short = packed(128 * 256, layout, 2)
    batches = [DeviceBatch([p], inputs_settled=True, output_idle=True) for p in (long, short)]
    x = torch.randint(-4, 5, (2048, 8192), device="cuda").to(BF16)
    w = torch.randint(-4, 5, (4096, 8192), device="cuda").to(BF16)
    z = torch.randint(-4, 5, (40, 256), device="cuda").to(BF16)
    z2 = torch.randint(-4, 5, (40, 4096), device="cuda").to(BF16)
    product, norm = Linear(w), RmsNorm(None, out_dtype=F32, device="cuda")
    y = torch.empty(2048, 4096, device="cuda")
    by_short, by_long = Linear(batches[1].output(0).view(128, 256)), Linear(batches[0].output(0).view(4096, 4096))
    want_y = (x.double() @ w.double().T).float()
    want_short = (z.double() @ torch.from_numpy(w_short.reshape(128, 256)).cuda().double().T).float()
    batches[0].decode()
    torch.cuda.synchronize()
    want_long = by_long(z2, out_dtype=F32)
    for _ in range(10):
        y.zero_()
        for b in batches:
            b.out_sets[0][0].zero_()
        torch.cuda.synchronize()                         # the outputs are idle from here on
        product(x, out=y)
        batches[0].decode()
        batches[1].decode()
        n = norm(y)[0]
        s, g = by_short(z, out_dtype=F32), by_long(z2, out_dtype=F32)
        torch.cuda.synchronize()
        assert torch.equal(y, want_y) and torch.equal(s, want_short) and torch.equal(g, want_long)
        assert torch.equal(n, norm(want_y)[0])
        assert batches[0].read_status() == 0 and batches[1].read_status() == 0
