"""Many requests at once through a decoder block from compressed weights: prompts of different lengths together, then all
requests token by token.  A step is

    page tables -> norm (8-bit rows) -> product q, k, v + each request's adapter -> cache -> attention over it
                -> product + residual + adapter -> norm (8-bit rows) -> product with gelu -> product + residual

The weights are those of decoder_block.py, shared by all requests; the adapters are the requests' own, bf16.  The steps of
single tokens run as one captured graph: lengths, tables and row ranges are made on the GPU, in place, so that a replay is the next step.

    python examples/decoder_requests.py [--width 1024] [--heads 8] [--requests 5] [--prompt 200] [--tokens 16] [--rank 16]

prints the norm of the deviation from the same requests in fp32, one by one, relative to the norm of their outputs, and the time of a step.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from decoder_block import BF16, E4M3, Weights  # noqa: E402
from paper_2406_06237_b200.runtime import Adapters, BlockCache, Linear, PageTables, RmsNorm  # noqa: E402


def make_adapters(width, rank, count, gen):
    """For the products q, k, v and out: {name: (a, b)}."""
    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=gen)
    return {name: ((normal(count, rank, width) / width ** 0.5).to(BF16), (0.3 * normal(count, n, rank) / rank ** 0.5).to(BF16))
            for name, n in (("qkv", 3 * width), ("out", width))}


class Server:
    def __init__(self, weights, adapters, scales, width, heads, requests, pages, page):
        self.heads, self.dim, self.requests = heads, width // heads, requests
        norms = torch.ones(width, dtype=BF16, device="cuda")
        self.norm1, self.norm2 = RmsNorm(norms, out_dtype=E4M3), RmsNorm(norms, out_dtype=E4M3)

        def linear(name, activation="none"):
            w, scale = weights.matrix(name)
            return Linear(w, scales=scale, activation=activation, settled=True)

        self.qkv, self.out, self.up, self.down = linear("qkv"), linear("out"), linear("up", "gelu"), linear("down")
        self.qkv_own, self.out_own = (Adapters(*adapters[name], scales) for name in ("qkv", "out"))
        self.cache = BlockCache(pages, page, heads, self.dim)
        self.pages = PageTables(page)
        self.tables = torch.zeros(requests, -(-pages // requests) + 1, dtype=torch.int32, device="cuda")
        self.free = torch.randperm(pages, device="cuda").to(torch.int32)
        self.lengths = torch.zeros(requests, dtype=torch.int32, device="cuda")
        self.taken = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.buffers = {}

    def __call__(self, x, new, which, longest):
        """x: [rows, width] bf16, the requests' new tokens in a row; new, which: [requests] int32.  Returns the residual stream."""
        rows = x.shape[0]
        if rows not in self.buffers:
            self.buffers[rows] = self.pages.buffers(self.requests, rows)._replace(lengths=self.lengths, taken=self.taken)
        batch = self.pages(self.tables, self.lengths, new, self.free, self.taken, out=self.buffers[rows])
        y, scales, _ = self.norm1(x)
        qkv = self.qkv(y, x_scales=scales)
        self.qkv_own(y, qkv, which, batch.starts, x_scales=scales, out=qkv)
        q, k, v = qkv.unflatten(1, (3, self.heads, self.dim)).unbind(1)
        self.cache.write(k, v, self.tables, batch.lengths, batch.starts)
        mixed = self.cache.attend(q, self.tables, batch.lengths, batch.starts, longest=longest).flatten(1)
        x = self.out(mixed, residual=x)
        self.out_own(mixed, x, which, batch.starts, out=x)
        y, scales, _ = self.norm2(x)
        return self.down(self.up(y, x_scales=scales), residual=x)

    def parts(self):
        return (self.qkv, self.out, self.up, self.down, self.qkv_own, self.out_own, self.cache, self.pages)


def plain(weights, adapters, scales, which, x, heads):
    """One request in fp32, its whole sequence at once."""
    def w(name):
        m, scale = weights.matrix(name)
        m = m.float() * (scale or 1)
        if which >= 0 and name in adapters:
            m = m + scales[which] * adapters[name][1][which].float() @ adapters[name][0][which].float()
        return m

    def norm(h):
        return h * torch.rsqrt((h * h).mean(1, keepdim=True) + 1e-6)

    tokens, width = x.shape
    q, k, v = (norm(x) @ w("qkv").T).unflatten(1, (3, heads, width // heads)).unbind(1)
    score = torch.einsum("qhd,khd->hqk", q, k) * (width // heads) ** -0.5
    later = torch.ones(tokens, tokens, dtype=torch.bool, device="cuda").triu(1)
    x = x + torch.einsum("hqk,khd->qhd", score.masked_fill(later, float("-inf")).softmax(2), v).flatten(1) @ w("out").T
    return x + torch.nn.functional.gelu(norm(x) @ w("up").T) @ w("down").T


def run(width=1024, heads=8, requests=5, prompt=200, tokens=16, rank=16, page=16, seed=0):
    """Returns (relative deviation from fp32, seconds a step of one token a request)."""
    weights = Weights(width, 4 * width, seed)
    gen = torch.Generator("cuda").manual_seed(seed)
    count = requests
    adapters, scales = make_adapters(width, rank, count, gen), 0.5 + torch.rand(count, device="cuda", generator=gen)
    which = [i if i % 3 != 2 else -1 for i in range(requests)]                 # some without an adapter
    prompts = [prompt - prompt * i // (2 * requests) for i in range(requests)]
    pages = sum(-(-(p + tokens) // page) for p in prompts) + requests * -(-(prompt + tokens) // page)
    server = Server(weights, adapters, scales, width, heads, requests, pages, page)
    x = [torch.randn(p + tokens, width, device="cuda", generator=gen).to(BF16) for p in prompts]
    ids = torch.tensor(which, dtype=torch.int32, device="cuda")
    new = torch.tensor(prompts, dtype=torch.int32, device="cuda")
    got = [list(server(torch.cat([s[:p] for s, p in zip(x, prompts)]), new, ids, prompt).split(prompts))]

    def rows(step):
        return torch.stack([s[p + step] for s, p in zip(x, prompts)])

    new.fill_(1)
    if tokens:
        got.append(list(server(rows(0), new, ids, 1).split(1)))
    if tokens > 1:
        given = rows(1).clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            result = server(given, new, ids, 1)
        torch.cuda.synchronize()
        began = time.perf_counter()
        for step in range(1, tokens):
            given.copy_(rows(step))
            graph.replay()
            got.append(list(result.clone().split(1)))
        torch.cuda.synchronize()
    each = (time.perf_counter() - began) / (tokens - 1) if tokens > 1 else 0.0
    for part in server.parts():
        if part.read_status():
            raise RuntimeError("a kernel reported a fault")
    off = whole = 0.0
    for i, s in enumerate(x):
        want = plain(weights, adapters, scales, which[i], s.float(), heads)
        mine = torch.cat([part[i] for part in got]).float()
        off, whole = off + float((mine - want).square().sum()), whole + float(want.square().sum())
    return (off / whole) ** 0.5, each


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("width", 1024), ("heads", 8), ("requests", 5), ("prompt", 200), ("tokens", 16), ("rank", 16)):
        p.add_argument("--" + name, type=int, default=value)
    off, each = run(**vars(p.parse_args()))
    print(f"relative deviation from fp32 {off:.4f}; {each * 1e6:.0f} us a step")
