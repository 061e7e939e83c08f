"""A language model's decoder block from compressed weights: every matrix stays entropy coded until it is loaded, then

    norm (8-bit rows) -> product q, k, v -> cache -> attention -> product + residual
    norm (8-bit rows) -> product with gelu -> product + residual

for a prompt and then token by token.  The weights that meet 8-bit rows are 4-bit symbols, held as e4m3 values
q - zero_point; the others are decoded to bf16.  The attention itself is plain torch on what the cache reads back.

    python examples/decoder_block.py [--width 1024] [--heads 8] [--prompt 200] [--tokens 16] [--bits 8]

prints the norm of the deviation from the same block in fp32 (unquantised activations and cache), relative to the norm of its
output, and the time of a token.
"""
import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2406_06237_b200 as ans  # noqa: E402
from paper_2406_06237_b200.runtime import DeviceBatch, Linear, PagedCache, RmsNorm, pack_layer, symbols_to_e4m3  # noqa: E402

BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn


def draw_symbols(rng, n, k, bits):
    """Laplacian symbols around the zero-point, as a zero-point quantiser leaves them."""
    zero = 1 << (bits - 1)
    q = np.rint(rng.laplace(0, 1.3 if bits <= 4 else 12, size=(n, k))) + zero
    return np.clip(q, 0, (1 << bits) - 1).astype(np.uint8)


class Weights:
    """Four matrices, packed, put on the GPU in compressed form and decoded by one launch."""

    def __init__(self, width, hidden, seed):
        rng = np.random.default_rng(seed)
        #            name   shape             bits  decoded to
        self.plan = [("qkv", (3 * width, width), 4, ans.ANS_U8), ("out", (width, width), 6, ans.ANS_BF16),
                     ("up", (hidden, width), 4, ans.ANS_U8), ("down", (width, hidden), 6, ans.ANS_BF16)]
        packed = []
        for _, (n, k), bits, dtype in self.plan:
            sym = draw_symbols(rng, n, k, bits)
            scale = 1.0 / (float(sym.std()) * k ** 0.5)
            packed.append(pack_layer(sym.reshape(-1), 1 << bits, 12, 16384, 32, ans.ANS_LAYOUT_QUADS, bits, 1 << (bits - 1), scale, dtype))
        self.batch = DeviceBatch(packed)
        self.batch.decode()
        if self.batch.read_status():
            raise RuntimeError("a compressed stream did not decode soundly")
        self.scale = {name: p.scale for (name, *_), p in zip(self.plan, packed)}
        self.bits = 8 * self.batch.compressed_bytes() / self.batch.n_symbols()

    def matrix(self, name):
        """(operand, scale): e4m3 values with the layer's scale, or bf16 weights and no scale."""
        i = [p[0] for p in self.plan].index(name)
        _, shape, bits, dtype = self.plan[i]
        if dtype == ans.ANS_BF16:
            return self.batch.output(i).view(shape), None
        return symbols_to_e4m3(self.batch.decode_symbols(i).view(shape), 1 << (bits - 1)), self.scale[name]


class Block:
    def __init__(self, weights, width, heads, pages, page, bits):
        self.heads, self.dim, self.page = heads, width // heads, page
        norms = torch.ones(width, dtype=BF16, device="cuda")
        self.norm1, self.norm2 = RmsNorm(norms, out_dtype=E4M3), RmsNorm(norms, out_dtype=E4M3)

        def linear(name, activation="none"):
            w, scale = weights.matrix(name)
            return Linear(w, scales=scale, activation=activation, settled=True)

        self.qkv, self.out, self.up, self.down = linear("qkv"), linear("out"), linear("up", "gelu"), linear("down")
        self.cache = PagedCache(pages, page, heads, self.dim, bits)
        self.table = torch.randperm(pages, device="cuda").to(torch.int32)[None]
        self.length = 0

    def __call__(self, x):
        """x: [tokens, width] bf16, the tokens after those seen so far; returns the residual stream behind the block."""
        tokens = x.shape[0]
        rows, scales, _ = self.norm1(x)
        q, k, v = self.qkv(rows, x_scales=scales).unflatten(1, (3, self.heads, self.dim)).unbind(1)
        at = torch.arange(self.length, self.length + tokens, device="cuda")
        self.cache.write(k, v, self.table[0, at // self.page].long() * self.page + at % self.page)
        self.length += tokens
        k, v = self.cache.read(self.table, torch.tensor([0, self.length], dtype=torch.int32, device="cuda"), self.length)
        score = torch.einsum("qhd,khd->hqk", q.float(), k.float()) * self.dim ** -0.5
        later = torch.arange(self.length, device="cuda") > at[:, None]
        mixed = torch.einsum("hqk,khd->qhd", score.masked_fill(later, float("-inf")).softmax(2), v.float())
        x = self.out(mixed.flatten(1).to(BF16), residual=x)
        rows, scales, _ = self.norm2(x)
        return self.down(self.up(rows, x_scales=scales), residual=x)


def plain(weights, x, heads):
    """The same block on a whole sequence in fp32."""
    def w(name):
        m, scale = weights.matrix(name)
        return m.float() * (scale or 1)

    def norm(h):
        return h * torch.rsqrt((h * h).mean(1, keepdim=True) + 1e-6)

    tokens, width = x.shape
    q, k, v = (norm(x) @ w("qkv").T).unflatten(1, (3, heads, width // heads)).unbind(1)
    score = torch.einsum("qhd,khd->hqk", q, k) * (width // heads) ** -0.5
    later = torch.ones(tokens, tokens, dtype=torch.bool, device="cuda").triu(1)
    x = x + torch.einsum("hqk,khd->qhd", score.masked_fill(later, float("-inf")).softmax(2), v).flatten(1) @ w("out").T
    return x + torch.nn.functional.gelu(norm(x) @ w("up").T) @ w("down").T


def run(width=1024, heads=8, prompt=200, tokens=16, bits=8, page=16, seed=0):
    """Returns (relative deviation from fp32, seconds a token, bits a weight)."""
    weights = Weights(width, 4 * width, seed)
    pages = -(-(prompt + tokens) // page) + 2
    block = Block(weights, width, heads, pages, page, bits)
    x = torch.randn(prompt + tokens, width, device="cuda", generator=torch.Generator("cuda").manual_seed(seed)).to(BF16)
    got = [block(x[:prompt])]
    torch.cuda.synchronize()
    began = time.perf_counter()
    for i in range(prompt, prompt + tokens):
        got.append(block(x[i:i + 1]))
    torch.cuda.synchronize()
    each = (time.perf_counter() - began) / max(tokens, 1)
    for part in (block.qkv, block.out, block.up, block.down, block.cache):
        if part.read_status():
            raise RuntimeError("a kernel reported a fault")
    want = plain(weights, x.float(), heads)
    off = float((torch.cat(got).float() - want).norm() / want.norm())
    return off, each, weights.bits


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("width", 1024), ("heads", 8), ("prompt", 200), ("tokens", 16), ("bits", 8)):
        p.add_argument("--" + name, type=int, default=value)
    off, each, weight_bits = run(**vars(p.parse_args()))
    print(f"weights at {weight_bits:.2f} bits; relative deviation from fp32 {off:.4f}; {each * 1e6:.0f} us a token")
