"""Serving an attention block with static quantization: the linears q, k, v and o from this library's W8A8 kernels, the rotation, the
paged key/value cache and the attention between them.

    python examples/serve_attention.py [--int8]

Three users' prompts of different lengths go in together, then tokens one at a time; a fourth user's prompt arrives in chunks beside
them.  At the end every output is compared with that of the same block run over each user's whole text at once.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2512_14481_amd import binding as B  # noqa: E402


class Linear:
    """A frozen W8A8 linear with its static activation factor."""

    def __init__(self, out_features: int, in_features: int, generator: torch.Generator, s: float):
        w = torch.randn(out_features, in_features, generator=generator, device="cuda") * in_features ** -0.5
        self.wq = torch.empty(out_features, in_features, dtype=torch.int8, device="cuda")
        self.s_w = torch.empty(out_features, device="cuda")
        B.sasq_quantize_weight(w, self.wq, self.s_w)
        self.s = torch.tensor([s], device="cuda")

    def __call__(self, x: torch.Tensor) -> torch.Tensor:
        (m, k), n = x.shape, self.wq.shape[0]
        y = torch.empty(m, n, dtype=x.dtype, device="cuda")
        B.sasq_static_linear(x, self.s, self.wq, self.s_w, None, y, B.SASQ_W_INT8, B.new_workspace(B.sasq_static_linear_workspace(m, n, k, B.SASQ_W_INT8)))
        return y


class Pages:
    """Which pages of a cache belong to which user."""

    def __init__(self, pages: int, page_size: int, users: int, most: int):
        self.free, self.page_size = list(range(pages)), page_size
        self.length = [0] * users
        self.table = torch.full((users, -(-most // page_size)), -1, dtype=torch.int32)

    def step(self, new: list[int]) -> B.KVBatch:
        """Makes room for so many new tokens of each user; the step's batch."""
        for u, n in enumerate(new):
            self.length[u] += n
            for i in range(-(-self.length[u] // self.page_size)):
                if self.table[u, i] < 0:
                    self.table[u, i] = self.free.pop()
        cu = torch.tensor([0] + new).cumsum(0).to(torch.int32)
        return B.KVBatch(cu.cuda(), torch.tensor(self.length, dtype=torch.int32).cuda(), self.table.cuda(), sum(new), max_q=max(new), max_kv=max(self.length))


class AttentionBlock:
    def __init__(self, hidden: int, heads: int, kv_heads: int, positions: int, pages: int, page_size: int, dtype: torch.dtype, int8: bool, seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.heads, self.kv_heads, self.dim = heads, kv_heads, hidden // heads
        self.qkv = Linear((heads + 2 * kv_heads) * self.dim, hidden, g, 4 / 127)
        self.o = Linear(hidden, heads * self.dim, g, 2 / 127)
        half = self.dim // 2
        angle = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
        self.cos, self.sin = angle.cos().float(), angle.sin().float()
        shape = (pages, kv_heads, page_size, self.dim)
        if int8:                                                     # static factors, one for each kv head
            k, v = torch.zeros(shape, dtype=torch.int8, device="cuda"), torch.zeros(shape, dtype=torch.int8, device="cuda")
            scales = (torch.full((kv_heads,), 5 / 127, device="cuda"), torch.full((kv_heads,), 5 / 127, device="cuda"))
        else:
            k, v, scales = torch.empty(shape, dtype=dtype, device="cuda"), torch.empty(shape, dtype=dtype, device="cuda"), (None, None)
        self.cache = B.KVCache(k.transpose(1, 2), v.transpose(1, 2), *scales)

    def __call__(self, x: torch.Tensor, batch: B.KVBatch) -> torch.Tensor:
        """x [tokens, hidden] of the batch's rows."""
        H, Hk, D = self.heads, self.kv_heads, self.dim
        qkv = self.qkv(x).view(-1, H + 2 * Hk, D)
        q = torch.empty(len(x), H, D, dtype=x.dtype, device="cuda")
        B.sasq_kv_append(qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:], q, self.cache, batch, self.cos, self.sin)
        a = torch.empty_like(q)
        workspace = B.new_workspace(B.sasq_paged_attention_workspace(self.cache, batch, H))
        B.sasq_paged_attention(q, a, self.cache, batch, workspace, D ** -0.5)
        return self.o(a.view(len(x), H * D))


def main(int8: bool = False, hidden: int = 1024, heads: int = 8, kv_heads: int = 2, dtype: torch.dtype = torch.float16) -> float:
    """The largest difference between serving in steps and all at once, relative to the outputs' root mean square."""
    prompts, chunks, tokens, page_size = [70, 1, 200], [64, 64, 33], 5, 16
    texts = [n + len(chunks) + tokens for n in prompts] + [sum(chunks) + tokens]
    g = torch.Generator(device="cuda").manual_seed(1)
    text = [torch.randn(n, hidden, generator=g, device="cuda").to(dtype) for n in texts]
    make = lambda: AttentionBlock(hidden, heads, kv_heads, max(texts), 64, page_size, dtype, int8)
    layer, pages = make(), Pages(64, page_size, 4, max(texts))
    at, served = [0] * 4, [[] for _ in range(4)]

    def step(new):
        x = torch.cat([text[u][at[u]:at[u] + n] for u, n in enumerate(new)])
        y = layer(x, pages.step(new))
        for u, part in enumerate(y.split(new)):
            at[u] += new[u]
            served[u].append(part)

    step(prompts + [0])                                              # three prompts together
    for n in chunks:                                                 # a token for each of them, the fourth prompt's chunks beside
        step([1, 1, 1, n])
    for _ in range(tokens):
        step([1, 1, 1, 1])
    whole = make()(torch.cat(text), Pages(64, page_size, 4, max(texts)).step(texts))
    steps = torch.cat([torch.cat(parts) for parts in served])
    return ((steps.double() - whole.double()).abs().max() / whole.double().square().mean().sqrt()).item()


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    parser.add_argument("--int8", action="store_true", help="keep keys and values as int8 codes with static factors")
    print(f"served in steps against all at once: largest difference {main(parser.parse_args().int8):.2e} of the outputs' root mean square")
