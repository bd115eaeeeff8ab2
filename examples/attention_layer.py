"""An attention layer in 8 bits: trained for some steps, then served.

Training: the four projections are `TokenLinear`s, so their products and both gradients run on 8-bit codes with a scale for each token
and output channel; the scores of whole sequences are elementary torch operations here.  Serving: the projections' weights are laid
out once (`ServedLinear`), keys and values go into a `PagedCache` as they arrive - prompts in chunks of unequal requests, then one token
of every request at a time - and new tokens attend over it.

    python examples/attention_layer.py                 # needs a GPU
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1912_12607_amd.tokens import PagedCache, TokenLinear  # noqa: E402


class Attention(torch.nn.Module):
    """Causal attention; `heads` query heads share `kv_heads` heads of keys and values."""

    def __init__(self, width: int, heads: int, kv_heads: int, dim: int, dtype=torch.bfloat16, device="cuda:0"):
        super().__init__()
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        self.q = TokenLinear(width, heads * dim, dtype=dtype, device=device, name="q")
        self.k = TokenLinear(width, kv_heads * dim, dtype=dtype, device=device, name="k")
        self.v = TokenLinear(width, kv_heads * dim, dtype=dtype, device=device, name="v")
        self.o = TokenLinear(heads * dim, width, dtype=dtype, device=device, name="o")

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        """x (sequences, length, width)"""
        n, L, _ = x.shape

        def split(y, heads):                       # (sequences * query heads, length, dim); shared heads repeated for their group
            y = y.float().view(n, L, heads, self.dim).transpose(1, 2)
            return y.repeat_interleave(self.heads // heads, 1).reshape(n * self.heads, L, self.dim)
        q, k, v = split(self.q(x), self.heads), split(self.k(x), self.kv_heads), split(self.v(x), self.kv_heads)
        scores = torch.bmm(q, k.transpose(1, 2).contiguous()) * self.dim ** -0.5
        later = torch.ones(L, L, dtype=torch.bool, device=x.device).triu(1)
        out = torch.bmm(scores.masked_fill(later, float("-inf")).softmax(-1), v)
        return self.o(out.view(n, self.heads, L, self.dim).transpose(1, 2).reshape(n, L, -1).to(x.dtype))


class Served:
    """An `Attention` in use: a cache with `pages` pages, dealt out to requests as they grow."""

    def __init__(self, layer: Attention, requests: int, pages: int, page_size: int = 16):
        self.layer = layer
        self.q, self.k, self.v, self.o = (m.served() for m in (layer.q, layer.k, layer.v, layer.o))
        device = layer.q.weight.device
        self.cache = PagedCache.empty(pages, page_size, layer.kv_heads, layer.dim, device)
        self.free = list(range(pages))[::-1]
        self.pages = [[] for _ in range(requests)]
        self.lengths = [0] * requests

    def place(self, counts: list[int]):
        """Places for counts[b] more tokens of each request b: (slots, starts, lengths, table) on the device, and the longest length."""
        size, slots, starts = self.cache.page_size, [], [0]
        for b, n in enumerate(counts):
            for at in range(self.lengths[b], self.lengths[b] + n):
                if at // size == len(self.pages[b]):
                    self.pages[b].append(self.free.pop())
                slots.append(self.pages[b][at // size] * size + at % size)
            self.lengths[b] += n
            starts.append(starts[-1] + n)
        wide = max(1, max(map(len, self.pages)))
        table = [p + [-1] * (wide - len(p)) for p in self.pages]
        device = self.cache.kq.device
        ints = [torch.tensor(t, dtype=torch.int32).to(device) for t in (starts, self.lengths, table)]
        return torch.tensor(slots, dtype=torch.int64).to(device), *ints, max(self.lengths)

    def step(self, x: torch.Tensor, counts: list[int]) -> torch.Tensor:
        """New tokens of all requests, one request's after another's: x (sum of counts, width)."""
        slots, starts, lengths, table, longest = self.place(counts)
        T, L = x.shape[0], self.layer
        self.cache.write(self.k(x).view(T, L.kv_heads, L.dim), self.v(x).view(T, L.kv_heads, L.dim), slots)
        out = self.cache.attend(self.q(x).view(T, L.heads, L.dim), starts, lengths, table, longest=longest)
        return self.o(out.view(T, -1))


def train(layer: Attention, steps: int, sequences: int = 4, length: int = 64, rate: float = 1e-3) -> list[float]:
    """Fits the layer to `mean of the tokens so far`; the loss of each step."""
    device, width = layer.q.weight.device, layer.q.in_features
    g = torch.Generator(device=device).manual_seed(1)
    optimiser = torch.optim.Adam(layer.parameters(), lr=rate)
    losses = []
    for _ in range(steps):
        x = torch.randn(sequences, length, width, generator=g, device=device)
        target = x.cumsum(1) / torch.arange(1, length + 1, device=device).view(1, -1, 1)
        optimiser.zero_grad()
        loss = (layer(x.to(layer.q.weight.dtype)).float() - target).square().mean()
        loss.backward()
        optimiser.step()
        losses.append(loss.item())
    return losses


def serve(layer: Attention, x: list[torch.Tensor], chunk: int, singles: int, page_size: int = 16) -> list[torch.Tensor]:
    """Outputs for the tokens of each request x[b] (length, width): all but the last `singles` in chunks, these one at a time."""
    served = Served(layer, len(x), sum(-(-t.shape[0] // page_size) for t in x), page_size)
    done, outs = [0] * len(x), [[] for _ in x]
    while any(n < t.shape[0] for n, t in zip(done, x)):
        counts = [min(chunk, t.shape[0] - singles - n) if n < t.shape[0] - singles else min(1, t.shape[0] - n) for n, t in zip(done, x)]
        y = served.step(torch.cat([t[n:n + c] for t, n, c in zip(x, done, counts)]), counts)
        for b, part in enumerate(y.split(counts)):
            outs[b].append(part)
            done[b] += counts[b]
    return [torch.cat(o) for o in outs]


def main(argv=None) -> dict:
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--width", type=int, default=512)
    p.add_argument("--heads", type=int, default=8)
    p.add_argument("--kv-heads", type=int, default=2)
    p.add_argument("--dim", type=int, default=64)
    p.add_argument("--steps", type=int, default=100)
    p.add_argument("--lengths", type=int, nargs="+", default=[200, 33, 117, 64])
    p.add_argument("--chunk", type=int, default=48)
    p.add_argument("--singles", type=int, default=16)
    a = p.parse_args(argv)
    torch.manual_seed(0)
    layer = Attention(a.width, a.heads, a.kv_heads, a.dim)
    losses = train(layer, a.steps)
    print(f"training: loss {losses[0]:.4f} -> {losses[-1]:.4f} in {a.steps} steps", flush=True)
    x = [torch.randn(n, a.width, device="cuda:0").bfloat16() for n in a.lengths]
    with torch.no_grad():
        whole = [layer(t[None])[0].float() for t in x]
        serve(layer, x, a.chunk, a.singles)                    # (first calls load code)
        torch.cuda.synchronize()
        begin = time.perf_counter()
        out = serve(layer, x, a.chunk, a.singles)
        torch.cuda.synchronize()
        seconds = time.perf_counter() - begin
    error = max(float((y.float() - w).norm() / w.norm()) for y, w in zip(out, whole))
    print(f"serving: {len(x)} requests, {sum(a.lengths)} tokens in {1e3 * seconds:.1f} ms; from whole sequences with keys and values in {x[0].dtype}: {100 * error:.2f} %", flush=True)
    return {"losses": losses, "error": error}


if __name__ == "__main__":
    main()
