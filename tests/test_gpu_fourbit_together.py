"""The operators as a program uses them together: prompts and then single tokens of several requests through a layer in 4 bits, with rotary positions, pages found on the
GPU and a cache in 4 bits; eager, on another stream, and captured into a graph."""
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import fourbit_reference as R  # noqa: E402
from paper_1912_12607_amd import fourbit  # noqa: E402
from paper_1912_12607_amd.positions import PageTable, Rotary  # noqa: E402

DEV = torch.device("cuda:0")
HEADS, GROUP, DIM, PAGE, WIDE = 2, 2, 64, 16, 96
HQ = HEADS * GROUP


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class Layer:
    def __init__(self, seed, requests, width, pages):
        gen = torch.Generator().manual_seed(seed)
        self.w = torch.randn((HQ + 2 * HEADS) * DIM, WIDE, generator=gen) * 0.1
        self.wo = torch.randn(WIDE, HQ * DIM, generator=gen) * 0.06
        self.qkv, self.out = fourbit.ServedLinear4.of(self.w.to(DEV)), fourbit.ServedLinear4.of(self.wo.to(DEV))
        self.rotary = Rotary(DIM // 2, layout="interleaved").to(DEV)
        self.cache = fourbit.PagedCache4.empty(pages, PAGE, HEADS, DIM, DEV)
        self.pages = PageTable.empty(requests, width, pages, PAGE)

    def __call__(self, x, new, longest=None):
        step = self.pages.extend(new, x.shape[0])
        q, k, v = self.qkv(x).view(-1, HQ + 2 * HEADS, DIM).split([HQ, HEADS, HEADS], 1)
        self.rotary.turn_(q, k, step.positions)
        self.cache.write(k, v, step.slots)
        o = self.cache.attend(q, step.starts, step.lengths, self.pages.table, longest=longest)
        self.pages.accept(step)
        return self.out(o.view(-1, HQ * DIM))


def turned(x, positions):
    f = 10000.0 ** (-np.arange(0, DIM // 2, 2) / (DIM // 2))
    t = positions[:, None, None] * f
    a, b = x[..., 0:DIM // 2:2], x[..., 1:DIM // 2:2]
    y = x.copy()
    y[..., 0:DIM // 2:2], y[..., 1:DIM // 2:2] = a * np.cos(t) - b * np.sin(t), a * np.sin(t) + b * np.cos(t)
    return y


def plain(layer, xs):
    """Every request's tokens at once, in 64 bits: codes where codes are made, no other rounding.  A value next to the border of two codes falls to the other side in fp32 now
    and then (a step of a code, 1/6 of a block's largest at most), so this is near, not equal."""
    out = []
    for x in xs:
        n = x.shape[0]
        y = (R.rounded(x) @ R.rounded(layer.w.double().numpy()).T).reshape(n, -1, DIM)
        q, k, v = y[:, :HQ], y[:, HQ:HQ + HEADS], y[:, HQ + HEADS:]
        q, k = turned(q, np.arange(n)), turned(k, np.arange(n))
        k, v = (R.rounded(t.reshape(-1, DIM)).reshape(t.shape) for t in (k, v))
        o = np.zeros((n, HQ, DIM))
        for h in range(HQ):
            s = q[:, h] @ k[:, h // GROUP].T / DIM**0.5
            s[np.arange(n)[:, None] < np.arange(n)[None]] = -np.inf
            p = np.exp(s - s.max(1, keepdims=True))
            o[:, h] = p / p.sum(1, keepdims=True) @ v[:, h // GROUP]
        out.append(R.rounded(o.reshape(n, -1)) @ R.rounded(layer.wo.double().numpy()).T)
    return out


def test_prompts_and_single_tokens():
    prompts, steps = [37, 1, 16, 60], 20
    xs = [torch.randn(n + steps, WIDE, generator=torch.Generator().manual_seed(10 + i)) for i, n in enumerate(prompts)]
    layer = Layer(1, 4, 8, 24)
    got = [[] for _ in prompts]
    y = layer(torch.cat([x[:n] for x, n in zip(xs, prompts)]).to(DEV), ints(prompts))
    for b, part in enumerate(y.split(prompts)):
        got[b].append(part)
    for t in range(steps):
        y = layer(torch.stack([x[n + t] for x, n in zip(xs, prompts)]).to(DEV), ints([1] * 4))
        for b in range(4):
            got[b].append(y[b:b + 1])
    for b, want in enumerate(plain(layer, [x.double().numpy() for x in xs])):
        off = torch.cat(got[b]).double().cpu().numpy() - want
        # codes that fall to the other side: a few per thousand, each some per cent of a result
        assert np.sqrt((off**2).mean()) <= 0.02 * np.sqrt((want**2).mean())


def test_captured_steps_follow_eager_ones():
    """Single tokens with requests that pause, captured once with room for more tokens than there are, replayed beside eager work; equal to an eager layer of its own."""
    captured, eager = Layer(2, 3, 6, 20), Layer(2, 3, 6, 20)
    prompts = [30, 5, 17]
    x0 = torch.randn(sum(prompts), WIDE, generator=torch.Generator().manual_seed(3)).to(DEV)
    assert torch.equal(captured(x0, ints(prompts)), eager(x0, ints(prompts)))
    x, new = torch.zeros(4, WIDE, device=DEV), ints([0, 0, 0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        captured(x, new, longest=96)                           # (no new tokens: nothing changes)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = captured(x, new, longest=96)
    for t in range(6):
        n = [1, t % 2, 2 if t == 3 else 1]
        x.copy_(torch.randn(4, WIDE, generator=torch.Generator().manual_seed(20 + t)))
        new.copy_(ints(n))
        graph.replay()
        torch.cuda.synchronize()
        want = eager(x, ints(n), longest=96)
        assert torch.equal(y[:sum(n)], want[:sum(n)])
        assert captured.pages.lengths.tolist() == eager.pages.lengths.tolist()
        for a, b in zip(captured.cache._tensors, eager.cache._tensors):
            assert torch.equal(a, b)


def test_training_through_layers_and_rotary():
    """Two projections in 4 bits with rotary positions between: gradients reach both weights and the input, and go by the formulas' chain."""
    x = torch.randn(40, WIDE, generator=torch.Generator().manual_seed(1)).to(DEV).requires_grad_(True)
    w1 = (torch.randn(HQ * DIM, WIDE, generator=torch.Generator().manual_seed(2)) * 0.1).to(DEV).requires_grad_(True)
    w2 = (torch.randn(WIDE, HQ * DIM, generator=torch.Generator().manual_seed(3)) * 0.06).to(DEV).requires_grad_(True)
    at = torch.arange(40, dtype=torch.int32, device=DEV)
    g = torch.randn(40, WIDE, generator=torch.Generator().manual_seed(4)).to(DEV)
    rotary = Rotary(DIM)
    h = fourbit.linear4(x, w1, seed=5)
    r = rotary(h.view(40, HQ, DIM), None, at)
    y = fourbit.linear4(r.reshape(40, -1), w2, seed=6)
    dx, dw1, dw2 = torch.autograd.grad(y, [x, w1, w2], g)
    # the same, call by call
    r1 = r.detach().reshape(40, -1).requires_grad_(True)
    dr, dw2_ = torch.autograd.grad(fourbit.linear4(r1, w2, seed=6), [r1, w2], g)
    h1 = h.detach().requires_grad_(True)
    dh, = torch.autograd.grad(rotary(h1.view(40, HQ, DIM), None, at), h1, dr.view(40, HQ, DIM))
    dx_, dw1_ = torch.autograd.grad(fourbit.linear4(x, w1, seed=5), [x, w1], dh)
    assert torch.equal(dx, dx_) and torch.equal(dw1, dw1_) and torch.equal(dw2, dw2_)
