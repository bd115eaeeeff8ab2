"""Rotary positions and page tables against plain implementations on the CPU: rotations in 64 bits, pages request after request.  Whole numbers have to be equal."""
import math
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

from paper_1912_12607_amd import binding as B  # noqa: E402
from paper_1912_12607_amd.positions import PageTable, Rotary  # noqa: E402

DEV = torch.device("cuda:0")
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
HALF = {F32: 2.0**-24, BF16: 2.0**-8, F16: 2.0**-11}


# ---- rotary positions ------------------------------------------------------------------------------------------------------------
def turned(x, positions, frequencies, layout, amplitude=1.0, back=False):
    """(result, sum of the magnitudes of the two products that make a value), 64 bits."""
    x = x.detach().cpu().double()
    r = 2 * len(frequencies)
    t = positions.cpu().double()[..., None, None] * torch.as_tensor(frequencies, dtype=torch.float64)
    c, s = t.cos() * amplitude, t.sin() * amplitude * (-1 if back else 1)
    ia, ib = (slice(0, r // 2), slice(r // 2, r)) if layout == "half" else (slice(0, r, 2), slice(1, r, 2))
    a, b = x[..., ia], x[..., ib]
    y, size = x.clone(), x.abs()
    y[..., ia], y[..., ib] = a * c - b * s, a * s + b * c
    size[..., ia], size[..., ib] = (a.abs() + b.abs()) * abs(amplitude), (a.abs() + b.abs()) * abs(amplitude)
    return y, size


def close(got, want, size, dtype):
    """Sines and cosines are off by 4 steps of 2^-24 at most (two of the function, one of the product with the amplitude, one of the term that makes up for the angle's rounding),
    the products and their sum by one each: 6 2^-24 of the products' magnitudes; the result by half a step of its type."""
    assert got.dtype == dtype and got.shape == want.shape
    bound = 6 * 2.0**-24 * size + HALF[dtype] * 1.01 * want.abs() + (2.0**-25 if dtype is F16 else 0.0)
    off = (got.detach().cpu().double() - want).abs()
    assert bool((off <= bound).all()), (off / bound.clamp(min=1e-300)).max()


def normal(shape, seed, dtype):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


CASES = [(1, 1, 1, 2, 2), (1, 32, 8, 128, 128), (3, 5, 1, 80, 80), (70, 6, 2, 96, 48), (33, 3, 3, 64, 34), (17, 2, 1, 20, 18), (5, 1, 2, 256, 64), (1500, 4, 2, 64, 64), (2, 1, 1, 19, 6)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T,hq,hk,dim,rot", CASES)
def test_rotary_and_its_gradient(dtype, layout, T, hq, hk, dim, rot):
    q, k = normal((T, hq, dim), 1, dtype), normal((T, hk, dim), 2, dtype)
    gq, gk = normal((T, hq, dim), 3, dtype), normal((T, hk, dim), 4, dtype)
    at = torch.randint(0, 1 << 20, (T,), generator=torch.Generator().manual_seed(5), dtype=torch.int32).to(DEV)
    at[0] = 0
    rotary = Rotary(rot, layout=layout)
    f = [10000.0 ** (-2.0 * i / rot) for i in range(rot // 2)]
    q.requires_grad_(True), k.requires_grad_(True)
    yq, yk = rotary(q, k, at)
    for x, y in ((q, yq), (k, yk)):
        close(y, *turned(x, at, f, layout), dtype)
    dq, dk = torch.autograd.grad([yq, yk], [q, k], [gq, gk])
    for g, d in ((gq, dq), (gk, dk)):
        close(d, *turned(g, at, f, layout, back=True), dtype)
    # one alone, and one gradient alone, give the same
    assert torch.equal(rotary(q.detach(), None, at), yq) and torch.equal(rotary(k.detach(), None, at), yk)
    assert torch.equal(torch.autograd.grad(rotary(q.detach(), k, at)[1], k, gk)[0], dk)
    assert torch.equal(torch.autograd.grad(rotary(q, k, at)[0], q, gq)[0], dq)
    assert torch.equal(torch.autograd.grad(rotary(q, None, at), q, gq)[0], dq)
    # in place
    a, b = q.detach().clone(), k.detach().clone()
    rotary.turn_(a, b, at)
    assert torch.equal(a, yq) and torch.equal(b, yk)


def test_rotary_gradient_against_differences():
    """A turn is linear in what is turned: differences of <g, y> over a step of 1 are its gradient, but for fp32's rounding of y (2^-22 of the sums of magnitudes)."""
    T, h, dim, rot = 4, 2, 24, 20
    for layout in ("half", "interleaved"):
        rotary = Rotary(rot, layout=layout, amplitude=1.3, factor=2.0)
        q, g = normal((T, h, dim), 1, F32), normal((T, h, dim), 2, F32)
        at = torch.tensor([0, 3, 1000, 70000], dtype=torch.int32, device=DEV)
        x = q.clone().requires_grad_(True)
        dq, = torch.autograd.grad(rotary(x, None, at), x, g)
        for i in ((0, 0, 3), (1, 1, 19), (2, 0, 10), (3, 1, 0), (3, 0, 23)):
            up = q.clone()
            up[i] += 1.0
            diff = ((rotary(up, None, at).double() - rotary(q, None, at).double()) * g.double()).sum()
            assert abs(float(diff - dq[i])) <= 2.0**-20 * float(g[i[0]].abs().sum() * (q[i[0]].abs().max() + 1))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_scaled_frequencies(layout):
    rot, T = 64, 40
    q = normal((T, 2, 64), 1, F32)
    at = torch.arange(0, T * 25000, 25000, dtype=torch.int32, device=DEV)
    base = [500000.0 ** (-2.0 * i / rot) for i in range(rot // 2)]

    def bands(f):
        turns = 4096 * f / (2 * math.pi)
        keep = min(1.0, max(0.0, (turns - 1.0) / (4.0 - 1.0)))
        return f * keep + f / 8.0 * (1 - keep)
    for args, f, amplitude in ((dict(factor=4.0), [v / 4.0 for v in base], 1.0), (dict(factor=8.0, original=4096, slow=1.0, fast=4.0), [bands(v) for v in base], 1.0),
                               (dict(amplitude=1.2079), base, 1.2079), (dict(frequencies=[0.1 * i for i in range(32)]), [0.1 * i for i in range(32)], 1.0)):
        close(Rotary(rot, base=500000.0, layout=layout, **args)(q, None, at), *turned(q, at, f, layout, float(np.float32(amplitude))), F32)


@pytest.mark.parametrize("dtype", TYPES)
def test_rotary_at_the_farthest_positions(dtype):
    """Angles of 2^31 radians: 64 bits leave 2^-21 of a radian, as the reference's do (its own rounding of the angle is 2^-22), which the bound allows for."""
    at = torch.tensor([2**31 - 1, 2**31 - 2, 2**30 + 1, -1, -70000], dtype=torch.int32, device=DEV)
    q = normal((5, 3, 32), 1, dtype)
    want, size = turned(q, at, [10000.0 ** (-2.0 * i / 32) for i in range(16)], "half")
    got = Rotary(32)(q, None, at).cpu().double()
    assert bool(((got - want).abs() <= (6 * 2.0**-24 + 2.0**-20) * size + HALF[dtype] * 1.01 * want.abs() + 2.0**-25).all())


def test_rotary_of_strides_dimensions_and_nothing():
    rotary = Rotary(48)
    qkv = normal((9, 7, 64), 1, BF16)                    # queries, keys, values of a token side by side
    at = torch.arange(9, dtype=torch.int32, device=DEV) * 11
    q, k = qkv[:, :4], qkv[:, 4:6]
    wq, wk = rotary(q.contiguous(), k.contiguous(), at)
    yq, yk = rotary(q, k, at)
    assert torch.equal(yq, wq) and torch.equal(yk, wk)
    v = qkv[:, 6].clone()
    rotary.turn_(q, k, at)
    assert torch.equal(qkv[:, :4], wq) and torch.equal(qkv[:, 4:6], wk) and torch.equal(qkv[:, 6], v)
    x = normal((2, 3, 5, 64), 2, F16)
    at2 = torch.arange(6, dtype=torch.int32, device=DEV).view(2, 3) * 5
    want = rotary(x.view(6, 5, 64), None, at2.view(6)).view(2, 3, 5, 64)
    assert torch.equal(rotary(x, None, at2), want)
    swapped = x.transpose(1, 2).contiguous().transpose(1, 2)
    assert torch.equal(rotary(swapped, None, at2), want)
    y = x.clone()
    rotary.turn_(y, None, at2)
    assert torch.equal(y, want)
    odd = normal((9, 3, 65), 3, BF16)[..., 1:]            # heads off 16 bytes
    assert torch.equal(rotary(odd, None, at), rotary(odd.contiguous(), None, at))
    none = torch.zeros(0, 3, 64, device=DEV, requires_grad=True)
    y = rotary(none, None, torch.zeros(0, dtype=torch.int32, device=DEV))
    assert y.shape == (0, 3, 64) and torch.autograd.grad(y, none, torch.zeros_like(y))[0].shape == (0, 3, 64)


def test_turning_in_place_what_a_graph_has_kept_is_noticed():
    x = normal((3, 2, 16), 1, F32).requires_grad_(True)
    h = x * 2.0
    y = h * h                                            # keeps h
    with torch.no_grad():
        Rotary(16).turn_(h, None, torch.arange(3, dtype=torch.int32, device=DEV))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_rotary_of_what_is_not_finite():
    q = normal((3, 2, 16), 1, F32)
    q[1, 1, 2] = float("nan")
    y = Rotary(8)(q, None, torch.arange(3, dtype=torch.int32, device=DEV))
    bad = torch.zeros(3, 2, 16, dtype=torch.bool, device=DEV)
    bad[1, 1, 2], bad[1, 1, 6] = True, True
    assert torch.equal(torch.isnan(y), bad)


def test_rotary_refusals():
    r = Rotary(32)
    q, at = torch.zeros(4, 2, 64, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV)
    for call in (lambda: r(q, None, at.long()), lambda: r(q, None, at[:3]), lambda: r(q.cpu(), None, at), lambda: r(q, q.half(), at), lambda: r(q, q[:3], at), lambda: r(q, None, at.cpu()),
                 lambda: r(q[..., :16], None, at), lambda: r(q[0], None, at), lambda: r(q[:, :0], None, at), lambda: r.turn_(q, q, at), lambda: r.turn_(q[:, :1].expand(4, 2, 64), None, at),
                 lambda: r.turn_(q.clone().requires_grad_(True), None, at), lambda: r.turn_(torch.zeros(4, 64, 2, device=DEV).transpose(1, 2), None, at),
                 lambda: r.turn_(q[:, :2], q[:, 1:], at)):
        with pytest.raises(RuntimeError):
            call()
    with pytest.raises(TypeError):
        r(q.double(), None, at)
    x = q.clone().requires_grad_(True)
    with pytest.raises(RuntimeError, match="once"):
        torch.autograd.grad(r(x, None, at).sum(), x, create_graph=True)


# ---- pages -----------------------------------------------------------------------------------------------------------------------
class Plain:
    """The same, one request after the other."""

    def __init__(self, requests, width, pages, page_size):
        self.table, self.lengths, self.free, self.P, self.width = [[-1] * width for _ in range(requests)], [0] * requests, list(range(pages - 1, -1, -1)), page_size, width

    def extend(self, new, tokens):
        starts, slots, positions, lengths, asked, without, there = [0], [-1] * tokens, [0] * tokens, list(self.lengths), 0, 0, len(self.free)
        taken = 0
        for b, n in enumerate(new):
            n, h, begin = max(0, n), max(0, self.lengths[b]), starts[-1]
            starts.append(begin + n)
            held, want = -(-h // self.P), -(-(h + n) // self.P)
            fits = want <= self.width and begin + n <= tokens
            if fits:
                asked += want - held
            if not fits or (want > held and asked > there):
                without += 1
                continue
            for i in range(want - held):
                self.table[b][held + i] = self.free[there - 1 - (asked - (want - held) + i)]
            if want > held:
                taken = asked
            lengths[b] = h + n
            for i in range(n):
                slots[begin + i], positions[begin + i] = self.table[b][(h + i) // self.P] * self.P + (h + i) % self.P, h + i
        return lengths, there - taken, starts, slots, positions, without

    def accept(self, step):
        self.lengths, self.free = step[0], self.free[:step[1]]

    def shrink(self, stay):
        for b, n in enumerate(stay):
            n = max(0, min(n, self.lengths[b]))
            for k in range(-(-n // self.P), -(-self.lengths[b] // self.P)):
                self.free.append(self.table[b][k])
            self.lengths[b] = n


def same(step, want):
    for got, w in zip((step.lengths, step.available, step.starts, step.slots, step.positions, step.without), want):
        assert got.cpu().tolist() == (w if isinstance(w, list) else [w])


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("requests,width,pages,page", [(1, 4, 4, 16), (5, 9, 20, 7), (64, 20, 300, 16), (300, 8, 900, 24), (700, 40, 9000, 1), (3, 2000, 5000, 3)])
def test_pages_through_a_life(requests, width, pages, page):
    """Steps of all sizes, drafts that are not accepted, tokens taken back, requests that end, too few pages."""
    r = np.random.default_rng(requests)
    plain, pt = Plain(requests, width, pages, page), PageTable.empty(requests, width, pages, page)
    for i in range(14):
        most = [1, 3, page, 4 * page, width * page // 2][i % 5]
        new = r.integers(0, most + 1, requests).tolist()
        if i == 6:
            new[0] = width * page + 1                   # does not fit its row
        tokens = max(0, sum(new) + [0, 5, 1100, -3][i % 4])
        want = plain.extend(new, tokens)
        step = pt.extend(ints(new), tokens)
        same(step, want)
        assert pt.table.cpu().tolist() == plain.table and pt.lengths.cpu().tolist() == plain.lengths
        live = [s for s in step.slots.tolist() if s >= 0]
        assert len(set(live)) == len(live)
        if i % 4 != 3:
            pt.accept(step)
            plain.accept(want)
        if i % 3 == 2:
            stay = [int(r.integers(0, n + 3)) if r.random() < 0.5 else 0 for n in plain.lengths]
            pt.shrink(ints(stay))
            plain.shrink(stay)
            n = int(pt.available)
            assert n == len(plain.free) and pt.free.cpu().tolist()[:n] == plain.free and pt.lengths.cpu().tolist() == plain.lengths
    pt.shrink(ints([0] * requests))
    assert int(pt.available) == pages and sorted(pt.free.cpu().tolist()) == list(range(pages))


def test_pages_at_the_edges():
    pt = PageTable.empty(3, 4, 6, 16)
    # nothing new; more rows than tokens; none at all
    same(pt.extend(ints([0, 0, 0]), 0), ([0, 0, 0], 6, [0, 0, 0, 0], [], [], 0))
    same(pt.extend(ints([0, -7, 0]), 3), ([0, 0, 0], 6, [0, 0, 0, 0], [-1] * 3, [0] * 3, 0))
    # whole pages, then one more token: the next page
    step = pt.extend(ints([16, 1, 32]), 49)
    assert step.slots.tolist()[:16] == list(range(16)) and step.slots.tolist()[16] == 16 and int(step.available) == 2
    pt.accept(step)
    step = pt.extend(ints([1, 1, 1]), 3)
    assert step.positions.tolist() == [16, 1, 32] and int(step.available) == 0 and step.slots.tolist() == [4 * 16, 17, 5 * 16]
    pt.accept(step)
    # no page is left: those that need none go on
    step = pt.extend(ints([1, 14, 16]), 31)
    assert step.without.tolist() == [1] and step.lengths.tolist() == [18, 16, 33] and step.slots.tolist()[15:] == [-1] * 16
    step = pt.extend(ints([48, 14, 1]), 63)
    assert step.without.tolist() == [1] and step.lengths.tolist() == [17, 16, 34]
    # the batch ends inside a request
    step = pt.extend(ints([1, 2, 3]), 5)
    assert step.without.tolist() == [1] and step.lengths.tolist() == [18, 4, 33] and step.slots.tolist()[3:] == [-1, -1]
    empty = PageTable.empty(0, 1, 4, 16)
    same(empty.extend(ints([]), 2), ([], 4, [0], [-1, -1], [0, 0], 0))
    empty.shrink(ints([]))
    none = PageTable.empty(2, 0, 0, 16)
    same(none.extend(ints([1, 0]), 1), ([0, 0], 0, [0, 1, 1], [-1], [0], 1))


def test_pages_in_a_graph_and_on_another_stream():
    requests, width, pages, page = 5, 30, 100, 4
    pt, plain = PageTable.empty(requests, width, pages, page), Plain(requests, width, pages, page)
    new = ints([1] * requests)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step = pt.extend(new, 8)
    torch.cuda.current_stream().wait_stream(side)
    same(step, plain.extend([1] * requests, 8))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step = pt.extend(new, 8)
        pt.accept(step)
    for i in range(8):
        n = [(i + b) % 3 for b in range(requests)]
        new.copy_(ints(n))
        graph.replay()
        torch.cuda.synchronize()
        want = plain.extend(n, 8)
        plain.accept(want)
        same(step, want)
        assert pt.lengths.tolist() == plain.lengths and pt.table.cpu().tolist() == plain.table


def test_pages_refusals():
    pt = PageTable.empty(3, 4, 6, 16)
    t, n, f, a = pt.table, pt.lengths, pt.free, pt.available
    for call in (lambda: pt.extend(ints([1, 2]), 3), lambda: pt.extend(ints([1, 2, 3]).long(), 3), lambda: pt.extend(ints([1, 2, 3]).cpu(), 3), lambda: pt.extend(ints([1, 2, 3]), -1),
                 lambda: pt.shrink(ints([1, 2])), lambda: PageTable(t.cpu(), n, f, a, 16), lambda: PageTable(t, n[:2], f, a, 16), lambda: PageTable(t, n.long(), f, a, 16),
                 lambda: PageTable(t[:, ::2], n, f, a, 16), lambda: PageTable(t, n, f, a[:0], 16), lambda: PageTable(t, n, f, a, 0), lambda: PageTable(t, n, f, a, 1 << 30)):
        with pytest.raises(RuntimeError):
            call()
    with pytest.raises(B.Int8tError):
        pt.extend(ints([1, 2, 3]), 2**31 - 1)


@pytest.mark.parametrize("requests,width,pages,page", [(1, 3000, 3000, 4), (40, 700, 20000, 16), (1025, 9, 5000, 8), (2500, 300, 20000, 1)])
def test_many_pages_go_back(requests, width, pages, page):
    """Requests of many pages and many requests: some end, some keep a part, and then their pages are used again."""
    r = np.random.default_rng(pages)
    plain, pt = Plain(requests, width, pages, page), PageTable.empty(requests, width, pages, page)
    for _ in range(3):
        new = [int(min(n, max(0, width * page - h))) for n, h in zip(r.integers(0, 2 * pages * page // requests + 1, requests), plain.lengths)]
        want, step = plain.extend(new, sum(new)), pt.extend(ints(new), sum(new))
        same(step, want)
        pt.accept(step)
        plain.accept(want)
        stay = [int(r.integers(0, n + 1)) if r.random() < 0.3 else n if r.random() < 0.2 else 0 for n in plain.lengths]
        pt.shrink(ints(stay))
        plain.shrink(stay)
        n = int(pt.available)
        assert n == len(plain.free) and pt.free.cpu().tolist()[:n] == plain.free and pt.lengths.cpu().tolist() == plain.lengths
