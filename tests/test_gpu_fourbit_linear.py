"""Linear layers in microscaled 4-bit codes, served and trained, against plain implementations in 64 bits."""
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
from paper_1912_12607_amd import binding as B  # noqa: E402
from paper_1912_12607_amd import fourbit, tokens  # noqa: E402

DEV = torch.device("cuda:0")
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
HALF = {F32: 2.0**-24, BF16: 2.0**-8, F16: 2.0**-11}


def values(shape, seed, dtype=F32, spread=1.0):
    r = np.random.default_rng(seed)
    x = r.standard_normal(shape) * np.exp(spread * r.standard_normal(shape[:-1] + (1,)))
    t = torch.from_numpy(x.astype(np.float32)).to(dtype)
    return t, t.double().numpy()


def near(got, a, b, dtype, bias=None):
    """got = a b^T + bias: each of the additions rounds (or cuts) by 2^-23 of what is summed at most, the result by half a step; fp16 has steps of 2^-24 below its range."""
    want, size = a @ b.T, np.abs(a) @ np.abs(b).T
    if bias is not None:
        want, size = want + bias, size + np.abs(bias)
    bound = (a.shape[1] + 1) * 2.0**-23 * size + HALF[dtype] * np.abs(want) * 1.01 + (2.0**-25 if dtype is F16 else 0.0)
    assert got.dtype == dtype and got.shape == want.shape
    off = np.abs(got.detach().double().cpu().numpy() - want)
    assert (off <= bound).all(), (off / np.maximum(bound, 1e-300)).max()


# few tokens, tiles of each size, odd everything
SERVED = [(1, 1, 1), (1, 4096, 4096), (2, 33, 17), (3, 300, 1000), (9, 2048, 1000), (16, 4096, 100), (17, 64, 40), (16, 8192, 33), (40, 1000, 300), (130, 520, 515), (1, 33000, 5), (16, 2048, 100), (16, 3000, 33), (3, 2048, 5001),
          (2, 500, 9000)]


@pytest.mark.parametrize("M,K,N", SERVED)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bias", [False, True])
def test_served_linear(M, K, N, dtype, bias):
    (x, x64), (w, w64) = values((M, K), 1, dtype), values((N, K), 2, dtype, 0.3)
    b = np.random.default_rng(3).standard_normal(N).astype(np.float32) if bias else None
    layer = fourbit.ServedLinear4.of(w.to(DEV), None if b is None else torch.from_numpy(b).to(DEV))
    code, byte = R.quantise(w64)
    assert np.array_equal(layer.codes.cpu().numpy(), R.packed(code)) and np.array_equal(layer.scales.cpu().numpy(), byte)
    near(layer(x.to(DEV)), R.rounded(x64), R.stands_for(code, byte, K), dtype, b)
    # the same from codes that were made elsewhere; what is behind the blocks does not matter
    more = torch.cat([layer.scales, torch.full((N, 5), 255, dtype=torch.uint8, device=DEV)], 1)
    again = fourbit.ServedLinear4(layer.codes, more, K, layer.bias)
    assert torch.equal(again(x.to(DEV)), layer(x.to(DEV)))


def test_served_linear_of_strided_and_many_dimensional_inputs():
    layer = fourbit.ServedLinear4.of(values((40, 96), 5)[0].to(DEV))
    x = values((5, 7, 200), 6, BF16)[0].to(DEV)
    want = layer(x[..., 3:99].contiguous())
    assert want.shape == (5, 7, 40) and torch.equal(layer(x[..., 3:99]), want)
    rows = x[0, :, :96]                                   # rows 200 apart
    assert torch.equal(layer(rows), layer(rows.contiguous()))
    assert torch.equal(layer(x[0, 0, :96].expand(9, 96)), layer(x[0, 0, :96].repeat(9, 1)))
    assert torch.equal(layer(x[1].t()[:96].t()), layer(x[1, :, :96].contiguous()))
    assert layer(torch.zeros(2, 0, 96, device=DEV)).shape == (2, 0, 40)


@pytest.mark.parametrize("M", [2, 70])
def test_served_linear_of_what_is_not_finite(M):
    w, _ = values((40, 100), 5)
    w[7, 50] = float("inf")
    x, _ = values((M, 100), 6)
    x[1, 99] = float("nan")
    y = fourbit.ServedLinear4.of(w.to(DEV))(x.to(DEV)).cpu()
    want = torch.zeros(M, 40, dtype=torch.bool)
    want[1], want[:, 7] = True, True
    assert torch.equal(torch.isnan(y), want)


def _train(x, w, b, g, seed):
    x, w = (t.to(DEV).requires_grad_(True) for t in (x, w))
    b = None if b is None else torch.from_numpy(b).to(DEV).requires_grad_(True)
    y = fourbit.linear4(x, w, b, seed=seed)
    grads = torch.autograd.grad(y, [x, w] + ([] if b is None else [b]), g.to(DEV))
    return y, grads


def _drawn(g64, seed):
    """The gradient's codes for dx and (transposed) for dw."""
    index = np.arange(g64.size).reshape(g64.shape)
    return R.rounded(g64, R.draws(index, seed)), R.rounded(g64.T, R.draws(index, seed ^ (1 << 63)).T)


@pytest.mark.parametrize("M,K,N", [(1, 16, 16), (1, 1, 1), (2, 33, 5), (70, 130, 65), (256, 512, 1000), (300, 64, 40), (1030, 144, 272), (33, 2100, 31)])
@pytest.mark.parametrize("dtype,wtype", [(F32, F32), (BF16, BF16), (F16, F16), (BF16, F32), (F32, F16)])
def test_linear_and_gradients(M, K, N, dtype, wtype):
    seed = 12345678901234567
    (x, x64), (w, w64), (g, g64) = values((M, K), 9, dtype), values((N, K), 10, wtype, 0.3), values((M, N), 11, dtype)
    b = np.random.default_rng(12).standard_normal(N).astype(np.float32)
    y, (dx, dw, db) = _train(x, w, b, g, seed)
    near(y, R.rounded(x64), R.rounded(w64), dtype, b)
    a, h = _drawn(g64, seed)
    near(dx, a, R.rounded(w64.T), dtype)
    near(dw, h, R.rounded(x64.T), wtype)
    assert np.all(np.abs(db.cpu().numpy() - g64.sum(0)) <= 33 * 2.0**-24 * np.abs(g64).sum(0) + 1e-30)


def test_gradients_against_differences():
    """Differences of the loss <g, x W^T + b> in 64 bits against the gradients.  Nothing is clipped: a drawn code of g is off by less than its step, a nearest one of W by half
    a step; a step is at most 2 2^e in a block of scale 2^e.  |error| <= sum_n (step_g |w'| + |g| step_w / 2), w' = Q'(W); likewise dw over the tokens."""
    M, K, N, h = 24, 40, 32, 1e-4
    (x, x64), (w, w64), (g, g64) = values((M, K), 13), values((N, K), 14, F32, 0.3), values((M, N), 15)
    y, (dx, dw, db) = _train(x, w, np.zeros(N, np.float32), g, 5)

    def step(v):
        byte = R.quantise(v)[1]
        return np.repeat(2 * np.ldexp(1.0, byte - 127), 32, 1)[:, :v.shape[1]]

    def loss(x, w, b):
        return float((g64 * (x @ w.T + b)).sum())
    bx = step(g64) @ np.abs(R.rounded(w64.T)).T + np.abs(g64) @ (step(w64.T) / 2).T
    bw = step(g64.T) @ np.abs(R.rounded(x64.T)).T + np.abs(g64.T) @ (step(x64.T) / 2).T
    r = np.random.default_rng(16)
    for _ in range(20):
        m, k, n = r.integers(M), r.integers(K), r.integers(N)
        for at, got, bound, arg in (((m, k), dx, bx, 0), ((n, k), dw, bw, 1), ((n,), db, np.full(N, 1e-4), 2)):
            args = [[x64, w64, np.zeros(N)], [x64, w64, np.zeros(N)]]
            for side, sign in ((0, 1), (1, -1)):
                args[side] = [v.copy() for v in args[side]]
                args[side][arg][at] += sign * h
            diff = (loss(*args[0]) - loss(*args[1])) / (2 * h)
            assert abs(float(got[at]) - diff) <= bound[at] * (1 + 1e-6) + 1e-6 * abs(diff) + 1e-6


def test_gradients_are_unbiased():
    """The mean over draws meets the gradient with the same codes of x and W and no rounding of g: a rounded value has variance at most (step / 2)^2, so the mean of R draws
    is within 6 sqrt(sum (step / 2)^2 w'^2 / R) for all but one in 5e8 elements."""
    M, K, N, T = 6, 48, 40, 256
    (x, x64), (w, w64), (g, g64) = values((M, K), 17), values((N, K), 18, F32, 0.3), values((M, N), 19)
    mx, mw = torch.zeros(M, K, dtype=torch.float64, device=DEV), torch.zeros(N, K, dtype=torch.float64, device=DEV)
    for seed in range(T):
        _, (dx, dw) = _train(x, w, None, g, seed)
        mx += dx.double() / T
        mw += dw.double() / T

    def step(v):
        return np.repeat(2 * np.ldexp(1.0, R.quantise(v)[1] - 127), 32, 1)[:, :v.shape[1]]
    for got, a, b in ((mx, g64, R.rounded(w64.T)), (mw, g64.T, R.rounded(x64.T))):
        var = (step(a) / 2) ** 2 @ (b ** 2).T
        assert np.all(np.abs(got.cpu().numpy() - a @ b.T) <= 6 * np.sqrt(var / T) + 1e-6)


def test_linear_of_no_tokens_single_gradients_and_broadcast_ones():
    x, w = torch.zeros(0, 48, device=DEV, requires_grad=True), torch.randn(20, 48, device=DEV, requires_grad=True)
    b = torch.zeros(20, device=DEV, requires_grad=True)
    y = fourbit.linear4(x, w, b)
    assert y.shape == (0, 20)
    dx, dw, db = torch.autograd.grad(y, [x, w, b], torch.zeros(0, 20, device=DEV))
    assert dx.shape == (0, 48) and not dw.any() and not db.any()
    xs, g = torch.randn(33, 48, device=DEV, requires_grad=True), torch.randn(33, 20, device=DEV)
    everything = torch.autograd.grad(fourbit.linear4(xs, w, b, seed=4), [xs, w, b], g)
    assert torch.equal(torch.autograd.grad(fourbit.linear4(xs, w.detach(), None, seed=4), xs, g)[0], everything[0])
    assert torch.equal(torch.autograd.grad(fourbit.linear4(xs.detach(), w, None, seed=4), w, g)[0], everything[1])
    assert torch.equal(torch.autograd.grad(fourbit.linear4(xs.detach(), w.detach(), b, seed=4), b, g)[0], everything[2])
    row = torch.randn(20, device=DEV)
    a = torch.autograd.grad(fourbit.linear4(xs, w, b, seed=4), [xs, w, b], row.expand(33, 20))
    c = torch.autograd.grad(fourbit.linear4(xs, w, b, seed=4), [xs, w, b], row.repeat(33, 1))
    assert all(torch.equal(p, q) for p, q in zip(a, c))
    # a leaf in two layers: its gradient is the sum
    y = fourbit.linear4(xs, w, None, seed=1).sum() + fourbit.linear4(xs, w, None, seed=2).sum()
    one = torch.ones(33, 20, device=DEV)
    parts = [torch.autograd.grad(fourbit.linear4(xs, w, None, seed=s), w, one)[0] for s in (1, 2)]
    assert torch.equal(torch.autograd.grad(y, w)[0], parts[0] + parts[1])


@pytest.mark.parametrize("M,K,N", [(200, 64, 48), (300, 64, 40), (1030, 130, 600), (700, 2100, 31)])
def test_each_gradient_by_itself(M, K, N):
    """The same numbers whichever of the gradients are wanted."""
    x, w, b = torch.randn(M, K, device=DEV, dtype=BF16), torch.randn(N, K, device=DEV, dtype=BF16), torch.randn(N, device=DEV)
    dy = torch.randn(M, N, device=DEV, dtype=BF16)

    def grads(want):
        leaves = [t.clone().requires_grad_(n in want) for t, n in ((x, "x"), (w, "w"), (b, "b"))]
        fourbit.linear4(*leaves, seed=5).backward(dy)
        return [t.grad for t in leaves]
    all_ = grads("xwb")
    assert torch.equal(all_[2], grads("b")[2])
    exact = dy.double().sum(0)
    # (a part of 256 rows: 7 sums of a lane, 3 of lanes, 2 of waves in a row; parts in 64 bits, rounded once)
    assert ((all_[2].double() - exact).abs() <= 13.1 * 2.0**-24 * dy.double().abs().sum(0)).all()
    for want in ("x", "w", "xw", "xb", "wb"):
        for got, ref, name in zip(grads(want), all_, "xwb"):
            assert (got is None) == (name not in want) and (got is None or torch.equal(got, ref)), (want, name)


@pytest.mark.parametrize("M", [1, 3, 40])
def test_weights_laid_out_and_tokens_kept(M):
    """Through the binding: codes of W that are there, codes of x kept for dw (few tokens too)."""
    K, N = 70, 50
    (x, x64), (w, w64), (g, g64) = values((M, K), 1), values((N, K), 2), values((M, N), 3)
    layer = fourbit.ServedLinear4.of(w.to(DEV))
    xd, gd = x.to(DEV), g.to(DEV)
    xt, sxt = torch.zeros(K, 16 * R.blocks_of(M), dtype=torch.uint8, device=DEV), torch.zeros(R.panels_of(M), K, 8, dtype=torch.uint8, device=DEV)
    y, dw = torch.empty(M, N, device=DEV), torch.empty(N, K, device=DEV)
    d = B.LinearDesc(M, K, N, B.F32, B.F32)
    b = B.Mx4LinearBuffers.from_buffer_copy(layer._b)
    b.x, b.x_pitch, b.y, b.y_pitch, b.xt, b.sxt, b.dy, b.dy_pitch, b.dw = xd.data_ptr(), K, y.data_ptr(), N, xt.data_ptr(), sxt.data_ptr(), gd.data_ptr(), N, dw.data_ptr()
    ws = torch.empty(max(B.int8t_mx4_linear_workspace_bytes(d, i) for i in (0, 1)), dtype=torch.uint8, device=DEV)
    b.ws, b.ws_bytes = ws.data_ptr(), ws.numel()
    B.int8t_mx4_linear_fwd(d, b)
    B.int8t_mx4_linear_bwd(d, b, 9)
    near(y, R.rounded(x64), R.rounded(w64), F32)
    near(dw, _drawn(g64, 9)[1], R.rounded(x64.T), F32)


def test_more_tokens_than_a_backward_pass_takes_are_refused_before_it():
    x, w = torch.zeros(131073, 1, device=DEV), torch.zeros(1, 1, device=DEV)
    b = torch.zeros(1, device=DEV)
    assert fourbit.linear4(x, w, b).shape == (131073, 1)
    for args in ((x, w.clone().requires_grad_(True), b), (x, w, b.clone().requires_grad_(True))):
        with pytest.raises(RuntimeError, match="not served"):
            fourbit.linear4(*args)


def test_gradients_of_what_is_not_finite():
    """NaN in the gradient of one token: its dx, and dw and db of its output; in fp16 training a program sees the overflow."""
    (x, _), (w, _), (g, _) = values((40, 50), 1), values((30, 50), 2), values((40, 30), 3)
    g[5, 7] = float("inf")
    _, (dx, dw, db) = _train(x, w, np.zeros(30, np.float32), g, 1)
    assert torch.isnan(dx[5]).all() and not torch.isnan(dx[torch.arange(40) != 5]).any()
    assert torch.isnan(dw[7]).all() and not torch.isnan(dw[torch.arange(30) != 7]).any()
    assert not torch.isfinite(db[7]) and torch.isfinite(db[torch.arange(30) != 7]).all()


def test_token_linear_module():
    m = fourbit.TokenLinear4(96, 40, dtype=BF16, name="proj")
    assert isinstance(m, tokens.TokenLinear)
    x = torch.randn(7, 96, device=DEV, dtype=BF16)
    seed = m._seed
    y = m(x)
    assert m._seed == seed + 1 and torch.equal(y, fourbit.linear4(x, m.weight, m.bias, seed + 1))
    with torch.no_grad():
        m(x)
    assert m._seed == seed + 1
    y.float().square().mean().backward()
    assert m.weight.grad.dtype is BF16 and m.bias.grad.dtype is F32 and torch.isfinite(m.weight.grad).all()
    assert torch.equal(m.served()(x), y.detach())
    with pytest.raises(RuntimeError, match="once"):
        z = m(x).float().sum()
        gw, = torch.autograd.grad(z, m.weight, create_graph=True)


def test_training_pass_in_a_graph():
    """Captured and replayed with other values, beside an eager pass of other leaves, every replay equal to the eager result."""
    x, w = torch.randn(70, 96, device=DEV, dtype=BF16), (torch.randn(130, 96, device=DEV) * 0.1).to(BF16)
    g = torch.randn(70, 130, device=DEV, dtype=BF16)
    b = torch.randn(130, device=DEV)

    def step():
        leaves = [t.detach().requires_grad_(True) for t in (x, w, b)]
        y = fourbit.linear4(*leaves, seed=3)
        return (y.detach(),) + torch.autograd.grad(y, leaves, g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(other, step()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        gen = torch.Generator().manual_seed(i)
        for t in (x, w, g, b):
            t.copy_(torch.randn(t.shape, generator=gen))
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in out]
        assert all(torch.equal(p, q) for p, q in zip(replayed, step()))


def test_refusals():
    layer = fourbit.ServedLinear4.of(torch.randn(8, 40, device=DEV))
    x = torch.zeros(2, 40, device=DEV)
    for call in (lambda: layer(torch.zeros(2, 39, device=DEV)), lambda: layer(torch.zeros(2, 40)), lambda: fourbit.linear4(x, torch.zeros(4, 39, device=DEV)),
                 lambda: fourbit.linear4(x, torch.zeros(4, 40, device=DEV), torch.zeros(5, device=DEV)), lambda: fourbit.linear4(x, torch.zeros(4, 40)),
                 lambda: fourbit.linear4(x, torch.zeros(4, 40, device=DEV), torch.zeros(4, device=DEV, dtype=BF16)),
                 lambda: fourbit.ServedLinear4(layer.codes, layer.scales[:4], 40), lambda: fourbit.ServedLinear4(layer.codes, layer.scales, 70),
                 lambda: fourbit.ServedLinear4(layer.codes, layer.scales[:, :1], 40), lambda: fourbit.ServedLinear4(layer.codes.char(), layer.scales, 40),
                 lambda: fourbit.ServedLinear4(layer.codes, layer.scales.cpu(), 40)):
        with pytest.raises(RuntimeError):
            call()
    for call in (lambda: layer(x.double()), lambda: fourbit.linear4(x, torch.zeros(4, 40, device=DEV).double())):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(B.Int8tError) as e:
        fourbit.ServedLinear4.of(torch.zeros(1, 131104, device=DEV))
    assert e.value.status == 2
