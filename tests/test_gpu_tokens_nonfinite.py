"""NaN and infinities in tokens, weights, gradients and cached rows show in what is computed from them, and in nothing else."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_1912_12607_amd import tokens  # noqa: E402

DEV = torch.device("cuda:0")
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
BAD = [float("nan"), float("inf"), float("-inf")]


def normal(*shape, dtype=F32, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


def only(got, clean, hit):
    """NaN at `hit`, the clean result to the bit elsewhere."""
    assert bool(got[hit].isnan().all()) and torch.equal(got[~hit], clean[~hit])


# few tokens (one by all waves, by two, by one, rows read twice), many; rows that a block holds and longer ones
@pytest.mark.parametrize("M,K,N", [(1, 300, 40), (1, 20000, 33), (4, 130, 17), (7, 64, 33), (13, 2040, 50), (40, 1000, 72), (70, 4096, 96), (3, 40000, 20)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", BAD)
def test_served_tokens(M, K, N, dtype, bad):
    layer = tokens.ServedLinear.of(normal(N, K, seed=1), normal(N, seed=2))
    x = normal(M, K, dtype=dtype, seed=3)
    clean = layer(x)
    m, hit = M // 2, torch.zeros(M, N, dtype=torch.bool, device=DEV)
    hit[m] = True
    for k in (0, K // 2, K - 1):
        y = x.clone()
        y[m, k] = bad
        only(layer(y), clean, hit)
    w = normal(N, K, dtype=dtype, seed=1)
    w[N - 1, K // 3] = bad
    assert bool(tokens.ServedLinear.of(w)(x)[:, N - 1].isnan().all()) and not tokens.ServedLinear.of(w)(x)[:, :N - 1].isnan().any()


@pytest.mark.parametrize("M,K,N", [(2, 33, 5), (70, 130, 65), (256, 512, 1000), (300, 64, 1504), (40, 48, 9001)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", BAD)
def test_gradients(M, K, N, dtype, bad):
    x0, w0, g0 = normal(M, K, dtype=dtype, seed=4), normal(N, K, dtype=dtype, seed=5), normal(M, N, dtype=dtype, seed=6)

    def run(x, w, g):
        x, w, b = x.clone().requires_grad_(True), w.clone().requires_grad_(True), torch.zeros(N, device=DEV, requires_grad=True)
        y = tokens.linear(x, w, b, seed=7)
        return [y.detach(), *torch.autograd.grad(y, [x, w, b], g)]
    clean = run(x0, w0, g0)
    m, k, n = M - 1, K // 2, N // 2
    rows, cols = torch.zeros(M, 1, dtype=torch.bool, device=DEV), torch.zeros(N, dtype=torch.bool, device=DEV)
    rows[m], cols[n] = True, True
    # a gradient: its token's dx, its channel's dw and bias
    g = g0.clone()
    g[m, n] = bad
    y, dx, dw, db = run(x0, w0, g)
    assert torch.equal(y, clean[0])
    only(dx, clean[1], rows.expand(M, K))
    only(dw, clean[2], cols[:, None].expand(N, K))
    assert not db[n].isfinite() and torch.equal(db[~cols], clean[3][~cols])
    # a token: its y; every channel's gradient has met it
    x = x0.clone()
    x[m, k] = bad
    y, dx, dw, db = run(x, w0, g0)
    only(y, clean[0], rows.expand(M, N))
    assert torch.equal(dx, clean[1]) and bool(dw.isnan().all()) and torch.equal(db, clean[3])
    # a channel: its y; every token's gradient has met it
    w = w0.clone()
    w[n, k] = bad
    y, dx, dw, db = run(x0, w, g0)
    only(y, clean[0], cols.expand(M, N))
    assert bool(dx.isnan().all()) and torch.equal(dw, clean[2]) and torch.equal(db, clean[3])


@pytest.mark.parametrize("heads,dim", [(2, 64), (3, 128), (1, 208)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", BAD)
def test_cached_rows(heads, dim, dtype, bad):
    cache = tokens.PagedCache.empty(2, 16, heads, dim, DEV)
    k, v = normal(20, heads, dim, dtype=dtype, seed=8), normal(20, heads, dim, dtype=dtype, seed=9)
    slots = torch.arange(20, device=DEV)
    cache.write(k, v, slots)
    clean = cache.read(slots, dtype)
    hit = torch.zeros(20, heads, dim, dtype=torch.bool, device=DEV)
    hit[11, heads - 1] = True
    for d in (0, dim - 1):
        kk, vv = k.clone(), v.clone()
        kk[11, heads - 1, d] = vv[11, heads - 1, d] = bad
        cache.write(kk, vv, slots)
        for got, want in zip(cache.read(slots, dtype), clean):
            only(got, want, hit)
